"""Inputs of any strides: broadcast rows, overlapping rows, reversed and transposed layouts, give the bits of their contiguous
copies, as SparseLinear gives them."""
import pytest
import torch

from paper_2607_08786_amd import linear, usp

K, M, N = 32, 24, 6


def layouts(rows, width, device):
    """[rows, width] fp16 tensors that are not rows of their own memory."""
    g = torch.Generator().manual_seed(rows * width)
    flat = torch.randn(2 * rows * width, generator=g).half().to(device)
    return {
        "one row for all": flat[:width].expand(rows, width),
        "one value per row": flat[:rows, None].expand(rows, width),
        "one value": flat[:1].expand(rows, width),
        "overlapping": flat.as_strided((rows, width), (3, 1)),
        "nearly apart": flat.as_strided((rows, width), (width - 1, 1)),
        "transposed": flat[:rows * width].reshape(width, rows).t(),
        "every other": flat.reshape(rows, 2 * width)[:, ::2],
        "three dimensions": flat[:width].expand(2, rows // 2, width),
    }


@pytest.mark.parametrize("name", layouts(N, K, "cpu"))
def test_rows_of(name):
    x = layouts(N, K, "cpu")[name]
    rows = linear._rows_of(x, K)
    assert rows.shape == (N, K) and rows.stride(1) == 1 and rows.stride(0) >= K
    assert torch.equal(rows, x.reshape(N, K))


def test_rows_apart_are_not_copied():
    wide = torch.zeros(N, K + 5, dtype=torch.float16)
    for x in (wide[:, :K], wide[:, 3:3 + K], wide[:1, :K], wide[:1, :K].expand(1, K), wide[::2, :K]):
        assert linear._rows_of(x, K).data_ptr() == x.data_ptr()


def test_gate_of_a_channel(monkeypatch):
    """A gate [features] of any type and stride, as one for each token may be."""
    seen = []

    def norm(residual, y, gate, *args, **kw):
        seen.append(gate)

    monkeypatch.setattr(usp, "usp_norm", norm)
    mod = linear.BlockNorm(K, device="cpu")
    x = torch.zeros(N, K, dtype=torch.float16)
    values = torch.randn(2 * K)
    for gate in (values[:K], values[::2].half(), values[:1].half().expand(K), values[:K].half()):
        mod(x, x, gate)
        assert seen[-1].dtype == torch.float16 and seen[-1].is_contiguous() and torch.equal(seen[-1], gate.half())
    assert seen[-1] is gate
    with pytest.raises(ValueError):
        mod(x, x, values[:K - 1].half())


@pytest.mark.gpu
@pytest.mark.parametrize("name", layouts(N, K, "cpu"))
def test_modules_on_the_gpu(name):
    g = torch.Generator().manual_seed(1)
    codes, mask = torch.randint(-9, 9, (M, K), generator=g).to(torch.int8), torch.rand(M, K, generator=g) < 0.5
    layer = linear.SparseLinearQ(codes, mask, torch.full((M,), 0.01))
    experts = linear.SparseExperts([torch.randn(M, K, generator=g)] * 2, [mask, mask])
    norm = linear.BlockNorm(K, post="rms")
    offsets = torch.tensor([0, 2, N], dtype=torch.int32, device="cuda")
    x, r = layouts(N, K, "cuda")[name], layouts(N, M, "cuda")[name]
    for call in (lambda x, r: layer(x, r), lambda x, r: experts(x, offsets), lambda x, r: norm(x, x)[1], lambda x, r: norm(x, x, x)[0]):
        assert torch.equal(call(x, r), call(x.contiguous(), r.contiguous()))
