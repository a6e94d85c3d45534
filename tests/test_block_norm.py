"""usp_norm, usp_quantize and BlockNorm against the plain form in 64 bits (GPU)."""
import numpy as np
import pytest
import torch

import blocks64
from paper_2607_08786_amd import linear, usp

pytestmark = pytest.mark.gpu


def f64(t):
    return None if t is None else t.double().cpu().numpy()


def draw(seed, *shape, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(*shape, generator=g) * scale).half().cuda()


# K on every path: one thread's chunk, 256 and 1024 threads with 1 to 4 chunks, rows that are read again, odd sizes.
SIZES = [(1, 1), (3, 7), (2, 8), (5, 64), (4, 1000), (33, 2048), (2, 2049), (7, 5120), (1, 8192), (3, 8200), (2, 20001),
         (1, 32768), (2, 32776), (1, 70001)]


@pytest.mark.parametrize("N,K", SIZES)
@pytest.mark.parametrize("post,pre,gate,act", [("none", "rms", "none", "none"), ("rms", "layer", "channel", "sigmoid"),
                                               ("layer", "rms", "token", "silu"), ("rms", "none", "token", "tanh"),
                                               ("layer", "layer", "none", "none")])
def test_norm(N, K, post, pre, gate, act):
    R, y = draw(1, N, K, scale=3.0), draw(2, N, K)
    y += 5.0  # a mean far from zero
    g = None if gate == "none" else draw(3, K) if gate == "channel" else draw(3, N, K)
    vec = [draw(4 + i, K) for i in range(4)]
    r, h, hq, hs = torch.empty_like(R), torch.empty_like(R), torch.empty_like(R, dtype=torch.int8), torch.empty(N, device="cuda")
    usp.usp_norm(R, y, g, 0.7, post, vec[0], vec[1], pre, vec[2], vec[3], 1e-5, act, residual_out=r, out=h, out_q=hq,
                 out_scale=hs)
    want = blocks64.norm(f64(R), f64(y), f64(g), float(np.float32(0.7)), post, f64(vec[0]) if post != "none" else None,
                         f64(vec[1]) if post != "none" else None, pre, f64(vec[2]), f64(vec[3]), 1e-5, act)
    blocks64.close(r.cpu().numpy(), want[0], want[1])
    blocks64.close(h.cpu().numpy(), want[2], want[3])
    codes, scales = blocks64.quantize(h.cpu().numpy())  # of the fp16 h, bit for bit
    assert np.array_equal(hq.cpu().numpy(), codes) and np.array_equal(hs.cpu().numpy(), scales)


@pytest.mark.parametrize("N,K", [(1, 1), (5, 33), (300, 5120), (2, 40001)])
def test_quantize_bits(N, K):
    x = draw(9, N, K, scale=2.0)
    if K > 1:
        x[0] = 0  # a token of zeros
    xq, s = torch.empty(N, K, dtype=torch.int8, device="cuda"), torch.empty(N, device="cuda")
    usp.usp_quantize(x, xq, s)
    codes, scales = blocks64.quantize(x.cpu().numpy())
    assert np.array_equal(xq.cpu().numpy(), codes) and np.array_equal(s.cpu().numpy(), scales)


def test_quantize_extremes():
    """The largest and smallest magnitudes, and tokens that are not finite: zeros and the scale NaN."""
    x = torch.zeros(6, 70, dtype=torch.float16)
    x[0, 3], x[0, 5] = 65504, -65504
    x[1, 3] = 6e-8  # the smallest subnormal
    x[2, 9] = float("inf")
    x[3, 9] = float("nan")
    x[4, :] = -1.5
    xq, s = torch.full((6, 70), 9, dtype=torch.int8, device="cuda"), torch.empty(6, device="cuda")
    usp.usp_quantize(x.cuda(), xq, s)
    codes, scales = blocks64.quantize(x.numpy())
    assert np.array_equal(xq.cpu().numpy(), codes)
    assert np.array_equal(s.cpu().numpy(), scales, equal_nan=True)
    assert np.isnan(scales[[2, 3]]).all() and codes[0, 3] == 127 and codes[0, 5] == -127 and codes[1, 3] == 127


def test_strides_alignment_and_in_place():
    """Rows of larger buffers at odd addresses; the update in place; what lies between the rows stays."""
    N, K = 9, 515
    base = draw(11, N, 600)
    want = blocks64.norm(f64(base[:, 3:3 + K]), f64(base[:, 3:3 + K]), None, 0.5, pre="rms")
    r = base.clone()
    h = torch.full((N, 700), 7.0, dtype=torch.float16, device="cuda")
    view = r[:, 3:3 + K]
    usp.usp_norm(view, view, scale=0.5, pre="rms", residual_out=view, out=h[:, 1:1 + K])
    blocks64.close(view.cpu().numpy(), want[0], want[1])
    blocks64.close(h[:, 1:1 + K].cpu().numpy(), want[2], want[3])
    keep = torch.ones(600, dtype=torch.bool)
    keep[3:3 + K] = False
    assert torch.equal(r[:, keep], base[:, keep])
    assert (h[:, 0] == 7).all() and (h[:, 1 + K:] == 7).all()


def test_without_block_output():
    """No y: r is the residual, h its norm; each output alone gives the same bits."""
    R = draw(12, 4, 640)
    w = draw(13, 640)
    h, h2, r = torch.empty_like(R), torch.empty_like(R), torch.empty_like(R)
    usp.usp_norm(R, pre="layer", pre_weight=w, out=h)
    usp.usp_norm(R, pre="layer", pre_weight=w, out=h2, residual_out=r)
    assert torch.equal(h, h2) and torch.equal(r, R)
    want = blocks64.norm(f64(R), pre="layer", pre_weight=f64(w))
    blocks64.close(h.cpu().numpy(), want[2], want[3])


def test_nonfinite_tokens_stay_apart():
    """A NaN or an infinity in one token leaves the others' bits alone."""
    R, y = draw(14, 6, 256), draw(15, 6, 256)
    clean = [torch.empty_like(R), torch.empty_like(R)]
    usp.usp_norm(R, y, pre="rms", residual_out=clean[0], out=clean[1])
    y[2, 5], y[4, 0] = float("nan"), float("inf")
    got = [torch.empty_like(R), torch.empty_like(R)]
    usp.usp_norm(R, y, pre="rms", residual_out=got[0], out=got[1])
    others = [0, 1, 3, 5]
    assert all(torch.equal(a[others], b[others]) for a, b in zip(clean, got))
    assert torch.isnan(got[1][2]).all() and torch.isnan(got[1][4, 0]) and torch.isinf(got[0][4, 0])


def test_captured_and_replayed():
    R, y = draw(16, 5, 1024), draw(17, 5, 1024)
    r, hq, hs = torch.empty_like(R), torch.empty_like(R, dtype=torch.int8), torch.empty(5, device="cuda")

    def step():
        usp.usp_norm(R, y, post="rms", pre="rms", residual_out=r, out_q=hq, out_scale=hs)

    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for k in range(4):
        R.copy_(draw(20 + k, 5, 1024))
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (r, hq, hs)]
        step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, (r, hq, hs)))


def test_module():
    mod = linear.BlockNorm(320, post="rms", pre="layer", scale=0.5, gate_activation="sigmoid")
    for i, name in enumerate(("post_weight", "pre_weight", "pre_bias")):
        getattr(mod, name).copy_(draw(30 + i, 320))
    x, y, g = draw(33, 2, 3, 320), draw(34, 2, 3, 320), draw(35, 320)
    r, h = mod(x, y, g)
    want = blocks64.norm(f64(x).reshape(6, 320), f64(y).reshape(6, 320), f64(g), 0.5, "rms", f64(mod.post_weight), None,
                         "layer", f64(mod.pre_weight), f64(mod.pre_bias), 1e-5, "sigmoid")
    assert r.shape == h.shape == x.shape
    blocks64.close(r.reshape(6, 320).cpu().numpy(), want[0], want[1])
    blocks64.close(h.reshape(6, 320).cpu().numpy(), want[2], want[3])
    r2, (hq, hs) = mod(x, y, g, quantize=True)
    codes, scales = blocks64.quantize(h.reshape(6, 320).cpu().numpy())
    assert torch.equal(r, r2) and np.array_equal(hq.cpu().numpy(), codes) and np.array_equal(hs.cpu().numpy(), scales)
    first, _ = mod(x)
    assert torch.equal(first, x)
    assert mod(x[:0])[0].shape == (0, 3, 320)


def test_binding_refusals():
    R = draw(40, 4, 64)
    out = torch.empty_like(R)
    for bad in (dict(y=R[:, :32]), dict(y=R.float()), dict(gate=R[0, :10]), dict(pre_weight=R[0].float()), dict(y=R.cpu())):
        with pytest.raises((TypeError, ValueError)):
            usp.usp_norm(R, **{"pre": "rms", "out": out, **bad})
    with pytest.raises(usp.UspError):
        usp.usp_norm(R, pre="rms")
    with pytest.raises(usp.UspError):
        usp.usp_norm(R, gate=R, out=out)


@pytest.mark.parametrize("offset,gap", [(0, 0), (1, 0), (2, 3), (3, 1), (5, 2)])
@pytest.mark.parametrize("K", [1, 7, 8, 33, 510, 1000, 5123, 8191, 32776, 33001])
def test_every_alignment(K, offset, gap):
    """Rows that start at any element, between NaN: the bits of aligned copies, and nothing written beside them."""
    N = 3
    g = torch.Generator(device="cuda").manual_seed(K)
    rows = [torch.randn(N, K, device="cuda", generator=g).half() for _ in range(3)]
    vectors = [torch.randn(K, device="cuda", generator=g).half() for _ in range(4)]

    def placed(t, fill):
        buf = torch.full((offset + t.numel() + N * gap + 16,), fill, dtype=t.dtype, device="cuda")
        at = torch.as_strided(buf, t.shape, (t.shape[-1] + gap, 1)[-t.dim():], offset)
        at.copy_(t)
        return buf, at

    def call(residual, y, gate, vec, r, h, q, s):
        usp.usp_norm(residual, y, gate, 0.5, "layer", vec[0], vec[1], "rms", vec[2], vec[3], residual_out=r, out=h,
                     out_q=q, out_scale=s, gate_activation="sigmoid")

    want = [torch.empty(N, K, dtype=d, device="cuda") for d in (torch.float16, torch.float16, torch.int8)]
    want_s = torch.empty(N, device="cuda")
    call(*rows, vectors, *want, want_s)
    outs = [placed(torch.zeros(N, K, dtype=d, device="cuda"), 9) for d in (torch.float16, torch.float16, torch.int8)]
    s = torch.empty(N, device="cuda")
    nan = float("nan")
    call(*[placed(t, nan)[1] for t in rows], [placed(t, nan)[1] for t in vectors], *[o[1] for o in outs], s)
    assert torch.equal(s, want_s) and torch.isfinite(s).all()
    for (buf, at), w in zip(outs, want):
        assert torch.equal(at, w)
        at.fill_(9)
        assert (buf == 9).all()
