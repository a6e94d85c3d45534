"""Tokens that are not finite stay visible through the epilogues of the 8-bit and grouped products (GPU)."""
import numpy as np
import pytest
import torch

from paper_2607_08786_amd import usp

pytestmark = pytest.mark.gpu

ACTS = ["none", "relu", "gelu_tanh", "silu"]
# (kernel, M, K, N)
PLACES = [("product", 64, 512, 20), ("product", 40, 300, 1), ("wide-product", 941, 1144, 1652)]


def half(seed, *shape):
    return torch.from_numpy(np.random.default_rng(seed).standard_normal(shape).astype(np.float16)).cuda()


def matrix(seed, M, K, q):
    rng = np.random.default_rng(seed)
    mask = (rng.random((M, K)) < 0.5).astype(np.uint8)
    mask[:, :2] = 1  # every row keeps the columns that the tests make NaN
    if q:
        return usp.SparseMatrixQ(rng.integers(-127, 128, (M, K)).astype(np.int8), mask, np.full(M, 1e-3, np.float32))
    return usp.SparseMatrix((rng.standard_normal((M, K)) * 0.1).astype(np.float16), mask)


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("kernel,M,K,N", PLACES)
def test_8_bit_tokens(kernel, M, K, N, act):
    """A token whose scale is NaN, and an fp16 token with a NaN or an infinity, give NaN in every output."""
    A = matrix(1, M, K, True)
    assert A.plan(N).startswith(kernel + " ")
    x, bias = half(2, N, K), half(3, M)
    clean = A.spmm(x, bias=bias, activation=act)
    for value in (float("nan"), float("inf"), float("-inf")):
        n = N // 2
        bad = x.clone()
        bad[n, 1] = value
        xq, s = torch.empty(N, K, dtype=torch.int8, device="cuda"), torch.empty(N, device="cuda")
        usp.usp_quantize(bad, xq, s)
        keep = (torch.arange(N) != n).cuda()
        for got in (A.spmm(bad, bias=bias, activation=act), A.spmm(xq, s, bias=bias, activation=act)):
            assert torch.isnan(got[n]).all()
            assert torch.equal(got[keep], clean[keep])


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("q", [False, True])
@pytest.mark.parametrize("kernel,M,K,T", [("product", 64, 512, 20), ("wide-product", 700, 776, 8192)])
def test_grouped_rows(kernel, M, K, T, q, act):
    G = usp.ExpertGroup([matrix(4 + e, M, K, q) for e in range(2)])
    assert G.plan(T).startswith(kernel)
    offsets = torch.tensor([0, T // 4, T], dtype=torch.int32, device="cuda")
    x, s = half(6, T, K), None
    if q:
        x, s = torch.randint(-128, 128, (T, K), device="cuda").to(torch.int8), torch.full((T,), 0.01, device="cuda")
    clean = G.spmm(x, offsets, x_scale=s, activation=act)
    n = T // 3
    if q:
        s = s.clone()
        s[n] = float("nan")
    else:
        x = x.clone()
        x[n, 1] = float("nan")
    got = G.spmm(x, offsets, x_scale=s, activation=act)
    keep = (torch.arange(T) != n).cuda()
    assert torch.isnan(got[n]).all()
    assert torch.equal(got[keep], clean[keep])
