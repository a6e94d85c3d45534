"""Scales whose product leaves the range of fp32 (GPU): a sum of zero stays zero, others follow the formula."""
import numpy as np
import pytest
import torch

from paper_2607_08786_amd import usp

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kernel,M,K,N", [("product", 40, 300, 5), ("wide-product", 941, 1144, 1652)])
@pytest.mark.parametrize("x_scale,w_scale", [(100.0, 1e38), (1e30, 1e30), (3e38, 3e38)])
def test_empty_rows(kernel, M, K, N, x_scale, w_scale):
    """A row of the weight that keeps nothing, or a token of zero codes, gives the bias."""
    rng = np.random.default_rng(1)
    W, mask = rng.integers(1, 9, (M, K)).astype(np.int8), np.ones((M, K), np.uint8)
    mask[3] = 0
    scale = np.full(M, 1e-3, np.float32)
    scale[3] = w_scale
    A = usp.SparseMatrixQ(W, mask, scale)
    assert A.plan(N).startswith(kernel + " ")
    x = torch.from_numpy(rng.integers(1, 9, (N, K)).astype(np.int8)).cuda()
    s = torch.full((N,), 1e-3, device="cuda")
    s[2] = x_scale
    b = torch.from_numpy(rng.standard_normal(M).astype(np.float16)).cuda()
    G = usp.ExpertGroup([A])
    offsets = torch.tensor([0, N], dtype=torch.int32, device="cuda")
    for y in (A.spmm(x, s, bias=b), G.spmm(x, offsets, x_scale=s, bias=b[None])):
        assert torch.equal(y[:, 3], b[3].expand(N))
    x[2] = 0
    A = usp.SparseMatrixQ(W, np.ones_like(mask), np.full(M, w_scale, np.float32))
    assert torch.equal(A.spmm(x, s, bias=b)[2], b)


@pytest.mark.parametrize("x_scale,w_scale", [(1e30, 1e-31), (2.0 ** 100, 2.0 ** -104), (1e-20, 1e18), (300.0, 1e36), (1e-30, 1e-12)])
def test_sums_that_are_not_zero(x_scale, w_scale):
    """The formula in 64 bits, rounded to fp16 (an infinity beyond 65520)."""
    rng = np.random.default_rng(2)
    W = rng.integers(-9, 9, (32, 200)).astype(np.int8)
    A = usp.SparseMatrixQ(W, np.ones((32, 200), np.uint8), np.full(32, w_scale, np.float32))
    x = rng.integers(-9, 9, (4, 200)).astype(np.int8)
    y = A.spmm(torch.from_numpy(x).cuda(), torch.full((4,), x_scale, device="cuda")).cpu().numpy().astype(np.float64)
    want = (x.astype(np.float64) @ W.T.astype(np.float64)) * float(np.float32(x_scale)) * float(np.float32(w_scale))
    big = np.abs(want) >= 65520
    assert np.array_equal(y[big], np.sign(want[big]) * np.inf)
    # One rounding to fp16 and four in fp32: the sum's conversion, the two scales' product, the product with the sum, none lost.
    tol = 2.0 ** -11 * np.abs(want) + 2.0 ** -25 + 4 * 2.0 ** -24 * np.abs(want)
    assert (np.abs(y - want)[~big] <= tol[~big]).all()


@pytest.mark.parametrize("kernel,M,K,N", [("product", 40, 300, 5), ("wide-product", 941, 1144, 1652)])
def test_infinite_token_scale(kernel, M, K, N):
    """As of a token with an infinity, whose codes are then zero: NaN, and infinities where codes are not."""
    rng = np.random.default_rng(3)
    W = rng.integers(1, 9, (M, K)).astype(np.int8)
    A = usp.SparseMatrixQ(W, np.ones((M, K), np.uint8), np.full(M, 1e-3, np.float32))
    assert A.plan(N).startswith(kernel + " ")
    x = torch.from_numpy(rng.integers(1, 9, (N, K)).astype(np.int8)).cuda()
    s = torch.full((N,), 1e-3, device="cuda")
    clean = A.spmm(x, s)
    x[2], s[2], s[4] = 0, float("inf"), float("-inf")
    y = A.spmm(x, s)
    assert torch.isnan(y[2]).all() and (y[4] == float("-inf")).all()
    keep = [n for n in range(N) if n not in (2, 4)]
    assert torch.equal(y[keep], clean[keep])
