"""Products on 8-bit weights and tokens against the plain form in 64 bits (GPU)."""
import numpy as np
import pytest
import torch

import blocks64
from paper_2607_08786_amd import linear, usp

pytestmark = pytest.mark.gpu


def matrix(seed, M, K, keep, low=-127):
    rng = np.random.default_rng(seed)
    W = rng.integers(low, 128, (M, K)).astype(np.int8)
    mask = (rng.random((M, K)) < keep).astype(np.uint8)
    scale = (rng.random(M) * 2e-3 + 1e-5).astype(np.float32)
    return usp.SparseMatrixQ(W, mask, scale), np.where(mask != 0, W, 0).astype(np.float64) * scale[:, None].astype(np.float64)


def tokens(seed, N, K, ld=None, offset=0):
    """Codes over the whole int8 range in a buffer of garbage, and scales."""
    rng = np.random.default_rng(seed)
    ld = K if ld is None else ld
    buf = torch.from_numpy(rng.integers(-128, 128, N * ld + offset + 64).astype(np.int8)).cuda()
    xq = torch.as_strided(buf, (N, K), (ld, 1), offset)
    s = torch.from_numpy((rng.random(N) * 0.05 + 1e-3).astype(np.float32)).cuda()
    return xq, s, xq.cpu().numpy().astype(np.float64) * s.cpu().numpy().astype(np.float64)[:, None]


def half(seed, *shape):
    return torch.from_numpy(np.random.default_rng(seed).standard_normal(shape).astype(np.float16)).cuda()


def f64(t):
    return None if t is None else t.detach().double().cpu().numpy()


# Rows and columns around a tile, K across several tiles, tokens around every block and route.
SHAPES = [(1, 1), (15, 3), (16, 256), (17, 257), (100, 255), (64, 1000), (1500, 2050), (257, 5000), (640, 8192)]


@pytest.mark.parametrize("M,K", SHAPES)
@pytest.mark.parametrize("N", [1, 2, 15, 16, 17, 32, 33, 64, 65, 129, 257, 513])
def test_shapes(M, K, N):
    A, w = matrix(M + K, M, K, 0.5)
    xq, s, x = tokens(N, N, K)
    want, tol = blocks64.product(x, w)
    blocks64.close(A.spmm(xq, s).cpu().numpy(), want, tol)


@pytest.mark.parametrize("keep", [0.0, 0.02, 0.3, 0.6, 1.0])
@pytest.mark.parametrize("N", [1, 40, 300])
def test_densities(keep, N):
    """An empty matrix gives the bias alone; a full one has the longest records."""
    A, w = matrix(7, 200, 1300, keep, low=-128)
    xq, s, x = tokens(8, N, 1300)
    b = half(9, 200)
    want, tol = blocks64.product(x, w, f64(b))
    blocks64.close(A.spmm(xq, s, bias=b).cpu().numpy(), want, tol)


@pytest.mark.parametrize("act", ["none", "relu", "gelu_tanh", "silu"])
@pytest.mark.parametrize("N", [1, 21, 200])
def test_epilogue(act, N):
    M, K = 333, 777
    A, w = matrix(11, M, K, 0.5)
    xq, s, x = tokens(12, N, K)
    b, r = half(13, M + 1)[1:], half(14, N, M + 3)[:, :M]  # unaligned bias, strided residual
    want, tol = blocks64.product(x, w, f64(b), act, f64(r))
    blocks64.close(A.spmm(xq, s, bias=b, residual=r, activation=act).cpu().numpy(), want, tol)
    y = r.contiguous().clone()  # the residual in place
    assert torch.equal(A.spmm(xq, s, Y=y, bias=b, residual=y, activation=act), A.spmm(xq, s, bias=b, residual=r, activation=act))


@pytest.mark.parametrize("ld,offset", [(1000, 0), (1001, 0), (1002, 2), (1004, 4), (1016, 1), (1003, 3)])
@pytest.mark.parametrize("N", [1, 50, 400])
def test_strides_and_alignment(ld, offset, N):
    """The same codes wherever they lie give the same bits; rows of Y between the written columns stay."""
    M, K = 150, 1000
    A, w = matrix(15, M, K, 0.5)
    xq, s, x = tokens(16, N, K, ld, offset)
    want, tol = blocks64.product(x, w)
    wide = torch.full((N, M + 5), 3.0, dtype=torch.float16, device="cuda")
    usp.usp_spmm_q(A.handle, xq, s, wide[:, 2:2 + M], A.make_workspace(N))
    blocks64.close(wide[:, 2:2 + M].cpu().numpy(), want, tol)
    assert (wide[:, :2] == 3).all() and (wide[:, 2 + M:] == 3).all()
    assert torch.equal(wide[:, 2:2 + M], A.spmm(xq.contiguous(), s))


def test_largest_sums():
    """-128 times -128 over many columns: the integer sums reach beyond 2^24 and stay exact."""
    M, K = 32, 40000
    W, mask = np.full((M, K), -128, np.int8), np.ones((M, K), np.uint8)
    A = usp.SparseMatrixQ(W, mask, np.full(M, 2.0 ** -22, np.float32))
    for N in (1, 70, 600):
        xq = torch.full((N, K), -128, dtype=torch.int8, device="cuda")
        y = A.spmm(xq, torch.ones(N, device="cuda"))
        assert (y == 128 * 128 * K / 2 ** 22).all()  # 156.25, exact in fp16


def test_nan_scale_stays_in_its_token():
    A, _ = matrix(17, 64, 512, 0.5)
    xq, s, _ = tokens(18, 20, 512)
    clean = A.spmm(xq, s)
    s2 = s.clone()
    s2[7] = float("nan")
    got = A.spmm(xq, s2)
    assert torch.isnan(got[7]).all()
    keep = torch.arange(20) != 7
    assert torch.equal(got[keep.cuda()], clean[keep.cuda()])


def test_densify_and_decode():
    rng = np.random.default_rng(19)
    W, mask = rng.integers(-128, 128, (70, 530)).astype(np.int8), (rng.random((70, 530)) < 0.5).astype(np.uint8)
    scale = (rng.random(70) * 0.01).astype(np.float32)
    A = usp.SparseMatrixQ(W, mask, scale)
    kept = np.where(mask != 0, W, 0).astype(np.int8)
    Wo, mo, so = A.decode()
    assert np.array_equal(Wo, kept) and np.array_equal(mo, mask) and np.array_equal(so, scale)
    assert np.array_equal(A.densify().cpu().numpy(), (kept.astype(np.float32) * scale[:, None]).astype(np.float16))
    info = A.info()
    assert info["format_version"] == 3 and info["nnz"] == mask.sum()


def test_value_types_are_told_apart():
    A, _ = matrix(20, 32, 256, 0.5)
    B = usp.SparseMatrix(np.zeros((32, 256), np.uint16), np.ones((32, 256), np.uint8))
    x16, y = half(21, 4, 256), torch.empty(4, 32, dtype=torch.float16, device="cuda")
    xq, s, _ = tokens(22, 4, 256)
    ws = torch.zeros(1 << 20, dtype=torch.uint8, device="cuda")
    for call in (lambda: usp.usp_spmm(A.handle, x16, y, ws), lambda: usp.usp_spmm_noalloc(A.handle, x16, y),
                 lambda: usp.usp_decode(A.handle), lambda: usp.usp_decode_q(B.handle),
                 lambda: usp.usp_spmm_q(B.handle, xq, s, y, ws)):
        with pytest.raises(usp.UspError) as e:
            call()
        assert e.value.status == 1


def test_refusals():
    A, _ = matrix(23, 32, 256, 0.5)
    xq, s, _ = tokens(24, 4, 256)
    y, ws = torch.empty(4, 32, dtype=torch.float16, device="cuda"), A.make_workspace(4)
    need = A.workspace_size(4)
    if need:
        with pytest.raises(usp.UspError):
            usp.usp_spmm_q(A.handle, xq, s, y, None)
        with pytest.raises(usp.UspError):
            usp.usp_spmm_q(A.handle, xq, s, y, torch.zeros(need - 1, dtype=torch.uint8, device="cuda"))
    for bad in (dict(x_scale=s[:3]), dict(x_scale=s.half()), dict(Xq=xq.half()), dict(Xq=xq[:3]), dict(bias=half(1, 31)),
                dict(residual=half(2, 4, 31)), dict(Xq=xq.cpu())):
        with pytest.raises((TypeError, ValueError)):
            usp.usp_spmm_q(A.handle, **{"Xq": xq, "x_scale": s, "Y": y, "workspace": ws, **bad})
    with pytest.raises(usp.UspError):
        usp.usp_spmm_q(A.handle, xq[:, :100].contiguous(), s, y, ws)  # fewer columns than the weight
    with pytest.raises(usp.UspError):
        usp.usp_spmm_q(A.handle, xq, s, y, ws, activation=9)


def test_workspace_shared_with_fp16_products():
    """One workspace, cleared once, serves both kinds in turn."""
    A, w = matrix(25, 320, 1001, 0.5)
    W16 = np.random.default_rng(26).standard_normal((512, 1024)).astype(np.float16)
    B = usp.SparseMatrix(W16, np.random.default_rng(27).integers(0, 2, (512, 1024)).astype(np.uint8))
    N = 48
    x16 = half(28, N, 1024)
    xq, s, x = tokens(29, N, 1001)
    ws = torch.zeros(max(A.workspace_size(N), B.workspace_size(N)), dtype=torch.uint8, device="cuda")
    want16, want, tol = B.spmm(x16), *blocks64.product(x, w)
    for _ in range(3):
        blocks64.close(A.spmm(xq, s, workspace=ws).cpu().numpy(), want, tol)
        assert torch.equal(B.spmm(x16, workspace=ws), want16)


@pytest.mark.parametrize("N", [4, 100, 400])
def test_captured_and_replayed(N):
    A, _ = matrix(30, 500, 1030, 0.5)
    xq, s, _ = tokens(31, N, 1030)
    y, ws = torch.empty(N, 500, dtype=torch.float16, device="cuda"), A.make_workspace(N)
    usp.usp_spmm_q(A.handle, xq, s, y, ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        usp.usp_spmm_q(A.handle, xq, s, y, ws)
    for k in range(4):
        s.mul_(1.25)
        xq.copy_(tokens(40 + k, N, 1030)[0])
        graph.replay()
        torch.cuda.synchronize()
        got = y.clone()
        assert torch.equal(got, A.spmm(xq, s))
        torch.cuda.synchronize()


def test_module():
    lin = torch.nn.Linear(300, 90).half().cuda()
    mask = torch.rand(90, 300) < 0.5
    mod = linear.SparseLinearQ.from_linear(lin, mask, activation="silu")
    codes, scale = linear.quantize_rows(lin.weight, mask)
    w = f64(codes) * f64(scale)[:, None]
    x, r = half(50, 2, 7, 300), half(51, 2, 7, 90)
    xq, xs = blocks64.quantize(x.reshape(14, 300).cpu().numpy())
    x64 = xq.astype(np.float64) * xs.astype(np.float64)[:, None]
    want, tol = blocks64.product(x64, w, f64(lin.bias), "silu", f64(r).reshape(14, 90))
    y = mod(x, r)
    assert y.shape == (2, 7, 90)
    blocks64.close(y.reshape(14, 90).cpu().numpy(), want, tol)
    pair = (torch.from_numpy(xq).cuda(), torch.from_numpy(xs).cuda())
    assert torch.equal(mod(pair, r.reshape(14, 90)), y.reshape(14, 90))
    assert mod(x[:, :0]).shape == (2, 0, 90)
    with torch.cuda.stream(torch.cuda.Stream()):
        z = mod(x, r)
    torch.cuda.synchronize()
    assert torch.equal(z, y)
    with pytest.raises(TypeError):
        linear.SparseLinearQ(lin.weight, mask, scale)


def test_module_captured():
    """A capture after a warm-up, then eager calls of other sizes, then replays."""
    w = torch.randn(400, 515).half().cuda()
    mask = torch.rand(400, 515) < 0.5
    codes, scale = linear.quantize_rows(w, mask)
    mod = linear.SparseLinearQ(codes, mask, scale)
    x = half(60, 9, 515)
    mod(x)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = mod(x)
    for k in range(4):
        x.copy_(half(61 + k, 9, 515))
        graph.replay()
        torch.cuda.synchronize()
        got = y.clone()
        mod(half(70, 900, 515))
        assert torch.equal(mod(x), got)
        torch.cuda.synchronize()
