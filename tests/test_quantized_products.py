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


@pytest.mark.parametrize("K", [64512, 65000, 129024])
@pytest.mark.parametrize("N", [1, 50, 300])
def test_most_columns(K, N):
    """A wavefront's share of the column tiles up to what its offsets' lanes hold, and the limit itself."""
    rng = np.random.default_rng(K)
    W, mask = rng.integers(-3, 4, (20, K)).astype(np.int8), (rng.random((20, K)) < 0.5).astype(np.uint8)
    A = usp.SparseMatrixQ(W, mask, np.full(20, 0.01, np.float32))
    xq = torch.from_numpy(rng.integers(-3, 4, (N, K)).astype(np.int8)).cuda()
    want, tol = blocks64.product(f64(xq), np.where(mask != 0, W, 0).astype(np.float64) * np.float64(np.float32(0.01)))
    blocks64.close(A.spmm(xq, torch.ones(N, device="cuda")).cpu().numpy(), want, tol)


def test_too_many_columns():
    one = np.ones((1, usp.MAX_K_Q + 1), np.int8)
    with pytest.raises(usp.UspError) as e:
        usp.SparseMatrixQ(one, one.astype(np.uint8), np.ones(1, np.float32))
    assert e.value.status == 2


def test_fp16_tokens_are_quantised():
    """Without scales the tokens are fp16: the bits of usp_quantize and the product after it."""
    A, _ = matrix(80, 130, 701, 0.5)
    for N in (1, 30, 500):
        x = half(81 + N, N, 703)[:, 1:702]
        xq, s = torch.empty(N, 701, dtype=torch.int8, device="cuda"), torch.empty(N, device="cuda")
        usp.usp_quantize(x, xq, s)
        assert torch.equal(A.spmm(x), A.spmm(xq, s))


# Every kernel of the planner at a small shape that takes it: (plan, M, K, N), for records of up to 3 KB and larger ones.
KERNELS = [
    ("product R=1 W=4 nb=1", 16, 203, 1),
    ("product R=1 W=4 nb=2", 76, 6750, 1371),
    ("product R=1 W=4 nb=4", 68, 4185, 1992),
    ("product R=1 W=8 nb=1", 16, 3101, 3),
    ("product R=1 W=8 nb=2", 36, 12276, 1462),
    ("product R=2 W=4 nb=1", 37, 370, 1365),
    ("product R=2 W=4 nb=2", 390, 960, 1221),
    ("product R=2 W=4 nb=4", 135, 1636, 1923),
    ("product R=2 W=8 nb=1", 39, 1343, 1364),
    ("product R=2 W=8 nb=2", 152, 8618, 1623),
    ("product R=4 W=4 nb=1", 133, 629, 1654),
    ("product R=4 W=4 nb=2", 1258, 620, 794),
    ("product R=4 W=8 nb=1", 70, 1908, 1726),
    ("product R=4 W=8 nb=2", 292, 2857, 1606),
    ("product R=4 W=8 nb=4", 261, 1280, 1928),
    ("wide-product R=4 nb=2", 941, 1144, 1652),
    ("wide-product R=4 nb=4", 1058, 2886, 2004),
    ("wide-product R=8 nb=2", 16605, 292, 130),
    ("wide-product R=8 nb=4", 11706, 280, 518),
]
KERNELS_DENSE = [
    ("product R=1 W=4 nb=1", 16, 200, 3),
    ("product R=1 W=4 nb=2", 71, 4017, 1373),
    ("product R=1 W=4 nb=4", 69, 2102, 1651),
    ("product R=1 W=8 nb=1", 16, 1036, 2),
    ("product R=1 W=8 nb=2", 36, 8044, 1381),
    ("product R=2 W=4 nb=1", 36, 595, 1393),
    ("product R=2 W=4 nb=2", 403, 660, 1231),
    ("product R=2 W=4 nb=4", 137, 787, 1820),
    ("product R=2 W=8 nb=1", 36, 1359, 1407),
    ("product R=2 W=8 nb=2", 152, 3871, 1618),
    ("product R=4 W=4 nb=1", 196, 603, 1765),
    ("product R=4 W=4 nb=2", 1654, 608, 594),
    ("product R=4 W=8 nb=1", 69, 1746, 1659),
    ("product R=4 W=8 nb=2", 304, 1349, 1617),
    ("product R=4 W=8 nb=4", 280, 850, 1816),
    ("wide-product R=4 nb=2", 590, 770, 1739),
    ("wide-product R=4 nb=4", 1201, 2678, 1738),
    ("wide-product R=8 nb=2", 16822, 204, 129),
    ("wide-product R=8 nb=4", 16545, 213, 277),
]


@pytest.mark.parametrize("keep,plan,M,K,N", [(0.5, *k) for k in KERNELS] + [(0.9, *k) for k in KERNELS_DENSE])
def test_every_kernel(keep, plan, M, K, N):
    A, w = matrix(M + N, M, K, keep, low=-128)
    assert A.plan(N).startswith(plan + " "), A.plan(N)
    xq, s, x = tokens(M, N, K)
    b = half(3, M)
    want, tol = blocks64.product(x, w, f64(b), "relu")
    y = A.spmm(xq, s, bias=b, activation="relu")
    blocks64.close(y.cpu().numpy(), want, tol)
    assert torch.equal(A.spmm(xq, s, bias=b, activation="relu"), y)  # bitwise reproducible


@pytest.mark.parametrize("N", [200, 900, 2048])
@pytest.mark.parametrize("keep", [0.5, 0.9])
def test_wide_kernels(N, keep):
    """Many tokens on enough rows for every form of the wide kernel, with the whole epilogue."""
    M, K = 2500, 515
    A, w = matrix(95, M, K, keep)
    xq, s, x = tokens(96, N, K)
    b, r = half(97, M), half(98, N, M)
    want, tol = blocks64.product(x, w, f64(b), "silu", f64(r))
    blocks64.close(A.spmm(xq, s, bias=b, residual=r, activation="silu").cpu().numpy(), want, tol)
    wide = torch.full((N, M + 7), 3.0, dtype=torch.float16, device="cuda")  # no vector stores
    usp.usp_spmm_q(A.handle, xq, s, wide[:, 1:1 + M], A.make_workspace(N), b, r, "silu")
    assert torch.equal(wide[:, 1:1 + M], A.spmm(xq, s, bias=b, residual=r, activation="silu"))
    assert (wide[:, 0] == 3).all() and (wide[:, 1 + M:] == 3).all()


def test_two_streams():
    """Two modules' calls on two streams at once, and one module's."""
    w = torch.randn(1500, 2000).half().cuda()
    mask = torch.rand(1500, 2000) < 0.5
    codes, scale = linear.quantize_rows(w, mask)
    mod = linear.SparseLinearQ(codes, mask, scale)
    xs = [half(100 + i, 64 + 200 * i, 2000) for i in range(2)]
    want = [mod(x) for x in xs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in xs]
    got = [[], []]
    for _ in range(10):
        for i, x in enumerate(xs):
            with torch.cuda.stream(streams[i]):
                got[i].append(mod(x))
    torch.cuda.synchronize()
    assert all(torch.equal(g, want[i]) for i in range(2) for g in got[i])


@pytest.mark.parametrize("K,ld,offset", [(8, 8, 0), (16, 24, 8), (100, 104, 0), (2056, 2056, 0), (8191, 8200, 0), (8200, 8208, 0),
                                         (8200, 8201, 0), (8448, 8448, 4), (20000, 20008, 0), (33001, 33001, 1)])
@pytest.mark.parametrize("N", [17, 35, 300])
def test_fp16_tokens_at_every_width(K, ld, offset, N):
    """Rows shorter and longer than what a thread keeps, aligned and not, in a buffer of NaN,
    with tokens of zeros, of a NaN and of an infinity: the bits of the two calls."""
    A, _ = matrix(90, 40, K, 0.5)
    buf = torch.full((N * ld + offset + 64,), float("nan"), dtype=torch.float16, device="cuda")
    x = torch.as_strided(buf, (N, K), (ld, 1), offset)
    x.copy_(half(91, N, K))
    x[2] = 0
    x[5, K // 2] = float("nan")
    x[N - 1, K - 1] = float("-inf")
    xq, s = torch.empty(N, K, dtype=torch.int8, device="cuda"), torch.empty(N, device="cuda")
    usp.usp_quantize(x, xq, s)
    got, want = A.spmm(x), A.spmm(xq, s)
    bad = torch.isnan(want).all(1).nonzero().flatten().tolist()
    assert bad == [5, N - 1] and torch.isnan(got[bad]).all()
    keep = [n for n in range(N) if n not in bad]
    assert torch.equal(got[keep], want[keep])
