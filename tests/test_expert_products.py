"""Products grouped by expert against the plain form in 64 bits, and the norms, experts and 8-bit layers together
(GPU)."""
import numpy as np
import pytest
import torch

import blocks64
from paper_2607_08786_amd import linear, usp

pytestmark = pytest.mark.gpu


def group(seed, E, M, K, q, keep=0.5):
    rng = np.random.default_rng(seed)
    mats, dense = [], []
    for _ in range(E):
        mask = (rng.random((M, K)) < keep).astype(np.uint8)
        if q:
            W, s = rng.integers(-128, 128, (M, K)).astype(np.int8), (rng.random(M) * 2e-3 + 1e-5).astype(np.float32)
            mats.append(usp.SparseMatrixQ(W, mask, s))
            dense.append(np.where(mask != 0, W, 0).astype(np.float64) * s[:, None].astype(np.float64))
        else:
            W = (rng.standard_normal((M, K)) * 0.1).astype(np.float16)
            mats.append(usp.SparseMatrix(W, mask))
            dense.append(np.where(mask != 0, W, 0).astype(np.float64))
    return usp.ExpertGroup(mats), dense


def inputs(seed, n, K, q):
    rng = np.random.default_rng(seed)
    if not q:
        x = rng.standard_normal((n, K)).astype(np.float16)
        return torch.from_numpy(x).cuda(), None, x.astype(np.float64)
    x, s = rng.integers(-128, 128, (n, K)).astype(np.int8), (rng.random(n) * 0.05 + 1e-3).astype(np.float32)
    return torch.from_numpy(x).cuda(), torch.from_numpy(s).cuda(), x.astype(np.float64) * s.astype(np.float64)[:, None]


def i32(v):
    return torch.tensor(np.asarray(v), dtype=torch.int32, device="cuda")


def plain(dense, x, ends, K, q, rows=None, bias=None, act="none", weight=None, untouched=0.0):
    """ends: (first, last + 1) of every expert's rows."""
    T = len(rows) if rows is not None else x.shape[0]
    want, tol = np.full((T, dense[0].shape[0]), untouched), np.zeros((T, dense[0].shape[0]))
    if rows is not None:
        x = np.stack([x[r] if 0 <= r < x.shape[0] else np.zeros(K) for r in rows])
    for e, (lo, hi) in enumerate(ends):
        if hi > lo:
            want[lo:hi], tol[lo:hi] = blocks64.product(x[lo:hi], dense[e], None if bias is None else bias[e], act, None,
                                                       None if weight is None else weight[lo:hi],
                                                       32 if q else blocks64.f16_sums(K))
    return want, tol


# Counts of rows per expert: none at all, one, around a block of 16 and of 32, one expert with nearly all, many experts.
COUNTS = {
    "one": [1],
    "empty": [0, 0, 0],
    "gaps": [0, 3, 0, 1, 17, 0],
    "edges": [16, 15, 17, 32, 31, 33],
    "skewed": [2, 300, 0, 1],
    "many": [(7 * e) % 5 for e in range(130)],
    "long": [520, 129, 65],
}


@pytest.mark.parametrize("q", [False, True])
@pytest.mark.parametrize("name", sorted(COUNTS))
@pytest.mark.parametrize("M,K", [(1, 8), (33, 264), (200, 1111), (70, 2048)])
def test_counts(name, M, K, q):
    counts = COUNTS[name]
    ends = np.cumsum([0] + counts)
    G, dense = group(len(counts), len(counts), M, K, q)
    T = max(1, int(ends[-1]))
    X, s, x = inputs(3, T, K, q)
    Y = torch.full((T, M), 7.0, dtype=torch.float16, device="cuda")
    usp.usp_spmm_grouped(G.handle, X, i32(ends), Y, G.make_workspace(T), x_scale=s)
    want, tol = plain(dense, x, list(zip(ends[:-1], ends[1:])), K, q, untouched=7.0)
    blocks64.close(Y.cpu().numpy(), want, tol)


@pytest.mark.parametrize("q", [False, True])
@pytest.mark.parametrize("K", [256, 300, 515])
def test_gather_bias_weight(K, q):
    """Rows gathered with repeats, an activation, biases and weights per row; indices outside X are rows of zeros."""
    E, M, T = 5, 130, 77
    counts = [20, 0, 30, 7, 20]
    ends = np.cumsum([0] + counts)
    G, dense = group(21, E, M, K, q)
    X, s, x = inputs(22, 40, K, q)
    rng = np.random.default_rng(23)
    rows = rng.integers(0, 40, T)
    rows[5], rows[33], rows[76] = -1, 40, 2 ** 31 - 1
    b, w = rng.standard_normal((E, M + 1)).astype(np.float16), rng.random(T).astype(np.float32)
    bias = torch.from_numpy(b).cuda()[:, 1:]
    Y = torch.empty(T, M, dtype=torch.float16, device="cuda")
    usp.usp_spmm_grouped(G.handle, X, i32(ends), Y, G.make_workspace(T), x_scale=s, rows=i32(rows), bias=bias,
                         row_weight=torch.from_numpy(w).cuda(), activation="silu")
    want, tol = plain(dense, x, list(zip(ends[:-1], ends[1:])), K, q, rows, b[:, 1:].astype(np.float64), "silu",
                      w.astype(np.float64))
    blocks64.close(Y.cpu().numpy(), want, tol)


@pytest.mark.parametrize("q", [False, True])
def test_offsets_of_any_value(q):
    """Offsets outside [0, T] count as the nearer end, decreasing ones as the one before; rows before the first offset
    and behind the last are left alone."""
    M, K, T = 48, 256, 60
    G, dense = group(31, 6, M, K, q)
    X, s, x = inputs(32, T, K, q)
    for off in ([4, 10, 7, 30, 30, 41, 50], [-5, 10, 2 ** 31 - 1, 3, 70, 60, -1], [60] * 7, [0] * 7):
        seen = np.maximum.accumulate(np.clip(off, 0, T))
        Y = torch.full((T, M), 7.0, dtype=torch.float16, device="cuda")
        usp.usp_spmm_grouped(G.handle, X, i32(off), Y, G.make_workspace(T), x_scale=s)
        want, tol = plain(dense, x, list(zip(seen[:-1], seen[1:])), K, q, untouched=7.0)
        blocks64.close(Y.cpu().numpy(), want, tol)


@pytest.mark.parametrize("ld,offset", [(520, 0), (513, 0), (514, 2), (522, 1)])
@pytest.mark.parametrize("q", [False, True])
@pytest.mark.parametrize("K", [512, 509])
def test_strides(ld, offset, q, K):
    """X and Y inside larger buffers; what follows a row of X may be anything (NaN)."""
    counts = [10, 0, 25]
    ends = np.cumsum([0] + counts)
    G, dense = group(41, 3, 64, K, q)
    X, s, x = inputs(42, 35, K, q)
    buf = torch.full((35 * ld + offset + 64,), 99 if q else float("nan"), dtype=X.dtype, device="cuda")
    view = torch.as_strided(buf, (35, K), (ld, 1), offset)
    view.copy_(X)
    Y = torch.full((35, 70), 7.0, dtype=torch.float16, device="cuda")
    usp.usp_spmm_grouped(G.handle, view, i32(ends), Y[:, 3:67], G.make_workspace(35), x_scale=s)
    want, tol = plain(dense, x, list(zip(ends[:-1], ends[1:])), K, q)
    blocks64.close(Y[:, 3:67].cpu().numpy(), want, tol)
    assert (Y[:, :3] == 7).all() and (Y[:, 67:] == 7).all()


def test_nan_stays_in_its_row():
    for q in (False, True):
        G, _ = group(51, 2, 40, 300, q)
        X, s, _ = inputs(52, 30, 300, q)
        off = i32([0, 12, 30])
        clean = G.spmm(X, off, x_scale=s)
        if q:
            s = s.clone()
            s[5] = float("nan")
        else:
            X[5, 7] = float("nan")
        got = G.spmm(X, off, x_scale=s)
        keep = (torch.arange(30) != 5).cuda()
        assert torch.isnan(got[5]).any() and torch.equal(got[keep], clean[keep])


@pytest.mark.parametrize("q", [False, True])
@pytest.mark.parametrize("T", [24, 400])
def test_captured_with_other_counts(q, T):
    """A replay serves the counts that the offsets hold then."""
    G, dense = group(61, 4, 96, 515, q)
    X, s, x = inputs(62, T, 515, q)
    off, rows = i32([0] * 5), i32(np.arange(T))
    Y, ws = torch.empty(T, 96, dtype=torch.float16, device="cuda"), G.make_workspace(T)
    usp.usp_spmm_grouped(G.handle, X, off, Y, ws, x_scale=s, rows=rows)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        usp.usp_spmm_grouped(G.handle, X, off, Y, ws, x_scale=s, rows=rows)
    rng = np.random.default_rng(63)
    for cuts in ([0, T, T, T], [1, 2, 3, T], [T // 2, T // 2, T - 5, T - 1]):
        ends = np.array([0] + cuts)
        off.copy_(i32(ends))
        index = rng.integers(0, T, T)
        rows.copy_(i32(index))
        Y.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        want, tol = plain(dense, x, list(zip(ends[:-1], ends[1:])), 515, q, index, untouched=7.0)
        blocks64.close(Y.cpu().numpy(), want, tol)


def test_same_expert_twice_and_lifetime():
    """An expert may occur twice; a handle that a group holds is not freed; a freed group is refused."""
    G, dense = group(71, 2, 32, 256, False)
    a, b = G.experts
    H = usp.ExpertGroup([a, b, a])
    X, _, x = inputs(72, 9, 256, False)
    want, tol = plain([dense[0], dense[1], dense[0]], x, [(0, 3), (3, 6), (6, 9)], 256, False)
    blocks64.close(H.spmm(X, i32([0, 3, 6, 9])).cpu().numpy(), want, tol)
    handle = H.handle
    for _ in range(2):
        with pytest.raises(usp.UspError):
            usp.usp_free(a.handle)
        H.free()
    with pytest.raises(usp.UspError):
        usp.usp_spmm_grouped(handle, X, i32([0, 3, 6, 9]), torch.empty(9, 32, dtype=torch.float16, device="cuda"))
    with pytest.raises(usp.UspError):
        usp.usp_group_free(handle)
    G.free()
    a.free()
    assert a.handle is None


def test_refusals():
    G, _ = group(81, 2, 32, 256, False)
    X, _, _ = inputs(82, 9, 256, False)
    off, Y = i32([0, 3, 9]), torch.empty(9, 32, dtype=torch.float16, device="cuda")
    ws = G.make_workspace(9)
    usp.usp_spmm_grouped(G.handle, X, off, Y, ws)
    for bad in (dict(offsets=off[:2]), dict(offsets=i32([0, 3, 9, 9])), dict(X=X[:4]), dict(activation=7),
                dict(x_scale=torch.ones(9, device="cuda"), X=X.to(torch.int8))):
        with pytest.raises(usp.UspError):
            usp.usp_spmm_grouped(G.handle, **{"X": X, "offsets": off, "Y": Y, "workspace": ws, **bad})
    for bad in (dict(offsets=off.long()), dict(rows=i32([0])), dict(bias=X[:2, :31]), dict(row_weight=torch.ones(8, device="cuda")),
                dict(offsets=off.cpu())):
        with pytest.raises((TypeError, ValueError)):
            usp.usp_spmm_grouped(G.handle, **{"X": X, "offsets": off, "Y": Y, "workspace": ws, **bad})
    Y.fill_(5.0)
    usp.usp_spmm_grouped(G.handle, X[:0].expand(0, 256), off, Y[:0], ws)  # no rows: nothing is done
    assert (Y == 5).all()
    other, _ = group(83, 1, 32, 512, False)
    eight, _ = group(84, 1, 32, 256, True)
    for m in (other.experts[0], eight.experts[0]):
        with pytest.raises(usp.UspError):
            usp.ExpertGroup([G.experts[0], m])


@pytest.mark.parametrize("q", [False, True])
def test_module_of_a_routed_block(q):
    """Norm, experts on the tokens' two best choices, their sum back to tokens, norm with 8-bit output, an 8-bit
    layer: as a decoder block uses them, against 64 bits step by step."""
    hidden, ffn, E, n, top = 256, 320, 6, 20, 2
    rng = np.random.default_rng(91)

    def experts(M, K, act):
        w = [torch.from_numpy((rng.standard_normal((M, K)) * 0.05).astype(np.float16)).cuda() for _ in range(E)]
        m = [torch.from_numpy(rng.random((M, K)) < 0.5).cuda() for _ in range(E)]
        if not q:
            return linear.SparseExperts(w, m, activation=act), [(a * b).double().cpu().numpy() for a, b in zip(w, m)]
        coded = [linear.quantize_rows(a, b) for a, b in zip(w, m)]
        return (linear.SparseExperts([c for c, _ in coded], m, [s for _, s in coded], activation=act),
                [(c * b).double().cpu().numpy() * s.double().cpu().numpy()[:, None] for (c, s), b in zip(coded, m)])

    up, up_w = experts(ffn, hidden, "silu")
    down, down_w = experts(hidden, ffn, "none")
    before, after = linear.BlockNorm(hidden, pre="rms"), linear.BlockNorm(hidden, post="rms", pre="rms", scale=0.5)
    out_w = torch.from_numpy((rng.standard_normal((100, hidden)) * 0.05).astype(np.float16)).cuda()
    out_mask = torch.from_numpy(rng.random((100, hidden)) < 0.5).cuda()
    codes, scale = linear.quantize_rows(out_w, out_mask)
    out = linear.SparseLinearQ(codes, out_mask, scale)

    x = torch.from_numpy(rng.standard_normal((n, hidden)).astype(np.float16)).cuda()
    choice = torch.from_numpy(np.stack([rng.permutation(E)[:top] for _ in range(n)])).cuda()
    share = torch.from_numpy(rng.random((n, top)).astype(np.float32)).cuda()
    flat = choice.reshape(-1)
    order = torch.argsort(flat, stable=True)
    rows, weight = (order // top).to(torch.int32), share.reshape(-1)[order].contiguous()
    offsets = torch.zeros(E + 1, dtype=torch.int32, device="cuda")
    offsets[1:] = torch.bincount(flat, minlength=E).cumsum(0)

    _, h = before(x, quantize=q)
    u = up(h, offsets, rows)
    d = down(u, offsets, row_weight=weight)
    y = torch.empty_like(d).index_copy_(0, order, d).reshape(n, top, hidden).float().sum(1).half()
    r, h2 = after(x, y, quantize=True)
    z = out(h2)

    ends = list(zip(offsets[:-1].tolist(), offsets[1:].tolist()))
    stands = lambda t: t[0].double().cpu().numpy() * t[1].double().cpu().numpy()[:, None] if isinstance(t, tuple) else t.double().cpu().numpy()  # noqa: E731
    want, tol = plain(up_w, stands(h), ends, hidden, q, rows.cpu().numpy(), act="silu")
    blocks64.close(u.cpu().numpy(), want, tol)
    u64 = u.cpu().numpy()
    if q:
        c, s = blocks64.quantize(u64)
        u64 = c.astype(np.float64) * s.astype(np.float64)[:, None]
    want, tol = plain(down_w, u64.astype(np.float64), ends, ffn, q, weight=weight.double().cpu().numpy())
    blocks64.close(d.cpu().numpy(), want, tol)
    ones = np.ones(hidden)
    want = blocks64.norm(x.double().cpu().numpy(), y.double().cpu().numpy(), None, 0.5, "rms", ones, None, "rms", ones)
    blocks64.close(r.cpu().numpy(), want[0], want[1])
    want, tol = blocks64.product(stands(h2), (codes * out_mask).double().cpu().numpy() * scale.double().cpu().numpy()[:, None])
    blocks64.close(z.cpu().numpy(), want, tol)


@pytest.mark.parametrize("q", [False, True])
@pytest.mark.parametrize("keep", [0.5, 1.0])
def test_prefill(q, keep):
    """Many ragged rows on the wide kernel, gathered, weighted, with a bias per expert; dense records too."""
    E, M, K = 4, 700, 776
    counts = [700, 0, 33, 515]
    ends = np.cumsum([0] + counts)
    T = int(ends[-1])
    G, dense = group(101, E, M, K, q, keep)
    assert G.plan(8192).startswith("wide-product")
    X, s, x = inputs(102, 900, K, q)
    rng = np.random.default_rng(103)
    rows, w = rng.integers(0, 900, T), rng.random(T).astype(np.float32)
    b = rng.standard_normal((E, M)).astype(np.float16)
    for total in (T, 8192):  # the second with rows behind the last expert's
        Y = torch.full((total, M), 7.0, dtype=torch.float16, device="cuda")
        index = np.zeros(total, np.int64)
        index[:T] = rows
        weight = np.ones(total, np.float32)
        weight[:T] = w
        usp.usp_spmm_grouped(G.handle, X, i32(ends), Y, G.make_workspace(total), x_scale=s, rows=i32(index),
                             bias=torch.from_numpy(b).cuda(), row_weight=torch.from_numpy(weight).cuda(), activation="silu")
        want, tol = plain(dense, x, list(zip(ends[:-1], ends[1:])), K, q, index, b.astype(np.float64), "silu",
                          weight.astype(np.float64), untouched=7.0)
        blocks64.close(Y.cpu().numpy(), want, tol)



# Every fp16 kernel of the planner at a small shape that takes it: (plan, M, K, T, experts), for records of up to 5 KB and
# larger ones.
KERNELS = [
    ("product R=1 W=4 nb=1", 16, 206, 1, 1),
    ("product R=1 W=4 nb=2", 37, 8860, 1432, 1),
    ("product R=1 W=8 nb=1", 16, 1038, 2, 1),
    ("product R=2 W=4 nb=1", 22, 814, 2041, 2),
    ("product R=2 W=4 nb=2", 197, 747, 2045, 2),
    ("product R=2 W=8 nb=1", 22, 1554, 2035, 2),
    ("product R=2 W=8 nb=2", 68, 4491, 1979, 1),
    ("product R=4 W=4 nb=1", 262, 635, 1363, 1),
    ("product R=4 W=4 nb=2", 391, 520, 1906, 1),
    ("product R=4 W=8 nb=1", 76, 1689, 1757, 1),
    ("product R=4 W=8 nb=2", 141, 2892, 1955, 1),
    ("wide-product R=4 nb=2", 434, 1085, 1759, 1),
    ("wide-product R=4 nb=4", 2068, 365, 1978, 1),
    ("wide-product R=8 nb=2", 2648, 246, 1510, 1),
]
KERNELS_DENSE = [
    ("product R=1 W=4 nb=1", 16, 205, 1, 1),
    ("product R=1 W=4 nb=2", 38, 6019, 1545, 1),
    ("product R=1 W=8 nb=1", 16, 1053, 4, 1),
    ("product R=1 W=8 nb=2", 38, 7405, 2042, 1),
    ("product R=2 W=4 nb=1", 20, 815, 2043, 3),
    ("product R=2 W=4 nb=2", 271, 670, 1655, 1),
    ("product R=2 W=8 nb=1", 23, 1419, 2046, 1),
    ("product R=2 W=8 nb=2", 56, 3078, 2041, 1),
    ("product R=4 W=4 nb=1", 204, 604, 1816, 1),
    ("product R=4 W=4 nb=2", 2622, 270, 476, 6),
    ("product R=4 W=8 nb=1", 70, 1788, 1788, 1),
    ("product R=4 W=8 nb=2", 132, 2371, 1838, 1),
    ("wide-product R=4 nb=2", 306, 561, 1679, 1),
    ("wide-product R=4 nb=4", 1095, 208, 1706, 2),
]


@pytest.mark.parametrize("keep,plan,M,K,T,E", [(0.5, *k) for k in KERNELS] + [(0.95, *k) for k in KERNELS_DENSE])
def test_every_kernel(keep, plan, M, K, T, E):
    G, dense = group(M + T, E, M, K, False, keep)
    assert G.plan(T).startswith(plan + " "), G.plan(T)
    ends = np.linspace(0, T, E + 1).astype(np.int64)
    X, _, x = inputs(T, T, K, False)
    Y = G.spmm(X, i32(ends))
    want, tol = plain(dense, x, list(zip(ends[:-1], ends[1:])), K, False)
    blocks64.close(Y.cpu().numpy(), want, tol)
    assert torch.equal(G.spmm(X, i32(ends)), Y)  # bitwise reproducible


def test_many_experts():
    """More experts than a wavefront has lanes, several times over, nearly all without rows."""
    G, dense = group(111, 3, 20, 256, False)
    E = 1000
    H = usp.ExpertGroup([G.experts[e % 3] for e in range(E)])
    counts = np.zeros(E, np.int64)
    counts[[0, 63, 64, 500, 999]] = [3, 20, 1, 40, 5]
    ends = np.cumsum(np.concatenate([[0], counts]))
    X, _, x = inputs(112, int(ends[-1]), 256, False)
    want, tol = plain([dense[e % 3] for e in range(E)], x, list(zip(ends[:-1], ends[1:])), 256, False)
    blocks64.close(H.spmm(X, i32(ends)).cpu().numpy(), want, tol)
    with pytest.raises(usp.UspError):
        usp.ExpertGroup([G.experts[0]] * 4097)
