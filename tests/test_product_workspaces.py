"""Workspaces of the 8-bit and grouped products (GPU): no larger than what is packed, filled with anything, of exactly the
stated size, with nothing written beside it or over the counters that fp16 products keep there."""
import numpy as np
import pytest
import torch

import test_expert_products as experts
import test_quantized_products as quantized
from paper_2607_08786_amd import usp

pytestmark = pytest.mark.gpu

COUNTERS = 256 << 10


def matrix_q(M, K):
    return usp.SparseMatrixQ(np.ones((M, K), np.int8), np.ones((M, K), np.uint8), np.ones(M, np.float32))


@pytest.mark.parametrize("K", [1000, 8192, 28672])
def test_sizes(K):
    """X packed in whole blocks of 16 tokens and what a workgroup may read past them: 4 blocks up to 16 tokens, 32 above."""
    A = matrix_q(16, K)
    B = usp.SparseMatrix(np.ones((16, K), np.uint16), np.ones((16, K), np.uint8))
    for N in (1, 16, 17, 300, 2048):
        tiles, spare = -(-K // 256), 4 if N <= 16 else 32
        block = 16 * 256 * tiles
        assert A.workspace_size(N) <= COUNTERS + (-(-N // 16) + spare) * block + 4 * N
        for group, value, count in ((usp.ExpertGroup([A] * 3), 1, 3), (usp.ExpertGroup([B] * 40), 2, 40)):
            assert group.workspace_size(N) <= COUNTERS + (N // 16 + min(count, N) + spare) * block * value


def guarded(need):
    """`need` bytes of NaN patterns between guards, and the whole buffer."""
    buf = torch.full((need + 8192,), 0xFF, dtype=torch.uint8, device="cuda")
    return buf, buf[4096:4096 + need]


def untouched(buf, ws):
    return bool((buf[:4096 + COUNTERS] == 0xFF).all()) and bool((buf[4096 + ws.numel():] == 0xFF).all())


@pytest.mark.parametrize("keep,plan,M,K,N", [(0.5, *k) for k in quantized.KERNELS] + [(0.9, *k) for k in quantized.KERNELS_DENSE])
def test_8_bit(keep, plan, M, K, N):
    A, _ = quantized.matrix(M + N, M, K, keep)
    xq, s, _ = quantized.tokens(M, N, K)
    odd, s_odd, _ = quantized.tokens(M, N, K, K + 3, 1)  # packed whatever the plan
    x16 = quantized.half(M, N, K)
    for x, scale in ((xq, s), (odd, s_odd), (x16, None)):
        want = A.spmm(x, scale)
        buf, ws = guarded(A.workspace_size(N))
        assert torch.equal(A.spmm(x, scale, workspace=ws), want)
        assert untouched(buf, ws)


@pytest.mark.parametrize("keep,plan,M,K,T,E", [(0.5, *k) for k in experts.KERNELS] + [(0.95, *k) for k in experts.KERNELS_DENSE])
def test_grouped(keep, plan, M, K, T, E):
    G, _ = experts.group(M + T, E, M, K, False, keep)
    ends = experts.i32(np.linspace(0, T, E + 1).astype(np.int64))
    wide = torch.full((T, K + 3), float("nan"), dtype=torch.float16, device="cuda")
    wide[:, 1:K + 1] = experts.inputs(T, T, K, False)[0]
    for x in (wide[:, 1:K + 1].contiguous(), wide[:, 1:K + 1]):
        want = G.spmm(x, ends)
        buf, ws = guarded(G.workspace_size(T))
        assert torch.equal(G.spmm(x, ends, workspace=ws), want)
        assert untouched(buf, ws)


@pytest.mark.parametrize("group", [False, True])
def test_only_the_counters_are_cleared(group):
    """usp_spmm needs those; the rest would be megabytes for every module, stream and replay."""
    A = matrix_q(16, 8192)
    A = usp.ExpertGroup([A]) if group else A
    N = 300
    need = A.workspace_size(N)
    torch.cuda.empty_cache()
    torch.full((need,), 0xFF, dtype=torch.uint8, device="cuda")  # its memory is the next tensor's
    ws = A.make_workspace(N)
    assert (ws[:COUNTERS] == 0).all() and (ws[COUNTERS:] == 0xFF).any()


@pytest.mark.parametrize("N", [3, 40, 700])
def test_capture_without_a_warm_up(N):
    """The graph allocates its workspaces itself; replays between eager calls give the eager bits."""
    from paper_2607_08786_amd import linear
    g = torch.Generator().manual_seed(N)
    codes, mask = torch.randint(-9, 9, (3, 300, 515), generator=g).to(torch.int8), torch.rand(3, 300, 515, generator=g) < 0.5
    scale = torch.full((300,), 0.01)
    layer = linear.SparseLinearQ(codes[0], mask[0], scale)
    routed = linear.SparseExperts(list(codes[1:]), list(mask[1:]), [scale, scale])
    offsets = experts.i32([0, N // 3, N])
    x = quantized.half(1, N, 515)
    usp.usp_quantize(x, torch.empty(N, 515, dtype=torch.int8, device="cuda"), torch.empty(N, device="cuda"))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y, z = layer(x), routed(x, offsets)
    for k in range(4):
        x.copy_(quantized.half(2 + k, N, 515))
        graph.replay()
        torch.cuda.synchronize()
        got = y.clone(), z.clone()
        assert torch.equal(layer(x), got[0]) and torch.equal(routed(x, offsets), got[1])
        torch.cuda.synchronize()
