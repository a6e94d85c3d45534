"""Records of 8-bit values on the CPU (the library's encoder built with g++): bit-exact round trips, the record's
layout as usp_format.h states it, and the refusals of the entry points that need no GPU."""
import ctypes
import os
import subprocess

import numpy as np
import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def hlib(tmp_path_factory):
    out = str(tmp_path_factory.mktemp("hostq") / "libq.so")
    src = [os.path.join(ROOT, "tests", "native", "encode_q_test.cpp"),
           os.path.join(ROOT, "paper_2607_08786_amd", "csrc", "usp_encode.cpp")]
    subprocess.run(["g++", "-O1", "-g", "-std=c++17", "-fPIC", "-shared", "-fsanitize=undefined",
                    "-fno-sanitize-recover=all", "-I", os.path.join(ROOT, "include"), *src, "-o", out, "-lpthread"],
                   check=True)
    lib = ctypes.CDLL(out)
    p, i64 = ctypes.c_void_p, ctypes.c_int64
    lib.usp_test_q.argtypes = [p, i64, p, i64, i64, i64, p, p, p, p, i64, p]
    return lib


def encode(lib, W, mask, pad=0):
    M, K = W.shape
    Wl, ml = np.full((M, K + pad), 77, np.int8), np.ones((M, K + pad), np.uint8)
    Wl[:, :K], ml[:, :K] = W, mask
    tiles = -(-M // 16) * -(-K // 256)
    Wo, mo, nnz = np.empty_like(W), np.empty((M, K), np.uint8), ctypes.c_int64()
    stream, off = np.zeros(tiles * (528 + 4096), np.uint8), np.zeros(tiles + 1, np.uint32)
    rc = lib.usp_test_q(Wl.ctypes.data, K + pad, ml.ctypes.data, K + pad, M, K, Wo.ctypes.data, mo.ctypes.data,
                        ctypes.byref(nnz), stream.ctypes.data, stream.size, off.ctypes.data)
    assert rc == 0, rc
    return Wo, mo, nnz.value, stream, off


@pytest.mark.parametrize("M,K,keep,pad", [(1, 1, 1.0, 0), (16, 256, 0.5, 0), (17, 257, 0.5, 3), (33, 700, 0.0, 0),
                                          (48, 512, 1.0, 0), (5, 15, 0.3, 1), (64, 1030, 0.6, 7)])
def test_round_trip(hlib, M, K, keep, pad):
    rng = np.random.default_rng(M * 1000 + K)
    W = rng.integers(-128, 128, (M, K)).astype(np.int8)
    mask = (rng.random((M, K)) < keep).astype(np.uint8) * rng.integers(1, 256, (M, K)).astype(np.uint8)
    Wo, mo, nnz, _, off = encode(hlib, W, mask, pad)
    kept = mask != 0
    assert np.array_equal(Wo, np.where(kept, W, 0)) and np.array_equal(mo, kept.astype(np.uint8))
    assert nnz == kept.sum()
    RB, KT = -(-M // 16), -(-K // 256)
    padded = np.zeros((RB * 16, KT * 256), bool)
    padded[:M, :K] = kept
    per_tile = padded.reshape(RB, 16, KT, 256).sum(axis=(1, 3)).reshape(-1)
    assert np.array_equal(np.diff(off.astype(np.int64)) * 16, 528 + (per_tile + 15) // 16 * 16)


def test_layout(hlib):
    """Position (r, 64 s + 16 g + j) is bit 16 s + j of lane 16 g + r; its value lies in the block of its mask byte behind
    those of the lanes before and of the byte's bits before; the blocks' starts stand between mask and values."""
    rng = np.random.default_rng(5)
    W = rng.integers(-128, 128, (16, 256)).astype(np.int8)
    mask = (rng.random((16, 256)) < 0.5).astype(np.uint8)
    _, _, _, stream, _ = encode(hlib, W, mask)
    lanes = stream[:512].reshape(64, 8).copy().view(np.uint64)[:, 0]
    values, starts = [], []
    for y in range(8):
        starts.append(528 + len(values))
        for lane in range(64):
            r, g = lane % 16, lane // 16
            for j in range(8):
                bit = 8 * y + j
                col = 64 * (bit // 16) + 16 * g + bit % 16
                assert (int(lanes[lane]) >> bit & 1) == mask[r, col]
                if mask[r, col]:
                    values.append(W[r, col])
    assert np.array_equal(stream[528:528 + len(values)].view(np.int8), np.array(values, np.int8))
    assert stream[512:528].view(np.uint16).tolist() == [starts[y] for y in (0, 2, 1, 3, 4, 6, 5, 7)]


def test_refusals_without_device():
    """Every refusal below comes before a device is looked for."""
    from paper_2607_08786_amd import usp
    lib, p = usp.load_library(), ctypes.c_void_p
    h = p()
    buf, mb, sc = (ctypes.c_int8 * 16)(), (ctypes.c_uint8 * 16)(), (ctypes.c_float * 4)(1, 1, 1, 1)

    def err(code, rc, text):
        assert rc == code, (rc, usp.usp_last_error())
        assert text in usp.usp_last_error()

    err(1, lib.usp_encode_q(buf, 4, mb, 4, None, 4, 4, 0, ctypes.byref(h)), "null")
    err(1, lib.usp_encode_q(None, 4, mb, 4, sc, 4, 4, 0, ctypes.byref(h)), "null")
    err(1, lib.usp_encode_q(buf, 3, mb, 4, sc, 4, 4, 0, ctypes.byref(h)), "ldw")
    err(2, lib.usp_encode_q(buf, 1 << 20, mb, 1 << 20, sc, 4, usp.MAX_K_Q + 1, 0, ctypes.byref(h)), "USP_MAX_K_Q")
    bad = (ctypes.c_float * 4)(1, float("inf"), 1, 1)
    err(1, lib.usp_encode_q(buf, 4, mb, 4, bad, 4, 4, 0, ctypes.byref(h)), "finite")
    assert h.value is None
    junk = ctypes.cast(ctypes.create_string_buffer(b"\xff" * 512), p)
    err(1, lib.usp_decode_q(junk, buf, mb, sc), "invalid or freed")
    err(1, lib.usp_spmm_q(junk, junk, 8, junk, junk, 8, 1, None, None, 0, 0, None, 0, None), "invalid or freed")
    g = p()
    err(1, lib.usp_group_create(None, 1, ctypes.byref(g)), "null")
    err(1, lib.usp_group_create(ctypes.byref(junk), 0, ctypes.byref(g)), "E must be")
    err(1, lib.usp_group_create(ctypes.byref(junk), 1, ctypes.byref(g)), "invalid or freed")
    assert g.value is None and lib.usp_group_free(None) == 0
    err(1, lib.usp_group_free(junk), "already freed")
    assert lib.usp_group_workspace_size(junk, 16) == 0 and lib.usp_group_workspace_size(None, 16) == 0
    err(1, lib.usp_spmm_grouped(junk, junk, 8, 1, None, None, junk, 1, junk, 8, 1, None, 0, None, 0, None, 0, None),
        "invalid or freed")
    err(1, lib.usp_quantize(None, 8, 1, 8, junk, 8, junk, 0, None), "null")
    err(1, lib.usp_quantize(junk, 8, 0, 8, junk, 8, junk, 0, None), "N and K")
    err(1, lib.usp_quantize(junk, 7, 1, 8, junk, 8, junk, 0, None), "strides")
    err(1, lib.usp_quantize(junk, 8, 1, 8, junk, 8, p(junk.value + 1), 0, None), "aligned")
    err(2, lib.usp_quantize(junk, 8, (1 << 20) + 1, 8, junk, 8, junk, 0, None), "N above")
    err(1, lib.usp_norm(None, 1, 8, 0, None), "null")


@pytest.mark.parametrize("change,text", [
    (dict(residual=None), "null input"), (dict(out=None), "no output"), (dict(out_q=1), "out_scale"),
    (dict(pre_kind=3), "unknown norm"), (dict(post_kind=-1), "unknown norm"), (dict(gate_activation=4), "unknown gate"),
    (dict(post_kind=1, y=None), "need y"), (dict(gate=1, y=None), "need y"), (dict(eps=-1.0), "eps"),
    (dict(eps=float("nan")), "eps"), (dict(ld_out=7), "strides"), (dict(ld_residual=0), "strides"),
    (dict(gate=1, ld_gate=7), "strides"), (dict(y=3), "aligned"), (dict(pre_weight=3), "aligned"),
])
def test_norm_refusals_without_device(change, text):
    from paper_2607_08786_amd import usp
    keep = ctypes.create_string_buffer(64)
    base = ctypes.addressof(keep) + 15 & ~15
    a = usp.usp_norm_args(residual=base, y=base, out=base, ld_residual=8, ld_y=8, ld_out=8, ld_out_q=8, ld_gate=8,
                          scale=1.0, eps=0.0)
    for k, v in change.items():
        pointer = k in ("residual", "y", "gate", "out", "out_q", "pre_weight")
        setattr(a, k, None if v is None else base + (v if v == 3 else 0) if pointer else v)
    assert usp.load_library().usp_norm(ctypes.byref(a), 1, 8, 0, None) == 1
    assert text in usp.usp_last_error()


def test_operators_are_registered():
    import torch
    from torch._subclasses.fake_tensor import FakeTensorMode
    import paper_2607_08786_amd.linear  # noqa: F401
    with FakeTensorMode():
        x = torch.empty(7, 64, dtype=torch.float16)
        y = torch.ops.usp.sparse_linear_q(x, None, 0, 33, None, None, 1, None)
        off = torch.empty(3, dtype=torch.int32)
        z = torch.ops.usp.sparse_experts(x, None, off, None, None, 0, 33, True, None, 0, None)
        r, h, s = torch.ops.usp.block_norm(x, x, None, 1.0, "rms", None, None, "rms", None, None, 1e-5, "none", True)
    assert tuple(y.shape) == (7, 33) and y.dtype == torch.float16
    assert tuple(z.shape) == (7, 33) and z.dtype == torch.float16
    assert tuple(r.shape) == tuple(h.shape) == (7, 64) and h.dtype == torch.int8 and tuple(s.shape) == (7,)


def test_quantize_rows():
    """Codes of kept entries within half a step, the largest magnitude at 127, an empty row at scale 0."""
    import torch
    from paper_2607_08786_amd import linear
    g = torch.Generator().manual_seed(3)
    w = torch.randn(9, 50, generator=g)
    mask = torch.rand(9, 50, generator=g) < 0.5
    mask[4] = False
    codes, scale = linear.quantize_rows(w, mask)
    kept = torch.where(mask, w, torch.zeros(()))
    assert codes.dtype == torch.int8 and scale.dtype == torch.float32 and scale[4] == 0 and not codes[4].any()
    assert ((codes * scale[:, None] - kept).abs() <= scale[:, None] * (0.5 + 1e-4)).all()
    full = mask.any(1)
    assert (codes.abs().amax(1)[full] == 127).all()


def test_workspaces_go_by_the_stream_of_the_layers_device(monkeypatch):
    """A layer on another GPU than the current one enqueues on that GPU's current stream, and its workspaces are
    told apart by it: two streams there must not share one."""
    import types

    import torch

    from paper_2607_08786_amd import linear

    current = {0: 5, 1: 100}
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: False)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda device: current[device], raising=False)
    for cls in (linear.SparseLinearQ, linear.SparseExperts):
        layer = cls.__new__(cls)
        torch.nn.Module.__init__(layer)
        layer.matrix = types.SimpleNamespace(device=1, workspace_size=lambda N: 16,
                                             make_workspace=lambda N: torch.zeros(16, dtype=torch.uint8))
        layer._ws, layer._graph_ws = {}, []
        current[1] = 100
        first = layer.workspace(1)
        current[1] = 101
        assert layer.workspace(1) is not first
        current[1] = 100
        assert layer.workspace(1) is first


def test_width_of_the_input_is_checked():
    import types

    import torch

    from paper_2607_08786_amd import linear

    layer = linear.SparseLinearQ.__new__(linear.SparseLinearQ)
    torch.nn.Module.__init__(layer)
    layer.in_features, layer.out_features, layer.matrix = 8, 4, types.SimpleNamespace(device=0)
    with pytest.raises(ValueError, match="features"):
        layer(torch.zeros(2, 16, dtype=torch.float16))
    norm = linear.BlockNorm(8, device="cpu")
    with pytest.raises(ValueError, match="features"):
        norm(torch.zeros(2, 16, dtype=torch.float16))
