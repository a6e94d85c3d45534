"""Operands of another width than the weight's are refused: the C calls know strides alone, and rows of 8-bit tokens are
padded, so that the stride of too narrow ones can be wide enough."""
from types import SimpleNamespace

import numpy as np
import pytest
import torch

from paper_2607_08786_amd import linear, usp

M, K, N = 48, 110, 5


class Calls:
    """In place of the library: every call succeeds and is counted."""

    def __init__(self):
        self.made = 0

    def __getattr__(self, name):
        def call(*args):
            self.made += 1
            return 0
        return call


@pytest.fixture
def calls(monkeypatch):
    lib = Calls()
    monkeypatch.setattr(usp, "_lib", lib)
    monkeypatch.setattr(usp, "load_library", lambda: lib)
    monkeypatch.setattr(usp, "_gpu", lambda t, name: -1)
    monkeypatch.setattr(usp, "_stream_of", lambda stream, dev: 0)
    monkeypatch.setattr(usp, "_shapes", {1: (M, K), 2: (M, K)}, raising=False)
    return lib


def padded(rows, width, dtype=torch.int8):
    """Rows 128 elements apart: wide enough for the weight whatever their width."""
    return torch.zeros((rows, 128), dtype=dtype)[:, :width]


def module(cls, **also):
    m = cls.__new__(cls)
    torch.nn.Module.__init__(m)
    m._set_up((M, K), None, "none", 0)
    m.matrix = SimpleNamespace(handle=1 if cls is linear.SparseLinearQ else 2, device=0, workspace_size=lambda n: 0, **also)
    return m


@pytest.mark.parametrize("rows", [1, N])
@pytest.mark.parametrize("x_width,y_width", [(100, M), (K - 1, M), (K + 1, M), (K, M - 8), (K, M + 1)])
def test_bindings(calls, rows, x_width, y_width):
    y = padded(rows, y_width, torch.float16)
    offsets = torch.tensor([0, rows], dtype=torch.int32)
    for x, s in ((padded(rows, x_width), torch.ones(rows)), (padded(rows, x_width, torch.float16), None)):
        with pytest.raises(usp.UspError) as e:
            usp.usp_spmm_q(1, x, s, y)
        assert e.value.status == 1
        with pytest.raises(usp.UspError) as e:
            usp.usp_spmm_grouped(2, x, offsets, y, x_scale=s)
        assert e.value.status == 1
    assert calls.made == 0
    usp.usp_spmm_q(1, padded(rows, K), torch.ones(rows), padded(rows, M, torch.float16))
    usp.usp_spmm_grouped(2, padded(rows, K), offsets, padded(rows, M, torch.float16), x_scale=torch.ones(rows))
    assert calls.made == 2


@pytest.mark.parametrize("width", [100, K - 1, K + 1, 128])
def test_modules(calls, width):
    x, s = linear._int8_tokens(N, width, "cpu"), torch.ones(N)
    with pytest.raises(ValueError):
        module(linear.SparseLinearQ)((x, s))
    offsets = torch.tensor([0, N], dtype=torch.int32)
    experts = module(linear.SparseExperts, experts=[None])
    experts.eight_bit = True
    with pytest.raises(ValueError):
        experts((x, s), offsets)
    assert calls.made == 0


def test_shapes_follow_the_handles(monkeypatch):
    """A handle's shape is known from its making to its end, and a refused end keeps it."""
    status = [0]

    class Lib:
        def usp_encode_q(self, *args):
            args[-1]._obj.value = 77
            return 0

        def usp_group_create(self, handles, count, out):
            out._obj.value = 99
            return 0

        def usp_free(self, handle):
            return status[0]

        usp_group_free = usp_free

        def usp_last_error(self):
            return b"refused"

    lib = Lib()
    monkeypatch.setattr(usp, "_lib", lib)
    monkeypatch.setattr(usp, "load_library", lambda: lib)
    monkeypatch.setattr(usp, "_shapes", {})
    one = np.ones((3, 7), np.int8)
    h = usp.usp_encode_q(one, one.astype(np.uint8), np.ones(3, np.float32))
    g = usp.usp_group_create([h])
    assert usp._shapes == {77: (3, 7), 99: (3, 7)} and (h, g) == (77, 99)
    status[0] = 1
    with pytest.raises(usp.UspError):
        usp.usp_free(h)
    assert usp._shapes[h] == (3, 7)
    status[0] = 0
    usp.usp_group_free(g)
    usp.usp_free(h)
    assert usp._shapes == {}


@pytest.mark.gpu
def test_on_the_gpu():
    """Too narrow and too wide operands with strides that would do, and the output beside them left alone."""
    rng = np.random.default_rng(3)
    W, mask = rng.integers(-9, 9, (M, K)).astype(np.int8), (rng.random((M, K)) < 0.5).astype(np.uint8)
    A = usp.SparseMatrixQ(W, mask, np.full(M, 0.01, np.float32))
    G = usp.ExpertGroup([A])
    s = torch.ones(N, device="cuda")
    offsets = torch.tensor([0, N], dtype=torch.int32, device="cuda")
    for x_width, y_width in ((100, M), (K + 1, M), (K, M - 8), (K, M + 1)):
        y = torch.full((N, 128), 3.0, dtype=torch.float16, device="cuda")
        x = torch.zeros((N, 128), dtype=torch.int8, device="cuda")[:, :x_width]
        with pytest.raises(usp.UspError):
            usp.usp_spmm_q(A.handle, x, s, y[:, :y_width], A.make_workspace(N))
        with pytest.raises(usp.UspError):
            usp.usp_spmm_grouped(G.handle, x, offsets, y[:, :y_width], G.make_workspace(N), x_scale=s)
        torch.cuda.synchronize()
        assert (y == 3).all()
    mod = linear.SparseLinearQ(torch.from_numpy(W), mask, torch.full((M,), 0.01))
    _, tokens = linear.BlockNorm(100)(torch.zeros(N, 100, dtype=torch.float16, device="cuda"), quantize=True)
    assert tokens[0].stride(0) >= K
    with pytest.raises(ValueError):
        mod(tokens)
