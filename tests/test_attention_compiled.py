"""usp::paged_attention and the modules under torch.compile. On the CPU, the binding replaced by plain writes."""
from types import SimpleNamespace

import pytest
import torch

from paper_2607_08786_amd import attention, linear, usp

KV, HEADS, D, T = 2, 4, 64, 5


@pytest.fixture(autouse=True)
def plain_writes(monkeypatch):
    """out = 2 q, written behind the tensors as the library writes."""
    def attend(cache, rows, q, out, *args, **kw):
        out.detach().numpy()[:] = 2 * q.detach().numpy()

    monkeypatch.setattr(usp, "usp_attention", attend)
    monkeypatch.setattr(usp, "_gpu", lambda t, name: 0)
    monkeypatch.setattr(usp, "current_stream_handle", lambda device=None: 0)
    monkeypatch.setattr(usp, "CacheRows", lambda table, lengths, offsets=None: SimpleNamespace(table=table, lengths=lengths, offsets=offsets, device=0))
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: False)
    torch._dynamo.reset()
    yield
    torch._dynamo.reset()


def operands():
    data = torch.zeros(1, 2, KV * 64 * 64 * 2, dtype=torch.uint8)
    return data, [KV, D, 32, 0], torch.zeros(T, 1, dtype=torch.int32), torch.ones(T, dtype=torch.int32)


def called(q, offsets=None, workspace=None):
    data, geometry, table, lengths = operands()
    return torch.ops.usp.paged_attention(q, data, geometry, table, lengths, offsets, workspace, 0, None, 0.0, None, 0, None, None)


@pytest.mark.parametrize("backend", ["aot_eager", "inductor"])
@pytest.mark.parametrize("offsets", [False, True])
@pytest.mark.parametrize("layout", ["rows first", "heads first", "channels apart"])
def test_compiled_operator(layout, offsets, backend):
    """The result lies as the compiler is told, whatever q's strides are."""
    q = torch.randn(T, HEADS, D).half()
    if layout == "heads first":
        q = q.transpose(0, 1).contiguous().transpose(0, 1)
    elif layout == "channels apart":
        q = torch.randn(T, HEADS, D + 8).half()[..., :D]
    where = torch.arange(T + 1, dtype=torch.int32) if offsets else None
    workspace = torch.zeros(16, dtype=torch.uint8)
    compiled = torch.compile(lambda q: called(q, where, workspace).flatten(1) + 1, backend=backend, fullgraph=True)
    assert torch.equal(compiled(q), 2 * q.flatten(1) + 1)
    got = called(q, where, workspace)
    assert got.is_contiguous() and torch.equal(got, 2 * q)


def attention_module(need):
    data, _, table, lengths = operands()
    cache = SimpleNamespace(kv_heads=KV, head_dim=D, page_tokens=32, dtype=torch.float16, device=0, data=data, workspace_size=lambda *a: need,
                            make_workspace=lambda *a: torch.zeros(need, dtype=torch.uint8))
    rows = SimpleNamespace(table=table, lengths=lengths, offsets=None)
    module = attention.PagedAttention(HEADS, KV, D)
    return lambda q: module(q, cache, rows), torch.randn(T, HEADS * D).half(), lambda q: 2 * q


IN, OUT = 32, 24


def layer(cls, need, **also):
    m = cls.__new__(cls)
    torch.nn.Module.__init__(m)
    m._set_up((OUT, IN), None, "none", 0)
    m.matrix = SimpleNamespace(handle=1, device=0, workspace_size=lambda n: need, make_workspace=lambda n: torch.zeros(need, dtype=torch.uint8), **also)
    return m


def linear_module(need):
    return layer(linear.SparseLinear, need), torch.randn(T, IN).half(), lambda x: 2 * x[:, :OUT]


def linear_q_module(need):
    return layer(linear.SparseLinearQ, need), torch.randn(T, IN).half(), lambda x: 2 * x[:, :OUT]


def experts_module(need):
    m = layer(linear.SparseExperts, need, experts=[None])
    m.eight_bit = False
    offsets = torch.tensor([0, T], dtype=torch.int32)
    return lambda x: m(x, offsets), torch.randn(T, IN).half(), lambda x: 2 * x[:, :OUT]


@pytest.mark.parametrize("backend", ["aot_eager", "inductor"])
@pytest.mark.parametrize("need", [0, 16])
@pytest.mark.parametrize("make", [attention_module, linear_module, linear_q_module, experts_module])
def test_compiled_modules(make, need, backend, monkeypatch):
    """Also where a step needs no workspace."""
    for name, at in (("usp_spmm_ex", 2), ("usp_spmm_q", 3), ("usp_spmm_grouped", 3)):
        def product(*args, at=at, **kw):
            args[at].detach().numpy()[:] = 2 * args[1].detach().numpy()[:, :OUT]
        monkeypatch.setattr(usp, name, product)
    module, x, want = make(need)
    compiled = torch.compile(lambda x: module(x) + 1, backend=backend)
    for factor in (1, 3):
        assert torch.equal(compiled(x * factor), want(x * factor) + 1)
        assert torch.equal(module(x * factor), want(x * factor))
