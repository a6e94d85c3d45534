"""The modules inside tracers, dispatch modes and function transforms: what looks at a program's operators finds the
modules' own. On the CPU, the binding replaced by plain writes."""
from types import SimpleNamespace

import pytest
import torch
from torch._subclasses.fake_tensor import FakeTensorMode
from torch.fx.experimental.proxy_tensor import make_fx
from torch.overrides import TorchFunctionMode
from torch.utils._python_dispatch import TorchDispatchMode

from paper_2607_08786_amd import linear, usp

K, M, N = 32, 24, 6


@pytest.fixture(autouse=True)
def plain_writes(monkeypatch, request):
    """y = 2 x (first columns) of the products, r = residual + y and h = 3 r of the norm, written into the memory behind the
    tensors, as the library writes: no tracer sees it."""
    if request.node.get_closest_marker("gpu"):
        return

    def at(t):
        return t.detach().numpy()

    def spmm_q(handle, x, x_scale, y, *args, **kw):
        at(y)[:] = 2 * at(x)[:, :M]

    def grouped(group, x, offsets, y, *args, **kw):
        at(y)[:] = 2 * at(x)[:, :M]

    def norm(residual, y, *args, residual_out, out, **kw):
        at(residual_out)[:] = at(residual) + (0 if y is None else at(y))
        at(out)[:] = 3 * at(residual_out)

    monkeypatch.setattr(usp, "usp_spmm_q", spmm_q)
    monkeypatch.setattr(usp, "usp_spmm_grouped", grouped)
    monkeypatch.setattr(usp, "usp_norm", norm)


def bare(cls, **also):
    m = cls.__new__(cls)
    torch.nn.Module.__init__(m)
    m._set_up((M, K), None, "none", 0)
    m.matrix = SimpleNamespace(handle=1, device=0, workspace_size=lambda n: 0, **also)
    return m


OFFSETS = torch.tensor([0, N], dtype=torch.int32)


def layer():
    return bare(linear.SparseLinearQ)


def experts():
    m = bare(linear.SparseExperts, experts=[None])
    m.eight_bit = False
    return lambda x: m(x, OFFSETS)


def norm():
    m = linear.BlockNorm(K, device="cpu")
    return lambda x: m(x, x)[1]


MODULES = {"sparse_linear_q": (layer, lambda x: 2 * x[:, :M]), "sparse_experts": (experts, lambda x: 2 * x[:, :M]),
           "block_norm": (norm, lambda x: 3 * (x + x))}


def draw(seed=0):
    return torch.randint(-9, 9, (N, K), generator=torch.Generator().manual_seed(seed)).half()


@pytest.mark.parametrize("name", MODULES)
def test_jit_trace(name):
    make, want = MODULES[name]
    call = make()
    traced = torch.jit.trace(lambda x: call(x), draw())
    assert f"usp::{name}" in str(traced.inlined_graph)
    for seed in (1, 2):
        assert torch.equal(traced(draw(seed)), want(draw(seed)))


@pytest.mark.parametrize("name", MODULES)
@pytest.mark.parametrize("mode", ["real", "fake"])
def test_make_fx(name, mode):
    make, want = MODULES[name]
    traced = make_fx(make(), tracing_mode=mode, _allow_non_fake_inputs=True)(draw())
    assert any(f"usp.{name}" in str(n.target) for n in traced.graph.nodes)
    assert torch.equal(traced(draw(1)), want(draw(1)))


@pytest.mark.parametrize("name", MODULES)
def test_modes_see_the_call(name):
    seen = []

    class Dispatch(TorchDispatchMode):
        def __torch_dispatch__(self, func, types, args=(), kwargs=None):
            seen.append(str(func))
            return func(*args, **(kwargs or {}))

    class Function(TorchFunctionMode):
        def __torch_function__(self, func, types, args=(), kwargs=None):
            seen.append(str(func))
            return func(*args, **(kwargs or {}))

    make, want = MODULES[name]
    for mode in (Dispatch, Function):
        seen.clear()
        with mode():
            y = make()(draw())
        assert any(f"usp.{name}" in s for s in seen), seen
        assert torch.equal(y, want(draw()))


@pytest.mark.parametrize("name", MODULES)
def test_fake_tensors(name):
    make, want = MODULES[name]
    with FakeTensorMode(allow_non_fake_inputs=True) as mode:
        x = mode.from_tensor(draw())
        inside = make()(x)
    outside = make()(x)  # a fake tensor by itself
    for y in (inside, outside):
        assert type(y) is type(x) and y.shape == want(draw()).shape and y.dtype == torch.float16


def test_tensor_subclass():
    seen = []

    class Seen(torch.Tensor):
        @classmethod
        def __torch_function__(cls, func, types, args=(), kwargs=None):
            seen.append(str(func))
            return super().__torch_function__(func, types, args, kwargs or {})

    norm()(draw().as_subclass(Seen))
    assert any("usp.block_norm" in s for s in seen)


@pytest.mark.parametrize("name", MODULES)
def test_negated_views(name):
    """A tensor whose memory holds the opposite values until something resolves it."""
    make, want = MODULES[name]
    x = torch._neg_view(draw())
    assert x.is_neg()
    assert torch.equal(make()(x), want(-draw()))


def test_vmap():
    x = torch.stack([draw(i) for i in range(3)])
    assert torch.equal(torch.func.vmap(norm())(x), 3 * (x + x))


@pytest.mark.parametrize("name", MODULES)
@pytest.mark.parametrize("context", [torch.no_grad, torch.inference_mode, torch.enable_grad])
def test_plain_calls_spare_the_dispatcher(name, context, monkeypatch):
    make, want = MODULES[name]

    def op(*args):
        raise AssertionError("the operator was called")

    monkeypatch.setattr(linear, name, op)
    with context():
        assert torch.equal(make()(draw()), want(draw()))


@pytest.mark.gpu
def test_traced_on_the_gpu():
    """A block of the three modules, traced: the bits of the eager calls on other inputs."""
    g = torch.Generator().manual_seed(5)
    codes, mask = torch.randint(-9, 9, (4, 64, 64), generator=g).to(torch.int8), torch.rand(4, 64, 64, generator=g) < 0.5
    scale = torch.full((64,), 0.01)
    up = linear.SparseLinearQ(codes[0], mask[0], scale, activation="silu")
    both = linear.SparseExperts(list(codes[1:3]), list(mask[1:3]), [scale, scale])
    between = linear.BlockNorm(64, post="rms")
    offsets = torch.tensor([0, 3, 7], dtype=torch.int32, device="cuda")

    def block(x):
        r, tokens = between(x, up(x), quantize=True)
        return r, both(tokens, offsets)

    xs = [torch.randn(7, 64, generator=g).half().cuda() for _ in range(3)]
    want = [block(x) for x in xs]
    traced = torch.jit.trace(block, xs[0])
    for name in MODULES:
        assert f"usp::{name}" in str(traced.graph)
    for x, w in zip(xs, want):
        assert all(torch.equal(a, b) for a, b in zip(traced(x), w))
