"""What the paged cache does without a GPU: refusals of the C ABI, workspace sizes and plans, the bookkeeping of pages, the
module in tracers."""
import ctypes
import random
from types import SimpleNamespace

import pytest
import torch
from torch._subclasses.fake_tensor import FakeTensorMode
from torch.fx.experimental.proxy_tensor import make_fx

from paper_2607_08786_amd import attention, usp


def described(**change):
    keep = ctypes.create_string_buffer(256)
    base = ctypes.addressof(keep) + 63 & ~63
    c = usp.usp_cache(base, 2, 8, 4, 64, 32, 2, 0)
    r = usp.usp_cache_rows(base, 300, 300, base, base, 2, 5)
    a = usp.usp_attention_args(base, base, None, None, None, 8 * 64, 64, 8 * 64, 64, 1, 0, 8, 0.1, 0.0)
    for name, v in change.items():
        where, field = name.split("_", 1)
        setattr(dict(c=c, r=r, a=a)[where], field, v if v is None or abs(v) > 3 or field not in ("data", "table", "lengths", "offsets", "q", "out", "first", "slopes") else base + v)
    return keep, base, c, r, a


@pytest.mark.parametrize("change,text", [
    (dict(c_data=None), "16-byte"), (dict(c_data=2), "16-byte"), (dict(c_layers=0), "layers"), (dict(c_pages=0), "layers"),
    (dict(c_pages=2 ** 31), "layers"), (dict(c_kv_heads=0), "kv_heads"), (dict(c_kv_heads=4097), "kv_heads"), (dict(c_head_dim=12), "head_dim"),
    (dict(c_head_dim=264), "head_dim"), (dict(c_head_dim=0), "head_dim"), (dict(c_page_tokens=48), "page_tokens"),
    (dict(c_page_tokens=8192), "page_tokens"), (dict(c_value_bytes=4), "value_bytes"), (dict(r_table=None), "null table"),
    (dict(r_lengths=None), "null table"), (dict(r_lengths=2), "4-byte"), (dict(r_table_pages=0), "table_pages"),
    (dict(r_table_pages=2 ** 26), "table_pages"), (dict(r_ld_table=2), "ld_table"), (dict(r_sequences=0), "sequences"),
    (dict(r_sequences=2 ** 20 + 1), "sequences"), (dict(r_rows=-1), "rows must"), (dict(r_rows=2 ** 20 + 1), "rows must"),
    (dict(r_offsets=None), "one row for each"), (dict(a_heads=6), "multiple"), (dict(a_heads=0), "multiple"), (dict(a_heads=65540), "multiple"),
    (dict(a_layer=2), "layer"), (dict(a_layer=-1), "layer"), (dict(a_scale=float("nan")), "scale"), (dict(a_scale=2.0 ** 127.5), "scale"), (dict(a_cap=float("inf")), "cap"),
    (dict(a_cap=-1.0), "cap"), (dict(a_cap=1e-45), "scale / cap"), (dict(a_window=-1), "window"), (dict(a_q=None), "null q"),
    (dict(a_out=None), "null q"), (dict(a_q=1), "2-byte"), (dict(a_first=2), "4-byte"), (dict(a_slopes=2), "4-byte"),
    (dict(a_ld_q=-1), "strides"), (dict(a_ld_out=63), "apart"), (dict(a_head_out=32), "apart"), (dict(a_ld_out=7 * 64), "apart"),
    (dict(c_device=99), "no such device"),
])
def test_attention_refusals(change, text):
    keep, base, c, r, a = described(**change)
    lib = usp.load_library()
    status = lib.usp_attention(c, r, a, base, 1 << 40, None)
    assert status == 1 and text in usp.usp_last_error(), usp.usp_last_error()
    if not any(k.startswith("a_") for k in change):
        assert lib.usp_cache_append(c, r, 0, base, 256, 64, base, 256, 64, None) == 1 and text in usp.usp_last_error()
        assert lib.usp_cache_read(c, r, 0, base, 256, 64, base, 256, 64, None) == 1 and text in usp.usp_last_error()


def test_more_refusals():
    keep, base, c, r, a = described()
    lib = usp.load_library()
    err = lambda status, text: (status == 1 and text in usp.usp_last_error()) or pytest.fail(usp.usp_last_error())  # noqa: E731
    err(lib.usp_attention(None, r, a, None, 0, None), "null cache")
    err(lib.usp_attention(c, None, a, None, 0, None), "null rows")
    err(lib.usp_attention(c, r, None, None, 0, None), "null arguments")
    err(lib.usp_attention(c, r, a, None, 1 << 40, None), "workspace too small")
    err(lib.usp_attention(c, r, a, base, 256 << 10, None), "workspace too small")
    err(lib.usp_attention(c, r, a, base + 8, 1 << 40, None), "16-byte aligned")
    err(lib.usp_cache_append(c, r, 2, base, 256, 64, base, 256, 64, None), "layer")
    err(lib.usp_cache_append(c, r, 0, None, 256, 64, base, 256, 64, None), "null K")
    err(lib.usp_cache_append(c, r, 0, base, -1, 64, base, 256, 64, None), "strides")
    err(lib.usp_cache_append(c, r, 0, base + 1, 256, 64, base, 256, 64, None), "2-byte")
    err(lib.usp_cache_read(c, r, 0, base, 255, 64, base, 256, 64, None), "apart")
    err(lib.usp_cache_read(c, r, 0, base, 256, 64, base, 256, 63, None), "apart")
    pages = (ctypes.c_int32 * 3)(0, 1, 2)
    twice = (ctypes.c_int32 * 3)(4, 5, 4)
    after = (ctypes.c_int32 * 3)(1, 2, 3)
    err(lib.usp_cache_copy(c, pages, twice, 3, None), "named twice")
    err(lib.usp_cache_copy(c, pages, after, 3, None), "both a source")
    err(lib.usp_cache_copy(c, pages, (ctypes.c_int32 * 3)(4, 5, 8), 3, None), "destination is no page")
    err(lib.usp_cache_copy(c, (ctypes.c_int32 * 3)(0, -1, 2), (ctypes.c_int32 * 3)(4, 5, 6), 3, None), "source is no page")
    err(lib.usp_cache_copy(c, None, after, 3, None), "null pages")
    err(lib.usp_cache_copy(c, pages, after, 9, None), "n must be")
    assert lib.usp_cache_copy(c, None, None, 0, None) == 0
    buf = ctypes.create_string_buffer(64)
    err(lib.usp_attention_plan(c, r, 7, buf, 64), "multiple")
    assert lib.usp_attention_plan(c, r, 16, buf, 64) == 0 and buf.value.startswith(b"rows")
    assert lib.usp_attention_plan(c, r, 8, buf, 64) == 0 and buf.value.startswith(b"tiles")
    r.rows = 0  # nothing to do, whatever else
    assert lib.usp_attention(c, r, a, None, 0, None) == 0 and lib.usp_attention_workspace_size(c, r, 8) == 0
    assert lib.usp_cache_append(c, r, 0, None, 0, 0, None, 0, 0, None) == 0


def test_too_many_workgroups():
    keep, base, c, r, a = described(c_kv_heads=4096, a_heads=65536, r_rows=2 ** 20, r_sequences=2 ** 20, r_offsets=None, a_ld_out=2 ** 23, a_ld_q=2 ** 23)
    assert usp.load_library().usp_attention(c, r, a, base, 1 << 50, None) == 2 and "too many" in usp.usp_last_error()


@pytest.mark.parametrize("table_pages", [0, -1, 2 ** 26, 2 ** 62])
def test_sizes_of_no_table(table_pages):
    """A table of no or too many pages has no workspace and no plan."""
    keep, base, c, r, a = described(r_table_pages=table_pages, r_ld_table=2 ** 62, r_offsets=None, r_rows=1, r_sequences=1)
    lib, buf = usp.load_library(), ctypes.create_string_buffer(64)
    assert lib.usp_attention_workspace_size(c, r, 8) == 0
    assert lib.usp_attention_plan(c, r, 8, buf, 64) == 1 and "table_pages" in usp.usp_last_error()


def test_launches_beyond_the_grid():
    """A launch has fewer than 2^32 threads: 2^24 workgroups of 256 are refused, not cut."""
    lib = usp.load_library()
    for offsets in (None, "r_offsets"):
        change = dict(c_kv_heads=256, a_heads=256, r_rows=2 ** 20, r_sequences=2 ** 20, a_ld_out=2 ** 15, a_ld_q=2 ** 15)
        keep, base, c, r, a = described(**change, **({"r_offsets": None} if offsets is None else {}))
        assert lib.usp_attention(c, r, a, base, 1 << 50, None) == 2 and "too many" in usp.usp_last_error()
        for call in (lib.usp_cache_append, lib.usp_cache_read):
            assert call(c, r, 0, base, 2 ** 15, 64, base, 2 ** 15, 64, None) == 2 and "too many" in usp.usp_last_error()


def test_sizes():
    lib = usp.load_library()
    for value_bytes, D, block in ((2, 128, 64 * 128 * 2), (1, 128, 64 * 128 + 256), (2, 40, 64 * 64 * 2), (1, 136, 64 * 192 + 256), (2, 256, 64 * 512)):
        assert lib.usp_cache_page_bytes(usp.usp_cache(None, 0, 0, 5, D, 96, value_bytes, 0)) == 5 * 3 * block
    assert lib.usp_cache_page_bytes(None) == 0
    # The largest workspace over numbers of sequences stays small, and none is needed for prompts or many rows.
    keep, base, c, r, a = described(r_offsets=None)
    sizes = []
    for n in (1, 7, 64, 512, 4096, 4097, 2 ** 20):
        r.rows = r.sequences = n
        sizes.append(lib.usp_attention_workspace_size(c, r, 64))
    assert 0 < sizes[0] <= max(sizes) < 64 << 20 and sizes[-1] == 0


# ---- bookkeeping


class Host(attention.PagedCache):
    """A PagedCache without a GPU: tokens are numbers in a list of pages, copies are made there."""

    def __init__(self, pages, page_tokens):
        self.pages, self.page_tokens, self._data = pages, page_tokens, torch.empty(0)
        self._free, self._users = list(range(pages)), [0] * pages
        self._pages, self._lengths, self._next = {}, {}, 0
        self.memory = [[None] * page_tokens for _ in range(pages)]

    def copy(self, src, dst, stream=None):
        assert len(set(dst)) == len(dst) and not set(src) & set(dst)
        for a, b in zip(src, dst):
            self.memory[b] = list(self.memory[a])

    def rows(self, sequences, tokens=None):
        return self._step(sequences, tokens)


def test_bookkeeping_against_lists():
    """Random adds, forks, steps, cuts, frees and compactions: every sequence keeps its tokens, every page its users."""
    rng = random.Random(5)
    cache, held, token, refused = Host(30, 4), {}, 0, 0
    for _ in range(4000):
        ids = list(held)
        what = rng.choice(["add", "fork", "extend", "extend", "extend", "truncate", "free", "compact"])
        if what == "add" and len(ids) < 8:
            held[cache.add()] = []
        elif what == "fork" and ids and len(ids) < 8:
            s = rng.choice(ids)
            held[cache.fork(s)] = list(held[s])
        elif what == "extend" and ids:
            some = rng.sample(ids, rng.randint(1, len(ids)))
            counts = [rng.randint(0, 6) for _ in some]
            before = ({s: list(p) for s, p in cache._pages.items()}, dict(cache._lengths), sorted(cache._free), list(cache._users))
            try:
                tables, lengths, offsets = cache.extend(some, counts)
            except attention.OutOfPages:
                refused += 1
                assert before == (cache._pages, cache._lengths, sorted(cache._free), cache._users)
                continue
            assert offsets == [sum(counts[:i]) for i in range(len(counts) + 1)]
            for s, n, L in zip(some, counts, lengths):
                assert L == len(held[s]) + n == cache.length(s)
                for j in range(L - n, L):
                    cache.memory[cache.pages_of(s)[j // 4]][j % 4] = token
                    held[s].append(token)
                    token += 1
        elif what == "truncate" and ids:
            s = rng.choice(ids)
            n = rng.randint(0, len(held[s]))
            cache.truncate(s, n)
            held[s] = held[s][:n]
        elif what == "free" and ids:
            s = rng.choice(ids)
            cache.free(s)
            del held[s]
        elif what == "compact":
            used = cache.compact()
            assert all(p < used for s in held for p in cache.pages_of(s)) and cache.free_pages == 30 - used
        users = [0] * 30
        for s, want in held.items():
            pages = cache.pages_of(s)
            assert len(pages) == -(-len(want) // 4) and len(set(pages)) == len(pages)
            assert [cache.memory[pages[j // 4]][j % 4] for j in range(len(want))] == want
            for p in pages:
                users[p] += 1
        assert users == cache._users and sorted(cache._free) == [p for p in range(30) if not users[p]]
    assert refused > 10 and token > 1000


def test_bookkeeping_refusals():
    cache = Host(4, 32)
    a = cache.add()
    for bad in (lambda: cache.extend([a, a]), lambda: cache.extend([a], [1, 2]), lambda: cache.extend([a], [-1]), lambda: cache.truncate(a, 1),
                lambda: cache.extend([a], [2 ** 31]), lambda: cache.rows([]), lambda: cache.rows([a], [1])):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(attention.OutOfPages):
        cache.extend([a], [129])
    assert cache.length(a) == 0 and cache.free_pages == 4
    for bad in (lambda: cache.extend([7]), lambda: cache.fork(7), lambda: cache.free(7), lambda: cache.length(7)):
        with pytest.raises(KeyError):
            bad()


# ---- the module in tracers


KV, HEADS, D = 2, 4, 8


@pytest.fixture
def plain_writes(monkeypatch):
    """out = 2 q, and the cache's first bytes count the appends, written behind the tensors as the library writes."""
    def attend(cache, rows, q, out, *args, **kw):
        out.detach().numpy()[:] = 2 * q.detach().numpy()

    def append(cache, rows, k, v, layer=0, stream=None):
        cache.data.detach().numpy()[..., 0] += 1

    monkeypatch.setattr(usp, "usp_attention", attend)
    monkeypatch.setattr(usp, "usp_cache_append", append)
    monkeypatch.setattr(usp, "_gpu", lambda t, name: 0)
    monkeypatch.setattr(usp, "CacheRows", lambda table, lengths, offsets=None: SimpleNamespace(table=table, lengths=lengths, offsets=offsets, device=0))
    return SimpleNamespace(
        cache=SimpleNamespace(kv_heads=KV, head_dim=D, page_tokens=32, dtype=torch.float16, device=0, workspace_size=lambda *a: 0,
                              data=torch.zeros(1, 2, KV * 64 * 32 * 2, dtype=torch.uint8)),
        rows=SimpleNamespace(table=torch.zeros(3, 1, dtype=torch.int32), lengths=torch.ones(3, dtype=torch.int32), offsets=None))


@pytest.mark.parametrize("mode", ["eager", "trace", "make_fx"])
def test_module_in_tracers(plain_writes, mode):
    mod = attention.PagedAttention(HEADS, KV, D)
    call = lambda q, k: mod(q, plain_writes.cache, plain_writes.rows, k, k)  # noqa: E731
    q, k = torch.randn(3, HEADS * D).half(), torch.randn(3, KV, D).half()
    if mode == "trace":
        call = torch.jit.trace(call, (q, k), check_trace=False)
        assert "usp::paged_attention" in str(call.inlined_graph) and "usp::cache_append" in str(call.inlined_graph)
    elif mode == "make_fx":
        call = make_fx(call)(q, k)
        names = [str(n.target) for n in call.graph.nodes]
        assert any("paged_attention" in n for n in names) and any("cache_append" in n for n in names)
    plain_writes.cache.data.zero_()
    for i in range(2):
        x = torch.randn(3, HEADS * D).half()
        assert torch.equal(call(x, k), 2 * x)
        assert (plain_writes.cache.data[..., 0] == i + 1).all()


def test_fake_shapes():
    with FakeTensorMode():
        q = torch.empty(3, HEADS, D, dtype=torch.bfloat16)
        data, table = torch.empty(1, 2, KV * 64 * 32 * 2, dtype=torch.uint8), torch.empty(3, 1, dtype=torch.int32)
        out = torch.ops.usp.paged_attention(q, data, [KV, D, 32, 0], table, table[:, 0], None, None, 0, None, 0.0, None, 0, None, None)
    assert out.shape == (3, HEADS, D) and out.dtype == torch.float16


def test_module_refusals(plain_writes):
    mod = attention.PagedAttention(HEADS, KV, D)
    q, k = torch.zeros(3, HEADS, D).half(), torch.zeros(3, KV, D).half()
    for bad in (lambda: mod(q[:, :2], plain_writes.cache, plain_writes.rows), lambda: mod(q, plain_writes.cache, plain_writes.rows, k),
                lambda: mod(q, plain_writes.cache, plain_writes.rows, k[..., :4], k),
                lambda: attention.PagedAttention(HEADS, KV, 16)(q, plain_writes.cache, plain_writes.rows),
                lambda: attention.PagedAttention(5, 2, 8), lambda: attention.PagedAttention(4, 2, 8, slopes=torch.zeros(3))):
        with pytest.raises(ValueError):
            bad()


def test_workspaces_go_by_device_and_stream(monkeypatch):
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: False)
    current = {0: 5, 1: 5}
    monkeypatch.setattr(usp, "current_stream_handle", lambda device=None: current[device])
    mod = attention.PagedAttention(HEADS, KV, D)
    cache = lambda device: SimpleNamespace(device=device, workspace_size=lambda *a: 16, make_workspace=lambda *a: torch.zeros(16))  # noqa: E731
    first = mod._workspace_of(cache(0), None, 3)
    assert mod._workspace_of(cache(0), None, 3) is first and mod._workspace_of(cache(1), None, 3) is not first
    current[0] = 6
    assert mod._workspace_of(cache(0), None, 3) is not first
