"""usp_attention where one call's tiles are cut into several pieces and joined, at every width and in both caches, and steps
that mix single tokens with prompts, against the plain form in 64 bits (GPU)."""
import re

import pytest
import torch

import attention64
from test_paged_attention import Setting, draw, on_gpu, operands

pytestmark = pytest.mark.gpu


def pieces_of(plan):
    found = re.search(r"pieces=(\d+)", plan)
    return int(found.group(1)) if found else 1


# heads, kv_heads, head_dim, page, lengths, rows of each: tiles of 6 blocks a piece at least, so more than two pieces each
TILES = [(2, 1, 32, 32, [900], [40]), (4, 2, 64, 64, [700, 30, 1100], [50, 0, 33]), (3, 1, 88, 32, [650, 1000], [64, 200]),
         (8, 1, 128, 128, [1301], [70]), (2, 2, 168, 64, [777], [300]), (1, 1, 256, 32, [640], [129])]


@pytest.mark.parametrize("values", ["f16", "q"])
@pytest.mark.parametrize("mods", ["plain", "bias", "window", "all"])
@pytest.mark.parametrize("heads,kv,D,page,lengths,counts", TILES)
def test_tiles_in_pieces(heads, kv, D, page, lengths, counts, mods, values):
    s = Setting(lengths, kv, D, page, values, seed=D + heads).fill()
    T = sum(counts)
    rows, kw = s.rows(counts), operands(mods, heads)
    plan = s.cache.plan(rows, T, heads)
    assert plan.startswith("tiles") and pieces_of(plan) > 2
    q = draw(11, T, heads, D, scale=2.0)
    attention64.close(s.cache.attention(rows, q.cuda(), **on_gpu(kw)), *s.want(q, counts, **kw))


@pytest.mark.parametrize("values", ["f16", "q"])
def test_tiles_in_pieces_with_masks(values):
    """Documents, prefixes and rows that see nothing: some pieces of a tile see nothing, some columns none of any piece."""
    heads, kv, D, lengths, counts = 4, 1, 64, [1500, 800], [300, 120]
    s = Setting(lengths, kv, D, 32, values, seed=3)
    for V, L in zip(s.V, lengths):
        V[L // 2, :, 3] = float("inf")
    s.fill()
    T = sum(counts)
    rows, q = s.rows(counts), draw(12, T, heads, D)
    assert pieces_of(s.cache.plan(rows, T, heads)) > 2
    position = torch.cat([torch.arange(L - n, L) for L, n in zip(lengths, counts)])
    g = torch.Generator().manual_seed(3)
    first, last = torch.randint(-3, 1700, (T,), generator=g).int(), torch.randint(-5, 1700, (T,), generator=g).int()
    for kw in (dict(first=first, last=last), dict(first=(position // 400 * 400).int()), dict(last=torch.maximum(position + 1, torch.tensor(1400)).int()),
               dict(first=position.int() + 1)):
        want, tol = s.want(q, counts, **kw)
        attention64.close(s.cache.attention(rows, q.cuda(), **on_gpu(kw)), want, torch.where(tol.isnan(), torch.zeros_like(tol), tol))


@pytest.mark.parametrize("values", ["f16", "q"])
@pytest.mark.parametrize("mods", ["plain", "all"])
@pytest.mark.parametrize("D", [64, 200])
@pytest.mark.parametrize("counts", [[4, 1, 3], [2, 0, 2]])
def test_few_rows_in_pieces(counts, D, mods, values):
    """Up to four rows a sequence of heads that share one, in pieces of the rows kernel."""
    heads, kv, lengths = 16, 2, [3000, 257, 1400]
    s = Setting(lengths, kv, D, 64, values, seed=D).fill()
    T = sum(counts)
    rows, kw = s.rows(counts), operands(mods, heads)
    plan = s.cache.plan(rows, T, heads)
    assert plan.startswith("rows") and pieces_of(plan) > 2
    q = draw(13, T, heads, D, scale=2.0)
    attention64.close(s.cache.attention(rows, q.cuda(), **on_gpu(kw)), *s.want(q, counts, **kw))


@pytest.mark.parametrize("values", ["f16", "q"])
def test_prompts_beside_single_tokens(values):
    """One call of a step that mixes them: every row as if its sequence were alone."""
    heads, kv, D, lengths, counts = 8, 2, 128, [150, 4000, 61, 900], [150, 1, 1, 20]
    s = Setting(lengths, kv, D, 64, values, seed=6).fill()
    T = sum(counts)
    q = draw(14, T, heads, D, scale=2.0)
    rows = s.rows(counts)
    assert s.cache.plan(rows, T, heads).startswith("tiles")
    attention64.close(s.cache.attention(rows, q.cuda()), *s.want(q, counts))


def test_empty_workspace():
    """An empty tensor where a step needs no workspace, as compiled programs have it."""
    s = Setting([200, 60], 2, 64, 64, seed=7).fill()
    q, rows = draw(15, 2, 8, 64).cuda(), s.rows()
    assert s.cache.workspace_size(rows, 2, 8) == 0
    none = torch.empty(0, dtype=torch.uint8, device="cuda")
    assert torch.equal(s.cache.attention(rows, q, workspace=none), s.cache.attention(rows, q))
