"""Which kernel usp_attention takes and into how many pieces it cuts, on both sides of each of the planner's rules (CPU)."""
import ctypes
import re

import pytest

from paper_2607_08786_amd import usp


def plan(S, T, kv=1, group=1, D=64, tokens=64 * 64, eight_bit=False, offsets=True):
    """(kernel, pieces aimed at or None, workgroups) of S sequences with T rows and room for so many tokens each."""
    cache = usp.usp_cache(None, 1, 1, kv, D, 32, 1 if eight_bit else 2, 0)
    rows = usp.usp_cache_rows(None, tokens // 32, tokens // 32, None, 1 if offsets else None, S, T)
    buf = ctypes.create_string_buffer(128)
    assert usp.load_library().usp_attention_plan(cache, rows, kv * group, buf, 128) == 0, usp.usp_last_error()
    text = buf.value.decode()
    pieces = re.search(r"pieces=(\d+)", text)
    assert f"W={usp.cache_width(D)}" in text
    return text.split()[0], int(pieces.group(1)) if pieces else None, int(re.search(r"grid=(\d+)", text).group(1))


@pytest.mark.parametrize("S,T,kv,group,want", [
    (1, 1, 1, 1, "rows"), (7, 7, 40, 1, "rows"), (300, 300, 40, 8, "rows"),  # a row a sequence, or fewer
    (9, 5, 8, 1, "rows"), (8, 9, 8, 1, "tiles"), (1, 2, 1, 1, "tiles"),
    (8, 32, 8, 4, "rows"), (8, 33, 8, 4, "tiles"),                            # up to four of them
    (8, 32, 8, 3, "tiles"),                                                   # where four heads share one
    (64, 65, 1, 4, "rows"), (65, 66, 1, 4, "tiles"), (2, 8, 32, 4, "rows"), (2, 8, 33, 4, "tiles")])  # and 64 heads of sequences at most
def test_kernel(S, T, kv, group, want):
    assert plan(S, T, kv, group)[0] == want


@pytest.mark.parametrize("S,kv,group,tokens,pieces", [
    (1, 1, 1, 257, 512), (1, 1, 1, 256, None),              # 8 blocks a piece at least
    (128, 1, 1, 4096, 512), (16, 8, 16, 4096, 512),         # 128 tiles are few
    (129, 1, 1, 4096, 1024), (16, 8, 17, 4096, 1024),
    (129, 1, 1, 1024, None), (129, 1, 1, 1056, 1024),       # of many, 32 blocks
    (4096, 4, 1, 4096, 1024), (4096, 5, 1, 4096, None),     # 16384 tiles at most
    (4096, 1, 1, 4096, 1024), (4097, 1, 1, 4096, None)])    # and 4096 sequences
def test_cuts_of_few_rows(S, kv, group, tokens, pieces):
    tokens = -(-tokens // 32) * 32
    kernel, got, grid = plan(S, S, kv, group, tokens=tokens, offsets=False)
    tiles = S * -(-group // 16)
    assert kernel == "rows" and got == pieces
    assert grid == (tiles + (pieces // kv if pieces else 0)) * kv


@pytest.mark.parametrize("eight_bit,places", [(False, 768), (True, 512)])
@pytest.mark.parametrize("S,T,kv,group", [(1, 40, 1, 1), (1, 512, 8, 8), (3, 700, 2, 3), (1, 4096, 8, 8), (16, 2048, 8, 8), (5, 333, 40, 1)])
def test_cuts_of_many_rows(S, T, kv, group, eight_bit, places):
    """As many pieces of a tile of 128 columns as there are places for, 1 to 16."""
    kernel, pieces, grid = plan(S, T, kv, group, eight_bit=eight_bit)
    tiles = -(-T * group // 128) + S - 1
    assert kernel == "tiles" and pieces == max(1, min(16, places // (tiles * kv))) and grid == tiles * kv * pieces
