"""usp_attention where the arithmetic of its softmax could go wrong: long chains of blocks, large scores, weights far below
the largest, extreme scales (GPU). Each case has an answer in closed form or by sums in 64 bits, and a tolerance of its own."""
import pytest
import torch

import attention64
from paper_2607_08786_amd import usp

pytestmark = pytest.mark.gpu

PAGE = 4096


def draw(seed, *shape, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(*shape, generator=g) * scale).half()


def int32(values):
    return torch.as_tensor(values, dtype=torch.int32).cuda()


def one_sequence(K, V, values, page=64):
    """A cache that holds one sequence's K and V [L, kv, D], and a function that makes the rows of its last n tokens."""
    L, kv, D = K.shape
    pages = -(-L // page)
    cache = usp.KVCache(pages, kv, D, page, dtype=torch.int8 if values == "q" else torch.float16)
    table, length = int32([list(range(pages))]), int32([L])
    cache.append(usp.CacheRows(table, length, int32([0, L])), K.cuda(), V.cuda())
    return cache, lambda n: usp.CacheRows(table, length, None if n == 1 else int32([0, n]))


def uncut(cache, tables):
    """Rows of one token for each of 4097 sequences, of which the first have the pages of `tables` and the others nothing: too
    many sequences for tiles to be cut, so that one workgroup takes each of the first ones whole."""
    table = torch.zeros(4097, len(tables[0]), dtype=torch.int32)
    lengths = torch.zeros(4097, dtype=torch.int32)
    table[:len(tables)], lengths[:len(tables)] = torch.tensor(tables, dtype=torch.int32), PAGE * len(tables[0])
    rows = usp.CacheRows(table.cuda(), lengths.cuda())
    plan = cache.plan(rows, 4097, cache.kv_heads)
    assert plan.startswith("rows") and "pieces" not in plan
    return rows


@pytest.mark.parametrize("values", ["f16", "q"])
@pytest.mark.parametrize("score", [300.0, 1e4, 1e8])
def test_long_chains_of_equal_scores(score, values):
    """1024 blocks a wavefront, values 1 in the first half of the keys and 0 in the second: 1 / 2 whatever the score. Weights
    are equal, so their roundings cancel. What is left: the result's rounding, 2^-12; sums of 1024 terms of one size each,
    1024 2^-24 = 2^-14 of 1 / 2 for the numerator and the same for the sum of weights."""
    D = 64
    cache = usp.KVCache(2, 1, D, PAGE, dtype=torch.int8 if values == "q" else torch.float16)
    K, V = torch.zeros(2 * PAGE, 1, D).half(), torch.zeros(2 * PAGE, 1, D).half()
    K[..., :61], V[:PAGE] = 1, 1
    cache.append(usp.CacheRows(int32([[0, 1]]), int32([2 * PAGE]), int32([0, 2 * PAGE])), K.cuda(), V.cuda())
    rows = uncut(cache, [[0] * 16 + [1] * 16])
    q = torch.ones(4097, 1, D, dtype=torch.float16, device="cuda")
    got = cache.attention(rows, q, scale=score / 61)
    assert (got[1:] == 0).all()
    assert ((got[0].double() - 0.5).abs() <= 2.0 ** -12 + 2.0 ** -14).all(), got[0, 0, :4]


def test_long_chains_in_units_of_a_scale():
    """32768 blocks a wavefront of an 8-bit cache, values v in the first half of the keys and 0 in the second: v / 2. All
    weights are 1, so the sums are of whole numbers below 2^24 times a power of two, and exact. What is left: the result's
    rounding, 2^-11 of it, the value's scale and the result's way back from its units, a few 2^-24 of it."""
    D, L = 32, 1024
    v = torch.linspace(1.0, 2.0, 17)[:16].half()
    cache = usp.KVCache(17, 1, D, PAGE, dtype=torch.int8)
    K, V = torch.zeros(17 * PAGE, 1, D).half(), torch.zeros(17, PAGE, 1, D).half()
    V[:16] = v[:, None, None, None]
    everything = usp.CacheRows(int32([list(range(17))]), int32([17 * PAGE]), int32([0, 17 * PAGE]))
    cache.append(everything, K.cuda(), V.view(17 * PAGE, 1, D).cuda())
    rows = uncut(cache, [[i] * (L // 2) + [16] * (L // 2) for i in range(16)])
    got = cache.attention(rows, torch.zeros(4097, 1, D, dtype=torch.float16, device="cuda"))
    want = attention64.held(V[:16, 0], True).view(16, 1, D) / 2
    assert ((got[:16].cpu().double() - want).abs() <= (2.0 ** -11 + 2.0 ** -20) * want).all(), (got[:16, 0, 0].cpu() / want[:, 0, 0] - 1)


@pytest.mark.parametrize("values", ["f16", "q"])
@pytest.mark.parametrize("n", [1, 40])
@pytest.mark.parametrize("L", [90, 4000])
@pytest.mark.parametrize("size,step", [(4096, 4), (57344, 32)])
def test_large_scores(size, step, L, n, values):
    """Scores of some 1e8 and 1e10 that lie far apart between seven kinds of keys and are one number within each: the mean
    of the values of the largest kind that a row sees. Products are multiples of size * step and their sums below 2^24 of
    them, so scores are exact up to their scale. (Values have one largest magnitude, so one scale in 8 bits.)
    Errors: the result's rounding; sums of up to L terms in fp32, twice over for the matrix unit; in 8 bits a weight's factor,
    the same for all here, 2^-14 of each."""
    D, kv, heads = 128, 2, 4
    kind = (torch.arange(L) * 3 + 1) % 7
    K = (size + step * kind.float())[:, None, None].expand(L, kv, D).half()
    V = draw(1, L, kv, D).clamp(-3, 3)
    V[..., 0] = 4
    q = torch.full((n, heads, D), float(size)).half()
    q[:, 1::2] *= -1  # half of the heads: the smallest kind, its score far below zero
    cache, rows = one_sequence(K, V, values)
    got = cache.attention(rows(n), q.cuda()).cpu().double()
    held = attention64.held(V, values == "q")
    for i in range(n):
        seen = kind[:L - n + i + 1]
        for h in range(heads):
            at = (seen == (seen.min() if h % 2 else seen.max())).nonzero()[:, 0]
            v = held[at, h // 2]
            want, A = v.mean(0), v.abs().mean(0)
            tol = 2.0 ** -25 + 2.0 ** -11 * want.abs() + (4 * (L + 40) * 2.0 ** -24 + (2.0 ** -13 if values == "q" else 0)) * A
            assert ((got[i, h] - want).abs() <= tol).all(), (i, h, got[i, h, :4], want[:4])


@pytest.mark.parametrize("values", ["f16", "q"])
@pytest.mark.parametrize("n", [1, 40])
def test_scores_beyond_fp32(n, values):
    """A score beyond fp32's range counts as an infinity: above, the row is NaN; below, the key has no weight; all below: zeros.
    Errors as above."""
    D, L = 64, 500
    sign = torch.where(torch.arange(L) % 5 == 0, 0.0, -1.0)  # scores of 0 and of -2^130
    K = (sign * 32)[:, None, None].expand(L, 1, D).half()
    V = draw(2, L, 1, D)
    V[..., 0] = 4
    V = V.clamp(-4, 4)
    cache, rows = one_sequence(K, V, values)
    q = torch.full((n, 3, D), 32.0).half()
    q[:, 1] *= -1
    scale = 2.0 ** 114
    first = torch.arange(L - n, L).int()
    got = cache.attention(rows(n), q.cuda(), scale=scale).cpu().double()
    assert got[:, 1].isnan().all()
    held = attention64.held(V, values == "q")[:, 0]
    for i in range(n):
        v = held[:L - n + i + 1][::5]
        want, A = v.mean(0), v.abs().mean(0)
        tol = 2.0 ** -25 + 2.0 ** -11 * want.abs() + (4 * (L + 40) * 2.0 ** -24 + (2.0 ** -13 if values == "q" else 0)) * A
        for h in (0, 2):
            assert ((got[i, h] - want).abs() <= tol).all()
    alone = cache.attention(rows(n), q.cuda(), scale=scale, first=first.cuda()).cpu()  # each row its own key alone
    for i in range(n):
        if (L - n + i) % 5:
            assert (alone[i, 0] == 0).all()
        else:
            want = held[L - n + i]
            assert ((alone[i, 0].double() - want).abs() <= 2.0 ** -25 + (2.0 ** -11 + 2.0 ** -13) * want.abs()).all()


@pytest.mark.parametrize("spread", [0.0, 1.0])
@pytest.mark.parametrize("values", ["f16", "q"])
@pytest.mark.parametrize("n", [1, 64])
@pytest.mark.parametrize("L", [16384, 131072])
def test_one_key_far_above_the_others(L, n, values, spread):
    """A first token that draws attention, its score 17.4 above the others', its value 0: the result is what the others add
    up to. Errors relative to it: its rounding 2^-11; each weight's rounding, 2^-11 in fp16 and 2^-14 more in 8 bits, in the
    numerator (in the sum of weights the others are less than 2^-4), and 2^-25 of the few that are subnormal, in units in which
    the others are 2^-10 and more, 2^-15; an exponent of up to 64 off by 8 roundings, 2^-15; the
    numerator's sum of two terms a block of 32 keys and the sum of weights' of one, (L / 16 + L / 32) 2^-24, twice over."""
    D = 64
    g = torch.Generator().manual_seed(L + n)
    K = torch.zeros(L, 1, D).half()
    K[1:, 0, 0] = (torch.randn(L - 1, generator=g) * spread).half()
    K[0, 0, 0] = 17.40625
    V = (torch.rand(L, 1, D, generator=g) + 0.5).half()
    V[0] = 0
    cache, rows = one_sequence(K, V, values, page=PAGE)
    q = torch.zeros(n, 1, D).half()
    q[..., 0] = 1
    assert cache.plan(rows(n), n, 1).startswith("rows" if n == 1 else "tiles")
    got = cache.attention(rows(n), q.cuda(), scale=1.0)[:, 0].cpu().double()
    s = attention64.held(K, values == "q")[:, 0, 0]
    w = torch.exp(s - s[0])
    v = attention64.held(V, values == "q")[:, 0]
    total, above = torch.cumsum(w, 0)[L - n:], torch.cumsum(w[:, None] * v, 0)[L - n:]
    want = above / total[:, None]
    assert total.max() < 1 + 2.0 ** -4
    off = (got / want - 1).abs().max()
    assert off <= 2.0 ** -11 + 2.0 ** -11 + 2.0 ** -14 + 2.0 ** -14 + 2 * (L / 16 + L / 32) * 2.0 ** -24, off


@pytest.mark.parametrize("modified", [False, True])
@pytest.mark.parametrize("n", [1, 40])
def test_scale_times_the_keys_scale(n, modified):
    """8 bits: a scale of 2^126 and keys of up to 60000. A score of 0 is 0, although the two scales' product is beyond fp32."""
    D, L = 64, 70
    K = torch.full((L, 1, D), 60000.0).half()
    V = draw(3, L, 1, D)
    cache, rows = one_sequence(K, V, "q")
    slopes = torch.zeros(2, device="cuda") if modified else None
    got = cache.attention(rows(n), torch.zeros(n, 2, D, dtype=torch.float16, device="cuda"), scale=2.0 ** 126, slopes=slopes)
    zero = cache.attention(rows(n), torch.zeros(n, 2, D, dtype=torch.float16, device="cuda"), scale=1.0, slopes=slopes)
    assert torch.isfinite(got).all() and torch.equal(got, zero)


@pytest.mark.parametrize("values", ["f16", "q"])
@pytest.mark.parametrize("L", [40, 130, 700])
def test_weights_of_few_rows(L, values):
    """Weights are not rounded to fp16 where a row is alone. q and K are whole numbers of few bits, so scores are exact up to
    their scale (8-bit keys: four values whose largest is 2, so codes and scales of one key are too), and V's signs leave a
    result far below its terms A = sum p |V|. Errors: the result's rounding, 2^-11 of it; weights, 2^-20 of A and it; scores
    off by 16 roundings, twice over; sums of L / 16 terms and a join, twice over."""
    D, heads, kv = 64, 8, 2
    g = torch.Generator().manual_seed(L)
    K = torch.randint(-2, 3, (L, kv, D), generator=g).half()
    K[..., 0] = 2
    q = torch.randint(-2, 3, (1, heads, D), generator=g).half()
    V = ((torch.rand(L, kv, D, generator=g) + 0.5) * (torch.randint(0, 2, (L, kv, D), generator=g) * 2 - 1)).half()
    cache, rows = one_sequence(K, V, values)
    got = cache.attention(rows(1), q.cuda(), scale=0.11).cpu().double()[0]
    k, v = attention64.held(K, values == "q"), attention64.held(V, values == "q")
    for h in range(heads):
        z = k[:, h // 4] @ q[0, h].double() * float(torch.tensor(0.11))
        w = torch.softmax(z, 0)
        out, A = w @ v[:, h // 4], w @ v[:, h // 4].abs()
        e = 16 * 2.0 ** -24 * (z.abs().max() + (D * 2.0 * 2.0 * 0.11 if values == "q" else 0))
        tol = 2.0 ** -25 + 2.0 ** -11 * out.abs() + 2.0 ** -20 * (A + out.abs()) + (2 * e + 2 * (L / 16 + 40) * 2.0 ** -24) * A
        assert ((got[h] - out).abs() <= tol).all(), ((got[h] - out).abs() / tol).max()


@pytest.mark.parametrize("n", [1, 40])
def test_infinite_values(n):
    """An infinity that a row sees is one, whatever its weight down to 2^-36 of the largest, and equal weights too; two of
    opposite signs are NaN."""
    D, L, heads = 64, 200, 40
    K = torch.zeros(L, 1, D).half()
    K[7, 0, 0] = -1  # head h: a score of -h / 40 of 24.95, 2^-36
    V = draw(5, L, 1, D)
    V[7, 0, 3], V[7, 0, 5], V[7, 0, 8] = float("inf"), float("-inf"), float("inf")
    V[9, 0, 8] = float("-inf")
    q = torch.zeros(n, heads, D).half()
    q[..., 0] = torch.arange(heads) / 40 * 24.95
    cache, rows = one_sequence(K, V, "f16")
    assert cache.plan(rows(n), n, heads).startswith("rows" if n == 1 else "tiles")
    got = cache.attention(rows(n), q.cuda(), scale=1.0).cpu()
    assert (got[..., 3] == float("inf")).all() and (got[..., 5] == -float("inf")).all() and got[..., 8].isnan().all()
    others = [d for d in range(D) if d not in (3, 5, 8)]
    assert torch.isfinite(got[..., others]).all()
    hidden = cache.attention(rows(n), q.cuda(), scale=1.0, first=int32([8] * n)).cpu()
    assert torch.isfinite(hidden[..., :8]).all() and (hidden[..., 8] == -float("inf")).all()


@pytest.mark.parametrize("values", ["f16", "q"])
@pytest.mark.parametrize("n", [1, 40])
@pytest.mark.parametrize("size,step", [(4096, 4), (57344, 32)])
def test_large_biased_scores(size, step, n, values):
    """Scores of 1e8 and 1e10 that pass the biases, here of nothing, and under a cap far above them: as without, to roundings."""
    D, L = 128, 900
    kind = (torch.arange(L) * 3 + 1) % 7
    K = (size + step * kind.float())[:, None, None].expand(L, 1, D).half()
    V = draw(6, L, 1, D).clamp(-3, 3)
    V[..., 0] = 4
    q = torch.full((n, 2, D), float(size)).half()
    q[:, 1] *= -1
    cache, rows = one_sequence(K, V, values)
    want = cache.attention(rows(n), q.cuda())
    for kw in (dict(slopes=torch.zeros(2, device="cuda")), dict(cap=1e30)):
        got = cache.attention(rows(n), q.cuda(), **kw)
        assert ((got - want).abs() <= 2.0 ** -10 * want.abs() + 2.0 ** -12).all()


@pytest.mark.parametrize("values", ["f16", "q"])
@pytest.mark.parametrize("biased", [False, True])
def test_neighbours_of_rows_that_are_not_finite(biased, values):
    """Rows with a NaN or an infinity in q are NaN, and all others keep their bits."""
    D, L, n, heads = 128, 700, 300, 4
    cache, rows = one_sequence(draw(8, L, 2, D), draw(9, L, 2, D), values)
    kw = dict(slopes=torch.full((heads,), 0.01, device="cuda")) if biased else {}
    q = draw(10, n, heads, D, scale=2.0)
    clean = cache.attention(rows(n), q.cuda(), **kw)
    assert torch.isfinite(clean).all()
    bad = torch.zeros(n, heads, dtype=torch.bool)
    for i, value in enumerate((float("nan"), float("inf"), -float("inf"))):
        for row in range(5 + i, n, 41):
            q[row, row % heads, 3 * i] = value
            bad[row, row % heads] = True
    got = cache.attention(rows(n), q.cuda(), **kw)
    assert got[bad.cuda()].isnan().all() and torch.equal(got[~bad.cuda()], clean[~bad.cuda()])
