"""Attention over a paged key-value cache, and the cache's own operations, as a serving program makes them.

A case is one pass through an operator:

* ``attention``: the rows of a step (one new token of each sequence, or ragged prompts and pieces of prompts) over the
  keys and values that the cache holds for them, the step's own included; fp16 or 8-bit caches; scores may be capped,
  biased by distance, and masked by a window, by documents and by a prefix;
* ``append``: the keys and values of new tokens written into their pages (in 8 bits: quantised first), and read back;
* ``copy``: pages copied to other pages in all layers, as a fork of a sequence or a compaction of the pool asks for.

Heads are those of the decoder blocks in ``workloads`` (40 of 128; 64 of 128 on 8 of keys and values) and generic ones.
Everything is drawn on the GPU from the seed alone. In their plain form pages are [tokens, heads, width] as a program
without a layout of its own holds them.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

_ATTENTION = dict(kind="attention", api="binding", values="f16", rows=1, past=0, page=64, cap=0.0, bias=False, window=0,
                  documents=0, prefix=0)
_13B = dict(kv=40, group=1, width=128)
_70B = dict(kv=8, group=8, width=128)


def listed():
    return [
        # One sequence's first steps: launch and host latency.
        dict(_ATTENTION, **_13B, name="decode13b_n1", S=1, past=100, api="module"),
        # A decode step of 16 sequences with 512 tokens of prompt and up to 512 produced.
        dict(_ATTENTION, **_13B, name="decode13b_n16", S=16, past=1023, api="module"),
        # One long document on shared heads: few rows, so the cache's length is the only thing to split.
        dict(_ATTENTION, **_70B, name="decode70b_long", S=1, past=131071),
        # A full serving batch over an 8-bit cache.
        dict(_ATTENTION, **_70B, name="decode70b_q_n64", S=64, past=8191, values="q"),
        # Odd heads and width, capped scores, bias by distance and a window.
        dict(_ATTENTION, name="decode_odd", kv=7, group=3, width=80, S=5, past=4097, page=32, cap=30.0, bias=True, window=1000),
        # A prompt at once.
        dict(_ATTENTION, **_70B, name="prompt70b_n4096", S=1, rows=4096),
        # Ragged prompts of packed documents behind a common prefix, capped, with a bias.
        dict(_ATTENTION, name="prompt_documents", kv=7, group=3, width=80, S=3, rows=1021, page=32, cap=30.0, bias=True,
             documents=3, prefix=77, api="module"),
        # A piece of a long prompt over an 8-bit cache.
        dict(_ATTENTION, **_70B, name="piece70b_q_n512", S=1, rows=512, past=16000, values="q"),
        # The new tokens of a decode step.
        dict(kind="append", name="append_n32", kv=8, width=128, S=32, rows=1, past=2000, page=64, values="f16"),
        # Prompts quantised into an 8-bit cache.
        dict(kind="append", name="append_q_n2048", kv=40, width=128, S=2, rows=1365, past=0, page=64, values="q"),
        # A fork: the last pages of four sequences in every layer.
        dict(kind="copy", name="fork_n4", kv=8, width=128, layers=8, pages=64, page=64, n=4, how="fork"),
        # A compaction: the upper pages of the pool into the holes below.
        dict(kind="copy", name="compact_n128", kv=8, width=128, layers=4, pages=320, page=64, n=128, how="compact"),
    ]


_MAX_BYTES = 131072 * 8 * 128 * 4
_MAX_PAIRS = 64 * 4096 * 4096 / 2 * 128
_MAX_POOL = 4 * 320 * 64 * 8 * 128 * 4


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["attention"] * 5 + ["append", "copy"])
    while True:
        kv, group = rng.choice([(40, 1), (8, 8), (10, 2), (7, 3), (2, 20)])
        case = dict(kind=kind, kv=kv, width=rng.choice([64, 80, 96, 128, 128, 256]), page=rng.choice([32, 64, 128]))
        if kind == "copy":
            case.update(width=rng.choice([64, 96, 128, 256]), layers=_log_int(rng, 1, 16), pages=_log_int(rng, 8, 512),
                        how=rng.choice(["fork", "compact"]))
            case["n"] = _log_int(rng, 1, case["pages"] // 2)
            if case["layers"] * case["pages"] * case["page"] * kv * case["width"] * 4 <= _MAX_POOL:
                return case
            continue
        prompt = rng.random() < 0.4
        case.update(S=_log_int(rng, 1, 16 if prompt else 128), rows=_log_int(rng, 2, 4096) if prompt else 1,
                    past=_log_int(rng, 1, 16384 if prompt else 131072) if rng.random() < 0.7 or not prompt else 0,
                    values=rng.choice(["f16", "q"]))
        if kind == "append":
            case["past"] = min(case["past"], 4096)
            if case["S"] * (case["rows"] + case["past"]) * kv * case["width"] * 4 <= _MAX_POOL:
                return case
            continue
        case.update(group=group, api=rng.choice(["binding", "module"]), cap=rng.choice([0.0, 0.0, 30.0]),
                    bias=rng.random() < 0.3, window=_log_int(rng, 16, 4096) if rng.random() < 0.2 else 0,
                    documents=rng.choice([0, 0, 2, 5]) if prompt else 0, prefix=_log_int(rng, 1, 512) if prompt and rng.random() < 0.3 else 0)
        w = work(case)
        held = sum(_lengths(case)) * kv * case["width"] * (4 if case["values"] == "f16" else 2)
        padded = case["S"] * max(_lengths(case)) * kv * group * case["rows"]
        if held <= _MAX_BYTES and w["flops"] / 4 <= _MAX_PAIRS and padded <= 2 * 64 * 4096 * 4096:
            return case


# ---- the sequences of a case


def _rows(case):
    """New tokens of each sequence: the most, falling to an eighth of it."""
    S, most = case["S"], case["rows"]
    return [max(1, most - most * 7 * i // (8 * S)) for i in range(S)]


def _lengths(case):
    """Tokens of each sequence in the cache, the new ones included."""
    S, most = case["S"], case["past"]
    return [r + most - most * 7 * i // (8 * S) for i, r in enumerate(_rows(case))]


def _spans(case):
    """(first, last) of each row: the keys that it sees are first <= k < last."""
    firsts, lasts = [], []
    for n, L in zip(_rows(case), _lengths(case)):
        p = np.arange(L - n, L)
        first, last = np.zeros(n, np.int64), p + 1
        if case["documents"]:
            d = case["documents"]
            first = -(-((p * d // L) * L) // d)
        if case["prefix"]:
            last = np.maximum(last, min(case["prefix"], L))
        if case["window"]:
            first = np.maximum(first, p - case["window"] + 1)
        firsts.append(np.maximum(first, 0))
        lasts.append(last)
    return np.concatenate(firsts), np.concatenate(lasts)


def _slopes(heads):
    return [2.0 ** (-8.0 * (i + 1) / heads) for i in range(heads)]


class _Draws:
    """Everything one case draws, in a fixed order from the seed."""

    def __init__(self, seed):
        self.g = torch.Generator(device="cuda")
        self.g.manual_seed(int(seed))

    def normal(self, *shape, scale=1.0):
        return torch.randn(*shape, generator=self.g, device="cuda", dtype=torch.float16).mul_(scale)

    def order(self, n):
        return torch.randperm(n, generator=self.g, device="cuda")


def _codes(x):
    """The last dimension in 8 bits with one scale, by the definition: a / 127 and rint(x * (127 / a)) in 32 bits, the
    division rounded once."""
    a = x.float().abs().amax(-1, keepdim=True)
    inverse = torch.where(a > 0, (127 / a.double()).float(), torch.zeros_like(a))
    return (x.float() * inverse).round().to(torch.int8), (a.double() / 127).float().squeeze(-1)


def _int32(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _sequences(case, d):
    """The page table (pages in any order), lengths, offsets, and a pool of so many pages."""
    lengths, rows = _lengths(case), _rows(case)
    need = [-(-L // case["page"]) for L in lengths]
    order = d.order(sum(need)).int()
    table = torch.zeros((len(need), max(need)), dtype=torch.int32, device="cuda")
    at = torch.arange(max(need), device="cuda")[None, :] < _int32(need)[:, None]
    table[at] = order
    return dict(table=table, lengths=_int32(lengths), offsets=_int32(np.concatenate([[0], np.cumsum(rows)])), pages=sum(need),
                longest=max(lengths), most=max(rows), T=sum(rows))


def _attention_inputs(case, seed):
    d = _Draws(seed)
    s = _sequences(case, d)
    heads, shape = case["kv"] * case["group"], (s["pages"], case["page"], case["kv"], case["width"])
    s["k"], s["v"] = d.normal(*shape), d.normal(*shape)
    s["q"] = d.normal(s["T"], heads, case["width"], scale=2.0)
    first, last = _spans(case)
    s["first"] = _int32(first) if case["documents"] else None
    s["last"] = _int32(last) if case["prefix"] else None
    s["slopes"] = torch.tensor(_slopes(heads), device="cuda") if case["bias"] else None
    s["spans"] = _int32(first), _int32(last)
    return s


def _append_inputs(case, seed):
    d = _Draws(seed)
    s = _sequences(case, d)
    s["k"], s["v"] = d.normal(s["T"], case["kv"], case["width"]), d.normal(s["T"], case["kv"], case["width"], scale=0.5)
    return s


def _copy_inputs(case, seed):
    d = _Draws(seed)
    shape = (case["layers"], case["pages"], case["page"], case["kv"], case["width"])
    n, pages = case["n"], case["pages"]
    if case["how"] == "fork":
        order = d.order(pages).tolist()
        src, dst = order[:n], order[n:2 * n]
    else:
        src, dst = list(range(pages - n, pages)), sorted(d.order(pages - n)[:n].tolist())
    return dict(k=d.normal(*shape), v=d.normal(*shape), src=src, dst=dst)


_INPUTS = dict(attention=_attention_inputs, append=_append_inputs, copy=_copy_inputs)


def prepare(case, seed):
    state = _INPUTS[case["kind"]](case, seed)
    state["case"] = case
    if own:
        _own_prepare(case, state)
    elif case["kind"] == "attention" and case["values"] == "q":
        for name in ("k", "v"):
            state[name], state[name + "_scale"] = _codes(state[name])
    elif case["kind"] == "append":
        shape = (state["pages"], case["page"], case["kv"], case["width"])
        for name in ("k", "v"):
            state[name + "_pool"] = torch.zeros(shape, dtype=torch.int8 if case["values"] == "q" else torch.float16, device="cuda")
            state[name + "_scale"] = torch.zeros(shape[:3], device="cuda") if case["values"] == "q" else None
    elif case["kind"] == "copy":
        state["src_on_gpu"], state["dst_on_gpu"] = _int32(state["src"]).long(), _int32(state["dst"]).long()
    return state


# ---- the framework's calls


def _own_prepare(case, s):
    """What a program keeps: the cache with what it holds so far, the step's rows, workspaces and output buffers."""
    from paper_2607_08786_amd import attention, usp

    pages = case["pages"] if case["kind"] == "copy" else s["pages"]
    eight_bit = case["kind"] != "copy" and case["values"] == "q"
    cache = usp.KVCache(pages, case["kv"], case["width"], page_tokens=case["page"], layers=case.get("layers", 1),
                        dtype=torch.int8 if eight_bit else torch.float16)
    s["cache"] = cache
    if case["kind"] == "copy":
        everything = usp.CacheRows(_int32([range(pages)]), _int32([pages * case["page"]]), _int32([0, pages * case["page"]]))
        for layer in range(case["layers"]):
            cache.append(everything, s["k"][layer].flatten(0, 1), s["v"][layer].flatten(0, 1), layer=layer)
        del s["k"], s["v"]
        return
    s["batch"] = usp.CacheRows(s["table"], s["lengths"], None if case["rows"] == 1 else s["offsets"])
    if case["kind"] == "append":
        shape = (s["T"], case["kv"], case["width"])
        s["k_out"], s["v_out"] = (torch.empty(shape, dtype=torch.float16, device="cuda") for _ in range(2))
        return
    # The pool's pages as the one sequence of a table that names each of them.
    everything = usp.CacheRows(_int32([range(pages)]), _int32([pages * case["page"]]), _int32([0, pages * case["page"]]))
    cache.append(everything, s["k"].flatten(0, 1), s["v"].flatten(0, 1))
    del s["k"], s["v"]
    heads = case["kv"] * case["group"]
    if case["api"] == "module":
        s["module"] = attention.PagedAttention(heads, case["kv"], case["width"], cap=case["cap"], window=case["window"],
                                               slopes=s["slopes"])
    else:
        s["ws"], s["out"] = cache.make_workspace(s["batch"], s["T"], heads), torch.empty_like(s["q"])


def _own_run(s):
    from paper_2607_08786_amd import usp

    case, cache = s["case"], s["cache"]
    if case["kind"] == "copy":
        usp.usp_cache_copy(cache, s["src"], s["dst"])
        return cache.blocks()
    if case["kind"] == "append":
        usp.usp_cache_append(cache, s["batch"], s["k"], s["v"])
        usp.usp_cache_read(cache, s["batch"], s["k_out"], s["v_out"])
        return s["k_out"], s["v_out"]
    if "module" in s:
        return s["module"](s["q"], cache, s["batch"], first=s["first"], last=s["last"])
    usp.usp_attention(cache, s["batch"], s["q"], s["out"], s["ws"], scale=_scale(case), cap=case["cap"], slopes=s["slopes"],
                      window=case["window"], first=s["first"], last=s["last"])
    return s["out"]


def _scale(case):
    return 1.0 / math.sqrt(case["width"])


# ---- the plain forms


def _of_tokens(s, most, last_rows):
    """(page, place in it, whether there is one) of tokens of every sequence: its first `most`, or its new rows."""
    size = s["case"]["page"]
    lengths, off = s["lengths"].long(), s["offsets"].long()
    i = torch.arange(most, device="cuda")[None, :]
    there = i < (off[1:] - off[:-1])[:, None] if last_rows else i < lengths[:, None]
    token = (lengths - (off[1:] - off[:-1]))[:, None] + i if last_rows else i.expand(lengths.shape[0], most)
    token = token.clamp(max=s["longest"] - 1)
    page = s["table"].long().gather(1, torch.where(there, token, 0) // size)
    return page, token % size, there


def _plain_attention(s):
    case = s["case"]
    S, R, L, G = case["S"], s["most"], s["longest"], case["group"]
    page, place, there = _of_tokens(s, L, False)
    k, v = (s[n][page, place].float() for n in ("k", "v"))  # [S, L, kv, width]
    if case["values"] == "q":
        k, v = k * s["k_scale"][page, place][..., None], v * s["v_scale"][page, place][..., None]
    v = v * there[:, :, None, None]
    off = s["offsets"].long()
    t = torch.arange(s["T"], device="cuda")
    seq = torch.searchsorted(off, t, right=True) - 1
    at = t - off[seq]
    q = torch.zeros((S, R, case["kv"], G, case["width"]), device="cuda")
    q[seq, at] = s["q"].float().view(s["T"], case["kv"], G, case["width"])
    first, last, position = (torch.zeros((S, R), dtype=torch.int64, device="cuda") for _ in range(3))
    first[seq, at], last[seq, at] = s["spans"][0].long(), s["spans"][1].long()
    position[seq, at] = s["lengths"].long()[seq] - (off[1:] - off[:-1])[seq] + at
    kt = k.permute(0, 2, 3, 1).contiguous()                                     # [S, kv, width, L]
    qt = q.permute(0, 2, 1, 3, 4).reshape(S, case["kv"], R * G, case["width"])
    x = torch.matmul(qt, kt).view(S, case["kv"], R, G, L).mul_(_scale(case))
    if case["cap"]:
        x = torch.tanh(x.div_(case["cap"])).mul_(case["cap"])
    key = torch.arange(L, device="cuda")
    if s["slopes"] is not None:
        distance = (position[:, :, None] - key).abs().float()                     # [S, R, L]
        x -= s["slopes"].view(1, case["kv"], 1, G, 1) * distance[:, None, :, None, :]
    seen = (key >= first[:, :, None]) & (key < last[:, :, None])
    x.masked_fill_(~seen[:, None, :, None, :], -torch.inf)
    top = x.amax(-1, keepdim=True)
    x = x.sub_(torch.where(top > -torch.inf, top, torch.zeros_like(top))).exp_()
    total = x.sum(-1, keepdim=True)
    vt = v.permute(0, 2, 1, 3).contiguous()                                     # [S, kv, L, width]
    out = torch.matmul(x.view(S, case["kv"], R * G, L), vt).view(S, case["kv"], R, G, case["width"])
    out = (out / total.clamp_min(1e-30)).permute(0, 2, 1, 3, 4)
    return out[seq, at].reshape(s["T"], case["kv"] * G, case["width"]).half()


def _plain_append(s):
    page, place, there = _of_tokens(s, s["most"], True)
    at = page[there], place[there]
    out = []
    for name in ("k", "v"):
        pool, scale = s[name + "_pool"], s[name + "_scale"]
        if scale is None:
            pool[at] = s[name]
            out.append(pool[at])
        else:
            pool[at], scale[at] = _codes(s[name])
            out.append((pool[at].float() * scale[at][..., None]).half())
    return tuple(out)


def _blocks(k, v):
    """Pools [layers, pages, tokens, heads, width] as the framework's views: blocks of 32 tokens, a key's place in its block
    by bits, eight of a width, and a value's in eights."""
    layers, pages, size, kv, width = k.shape
    k = k.view(layers, pages, size // 32, 2, 2, 2, 4, kv, width // 8, 8).permute(0, 1, 7, 2, 3, 4, 5, 6, 8, 9)
    v = v.view(layers, pages, size // 32, 4, 8, kv, width).permute(0, 1, 5, 2, 3, 4, 6)
    return k, v


def _plain_copy(s):
    for name in ("k", "v"):
        s[name][:, s["dst_on_gpu"]] = s[name][:, s["src_on_gpu"]]
    return _blocks(s["k"], s["v"])


_PLAIN = dict(attention=_plain_attention, append=_plain_append, copy=_plain_copy)


def run(state):
    if own:
        return _own_run(state)
    return _PLAIN[state["case"]["kind"]](state)


# ---- what a pass cannot do without


def work(case):
    if case["kind"] == "copy":
        return {"bytes": 2.0 * case["layers"] * case["n"] * case["page"] * case["kv"] * case["width"] * 4, "flops": 0.0}
    kv, width, value = case["kv"], case["width"], 2 if case["values"] == "f16" else 1
    held = 2 * (width * value + (4 if value == 1 else 0)) * kv  # of one token, its keys and values
    T, tables = sum(_rows(case)), 4 * sum(-(-L // case["page"]) for L in _lengths(case)) + 8 * case["S"]
    if case["kind"] == "append":
        return {"bytes": 2.0 * T * (2 * width * 2 * kv + held) + tables, "flops": 0.0}
    first, last = _spans(case)
    ends = np.cumsum([0] + _rows(case))
    keys = sum(int(last[a:b].max() - first[a:b].min()) for a, b in zip(ends[:-1], ends[1:]))
    heads = kv * case["group"]
    return {"bytes": float(keys * held + 2 * T * heads * width * 2 + tables),
            "flops": 4.0 * heads * width * float(np.maximum(last - first, 0).sum())}


# ---- the definitions in 64 bits


def _values64(x, values):
    """What the cache holds of x [..., width], in 64 bits."""
    if values == "f16":
        return x.double()
    top = x.float().abs().amax(-1, keepdim=True)
    inverse = torch.where(top > 0, (127.0 / top.double()).float(), torch.zeros_like(top)).double()
    return torch.round((x.double() * inverse).float().double()) * (top.double() / 127).float().double()


def _exact_attention(case, s):
    out, table, row = [], s["table"].tolist(), 0
    spans = [x.long() for x in s["spans"]]
    slopes = _slopes(case["kv"] * case["group"])
    for i, (n, L) in enumerate(zip(_rows(case), _lengths(case))):
        pages = table[i][:-(-L // case["page"])]
        first, last = spans[0][row:row + n, None], spans[1][row:row + n, None]
        key = torch.arange(L, device="cuda")[None, :]
        hidden = (key < first) | (key >= last)
        away = (torch.arange(L - n, L, device="cuda")[:, None] - key).abs().double()
        heads = []
        for h in range(case["kv"]):
            k, v = (_values64(s[x][pages, :, h].reshape(-1, case["width"])[:L], case["values"]) for x in ("k", "v"))
            for g in range(case["group"]):
                j = h * case["group"] + g
                x = (s["q"][row:row + n, j].double() @ k.t()) / math.sqrt(case["width"])
                if case["cap"]:
                    x = case["cap"] * torch.tanh(x / case["cap"])
                if case["bias"]:
                    x = x - float(np.float32(slopes[j])) * away
                heads.append(torch.softmax(x.masked_fill(hidden, -math.inf), 1) @ v)
        out.append(torch.stack(heads, 1))
        row += n
    return torch.cat(out)


def exact(case, seed):
    s = _INPUTS[case["kind"]](case, seed)
    if case["kind"] == "attention":
        return _exact_attention(case, s)
    if case["kind"] == "append":
        return _values64(s["k"], case["values"]), _values64(s["v"], case["values"])
    for name in ("k", "v"):
        for a, b in zip(s["src"], s["dst"]):
            s[name][:, b] = s[name][:, a]
    return tuple(x.double() for x in _blocks(s["k"], s["v"]))
