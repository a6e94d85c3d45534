"""The 8-bit products, the products grouped by expert and the block norms, as a program that uses them makes them.

A case is one pass through an operator:

* ``product``: a pruned layer with 8-bit weights (one scale per output channel) on tokens in 8 bits (one scale per token),
  through the binding on tokens that are 8-bit already, or through the module, which quantises fp16 tokens first;
* ``experts``: rows sorted by expert, each multiplied by its expert's pruned weight (fp16 or 8-bit), ragged row counts,
  experts without rows among them; rows may be gathered from the tokens and weighted by the router;
* ``norm``: the residual update after a block (norm of its output, gate, residual scale) and the norm before the next one;
  with ``then`` the norm writes 8-bit tokens and the next block's 8-bit product reads them.

Layer shapes are those of ``workloads`` and generic ones. Weights are N(0, 0.02) pruned by magnitude per row; everything is
drawn on the GPU from the seed alone.
"""
from __future__ import annotations

import math

import torch

own = False

_PRODUCT = dict(kind="product", api="spmm", sparsity=50, epilogue="")
_EXPERTS = dict(kind="experts", values="f16", sparsity=50, epilogue="")
_NORM = dict(kind="norm", post="none", pre="rms", gate="none", then=0)


def listed():
    return [
        # The smallest layer of the test workloads: launch and host latency.
        dict(_PRODUCT, name="q_tiny_n16", M=1024, K=1024, N=16),
        # One sequence's decode step on one GPU's share of the 70B FFN, as a module in a model.
        dict(_PRODUCT, name="q_ffn70b_shard8_n1", M=3584, K=8192, N=1, api="module"),
        # The benchmark's layer, 16 sequences, tokens quantised by the norm before it.
        dict(_PRODUCT, name="q_ffn70b_n16", M=28672, K=8192, N=16),
        # Nothing a multiple of anything, and the whole epilogue.
        dict(_PRODUCT, name="q_ragged_n21", M=4999, K=4093, N=21, api="module", epilogue="bias+silu+residual"),
        # Prefill of 1024 tokens through the module.
        dict(_PRODUCT, name="q_ffn13b_up_n1024", M=13824, K=5120, N=1024, api="module", epilogue="bias+gelu_tanh"),
        # Decode step of 32 sequences, two of eight large experts each: the FFN's first layer.
        dict(_EXPERTS, name="experts8_n32", E=8, M=3584, K=8192, tokens=32, top=2, epilogue="silu"),
        # Decode step of 16 sequences over many small 8-bit experts, most of which get no row: the second layer, with
        # the router's weights.
        dict(_EXPERTS, name="experts64_q_n16", E=64, M=2048, K=1024, tokens=16, top=2, values="q", epilogue="weight"),
        # An odd number of experts, odd sizes, rows in place.
        dict(_EXPERTS, name="experts7_q_ragged", E=7, M=1001, K=1499, tokens=301, top=1, values="q", epilogue="bias+relu"),
        # Prefill: the rows of 2048 tokens, two experts each.
        dict(_EXPERTS, name="experts16_n2048", E=16, M=2816, K=2048, tokens=2048, top=2),
        # The norm between two blocks of a 70B decoder for one sequence.
        dict(_NORM, name="norm_n1", N=1, K=8192),
        # Prefill: layer norms on both sides of the block and a gate for each token and channel.
        dict(_NORM, name="norm_n2048", N=2048, K=5120, post="layer", pre="layer", gate="token"),
        # A 13B block's norms, gate and 8-bit tokens, then the 8-bit projection that reads them.
        dict(_NORM, name="norm_q_attn13b_n32", N=32, K=5120, post="rms", gate="channel", then=5120),
    ]


_MAX_WEIGHTS = 28672 * 8192
_MAX_PRODUCT = 13824 * 5120 * 1024
_MAX_EXPERTS = 2816 * 2048 * 4096
_EPILOGUES = ("", "bias", "bias+relu", "bias+gelu_tanh", "bias+silu", "bias+residual", "residual", "bias+silu+residual")


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _side(rng, lo, hi):
    """A layer's side: a multiple of 64 as models have them, and one time in four any number."""
    v = _log_int(rng, lo, hi)
    return (v + 63) // 64 * 64 if rng.random() < 0.75 else v


def draw(rng):
    kind = rng.choice(["product", "product", "experts", "experts", "norm"])
    sparsity = rng.choice([40, 50, 60, 70])
    if kind == "product":
        while True:
            M, K, N = _side(rng, 256, 28672), _side(rng, 256, 28672), _log_int(rng, 1, 2048)
            if M * K <= _MAX_WEIGHTS and M * K * N <= _MAX_PRODUCT:
                return dict(kind=kind, api=rng.choice(["spmm", "module"]), sparsity=sparsity, M=M, K=K, N=N,
                            epilogue=rng.choice(_EPILOGUES))
    if kind == "experts":
        while True:
            E, M, K = _log_int(rng, 1, 64), _side(rng, 128, 8192), _side(rng, 128, 8192)
            tokens, top = _log_int(rng, 1, 4096), rng.choice([1, 2, 4])
            if E * M * K <= _MAX_WEIGHTS and M * K * tokens * top <= _MAX_EXPERTS and top <= E:
                return dict(kind=kind, E=E, M=M, K=K, tokens=tokens, top=top, values=rng.choice(["f16", "q"]),
                            sparsity=sparsity, epilogue=rng.choice(["", "bias", "bias+relu", "silu", "weight", "bias+weight"]))
    N, K = _log_int(rng, 1, 2048), _side(rng, 64, 8192)
    then = _side(rng, 256, 8192) if N <= 256 and rng.random() < 0.3 else 0
    return dict(kind="norm", N=N, K=K, post=rng.choice(["none", "rms", "layer"]), pre=rng.choice(["rms", "layer"]),
                gate=rng.choice(["none", "channel", "token"]), then=then)


_EPS = 1e-5
_RESIDUAL_SCALE = 0.7


class _Draws:
    """Everything one case draws, in a fixed order from the seed."""

    def __init__(self, seed):
        self.g = torch.Generator(device="cuda")
        self.g.manual_seed(int(seed))

    def normal(self, *shape, scale=1.0):
        return torch.randn(*shape, generator=self.g, device="cuda", dtype=torch.float16).mul_(scale)

    def weight(self, M, K, sparsity):
        """An fp16 weight and its keep-mask: the largest magnitudes of every row."""
        W = self.normal(M, K, scale=0.02)
        prune = max(1, K * sparsity // 100)
        mask = torch.empty((M, K), dtype=torch.bool, device="cuda")
        for r in range(0, M, 4096):
            a = W[r:r + 4096].abs()
            mask[r:r + 4096] = a > a.kthvalue(prune, dim=1, keepdim=True).values
        return W, mask

    def weight_q(self, M, K, sparsity):
        """The same in 8 bits: whole numbers up to 127, the mask, a scale for each row."""
        W, mask = self.weight(M, K, sparsity)
        scale = W.abs().amax(1).float() / 127
        q = torch.empty((M, K), dtype=torch.int8, device="cuda")
        for r in range(0, M, 4096):
            q[r:r + 4096] = (W[r:r + 4096].float() / scale[r:r + 4096, None]).round_().to(torch.int8)
        return q.mul_(mask), mask, scale

    def order(self, n):
        return torch.randperm(n, generator=self.g, device="cuda")

    def below(self, limit, n):
        return torch.randint(limit, (n,), generator=self.g, device="cuda", dtype=torch.int32)

    def uniform(self, n):
        return torch.rand(n, generator=self.g, device="cuda")


def _parts(case):
    return case["epilogue"].split("+") if case["epilogue"] else []


def _activation(case):
    return next((p for p in _parts(case) if p in ("relu", "gelu_tanh", "silu")), "none")


def _quantized(x):
    """Tokens in 8 bits and their scales."""
    amax = x.float().abs().amax(1)
    inverse = torch.where(amax > 0, 127 / amax, torch.zeros_like(amax))
    return (x.float() * inverse[:, None]).round().to(torch.int8), amax / 127


# ---- inputs


def _product_inputs(case, seed):
    d, parts = _Draws(seed), _parts(case)
    M, K, N = case["M"], case["K"], case["N"]
    w, mask, w_scale = d.weight_q(M, K, case["sparsity"])
    x = d.normal(N, K)
    s = dict(w=w, mask=mask, w_scale=w_scale, bias=d.normal(M) if "bias" in parts else None,
             residual=d.normal(N, M) if "residual" in parts else None, act=_activation(case))
    if case["api"] == "module":
        s["x"] = x
    else:
        s["xq"], s["x_scale"] = _quantized(x)
    return s


def _counts(case):
    """Rows of the experts by rank: shares falling with the rank, whole numbers that sum to all rows."""
    E, T = case["E"], case["tokens"] * case["top"]
    share = [1.0 / (r + 2) for r in range(E)]
    got = [int(T * x / sum(share)) for x in share]
    for i in range(T - sum(got)):
        got[i % E] += 1
    return got


def _experts_inputs(case, seed):
    d, parts = _Draws(seed), _parts(case)
    E, M, K, tokens = case["E"], case["M"], case["K"], case["tokens"]
    T = tokens * case["top"]
    weights, masks, scales = [], [], []
    for _ in range(E):
        if case["values"] == "q":
            w, mask, scale = d.weight_q(M, K, case["sparsity"])
            scales.append(scale)
        else:
            w, mask = d.weight(M, K, case["sparsity"])
            w = w.mul_(mask)
        weights.append(w)
        masks.append(mask)
    counts = torch.tensor(_counts(case), device="cuda")[d.order(E)]  # which expert has which rank
    offsets = torch.zeros(E + 1, dtype=torch.int32, device="cuda")
    offsets[1:] = counts.cumsum(0)
    x = d.normal(tokens, K)
    s = dict(w=torch.stack(weights), masks=masks, w_scale=torch.stack(scales) if scales else None, offsets=offsets,
             longest=max(_counts(case)), rows=d.below(tokens, T) if case["top"] > 1 else None, act=_activation(case),
             bias=d.normal(E, M) if "bias" in parts else None, weight=d.uniform(T) if "weight" in parts else None)
    if scales:
        s["x"], s["x_scale"] = _quantized(x)
    else:
        s["x"], s["x_scale"] = x, None
    return s


def _norm_inputs(case, seed):
    d, N, K = _Draws(seed), case["N"], case["K"]
    s = dict(residual=d.normal(N, K, scale=4.0), y=d.normal(N, K, scale=0.5),
             gate=None if case["gate"] == "none" else d.normal(K) if case["gate"] == "channel" else d.normal(N, K))
    for side in ("post", "pre"):
        kind = case[side]
        s[side] = kind
        s[side + "_weight"] = d.normal(K, scale=0.1).add_(1) if kind != "none" else None
        s[side + "_bias"] = d.normal(K, scale=0.1) if kind == "layer" else None
    if case["then"]:
        s["w"], s["mask"], s["w_scale"] = d.weight_q(case["then"], K, 50)
    return s


_INPUTS = dict(product=_product_inputs, experts=_experts_inputs, norm=_norm_inputs)


def prepare(case, seed):
    state = _INPUTS[case["kind"]](case, seed)
    state["kind"] = case["kind"]
    if own:
        _own_prepare(case, state)
    return state


# ---- the framework's calls


def _own_prepare(case, s):
    """What a program keeps: the encoded weights, workspaces and output buffers."""
    from paper_2607_08786_amd import linear, usp

    def encoded(w, mask, scale):
        host = mask.cpu().numpy()
        if scale is None:
            return usp.SparseMatrix(w.cpu().numpy(), host)
        return usp.SparseMatrixQ(w.cpu().numpy(), host, scale.cpu().numpy())

    def empty(*shape, dtype=torch.float16):
        return torch.empty(shape, dtype=dtype, device="cuda")

    if case["kind"] == "product":
        if case["api"] == "module":
            s["module"] = linear.SparseLinearQ(s["w"], s["mask"], s["w_scale"], s["bias"], s["act"])
        else:
            s["A"] = encoded(s["w"], s["mask"], s["w_scale"])
            s["ws"], s["out"] = s["A"].make_workspace(case["N"]), empty(case["N"], case["M"])
    elif case["kind"] == "experts":
        E, T = case["E"], case["tokens"] * case["top"]
        s["group"] = usp.ExpertGroup([encoded(s["w"][e], s["masks"][e], None if s["w_scale"] is None else s["w_scale"][e])
                                      for e in range(E)])
        s["ws"], s["out"] = s["group"].make_workspace(T), empty(T, case["M"])
    else:
        N, K = case["N"], case["K"]
        s["residual_out"] = empty(N, K)
        if case["then"]:
            s["A"] = encoded(s["w"], s["mask"], s["w_scale"])
            s["ws"], s["out"] = s["A"].make_workspace(N), empty(N, case["then"])
            s["hq"], s["h_scale"] = empty(N, K, dtype=torch.int8), empty(N, dtype=torch.float32)
        else:
            s["h"] = empty(N, K)


def _own_run(s):
    from paper_2607_08786_amd import usp

    if s["kind"] == "product":
        if "module" in s:
            return s["module"](s["x"], s["residual"])
        usp.usp_spmm_q(s["A"].handle, s["xq"], s["x_scale"], s["out"], s["ws"], s["bias"], s["residual"], s["act"])
        return s["out"]
    if s["kind"] == "experts":
        usp.usp_spmm_grouped(s["group"].handle, s["x"], s["offsets"], s["out"], s["ws"], x_scale=s["x_scale"],
                             rows=s["rows"], bias=s["bias"], row_weight=s["weight"], activation=s["act"])
        return s["out"]
    args = dict(y=s["y"], gate=s["gate"], scale=_RESIDUAL_SCALE, post=s["post"], post_weight=s["post_weight"],
                post_bias=s["post_bias"], pre=s["pre"], pre_weight=s["pre_weight"], pre_bias=s["pre_bias"], eps=_EPS,
                residual_out=s["residual_out"])
    if "A" not in s:
        usp.usp_norm(s["residual"], out=s["h"], **args)
        return s["residual_out"], s["h"]
    usp.usp_norm(s["residual"], out_q=s["hq"], out_scale=s["h_scale"], **args)
    usp.usp_spmm_q(s["A"].handle, s["hq"], s["h_scale"], s["out"], s["ws"])
    return s["residual_out"], s["out"]


# ---- the plain forms


def _act(v, act):
    if act == "relu":
        return v.clamp_min(0)
    if act == "gelu_tanh":
        return 0.5 * v * (1 + torch.tanh(math.sqrt(2 / math.pi) * (v + 0.044715 * v * v * v)))
    if act == "silu":
        return v / (1 + torch.exp(-v))
    return v


def _plain_product(xq, x_scale, s):
    v = (xq.float() @ s["w"].float().t()) * x_scale[:, None] * s["w_scale"]
    if s.get("bias") is not None:
        v = v + s["bias"].float()
    v = _act(v, s.get("act"))
    if s.get("residual") is not None:
        v = v + s["residual"].float()
    return v.half()


def _plain_experts(s):
    off, w = s["offsets"].long(), s["w"].float()
    T = s["rows"].numel() if s["rows"] is not None else s["x"].shape[0]
    t = torch.arange(T, device=w.device)
    expert = torch.searchsorted(off, t, right=True) - 1
    at = t - off[expert]
    x = s["x"].float()
    if s["x_scale"] is not None:
        x = x * s["x_scale"][:, None]
        w = w * s["w_scale"][:, :, None]
    padded = torch.zeros((w.shape[0], s["longest"], w.shape[2]), device=w.device)
    padded[expert, at] = x if s["rows"] is None else x[s["rows"].long()]
    v = torch.bmm(w, padded.transpose(1, 2).contiguous())[expert, :, at]
    if s["bias"] is not None:
        v = v + s["bias"].float()[expert]
    v = _act(v, s["act"])
    if s["weight"] is not None:
        v = v * s["weight"][:, None]
    return v.half()


def _plain_norm(v, kind, weight, bias):
    if kind == "none":
        return v
    if kind == "layer":
        v = v - v.mean(1, keepdim=True)
    v = v * torch.rsqrt((v * v).mean(1, keepdim=True) + _EPS) * weight.float()
    return v if bias is None else v + bias.float()


def _plain_block(s):
    v = _plain_norm(s["y"].float(), s["post"], s["post_weight"], s["post_bias"])
    if s["gate"] is not None:
        v = v * s["gate"].float()
    r = s["residual"].float() + _RESIDUAL_SCALE * v
    h = _plain_norm(r, s["pre"], s["pre_weight"], s["pre_bias"]).half()
    if "w" not in s:
        return r.half(), h
    return r.half(), _plain_product(*_quantized(h), dict(w=s["w"], w_scale=s["w_scale"]))


def run(state):
    if own:
        return _own_run(state)
    if state["kind"] == "product":
        xq, x_scale = _quantized(state["x"]) if "x" in state else (state["xq"], state["x_scale"])
        return _plain_product(xq, x_scale, state)
    if state["kind"] == "experts":
        return _plain_experts(state)
    return _plain_block(state)


# ---- what a pass cannot do without


def _kept(M, K, sparsity):
    return M * (K - K * sparsity // 100)


def _weight_bytes(M, K, sparsity, value):
    """One bit a position and the kept values (an 8-bit weight has a scale a row too)."""
    return M * K / 8 + value * _kept(M, K, sparsity) + (4 * M if value == 1 else 0)


def work(case):
    parts = _parts(case) if "epilogue" in case else []
    if case["kind"] == "product":
        M, K, N = case["M"], case["K"], case["N"]
        x = 2 * N * K if case["api"] == "module" else N * K + 4 * N
        extra = (2 * M if "bias" in parts else 0) + (2 * M * N if "residual" in parts else 0)
        return {"bytes": _weight_bytes(M, K, case["sparsity"], 1) + x + 2 * N * M + extra,
                "flops": 2.0 * _kept(M, K, case["sparsity"]) * N}
    if case["kind"] == "experts":
        M, K, T, value = case["M"], case["K"], case["tokens"] * case["top"], 1 if case["values"] == "q" else 2
        active = sum(c > 0 for c in _counts(case))
        per_row = 2 * M + (4 if case["top"] > 1 else 0) + (4 if "weight" in parts else 0)
        return {"bytes": active * (_weight_bytes(M, K, case["sparsity"], value) + (2 * M if "bias" in parts else 0)) +
                min(T, case["tokens"]) * (value * K + (4 if value == 1 else 0)) + T * per_row + 4 * (case["E"] + 1),
                "flops": 2.0 * _kept(M, K, case["sparsity"]) * T}
    N, K, M = case["N"], case["K"], case["then"]
    vectors = 2 * K * (("none", "rms", "layer").index(case["post"]) + ("none", "rms", "layer").index(case["pre"]))
    gate = 2 * K * {"none": 0, "channel": 1, "token": N}[case["gate"]]
    out = {"bytes": 3 * 2 * N * K + vectors + gate, "flops": 12.0 * N * K}
    if M:
        return {"bytes": out["bytes"] + _weight_bytes(M, K, 50, 1) + 2 * N * M, "flops": out["flops"] + 2.0 * _kept(M, K, 50) * N}
    return {"bytes": out["bytes"] + 2 * N * K, "flops": out["flops"]}


# ---- the definitions in 64 bits


def _product64(x, w):
    """x w^T in slices of rows that fit the card several times over."""
    out = torch.empty((x.shape[0], w.shape[0]), dtype=torch.float64, device=x.device)
    for r in range(0, w.shape[0], 4096):
        out[:, r:r + 4096] = x @ w[r:r + 4096].double().t()
    return out


def _act64(v, act):
    if act == "gelu_tanh":
        return torch.nn.functional.gelu(v, approximate="tanh")
    return {"relu": torch.relu, "silu": torch.nn.functional.silu}.get(act, lambda z: z)(v)


def _tokens64(x):
    """The values that the 8-bit tokens stand for."""
    top = x.double().abs().amax(1, keepdim=True)
    code = torch.where(top > 0, torch.round(x.double() * (127 / top)), torch.zeros_like(top))
    return code * (top / 127)


def exact(case, seed):
    s = _INPUTS[case["kind"]](case, seed)
    if case["kind"] == "product":
        x = _tokens64(s["x"]) if "x" in s else s["xq"].double() * s["x_scale"].double()[:, None]
        v = _product64(x, s["w"]) * s["w_scale"].double()
        if s["bias"] is not None:
            v += s["bias"].double()
        v = _act64(v, s["act"])
        return v if s["residual"] is None else v + s["residual"].double()
    if case["kind"] == "experts":
        off = s["offsets"].tolist()
        x = s["x"].double() if s["x_scale"] is None else s["x"].double() * s["x_scale"].double()[:, None]
        if s["rows"] is not None:
            x = x[s["rows"].long()]
        v = torch.empty((x.shape[0], case["M"]), dtype=torch.float64, device="cuda")
        for e in range(case["E"]):
            part = _product64(x[off[e]:off[e + 1]], s["w"][e])
            if s["w_scale"] is not None:
                part *= s["w_scale"][e].double()
            v[off[e]:off[e + 1]] = part if s["bias"] is None else part + s["bias"][e].double()
        v = _act64(v, s["act"])
        return v if s["weight"] is None else v * s["weight"].double()[:, None]

    def normed(v, side):
        kind = s[side]
        if kind == "none":
            return v
        w = s[side + "_weight"].double()
        if kind == "layer":
            return torch.nn.functional.layer_norm(v, (v.shape[1],), w, s[side + "_bias"].double(), _EPS)
        return w * v / torch.sqrt(torch.linalg.vector_norm(v, dim=1, keepdim=True) ** 2 / v.shape[1] + _EPS)

    v = normed(s["y"].double(), "post")
    r = s["residual"].double() + _RESIDUAL_SCALE * (v if s["gate"] is None else v * s["gate"].double())
    h = normed(r, "pre")
    return (r, h) if "w" not in s else (r, _product64(_tokens64(h.half()), s["w"]) * s["w_scale"].double())
