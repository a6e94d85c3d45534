"""Plain forms in 64 bits of the 8-bit products, the products grouped by expert and the block norms, with the error
that the kernels' arithmetic allows.

An output is rounded to fp16 once: half a step, 2^-11 of the value, or 2^-25 where it is subnormal. Before that, in
fp32 (2^-24 a rounding): for 8-bit products, exact integer sums, their conversion, two scales, bias, activation and
residual, fewer than 32 roundings of what is added up; for fp16 products also K additions in some order."""
import numpy as np

U = 2.0 ** -24


def act64(v, name):
    if name == "relu":
        return np.maximum(v, 0)
    if name == "gelu_tanh":
        return 0.5 * v * (1 + np.tanh(np.sqrt(2 / np.pi) * (v + 0.044715 * v ** 3)))
    if name == "silu":
        return v / (1 + np.exp(-v))
    return v


def round_tol(y):
    return 2.0 ** -11 * np.abs(y) + 2.0 ** -25


def quantize(x):
    """Codes and scales, in the fp32 operations of the definition (numpy's are correctly rounded)."""
    x = x.astype(np.float32)
    a = np.abs(x).max(1)
    with np.errstate(divide="ignore", invalid="ignore"):
        inv = np.where(a > 0, np.float32(127) / a, np.float32(0)).astype(np.float32)
        codes = np.rint(x * inv[:, None])
    good = np.isfinite(a)
    codes = np.where(good[:, None], codes, 0).astype(np.int8)
    return codes, np.where(good, a / np.float32(127), np.float32("nan")).astype(np.float32)


def product(x, w, bias=None, act="none", residual=None, weight=None, sums=32):
    """(y, tolerance) of weight * act(x w^T + bias) + residual, x [N, K] and w [M, K] in float64. sums: roundings of
    the sum itself."""
    v, size = x @ w.T, np.abs(x) @ np.abs(w).T
    if bias is not None:
        v, size = v + bias, size + np.abs(bias)
    y = act64(v, act)
    if weight is not None:
        y, size = y * weight[:, None], size * np.abs(weight[:, None])
    if residual is not None:
        y, size = y + residual, size + np.abs(residual)
    return y, round_tol(y) + sums * U * size


def f16_sums(K):
    return 2 * (K + 40)  # every product and addition, twice over for what the matrix unit drops


def _normed(v, size, kind, w, b, eps, roundings):
    """(norm of v, its error's size in fp32 roundings) for v known up to roundings * U * size."""
    w = np.ones(v.shape[1]) if w is None else w
    b = np.zeros(v.shape[1]) if b is None else b
    if kind == "none":
        return v, size
    m = v.mean(1, keepdims=True) if kind == "layer" else 0.0
    inv = 1 / np.sqrt(((v - m) ** 2).mean(1, keepdims=True) + eps)
    h = (v - m) * inv * w + b
    spread = np.abs(v) + size + (size.mean(1, keepdims=True) if kind == "layer" else 0)
    # The root mean square of the errors moves inv, relative to itself, by at most their ratio to 1 / inv.
    moved = np.sqrt((spread ** 2).mean(1, keepdims=True)) * inv
    return h, np.abs(w) * inv * spread + np.abs((v - m) * inv * w) * (1 + moved) + np.abs(b)


def norm(residual, y=None, gate=None, scale=1.0, post="none", post_weight=None, post_bias=None, pre="none",
         pre_weight=None, pre_bias=None, eps=1e-5, gate_activation="none"):
    """(r, tolerance, h, tolerance), operands in float64."""
    K = residual.shape[1]
    roundings = 64 + K // 1024 + 8  # the longest chain of additions to a sum, and what follows it
    r, size = residual, np.abs(residual)
    if y is not None:
        v, vs = _normed(y, np.abs(y), post, post_weight, post_bias, eps, roundings)
        if gate is not None:
            g = {"none": lambda z: z, "sigmoid": lambda z: 1 / (1 + np.exp(-z)), "tanh": np.tanh,
                 "silu": lambda z: z / (1 + np.exp(-z))}[gate_activation](gate)
            v, vs = v * g, vs * np.abs(g) + np.abs(v * g)
        r, size = residual + scale * v, size + abs(scale) * vs
    h, hs = _normed(r, size, pre, pre_weight, pre_bias, eps, roundings)
    return r, round_tol(r) + roundings * U * size, h, round_tol(h) + roundings * U * hs


def close(got, want, tol):
    got = got.astype(np.float64)
    assert got.shape == want.shape
    bad = ~(np.abs(got - want) <= tol)
    assert not bad.any(), (int(bad.sum()), got[bad][:4], want[bad][:4], (np.abs(got - want) / tol)[bad][:4])
