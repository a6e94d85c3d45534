"""Attention over a cache in its plain form in 64 bits, with the error that the kernels' arithmetic allows.

out = sum_k w_k V_k / sum_k w_k. With p_k = w_k / sum w and A = sum_k p_k |V_k| (per channel), the errors are
* the result's rounding to fp16: 2^-11 |out|, 2^-25 where it is subnormal;
* the weights' rounding to fp16, relative d_k of at most 2^-11 above and below the line alike: sum_k p_k d_k (V_k - out), so
  2^-11 (A + |out|), and 2^-25 each where they are subnormal, so 2^-25 sum |V_k| over sum w, which is at least 1 (weights
  are relative to the largest);
* in 8 bits a weight's factor f between 16 / 17 and 17 / 16, held as log2 f (below 0.0875, so half a step of fp16 is 2^-15) and as
  1 / f - 1 (the same): relative 2^-15 ln 2 + 2^-15 < 2^-14 of each weight, so 2^-14 (A + |out|);
* an error e of the scores, which moves p_k by p_k (e_k - sum p e), so at most 2 e A;
* fp32 sums over n keys and the rescaling of what was summed: fewer than 4 (n + 40) roundings of A.
e in roundings U = 2^-24: 2 (D + 40) of sum_d |q_d K_d| scale (products and their sum, twice over for what the matrix unit
drops), 16 of the largest score, cap and bias each (scaling, cap, bias, subtraction of the maximum, exponential). A cap
counts as at most 512 or 32 times the largest score: cap tanh(y) for |y| < 1 / 8 has a series, with an error relative to the
score itself, and elsewhere the cap is less than 9 times the score."""
import numpy as np
import torch

U = 2.0 ** -24


def held(x, eight_bit):
    """What the cache holds of x [..., D] fp16, in 64 bits."""
    x = x.float()
    if not eight_bit:
        return x.double()
    a = x.abs().amax(-1, keepdim=True)
    finite = torch.isfinite(a)
    inv = torch.where(a > 0, (127.0 / a.double()).float(), torch.zeros_like(a))
    codes = (x.double() * inv.double()).float().round()  # the fp32 product, rounded to even
    out = codes.double() * (a.double() / 127).float().double()
    return torch.where(finite, out, torch.full_like(out, float("nan")))


def spans(n, L, first=None, last=None, window=0):
    p = torch.arange(L - n, L)
    lo = torch.zeros(n, dtype=torch.int64) if first is None else first.long()
    if window:
        lo = torch.maximum(lo, p - window + 1)
    hi = p + 1 if last is None else last.long()
    hi = torch.where(p < 0, torch.zeros_like(hi), hi)
    return p, lo.clamp(min=0), hi.clamp(max=L)


def attend(q, K, V, scale=None, cap=0.0, slopes=None, first=None, last=None, window=0):
    """(out, tolerance) [n, heads, D] of the last n tokens of a sequence whose held keys and values are K, V [L, kv, D]."""
    n, heads, D = q.shape
    L, kv = K.shape[0], K.shape[1]
    scale = float(np.float32(D ** -0.5 if scale is None else scale))
    cap = float(np.float32(cap))
    p, lo, hi = spans(n, L, first, last, window)
    key = torch.arange(L)
    sees = (key >= lo[:, None]) & (key < hi[:, None])
    out = torch.zeros(n, heads, D, dtype=torch.float64)
    tol = torch.full_like(out, 2.0 ** -25)
    for h in range(heads):
        k, v, x = K[:, h * kv // heads], V[:, h * kv // heads], q[:, h].double()
        s = x @ k.T * scale
        size = x.abs() @ k.abs().T * abs(scale)
        if cap:
            s = cap * torch.tanh(s / cap)
        bias = torch.zeros_like(s)
        if slopes is not None:
            bias = float(slopes[h].float()) * (p[:, None] - key).abs().double()
        s = s - bias
        for i in range(n):
            at = sees[i].nonzero()[:, 0]
            if not len(at):
                continue
            z, vv = s[i, at], v[at]
            most = min(cap, max(512.0, 32 * float(z.abs().nan_to_num(0, 0).max())))
            top = z.max()
            w = torch.exp(z - (top if torch.isfinite(top) else 0))
            w = w / w.sum()
            out[i, h] = w @ vv
            A = w @ vv.abs()
            e = U * (2 * (D + 40) * size[i, at].max() + 16 * (z.abs().max() + most + bias[i, at].abs().max()))
            subnormal = 2.0 ** -25 * vv.abs().sum(0) * w.max()
            tol[i, h] = (2.0 ** -25 + 2.0 ** -11 * out[i, h].abs() + (2.0 ** -11 + 2.0 ** -14) * (A + out[i, h].abs()) + subnormal +
                         2 * e * A + 4 * (len(at) + 40) * U * A)
    return out, tol


def close(got, want, tol):
    got = got.double().cpu()
    assert got.shape == want.shape
    nan = want.isnan()
    assert torch.equal(got.isnan(), nan), (got[got.isnan() != nan][:4], want[got.isnan() != nan][:4])
    bad = ~((got - want).abs() <= tol) & ~nan & ~(want == got)
    assert not bad.any(), (int(bad.sum()), bad.nonzero()[:4], got[bad][:4], want[bad][:4], ((got - want).abs() / tol)[bad][:4])
