"""Causal attention over prompts and its gradient in plain 64 bits, one head at a time, with what the calls' results may be off by.

Errors.  U = 2^-8 is the most a rounding to bf16 changes a number by, relative to it; u = 2^-24 that to fp32.
  - A score is a sum of 128 products of exact operands in 32 bits, off by 130 u times the sum of their magnitudes, and its exponent
    is rounded (4 u of it): a weight is off by `each` = that, doubled for the row's maximum or lse, + 2^-20 for exponential,
    logarithm and sums of up to 2^12 terms a lane.
  - out = sum P v: P is rounded to bf16 (U) for the product: off by (U + 2 each) sum P |v| (numerator and denominator), and by U |out|
    for its own rounding.  lse: off by `each` and 4 u of itself.
  - dP - delta: delta is made of the rounded out, so off by sum |g| off(out) + 130 u (sum |g||v| + sum |g||out|).
  - dS = P (dP - delta): off by U |dS| for its rounding, each |dS|, P off(dP - delta).
  - dq, dk: sums of dS times exact numbers: off by sum off(dS) |k|, |q|; dv: by (U + 2 each) sum P |g|; their own rounding U.
  - A sum of n terms in 32 bits: n u of the sum of magnitudes; n below 2^13 here: 2^-11, of which the terms' own order makes a few; the
    matrix units add 16 terms at a time: n / 16 u + 16 u <= 2^-14."""
import math

import numpy as np

D = 128
U, u = 2.0 ** -8, 2.0 ** -24
SUM = 2.0 ** -14


def head(q, k, v, pos, g=None):
    """One query head's rows q [n, 128] at positions pos on keys k, v [L, 128]: a dict of (value, tolerance) of out, lse and, with g, dq,
    dk, dv.  Unseen pairs are left out, whatever they hold."""
    n, L = len(q), len(k)
    out, off_out = np.zeros((n, D)), np.zeros((n, D))
    lse, off_lse = np.full(n, -np.inf), np.zeros(n)
    dq, off_q = np.zeros((n, D)), np.zeros((n, D))
    dk, off_k, dv, off_v = (np.zeros((L, D)) for _ in range(4))
    c = 1 / math.sqrt(D)
    for i in range(n):
        m = min(L, int(pos[i]) + 1)
        if m <= 0:
            continue
        K, V = k[:m], v[:m]
        s = K @ q[i] * c
        lse[i] = np.log(np.exp(s - s.max()).sum()) + s.max()
        p = np.exp(s - lse[i])
        each = 2 * (130 * u * (np.abs(K) @ np.abs(q[i])).max() * c + 4 * u * np.abs(s).max()) + 2.0 ** -20
        out[i] = p @ V
        seen = p @ np.abs(V)
        off_out[i] = U * np.abs(out[i]) + (U + 2 * each + SUM) * seen
        off_lse[i] = each + 4 * u * abs(lse[i]) + 2.0 ** -20
        if g is None:
            continue
        dp, delta = V @ g[i], out[i] @ g[i]
        ds = p * (dp - delta)
        off_dp = np.abs(g[i]) @ off_out[i] + 130 * u * (np.abs(V) @ np.abs(g[i]) + np.abs(g[i]) @ np.abs(out[i]))
        off_ds = (U + each + SUM) * np.abs(ds) + p * off_dp
        dq[i] = c * ds @ K
        off_q[i] = U * np.abs(dq[i]) + c * off_ds @ np.abs(K)
        dk[:m] += c * np.outer(ds, q[i])
        off_k[:m] += c * np.outer(off_ds, np.abs(q[i]))
        dv[:m] += np.outer(p, g[i])
        off_v[:m] += (U + 2 * each + SUM) * np.outer(p, np.abs(g[i]))
    got = {"out": (out, off_out), "lse": (lse, off_lse)}
    if g is not None:
        got.update(dq=(dq, off_q), dk=(dk, off_k), dv=(dv, off_v))
    return got


def prompt(q, k, v, start, lens, g=None):
    """All heads: q [T, H_q, 128], k(b, h) and v(b, h) the keys [lens[b], 128] of request b's KV head h, and the number of KV heads as
    k.heads; gradients of k and v come back by request."""
    T, Hq, _ = q.shape
    H = k.heads
    G = Hq // H
    got = {"out": np.zeros((2, T, Hq, D)), "lse": np.zeros((2, Hq, T))}
    if g is not None:
        got["dq"] = np.zeros((2, T, Hq, D))
        got["dk"] = [np.zeros((2, L, H, D)) for L in lens]
        got["dv"] = [np.zeros((2, L, H, D)) for L in lens]
    for b, L in enumerate(lens):
        lo, hi = start[b], start[b + 1]
        pos = L - (hi - lo) + np.arange(hi - lo)
        for h in range(Hq):
            x = head(q[lo:hi, h], k(b, h // G), v(b, h // G), pos, None if g is None else g[lo:hi, h])
            got["out"][:, lo:hi, h] = x["out"]
            got["lse"][:, h, lo:hi] = x["lse"]
            if g is not None:
                got["dq"][:, lo:hi, h] = x["dq"]
                for name in ("dk", "dv"):
                    got[name][b][:, :, h // G] += x[name]
    if g is not None:
        for name in ("dk", "dv"):  # (the sum's own rounding)
            for x in got[name]:
                x[1] += U * np.abs(x[0])
    return got


class Keys:
    """Keys or values of a request's KV head, of a function (b, h) -> [L, 128]."""

    def __init__(self, heads, of):
        self.heads, self.of = heads, of

    def __call__(self, b, h):
        return self.of(b, h)


def dense(q, k, v, pos, g=None):
    """head() for long requests: the same formulas as products of whole matrices, of 64-bit torch tensors on any device."""
    import torch
    c = 1 / math.sqrt(D)
    m = torch.arange(len(k), device=q.device) <= pos.view(-1, 1)
    s = (q @ k.T) * c
    big = torch.where(m, q.abs() @ k.abs().T, 0.0).amax(1) * c
    each = (2 * (130 * u * big + 4 * u * torch.where(m, s.abs(), 0.0).amax(1)) + 2.0 ** -20).view(-1, 1)
    s = torch.where(m, s, -math.inf)
    lse = s.logsumexp(1)
    p = torch.where(m, (s - lse.view(-1, 1)).exp(), 0.0)
    out, seen = p @ v, p @ v.abs()
    off_out = U * out.abs() + (U + 2 * each + SUM) * seen
    got = {"out": (out, off_out), "lse": (lse, each[:, 0] + 4 * u * lse.abs() + 2.0 ** -20)}
    if g is not None:
        dp, delta = g @ v.T, (out * g).sum(1, keepdim=True)
        ds = p * (dp - delta)
        off_dp = (g.abs() * off_out).sum(1, keepdim=True) + 130 * u * (g.abs() @ v.abs().T + (g.abs() * out.abs()).sum(1, keepdim=True))
        off_ds = torch.where(m, (U + each + SUM) * ds.abs() + p * off_dp, 0.0)
        dq = c * ds @ k
        got["dq"] = (dq, U * dq.abs() + c * off_ds @ k.abs())
        got["dk"] = (c * ds.T @ q, c * off_ds.T @ q.abs())
        got["dv"] = (p.T @ g, ((U + 2 * each + SUM) * p).T @ g.abs())
    return got
