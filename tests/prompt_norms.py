"""How far results of attention over prompts may be off as a whole: the 2-norm over 128 rows of a head, where bounds entry by entry
grow with the sum of all terms' magnitudes and would let a block of them get lost.

A rounding to bf16 is off by a number spread evenly over half a step either way, independent from one number to the next: relative
to numbers whose leading digits are spread as those of products are (density 1 / (m ln 2) for m in [1, 2)), its root mean square is
    r = 2^-8 / sqrt(3) sqrt(integral of 1 / (m^3 ln 2)) = 2^-8 sqrt((3 / 8) / (3 ln 2)) = 0.00166.
What is rounded, and so the expected square of each result's error (squares of matrices entry by entry):
    out    P and out               r^2 (out^2 + P^2 v^2)
    delta  out as above            D_i = sum_d g^2 off(out)^2
    dq     dS, delta and dq        r^2 dq^2 + c^2 (r^2 dS^2 k^2 + D (P k)^2)      (delta's error is one for all keys of a row)
    dk     dS, delta and dk        r^2 dk^2 + c^2 (r^2 dS^2 + D P^2)^T q^2        c = 1 / sqrt(128)
    dv     P and dv                r^2 (dv^2 + (P^2)^T g^2)
Their sum over some thousand entries is near its expectation; the bound is twice its root, and 2^-13 of the result for 32 bits."""
import math

import torch

r = 2.0 ** -8 * math.sqrt(0.375 / (3 * math.log(2)))
ROWS = 128


def head(q, k, v, pos, g=None):
    """(value, expected square of the error) of one query head's out and, with g, dq, dk, dv: 64-bit tensors, rows q at positions pos on keys
    k, v.  Those of dk and dv are without their own rounding, which belongs to the sum over a KV head's query heads (whole)."""
    c = 1 / math.sqrt(q.shape[1])
    seen = torch.arange(len(k), device=q.device) <= pos.view(-1, 1)
    p = torch.where(seen, (q @ k.T) * c, -math.inf)
    p = torch.where(seen, (p - p.logsumexp(1, keepdim=True)).exp(), 0.0)
    out = p @ v
    off = r * r * (out ** 2 + p ** 2 @ v ** 2)
    got = {"out": (out, off)}
    if g is not None:
        ds = p * (g @ v.T - (out * g).sum(1, keepdim=True))
        delta = (g ** 2 * off).sum(1, keepdim=True)
        dq = c * ds @ k
        got["dq"] = (dq, r * r * dq ** 2 + c * c * (r * r * ds ** 2 @ k ** 2 + delta * (p @ k) ** 2))
        got["dk"] = (c * ds.T @ q, c * c * ((r * ds) ** 2 + delta * p ** 2).T @ q ** 2)
        got["dv"] = (p.T @ g, (r * p.T) ** 2 @ g ** 2)
    return got


def whole(parts):
    """dk or dv of a KV head from its query heads' parts."""
    value = sum(x for x, _ in parts)
    return value, sum(y for _, y in parts) + (r * value) ** 2


def near(got, want, what):
    value, off = want
    for at in range(0, len(value), ROWS):
        x, y, z = (t[at:at + ROWS] for t in (got, value, off))
        far, most = (x.double() - y).norm().item(), 2 * math.sqrt(z.sum().item()) + 2.0 ** -13 * y.norm().item()
        assert far <= most, "%s, rows from %d: off by %.3g of %.3g, more than %.3g" % (what, at, far, y.norm().item(), most)
