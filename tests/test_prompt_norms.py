"""The bounds of tests/prompt_norms.py without a GPU: results rounded as the kernels round pass them, and results that lack some work
do not."""
import math

import pytest
import torch

from tests import prompt_norms as N

C = 1 / math.sqrt(128)


def rounded(x):
    return x.to(torch.bfloat16).double()


def inputs(n, heads, sharp):
    gen = torch.Generator().manual_seed(n + heads)
    q, g = (rounded(torch.randn((heads, n, 128), dtype=torch.float64, generator=gen)) for _ in range(2))
    k, v = (rounded(torch.randn((n, 128), dtype=torch.float64, generator=gen)) for _ in range(2))
    return rounded(q * sharp), k, v, g, torch.arange(n)


def results(q, k, v, g, pos, lost=None):
    """What the kernels make of one KV head, in 64 bits but for the roundings to bf16; `lost`: a (rows, keys) block of pairs that is left
    out of the sums called so."""
    seen = torch.arange(len(k)) <= pos.view(-1, 1)
    got = {"out": [], "dq": [], "dk": 0, "dv": 0}
    for h in range(len(q)):
        s = torch.where(seen, q[h] @ k.T * C, -math.inf)
        lse = s.logsumexp(1, keepdim=True)
        p = torch.where(seen, (s - lse).exp(), 0.0)
        m = s.amax(1, keepdim=True)
        w = rounded(torch.where(seen, (s - m).exp(), 0.0))     # (as the forward pass measures them)
        left = {name: torch.ones_like(p) for name in got}
        if lost is not None:
            left[lost[0]][lost[1], lost[2]] = 0
        out = rounded((w * left["out"]) @ v * (m - lse).exp())
        ds = rounded(p * (g[h] @ v.T - (out * g[h]).sum(1, keepdim=True)))
        got["out"].append(out)
        got["dq"].append(rounded(C * (ds * left["dq"]) @ k))
        got["dk"] = got["dk"] + C * (ds * left["dk"]).T @ q[h]
        got["dv"] = got["dv"] + (rounded(p) * left["dv"]).T @ g[h]
    return dict(got, dk=rounded(got["dk"]), dv=rounded(got["dv"]))


def check(got, q, k, v, g, pos, names=("out", "dq", "dk", "dv")):
    want = [N.head(q[h], k, v, pos, g[h]) for h in range(len(q))]
    for name in names:
        if name in ("dk", "dv"):
            N.near(got[name], N.whole([w[name] for w in want]), name)
        else:
            for h, w in enumerate(want):
                N.near(got[name][h], w[name], "%s of head %d" % (name, h))


@pytest.mark.parametrize("n, heads, sharp", [(128, 1, 1.0), (300, 4, 0.3), (700, 2, 1.2), (1500, 1, 0.3), (1500, 1, 3.0)])
def test_rounded_results_pass(n, heads, sharp):
    x = inputs(n, heads, sharp)
    check(results(*x), *x)


@pytest.mark.parametrize("n, heads, sharp", [(700, 2, 1.2), (1500, 1, 0.3), (1500, 1, 3.0)])
@pytest.mark.parametrize("name", ["out", "dq", "dk", "dv"])
def test_a_lost_block_is_seen(n, heads, sharp, name):
    """64 keys that 64 rows near the end lack, wherever they lie; 64 rows that some keys lack."""
    x = inputs(n, heads, sharp)
    rows = slice(n - 100, n - 36)
    for first in range(0, n - 200, 192):
        with pytest.raises(AssertionError, match="off by"):
            check(results(*x, lost=(name, rows, slice(first, first + 64))), *x, names=(name,))


@pytest.mark.parametrize("name", ["out", "dq", "dk", "dv"])
def test_a_wrong_factor_is_seen(name):
    x = inputs(700, 2, 1.2)
    got = results(*x)
    got[name] = [1.03 * t for t in got[name]] if isinstance(got[name], list) else 1.03 * got[name]
    with pytest.raises(AssertionError, match="off by"):
        check(got, *x, names=(name,))
