"""Long calls of attention over prompts, whose work is cut into tiles, ranges and pieces, against tests/prompt_norms.py: a block that one of
them left out shows in the norm of a head's 128 rows."""

import pytest
import torch

from tests import paged_reference as P
from tests import prompt_norms as N
from tests.test_gpu_prompt import DEV, Packed, backward, ctx, forward, ints, one_like, paged_case, q4  # noqa: F401

pytestmark = pytest.mark.gpu


def check(s, lens, key, value, out, grads=None, g=None):
    """key(b, h), value(b, h): 64-bit tensors on the GPU; requests of fewer than 64 rows have too few for a norm to say much."""
    G = s.Hq // s.H
    for b, L in enumerate(lens):
        me = slice(int(s.start[b]), int(s.start[b + 1]))
        n = me.stop - me.start
        if n < 64:
            continue
        pos = torch.arange(L - n, L, device=DEV)
        for h in range(s.H):
            parts = []
            for x in range(h * G, h * G + G):
                want = N.head(s.q[me, x].double(), key(b, h), value(b, h), pos, None if g is None else g[me, x].double())
                what = " of request %d, head %d" % (b, x)
                N.near(out[me, x], want["out"], "out" + what)
                if g is not None:
                    N.near(grads[me, x], want["dq"], "dq" + what)
                    parts.append((want["dk"], want["dv"]))
            if g is not None:
                for i, name in enumerate(("dk", "dv")):
                    N.near(grads[me, s.Hq + i * s.H + h], N.whole([p[i] for p in parts]), "%s of request %d, KV head %d" % (name, b, h))


def packed(s, x):
    return lambda b, h: x[s.start[b]:s.start[b + 1], h].double()


@pytest.mark.parametrize("sharp", [0.3, 1.2, 3.0])
@pytest.mark.parametrize("new, q_heads, kv_heads", [
    ([1500], 1, 1),                  # row tiles and key tiles shared out
    ([1, 1650, 40, 0], 2, 2),
    ([1300, 1290], 3, 3),
    ([2600], 6, 2),
    ([3100, 70, 900], 2, 1),
    ([700, 129, 500], 8, 8),         # row tiles a workgroup each
    ([200] * 7, 8, 2),
    ([2100], 16, 1),
    ([65, 130, 999], 10, 2),
])
def test_packed_sequences_and_gradients(ctx, new, q_heads, kv_heads, sharp):  # noqa: F811
    s = Packed(101, new, q_heads, kv_heads, 2, 3, sharp=0.8)
    s.rows[:, :q_heads] = torch.randn((s.T, q_heads, 128), device=DEV, generator=s.gen).mul_(sharp).bfloat16()
    g = one_like(s)
    out, lse, p, ws = forward(ctx, s)
    grads = backward(ctx, s, p, out, lse, ws, g)
    check(s, new, packed(s, s.k), packed(s, s.v), out, grads, g)


@pytest.mark.parametrize("new, lens, cap, q_heads, kv_heads", [
    ([64], [6000], 6000, 4, 1),                          # pieces of keys, merged
    ([130, 1, 0, 70], [2100, 1500, 30, 70], 4000, 4, 1),
    ([90] * 9, [1400] * 8 + [5000], 5000, 2, 2),
    ([200, 1, 64], [200, 700, 90], 6000, 32, 2),         # might be shared, and is not
    ([700], [20000], 20000, 2, 2),
])
def test_pieces_over_a_cache(ctx, new, lens, cap, q_heads, kv_heads):  # noqa: F811
    s = Packed(102, new, q_heads, kv_heads, sharp=1.2)
    k, v = (torch.randn((len(new), kv_heads, cap, 128), device=DEV, generator=s.gen).bfloat16() for _ in range(2))
    out, _, _, _ = forward(ctx, s, ints(lens), k, v)
    check(s, lens, lambda b, h: k[b, h, :lens[b]].double(), lambda b, h: v[b, h, :lens[b]].double(), out)


@pytest.mark.parametrize("new, lens, q_heads, kv_heads, page", [
    ([64], [3000], 2, 1, 64),
    ([200, 1], [700, 2500], 4, 2, 16),
    ([300], [300], 8, 1, 256),
])
def test_pieces_over_the_paged_cache(ctx, new, lens, q_heads, kv_heads, page):  # noqa: F811
    s, p, table, cache = paged_case(103, new, lens, q_heads, kv_heads, page)
    out = q4(ctx, s, p, table, cache, lens)
    rows = {(b, h): [torch.from_numpy(x).to(DEV) for x in cache.rows(P.slots_of(table[b], n, page, p.n_pages), h)]
            for b, n in enumerate(lens) for h in range(kv_heads)}
    check(s, lens, lambda b, h: rows[b, h][0], lambda b, h: rows[b, h][1], out)
