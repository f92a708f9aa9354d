"""Calls whose row tiles are shared out in ranges, whole and in parts, and calls that might have shared theirs and do not, against
tests/prompt_reference.py; layouts, repetition and capture of both."""
import math

import numpy as np
import pytest
import torch

from tests import paged_reference as P
from tests import prompt_reference as R
from tests.test_gpu_prompt import DEV, Packed, backward, binding, ctx, forward, host, ints, near, one_like, paged_case, q4  # noqa: F401

pytestmark = pytest.mark.gpu


def to_host(pair):
    return tuple(x.cpu().numpy() for x in pair)


def check(s, lens, out, lse, key, value, grads=None, g=None):
    """All results of a batch; key(b, h) and value(b, h) in 64 bits on the GPU."""
    G = s.Hq // s.H
    for b, L in enumerate(lens):
        me = slice(int(s.start[b]), int(s.start[b + 1]))
        n = me.stop - me.start
        if n == 0:
            continue
        pos = torch.arange(L - n, L, device=DEV)
        for h in range(s.H):
            dk = dv = 0
            for x in range(h * G, h * G + G):
                want = R.dense(s.q[me, x].double(), key(b, h), value(b, h), pos, None if g is None else g[me, x].double())
                what = " of request %d, head %d" % (b, x)
                near(host(out)[me, x], to_host(want["out"]), "out" + what)
                near(host(lse)[x, me], to_host(want["lse"]), "lse" + what)
                if g is not None:
                    near(host(grads)[me, x], to_host(want["dq"]), "dq" + what)
                    dk, dv = dk + np.stack(to_host(want["dk"])), dv + np.stack(to_host(want["dv"]))
            if g is not None:
                for name, t, at in (("dk", dk, s.Hq + h), ("dv", dv, s.Hq + s.H + h)):
                    t[1] += R.U * np.abs(t[0])
                    near(host(grads)[me, at], tuple(t), "%s of request %d, head %d" % (name, b, h))
    lo, hi = int(s.start[0]), int(s.start[-1])
    for t in (out[:lo], out[hi:], lse[:, :lo], lse[:, hi:]):
        assert (t == 7).all(), "rows of no request were written"


def packed(s, x):
    return lambda b, h: x[s.start[b]:s.start[b + 1], h].double()


SHARED = [  # few tiles, the longest longer than a fair share of all
    ([1500], 1, 1, 0, 0),
    ([1290], 2, 1, 3, 1),
    ([1, 1650, 40, 0], 2, 2, 0, 5),
    ([1300, 1290], 3, 3, 0, 0),
    ([2600], 6, 2, 0, 0),
    ([16, 30], 1, 1, 0, 2),     # so few keys that they are one range, which needs no merge
    ([20, 0, 1], 3, 1, 1, 0),
    ([60, 5], 2, 2, 0, 0),
]


@pytest.mark.parametrize("new, q_heads, kv_heads, first, behind", SHARED)
def test_shared_tiles_and_their_gradients(ctx, new, q_heads, kv_heads, first, behind):  # noqa: F811
    s = Packed(71, new, q_heads, kv_heads, first, behind, sharp=1.2)
    out, lse, p, ws = forward(ctx, s)
    g = one_like(s)
    grads = backward(ctx, s, p, out, lse, ws, g)
    check(s, new, out, lse, packed(s, s.k), packed(s, s.v), grads, g)
    lo, hi = int(s.start[0]), int(s.start[-1])
    assert (grads[:lo] == 5).all() and (grads[hi:] == 5).all(), "rows of no request were written"
    again = forward(ctx, s)
    assert torch.equal(again[0], out) and torch.equal(again[1], lse)
    assert torch.equal(backward(ctx, s, p, out, lse, ws, g), grads)


@pytest.mark.parametrize("new, lens, cap, q_heads, kv_heads", [
    ([1], [2500], 2500, 1, 1),
    ([130, 1, 0, 7], [2100, 1500, 30, 7], 4000, 4, 1),   # parts of tiles and whole ones in a range
    ([9] * 40, [1400] * 39 + [5000], 5000, 2, 2),        # more tiles than a head's ranges
    ([5, 3], [40, 64], 9000, 8, 2),                      # might be shared, by the cache's size, and is not
    ([200, 1, 60], [200, 700, 90], 6000, 32, 2),
    ([1] * 256, [1 + 5 * b for b in range(255)] + [3500], 3500, 2, 1),
])
def test_ranges_over_a_cache(ctx, new, lens, cap, q_heads, kv_heads):  # noqa: F811
    s = Packed(72, new, q_heads, kv_heads, 0, 2)
    k, v = (torch.randn((len(new), kv_heads, cap, 128), device=DEV, generator=s.gen).bfloat16() for _ in range(2))
    for b, n in enumerate(lens):
        k[b, :, n:], v[b, :, n:] = math.nan, math.nan
    out, lse, _, _ = forward(ctx, s, ints(lens), k, v)
    check(s, lens, out, lse, lambda b, h: k[b, h, :lens[b]].double(), lambda b, h: v[b, h, :lens[b]].double())


@pytest.mark.parametrize("new, lens, page", [
    ([1, 40], [2700, 3100], 16),
    ([3, 0, 9], [5, 12, 2600], 128),
    ([20] * 5, [100] * 4 + [900], 256),                  # might be shared, by the table's width, and is not
])
def test_ranges_over_the_paged_cache(ctx, new, lens, page):  # noqa: F811
    s, p, table, cache = paged_case(73, new, lens, 6, 2, page, holes=[(len(new) - 1, 1, -1)], behind=1)
    out = q4(ctx, s, p, table, cache, lens)
    for b, n in enumerate(lens):
        if new[b] == 0:
            continue
        slots = P.slots_of(table[b], n, page, p.n_pages)
        there = np.nonzero(slots >= 0)[0]
        pos = np.searchsorted(there, n - new[b] + np.arange(new[b]), side="right") - 1   # (positions among those that are there)
        for h in range(6):
            k, v = (torch.from_numpy(np.ascontiguousarray(x, dtype=np.float64)) for x in cache.rows(slots[there], h // 3))
            me = slice(int(s.start[b]), int(s.start[b + 1]))
            want = R.dense(s.q[me, h].double().cpu(), k, v, torch.from_numpy(pos))["out"]
            near(host(out)[me, h], to_host(want), "out of request %d head %d" % (b, h))
    assert (out[int(s.start[-1]):] == 7).all()


@pytest.mark.parametrize("bad", [math.inf, math.nan])
@pytest.mark.parametrize("at", [0, 700, 1344, 1499])
def test_what_is_not_seen_has_no_influence_on_shared_tiles(ctx, bad, at):  # noqa: F811
    s = Packed(74, [1500], 2, 1, sharp=1.0)
    out, lse, p, ws = forward(ctx, s)
    g = one_like(s)
    clean = backward(ctx, s, p, out, lse, ws, g)
    s.v[at, 0, 3] = bad
    o, l, p, ws = forward(ctx, s)
    assert torch.equal(o[:at], out[:at]) and torch.equal(l, lse) and torch.equal(o[:, :, 4:], out[:, :, 4:])
    assert not torch.isfinite(o[at:, :, 3]).any()
    s.v[at, 0, 3] = 0.5
    s.k[at, 0, 9] = bad
    o, l, p, ws = forward(ctx, s)
    got = backward(ctx, s, p, o, l, ws, g)
    assert torch.equal(got[:at, :2], clean[:at, :2])


@pytest.mark.parametrize("n", [90, 1500])
def test_heads_before_tokens(ctx, n):  # noqa: F811
    """Queries, keys and their gradients as [head][token][128], and rows that lie further apart than they are long."""
    lb = binding()
    s = Packed(75, [n], 4, 2, sharp=1.2)
    g = one_like(s)
    out, lse, p, ws = forward(ctx, s)
    grads = backward(ctx, s, p, out, lse, ws, g)
    store = torch.empty((8, n, 160), dtype=torch.bfloat16, device=DEV)
    rows = store[:, :, :128].transpose(0, 1)
    rows.copy_(s.rows)
    q, k, v = rows.split((4, 2, 2), 1)
    p = lb.make_prompt(1, q, k)
    ws = lb.alloc_prompt_workspace(p)
    o, l = s.outputs()
    ctx.prompt_attn(p, q, k, v, s.d_start, None, o, l, ws)
    assert torch.equal(o, out) and torch.equal(l, lse)
    to = torch.full((8, n, 160), 5.0, dtype=torch.bfloat16, device=DEV)
    dq, dk, dv = to[:, :, :128].transpose(0, 1).split((4, 2, 2), 1)
    ctx.prompt_attn_backward(p, g, q, k, v, o, l, s.d_start, dq, dk, dv, ws)
    torch.cuda.synchronize()
    assert torch.equal(to[:, :, :128].transpose(0, 1), grads) and (to[:, :, 128:] == 5).all()


def test_graphs_of_shared_tiles_with_one_workspace(ctx):  # noqa: F811
    """Two captured graphs, forward and backward, that leave their partials in the same workspace, replayed in turn."""
    cases = []
    for seed, new in ((76, [1500]), (77, [40, 1300, 9])):
        s = Packed(seed, new, 2, 1, sharp=1.2)
        out, lse, p, ws = forward(ctx, s)
        g = one_like(s)
        cases.append([s, g, p, out, lse, backward(ctx, s, p, out, lse, ws, g), ws])
    ws = max((c[-1] for c in cases), key=lambda w: w.numel())
    stream, graphs = torch.cuda.Stream(), []
    for s, g, p, *_ in cases:
        o, l = s.outputs()
        to = torch.full_like(s.rows, 5.0)
        grads = to.split((s.Hq, s.H, s.H), 1)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            ctx.prompt_attn(p, s.q, s.k, s.v, s.d_start, None, o, l, ws)
            ctx.prompt_attn_backward(p, g, s.q, s.k, s.v, o, l, s.d_start, *grads, ws)
        graphs.append((graph, o, l, to))
    for _ in range(3):
        for (graph, o, l, to), (s, g, p, out, lse, want, own) in zip(graphs, cases):
            o.fill_(7), l.fill_(7), to.fill_(5), ws.fill_(0xFF)
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(o, out) and torch.equal(l, lse) and torch.equal(to, want)
            eager, l2, _, _ = forward(ctx, s, workspace=own, p=p)
            assert torch.equal(eager, out) and torch.equal(l2, lse)
