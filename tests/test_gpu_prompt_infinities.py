"""Attention over prompts where scores or values are infinite: rows whose every score is -infinity are NaN and not those that see nothing,
and an infinite value that a row sees reaches its output however small its weight, whole, rescaled or merged."""
import math

import numpy as np
import pytest
import torch

from tests import paged_reference as P
from tests import prompt_reference as R
from tests.test_gpu_prompt import DEV, Packed, backward, check_forward, ctx, forward, host, ints, near, one_like, paged_case, q4  # noqa: F401

pytestmark = pytest.mark.gpu


def nothing_but_minus_infinity(out, lse, rows, heads):
    assert torch.isnan(out[rows, heads]).all(), "rows whose scores are all -infinity"
    assert (lse[heads, rows] == -math.inf).all()


@pytest.mark.parametrize("n", [1, 50, 64, 130, 1500])
def test_scores_that_are_all_minus_infinity(ctx, n):  # noqa: F811
    """The last token's query is infinite in a dimension in which all keys are negative; one head of a KV head's two."""
    s = Packed(81, [n, 9], 2, 1, 1, 1)
    s.k[:, :, 7] = -s.k[:, :, 7].abs() - 0.5
    clean, clean_lse, _, _ = forward(ctx, s)
    s.q[n, 1, 7] = math.inf
    out, lse, _, _ = forward(ctx, s)
    nothing_but_minus_infinity(out, lse, n, 1)
    out[n, 1], lse[1, n] = clean[n, 1], clean_lse[1, n]
    assert torch.equal(out, clean) and torch.equal(lse, clean_lse)


def test_rows_that_see_nothing_are_zero_whatever_their_query(ctx):  # noqa: F811
    s = Packed(82, [7, 70, 3], 4, 2)
    lens = [3, 66, 0]
    k, v = (torch.randn((3, 2, 70, 128), device=DEV, generator=s.gen).bfloat16() for _ in range(2))
    k[..., 7] = -k[..., 7].abs() - 0.5
    s.q[:, :, 7] = math.inf
    out, lse, _, _ = forward(ctx, s, ints(lens), k, v)
    for b, n in enumerate(lens):
        first, new = int(s.start[b]), s.new[b]
        unseen = slice(first, first + new - n)
        assert (out[unseen] == 0).all() and (lse[:, unseen] == -math.inf).all()
        nothing_but_minus_infinity(out, lse, slice(first + new - n, first + new), slice(0, 4))


@pytest.mark.parametrize("length", [60, 200, 5000])
def test_scores_of_minus_infinity_among_others(ctx, length):  # noqa: F811
    """Keys whose scores are -infinity have no weight, also where a row's first blocks hold no others."""
    s = Packed(83, [3], 2, 1)
    k, v = (torch.randn((1, 1, length, 128), device=DEV, generator=s.gen).bfloat16() for _ in range(2))
    s.q[:, :, 5] = s.q[:, :, 5].abs() + 0.5
    gone = torch.arange(length, device=DEV) < length - 17
    gone[::11] = True
    k[0, 0, gone, 5] = -math.inf
    out, lse, _, _ = forward(ctx, s, ints([length]), k, v)
    there = torch.nonzero(~gone).flatten()
    K, V = host(k[0, 0, there]), host(v[0, 0, there])
    for h in range(2):
        pos = np.searchsorted(there.cpu().numpy(), length - 3 + np.arange(3), side="right") - 1   # (positions among the others)
        want = R.head(host(s.q[:, h]), K, V, pos)
        near(host(out[:, h]), want["out"], "out of head %d" % h)
        near(host(lse[h]), want["lse"], "lse of head %d" % h)


def test_minus_infinity_over_the_paged_cache(ctx):  # noqa: F811
    """The same, a token and its neighbours; and where a row's every page is absent it sees nothing."""
    lens, new = [100, 2500, 40], [4, 3, 2]
    s, p, table, cache = paged_case(84, new, lens, 4, 2, 16)
    cache.bytes[:, 3:2048:128] = (cache.bytes[:, 3:2048:128] & 0x0F) | 0xA0    # dimension 7 of every key: -1 times its scale
    table[2] = -1
    clean = q4(ctx, s, p, table, cache, lens)
    s.q[:, :, 7] = math.inf
    s.q[5, 2:, 7] = 1.0
    ordinary = q4(ctx, s, p, table, cache, lens)
    assert torch.isnan(ordinary[:5]).all() and torch.isnan(ordinary[6]).all() and torch.isnan(ordinary[5, :2]).all()
    assert torch.isfinite(ordinary[5, 2:]).all()
    assert (ordinary[7:] == 0).all() and (clean[7:] == 0).all()


@pytest.mark.parametrize("there", [0, 13, 150, 373])
def test_minus_infinity_in_one_of_many_pieces(ctx, there):  # noqa: F811
    """Rows over 6000 tokens of which a single page is there: merged from more than 16 pieces, of which one sees a key."""
    s, p, table, cache = paged_case(88, [3], [6000], 1, 1, 16)
    cache.bytes[:, 3:2048:128] = (cache.bytes[:, 3:2048:128] & 0x0F) | 0xA0
    kept = table[0, there]
    table[0, :] = -1
    s.q[:, :, 7] = math.inf
    assert (q4(ctx, s, p, table, cache, [6000]) == 0).all()
    table[0, there] = kept
    assert torch.isnan(q4(ctx, s, p, table, cache, [6000])).all()


@pytest.mark.parametrize("new, length, absent", [(20, 20, [0]), (70, 130, [4, 5]), (40, 40, [1]), (3, 300, range(18)), (3, 300, range(19))])
def test_rows_that_see_no_page_among_others(ctx, new, length, absent):  # noqa: F811
    """Of a block's rows those before its first page are zero, and the others, whose scores are all -infinity, NaN."""
    s, p, table, cache = paged_case(91, [new], [length], 2, 1, 16)
    cache.bytes[:, 3:2048:128] = (cache.bytes[:, 3:2048:128] & 0x0F) | 0xA0
    table[0, list(absent)] = -1
    s.q[:, :, 7] = math.inf
    out = q4(ctx, s, p, table, cache, [length])
    there = np.nonzero(P.slots_of(table[0], length, 16, p.n_pages) >= 0)[0]
    sees = torch.from_numpy(length - new + np.arange(new) >= (there[0] if len(there) else length)).to(DEV)
    assert torch.isnan(out[sees]).all() and (out[~sees] == 0).all()


def steep(s, k, low, high):
    """Queries and keys whose scores rise along the keys: low nats for the first, high for the last (rounded to bf16)."""
    root = math.sqrt(128)
    s.q[:, :, 0] = 16.0
    n = k.shape[-2]
    k[..., 0] = (torch.linspace(low, high, n, device=DEV) * root / 16).bfloat16()


@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
@pytest.mark.parametrize("new, length", [(3, 60), (3, 200), (70, 700), (2, 6000)])
def test_infinite_values_of_small_weight(ctx, bad, new, length):  # noqa: F811
    """Weights from e^-600 on: zero in 32 bits, not in the formula.  Rescaled within a range (from 65 keys on) and merged (6000)."""
    s = Packed(85, [new], 2, 1, sharp=0.3)
    k, v = (torch.randn((1, 1, length, 128), device=DEV, generator=s.gen).bfloat16() for _ in range(2))
    steep(s, k, -300.0, 300.0)
    v[0, 0, 2, 9] = bad
    v[0, 0, length - new - 1, 40] = bad
    out, lse, _, _ = forward(ctx, s, ints([length]), k, v)
    check_forward(s, out, lse, R.Keys(1, lambda b, h: host(k[b, h])), R.Keys(1, lambda b, h: host(v[b, h])), [length])


def test_infinite_values_of_both_signs(ctx):  # noqa: F811
    s = Packed(86, [300], 1, 1, sharp=0.3)
    steep(s, s.rows[:, 1:2].transpose(0, 1), -300.0, 300.0)
    s.v[2, 0, 9], s.v[200, 0, 9] = math.inf, -math.inf
    out, lse, _, _ = forward(ctx, s)
    check_forward(s, out, lse, s.keys(s.k), s.keys(s.v), [300])
    assert (out[2:200, 0, 9] == math.inf).all() and torch.isnan(out[200:, 0, 9]).all()


def test_infinite_values_of_small_weight_in_the_paged_cache(ctx):  # noqa: F811
    """A group under scale byte 255, which is NaN."""
    lens, new = [2600], [2]
    s, p, table, cache = paged_case(87, new, lens, 2, 1, 32)
    s.q[:] = 0
    s.q[:, :, 0] = 16.0
    slots = P.slots_of(table[0], 2600, 32, p.n_pages)
    for t in range(2600):   # dimension 0 of the key: 6 times the scale, the scale's sign and size along the keys
        tile, r = cache._at(slots[t], 0)
        cache.bytes[tile, r * 128] = (cache.bytes[tile, r * 128] & 0xF0) | (0xF if t < 1300 else 0x7)
        cache.bytes[tile, 2048 + r] = 127 + (5 if 100 < t < 2500 else 6)
    tile, r = cache._at(slots[10], 0)
    cache.bytes[tile, 2048 + 5 * 16 + r] = 255
    out = q4(ctx, s, p, table, cache, lens)
    assert torch.isnan(out[:, :, 32:64]).all()
    k, v = cache.rows(slots, 0)
    want = R.prompt(host(s.q), R.Keys(1, lambda b, h: k), R.Keys(1, lambda b, h: v), s.start, lens)["out"]
    near(host(out)[..., :32], want[..., :32], "out")
    near(host(out)[..., 64:], want[..., 64:], "out")


@pytest.mark.parametrize("n", [90, 1500])
def test_gradients_of_rows_whose_scores_are_all_minus_infinity(ctx, n):  # noqa: F811
    """Such a row has no gradient (NaN), and neither have the keys that it sees; other heads and requests keep theirs."""
    s = Packed(89, [n, 70], 4, 2, sharp=1.2)
    s.k[:, :, 7] = -s.k[:, :, 7].abs() - 0.5
    g = one_like(s)
    out, lse, p, ws = forward(ctx, s)
    clean = backward(ctx, s, p, out, lse, ws, g)
    at = n // 2
    s.q[at, 1, 7] = math.inf
    out, lse, p, ws = forward(ctx, s)
    got = backward(ctx, s, p, out, lse, ws, g)
    (dq, dk, dv), (cq, ck, cv) = (x.split((4, 2, 2), 1) for x in (got, clean))
    assert torch.isnan(dq[at, 1]).all()
    dq[at, 1] = cq[at, 1]
    assert torch.equal(dq, cq)
    for x, y in ((dk, ck), (dv, cv)):
        assert torch.isnan(x[:at + 1, 0]).all()
        assert torch.equal(x[at + 1:], y[at + 1:]) and torch.equal(x[:, 1], y[:, 1])


@pytest.mark.parametrize("n, at", [(90, 10), (90, 64), (200, 3), (1500, 700)])
def test_gradients_of_keys_whose_scores_are_minus_infinity(ctx, n, at):  # noqa: F811
    """A key with an infinity has no weight and no gradient; for the rows that see it, dq is 0 times infinity there, which is NaN, and as
    without the key elsewhere."""
    s = Packed(90, [n], 2, 1, sharp=1.2)
    s.q[:, :, 9] = s.q[:, :, 9].abs() + 0.5
    s.k[at, 0, 9] = -math.inf
    g = one_like(s)
    out, lse, p, ws = forward(ctx, s)
    got = backward(ctx, s, p, out, lse, ws, g)
    dq, dk, dv = (host(x) for x in got.split((2, 1, 1), 1))
    assert np.isfinite(dq[:at]).all() and np.isnan(dq[at:, :, 9]).all()
    assert (dk[at] == 0).all() and (dv[at] == 0).all()
    others = np.arange(n) != at
    K, V = (x[:, 0].double()[torch.from_numpy(others).to(DEV)] for x in (s.k, s.v))
    pos = torch.arange(n, device=DEV) - (torch.arange(n, device=DEV) >= at).long()    # (positions among the others)
    dims = np.arange(128) != 9
    wk = wv = 0
    for h in range(2):
        want = R.dense(s.q[:, h].double(), K, V, pos, g[:, h].double())
        value, off = (x.cpu().numpy() for x in want["dq"])
        near(dq[:, h][:, dims], (value[:, dims], off[:, dims]), "dq of head %d" % h)
        near(dq[:at, h], (value[:at], off[:at]), "dq of head %d" % h)
        wk, wv = (a + np.stack([x.cpu().numpy() for x in want[name]]) for a, name in ((wk, "dk"), (wv, "dv")))
    for name, got, want in (("dk", dk, wk), ("dv", dv, wv)):
        want[1] += R.U * np.abs(want[0])
        near(got[others, 0], tuple(want), name)
