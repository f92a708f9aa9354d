"""Attention over prompts on the GPU against tests/prompt_reference.py, through the C ABI: every call by itself at the sizes and
masks where it can go wrong, then a run of them as serving and training make it."""
import math

import numpy as np
import pytest
import torch

from tests import paged_reference as P
from tests import prompt_reference as R

pytestmark = pytest.mark.gpu
DEV = "cuda"


def binding():
    from paper_2602_04541_amd import binding as lb
    return lb


@pytest.fixture(scope="module")
def ctx():
    c = binding().Context(0)
    yield c
    torch.cuda.synchronize()
    c.close()


def ints(v):
    return torch.as_tensor(np.ascontiguousarray(v), dtype=torch.int32, device=DEV).contiguous()


def host(t):
    return t.detach().double().cpu().numpy()


def starts(new, first=0):
    return first + np.concatenate(([0], np.cumsum(new)))


def near(got, want, what):
    """Within the reference's tolerance; equal where that is no number (infinite or NaN)."""
    value, off = want
    got = np.asarray(got)
    sure = np.isfinite(value) & np.isfinite(off)
    with np.errstate(invalid="ignore"):
        far = np.where(sure, np.abs(got - value) - off - 1e-30, -1.0)
    assert np.isfinite(got[sure]).all(), "%s: %d values are no numbers" % (what, (~np.isfinite(got[sure])).sum())
    assert (far <= 0).all(), "%s: off by %g more than %g at %s" % (what, far.max(), off.flat[far.argmax()], np.unravel_index(far.argmax(), far.shape))
    same = np.isfinite(value) | (got == value) | (np.isnan(got) & np.isnan(value))
    assert same.all(), "%s: %s where %s was expected" % (what, got[~same][:4], value[~same][:4])


class Packed:
    """Packed rows of a fused projection: `first` rows before and `behind` rows behind those of the requests."""

    def __init__(self, seed, new, q_heads, kv_heads, first=0, behind=0, sharp=2.0):
        gen = torch.Generator(DEV)
        gen.manual_seed(seed)
        self.gen, self.new, self.Hq, self.H = gen, list(new), q_heads, kv_heads
        self.start = starts(new, first)
        self.T = int(self.start[-1]) + behind
        self.rows = torch.randn((self.T, q_heads + 2 * kv_heads, 128), device=DEV, generator=gen)
        self.rows[:, :q_heads] *= torch.linspace(0.3, sharp, q_heads, device=DEV).view(1, -1, 1)
        self.rows = self.rows.bfloat16()
        self.q, self.k, self.v = self.rows.split((q_heads, kv_heads, kv_heads), 1)
        self.d_start = ints(self.start)

    def keys(self, x):
        rows = host(x)
        return R.Keys(self.H, lambda b, h: rows[self.start[b]:self.start[b + 1], h])

    def outputs(self):
        out = torch.full((self.T, self.Hq, 128), 7.0, dtype=torch.bfloat16, device=DEV)
        lse = torch.full((self.Hq, self.T), 7.0, device=DEV)
        return out, lse


def forward(ctx, s, lengths=None, k=None, v=None, lse=True, workspace=None, p=None):
    lb = binding()
    k, v = s.k if k is None else k, s.v if v is None else v
    p = p or lb.make_prompt(len(s.new), s.q, k)
    ws = lb.alloc_prompt_workspace(p) if workspace is None else workspace
    ws.fill_(0xFF)
    out, l = s.outputs()
    ctx.prompt_attn(p, s.q, k, v, s.d_start, lengths, out, l if lse else None, ws)
    torch.cuda.synchronize()
    return out, l, p, ws


def check_forward(s, out, lse, keys, values, lens):
    want = R.prompt(host(s.q), keys, values, s.start, lens)
    lo, hi = s.start[0], s.start[-1]
    near(host(out)[lo:hi], want["out"][:, lo:hi], "out")
    near(host(lse)[:, lo:hi], want["lse"][:, :, lo:hi], "lse")
    for t in (host(out)[:lo], host(out)[hi:], host(lse)[:, :lo], host(lse)[:, hi:]):
        assert (t == 7).all(), "rows of no request were written"


PACKED = [
    # new tokens of the requests, query heads, KV heads, rows before, rows behind
    ([1], 1, 1, 0, 0),
    ([2], 4, 1, 0, 3),
    ([77], 8, 2, 0, 0),
    ([63, 64, 65], 2, 2, 0, 0),
    ([0, 33, 0, 1, 32, 31, 0], 8, 2, 5, 9),
    ([129, 0, 1], 3, 3, 0, 1),
    ([40, 127], 5, 1, 2, 0),
    ([17, 3, 50], 16, 2, 0, 2),
    ([9, 41], 32, 2, 0, 0),
    ([300], 4, 2, 0, 0),
    ([1] * 70, 8, 8, 0, 1),
    ([0, 0], 4, 1, 3, 3),
    ([5, 2, 700], 6, 3, 0, 0),
]


@pytest.mark.parametrize("new, q_heads, kv_heads, first, behind", PACKED)
def test_packed_sequences(ctx, new, q_heads, kv_heads, first, behind):
    s = Packed(1, new, q_heads, kv_heads, first, behind)
    out, lse, _, _ = forward(ctx, s)
    check_forward(s, out, lse, s.keys(s.k), s.keys(s.v), new)


@pytest.mark.parametrize("new, lens, q_heads, kv_heads", [
    ([1], [1], 4, 1),
    ([1], [900], 4, 1),                  # a single token over a cache
    ([32], [5000], 8, 2),                # split over the keys
    ([3, 1, 0, 40], [4000, 1, 17, 40], 8, 2),
    ([5, 7], [3, 0], 4, 2),              # fewer keys than query tokens, and none: rows that see nothing
    ([70], [66], 2, 1),
    ([130, 2, 65], [1030, 2500, 64], 4, 4),
    ([1] * 20, list(range(0, 4000, 200)), 5, 1),
    ([2, 9], [2047, 2112], 32, 2),
    ([33], [8200], 1, 1),
])
def test_pieces_over_a_cache(ctx, new, lens, q_heads, kv_heads):
    s = Packed(2, new, q_heads, kv_heads, 1, 2)
    cap = max(lens) + 5
    k, v = (torch.randn((len(new), kv_heads, cap, 128), device=DEV, generator=s.gen).bfloat16() for _ in range(2))
    for b, n in enumerate(lens):  # what lies behind a request's keys is not read as one
        k[b, :, n:], v[b, :, n:] = math.nan, math.nan
    out, lse, _, _ = forward(ctx, s, ints(lens), k, v)
    hk, hv = host(k), host(v)
    check_forward(s, out, lse, R.Keys(kv_heads, lambda b, h: hk[b, h, :lens[b]]), R.Keys(kv_heads, lambda b, h: hv[b, h, :lens[b]]), lens)


def test_a_token_major_cache_and_lengths_out_of_range(ctx):
    s = Packed(3, [4, 6], 4, 2)
    store = torch.randn((2, 2, 100, 2, 128), device=DEV, generator=s.gen).bfloat16()   # [k or v][B][L][H][128]
    k, v = (store[i].transpose(1, 2) for i in range(2))
    out, lse, _, _ = forward(ctx, s, ints([1000, -3]), k, v)                           # clamped to 100 and 0
    hk, hv = host(k), host(v)
    lens = [100, 0]
    check_forward(s, out, lse, R.Keys(2, lambda b, h: hk[b, h, :lens[b]]), R.Keys(2, lambda b, h: hv[b, h, :lens[b]]), lens)


def test_starts_out_of_range_stay_among_the_rows(ctx):
    s = Packed(4, [6, 20], 4, 2, 0, 6)
    s.d_start = ints([-5, 6, 10 ** 6])                                                 # clamped to 0 and 32
    s.start, s.new = np.array([0, 6, 32]), [6, 26]
    out, lse, _, _ = forward(ctx, s)
    check_forward(s, out, lse, s.keys(s.k), s.keys(s.v), [6, 26])


@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
@pytest.mark.parametrize("lens, at", [([100], 70), ([130, 20], 129), ([64], 63), ([200], 64)])
def test_what_is_not_seen_has_no_influence(ctx, bad, lens, at):
    """A key and a value that are no numbers: rows before them are as without, rows behind as the formula has it."""
    s = Packed(5, lens, 8, 2)
    clean, _, _, _ = forward(ctx, s)
    s.v[at, 0, 5], s.v[at, 1, 127] = bad, bad
    out, lse, _, _ = forward(ctx, s)
    hv = host(s.v)
    check_forward(s, out, lse, s.keys(s.k), s.keys(s.v), lens)
    assert np.isnan(hv[at, 0, 5]) or not np.isfinite(host(out)[at:lens[0], :4, 5]).any()
    assert (out[:at] == clean[:at]).all()
    s.k[at, 0] = bad
    out, lse, _, _ = forward(ctx, s)
    assert (out[:at] == clean[:at]).all() and torch.isfinite(lse[:, :at]).all()
    assert (out[lens[0]:] == clean[lens[0]:]).all()


def test_far_apart_scores(ctx):
    """Scores of hundreds, and rows whose largest comes late: the running maximum."""
    s = Packed(6, [190], 4, 1, sharp=30.0)
    s.rows[:, 4] *= (1 + torch.arange(190, device=DEV) / 20).view(-1, 1).bfloat16()
    out, lse, _, _ = forward(ctx, s)
    check_forward(s, out, lse, s.keys(s.k), s.keys(s.v), [190])


# ------------------------------------------------------------------ gradients


def backward(ctx, s, p, out, lse, ws, g):
    grads = torch.full_like(s.rows, 5.0)
    dq, dk, dv = grads.split((s.Hq, s.H, s.H), 1)
    ws.fill_(0xFF)
    ctx.prompt_attn_backward(p, g, s.q, s.k, s.v, out, lse, s.d_start, dq, dk, dv, ws)
    torch.cuda.synchronize()
    return grads


def check_backward(s, grads, g):
    want = R.prompt(host(s.q), s.keys(s.k), s.keys(s.v), s.start, s.new, host(g))
    dq, dk, dv = (host(x) for x in grads.split((s.Hq, s.H, s.H), 1))
    lo, hi = s.start[0], s.start[-1]
    near(dq[lo:hi], want["dq"][:, lo:hi], "dq")
    for b in range(len(s.new)):
        near(dk[s.start[b]:s.start[b + 1]], want["dk"][b], "dk of request %d" % b)
        near(dv[s.start[b]:s.start[b + 1]], want["dv"][b], "dv of request %d" % b)
    assert (grads[:lo] == 5).all() and (grads[hi:] == 5).all(), "rows of no request were written"


def one_like(s):
    return torch.randn((s.T, s.Hq, 128), device=DEV, generator=s.gen).bfloat16()


@pytest.mark.parametrize("new, q_heads, kv_heads, first, behind", PACKED)
def test_gradients(ctx, new, q_heads, kv_heads, first, behind):
    s = Packed(7, new, q_heads, kv_heads, first, behind, sharp=1.2)
    g = one_like(s)
    out, lse, p, ws = forward(ctx, s)
    check_backward(s, backward(ctx, s, p, out, lse, ws, g), g)


@pytest.mark.parametrize("bad", [math.inf, math.nan])
@pytest.mark.parametrize("lens, at", [([100], 70), ([150, 20], 129), ([129], 0)])
def test_gradients_of_what_is_not_seen(ctx, bad, lens, at):
    """An output gradient, a query and a key that are no numbers reach what they are summed into, and nothing else."""
    s = Packed(8, lens, 4, 2, sharp=1.0)
    g = one_like(s)
    out, lse, p, ws = forward(ctx, s)
    clean = backward(ctx, s, p, out, lse, ws, g)
    g[at, 1, 3] = bad                                  # query head 1, of KV head 0
    got = backward(ctx, s, p, out, lse, ws, g)
    dq, dk, dv = got.split((4, 2, 2), 1)
    cq, ck, cv = clean.split((4, 2, 2), 1)
    assert (dq[:at] == cq[:at]).all() and (dq[at + 1:] == cq[at + 1:]).all() and (dq[at, 2:] == cq[at, 2:]).all()
    assert (dk[at + 1:] == ck[at + 1:]).all() and (dv[at + 1:] == cv[at + 1:]).all()        # keys that the row does not see
    assert (dk[:, 1] == ck[:, 1]).all() and (dv[:, 1] == cv[:, 1]).all()
    assert not torch.isfinite(dv[:at + 1, 0, 3]).any() and torch.isfinite(dv[:at + 1, 0, 4]).all()
    # a query and its row of outputs
    g = one_like(s)
    clean = backward(ctx, s, p, out, lse, ws, g)
    s.q[at, 1] = bad
    out, lse, p, ws = forward(ctx, s)
    got = backward(ctx, s, p, out, lse, ws, g)
    assert (got[at + 1:] == clean[at + 1:]).all()
    dq = got[:, :4]
    assert (dq[:at] == clean[:at, :4]).all() and torch.isnan(dq[at, 1]).all()
    # a key
    s = Packed(8, lens, 4, 2, sharp=1.0)
    out, lse, p, ws = forward(ctx, s)
    clean = backward(ctx, s, p, out, lse, ws, g)
    s.k[at, 0, 9] = bad
    out, lse, p, ws = forward(ctx, s)
    got = backward(ctx, s, p, out, lse, ws, g)
    assert (got[:at, :4] == clean[:at, :4]).all()
    assert (got[lens[0]:] == clean[lens[0]:]).all()


def test_gradients_against_differences(ctx):
    """The direction of the gradient: the loss, in 64 bits of the outputs, at inputs moved along it."""
    s = Packed(9, [50, 90], 8, 2, sharp=1.0)
    g = one_like(s)
    out, lse, p, ws = forward(ctx, s)
    grads = host(backward(ctx, s, p, out, lse, ws, g))
    rows, hg = host(s.rows), host(g)

    def loss(x):
        q, k, v = x[:, :8], x[:, 8:10], x[:, 10:]
        part = lambda t: R.Keys(2, lambda b, h: t[s.start[b]:s.start[b + 1], h])  # noqa: E731
        return (R.prompt(q, part(k), part(v), s.start, s.new)["out"][0] * hg).sum()

    d = grads / np.linalg.norm(grads)
    h = 1e-4
    slope = (loss(rows + h * d) - loss(rows - h * d)) / (2 * h)
    # the slope along d is <gradient, d>: the gradient's rounding, independent from entry to entry, hardly turns it; 2^-8 of it at most
    assert abs(slope - np.linalg.norm(grads)) <= 2.0 ** -8 * slope


# ------------------------------------------------------------------ the paged 4-bit cache


def paged_case(seed, new, lens, q_heads, kv_heads, page, holes=(), behind=0):
    lb = binding()
    s = Packed(seed, new, q_heads, kv_heads, 0, behind)
    rng = np.random.default_rng(seed)
    held = [-(-n // page) for n in lens]
    n_pages, width = sum(held) + 3, max(1, max(held) + 1)
    p = lb.make_paged(len(new), q_heads, kv_heads, n_pages, page, width, 1, width + 2)
    table = np.full((len(new), width + 2), -1, np.int32)
    pages = rng.permutation(n_pages)
    for b, n in enumerate(held):
        table[b, :n], pages = pages[:n], pages[n:]
    tiles = n_pages * kv_heads * (page // 16)
    data = rng.integers(0, 256, (tiles, 2176)).astype(np.uint8)
    data[:, 2048:] = rng.integers(125, 128, (tiles, 128))
    for b, e, value in holes:
        table[b, e] = value
    cache = P.Cache(n_pages, page, kv_heads)
    cache.bytes = data
    return s, p, table, cache


def q4(ctx, s, p, table, cache, lens):
    lb = binding()
    out, _ = s.outputs()
    ws = lb.alloc_q4_prompt_workspace(p, s.T)
    ws.fill_(0xFF)
    ctx.q4_prompt_attn(p, s.q, torch.from_numpy(cache.bytes).to(DEV), ints(table), ints(lens), s.d_start, out, ws)
    torch.cuda.synchronize()
    return out


@pytest.mark.parametrize("new, lens, q_heads, kv_heads, page", [
    ([1], [1], 4, 1, 16),
    ([17], [317], 8, 2, 64),
    ([1, 0, 30, 2], [63, 5, 100, 65], 8, 2, 16),
    ([64, 1], [64, 1300], 4, 4, 32),
    ([5], [3000], 16, 2, 256),           # split over the keys
    ([3, 8], [2, 0], 5, 1, 128),         # rows that see nothing
    ([130], [200], 32, 2, 64),
    ([1] * 33, list(range(10, 670, 20)), 8, 8, 16),
])
def test_pieces_over_the_paged_cache(ctx, new, lens, q_heads, kv_heads, page):
    s, p, table, cache = paged_case(11, new, lens, q_heads, kv_heads, page, behind=2)
    out = q4(ctx, s, p, table, cache, lens)
    rows = {(b, h): cache.rows(P.slots_of(table[b], n, page, p.n_pages), h) for b, n in enumerate(lens) for h in range(kv_heads)}
    keys = [R.Keys(kv_heads, lambda b, h, i=i: rows[b, h][i]) for i in range(2)]
    want = R.prompt(host(s.q), *keys, s.start, lens)
    hi = s.start[-1]
    near(host(out)[:hi], want["out"][:, :hi], "out")
    assert (out[hi:] == 7).all()


@pytest.mark.parametrize("page", [16, 64])
def test_absent_pages_are_left_out(ctx, page):
    """Entries that are no page, and scale bytes of NaN in places that are not seen."""
    lens, new = [6 * page + 9, 3 * page], [20, 3 * page]
    s, p, table, cache = paged_case(12, new, lens, 8, 2, page, holes=[(0, 1, -1), (0, 5, 10 ** 9), (1, 0, -7)])
    tail = table[0, 6]
    for tile in range(2 * page // 16):   # of the last page, tokens behind the request's last
        behind = 9 if tile % (page // 16) == 0 else 0
        cache.bytes[tail * (2 * page // 16) + tile, 2048:].reshape(8, 16)[:, behind:] = 255
    out = q4(ctx, s, p, table, cache, lens)
    for b, n in enumerate(lens):
        slots = P.slots_of(table[b], n, page, p.n_pages)
        there = np.nonzero(slots >= 0)[0]
        for h in range(8):
            k, v = cache.rows(slots[there], h // 4)
            pos = np.searchsorted(there, n - new[b] + np.arange(new[b]), side="right") - 1   # (positions among those that are there)
            want = R.head(host(s.q)[s.start[b]:s.start[b + 1], h], k, v, pos)["out"]
            near(host(out)[s.start[b]:s.start[b + 1], h], want, "out of request %d head %d" % (b, h))


def test_values_of_the_paged_cache_that_are_no_numbers(ctx):
    """A group under scale byte 255 is NaN for the rows that see its token, and nothing for the others."""
    lens, new = [100], [60]
    s, p, table, cache = paged_case(13, new, lens, 8, 2, 32)
    clean = q4(ctx, s, p, table, cache, lens)
    t, r = cache._at(P.slots_of(table[0], 100, 32, p.n_pages)[70], 1)
    cache.bytes[t, 2048 + 5 * 16 + r] = 255             # dimensions 32 .. 63 of the value of token 70, KV head 1
    out = q4(ctx, s, p, table, cache, lens)
    assert (out[:30] == clean[:30]).all() and (out[:, :4] == clean[:, :4]).all()
    assert torch.isnan(out[30:, 4:, 32:64]).all()
    assert (out[30:, 4:, :32] == clean[30:, 4:, :32]).all() and (out[30:, 4:, 64:] == clean[30:, 4:, 64:]).all()


# ------------------------------------------------------------------ together


def test_a_prompt_in_pieces_then_decoding(ctx):
    """A serving loop: pieces of two prompts planned, appended and attended to over the 4-bit cache, then single tokens; a piece's
    rows are those of the whole prompt, and a token's those of the decode call."""
    lb = binding()
    page, Hq, H = 32, 8, 2
    p = lb.make_paged(2, Hq, H, 40, page, 12, 1)
    cache = lb.alloc_q4_cache(p)
    lengths, table = torch.zeros(2, dtype=torch.int32, device=DEV), torch.full((2, 12), -1, dtype=torch.int32, device=DEV)
    free, count = torch.arange(40, dtype=torch.int32, device=DEV), ints([40])
    total = 310
    gen = torch.Generator(DEV)
    gen.manual_seed(21)
    rows = torch.randn((2, total, Hq + 2 * H, 128), device=DEV, generator=gen).bfloat16()
    seen = torch.zeros((2, total, Hq, 128), dtype=torch.bfloat16, device=DEV)
    ws = lb.alloc_q4_prompt_workspace(p, 256)
    decode_ws = lb.alloc_paged_workspace(p)
    for new in ([100, 7], [0, 130], [150, 1], [1, 1], [1, 1]):
        n, before = sum(new), lengths.tolist()
        slots, start, status = ints(np.zeros(n)), ints(np.zeros(3)), ints([0])
        ctx.plan_pages(p, lengths, ints(new), table, free, count, None, None, slots, start, status)
        step = torch.cat([rows[b, before[b]:before[b] + new[b]] for b in range(2)])
        q, k, v = step.split((Hq, H, H), 1)
        out = torch.zeros((n, Hq, 128), dtype=torch.bfloat16, device=DEV)
        ctx.q4_append(p, k, v, slots, cache)
        ctx.q4_prompt_attn(p, q, cache, table, lengths, start, out, ws)
        assert int(status) == 0 and lengths.tolist() == [a + b for a, b in zip(before, new)]
        at = 0
        for b in range(2):
            seen[b, before[b]:before[b] + new[b]] = out[at:at + new[b]]
            at += new[b]
        if new == [1, 1]:  # the decode call's single token
            alone = torch.zeros_like(out)
            ctx.q4_decode_attn(p, q.contiguous(), cache, table, lengths, None, None, alone, None, decode_ws)
            # both are within the tolerances of their references: a rounding of the weights (2^-8) and of the outputs (2^-8 each)
            k4, v4 = (torch.zeros((2, H, max(lengths.tolist()), 128), dtype=torch.bfloat16, device=DEV) for _ in range(2))
            ctx.q4_read(p, cache, table, None, lengths, k4, v4)
            size = host(v4.abs().float().amax(2)).repeat(Hq // H, 1)
            assert (np.abs(host(out) - host(alone)) <= 2.0 ** -8 * (2 * np.abs(host(alone)) + size) * 1.02).all()
    # all at once, on the rows that the cache stands for
    lens = lengths.tolist()
    k4, v4 = (torch.zeros((2, H, max(lens), 128), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    ctx.q4_read(p, cache, table, None, lengths, k4, v4)
    q = torch.cat([rows[b, :lens[b], :Hq] for b in range(2)]).contiguous()
    whole = R.prompt(host(q), R.Keys(H, lambda b, h: host(k4[b, h, :lens[b]])), R.Keys(H, lambda b, h: host(v4[b, h, :lens[b]])),
                             [0, lens[0], sum(lens)], lens)["out"]
    near(host(torch.cat([seen[b, :lens[b]] for b in range(2)])), whole, "pieces")
    # and the bf16 call on the same rows as a cache
    s = Packed(1, lens, Hq, H)
    s.q = q
    out, lse, _, _ = forward(ctx, s, lengths, k4, v4)
    near(host(out), whole, "over the bf16 cache")


def test_results_repeat_and_share_no_state(ctx):
    """The same bits again, on another context, with another workspace, and split or not as the launch decides."""
    s = Packed(31, [33, 900], 8, 2, sharp=1.0)
    g = one_like(s)
    out, lse, p, ws = forward(ctx, s)
    grads = backward(ctx, s, p, out, lse, ws, g)
    other = binding().Context(0)
    try:
        for c in (ctx, other):
            again, lse2, _, ws2 = forward(c, s)
            assert (again == out).all() and (lse2 == lse).all()
            assert (backward(c, s, p, out, lse, ws2, g) == grads).all()
            without, _, _, _ = forward(c, s, lse=False)
            assert (without == out).all()
    finally:
        other.close()


def test_captured_and_replayed_between_eager_calls(ctx):
    """A training step and a serving step in graphs that share a workspace each, replayed between eager calls, on other inputs."""
    lb = binding()
    s = Packed(41, [150, 40], 8, 2, sharp=1.0)
    g = one_like(s)
    out, lse, p, ws = forward(ctx, s)
    grads = torch.zeros_like(s.rows)
    dq, dk, dv = grads.split((8, 2, 2), 1)
    t, pg, table, cache = paged_case(42, [9, 1], [1200, 300], 8, 2, 64)
    d_cache, d_table, d_lens = torch.from_numpy(cache.bytes).to(DEV), ints(table), ints([1200, 300])
    out4, ws4 = torch.zeros_like(t.q.contiguous()), lb.alloc_q4_prompt_workspace(pg, t.T)

    def step():
        ctx.prompt_attn(p, s.q, s.k, s.v, s.d_start, None, out, lse, ws)
        ctx.prompt_attn_backward(p, g, s.q, s.k, s.v, out, lse, s.d_start, dq, dk, dv, ws)

    def serve():
        ctx.q4_prompt_attn(pg, t.q, d_cache, d_table, d_lens, t.d_start, out4, ws4)

    graphs = []
    for f in (step, serve, serve):
        f()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            f()
        graphs.append(graph)
    for seed in range(4):
        gen = torch.Generator(DEV)
        gen.manual_seed(seed)
        s.rows.copy_(torch.randn(s.rows.shape, device=DEV, generator=gen).bfloat16())
        t.rows.copy_(torch.randn(t.rows.shape, device=DEV, generator=gen).bfloat16())
        step()
        serve()
        want = [x.clone() for x in (out, lse, grads, out4)]
        torch.cuda.synchronize()
        for x in (out, lse, grads, out4):
            x.fill_(3)
        for graph in graphs:
            graph.replay()
        torch.cuda.synchronize()
        for a, b in zip((out, lse, grads, out4), want):
            assert (a == b).all()


def test_two_streams_at_once(ctx):
    """Calls on two contexts and streams, with workspaces of their own, while other work keeps the device busy."""
    lb = binding()
    both = [Packed(51 + i, [700, 50], 8, 2, sharp=1.0) for i in range(2)]
    gs = [one_like(s) for s in both]
    want = []
    for s, g in zip(both, gs):
        out, lse, p, ws = forward(ctx, s)
        want.append((out, backward(ctx, s, p, out, lse, ws, g)))
    others = [lb.Context(0) for _ in range(2)]
    try:
        streams = [torch.cuda.Stream() for _ in range(2)]
        kept = []
        for s, g, c, stream in zip(both, gs, others, streams):
            p = lb.make_prompt(2, s.q, s.k)
            out, lse = s.outputs()
            grads = torch.full_like(s.rows, 5.0)
            kept.append((out, lse, grads, lb.alloc_prompt_workspace(p), p))
        torch.cuda.synchronize()
        for _ in range(5):
            for s, g, c, stream, (out, lse, grads, ws, p) in zip(both, gs, others, streams, kept):
                with torch.cuda.stream(stream):
                    c.prompt_attn(p, s.q, s.k, s.v, s.d_start, None, out, lse, ws)
                    c.prompt_attn_backward(p, g, s.q, s.k, s.v, out, lse, s.d_start, *grads.split((8, 2, 2), 1), ws)
        torch.cuda.synchronize()
        for (out, grads), (got, _, got_grads, _, _) in zip(want, kept):
            assert (got == out).all() and (got_grads == grads).all()
    finally:
        torch.cuda.synchronize()
        for c in others:
            c.close()


def test_many_tiles_and_long_keys(ctx):
    """Sizes beyond the small cases, against 64 bits on the GPU: more tiles than a launch splits, and a long split row."""
    for new, lens, cached in (([2500, 700], [2500, 700], False), ([40, 3], [30000, 70000], True)):
        s = Packed(61, new, 8, 2, sharp=1.5)
        k = v = None
        if cached:
            k, v = (torch.randn((2, 2, max(lens), 128), device=DEV, generator=s.gen).bfloat16() for _ in range(2))
        out, lse, _, _ = forward(ctx, s, ints(lens) if cached else None, k, v)
        for b in range(2):
            me = slice(s.start[b], s.start[b + 1])
            pos = torch.arange(lens[b] - new[b], lens[b], device=DEV).view(-1, 1)
            for h in range(8):
                K, V = (x[b, h // 4, :lens[b]].double() for x in (k, v)) if cached else (x[me, h // 4].double() for x in (s.k, s.v))
                z = s.q[me, h].double() @ K.T.contiguous() / math.sqrt(128)
                z = torch.where(torch.arange(lens[b], device=DEV) <= pos, z, -math.inf)
                w = z.softmax(1)
                want, seen = w @ V, w @ V.abs()
                # (as in the reference: a rounding of the weights and one of the result; 2^-12 for what 32 bits lose)
                assert ((out[me, h].double() - want).abs() <= 2.0 ** -8 * want.abs() + (2.0 ** -8 + 2.0 ** -12) * seen).all()
                assert ((lse[h, me].double() - z.logsumexp(1)).abs() <= 2.0 ** -16).all()
