"""The paged 4-bit cache on the GPU against tests/paged_reference.py, through the C ABI: every call by itself at the sizes
where it can go wrong, then a run of them as a serving loop makes it."""
import numpy as np
import pytest
import torch

from tests import paged_reference as R

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


def bf16(x):
    """float64 values that bf16 holds, as a tensor on the GPU."""
    return torch.from_numpy(R.to_bf16_bits(x).view(np.int16)).view(torch.bfloat16).to(DEV)


def host(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


def draw(rng, shape, spread=1.0):
    """Normal values that bf16 holds."""
    return R.from_bf16_bits(R.to_bf16_bits(rng.standard_normal(shape) * spread))


class Made:
    """A cache with every request's tokens in pages of a shuffled pool; what no token lies in is `fill` bytes."""

    def __init__(self, seed, lens, q_heads, kv_heads, page, k=1, fill=0xFF, max_pages=None, page_tiles=0, spread=1.0, extra=3):
        lb = binding()
        self.rng = rng = np.random.default_rng(seed)
        self.lens = np.asarray(lens, np.int32)
        B = len(lens)
        held = -(-self.lens // page)
        self.max_pages = max_pages or max(1, int(held.max()) + 1)
        n_pages = int(held.sum()) + extra
        self.p = lb.make_paged(B, q_heads, kv_heads, n_pages, page, self.max_pages, k, self.max_pages + 2, page_tiles)
        self.table = np.full((B, self.max_pages + 2), -1, np.int32)
        pages = rng.permutation(n_pages)
        for b in range(B):
            self.table[b, :held[b]], pages = pages[:held[b]], pages[held[b]:]
        self.ref = R.Cache(n_pages, page, kv_heads, self.p.page_tiles, fill)
        # (codes and scales drawn at random: every code, scales of a few binades)
        for b in range(B):
            slots = R.slots_of(self.table[b], self.lens[b], page, n_pages)
            for g in range(kv_heads):
                for s in slots:
                    kv = [(rng.integers(0, 16, 128).astype(np.uint8), rng.integers(125, 128, 4).astype(np.uint8)) for _ in range(2)]
                    self.ref.write(s, g, *kv)
        self.q = draw(rng, (B, q_heads, 128), spread)
        self.cache = torch.from_numpy(self.ref.bytes).to(DEV)
        self.ws = lb.alloc_paged_workspace(self.p)

    def sets(self, k, kind="full"):
        """Sets of k entries: distinct positions, ascending, -1 behind them; or with entries that have to be ignored."""
        B, H = self.p.batch, self.p.n_kv_heads
        out = np.full((B, H, k), -1, np.int32)
        for b in range(B):
            for g in range(H):
                n = min(k, int(self.lens[b]))
                if kind == "short":
                    n = self.rng.integers(0, n + 1)
                at = np.sort(self.rng.permutation(int(self.lens[b]))[:n])
                out[b, g, :n] = at
                if kind == "wild" and n:
                    junk = self.rng.permutation(n)[:max(1, n // 3)]
                    out[b, g, junk] = self.rng.choice([-1, -7, int(self.lens[b]), 1 << 30, -(1 << 31)], len(junk))
        return out


def check_attn(ctx, m, mask=None, idx=None, scores=False, table=None, lens=None, stream=None):
    """Runs the attention on `m` and compares outputs and scores with the reference, element by element."""
    p, G, B, H = m.p, m.p.n_q_heads // m.p.n_kv_heads, m.p.batch, m.p.n_kv_heads
    table = m.table if table is None else table
    lens = m.lens if lens is None else lens
    out = torch.full((B, p.n_q_heads, 128), 7.5, dtype=torch.bfloat16, device=DEV)
    sc = torch.full((B, H, m.max_pages * p.page_size), 9.25, device=DEV) if scores else None
    d = dict(q=bf16(m.q), table=ints(table), lens=ints(lens), idx=None if idx is None else ints(idx))
    torch.cuda.synchronize()
    ctx.q4_decode_attn(p, d["q"], m.cache, d["table"], d["lens"], mask, d["idx"], out, sc, m.ws, stream=stream)
    torch.cuda.synchronize()
    got, types = host(out), np.ones(p.n_q_heads, np.uint8) if mask is None else mask
    gsc = sc.cpu().numpy() if scores else None
    for b in range(B):
        L = int(np.clip(lens[b], 0, m.max_pages * p.page_size))
        slots = R.slots_of(table[b], L, p.page_size, p.n_pages)
        for g in range(H):
            k, v = m.ref.rows(slots, g)
            heads = np.arange(g * G, (g + 1) * G)
            dense, sparse = heads[types[heads] == 1], heads[types[heads] == 0]
            for hs, rows in ((dense, np.nonzero(slots >= 0)[0]), (sparse, None)):
                if not len(hs):
                    continue
                if rows is None:
                    e = idx[b, g, :min(p.k, L)].astype(np.int64)
                    e = e[(e >= 0) & (e < L)]
                    rows = e[slots[e] >= 0]
                want, off, s, s_off = R.attend(m.q[b, hs], k[rows], v[rows])
                err = np.abs(got[b, hs] - want)
                assert (err <= off + 1e-30).all(), (b, g, hs, L, err.max(), off[np.unravel_index(err.argmax(), err.shape)])
                if scores and hs is dense:
                    full = np.full(L, -np.inf)
                    full[rows] = s.mean(0)
                    far = np.zeros(L)
                    far[rows] = s_off.mean(0) + 2.0 ** -22 * np.abs(s).max(0)
                    x = gsc[b, g].astype(np.float64)
                    fine = np.isfinite(full)
                    assert (x[:L][~fine] == -np.inf).all()
                    assert (np.abs(x[:L][fine] - full[fine]) <= far[fine] + 1e-30).all(), (b, g, np.abs(x[:L][fine] - full[fine]).max())
            if scores:
                assert (gsc[b, g, L if len(dense) else 0:] == 9.25).all()
    return got, gsc


# ------------------------------------------------------------------ append and read


@pytest.mark.parametrize("page,heads,tokens,tiles", [(16, 1, 1, 0), (16, 3, 37, 0), (64, 8, 65, 0), (128, 2, 300, 40), (256, 5, 129, 0), (32, 64, 9, 0)])
def test_append_writes_what_the_reference_writes(ctx, page, heads, tokens, tiles):
    lb = binding()
    rng = np.random.default_rng(tokens)
    n_pages = -(-tokens // page) + 2
    p = lb.make_paged(1, heads, heads, n_pages, page, 4, page_tiles=tiles)
    slots = rng.permutation(n_pages * page)[:tokens].astype(np.int32)
    skipped = np.arange(tokens) % 7 == 3
    slots[skipped] = rng.choice([-1, -5, n_pages * page, 2 ** 31 - 1, -2 ** 31], int(skipped.sum()))
    kv = draw(rng, (tokens, 2, heads, 128)) * 2.0 ** rng.integers(-6, 7, (tokens, 2, heads, 1))  # strides of a fused projection
    kv[:, :, :, 40] *= 16
    ref = R.Cache(n_pages, page, heads, tiles, 0xA5)
    for i, s in enumerate(slots):
        if not skipped[i]:
            for g in range(heads):
                codes = [R.quantise(kv[i, j, g][None]) for j in range(2)]
                ref.write(s, g, *[(c[0][0], c[1][0]) for c in codes])
    cache = torch.full((n_pages, p.page_tiles * 2176), 0xA5, dtype=torch.uint8, device=DEV)
    t = bf16(kv)
    ctx.q4_append(p, t[:, 0], t[:, 1], ints(slots), cache)
    got = cache.cpu().numpy().reshape(ref.bytes.shape)
    assert (got == ref.bytes).all(), np.argwhere(got != ref.bytes)[:5]


def test_append_of_extreme_values(ctx):
    lb = binding()
    rows = np.zeros((13, 128))
    tiny, big = 2.0 ** -133, 3.3895313892515355e38
    rows[1, :4] = [tiny, -tiny, 2.0 ** -127, -2.0 ** -126]      # subnormal: below the smallest scale's half step, and at it
    rows[2, 0], rows[2, 32], rows[2, 64] = big, -big, 1.5 * 2.0 ** 127
    rows[3, :] = -0.0
    rows[4, 5], rows[5, 37], rows[6, 70] = np.inf, -np.inf, np.nan
    rows[7, :8] = [6, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5]        # ties
    rows[8, :8] = [-6, -0.25, -0.75, -1.25, -1.75, -2.5, -3.5, -5]
    rows[9, 0], rows[9, 1] = 2.0 ** 127, 1.0                    # far apart in one group
    rows[10, :] = 1.5 * 2.0 ** -120                             # 6 * 2^-122 exactly
    rows[11, :] = 1.5078125 * 2.0 ** -120                       # the next number: a larger scale
    rows[12, 96:] = 2.0 ** -124                                 # near the smallest scale
    p = lb.make_paged(1, 1, 1, 1, 16, 1)
    cache = torch.zeros((1, 2176), dtype=torch.uint8, device=DEV)
    with np.errstate(invalid="ignore"):
        k = torch.from_numpy(R.to_bf16_bits(rows).view(np.int16)).view(torch.bfloat16).to(DEV)
    k = torch.where(torch.from_numpy(np.isnan(rows)).to(DEV), float("nan"), k)
    v = k.flip(0)
    ctx.q4_append(p, k.unsqueeze(1), v.unsqueeze(1), ints(np.arange(13)), cache)
    out = torch.full((2, 1, 1, 16, 128), 3.0, dtype=torch.bfloat16, device=DEV)
    ctx.q4_read(p, cache, ints([[0]]), None, ints([13]), out[0], out[1])
    want = R.dequantise(*R.quantise(rows))
    for got, w in ((host(out[0])[0, 0], want), (host(out[1])[0, 0], want[::-1])):
        assert np.array_equal(got[:13], w, equal_nan=True), np.argwhere(~((got[:13] == w) | np.isnan(w)))[:5]
        assert (got[13:] == 3.0).all()


def test_every_bf16_number_is_rounded_like_the_reference(ctx):
    lb = binding()
    bits = np.arange(65536, dtype=np.uint16).reshape(512, 128)
    x = R.from_bf16_bits(bits)
    p = lb.make_paged(1, 1, 1, 32, 16, 32)
    cache = lb.alloc_q4_cache(p)
    t = torch.from_numpy(bits.view(np.int16)).view(torch.bfloat16).to(DEV).view(512, 1, 128)
    ctx.q4_append(p, t, t, ints(np.arange(512)), cache)
    out = torch.zeros((2, 1, 1, 512, 128), dtype=torch.bfloat16, device=DEV)
    ctx.q4_read(p, cache, ints(np.arange(32)[None]), None, ints([512]), out[0], out[1])
    want = R.dequantise(*R.quantise(x))
    assert np.array_equal(host(out[0])[0, 0], want, equal_nan=True) and np.array_equal(host(out[1])[0, 0], want, equal_nan=True)


@pytest.mark.parametrize("page,heads,lens,first", [(16, 1, [1], None), (64, 2, [0, 5, 130], None), (32, 3, [100, 33, 64], [7, 33, 63]),
                                                   (256, 2, [600], [255]), (128, 1, [40, 41], [41, 60])])
def test_read(ctx, page, heads, lens, first):
    m = Made(3, lens, heads, heads, page)
    table = m.table.copy()
    if len(lens) == 3:
        table[2, 0] = m.p.n_pages  # no page: zeros
    n = max(1, max(lens) - 3)      # fewer rows than the longest has
    out = torch.full((2, len(lens), heads, n + 2, 136), -2.0, dtype=torch.bfloat16, device=DEV)[..., :128]
    ctx.q4_read(m.p, m.cache, ints(table), None if first is None else ints(first), ints(lens), out[0][:, :, :n], out[1][:, :, :n])
    got = host(out)
    for b, L in enumerate(lens):
        f = 0 if first is None else first[b]
        slots = R.slots_of(table[b], L, page, m.p.n_pages)[f:][:n]
        for g in range(heads):
            want = m.ref.rows(slots, g)
            assert (got[:, b, g, :len(slots)] == want).all() and (got[:, b, g, len(slots):] == -2.0).all()


def test_read_clamps_lengths_to_the_table(ctx):
    m = Made(4, [32], 1, 1, 16, max_pages=2)
    out = torch.zeros((2, 1, 1, 50, 128), dtype=torch.bfloat16, device=DEV)
    ctx.q4_read(m.p, m.cache, ints(m.table), ints([-9]), ints([2 ** 31 - 1]), out[0], out[1])
    want = m.ref.rows(R.slots_of(m.table[0], 32, 16, m.p.n_pages), 0)
    assert (host(out)[:, 0, 0, :32] == want).all() and (host(out)[:, 0, 0, 32:] == 0).all()


# ------------------------------------------------------------------ pages


def run_plan(ctx, p, lengths, new, table, free, count, n_slots, in_place):
    lb = binding()
    d = dict(l=ints(lengths), n=ints(new), t=ints(table), f=ints(free), c=ints([count]))
    o = dict(l=d["l"] if in_place else ints(np.zeros(len(lengths))), c=d["c"] if in_place else ints([0]))
    slots, start, status = ints(np.full(n_slots, 77)), ints(np.full(len(lengths) + 1, 77)), ints([77])
    ctx.plan_pages(p, d["l"], d["n"], d["t"], d["f"], d["c"], None if in_place else o["l"], None if in_place else o["c"], slots, start, status)
    n = lambda t: t.cpu().numpy()  # noqa: E731
    return n(o["l"]), n(o["c"])[0], n(d["t"]), n(slots), n(start), n(status)[0]


@pytest.mark.parametrize("batch,page,in_place", [(1, 16, True), (3, 64, False), (17, 16, True), (256, 32, True), (255, 256, False)])
def test_steps_of_a_serving_loop_are_planned_like_the_reference(ctx, batch, page, in_place):
    lb = binding()
    rng = np.random.default_rng(batch)
    max_pages, n_pages = 9, batch * 2 + 3
    p = lb.make_paged(batch, 1, 1, n_pages, page, max_pages, table_stride=max_pages + 1)
    lengths, table = np.zeros(batch, np.int64), np.full((batch, max_pages + 1), -1, np.int32)
    pool = R.Pool(rng.permutation(n_pages), page, max_pages, n_pages)
    stack = np.full(n_pages, -1, np.int32)
    short = 0
    for step in range(12):
        stack[:len(pool.free)] = pool.free
        done = (rng.random(batch) < 0.2).astype(np.uint8)
        d = [ints(lengths), ints(table), ints(stack), ints([len(pool.free)])]
        lo, co = (None, None) if in_place else (ints(np.zeros(batch)), ints([0]))
        ctx.release_pages(p, torch.from_numpy(done).to(DEV), d[0], d[1], d[2], d[3], lo, co)
        pool.release(done, lengths, table)
        got_stack = d[2].cpu().numpy()
        count = int((d[3] if in_place else co)[0])
        assert count == len(pool.free) and (got_stack[:count] == pool.free).all() and (got_stack[count:] == stack[count:]).all()
        assert ((d[0] if in_place else lo).cpu().numpy() == lengths).all() and (d[1].cpu().numpy() == table).all()
        stack = got_stack.copy()
        new = np.where(rng.random(batch) < 0.3, rng.integers(0, 3 * page, batch), rng.integers(0, 2, batch))
        new = np.minimum(new, max_pages * page - lengths)
        n_slots = int(new.sum()) + int(rng.integers(0, 9))
        before_len, before_table = lengths.copy(), table.copy()
        got = run_plan(ctx, p, before_len, new, before_table, stack, count, n_slots, in_place)
        status, slots, start = pool.plan(lengths, new, table, n_slots)
        short += status > 0
        assert got[5] == status and (got[0] == lengths).all() and got[1] == len(pool.free), (step, got[5], status)
        assert (got[2] == table).all() and (got[3] == slots).all() and (got[4] == start).all()
    assert batch < 17 or short > 0  # (some step asked for more pages than there were)


@pytest.mark.parametrize("in_place", [True, False])
def test_plans_that_are_refused_change_nothing(ctx, in_place):
    lb = binding()
    p = lb.make_paged(3, 1, 1, 8, 16, 4)
    table, free = np.arange(12).reshape(3, 4) % 8, np.arange(8)[::-1]
    for lengths, new, count, n_slots, want in (
            ([5, 64, 0], [1, 1, 1], 8, 9, -1), ([5, -1, 0], [1, 1, 1], 8, 9, -1), ([5, 1, 0], [1, -1, 1], 8, 9, -1),
            ([5, 65, 0], [1, 0, 1], 8, 9, -1), ([5, 1, 0], [1, 2 ** 31 - 1, 1], 8, 9, -1), ([5, 1, 0], [1, 1, 1], -1, 9, -1),
            ([5, 1, 0], [1, 1, 1], 9, 9, -1), ([5, 1, 0], [4, 4, 2], 8, 9, -2), ([16, 16, 0], [1, 1, 17], 1, 30, 3)):
        got = run_plan(ctx, p, lengths, new, table, free, count, n_slots, in_place)
        assert got[5] == want, (lengths, new, got[5])
        assert (got[0] == lengths).all() and got[1] == count and (got[2] == table).all()
        assert (got[3] == -1).all() and (got[4] == 0).all()


def test_a_plan_of_nothing_and_of_much(ctx):
    lb = binding()
    p = lb.make_paged(2, 1, 1, 5000, 16, 4000)
    table, free = np.full((2, 4000), -1), np.random.default_rng(0).permutation(5000)
    got = run_plan(ctx, p, [3, 0], [0, 0], table, free, 5000, 5, True)
    assert got[5] == 0 and (got[3] == -1).all() and (got[4] == 0).all() and got[0].tolist() == [3, 0]
    pool, lengths, t = R.Pool(free, 16, 4000, 5000), np.array([0, 7]), np.full((2, 4000), -1)
    t[1, 0] = 5001  # (a table that names no page: its tokens get no slot)
    got = run_plan(ctx, p, lengths, [63999, 12001], t.copy(), free, 5000, 80000, True)
    status, slots, start = pool.plan(lengths, np.array([63999, 12001]), t, 80000)
    assert got[5] == status == 0 and (got[2] == t).all() and (got[3] == slots).all() and (got[4] == start).all()
    assert (slots[63999:64008] == -1).all()


def test_pages_given_back_twice_do_not_leave_the_stack(ctx):
    lb = binding()
    p = lb.make_paged(2, 1, 1, 4, 16, 4)
    free, count, lens = ints([3, 2, 1, 0]), ints([3]), ints([64, 33])
    ctx.release_pages(p, torch.tensor([1, 1], dtype=torch.uint8, device=DEV), lens, ints(np.arange(8).reshape(2, 4)), free, count)
    assert count.tolist() == [4] and free.tolist() == [3, 2, 1, 0] and lens.tolist() == [0, 0]


# ------------------------------------------------------------------ attention


@pytest.mark.parametrize("group", [1, 2, 3, 4, 5, 8, 11, 16])
@pytest.mark.parametrize("page", [16, 64, 256])
def test_dense_attention_by_group_and_page(ctx, group, page):
    m = Made(group, [70, 1, 257], 2 * group, 2, page)
    check_attn(ctx, m)


@pytest.mark.parametrize("lens", [[1], [0], [15], [16], [17], [63], [64], [65], [128], [1000], [4099], [0, 0, 3], [300, 0, 2, 64, 129]])
def test_dense_attention_by_length(ctx, lens):
    m = Made(sum(lens), lens, 4, 1, 32)
    check_attn(ctx, m, scores=True)


@pytest.mark.parametrize("kind", ["full", "short", "wild"])
@pytest.mark.parametrize("k", [1, 5, 64, 100, 321])
def test_mixed_heads_over_sets(ctx, kind, k):
    m = Made(k, [200, 63, 0, 1, 320], 12, 3, 16, k=k)
    mask = np.array([1, 0, 0, 0, 0, 0, 0, 0, 1, 1, 1, 1], np.uint8)  # one retrieval head; none; no sparse head
    check_attn(ctx, m, mask, m.sets(k, kind), scores=True)


@pytest.mark.parametrize("group", [1, 7, 16])
def test_sparse_heads_only(ctx, group):
    m = Made(5, [500, 40], 2 * group, 2, 64, k=130)
    check_attn(ctx, m, np.zeros(2 * group, np.uint8), m.sets(130, "short"))


@pytest.mark.parametrize("group,scores", [(6, True), (16, True), (8, False)])
def test_mixed_heads_of_wide_groups(ctx, group, scores):
    m = Made(9, [150, 333], 2 * group, 2, 32, k=70)
    mask = (np.arange(2 * group) % 3 == 0).astype(np.uint8)
    check_attn(ctx, m, mask, m.sets(70, "wild"), scores=scores)


def test_sequences_cut_into_many_pieces(ctx):
    """Long enough for hundreds of workgroups, whose partials are merged; one head's pieces end inside others' runs."""
    m = Made(1, [9001, 17, 5003], 6, 2, 64, k=900)
    check_attn(ctx, m, scores=True)
    check_attn(ctx, m, np.array([1, 0, 0, 0, 0, 0], np.uint8), m.sets(900, "wild"), scores=True)


def test_many_short_requests(ctx):
    rng = np.random.default_rng(8)
    m = Made(2, rng.integers(0, 40, 256), 4, 1, 16, k=9)
    check_attn(ctx, m, np.array([1, 0, 1, 0], np.uint8), m.sets(9, "short"), scores=True)


@pytest.mark.parametrize("batch,heads", [(256, 3), (65, 6), (40, 7)])
def test_more_pieces_than_workgroups(ctx, batch, heads):
    """Workgroups take several pieces, whose requests are ordered by length; the same bits again after another launch."""
    rng = np.random.default_rng(batch)
    lens = rng.integers(0, 50, batch)
    lens[[3, batch // 2]] = [4000, 1500]   # (cut into pieces among the others)
    m = Made(batch, lens, 2 * heads, heads, 16, k=20)
    mask, idx = np.tile(np.array([1, 0], np.uint8), heads), m.sets(20, "wild")
    few = Made(5, [100, 20], 4, 2, 16)
    first = check_attn(ctx, m, mask, idx, scores=True)
    for _ in range(2):
        check_attn(ctx, few)
        again = check_attn(ctx, m, mask, idx, scores=True)
        assert (again[0] == first[0]).all() and (again[1] == first[1]).all()


@pytest.mark.parametrize("group", [1, 3, 6, 13])
def test_segments_of_many_partials(ctx, group):
    m = Made(20 + group, [30011], group, 1, 64, k=11003)
    check_attn(ctx, m, scores=True)
    if group > 1:
        check_attn(ctx, m, (np.arange(group) % 3 == 0).astype(np.uint8), m.sets(11003, "wild"))


def test_the_workspace_of_a_pending_selection_is_refused(ctx):
    lb = binding()
    m = Made(18, [70], 4, 2, 16)
    rng = np.random.default_rng(0)
    q, kv = bf16(draw(rng, (1, 4, 128))), [bf16(draw(rng, (1, 2, 96, 128))) for _ in range(2)]
    shape = lb.make_shape(1, 4, 2, 96, 16, kv[0])
    need = max(lb.step_workspace_bytes(shape, 2), lb.paged_workspace_bytes(m.p))
    ws = torch.empty(need, dtype=torch.uint8, device=DEV)
    mask, lens = np.ones(4, np.uint8), ints([96])
    plain, late, out, idx = ints(np.zeros((1, 2, 16))), ints(np.zeros((1, 2, 16))), torch.empty_like(q), ints(m.table)
    ctx.decode_attn(shape, q, kv[0], kv[1], mask, None, out, plain, lens, ws)
    ctx.decode_attn_deferred(shape, q, kv[0], kv[1], mask, None, out, late, lens, ws)
    with pytest.raises(lb.LycheeError) as e:
        ctx.q4_decode_attn(m.p, bf16(m.q), m.cache, idx, ints(m.lens), None, None, torch.empty_like(q), None, ws)
    assert e.value.code == lb.EINVAL
    check_attn(ctx, m)   # (on its own workspace it runs)
    ctx.select_flush()
    assert (late == plain).all()
    ctx.q4_decode_attn(m.p, bf16(m.q), m.cache, idx, ints(m.lens), None, None, torch.empty_like(q), None, ws)


@pytest.mark.parametrize("bad", [-1, 1 << 30, -(1 << 31)])
def test_pages_that_are_not_there_are_left_out(ctx, bad):
    m = Made(6, [200, 64, 48], 4, 1, 16, k=40)
    table = m.table.copy()
    table[0, [0, 5, 12]] = bad   # the first, one between and the last
    table[1, :] = m.p.n_pages    # nothing left: zeros
    mask = np.array([1, 1, 0, 0], np.uint8)
    check_attn(ctx, m, None, None, scores=True, table=table)
    check_attn(ctx, m, mask, m.sets(40), scores=True, table=table)


def test_lengths_beyond_the_table_are_clamped(ctx):
    m = Made(7, [64, 50], 4, 2, 16, max_pages=4)
    check_attn(ctx, m, lens=np.array([2 ** 31 - 1, -5], np.int32), scores=True)


def test_steep_and_flat_scores(ctx):
    m = Made(11, [400], 8, 2, 32, spread=40.0)    # one token takes all
    check_attn(ctx, m)
    m = Made(12, [5000], 8, 2, 32, spread=1e-3)   # every token counts the same
    check_attn(ctx, m)


def test_numbers_that_are_none_stay_in_their_request(ctx):
    m = Made(13, [100, 100, 100], 4, 1, 16)
    clean = check_attn(ctx, m)[0]
    slot = R.slots_of(m.table[1], 100, 16, m.p.n_pages)[37]
    t, r = m.ref._at(slot, 0)
    m.ref.bytes[t, 2048 + 5 * 16 + r] = 255   # a group of that token's value is NaN: dimensions 32 to 63
    m.cache.copy_(torch.from_numpy(m.ref.bytes))
    out = torch.zeros((3, 4, 128), dtype=torch.bfloat16, device=DEV)
    ctx.q4_decode_attn(m.p, bf16(m.q), m.cache, ints(m.table), ints(m.lens), None, None, out, None, m.ws)
    got = host(out)
    assert np.isnan(got[1, :, 32:64]).all() and (got[[0, 2]] == clean[[0, 2]]).all()
    assert (got[1, :, :32] == clean[1, :, :32]).all() and (got[1, :, 64:] == clean[1, :, 64:]).all()
    m.ref.bytes[t, 2048 + 0 * 16 + r] = 255   # and of its key: every output of the request
    m.cache.copy_(torch.from_numpy(m.ref.bytes))
    ctx.q4_decode_attn(m.p, bf16(m.q), m.cache, ints(m.table), ints(m.lens), None, None, out, None, m.ws)
    got = host(out)
    assert np.isnan(got[1]).all() and (got[[0, 2]] == clean[[0, 2]]).all()
    # the same token out of reach: the lengths end before it
    check_attn(ctx, m, lens=np.array([100, 37, 100], np.int32))


def test_interleaved_layers_and_shared_pages(ctx):
    """Pages of two layers side by side (page_tiles of both), and two requests that share their first pages."""
    lb = binding()
    m = Made(14, [96, 96], 4, 2, 32, page_tiles=11)
    m.table[1, :2] = m.table[0, :2]
    check_attn(ctx, m, scores=True)


def test_cache_whose_offsets_pass_32_bits(ctx):
    lb = binding()
    small = Made(15, [300, 65], 4, 1, 64, k=50)
    n_pages = 600_000                                     # 5.2 GB of pages
    p = lb.make_paged(2, 4, 1, n_pages, 64, small.max_pages, 50, small.max_pages + 2)
    cache = torch.empty((n_pages, p.page_tiles * 2176), dtype=torch.uint8, device=DEV)
    far = np.sort(np.random.default_rng(1).choice(np.arange(n_pages - 60_000, n_pages), small.p.n_pages, False))
    cache[torch.from_numpy(far).to(DEV)] = small.cache.view(small.p.n_pages, -1)
    table = np.where(small.table >= 0, far[np.maximum(small.table, 0)], -1)
    idx = small.sets(50)
    mask = np.array([1, 0, 0, 1], np.uint8)
    want = [check_attn(ctx, small), check_attn(ctx, small, mask, idx)]
    for w, (mk, ix) in zip(want, ((None, None), (mask, idx))):
        out = torch.zeros((2, 4, 128), dtype=torch.bfloat16, device=DEV)
        ctx.q4_decode_attn(p, bf16(small.q), cache, ints(table), ints(small.lens), mk, None if ix is None else ints(ix), out, None,
                           small.ws)
        assert (host(out) == w[0]).all()
    rows = torch.zeros((2, 2, 1, 300, 128), dtype=torch.bfloat16, device=DEV)
    ctx.q4_read(p, cache, ints(table), None, ints(small.lens), rows[0], rows[1])
    assert (host(rows)[:, 0, 0] == small.ref.rows(R.slots_of(small.table[0], 300, 64, small.p.n_pages), 0)).all()
    new = draw(np.random.default_rng(2), (1, 2, 1, 128))
    slot = int(far[-1]) * 64 + 63
    t = bf16(new)
    ctx.q4_append(p, t[:, 0], t[:, 1], ints([slot]), cache)
    one = torch.zeros((2, 1, 1, 64, 128), dtype=torch.bfloat16, device=DEV)
    p1 = lb.make_paged(1, 4, 1, n_pages, 64, 1)
    ctx.q4_read(p1, cache, ints([[far[-1]]]), ints([63]), ints([64]), one[0], one[1])
    assert (host(one)[:, 0, 0, 0] == R.dequantise(*R.quantise(new[0, :, 0]))).all()


def test_the_same_call_gives_the_same_bits_on_any_stream(ctx):
    m = Made(16, [3000, 700], 8, 2, 64, k=300)
    mask, idx = np.array([1, 0, 0, 0, 0, 0, 1, 1], np.uint8), m.sets(300)
    first = check_attn(ctx, m, mask, idx, scores=True)
    side = torch.cuda.Stream()
    for stream in (None, side, side):
        again = check_attn(ctx, m, mask, idx, scores=True, stream=stream)
        assert (again[0] == first[0]).all() and (again[1] == first[1]).all()


# ------------------------------------------------------------------ selection


def check_select(ctx, x, lens, k, mask=None, heads_per=2, idx=None):
    lb = binding()
    B, H, n = x.shape
    page = 16
    p = lb.make_paged(B, H * heads_per, H, 1, page, max(1, n // page), k)
    t = torch.from_numpy(np.ascontiguousarray(x, np.float32)).to(DEV)
    out = ints(np.full((B, H, k), 55))
    ctx.select_scores(p, t, ints(lens), mask, None if idx is None else ints(idx), out)
    got = out.cpu().numpy()
    for b in range(B):
        L = int(np.clip(lens[b], 0, p.max_pages * page))
        for g in range(H):
            if mask is not None and not mask[g * heads_per:(g + 1) * heads_per].any():
                assert (got[b, g] == idx[b, g]).all()
                continue
            want = np.full(k, -1)
            best = R.top(x[b, g, :L].astype(np.float32), k)
            want[:len(best)] = best
            assert (got[b, g] == want).all(), (b, g, L, np.nonzero(got[b, g] != want)[0][:5])
    return got


@pytest.mark.parametrize("L,k", [(16, 1), (48, 3), (64, 64), (1008, 1000), (4096, 17), (5008, 2500), (33008, 2048), (131072, 4096), (131072, 8192), (200000, 65000)])
def test_selection_by_size(ctx, L, k):
    rng = np.random.default_rng(L + k)
    x = rng.standard_normal((2, 2, L))
    check_select(ctx, x, [L, max(0, L - 13)], k)


@pytest.mark.parametrize("L", [1025, 2049, 8192, 8195, 33000, 131072, 140000])
@pytest.mark.parametrize("k", [1, 2, 16, 255, 256, 512, 513, 1024])
def test_selection_of_few(ctx, L, k):
    """Sets of up to one entry a thread: rows without order, rows whose high scores are all one thread's (a stride of 1024), or
    one wavefront's, more of them than are taken and than its list holds; and fewer positions than the rows are long."""
    rng = np.random.default_rng(L + k)
    n = -(-L // 16) * 16
    x = rng.standard_normal((1, 4, n))
    x[0, 1, 37::1024] += 30.0
    x[0, 2, np.arange(n) % 1024 < 64] += 30.0
    x[0, 3] = -np.abs(x[0, 3])
    x[0, 3, rng.permutation(n)[:3 * k]] = 0.0
    check_select(ctx, x, [L], k)
    check_select(ctx, x, [k + 1], k)


@pytest.mark.parametrize("what", ["equal", "two values", "duplicates", "steps", "extremes", "sorted", "reversed", "tiny", "planted"])
def test_selection_among_equals(ctx, what):
    rng = np.random.default_rng(3)
    n, k = 20000, 1500
    x = rng.standard_normal((1, 3, n)).astype(np.float32)
    if what == "equal":
        x[:] = -2.5
    elif what == "two values":
        x = np.where(rng.random((1, 3, n)) < 0.05, 1.0, np.where(rng.random((1, 3, n)) < 0.5, 0.0, -0.0)).astype(np.float32)
    elif what == "duplicates":
        x = x[:, :, rng.integers(0, 900, n)]
    elif what == "steps":
        x = np.round(x * 4) / 4
    elif what == "extremes":
        x = rng.choice([np.inf, -np.inf, np.nan, 3.4e38, -3.4e38, 1e-45, -1e-45, 0.0, -0.0, 1.0], (1, 3, n)).astype(np.float32)
        x[0, 2] = np.nan
    elif what == "sorted":
        x.sort(axis=2)
    elif what == "reversed":
        x = -np.sort(-x, axis=2)
    elif what == "tiny":
        x = (1.0 + rng.integers(0, 9, (1, 3, n)) * 2.0 ** -23).astype(np.float32)
    else:
        x[:, :, rng.permutation(n)[:k]] += 40.0
    for kk in (1, 63, k):
        check_select(ctx, x, [n - 7], kk)


@pytest.mark.parametrize("zeros", [0, 5000, 14999, 15000, 15001])
def test_selection_at_the_edge_below_zero(ctx, zeros):
    """The last ones taken are the smallest negative numbers there are, or the zeros above them; too many for the list."""
    rng = np.random.default_rng(zeros)
    n = 40000
    x = (-rng.integers(1, 1 << 23, (1, 2, n))).astype(np.float64) * 2.0 ** -149
    x[0, 1] = -rng.integers(1, 300, n) * 2.0 ** -149
    at = rng.permutation(n)[:zeros]
    x[:, :, at] = np.where(rng.random(zeros) < 0.5, 0.0, -0.0)
    check_select(ctx, x, [n - 9], 15000)
    x[:, :, at[:100]] = 3.0
    check_select(ctx, x, [n], 15000)


def test_selection_passes_over_every_kind_of_nan(ctx):
    rng = np.random.default_rng(17)
    for n in (5000, 20000, 140000):
        x = rng.standard_normal((1, 2, n)).astype(np.float32)
        bits = x.view(np.uint32)
        bits[rng.random(x.shape) < 0.4] = 0x7F800001   # signaling
        bits[rng.random(x.shape) < 0.2] = 0xFFFFFFFF
        for k in (40, n // 2, n - 32):
            check_select(ctx, x, [n], k)


def test_selection_of_a_batch_with_kept_sets_and_empty_requests(ctx):
    rng = np.random.default_rng(4)
    B, H, n, k = 40, 3, 2048, 100
    x = rng.standard_normal((B, H, n))
    lens = rng.integers(0, n, B)
    lens[:5] = [0, 1, k, k + 1, k - 1]
    lens[5], lens[6] = 2 ** 31 - 1, -3
    mask = np.array([0, 1, 0, 0, 1, 1], np.uint8)
    check_select(ctx, x, lens, k, mask, idx=rng.integers(-5, 5000, (B, H, k)))


# ------------------------------------------------------------------ counts that an int just holds


def test_a_set_and_a_copied_set_of_the_most_entries(ctx):
    lb = binding()
    k = 2 ** 31 - 1
    p = lb.make_paged(1, 1, 1, 1, 16, 2, k)
    room = torch.full((k + 2048,), 7, dtype=torch.int32, device=DEV)
    x = torch.arange(32, dtype=torch.float32, device=DEV).view(1, 1, 32)
    ctx.select_scores(p, x, ints([20]), None, None, room[1024:1024 + k].view(1, 1, k))
    assert room[1024:1044].tolist() == list(range(20)) and bool((room[1044:1024 + k] == -1).all())
    assert bool((room[:1024] == 7).all()) and bool((room[1024 + k:] == 7).all())
    out = torch.full((k + 2048,), 9, dtype=torch.int32, device=DEV)
    ctx.select_scores(p, x, ints([20]), np.zeros(1, np.uint8), room[1024:1024 + k].view(1, 1, k), out[1024:1024 + k].view(1, 1, k))
    assert torch.equal(out[1024:1024 + k], room[1024:1024 + k])
    assert bool((out[:1024] == 9).all()) and bool((out[1024 + k:] == 9).all())


@pytest.mark.parametrize("in_place", [True, False])
def test_a_plan_with_room_for_the_most_slots(ctx, in_place):
    lb = binding()
    n, ends = 2 ** 31 - 1, 1 << 18
    p = lb.make_paged(2, 1, 1, 8, 16, 4)
    room = torch.full((n + 2 * ends,), 7, dtype=torch.int32, device=DEV)
    slots = room[ends:ends + n]
    d = [ints([0, 0]), ints([3, 1]), ints(np.full((2, 4), -1)), ints(np.arange(8)), ints([8])]
    lo, co = (None, None) if in_place else (ints([0, 0]), ints([0]))
    start, status = ints([7] * 3), ints([7])
    ctx.plan_pages(p, *d, lo, co, slots, start, status)
    assert status.tolist() == [0] and start.tolist() == [0, 3, 4] and slots[:4].tolist() == [112, 113, 114, 96]
    assert bool((slots[4:] == -1).all()) and bool((room[:ends] == 7).all()) and bool((room[ends + n:] == 7).all())


# ------------------------------------------------------------------ together


def test_a_serving_loop_of_two_layers(ctx):
    """Requests come, grow and leave: pages planned, tokens written in both layers, layer 0's retrieval heads select the
    sets that layer 1's sparse heads read.  Against the reference at every step; the caches bit for bit."""
    lb = binding()
    rng = np.random.default_rng(21)
    B, H, G, page, k, max_pages, n_pages = 3, 2, 2, 16, 24, 6, 14
    p = lb.make_paged(B, H * G, H, n_pages, page, max_pages, k)
    masks = [np.ones(H * G, np.uint8), np.array([0, 0, 1, 0], np.uint8)]
    lens, table = np.zeros(B, np.int64), np.full((B, max_pages), -1, np.int32)
    pool = R.Pool(rng.permutation(n_pages), page, max_pages, n_pages)
    ref = [R.Cache(n_pages, page, H, 0, 0xFF) for _ in range(2)]
    d = dict(lens=ints(lens), table=ints(table), free=ints(np.asarray(pool.free)), count=ints([n_pages]), start=ints(np.zeros(B + 1)),
             status=ints([5]), sets=ints(np.zeros((B, H, k))), sets1=ints(np.zeros((B, H, k))))
    caches = [torch.full((n_pages, p.page_tiles * 2176), 0xFF, dtype=torch.uint8, device=DEV) for _ in range(2)]
    scores = torch.zeros((B, H, max_pages * page), device=DEV)
    ws = lb.alloc_paged_workspace(p)
    m = Made.__new__(Made)
    m.p, m.max_pages, m.ws = p, max_pages, ws
    for step, (new, gone) in enumerate([([40, 3, 0], []), ([1, 1, 64], []), ([1, 1, 1], []), ([1, 0, 1], [1]), ([0, 50, 1], [0]), ([1, 1, 1], [])]):
        done = np.isin(np.arange(B), gone).astype(np.uint8)
        pool.release(done, lens, table)
        ctx.release_pages(p, torch.from_numpy(done).to(DEV), d["lens"], d["table"], d["free"], d["count"])
        n_slots = sum(new) + 2
        slots = ints(np.zeros(n_slots))
        ctx.plan_pages(p, d["lens"], ints(new), d["table"], d["free"], d["count"], None, None, slots, d["start"], d["status"])
        status, want_slots, _ = pool.plan(lens, new, table, n_slots)
        assert status == 0 and int(d["status"][0]) == 0 and (slots.cpu().numpy() == want_slots).all()
        assert (d["table"].cpu().numpy() == table).all() and (d["lens"].cpu().numpy() == lens).all()
        sets = None
        for layer in range(2):
            kv = draw(rng, (n_slots, 2, H, 128))
            t = bf16(kv)
            ctx.q4_append(p, t[:, 0], t[:, 1], slots, caches[layer])
            for i, s in enumerate(want_slots):
                for g in range(H):
                    if s >= 0:
                        c = [R.quantise(kv[i, j, g][None]) for j in range(2)]
                        ref[layer].write(s, g, *[(x[0][0], x[1][0]) for x in c])
            assert (caches[layer].cpu().numpy().reshape(-1, 2176) == ref[layer].bytes).all()
            m.ref, m.cache, m.table, m.lens = ref[layer], caches[layer], table, lens.astype(np.int32)
            m.q = draw(rng, (B, H * G, 128))
            _, sc = check_attn(ctx, m, masks[layer], sets, scores=True)
            idx = torch.from_numpy(sc).to(DEV)
            ctx.select_scores(p, idx, d["lens"], masks[layer], None if sets is None else ints(sets), d["sets"])
            got = d["sets"].cpu().numpy()
            for b in range(B):
                for g in range(H):
                    want = np.full(k, -1)
                    best = R.top(sc[b, g, :lens[b]], k)
                    want[:len(best)] = best
                    assert (got[b, g] == (want if masks[layer][g * G:(g + 1) * G].any() else sets[b, g])).all()
            sets = got.copy()


def test_a_captured_step_replays_as_the_eager_calls_run(ctx):
    """Plan, append, attention and selection of a decode step in one graph, replayed token after token with eager work and
    waits in between, against the same calls made eagerly on a second set of buffers."""
    lb = binding()
    m = Made(17, [700, 33, 129], 8, 2, 16, k=40, max_pages=50, extra=30)
    B, H = 3, 2
    mask, idx0 = np.array([1, 0, 0, 0, 0, 1, 0, 0], np.uint8), m.sets(40)
    held = set(m.table[m.table >= 0].tolist())
    free = [i for i in range(m.p.n_pages) if i not in held]

    def state():
        s = dict(lens=ints(m.lens), table=ints(m.table), free=ints(np.asarray(free + [-1] * (m.p.n_pages - len(free)))),
                 count=ints([len(free)]), new=ints([1, 1, 1]), slots=ints([0] * 3), start=ints([0] * 4), status=ints([0]),
                 cache=m.cache.clone(), idx=ints(idx0), sets=ints(np.zeros_like(idx0)), ws=lb.alloc_paged_workspace(m.p),
                 kv=torch.zeros((3, 2, H, 128), dtype=torch.bfloat16, device=DEV),
                 q=torch.zeros((B, 8, 128), dtype=torch.bfloat16, device=DEV),
                 out=torch.zeros((B, 8, 128), dtype=torch.bfloat16, device=DEV),
                 scores=torch.zeros((B, H, 800), device=DEV))
        return s

    def step(c, s):
        c.plan_pages(m.p, s["lens"], s["new"], s["table"], s["free"], s["count"], None, None, s["slots"], s["start"], s["status"])
        c.q4_append(m.p, s["kv"][:, 0], s["kv"][:, 1], s["slots"], s["cache"])
        c.q4_decode_attn(m.p, s["q"], s["cache"], s["table"], s["lens"], mask, s["idx"], s["out"], s["scores"], s["ws"])
        c.select_scores(m.p, s["scores"], s["lens"], mask, s["idx"], s["sets"])

    eager, held_ctx = state(), lb.Context(0)
    try:
        graph_state, g = state(), torch.cuda.CUDAGraph()
        stream = torch.cuda.Stream()
        torch.cuda.synchronize()
        with torch.cuda.graph(g, stream=stream):
            step(held_ctx, graph_state)
        for i in range(20):
            gen = torch.Generator(DEV).manual_seed(i)
            for s in (eager, graph_state):
                gen.manual_seed(i)
                s["kv"].normal_(generator=gen)
                s["q"].normal_(generator=gen)
            step(ctx, eager)
            g.replay()
            torch.cuda.synchronize()
            for key in ("lens", "table", "count", "slots", "start", "status", "cache", "out", "scores", "sets"):
                assert torch.equal(eager[key], graph_state[key]), (i, key)
            if i % 5 == 0:
                torch.randn(1 << 20, device=DEV).sum().item()
        assert eager["lens"].tolist() == [720, 53, 149] and eager["status"].tolist() == [0]
        del g
    finally:
        torch.cuda.synchronize()
        held_ctx.close()


def test_the_rows_that_were_read_serve_the_bf16_calls(ctx):
    """A sequence handed to lychee_dense_decode_attn: on the values that the cache stands for both layers agree."""
    lb = binding()
    m = Made(18, [500, 90], 8, 2, 32)
    rows = torch.zeros((2, 2, 2, 512, 128), dtype=torch.bfloat16, device=DEV)
    ctx.q4_read(m.p, m.cache, ints(m.table), None, ints(m.lens), rows[0], rows[1])
    shape = lb.make_shape(2, 8, 2, 512, 1, kv=rows[0])
    out = torch.zeros((2, 8, 128), dtype=torch.bfloat16, device=DEV)
    ctx.dense_decode_attn(shape, bf16(m.q), rows[0], rows[1], out, ints(m.lens), lb.alloc_workspace(shape))
    mine = check_attn(ctx, m)[0]
    # (each is within half a bf16 step of the value and far less beside it)
    assert (np.abs(host(out) - mine) <= 2.0 ** -7 * np.abs(mine) + 1e-4).all()


def attn_call(c, m, mask, idx):
    """The tensors of a call on `m` and the call itself."""
    d = dict(q=bf16(m.q), table=ints(m.table), lens=ints(m.lens), idx=ints(idx), out=torch.zeros((m.p.batch, m.p.n_q_heads, 128), dtype=torch.bfloat16, device=DEV),
             sc=torch.zeros((m.p.batch, m.p.n_kv_heads, m.max_pages * m.p.page_size), device=DEV),
             sets=torch.zeros((m.p.batch, m.p.n_kv_heads, m.p.k), dtype=torch.int32, device=DEV))

    def run(ws):
        c.q4_decode_attn(m.p, d["q"], m.cache, d["table"], d["lens"], mask, d["idx"], d["out"], d["sc"], ws)
        c.select_scores(m.p, d["sc"], d["lens"], mask, d["idx"], d["sets"])

    def take():
        got = [d[n].cpu().clone() for n in ("out", "sc", "sets")]
        for n in ("out", "sc", "sets"):
            d[n].zero_()
        return got

    return run, take


def two_calls(c0, c1):
    mask = np.array([1, 0, 0, 0, 0, 0, 1, 1], np.uint8)
    big, wide = Made(31, [2500, 900], 8, 2, 64, k=200), Made(32, np.arange(20, 90, 3), 8, 2, 16, k=33)
    pairs = [attn_call(c, m, mask, m.sets(m.p.k)) for c, m in ((c0, big), (c1, wide))]
    want = []
    for (run, take), m in zip(pairs, (big, wide)):
        run(m.ws)
        want.append(take())
    torch.cuda.synchronize()
    return (big, wide), pairs, want


def test_two_contexts_on_two_streams(ctx):
    other = binding().Context(0)
    made, pairs, want = two_calls(ctx, other)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(5):
        for _ in range(4):
            for (run, _), m, s in zip(pairs, made, streams):
                with torch.cuda.stream(s):
                    run(m.ws)
        torch.cuda.synchronize()
        for (_, take), w in zip(pairs, want):
            assert all(torch.equal(a, b) for a, b in zip(take(), w))
        torch.cuda.synchronize()
    other.close()


def test_two_captured_graphs_share_a_context_and_a_workspace(ctx):
    made, pairs, want = two_calls(ctx, ctx)
    ws = max((m.ws for m in made), key=lambda t: t.numel())
    graphs = []
    for run, _ in pairs:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            run(ws)
        graphs.append(g)
    for turn in range(4):
        for i in (0, 1, 1, 0):
            graphs[i].replay()
            if turn & 1:
                pairs[1 - i][0](ws)   # (an eager call of the other between them)
        torch.cuda.synchronize()
        for (_, take), w in zip(pairs, want):
            assert all(torch.equal(a, b) for a, b in zip(take(), w))
        torch.cuda.synchronize()
