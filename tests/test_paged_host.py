"""The paged 4-bit cache without a GPU: checks of its shape, every refusal of its calls (they come before anything is
launched, and before the context is looked into), and the reference itself against hand-made values."""
import ctypes

import numpy as np
import pytest
import torch

from tests import paged_reference as R


@pytest.fixture(scope="module")
def lb():
    from paper_2602_04541_amd import binding
    return binding


def shape(lb, **kw):
    a = dict(batch=2, n_q_heads=8, n_kv_heads=2, n_pages=10, page_size=16, max_pages=4, k=5)
    a.update(kw)
    return lb.make_paged(**a)


def test_shapes(lb):
    assert lb.check_paged(shape(lb)) == lb.OK
    for page in (16, 32, 64, 128, 256):
        assert lb.check_paged(shape(lb, page_size=page)) == lb.OK
    for page in (0, 8, 24, 512):
        assert lb.check_paged(shape(lb, page_size=page, page_tiles=64)) == lb.EUNSUPPORTED
    for field in ("batch", "n_q_heads", "n_kv_heads", "n_pages", "max_pages", "k"):
        p = shape(lb)
        setattr(p, field, 0)
        assert lb.check_paged(p) == lb.EINVAL, field
        setattr(p, field, -3)
        assert lb.check_paged(p) == lb.EINVAL, field
    assert lb.check_paged(shape(lb, n_q_heads=7)) == lb.EINVAL
    assert lb.check_paged(shape(lb, head_dim=64)) == lb.EUNSUPPORTED
    assert lb.check_paged(shape(lb, batch=257)) == lb.EUNSUPPORTED
    assert lb.check_paged(shape(lb, n_q_heads=65, n_kv_heads=65)) == lb.EUNSUPPORTED
    assert lb.check_paged(shape(lb, table_stride=3)) == lb.EINVAL
    assert lb.check_paged(shape(lb, page_tiles=1)) == lb.EINVAL
    assert lb.check_paged(shape(lb, page_tiles=5, table_stride=9)) == lb.OK
    assert lb.check_paged(shape(lb, max_pages=1 << 20)) == lb.OK          # 2^24 tokens
    assert lb.check_paged(shape(lb, max_pages=(1 << 20) + 1)) == lb.EUNSUPPORTED
    assert lb.check_paged(shape(lb, n_pages=1 << 26)) == lb.OK            # 2^27 tiles
    assert lb.check_paged(shape(lb, n_pages=(1 << 26) + 1)) == lb.EUNSUPPORTED
    assert lb.check_paged(shape(lb, n_pages=1 << 23, page_size=256)) == lb.EUNSUPPORTED  # 2^31 slots


def test_head_types(lb):
    p = shape(lb)
    mixed = np.array([1, 0, 0, 0, 1, 1, 1, 1], np.uint8)
    assert lb.check_paged(p, np.ones(8, np.uint8), has_idx_in=False) == lb.OK
    assert lb.check_paged(p, mixed, has_idx_in=True) == lb.OK
    assert lb.check_paged(p, mixed, has_idx_in=False) == lb.EINVAL
    assert lb.check_paged(p, np.full(8, 2, np.uint8)) == lb.EINVAL


def test_workspace(lb):
    assert lb.paged_workspace_bytes(shape(lb, head_dim=64)) == 0
    small, large = lb.paged_workspace_bytes(shape(lb)), lb.paged_workspace_bytes(shape(lb, batch=200, n_q_heads=64, n_kv_heads=8))
    assert 0 < small < large and small % 256 == 0
    with pytest.raises(lb.LycheeError):
        lb.alloc_paged_workspace(shape(lb, k=0), "cpu")
    with pytest.raises(lb.LycheeError):
        lb.alloc_q4_cache(shape(lb, k=0), "cpu")
    assert lb.alloc_q4_cache(shape(lb), "cpu").shape == (10, 2 * 2176)


# Arguments of a call that would be accepted, by name, and the ones whose change is refused.  Addresses are made up:
# a refused call touches none of them.
A = 1 << 20
CALLS = {
    "lychee_release_pages": dict(done=A, lengths=A, table=A, free=A, count=A, lengths_out=A, count_out=A, stream=None),
    "lychee_plan_pages": dict(lengths=A, new=A, table=A, free=A, count=A, lengths_out=A, count_out=A, slots=A, n_slots=7,
                              start=A, status=A, stream=None),
    "lychee_q4_append": dict(k=A, v=A, stride_tok=256, stride_head=128, slots=A, n=7, cache=A, stream=None),
    "lychee_q4_read": dict(cache=A, table=A, first=A, last=A, k=A, v=A, stride_b=4096, stride_h=2048, stride_t=128, rows=9,
                           stream=None),
    "lychee_q4_decode_attn": dict(q=A, cache=A, table=A, lengths=A, mask=None, idx=A, out=A, scores=A, stride=64, ws=A,
                                  bytes=1 << 40, stream=None),
    "lychee_select_scores": dict(scores=A, stride=64, lengths=A, mask=None, idx_in=2 * A, idx_out=A, stream=None),
}
NULL = {
    "lychee_release_pages": "done lengths table free count lengths_out count_out",
    "lychee_plan_pages": "lengths new table free count lengths_out count_out slots start status",
    "lychee_q4_append": "k v slots cache",
    "lychee_q4_read": "cache table last k v",
    "lychee_q4_decode_attn": "q cache table lengths out",
    "lychee_select_scores": "scores lengths idx_out",
}
ODD = {  # alignment each pointer needs
    "lychee_release_pages": dict(lengths=4, table=4, free=4, count=4, lengths_out=4, count_out=4),
    "lychee_plan_pages": dict(lengths=4, new=4, table=4, free=4, count=4, lengths_out=4, count_out=4, slots=4, start=4, status=4),
    "lychee_q4_append": dict(k=16, v=16, slots=4, cache=128),
    "lychee_q4_read": dict(cache=128, table=4, first=4, last=4, k=16, v=16),
    "lychee_q4_decode_attn": dict(q=16, cache=128, table=4, lengths=4, idx=4, out=16, scores=4),
    "lychee_select_scores": dict(scores=4, lengths=4, idx_in=4, idx_out=4),
}


def refused(lb, name, p, ctx=True, **change):
    """The call's status, made on a context that must not be looked into (its bytes are no context)."""
    args = dict(CALLS[name])
    args.update(change)
    fake = ctypes.create_string_buffer(1 << 16)
    return getattr(lb._lib, name)(ctypes.addressof(fake) if ctx else None, ctypes.byref(p) if p is not None else None, *args.values())


@pytest.mark.parametrize("name", sorted(CALLS))
def test_null_and_misaligned_arguments_are_refused(lb, name):
    p = shape(lb)
    assert refused(lb, name, p, ctx=False) == lb.EINVAL
    assert refused(lb, name, None) == lb.EINVAL
    assert refused(lb, name, shape(lb, head_dim=64)) == lb.EUNSUPPORTED
    assert refused(lb, name, shape(lb, table_stride=3)) == lb.EINVAL
    for arg in NULL[name].split():
        assert refused(lb, name, p, **{arg: None}) == lb.EINVAL, arg
    for arg, align in ODD[name].items():
        assert refused(lb, name, p, **{arg: A + align // 2}) == lb.EINVAL, arg


@pytest.mark.parametrize("name", ["lychee_q4_decode_attn", "lychee_select_scores"])
def test_workspace_and_scores_are_checked(lb, name):
    p = shape(lb)
    if "attn" in name:
        assert refused(lb, name, p, ws=None) == lb.EWORKSPACE
        assert refused(lb, name, p, ws=A + 128) == lb.EWORKSPACE
        assert refused(lb, name, p, bytes=lb.paged_workspace_bytes(p) - 1) == lb.EWORKSPACE
    assert refused(lb, name, p, stride=63) == lb.EINVAL
    mask = np.array([1, 0, 0, 0, 0, 0, 0, 0], np.uint8)
    no_set = {"idx" if "attn" in name else "idx_in": None}
    assert refused(lb, name, p, mask=mask.ctypes.data, **no_set) == lb.EINVAL
    bad = np.full(8, 2, np.uint8)
    assert refused(lb, name, p, mask=bad.ctypes.data) == lb.EINVAL


@pytest.mark.parametrize("name", ["lychee_q4_decode_attn", "lychee_select_scores"])
@pytest.mark.parametrize("at", range(1, 8))
def test_every_head_type_is_checked(lb, name, at):
    """A value that is no head type is refused wherever it stands, behind a retrieval head of its group as well."""
    mask = np.array([1, 0, 0, 0, 1, 1, 1, 1], np.uint8)
    mask[at] = 7
    p = shape(lb)
    assert lb.check_paged(p, mask) == lb.EINVAL
    assert refused(lb, name, p, mask=mask.ctypes.data) == lb.EINVAL


def test_sizes_that_are_refused(lb):
    p = shape(lb)
    assert refused(lb, "lychee_plan_pages", p, n_slots=-1) == lb.EINVAL
    assert refused(lb, "lychee_q4_append", p, n=-1) == lb.EINVAL
    assert refused(lb, "lychee_q4_append", p, n=0) == lb.OK   # nothing to do, and nothing launched
    assert refused(lb, "lychee_q4_append", p, n=2 ** 31 - 1) == lb.EUNSUPPORTED
    for stride in (-8, 4, 129):
        assert refused(lb, "lychee_q4_append", p, stride_tok=stride) == lb.EINVAL
        assert refused(lb, "lychee_q4_append", p, stride_head=stride) == lb.EINVAL
        for s in ("stride_b", "stride_h", "stride_t"):
            assert refused(lb, "lychee_q4_read", p, **{s: stride}) == lb.EINVAL
    assert refused(lb, "lychee_q4_read", p, stride_t=120) == lb.EINVAL
    assert refused(lb, "lychee_q4_read", p, stride_h=0) == lb.EINVAL
    assert refused(lb, "lychee_q4_read", p, stride_b=0) == lb.EINVAL
    assert refused(lb, "lychee_q4_read", p, rows=-1) == lb.EINVAL
    assert refused(lb, "lychee_q4_read", p, rows=0) == lb.OK
    assert refused(lb, "lychee_q4_decode_attn", shape(lb, n_q_heads=34)) == lb.EUNSUPPORTED     # 17 heads a KV head
    wide = shape(lb, batch=256, n_q_heads=64, n_kv_heads=64, max_pages=1 << 20)
    assert refused(lb, "lychee_q4_decode_attn", wide, stride=1 << 24) == lb.EUNSUPPORTED          # 2^32 blocks
    assert refused(lb, "lychee_select_scores", p, idx_out=A, idx_in=A) == lb.EINVAL


# ------------------------------------------------------------------ what the binding refuses


def bound(lb, device=-1):
    """The binding's methods without a context: tensors of the CPU pass for the device's, and what is passed on the library
    refuses (EINVAL, since there is no context)."""
    c = object.__new__(lb.Context)
    c._h, c.device = None, device
    return c


def ints(*size):
    return torch.zeros(size, dtype=torch.int32)


def half(*size):
    return torch.zeros(size, dtype=torch.bfloat16)


def arguments(lb, p):
    """Tensors just large enough, by method and argument (shape(lb): 2 requests, 8 heads on 2, 10 pages of 16 tokens, 4 a
    request, sets of 5)."""
    pages = dict(lengths=ints(2), block_table=ints(2, 4), free_pages=ints(10), free_count=ints(1), lengths_out=ints(2),
                 free_count_out=ints(1))
    cache = torch.zeros((10, 2 * 2176), dtype=torch.uint8)
    mask = np.array([1, 0, 0, 0, 1, 1, 1, 1], np.uint8)
    kv, rows = half(7, 2, 2, 128), half(2, 2, 2, 9, 136)
    return {
        "release_pages": dict(done=torch.zeros(2, dtype=torch.uint8), **pages),
        "plan_pages": dict(pages, new_tokens=ints(2), slots=ints(7), token_start=ints(3), status=ints(1)),
        "q4_append": dict(k_new=kv[:, 0], v_new=kv[:, 1], slots=ints(7), cache=cache),
        "q4_read": dict(cache=cache, block_table=ints(2, 4), first=ints(2), last=ints(2), k_out=rows[0, ..., :128],
                        v_out=rows[1, ..., :128]),
        "q4_decode_attn": dict(q=half(2, 8, 128), cache=cache, block_table=ints(2, 4), lengths=ints(2), head_type_mask=mask,
                               idx_in=ints(2, 2, 5), out=half(2, 8, 128), scores=torch.zeros(2, 2, 64),
                               workspace=lb.alloc_paged_workspace(p, "cpu")),
        "select_scores": dict(scores=torch.zeros(2, 2, 64), lengths=ints(2), head_type_mask=mask, idx_in=ints(2, 2, 5),
                              idx_out=ints(2, 2, 5)),
    }


METHODS = ["release_pages", "plan_pages", "q4_append", "q4_read", "q4_decode_attn", "select_scores"]


def says(lb, p, method, args, device=-1):
    """What the call's error says: that the library refused it (there is no context), or which argument the binding did."""
    with pytest.raises(lb.LycheeError) as e:
        getattr(bound(lb, device), method)(p, stream=0, **args)
    assert e.value.code == lb.EINVAL
    return str(e.value)


@pytest.mark.parametrize("method", METHODS)
def test_the_binding_looks_at_types_sizes_layout_and_device(lb, method):
    p = shape(lb)
    passed = "lychee_%s failed" % method
    args = arguments(lb, p)[method]
    assert says(lb, p, method, args).startswith(passed)
    for name, t in args.items():
        if name == "head_type_mask":
            continue
        bad = [t.to(torch.int64) if t.element_size() == 4 or name == "done" else t.to(torch.float32)]
        if t.dim() == 1:
            bad.append(torch.stack((t, t), 1)[:, 0] if len(t) > 1 else None)    # every other entry
            bad.append(t[:-1] if name not in ("slots", "workspace") else None)
        else:
            bad.append(t.transpose(-1, -2).contiguous().transpose(-1, -2))         # rows that are columns
            bad += [t[:-1], t.narrow(t.dim() - 1, 0, t.shape[-1] - 1).contiguous()]
            if t.dim() == 3:
                bad.append(t[:, :-1].contiguous())
            if t.dim() > 2 and name not in ("k_new", "v_new", "k_out", "v_out", "scores"):
                bad.append(torch.stack((t, t), 1)[:, 0])                           # a view of a fused tensor
        bad = [b for b in bad if b is not None]
        assert bad
        if name == "workspace":
            bad = [torch.stack((t, t), 1)[:, 0]]
        for b in bad:
            assert "lychee_%s: %s is" % (method, name) in says(lb, p, method, dict(args, **{name: b})), (name, b.dtype, b.shape, b.stride())
    # a tensor of another device than the context's
    assert says(lb, p, method, args, device=0).startswith("lychee_%s: " % method)
    if "head_type_mask" in args:
        for m in (np.ones(7, np.uint8), np.ones((2, 4), np.uint8), np.full(8, 256), np.full(8, 0.5), np.full(8, -1)):
            assert "head_type_mask" in says(lb, p, method, dict(args, head_type_mask=m))
        for m in (np.ones(8, bool), np.ones(8), [1, 0, 0, 0, 1, 1, 1, 1], None):
            assert says(lb, p, method, dict(args, head_type_mask=m)).startswith(passed)


def test_layouts_that_the_binding_takes(lb):
    """Views that the calls read right: wide tables, interleaved layers, outputs of a larger batch, scores' first positions."""
    p = shape(lb, table_stride=6, page_tiles=6)
    a = arguments(lb, p)
    wide, pool = ints(2, 6), torch.zeros((10, 3, 2 * 2176), dtype=torch.uint8)
    for table in (wide, wide[:, :5], wide.view(-1), ints(3, 12)[:, :6], ints(3, 6), ints(10)):
        ok = table.dim() == 1 or table.stride(0) == 6
        said = says(lb, p, "q4_read", dict(a["q4_read"], block_table=table, cache=pool[:, 0]))
        assert said.startswith("lychee_q4_read failed") if ok else "block_table is" in said, (table.shape, table.stride())
    assert "block_table is" in says(lb, p, "q4_read", dict(a["q4_read"], block_table=ints(9), cache=pool[:, 0]))
    for cache, ok in ((pool[:, 2], True), (pool, True), (pool.view(-1)[2 * 4352:], True), (pool.view(-1)[2 * 4352 + 1:], False),
                      (torch.zeros((10, 2, 4352), dtype=torch.uint8)[:, 0], False), (pool.view(torch.int8)[:, 1], True)):
        said = says(lb, p, "q4_append", dict(a["q4_append"], cache=cache))
        assert said.startswith("lychee_q4_append failed") if ok else "cache is" in said, (cache.shape, cache.stride())
    p, a = shape(lb), arguments(lb, shape(lb))
    room = torch.zeros(2, 2, 80)
    tail = torch.zeros(4 * 80 - 17)                                              # 63 positions of the last row
    for x, ok in ((room, True), (room[..., :50], True), (torch.zeros(5, 2, 64), True), (torch.zeros(2, 3, 64), False),
                  (torch.zeros(2, 3, 64)[:, :2], False), (tail.as_strided((2, 2, 50), (160, 80, 1)), False),
                  (torch.zeros(2, 64), False)):
        for method in ("q4_decode_attn", "select_scores"):
            said = says(lb, p, method, dict(a[method], scores=x))
            assert said.startswith("lychee_%s failed" % method) if ok else "scores is" in said, (x.shape, x.stride())
    for method, names in (("release_pages", ("lengths_out", "free_count_out")), ("plan_pages", ("lengths_out", "free_count_out"))):
        assert says(lb, p, method, dict(a[method], **{n: None for n in names})).startswith("lychee_%s failed" % method)
    assert says(lb, p, "release_pages", dict(a["release_pages"], done=torch.zeros(2, dtype=torch.bool))).startswith("lychee_release_pages failed")
    assert says(lb, p, "q4_append", dict(a["q4_append"], slots=ints(8))).startswith("lychee_q4_append: k_new is")
    assert lb.check_paged(p, np.ones(7, np.uint8)) == lb.check_paged(p, np.full(8, 256)) == lb.EINVAL


@pytest.mark.parametrize("in_place", [True, False])
@pytest.mark.parametrize("method", ["release_pages", "plan_pages"])
def test_what_the_usual_and_the_other_way_pass_on(lb, method, in_place, monkeypatch):
    """A table that is not looked at first (a flat one) brings the call to the same arguments in the same places."""
    passed = []

    class Library:
        def __getattr__(self, name):
            return lambda *args: passed.append((name, args)) or 0

    p = shape(lb)
    a = arguments(lb, p)[method]
    if in_place:
        a.update(lengths_out=None, free_count_out=None)
    monkeypatch.setattr(lb, "_lib", Library())
    for table in (a["block_table"], a["block_table"].view(-1)):
        getattr(bound(lb), method)(p, stream=0, **dict(a, block_table=table))
    assert passed[0] == passed[1] and passed[0][0] == "lychee_" + method
    at = {k: None if t is None else t.data_ptr() for k, t in a.items()}
    at.update(lengths_out=at["lengths_out"] or at["lengths"], free_count_out=at["free_count_out"] or at["free_count"], n_slots=7)
    order = {"release_pages": "done lengths block_table free_pages free_count lengths_out free_count_out",
             "plan_pages": "lengths new_tokens block_table free_pages free_count lengths_out free_count_out slots n_slots token_start status"}
    assert list(passed[0][1][2:-1]) == [at[n] for n in order[method].split()]
    missing = dict(a, lengths=None, lengths_out=None)
    getattr(bound(lb), method)(p, stream=0, **missing)   # (None goes on to the library, which refuses it)
    assert passed[2][1][2:].count(None) == 3


# ------------------------------------------------------------------ the reference against hand-made values


def test_reference_format():
    x = np.zeros((1, 128))
    x[0, :8] = [6, -6, 0.25, 0.75, 1.25, 2.5, 3.5, 5]          # scale 1: ties go to the even code
    x[0, 32:34] = [6.0625, 1]                                 # just over 6: scale 2
    x[0, 64] = np.inf
    codes, scales = R.quantise(x)
    assert scales.tolist() == [[127, 128, 255, 2]]
    assert codes[0, :8].tolist() == [7, 15, 0, 2, 2, 4, 6, 6]
    back = R.dequantise(codes, scales)
    assert back[0, :8].tolist() == [6, -6, 0, 1, 1, 2, 4, 4]
    assert back[0, 32:34].tolist() == [6, 1]
    assert np.isnan(back[0, 64:96]).all() and (back[0, 96:] == 0).all()
    big = np.zeros((1, 128))
    big[0, 0] = 3.3895313892515355e38                          # bf16's largest: scale 2^125, 6 of them
    codes, scales = R.quantise(big)
    assert scales[0, 0] == 252 and R.dequantise(codes, scales)[0, 0] == 6 * 2.0 ** 125


def test_reference_cache_and_pool():
    c = R.Cache(3, 32, 2)
    rng = np.random.default_rng(0)
    k, v = R.quantise(rng.standard_normal((1, 128))), R.quantise(rng.standard_normal((1, 128)))
    c.write(2 * 32 + 17, 1, (k[0][0], k[1][0]), (v[0][0], v[1][0]))
    rows = c.rows([2 * 32 + 17, -1], 1)
    assert (rows[0, 0] == R.dequantise(*k)[0]).all() and (rows[1, 0] == R.dequantise(*v)[0]).all() and (rows[:, 1] == 0).all()
    pool = R.Pool([0, 1, 2, 3], 16, 4, 4)
    lengths, table = np.array([0, 16]), np.full((2, 4), -1)
    table[1, 0] = 9
    status, slots, start = pool.plan(lengths, [2, 17], table, 20)
    assert status == 0 and start.tolist() == [0, 2, 19] and lengths.tolist() == [2, 33]
    assert slots[:3].tolist() == [48, 49, 32] and slots[18] == 16 and slots[19] == -1 and pool.free == [0]
    assert pool.plan(lengths, [0, 31], table, 20)[0] == -2
    assert pool.plan(lengths, [0, 32], table, 40)[0] == -1
    assert pool.plan(lengths, [30, 20], table, 60)[0] == 1
    pool.release([0, 1], lengths, table)
    assert pool.free == [0, 9, 2, 1] and lengths.tolist() == [2, 0]
    assert R.top([1.0, 3.0, 3.0, np.nan, 0.0], 2).tolist() == [1, 2]
    assert R.top([1.0, 3.0, 3.0, 1.0], 3).tolist() == [0, 1, 2]
