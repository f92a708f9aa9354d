"""The paged 4-bit cache without a GPU: checks of its shape, every refusal of its calls (they come before anything is
launched, and before the context is looked into), and the reference itself against hand-made values."""
import ctypes

import numpy as np
import pytest

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
