"""Calls of attention over prompts that are refused on the host, without a GPU.  Calls that would be accepted are made without a
workspace, which is what they are refused for then: nothing is launched, and no context looked into."""
import itertools

import pytest
import torch

from tests.test_prompt_host import lb, paged, refused, shape  # noqa: F401

BACKWARD = "lychee_prompt_attn_backward"


def rows_meet(tokens, tok, heads, head):
    """Whether two of the rows [i * tok + h * head, + 128) have an element in common."""
    at = sorted(i * tok + h * head for i, h in itertools.product(range(tokens), range(heads)))
    return any(b - a < 128 for a, b in zip(at, at[1:]))


@pytest.mark.parametrize("tokens, tok, head", [
    (9, 1024, 128),            # as a projection leaves them
    (9, 1536, 128),
    (9, 128, 9 * 128),         # head after head
    (9, 160, 9 * 160),
    (9, 128, 128),             # every token's head where the next token's is
    (9, 128, 256),
    (9, 256, 128),
    (9, 896, 128),             # one head short of a row's
    (9, 1016, 128),            # eight elements short of it
    (9, 128, 8 * 128),         # one token short of a head's
    (9, 136, 136 * 8 + 120),
    (1, 128, 128),             # a single token
    (2, 128, 128),
    (2, 1000 * 8, 136),
    (3, 256, 384),             # rows that meet though neither stride holds all of the other's
    (2, 384, 256),
    (3, 16 * 128, 3 * 128),
    (5, 3 * 128, 5 * 128),     # and that do not
    (9, 128, 1 << 24),
    (0, 128, 128),
])
def test_gradients_whose_rows_meet_are_refused(lb, tokens, tok, head):  # noqa: F811
    """They would be written by several workgroups at once."""
    meet = rows_meet(tokens, tok, 8, head)
    p = shape(lb, n_tokens=tokens, q_stride_tok=tok, q_stride_head=head, kv_stride_tok=4096)
    assert refused(lb, BACKWARD, p, ws=None) == (lb.EINVAL if meet else lb.EWORKSPACE)
    assert refused(lb, "lychee_prompt_attn", p, ws=None) == lb.EWORKSPACE      # (reading them is no harm)
    p = shape(lb, n_q_heads=32, n_kv_heads=8, n_tokens=tokens, q_stride_tok=32 * 128, kv_stride_tok=tok, kv_stride_head=head)
    assert refused(lb, BACKWARD, p, ws=None) == (lb.EINVAL if meet else lb.EWORKSPACE)
    if meet:
        assert refused(lb, BACKWARD, p) == lb.EINVAL


def test_rows_that_meet_against_all_pairs(lb):  # noqa: F811
    for tokens, tok, head in itertools.product((2, 3, 7), range(128, 1200, 72), range(128, 1200, 56)):
        p = shape(lb, n_tokens=tokens, q_stride_tok=tok, q_stride_head=head, kv_stride_tok=4096)
        want = lb.EINVAL if rows_meet(tokens, tok, 8, head) else lb.EWORKSPACE
        assert refused(lb, BACKWARD, p, ws=None) == want, (tokens, tok, head)


def test_strides_of_key_heads_of_any_size(lb):  # noqa: F811
    for head in (1 << 40, 1 << 60, (1 << 63) - 8):
        p = shape(lb, kv_stride_tok=128, kv_stride_head=head)
        assert refused(lb, BACKWARD, p, ws=None) == lb.EWORKSPACE


# Arguments at addresses of their own, 16 MiB apart (made up: a refused call touches none of them).
OUTPUTS = {
    "lychee_prompt_attn": ("out lse", "q k v start lengths"),
    BACKWARD: ("dq dk dv", "d_out q k v out lse start"),
    "lychee_q4_prompt_attn": ("out", "q cache table lengths start"),
}


@pytest.mark.skipif(torch.cuda.is_available(), reason="an accepted call would be launched")
@pytest.mark.parametrize("name", sorted(OUTPUTS))
def test_outputs_at_the_address_of_another_argument_are_refused(lb, name):  # noqa: F811
    outputs, inputs = (x.split() for x in OUTPUTS[name])
    apart = {arg: (i + 1) << 24 for i, arg in enumerate(outputs + inputs)}
    p = paged(lb) if "q4" in name else shape(lb)
    ws = 1 << 30
    assert refused(lb, name, p, ws=ws, **apart) == lb.EHIP     # (taken, and no device to launch on)
    for i, out in enumerate(outputs):
        for other in outputs[:i] + inputs:
            assert refused(lb, name, p, ws=ws, **dict(apart, **{out: apart[other]})) == lb.EINVAL, (out, other)
        assert refused(lb, name, p, ws=apart[out], **apart) == lb.EINVAL, (out, "workspace")
    for arg in inputs:
        assert refused(lb, name, p, ws=apart[arg], **apart) == lb.EINVAL, (arg, "workspace")
    if name == BACKWARD:                                       # what is only read may be the same
        assert refused(lb, name, p, ws=ws, **dict(apart, d_out=apart["out"], q=apart["out"])) == lb.EHIP


@pytest.mark.parametrize("kv_heads, group, n", [(64, 4, 1 << 25), (64, 1, 1 << 26), (8, 16, 1 << 24), (8, 17, 9), (1, 4, 1 << 26)])
def test_sizes_without_a_workspace_are_those_that_are_refused(lb, kv_heads, group, n):  # noqa: F811
    """More tokens, heads or workgroups than a call over the paged cache takes: no size, and no buffer."""
    p = paged(lb, n_q_heads=kv_heads * group, n_kv_heads=kv_heads)
    name = "lychee_q4_prompt_attn"
    assert refused(lb, name, p, n=n, tok=1 << 20, ws=None) == lb.EUNSUPPORTED
    assert lb.q4_prompt_workspace_bytes(p, n) == 0
    with pytest.raises(lb.LycheeError) as e:
        lb.alloc_q4_prompt_workspace(p, n, "cpu")
    assert e.value.code == lb.EUNSUPPORTED
    fewer = max(1, n >> 3) if group <= 16 else 0
    if fewer:
        assert refused(lb, name, p, n=fewer, tok=1 << 20, ws=None) == lb.EWORKSPACE
        assert lb.q4_prompt_workspace_bytes(p, fewer) > 0


def half(*size):
    return torch.zeros(size, dtype=torch.bfloat16)


MAX = 1 << 24


@pytest.mark.parametrize("q, kv", [
    (half(8, 128, 1).permute(2, 0, 1), half(2, 128, 1).permute(2, 0, 1)),               # one token: a stride of 1
    (half(9, 128, 1).transpose(1, 2), half(9, 128, 1).transpose(1, 2)),                 # one head
    (half(9, 8, 128), half(2, 64, 128, 1).permute(3, 0, 1, 2)),                         # one request
    (half(9, 8, 128), half(1, 64, 128).unsqueeze(1)),
    (half(1, 8, 128), half(2, 2, 128, 1).permute(0, 1, 3, 2)),                          # a cache of one row
    (half(1, 8, 128), half(3, 128, 1).permute(0, 2, 1).unsqueeze(1)),                   # and one head
    (half(8 * 9 * 128).as_strided((9, 1, 128), (128, 2 * MAX, 1)), half(9, 1, 128)),    # one head of many that lie far apart
    (half(8, 128).as_strided((1, 8, 128), (2 * MAX, 128, 1)), half(1, 2, 128)),
])
def test_strides_of_dimensions_of_one_entry_do_not_count(lb, monkeypatch, q, kv):  # noqa: F811
    batch = kv.shape[0] if kv.dim() == 4 else 1
    p = lb.make_prompt(batch, q, kv)
    assert lb.check_prompt(p) == lb.OK
    for name, t, strides in (("q", q, (p.q_stride_tok, p.q_stride_head)), ("kv", kv, (p.kv_stride_tok, p.kv_stride_head))):
        dims = (0, 1) if t.dim() == 3 else (2, 1)
        assert all(t.shape[i] == 1 or t.stride(i) == s for i, s in zip(dims, strides)), name
    calls = []

    class Library:
        def __getattr__(self, name):
            return lambda *a: calls.append((name,) + a) or 0

    ws = lb.alloc_prompt_workspace(p, "cpu")
    monkeypatch.setattr(lb, "_lib", Library())
    c = object.__new__(lb.Context)
    c._h, c.device = None, -1
    T, H = q.shape[:2]
    start, lengths = torch.zeros(batch + 1, dtype=torch.int32), torch.zeros(batch, dtype=torch.int32)
    out, lse = half(T, H, 128), torch.zeros(H, T)
    c.prompt_attn(p, q, kv, kv, start, lengths if kv.dim() == 4 else None, out, lse, ws, stream=0)
    assert calls[-1][3:6] == (q.data_ptr(), kv.data_ptr(), kv.data_ptr())
    pg = lb.make_paged(1, H, kv.shape[1], 10, 16, 4)
    table, cache = torch.zeros((1, 4), dtype=torch.int32), torch.zeros((10, pg.page_tiles * lb.Q4_TILE_BYTES), dtype=torch.uint8)
    c.q4_prompt_attn(pg, q, cache, table, lengths[:1], start[:2], out, ws, stream=0)
    tok, head = calls[-1][4:6]
    assert calls[-1][3] == q.data_ptr() and 128 <= tok <= MAX and 0 <= head <= MAX and tok % 8 == 0 == head % 8
    assert (T == 1 or tok == q.stride(0)) and (H == 1 or head == q.stride(1))
    c._h = None
