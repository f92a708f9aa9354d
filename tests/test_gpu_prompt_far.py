"""Attention over prompts at the largest strides and at offsets beyond 32 bits: what a call reads and writes lies gigabytes apart, and the
rest of the memory is not touched (nor filled)."""
import pytest
import torch

from tests import prompt_norms as N
from tests.test_gpu_prompt import DEV, Packed, backward, binding, ctx, forward, ints, one_like, paged_case, q4  # noqa: F401

pytestmark = pytest.mark.gpu
FAR = 1 << 24  # elements, the largest stride of tokens and query heads


def far(x, tok, head):
    """A tensor [tokens, heads, 128] with these strides and x's values."""
    size = (x.shape[0] - 1) * tok + (x.shape[1] - 1) * head + 128
    return torch.empty(size, dtype=x.dtype, device=DEV).as_strided(x.shape, (tok, head, 1)).copy_(x)


@pytest.mark.parametrize("new, q_heads, kv_heads, tok, head", [
    ([150, 130], 2, 1, FAR, 128),              # a token's row 32 MB from the next: 4.7 G elements
    ([200], 4, 2, 128, FAR),                   # heads far apart
    ([70, 9], 8, 4, FAR, 4096 + 8),
])
def test_the_largest_strides(ctx, new, q_heads, kv_heads, tok, head):  # noqa: F811
    """The same bits as from rows side by side, forward and backward."""
    lb = binding()
    s = Packed(111, new, q_heads, kv_heads, sharp=1.2)
    g = one_like(s)
    out, lse, p, ws = forward(ctx, s)
    grads = backward(ctx, s, p, out, lse, ws, g).split((q_heads, kv_heads, kv_heads), 1)
    q, k, v = (far(x, tok, head) for x in (s.q, s.k, s.v))
    p = lb.make_prompt(len(new), q, k)
    assert lb.check_prompt(p) == lb.OK and p.q_stride_tok == tok == p.kv_stride_tok
    o, l = s.outputs()
    ctx.prompt_attn(p, q, k, v, s.d_start, None, o, l, ws)
    assert torch.equal(o, out) and torch.equal(l, lse)
    to = [far(torch.full_like(x, 5.0), tok, head) for x in (s.q, s.k, s.v)]
    ctx.prompt_attn_backward(p, g, q, k, v, o, l, s.d_start, *to, ws)
    torch.cuda.synchronize()
    for a, b in zip(to, grads):
        assert torch.equal(a, b)


def test_a_cache_of_more_than_32_bits(ctx):  # noqa: F811
    """[B][H][L_cap][128] of 4.3 G elements, its last head of its last request; and one token-major, 4.6 G elements along one head's keys."""
    s = Packed(112, [3, 70], 2, 2, sharp=1.2)
    k, v = (torch.empty((2, 2, 1 << 23, 128), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    lens = [90, 1300]
    for x in (k, v):
        for b, n in enumerate(lens):
            x[b, :, :n] = torch.randn((2, n, 128), device=DEV, generator=s.gen).bfloat16()
    out, lse, _, _ = forward(ctx, s, ints(lens), k, v)
    near, near_lse, _, _ = forward(ctx, s, ints(lens), k[:, :, :1300].contiguous(), v[:, :, :1300].contiguous())
    # (a wider cache may be cut otherwise: the sums' order, and with it the last bits, are its own)
    for h in range(2):
        for b, n in enumerate(lens):
            if s.new[b] >= 64:
                me = slice(int(s.start[b]), int(s.start[b + 1]))
                want = N.head(s.q[me, h].double(), k[b, h, :n].double(), v[b, h, :n].double(), torch.arange(n - s.new[b], n, device=DEV))
                N.near(out[me, h], want["out"], "out")
    # either is off by a rounding of its result and of its weights (2^-8), and sums in 32 bits by 2^-14 (tests/prompt_reference.py)
    most = max(x[b, :, :n].abs().max().item() for x in (v,) for b, n in enumerate(lens))
    assert ((out.float() - near.float()).abs() <= 2 * (2.0 ** -8 * near.float().abs() + (2.0 ** -8 + 2.0 ** -13) * most)).all()
    assert (lse - near_lse).abs().max() <= 2.0 ** -13
    del k, v
    s = Packed(113, [64], 1, 1, sharp=1.2)
    n = 140000
    rows = torch.empty((1, n, 256, 128), dtype=torch.bfloat16, device=DEV)
    rows[:, :, 254:] = torch.randn((1, n, 2, 128), device=DEV, generator=s.gen).bfloat16()
    k, v = rows[:, :, 254:255].transpose(1, 2), rows[:, :, 255:].transpose(1, 2)
    out, lse, _, _ = forward(ctx, s, ints([n]), k, v)
    want = N.head(s.q[:, 0].double(), k[0, 0].double(), v[0, 0].double(), torch.arange(n - 64, n, device=DEV))
    N.near(out[:, 0], want["out"], "out")


def test_pages_of_more_than_32_bits(ctx):  # noqa: F811
    """A paged cache of 4.6 GB whose last pages a request holds."""
    lb = binding()
    s, p, table, cache = paged_case(114, [70], [700], 4, 2, 256)
    want = q4(ctx, s, p, table, cache, [700])
    size = 66000
    big = lb.make_paged(1, 4, 2, size, 256, p.max_pages, 1, p.table_stride)
    data = torch.empty((size, big.page_tiles * lb.Q4_TILE_BYTES), dtype=torch.uint8, device=DEV)
    few = torch.from_numpy(cache.bytes).to(DEV).view(p.n_pages, -1)
    data[size - p.n_pages:] = few
    moved = ints(table)
    moved[moved >= 0] += size - p.n_pages
    assert int(moved.max()) * big.page_tiles * lb.Q4_TILE_BYTES > 1 << 32
    out, _ = s.outputs()
    ws = lb.alloc_q4_prompt_workspace(big, s.T)
    ctx.q4_prompt_attn(big, s.q, data, moved, ints([700]), s.d_start, out, ws)
    torch.cuda.synchronize()
    assert torch.equal(out, want)


def test_requests_that_share_pages(ctx):  # noqa: F811
    """Two requests whose tables begin with the same pages: a prompt's beginning kept once."""
    s, p, table, cache = paged_case(115, [40, 40], [200, 200], 4, 2, 64)
    table[1, :2] = table[0, :2]
    out = q4(ctx, s, p, table, cache, [200, 200])
    for b in range(2):
        one = Packed(115, [40], 4, 2)
        one.q.copy_(s.q[40 * b:40 * b + 40])
        mine = binding().make_paged(1, 4, 2, p.n_pages, 64, p.max_pages, 1, p.table_stride)
        got = q4(ctx, one, mine, table[b:b + 1], cache, [200])
        assert torch.equal(got, out[40 * b:40 * b + 40])
