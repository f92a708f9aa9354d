"""Attention over prompts without a GPU: checks of its shape, every refusal of its calls (they come before anything is launched,
and before the context is looked into), and the reference itself against differences."""
import ctypes

import numpy as np
import pytest
import torch

from tests import prompt_reference as R


@pytest.fixture(scope="module")
def lb():
    from paper_2602_04541_amd import binding
    return binding


def shape(lb, **kw):
    a = dict(batch=2, n_q_heads=8, n_kv_heads=2, head_dim=128, n_tokens=9, max_len=64, q_stride_tok=12 * 128, q_stride_head=128,
             kv_stride_batch=2 * 64 * 128, kv_stride_head=128, kv_stride_tok=12 * 128)
    a.update(kw)
    return lb.Prompt(**a)


def paged(lb, **kw):
    a = dict(batch=2, n_q_heads=8, n_kv_heads=2, n_pages=10, page_size=16, max_pages=4)
    a.update(kw)
    return lb.make_paged(**a)


def test_shapes(lb):
    assert lb.check_prompt(shape(lb)) == lb.OK
    for change in (dict(batch=0), dict(batch=-1), dict(n_q_heads=0), dict(n_q_heads=7), dict(n_kv_heads=0), dict(n_tokens=-1),
                   dict(max_len=-1), dict(q_stride_tok=120), dict(q_stride_tok=132), dict(q_stride_head=4), dict(q_stride_head=-128),
                   dict(kv_stride_tok=64), dict(kv_stride_tok=-256), dict(kv_stride_head=130), dict(kv_stride_batch=-8),
                   dict(kv_stride_batch=12)):
        assert lb.check_prompt(shape(lb, **change)) == lb.EINVAL, change
        assert lb.prompt_workspace_bytes(shape(lb, **change)) == 0
    for change in (dict(head_dim=64), dict(batch=257), dict(n_q_heads=34), dict(n_q_heads=65, n_kv_heads=65), dict(max_len=(1 << 24) + 1),
                   dict(q_stride_tok=(1 << 24) + 8), dict(q_stride_head=(1 << 24) + 8), dict(kv_stride_tok=(1 << 24) + 8),
                   dict(n_tokens=1 << 26), dict(n_tokens=1 << 26, n_q_heads=64, n_kv_heads=64)):
        assert lb.check_prompt(shape(lb, **change)) == lb.EUNSUPPORTED, change
        assert lb.prompt_workspace_bytes(shape(lb, **change)) == 0
    for change in (dict(n_tokens=0), dict(max_len=0), dict(n_q_heads=32), dict(max_len=1 << 24), dict(q_stride_tok=1 << 24),
                   dict(q_stride_head=0), dict(kv_stride_head=0), dict(kv_stride_batch=0), dict(n_tokens=(1 << 26) - 1)):
        assert lb.check_prompt(shape(lb, **change)) == lb.OK, change
        assert lb.prompt_workspace_bytes(shape(lb, **change)) > 0
    q, rows, cache = (torch.zeros(s, dtype=torch.bfloat16) for s in ((9, 12, 128), (9, 12, 128), (2, 2, 64, 128)))
    p = lb.make_prompt(2, q[:, :8], rows[:, 8:10])
    assert (p.n_q_heads, p.n_kv_heads, p.n_tokens, p.max_len) == (8, 2, 9, 0)
    assert (p.q_stride_tok, p.q_stride_head, p.kv_stride_batch, p.kv_stride_head, p.kv_stride_tok) == (1536, 128, 0, 128, 1536)
    p = lb.make_prompt(2, q[:, :8], cache)
    assert (p.n_kv_heads, p.max_len) == (2, 64)
    assert (p.kv_stride_batch, p.kv_stride_head, p.kv_stride_tok) == (16384, 8192, 128)


def test_workspace(lb):
    stats = lambda p: p.n_tokens * p.n_q_heads * 8  # noqa: E731
    many, long = shape(lb, n_tokens=1 << 20), shape(lb, max_len=1 << 20)
    for p in (shape(lb), many, long):
        n = lb.prompt_workspace_bytes(p)
        assert n >= stats(p) and n % 256 == 0
    for p in (many, long):                                             # (partials: as many as fill the device, however many tokens)
        assert lb.prompt_workspace_bytes(p) < stats(p) + (320 << 20)
    assert lb.prompt_workspace_bytes(long) > 1 << 20                   # few tiles over many keys
    assert lb.q4_prompt_workspace_bytes(paged(lb), 9) > 0
    assert lb.q4_prompt_workspace_bytes(paged(lb), 0) > 0
    assert lb.q4_prompt_workspace_bytes(paged(lb), -1) == 0
    assert lb.q4_prompt_workspace_bytes(paged(lb, n_q_heads=34), 9) == 0
    assert lb.q4_prompt_workspace_bytes(paged(lb, head_dim=64), 9) == 0
    with pytest.raises(lb.LycheeError):
        lb.alloc_prompt_workspace(shape(lb, batch=0), "cpu")
    with pytest.raises(lb.LycheeError):
        lb.alloc_q4_prompt_workspace(paged(lb, n_q_heads=34), 9, "cpu")


# Arguments of a call that would be accepted, by name.  Addresses are made up: a refused call touches none of them.
A = 1 << 20
WS = dict(ws=A, bytes=1 << 40, stream=None)
CALLS = {
    "lychee_prompt_attn": dict(q=A, k=A, v=A, start=A, lengths=A, out=A, lse=A, **WS),
    "lychee_prompt_attn_backward": dict(d_out=A, q=A, k=A, v=A, out=A, lse=A, start=A, dq=A, dk=A, dv=A, **WS),
    "lychee_q4_prompt_attn": dict(q=A, tok=1024, head=128, n=9, cache=A, table=A, lengths=A, start=A, out=A, **WS),
}
NULL = {
    "lychee_prompt_attn": "q k v start out",
    "lychee_prompt_attn_backward": "d_out q k v out lse start dq dk dv",
    "lychee_q4_prompt_attn": "q cache table lengths start out",
}
ODD = {
    "lychee_prompt_attn": dict(q=16, k=16, v=16, start=4, lengths=4, out=16, lse=4),
    "lychee_prompt_attn_backward": dict(d_out=16, q=16, k=16, v=16, out=16, lse=4, start=4, dq=16, dk=16, dv=16),
    "lychee_q4_prompt_attn": dict(q=16, cache=128, table=4, lengths=4, start=4, out=16),
}


def usual(lb, name, **kw):
    return (paged if "q4" in name else shape)(lb, **kw)


def refused(lb, name, p, ctx=True, **change):
    """The call's status, made on a context that must not be looked into (its bytes are no context)."""
    args = dict(CALLS[name])
    args.update(change)
    fake = ctypes.create_string_buffer(1 << 16)
    return getattr(lb._lib, name)(ctypes.addressof(fake) if ctx else None, ctypes.byref(p) if p is not None else None, *args.values())


@pytest.mark.parametrize("name", sorted(CALLS))
def test_null_and_misaligned_arguments_are_refused(lb, name):
    p = usual(lb, name)
    assert refused(lb, name, p, ctx=False) == lb.EINVAL
    assert refused(lb, name, None) == lb.EINVAL
    assert refused(lb, name, usual(lb, name, head_dim=64)) == lb.EUNSUPPORTED
    assert refused(lb, name, usual(lb, name, n_q_heads=7)) == lb.EINVAL
    assert refused(lb, name, usual(lb, name, n_q_heads=34)) == lb.EUNSUPPORTED   # 17 heads a KV head
    for arg in NULL[name].split():
        assert refused(lb, name, p, **{arg: None}) == lb.EINVAL, arg
    for arg, align in ODD[name].items():
        assert refused(lb, name, p, **{arg: A + align // 2}) == lb.EINVAL, arg
    assert refused(lb, name, p, ws=None) == lb.EWORKSPACE
    assert refused(lb, name, p, ws=A + 128) == lb.EWORKSPACE
    need = lb.q4_prompt_workspace_bytes(p, 9) if "q4" in name else lb.prompt_workspace_bytes(p)
    assert refused(lb, name, p, bytes=need - 1) == lb.EWORKSPACE


def test_sizes_that_are_refused(lb):
    for name in ("lychee_prompt_attn", "lychee_prompt_attn_backward"):
        assert refused(lb, name, shape(lb, n_tokens=0), q=None, k=None, v=None, out=None) == lb.OK   # nothing to do, nothing launched
        assert refused(lb, name, shape(lb, n_tokens=1 << 26)) == lb.EUNSUPPORTED
    # gradients of heads that share rows would overwrite one another
    assert refused(lb, "lychee_prompt_attn_backward", shape(lb, kv_stride_head=0)) == lb.EINVAL
    assert refused(lb, "lychee_prompt_attn_backward", shape(lb, q_stride_head=64)) == lb.EINVAL
    name, p = "lychee_q4_prompt_attn", paged(lb)
    assert refused(lb, name, p, n=-1) == lb.EINVAL
    assert refused(lb, name, p, n=0, q=None, out=None) == lb.OK
    assert refused(lb, name, p, n=1 << 26) == lb.EUNSUPPORTED
    for stride in (-8, 4, 129):
        assert refused(lb, name, p, tok=stride) == lb.EINVAL
        assert refused(lb, name, p, head=stride) == lb.EINVAL
    assert refused(lb, name, p, tok=120) == lb.EINVAL
    assert refused(lb, name, p, tok=(1 << 24) + 8) == lb.EUNSUPPORTED
    assert refused(lb, name, p, head=(1 << 24) + 8) == lb.EUNSUPPORTED
    assert refused(lb, name, paged(lb, table_stride=3)) == lb.EINVAL


# ------------------------------------------------------------------ what the binding refuses


def ints(*size):
    return torch.zeros(size, dtype=torch.int32)


def half(*size):
    return torch.zeros(size, dtype=torch.bfloat16)


def arguments(lb, cached):
    rows = half(9, 12, 128)
    q, k, v = rows.split((8, 2, 2), 1)
    if cached:
        k, v = half(2, 2, 64, 128), half(2, 2, 64, 128)
    p = lb.make_prompt(2, q, k)
    ws = lb.alloc_prompt_workspace(p, "cpu")
    grads = half(9, 12, 128).split((8, 2, 2), 1)
    return p, {
        "prompt_attn": dict(q=q, k=k, v=v, token_start=ints(3), lengths=ints(2) if cached else None, out=half(9, 8, 128),
                            lse=torch.zeros(8, 9), workspace=ws),
        "prompt_attn_backward": dict(d_out=half(9, 8, 128), q=q, k=k, v=v, out=half(9, 8, 128), lse=torch.zeros(8, 9), token_start=ints(3),
                                     dq=grads[0], dk=grads[1], dv=grads[2], workspace=ws),
        "q4_prompt_attn": dict(q=q, cache=torch.zeros((10, 2 * 2176), dtype=torch.uint8), block_table=ints(2, 4), lengths=ints(2),
                               token_start=ints(3), out=half(9, 8, 128), workspace=lb.alloc_q4_prompt_workspace(paged(lb), 9, "cpu")),
    }


def says(lb, p, method, args, device=-1):
    """What the call's error says: that the library refused it (there is no context), or which argument the binding did."""
    c = object.__new__(lb.Context)
    c._h, c.device = None, device
    with pytest.raises(lb.LycheeError) as e:
        getattr(c, method)(p, stream=0, **args)
    assert e.value.code == lb.EINVAL
    return str(e.value)


@pytest.mark.parametrize("method, cached", [("prompt_attn", False), ("prompt_attn", True), ("prompt_attn_backward", False), ("q4_prompt_attn", False)])
def test_the_binding_looks_at_types_sizes_layout_and_device(lb, method, cached):
    p, every = arguments(lb, cached)
    p = paged(lb) if "q4" in method else p
    args = every[method]
    passed = "lychee_%s failed" % method
    assert says(lb, p, method, args).startswith(passed)
    for name, t in args.items():
        if t is None or name in ("cache", "block_table"):
            continue
        bad = [t.to(torch.int64) if t.dtype == torch.int32 else t.to(torch.float16) if t.element_size() == 2 else None]
        if name == "workspace":
            bad = [torch.stack((t, t), 1)[:, 0]]
        elif t.dim() == 1:
            bad += [torch.stack((t, t), 1)[:, 0], t[:-1]]
        else:
            bad.append(t.transpose(-1, -2).contiguous().transpose(-1, -2))
            bad.append(t.narrow(t.dim() - 1, 0, t.shape[-1] - 1))
            if name != "q" or "q4" not in method:
                bad += [t[:-1], torch.stack((t, t), -2).flatten(-3, -2)[..., ::2, :] if t.dim() == 4 else t[:, :-1]]
        for x in (x for x in bad if x is not None):
            assert "lychee_%s: %s is" % (method, name) in says(lb, p, method, dict(args, **{name: x})), (name, x.dtype, x.shape, x.stride())
    assert says(lb, p, method, args, device=0).startswith("lychee_%s: " % method)
    for name in ("lse", "lengths"):  # (None goes on to the library)
        if name in args:
            assert says(lb, p, method, dict(args, **{name: None})).startswith("lychee_%s" % method)


def test_layouts_that_the_binding_takes(lb):
    p, every = arguments(lb, False)
    one = half(9, 1, 128)
    p1 = lb.make_prompt(2, half(9, 1, 128), half(9, 12, 128)[:, 4:5])       # a single head: its stride does not count
    a = dict(every["prompt_attn"], q=one.as_strided((9, 1, 128), (128, 8, 1)), k=half(9, 12, 128)[:, 4:5], v=half(9, 12, 128)[:, 5:6],
             out=one, lse=torch.zeros(1, 9))
    assert says(lb, p1, "prompt_attn", a).startswith("lychee_prompt_attn failed")
    p0 = lb.make_prompt(2, half(0, 8, 128), half(0, 2, 128))                # no tokens: nothing is launched, without a context too
    a = dict(every["prompt_attn"], q=half(0, 8, 128), k=half(0, 2, 128), v=half(0, 2, 128), out=half(0, 8, 128), lse=torch.zeros(8, 0))
    assert says(lb, p0, "prompt_attn", a).startswith("lychee_prompt_attn failed")


@pytest.mark.parametrize("method, cached", [("prompt_attn", False), ("prompt_attn", True), ("prompt_attn_backward", False)])
def test_usual_and_unusual_layouts_go_on_alike(lb, monkeypatch, method, cached):
    """One row: its stride to the next does not count, but the binding looks at such arguments one by one."""
    H, Hkv = 8, 2
    rows = half(1, 12, 128)
    q, k, v = rows.split((H, Hkv, Hkv), 1)
    if cached:
        k, v = half(1, Hkv, 64, 128), half(1, Hkv, 64, 128)
    p = lb.make_prompt(1, q, k)
    grads = half(1, 12, 128).split((H, Hkv, Hkv), 1)
    args = dict(q=q, k=k, v=v, token_start=ints(2), out=half(1, H, 128), lse=torch.zeros(H, 1), workspace=lb.alloc_prompt_workspace(p, "cpu"))
    args.update(dict(lengths=ints(1) if cached else None) if method == "prompt_attn" else dict(zip(("dq", "dk", "dv"), grads), d_out=half(1, H, 128)))
    passed = []

    class Library:
        def __getattr__(self, name):
            return lambda *a: passed.append((name,) + a) or 0

    monkeypatch.setattr(lb, "_lib", Library())
    c = object.__new__(lb.Context)
    c._h, c.device = None, -1
    getattr(c, method)(p, stream=0, **args)
    for name in ("q", "k", "dv"):
        if name in args:
            t = args[name]
            odd = t.as_strided(t.shape, (t.stride(0) + 8,) + t.stride()[1:], t.storage_offset())
            getattr(c, method)(p, stream=0, **dict(args, **{name: odd}))
    assert len(passed) >= 3 and all(x == passed[0] for x in passed)
    c._h = None


# ------------------------------------------------------------------ the reference


def test_reference_gradients_against_differences():
    rng = np.random.default_rng(3)
    n, h = 5, 1e-5
    q, k, v, g = (rng.standard_normal((n, 128)) for _ in range(4))
    pos = np.arange(n)
    got = R.head(q, k, v, pos, g)
    loss = lambda *x: (R.head(*x, pos)["out"][0] * g).sum()  # noqa: E731
    for name, at in (("dq", 0), ("dk", 1), ("dv", 2)):
        for _ in range(12):
            i, d = rng.integers(n), rng.integers(128)
            both = []
            for sign in (1, -1):
                x = [q.copy(), k.copy(), v.copy()]
                x[at][i, d] += sign * h
                both.append(loss(*x))
            # (the third derivative's part is h^2, rounding 2^-52 / h of a loss of some tens)
            assert abs((both[0] - both[1]) / (2 * h) - got[name][0][i, d]) < 1e-8


def test_reference_leaves_out_what_is_not_seen():
    rng = np.random.default_rng(4)
    q, k, v = (rng.standard_normal((4, 128)) for _ in range(3))
    want = R.head(q, k, v, np.array([-1, 0, 1, 9]))
    assert (want["out"][0][0] == 0).all() and want["lse"][0][0] == -np.inf
    assert np.allclose(want["out"][0][1], v[0])
    v[2:] = np.nan
    got = R.head(q, k, v, np.array([-1, 0, 1, 9]))
    assert (got["out"][0][:3] == want["out"][0][:3]).all() and np.isnan(got["out"][0][3]).all()


def test_reference_in_matrices():
    gen = torch.Generator().manual_seed(3)
    q, g = (torch.randn((9, 128), dtype=torch.float64, generator=gen) for _ in range(2))
    k, v = (torch.randn((30, 128), dtype=torch.float64, generator=gen) for _ in range(2))
    pos = torch.arange(21, 30)
    one, two = R.head(*(x.numpy() for x in (q, k, v, pos, g))), R.dense(q, k, v, pos, g)
    assert one.keys() == two.keys()
    for name in one:
        for a, b in zip(one[name], two[name]):
            assert abs(a - b.numpy()).max() <= 1e-12, name


def test_a_workspace_serves_smaller_calls(lb):
    """Fewer tokens, requests or keys need no more, whether a call shares its tiles out or not."""
    for batch in (1, 3, 256):
        for max_len in (1, 700, 5000, 1 << 20):
            sizes = [lb.prompt_workspace_bytes(shape(lb, batch=batch, n_tokens=n, max_len=max_len)) for n in (1, 77, 300, 2000, 5000, 70000, 1 << 20)]
            assert sizes == sorted(sizes) and sizes[0] > 0
        sizes = [lb.q4_prompt_workspace_bytes(paged(lb, batch=batch), n) for n in (0, 1, 77, 300, 2000, 70000)]
        assert sizes == sorted(sizes)
    for n in (1, 300, 5000):
        sizes = [lb.prompt_workspace_bytes(shape(lb, batch=b, n_tokens=n, max_len=m)) for b, m in ((1, 1), (1, 900), (2, 900), (2, 9000), (9, 9000), (256, 1 << 20))]
        assert sizes == sorted(sizes)
