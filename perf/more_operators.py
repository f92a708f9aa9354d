"""The calls that work on whole prompts: causal attention of packed sequences and of prompt pieces over a cache, its
gradient, and the same attention over the paged 4-bit cache, from a few tokens of a small model to a piece at 128K.

Request b of a batch has the query tokens token_start[b] .. token_start[b+1]-1 of the packed rows q [n_tokens, H_q, 128].
Its query number i sits at position p = L_b - n_b + i of the request's L_b keys (n_b query tokens; L_b = n_b where the keys
are packed like the queries) and attends, query head h with KV head h / (H_q / H_kv), to the positions up to its own:

    s_j = q . k_j / sqrt(128),  P_j = exp(s_j - lse),  lse = log sum_j exp s_j,  out = sum_j P_j v_j     (j <= p)

and with g the gradient of out, summed over the query heads of a KV head and over the queries:

    dP_j = g . v_j,  delta = g . out,  dS_j = P_j (dP_j - delta),
    dq = sum_j dS_j k_j / sqrt(128),  dk_j = sum dS_j q / sqrt(128),  dv_j = sum P_j g

A case is a dict of sizes:
  op        "prompt"  packed sequences; keys packed like the queries, or (`cached`) in a bf16 cache [B, H_kv, L_cap, 128]
            "train"   packed sequences, forward and backward
            "q4"      pieces of prompts over the paged 4-bit cache
  batch, q_heads, kv_heads
  new_lo, new_hi   query tokens of the requests are spread over this range ("q4": of every `chunked`-th, the others have one)
  len_lo, len_hi   keys they have in front of these ("q4" and `cached`)
  page             tokens of a page ("q4")

Lengths and token counts belong to the case; values and pages come from the seed.
"""
from __future__ import annotations

import math
import random

import torch

own = False

D = 128
TILE = 16
TILE_BYTES = 16 * 128 + 8 * 16
DEV = "cuda"


def _case(name=None, **kw):
    c = dict(op="prompt", batch=1, q_heads=32, kv_heads=8, new_lo=1, new_hi=1, len_lo=0, len_hi=0, cached=False, page=64, chunked=1)
    c.update(kw)
    c["new_lo"] = kw.get("new_lo", c["new_hi"])
    c["len_lo"] = kw.get("len_lo", c["len_hi"])
    if name is not None:
        c["name"] = name
    return c


def listed():
    return [
        # a short question to a small model: what a call costs at least
        _case("prompt_77", q_heads=8, kv_heads=2, new_hi=77),
        # a batch of ordinary prompts of unequal lengths
        _case("prompt_b16_short", batch=16, new_lo=61, new_hi=3001),
        # one long prompt
        _case("prompt_16k", new_hi=16384),
        # the last 32 decoded tokens once more, over a bf16 cache at 32K
        _case("prompt_cache_32_at_32k", new_hi=32, len_hi=32736, cached=True),
        # prompts that come in pieces, each over what its request holds already
        _case("prompt_cache_pieces", batch=4, new_lo=1021, new_hi=2048, len_lo=4099, len_hi=30011, cached=True),
        # a training batch of short texts, a small model
        _case("train_b4_short", op="train", batch=4, q_heads=8, kv_heads=2, new_lo=93, new_hi=311),
        # a training batch of packed documents
        _case("train_b8_4k", op="train", batch=8, new_lo=511, new_hi=4099),
        # one long document
        _case("train_8k", op="train", new_hi=8192),
        # a few tokens of a short conversation, a small model
        _case("q4_17_at_300", op="q4", q_heads=8, kv_heads=2, new_hi=17, len_hi=300),
        # the last 32 decoded tokens once more, at 128K
        _case("q4_32_at_128k", op="q4", new_hi=32, len_hi=131040),
        # a serving step: every sixteenth request brings a piece of its prompt, the others a token; eight heads a KV head
        _case("q4_b64_mixed", op="q4", batch=64, q_heads=64, page=16, new_lo=509, new_hi=2048, len_lo=61, len_hi=8191, chunked=16),
        # large pieces of long prompts
        _case("q4_b2_4k_at_64k", op="q4", batch=2, new_lo=4001, new_hi=4096, len_lo=32771, len_hi=61440, page=256),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the same ranges: any of the calls, 1 to 64 requests of 1 to 16K new tokens over up to 128K, 1 to 16 KV
    heads, groups of 1 to 16 query heads, pages of 16 to 256 tokens; sizes mostly odd."""
    op = rng.choice(["prompt", "prompt", "cached", "cached", "train", "train", "train", "q4", "q4", "q4"])
    kv = rng.choice([1, 2, 3, 4, 8, 8, 8, 16])
    group = rng.choice([1, 2, 4, 4, 4, 5, 8, 16] if kv < 8 else [1, 2, 4, 4, 4, 5, 8])
    batch = rng.choice([1, 1, 1, 2, 3, 8, 17, 64])
    new = _log(rng, 1 if op in ("cached", "q4") else 16, 16384)
    c = dict(op="prompt" if op == "cached" else op, cached=op == "cached", batch=batch, q_heads=kv * group, kv_heads=kv)
    c["page"] = rng.choice([16, 32, 64, 64, 128, 256]) if op == "q4" else 64
    c["chunked"] = rng.choice([1, 1, 4, 16]) if op == "q4" else 1
    spread, before = rng.uniform(0.05, 0.95), rng.uniform(0.05, 0.95)
    length = _log(rng, 16, 131072) if op in ("cached", "q4") else 0
    while True:
        c.update(new_hi=new, new_lo=max(1, int(new * spread)), len_hi=length, len_lo=int(length * before))
        w = work(_case(**c))
        if w["flops"] <= 2.0e12 and w["bytes"] <= 1.0e9:
            return _case(**c)
        if length > 2 * new:
            length = max(1, int(length * 0.8))
        else:
            new = max(1, int(new * 0.8))


# ------------------------------------------------------------------ what belongs to the case


def _spread(lo, hi, n, key):
    v = [hi if n == 1 else lo + (hi - lo) * i // (n - 1) for i in range(n)]
    random.Random(key).shuffle(v)
    return v


def _new(c):
    big = _spread(c["new_lo"], c["new_hi"], -(-c["batch"] // c["chunked"]), 3)
    return [big[b // c["chunked"]] if b % c["chunked"] == 0 else 1 for b in range(c["batch"])]


def _lengths(c):
    """Keys of the requests, their new tokens' among them."""
    return [a + b for a, b in zip(_spread(c["len_lo"], c["len_hi"], c["batch"], 7), _new(c))]


def _ceil(a, b):
    return -(-a // b)


def _max_pages(c):
    return _ceil(max(_lengths(c)), c["page"]) + 1


def work(case):
    c = case
    new, lens = _new(c), _lengths(c)
    pairs = sum(n * (L - n) + n * (n + 1) // 2 for n, L in zip(new, lens)) * c["q_heads"]
    rows = sum(new) * c["q_heads"] * D * 2
    keys = sum(lens) * c["kv_heads"] * (136 if c["op"] == "q4" else 4 * D)
    if c["op"] == "train":  # in: q, g, k, v; out: out, lse, dq, dk, dv
        return {"bytes": 4 * rows + 2 * keys + 4 * sum(new) * c["q_heads"], "flops": 14 * D * pairs}
    return {"bytes": 2 * rows + keys, "flops": 4 * D * pairs}


# ------------------------------------------------------------------ values


def _packed(n, heads, gen):
    return torch.randn((n, heads, D), dtype=torch.bfloat16, device=DEV, generator=gen)


def _quantised(n, gen):
    """n tiles of N(0, 1) tokens as the cache holds them."""
    out = torch.empty((n, TILE_BYTES), dtype=torch.uint8, device=DEV)
    edges = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0], device=DEV)
    for part in out.split(1 << 15):
        x = torch.randn((len(part), TILE, 8, 32), device=DEV, generator=gen)
        e = torch.ceil(torch.log2(x.abs().amax(-1) / 6))
        x = torch.ldexp(x, -e.unsqueeze(-1))
        code = (torch.bucketize(x.abs(), edges) + 8 * torch.signbit(x)).to(torch.uint8).flatten(1)
        part[:, :2048] = code[:, 0::2] | (code[:, 1::2] << 4)
        part[:, 2048:] = (e + 127).to(torch.uint8).transpose(1, 2).flatten(1)
    return out


def prepare(case, seed):
    c = case
    B, H, P = c["batch"], c["kv_heads"], c["page"]
    gen = torch.Generator(DEV)
    gen.manual_seed(seed)
    new, lens = _new(c), _lengths(c)
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device=DEV)  # noqa: E731
    start = [0]
    for n in new:
        start.append(start[-1] + n)
    T = start[-1]
    s = {"case": c, "start": ints(start), "lens": ints(lens)}
    sharp = torch.linspace(0.5, 2.5, c["q_heads"], device=DEV).view(1, -1, 1)  # heads look far and wide, or at a few tokens
    if c["op"] == "q4":
        s["q"] = (_packed(T, c["q_heads"], gen) * sharp).bfloat16()
        held = [_ceil(n, P) for n in lens]
        size = sum(held) + 8
        s["table"] = torch.full((B, _max_pages(c)), -1, dtype=torch.int32, device=DEV)
        mine = torch.arange(_max_pages(c), device=DEV) < ints(held).unsqueeze(1)
        s["table"][mine] = torch.randperm(size, device=DEV, generator=gen)[:sum(held)].int()
        s["cache"] = _quantised(size * H * (P // TILE), gen).view(size, -1)
    else:  # q, k and v as one projection leaves them
        rows = _packed(T, c["q_heads"] + 2 * H, gen)
        rows[:, :c["q_heads"]] = (rows[:, :c["q_heads"]] * sharp).bfloat16()
        s["rows"] = rows
        s["q"], s["k"], s["v"] = rows.split((c["q_heads"], H, H), 1)
        if c["cached"]:
            cap = _ceil(max(lens), 64) * 64
            s["k"], s["v"] = (torch.randn((B, H, cap, D), dtype=torch.bfloat16, device=DEV, generator=gen) for _ in range(2))
    s["out"] = torch.zeros((T, c["q_heads"], D), dtype=torch.bfloat16, device=DEV)
    if c["op"] == "train":
        s["g"] = _packed(T, c["q_heads"], gen)
        s["lse"] = torch.zeros((c["q_heads"], T), device=DEV)
        s["grads"] = torch.zeros_like(s["rows"])
    return s


# ------------------------------------------------------------------ the plain forms


def _of_pages(s, c, b, L):
    """K and V [H, L, 128] of a request, in 32 bits."""
    H, t = c["kv_heads"], c["page"] // TILE
    pages = s["table"][b, :_ceil(L, c["page"])].long()
    tiles = s["cache"].view(-1, H, t, TILE_BYTES)[pages].transpose(0, 1).reshape(H, -1, TILE_BYTES)
    code = tiles[..., :2048]
    grid = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6, 0, -0.5, -1, -1.5, -2, -3, -4, -6], device=DEV)
    x = grid[torch.stack((code & 15, code >> 4), -1).int()].view(H, -1, 8, 32)
    scale = torch.exp2(tiles[..., 2048:].unflatten(-1, (8, TILE)).transpose(2, 3).reshape(H, -1, 8, 1).float() - 127)
    x = (x * scale).flatten(2)[:, :L]
    return x[..., :D], x[..., D:]


def _keys(s, c, b, first, n, L):
    if c["op"] == "q4":
        return _of_pages(s, c, b, L)
    if c["cached"]:
        return s["k"][b, :, :L].float(), s["v"][b, :, :L].float()
    return s["k"][first:first + n].float().transpose(0, 1), s["v"][first:first + n].float().transpose(0, 1)


def _plain(s):
    c = s["case"]
    H, G, scale = c["kv_heads"], c["q_heads"] // c["kv_heads"], 1 / math.sqrt(D)
    grads = s["grads"].view(len(s["grads"]), -1, D) if c["op"] == "train" else None
    at = 0
    for b, (n, L) in enumerate(zip(_new(c), _lengths(c))):
        k, v = _keys(s, c, b, at, n, L)
        here = slice(at, at + n)
        at += n
        hidden = (torch.arange(L, device=DEV) > torch.arange(L - n, L, device=DEV).unsqueeze(1)).repeat(G, 1)
        step = max(1, (1 << 30) // (G * n * L))  # as many heads at a time as memory takes
        for h in range(0, H, step):
            m = min(step, H - h)
            heads = slice(h * G, (h + m) * G)
            rows = lambda x: x[here, heads].float().transpose(0, 1).reshape(m, G * n, D)  # noqa: E731, B023
            q, kh, vh = rows(s["q"]), k[h:h + m], v[h:h + m]
            z = (torch.matmul(q, kh.transpose(1, 2)) * scale).masked_fill_(hidden, -math.inf)
            top = z.amax(-1, keepdim=True)
            p = z.sub_(top).exp_()
            total = p.sum(-1, keepdim=True)
            p = p.div_(total)
            o = torch.matmul(p, vh)
            s["out"][here, heads] = o.view(m * G, n, D).transpose(0, 1).bfloat16()
            if grads is None:
                continue
            s["lse"][heads, here] = (top + total.log()).view(m * G, n)
            g = rows(s["g"])
            grads[here, H * G + H + h:H * G + H + h + m] = torch.matmul(p.transpose(1, 2), g).transpose(0, 1).bfloat16()
            ds = torch.matmul(g, vh.transpose(1, 2)).sub_((g * o).sum(-1, keepdim=True)).mul_(p).mul_(scale)
            grads[here, heads] = torch.matmul(ds, kh).view(m * G, n, D).transpose(0, 1).bfloat16()
            grads[here, H * G + h:H * G + h + m] = torch.matmul(ds.transpose(1, 2), q).transpose(0, 1).bfloat16()
    return _named(s)


def _named(s):
    c = s["case"]
    if c["op"] != "train":
        return {"out": s["out"]}
    dq, dk, dv = s["grads"].split((c["q_heads"], c["kv_heads"], c["kv_heads"]), 1)
    return {"out": s["out"], "lse": s["lse"], "dq": dq, "dk": dk, "dv": dv}


# ------------------------------------------------------------------ the framework's calls

_context = []


def _own(s):
    from paper_2602_04541_amd import binding as lb
    c = s["case"]
    if not _context:
        _context.append(lb.Context(0))
    ctx = _context[0]
    if c["op"] == "q4":
        if "paged" not in s:  # what a program keeps beside its cache: the shape, and the workspace of its calls
            s["paged"] = lb.make_paged(c["batch"], c["q_heads"], c["kv_heads"], s["cache"].shape[0], c["page"], _max_pages(c))
            s["ws"] = lb.alloc_q4_prompt_workspace(s["paged"], len(s["q"]), DEV)
        ctx.q4_prompt_attn(s["paged"], s["q"], s["cache"], s["table"], s["lens"], s["start"], s["out"], s["ws"])
        return _named(s)
    if "prompt" not in s:
        s["prompt"] = lb.make_prompt(c["batch"], s["q"], s["k"])
        s["ws"] = lb.alloc_prompt_workspace(s["prompt"], DEV)
    ctx.prompt_attn(s["prompt"], s["q"], s["k"], s["v"], s["start"], s["lens"] if c["cached"] else None, s["out"], s.get("lse"), s["ws"])
    if c["op"] == "train":
        dq, dk, dv = s["grads"].split((c["q_heads"], c["kv_heads"], c["kv_heads"]), 1)
        ctx.prompt_attn_backward(s["prompt"], s["g"], s["q"], s["k"], s["v"], s["out"], s["lse"], s["start"], dq, dk, dv, s["ws"])
    return _named(s)


def run(state):
    return _own(state) if own else _plain(state)


# ------------------------------------------------------------------ the same in 64 bits


def _decoded(rows, scales):
    """What 64 packed bytes a row stand for under four scale bytes a row."""
    value = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], dtype=torch.float64, device=DEV)
    out = torch.empty((len(rows), D), dtype=torch.float64, device=DEV)
    for half, nibble in ((0, rows % 16), (1, rows // 16)):
        out[:, half::2] = torch.where(nibble >= 8, -1.0, 1.0) * value[(nibble % 8).long()]
    return out * torch.pow(2.0, scales.double() - 127).repeat_interleave(32, 1)


def exact(case, seed):
    c = case
    s = prepare(c, seed)
    H, G, Hq = c["kv_heads"], c["q_heads"] // c["kv_heads"], c["q_heads"]
    T = len(s["q"])
    zeros = lambda *shape: torch.zeros(shape, dtype=torch.float64, device=DEV)  # noqa: E731
    out, lse, dq, dk, dv = zeros(T, Hq, D), zeros(Hq, T), zeros(T, Hq, D), zeros(T, H, D), zeros(T, H, D)
    at = 0
    for b, (n, L) in enumerate(zip(_new(c), _lengths(c))):
        for kv in range(H):
            if c["op"] == "q4":
                tiles = s["cache"].view(s["cache"].shape[0], H, -1, TILE_BYTES)[s["table"][b, :_ceil(L, c["page"])].long(), kv].reshape(-1, TILE_BYTES)
                rows = tiles[:, :2048].reshape(-1, 128)[:L]
                scales = tiles[:, 2048:].reshape(-1, 8, 16).permute(0, 2, 1).reshape(-1, 8)[:L]
                K, V = _decoded(rows[:, :64], scales[:, :4]), _decoded(rows[:, 64:], scales[:, 4:])
            elif c["cached"]:
                K, V = s["k"][b, kv, :L].double(), s["v"][b, kv, :L].double()
            else:
                K, V = s["k"][at:at + n, kv].double(), s["v"][at:at + n, kv].double()
            for h in range(kv * G, (kv + 1) * G):
                for lo in range(0, n, 4096):
                    hi = min(n, lo + 4096)
                    me, seen = slice(at + lo, at + hi), L - n + hi
                    q = s["q"][me, h].double()
                    logit = q @ K[:seen].T / math.sqrt(D)
                    logit += torch.full_like(logit, -math.inf).triu(L - n + lo + 1)
                    lse[h, me] = logit.logsumexp(1)
                    p = torch.exp(logit - lse[h, me].unsqueeze(1))
                    out[me, h] = p @ V[:seen]
                    if c["op"] == "train":
                        g = s["g"][me, h].double()
                        ds = p * (g @ V[:seen].T - (g * out[me, h]).sum(1, keepdim=True)) / math.sqrt(D)
                        dq[me, h] = ds @ K[:seen]
                        dk[at:at + seen, kv] += ds.T @ q
                        dv[at:at + seen, kv] += p.T @ g
        at += n
    return {"out": out, "lse": lse, "dq": dq, "dk": dk, "dv": dv} if c["op"] == "train" else {"out": out}
