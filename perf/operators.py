"""Performance cases of the operators that surround a Test-Time Control block in a decoder layer: rotary positions, the paged
key-value cache in 4 bits and the attention over it.

Families (``case["op"]``):

    rope        ttc_rope, or with backward=True ttc_rope_backward: positions of a tensor of heads
    append      ttc_kv_append (keys rotated and quantised, values quantised, queries rotated: one launch), and ttc_kv_read of
                the same tokens, which gives what the cache holds as numbers
    attention   ttc_attention over a paged cache: single tokens (q = 1), or prompts and chunks of them

With ``own`` false the same results come from elementary torch operations in float32.  Sequence lengths are a function of the
case alone; values, page orders and positions are drawn from the seed.
"""
from __future__ import annotations

import math

import torch

DEV = "cuda:0"
own = False

GRID = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)   # magnitudes of a 4-bit code; bit 3 is the sign
BLOCK = 32                                        # entries of a head that share one exponent byte


def listed():
    return [
        # One decoding step of 32 sequences far into their contexts, 32 heads of 128: launch latency.
        dict(name="rope_decode", op="rope", tokens=32, heads=32, of=32, d=128, rot=128, layout="half", dtype="bf16",
             backward=False, far=131072),
        # Prompt of 2 x 8192 tokens: 32 query and 8 key heads rotated where the fused projection left them (its 8 value heads lie behind).
        dict(name="rope_prompt", op="rope", tokens=16384, heads=40, of=48, d=128, rot=128, layout="half", dtype="bf16",
             backward=False, far=8192),
        # Training step in float32: gradient of 16 heads of 64 of which one half is rotated, odd number of tokens.
        dict(name="rope_part_backward", op="rope", tokens=4099, heads=16, of=16, d=64, rot=32, layout="interleaved",
             dtype="f32", backward=True, far=4099),
        # One decoding step of 32 sequences: a token each to its page.
        dict(name="append_decode", op="append", tokens=32, heads_q=32, heads=8, d=128, page=64, rot=128, layout="half",
             dtype="bf16", far=131072),
        # Prompt of 2 x 8192 tokens.
        dict(name="append_prompt", op="append", tokens=16384, heads_q=32, heads=8, d=128, page=64, rot=128, layout="half",
             dtype="bf16", far=8192),
        # float32 features, 16 heads of 64, small pages, an odd number of tokens, half of each head rotated.
        dict(name="append_small_head", op="append", tokens=4099, heads_q=16, heads=16, d=64, page=16, rot=32,
             layout="interleaved", dtype="f32", far=4099),
        # One sequence's next token after 4099 others: latency.
        dict(name="attn_decode_one", op="attention", seqs=1, kv_lo=4099, kv_hi=4099, q_lo=1, q_hi=1, heads_q=32, heads=8, d=128,
             page=64, window=0, dtype="bf16"),
        # A serving batch: 64 sequences between 257 and 16384 tokens.
        dict(name="attn_decode_batch", op="attention", seqs=64, kv_lo=257, kv_hi=16384, q_lo=1, q_hi=1, heads_q=32, heads=8,
             d=128, page=64, window=0, dtype="bf16"),
        # Few sequences with long contexts.
        dict(name="attn_decode_long", op="attention", seqs=4, kv_lo=131072, kv_hi=131072, q_lo=1, q_hi=1, heads_q=32, heads=8,
             d=128, page=256, window=0, dtype="bf16"),
        # float32, a cache head for every query head, small pages, contexts from nothing to 4099 tokens.
        dict(name="attn_decode_f32", op="attention", seqs=24, kv_lo=0, kv_hi=4099, q_lo=1, q_hi=1, heads_q=16, heads=16, d=64,
             page=16, window=0, dtype="f32"),
        # A chunk of 4096 prompt tokens behind 8192 that the cache holds already.
        dict(name="attn_prompt_chunk", op="attention", seqs=1, kv_lo=12288, kv_hi=12288, q_lo=4096, q_hi=4096, heads_q=32,
             heads=8, d=128, page=64, window=0, dtype="bf16"),
        # Eight short prompts of odd lengths, 64-wide heads, one cache head, a sliding window.
        dict(name="attn_prompt_ragged", op="attention", seqs=8, kv_lo=301, kv_hi=2047, q_lo=17, q_hi=1500, heads_q=16, heads=1,
             d=64, page=32, window=512, dtype="bf16"),
    ]


def _log(rng, lo, hi):
    """A whole number between lo and hi, spread over the logarithm; odd ones as likely as even ones."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    """A case of the same families: any supported head, lengths spread over the listed range."""
    op = rng.choice(["rope", "append", "attention", "attention", "attention", "attention"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if op == "rope":
        d = rng.choice([64, 80, 96, 128, 256])
        heads = rng.randint(1, 40)
        rot = rng.choice([d, d, d // 2, d // 4])
        tokens = _log(rng, 1, max(1, min(32768, 40_000_000 // (heads * d))))
        return dict(op=op, tokens=tokens, heads=heads, of=heads + rng.choice([0, 0, 8]), d=d, rot=rot,
                    layout=rng.choice(["half", "interleaved"]), dtype=dtype, backward=rng.random() < 0.5, far=_log(rng, 1, 131072))
    d = rng.choice([64, 128, 128, 256])
    page = rng.choice([16, 32, 64, 128, 256])
    heads = rng.choice([1, 2, 4, 5, 8, 16])
    if op == "append":
        tokens = _log(rng, 1, 8388608 // (heads * d))
        return dict(op=op, tokens=tokens, heads_q=heads * rng.choice([1, 2, 4]), heads=heads, d=d, page=page,
                    rot=rng.choice([d, d, d // 2]), layout=rng.choice(["half", "interleaved"]), dtype=dtype,
                    far=_log(rng, 1, 131072))
    heads_q = heads * rng.choice([1, 2, 3, 4, 7, 8, 16])
    if heads_q > 64:
        heads_q = heads * (64 // heads)
    if rng.random() < 0.6:      # decoding
        seqs = _log(rng, 1, 128)
        kv_hi = _log(rng, 1, max(1, min(131072, 400_000_000 // (seqs * heads * d))))
        return dict(op=op, seqs=seqs, kv_lo=rng.choice([0, max(0, kv_hi // 8), kv_hi]), kv_hi=kv_hi, q_lo=1, q_hi=1, heads_q=heads_q,
                    heads=heads, d=d, page=page, window=rng.choice([0, 0, 0, 1024]), dtype=dtype)
    seqs = _log(rng, 1, 8)      # a few tokens a sequence, prompts
    kv_hi = _log(rng, 2, 8192 // seqs)
    q_hi = _log(rng, 2, max(2, min(kv_hi, 4096, 160_000_000_000 // (seqs * kv_hi * heads_q * d))))
    return dict(op=op, seqs=seqs, kv_lo=rng.choice([max(1, kv_hi // 4), kv_hi]), kv_hi=kv_hi, q_lo=rng.choice([1, q_hi]), q_hi=q_hi,
                heads_q=heads_q, heads=heads, d=d, page=page, window=rng.choice([0, 0, 256]), dtype=dtype)


def _spread(lo, hi, n):
    """n whole numbers between lo and hi, both ends among them (hi alone where n is 1), in no order."""
    at = [(i * 0.6180339887498949) % 1.0 for i in range(n)]
    first, last = min(at), max(at)
    return [hi if n == 1 else lo + int(round((hi - lo) * (a - first) / (last - first))) for a in at]


def _lengths(case):
    """(tokens in the cache, new tokens) of each sequence: the new ones are the last of those in the cache."""
    kv = _spread(case["kv_lo"], case["kv_hi"], case["seqs"])
    q = _spread(case["q_lo"], case["q_hi"], case["seqs"])
    return kv, q


def _visible(kv, q, window):
    """Pairs of a query and a key that it sees, for one sequence: query i is token kv - q + i."""
    last = [kv - q + i + 1 for i in range(q)]
    return sum(max(0, min(n, window) if window else n) for n in last)


# ---------------------------------------------------------------------------------------------------------------
# inputs

def _gen(seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    return gen


def _type(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _table(rows, rot):
    """cos and sin of position times frequency, formed in float64: (rows, rot / 2, 2)."""
    freq = 10000.0 ** (-torch.arange(0, rot, 2, device=DEV, dtype=torch.float64) / rot)
    angle = torch.arange(rows, device=DEV, dtype=torch.float64)[:, None] * freq
    return torch.stack([angle.cos(), angle.sin()], -1).float()


def _heads(gen, n, heads, d, dtype):
    """Features of n tokens, some channels larger than others as a projection leaves them."""
    channel = torch.exp(0.5 * torch.randn((heads, d), generator=gen, device=DEV))
    return (torch.randn((n, heads, d), generator=gen, device=DEV) * channel).to(dtype)


def _views(cache, d):
    """The four parts of a cache (pages, heads, page * (d + d / 16) bytes): codes of the keys (.., token, d / 2), codes of the
    values (.., four tokens, lane of 16, token of the four, d / 32), exponents of the keys (.., token, d / 32) and of the values
    (.., four tokens, d / 32, token of the four)."""
    pages, heads, nbytes = cache.shape
    page = nbytes // (d + d // 16)
    code, exp = page * d // 2, page * d // BLOCK
    lead = (pages, heads)
    return (cache[..., :code].view(*lead, page, d // 2), cache[..., code:2 * code].view(*lead, page // 4, 16, 4, d // 32),
            cache[..., 2 * code:2 * code + exp].view(*lead, page, d // BLOCK),
            cache[..., 2 * code + exp:].view(*lead, page // 4, d // BLOCK, 4))


def _quantise(x):
    """Codes (0 .. 15, uint8) and exponent bytes of the blocks of 32 of the last axis of a float32 tensor."""
    b = x.reshape(*x.shape[:-1], x.shape[-1] // BLOCK, BLOCK)
    bits = b.abs().amax(-1).view(torch.int32)
    e = torch.where(bits >= 0x7f800000, 255, (((bits + 0x200000) >> 23) - 2).clamp_(min=0))
    inverse = ((254 - e.clamp(max=253)) << 23).view(torch.float32)
    y = (b * inverse[..., None]).abs()
    m = torch.where(y < 2, torch.round(2 * y), torch.where(y < 4, torch.round(y) + 2, torch.round(0.5 * y).clamp(max=3) + 4))
    code = torch.where(torch.isfinite(m), m, 0).to(torch.uint8) | (torch.signbit(b).to(torch.uint8) << 3)
    return code.reshape(x.shape), e.to(torch.uint8)


def _pack(code):
    """Two codes to a byte, the first in the low half."""
    return code[..., 0::2] | (code[..., 1::2] << 4)


def _values(packed, e):
    """The float32 numbers that packed codes (.., d / 2) and exponents (.., d / 32) stand for."""
    grid = torch.tensor(GRID + tuple(-g for g in GRID), device=packed.device)
    code = torch.stack([packed & 15, packed >> 4], -1).reshape(*packed.shape[:-1], -1)
    scale = torch.where(e == 255, math.nan, torch.exp2(e.float() - 127.0))
    x = grid[code.int()]
    return (x.view(*x.shape[:-1], e.shape[-1], BLOCK) * scale[..., None]).view(x.shape)


def _fill(gen, pages, heads, page, d):
    """A cache whose every token was written by a model: keys with channels of unlike size, values without."""
    cache = torch.empty((pages, heads, page * (d + d // 16)), dtype=torch.uint8, device=DEV)
    kc, vc, ke, ve = _views(cache, d)
    x = torch.randn((pages, heads, page, d), generator=gen, device=DEV)
    code, e = _quantise(x * torch.exp(0.5 * torch.randn((heads, 1, d), generator=gen, device=DEV)))
    kc.copy_(_pack(code))
    ke.copy_(e)
    code, e = _quantise(x.normal_(generator=gen))
    vc.copy_(_pack(code).view(pages, heads, page // 4, 4, 16, d // 32).transpose(3, 4))
    ve.copy_(e.view(pages, heads, page // 4, 4, d // BLOCK).transpose(3, 4))
    return cache


def prepare(case, seed):
    op, d, dtype, gen = case["op"], case["d"], _type(case), _gen(seed)
    if op == "rope":
        x = _heads(gen, case["tokens"], case["of"], d, dtype)[:, :case["heads"]]
        positions = torch.randint(0, case["far"], (case["tokens"],), generator=gen, device=DEV)
        return dict(op=op, x=x, positions=positions, table=_table(case["far"], case["rot"]), layout=case["layout"],
                    backward=case["backward"])
    page, heads, heads_q = case["page"], case["heads"], case["heads_q"]
    if op == "append":
        n = case["tokens"]
        k, v, q = (_heads(gen, n, h, d, dtype) for h in (heads, heads, heads_q))
        if n <= 128:    # a token of each of n sequences
            pages = n + 1
            slots = torch.randperm(pages, generator=gen, device=DEV)[:n] * page + torch.randint(0, page, (n,), generator=gen, device=DEV)
            positions = torch.randint(0, case["far"], (n,), generator=gen, device=DEV)
        else:           # a prompt that begins inside a page
            start = 3
            pages = (start + n + page - 1) // page + 1
            at = torch.arange(start, start + n, device=DEV)
            slots = torch.randperm(pages, generator=gen, device=DEV)[at // page] * page + at % page
            positions = torch.arange(n, device=DEV) % case["far"]
        cache = torch.randint(0, 256, (pages, heads, page * (d + d // 16)), generator=gen, device=DEV, dtype=torch.uint8)
        return dict(op=op, d=d, cache=cache, k=k, v=v, q=q, slots=slots, positions=positions,
                    table=_table(case["far"], case["rot"]), layout=case["layout"])
    kv, new = _lengths(case)
    count = [-(-n // page) for n in kv]
    total, width = sum(count) + 1, max(1, max(count))
    cache = _fill(gen, total, heads, page, d)
    order = torch.randperm(total, generator=gen, device=DEV).to(torch.int32).cpu()
    table, at = torch.full((len(kv), width), -1, dtype=torch.int32), 0
    for i, c in enumerate(count):
        table[i, :c] = order[at:at + c]
        at += c
    # what lies behind a sequence's last token in its last page was never written: any bytes, NaN among them
    ends = [(int(table[i, c - 1]), n % page // 4 * 4 + 4) for i, (n, c) in enumerate(zip(kv, count)) if n % page]
    for p, first in ends:
        for part in _views(cache, d)[0::2]:
            part[p, :, first:] = 255
        for part in _views(cache, d)[1::2]:
            part[p, :, first // 4:] = 255
    q = _heads(gen, sum(new), heads_q, d, dtype)
    cu = torch.tensor([0] + new, dtype=torch.int32).cumsum(0, dtype=torch.int32)
    return dict(op=op, d=d, q=q, cache=cache, table=table.to(DEV), kv_len=torch.tensor(kv, dtype=torch.int32, device=DEV),
                cu_q=None if max(new) == 1 and min(new) == 1 else cu.to(DEV), max_q=max(new), max_kv=max(kv),
                scale=1.0 / math.sqrt(d), window=case["window"])


# ---------------------------------------------------------------------------------------------------------------
# one pass

def _plain_rope(x, positions, table, layout, backward=False):
    """float32 rotation of the first entries of each head of x (tokens, heads, d), by the table's row of each token."""
    half = table.shape[1]
    cos, sin = table[positions][:, None].unbind(-1)
    if backward:
        sin = -sin
    x = x.float()
    part = x[..., :2 * half]
    a, b = (part[..., :half], part[..., half:]) if layout == "half" else (part[..., 0::2], part[..., 1::2])
    y = (a * cos - b * sin, b * cos + a * sin)
    y = torch.cat(y, -1) if layout == "half" else torch.stack(y, -1).flatten(-2)
    return torch.cat([y, x[..., 2 * half:]], -1)


def _plain_append(s):
    d, cache, n = s["d"], s["cache"], s["k"].shape[0]
    heads = s["k"].shape[1]
    kc, vc, ke, ve = _views(cache, d)
    page = kc.shape[2]
    p, t = s["slots"] // page, s["slots"] % page
    code, e = _quantise(_plain_rope(s["k"], s["positions"], s["table"], s["layout"]))
    kc[p, :, t] = _pack(code)
    ke[p, :, t] = e
    code, e = _quantise(s["v"].float())
    vc[p, :, t // 4, :, t % 4] = _pack(code).view(n, heads, 16, d // 32)
    ve[p, :, t // 4, :, t % 4] = e
    k = _values(kc[p, :, t], ke[p, :, t])
    v = _values(vc[p, :, t // 4, :, t % 4].reshape(n, heads, d // 2), ve[p, :, t // 4, :, t % 4])
    q = _plain_rope(s["q"], s["positions"], s["table"], s["layout"])
    return {"q": q.to(s["q"].dtype), "k": k.to(torch.bfloat16), "v": v.to(torch.bfloat16)}


def _plain_attention(s):
    d, q, table, kv_len = s["d"], s["q"], s["table"], s["kv_len"].long()
    seqs, width = table.shape
    tokens, heads_q, _ = q.shape
    kc, vc, ke, ve = _views(s["cache"], d)
    heads, page = kc.shape[1], kc.shape[2]
    group, length, most = heads_q // heads, width * page, s["max_q"]
    at = table.clamp(min=0).long()
    j = torch.arange(length, device=q.device)

    def rows(x):        # (seqs, pages, heads, page, ..) -> (seqs, heads, tokens, ..)
        return x.transpose(1, 2).reshape(seqs, heads, length, x.shape[-1])

    there = (j < kv_len[:, None])[:, None, :, None]
    k = torch.where(there, _values(rows(kc[at]), rows(ke[at])), 0.0)
    values = vc[at].transpose(4, 5).reshape(seqs, width, heads, page, d // 2)
    v = torch.where(there, _values(rows(values), rows(ve[at].transpose(4, 5).reshape(seqs, width, heads, page, d // BLOCK))), 0.0)
    # the new tokens of each sequence, padded to `most`
    cu = torch.arange(seqs + 1, device=q.device) if s["cu_q"] is None else s["cu_q"].long()
    new = cu[1:] - cu[:-1]
    i = torch.arange(most, device=q.device)
    real = i < new[:, None]
    row = (cu[:-1, None] + i).clamp(max=tokens - 1)
    x = q.float()[row].view(seqs, most, heads, group, d).permute(0, 2, 3, 1, 4).reshape(seqs, heads, group * most, d)
    z = torch.matmul(x, k.transpose(-1, -2)).view(seqs, heads, group, most, length)
    z *= s["scale"]
    last = (kv_len - new)[:, None] + i
    seen = (j <= last[..., None]) & (j < kv_len[:, None, None])
    if s["window"]:
        seen &= j > last[..., None] - s["window"]
    z.masked_fill_(~seen[:, None, None], -math.inf)
    top = z.amax(-1, keepdim=True)
    top = torch.where(torch.isfinite(top), top, 0.0)
    z.sub_(top).exp_()
    total = z.sum(-1, keepdim=True)
    o = torch.matmul(z.view(seqs, heads, group * most, length), v).view(seqs, heads, group, most, d)
    o = torch.where(total > 0, o / total, 0.0)
    lse = (top + torch.log(total)).squeeze(-1)
    o, lse = o.permute(0, 3, 1, 2, 4)[real], lse.permute(0, 3, 1, 2)[real]
    return {"out": o.reshape(tokens, heads_q, d).to(q.dtype), "lse": lse.reshape(tokens, heads_q)}


def run(state):
    s = state
    if not own:
        if s["op"] == "rope":
            return _plain_rope(s["x"], s["positions"], s["table"], s["layout"], s["backward"]).to(s["x"].dtype)
        return _plain_append(s) if s["op"] == "append" else _plain_attention(s)
    from paper_2603_09221_amd import binding
    if s["op"] == "rope":
        call = binding.ttc_rope_backward if s["backward"] else binding.ttc_rope
        return call(s["x"], s["positions"], s["table"], layout=s["layout"])
    if s["op"] == "append":
        q = binding.ttc_kv_append(s["cache"], s["k"], s["v"], s["slots"], s["positions"], s["table"], layout=s["layout"], q=s["q"])
        k, v = binding.ttc_kv_read(s["cache"], s["slots"], s["d"])
        return {"q": q, "k": k, "v": v}
    return binding.ttc_attention(s["q"], s["cache"], s["table"], s["kv_len"], cu_q=s["cu_q"], max_q=s["max_q"], max_kv=s["max_kv"],
                                 scale=s["scale"], window=s["window"])


# ---------------------------------------------------------------------------------------------------------------
# what a pass cannot do without

def work(case):
    op, d = case["op"], case["d"]
    e = 2 if case["dtype"] == "bf16" else 4
    if op == "rope":
        n, rows = case["tokens"], min(case["tokens"], case["far"])
        return {"bytes": 2 * n * case["heads"] * d * e + 8 * n + rows * case["rot"] * 4,
                "flops": 3.0 * n * case["heads"] * case["rot"]}
    token = d // 2 + d // BLOCK     # bytes of a token's keys, or values, in the cache, per head
    if op == "append":
        n, heads, rows = case["tokens"], case["heads"], min(case["tokens"], case["far"])
        return {"bytes": 2 * n * case["heads_q"] * d * e + 2 * n * heads * (d * e + 2 * token + d * 2) + 16 * n + rows * case["rot"] * 4,
                "flops": n * (3.0 * (case["heads_q"] + heads) * case["rot"] + 6.0 * heads * d)}
    kv, new = _lengths(case)
    tokens = sum(min(n, case["window"] + m - 1) if case["window"] else n for n, m in zip(kv, new))
    pairs = sum(_visible(n, m, case["window"]) for n, m in zip(kv, new))
    return {"bytes": 2 * tokens * case["heads"] * token + sum(new) * case["heads_q"] * (2 * d * e + 4),
            "flops": 4.0 * d * case["heads_q"] * pairs}


# ---------------------------------------------------------------------------------------------------------------
# the definitions in 64 bits

def _exact_rope(x, positions, table, layout, backward=False):
    """Complex multiplication: the pair (a, b) is a + ib, the position a factor of cos + i sin."""
    x = x.double()
    rot = 2 * table.shape[1]
    w = torch.view_as_complex(table[positions].double())[:, None]
    part = x[..., :rot]
    pair = part.unflatten(-1, (2, rot // 2)).transpose(-1, -2) if layout == "half" else part.unflatten(-1, (rot // 2, 2))
    y = torch.view_as_real(torch.view_as_complex(pair.contiguous()) * (w.conj() if backward else w))
    y = (y.transpose(-1, -2) if layout == "half" else y).flatten(-2)
    return torch.cat([y, x[..., rot:]], -1)


def _exact_rounded(x):
    """The number nearest to each entry among those that the block's exponent allows, in float64."""
    b = x.unflatten(-1, (-1, BLOCK))
    top = b.abs().amax(-1, keepdim=True)
    f, k = torch.frexp(top)                 # top = f * 2^k, 1/2 <= f < 1
    k = torch.where(f >= 0.875, k, k - 1) - 2
    scale = torch.ldexp(torch.ones_like(top), torch.where(top > 0, k, 0))
    y = b / scale
    step = torch.where(y.abs() < 2, 0.5, torch.where(y.abs() < 4, 1.0, 2.0))
    return (scale * (torch.round(y / step) * step).clamp(-6, 6)).flatten(-2)


def _exact_tokens(codes, e):
    """float64 numbers of codes (.., d / 2 bytes) and exponents, by the code's sign, exponent and mantissa bits."""
    c = torch.stack([codes % 16, codes // 16], -1).flatten(-2).int()
    m, k = (c % 2).double(), (c // 2 % 4).double()
    x = torch.where(k == 0, 0.5 * m, (1 + 0.5 * m) * 2.0 ** (k - 1)) * (1 - 2 * (c // 8)).double()
    return x * torch.repeat_interleave(2.0 ** (e.double() - 127), BLOCK, -1)


def exact(case, seed):
    s = prepare(case, seed)
    if s["op"] == "rope":
        return _exact_rope(s["x"], s["positions"], s["table"], s["layout"], s["backward"])
    if s["op"] == "append":
        k = _exact_rope(s["k"], s["positions"], s["table"], s["layout"])
        return {"q": _exact_rope(s["q"], s["positions"], s["table"], s["layout"]), "k": _exact_rounded(k),
                "v": _exact_rounded(s["v"].double())}
    d, q = s["d"], s["q"].double()
    kc, vc, ke, ve = _views(s["cache"], d)
    page, heads = kc.shape[2], kc.shape[1]
    group = q.shape[1] // heads
    kv = s["kv_len"].tolist()
    cu = list(range(len(kv) + 1)) if s["cu_q"] is None else s["cu_q"].tolist()
    out, lse = torch.zeros_like(q), torch.full(q.shape[:2], -math.inf, dtype=torch.float64, device=q.device)
    for i, n in enumerate(kv):
        new = cu[i + 1] - cu[i]
        if not n or not new:
            continue
        at = s["table"][i, :-(-n // page)].long()
        j, last = torch.arange(n, device=q.device), n - new + torch.arange(new, device=q.device)[:, None]
        seen = (j <= last) & (j > last - s["window"]) if s["window"] else j <= last
        for h in range(heads):
            k = _exact_tokens(kc[at, h].flatten(0, 1)[:n], ke[at, h].flatten(0, 1)[:n])
            v = _exact_tokens(vc[at, h].transpose(2, 3).reshape(-1, d // 2)[:n], ve[at, h].transpose(2, 3).reshape(-1, d // BLOCK)[:n])
            for g in range(h * group, (h + 1) * group):
                z = (q[cu[i]:cu[i + 1], g] @ k.T * s["scale"]).masked_fill(~seen, -math.inf)
                total = torch.logsumexp(z, -1)
                lse[cu[i]:cu[i + 1], g] = total
                out[cu[i]:cu[i + 1], g] = torch.where(torch.isfinite(total)[:, None], torch.exp(z - total[:, None]), 0.0) @ v
    return {"out": out, "lse": lse}
