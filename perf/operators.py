"""The attention sublayer of a cached decoding loop: operators, cases, plain forms.

A masked-diffusion model that decodes block by block runs its model call on
the active block against a cache of the other positions' keys and values; the
cache is filled once by a call over the whole prompt.  Three operators around
that cache, each through the public entry points of ``paper_2606_02955_amd``:

* ``rope``: the RMS norm of every query and key head and the rotation by
  position, in one pass; the queries (and, for a prompt, the keys) come out in
  16 bits, the keys and values go into the cache in 4.  The pass reads back
  what the cache now holds for those tokens.
* ``cache``: attention of one to a few dozen query tokens per sequence over
  the 4-bit cache, read page by page.
* ``prompt``: attention over whole packed sequences in 16 bits.

The 4-bit cache, ``[pages, kv heads, tile]`` bytes.  A page holds 64 tokens; a
tile is one page of one head: key codes, value codes, key scales, value scales.

* Codes: ``[D / 32 groups][64 tokens][16 bytes]``.  Byte n of a group holds
  elements 2n (low nibble) and 2n + 1 of its 32, as E2M1: a sign bit and a
  magnitude out of 0, 0.5, 1, 1.5, 2, 3, 4, 6.
* Scales: ``[64 tokens][S]`` bytes, S = D / 32 rounded up to a multiple of 4;
  byte g is 127 + e (E8M0) of group g: element = 2^e * code.
* Writing a group: the smallest e (from -126) with amax <= 7 * 2^e, then
  x / 2^e rounded to the nearest code, ties to the even code, over 6 to 6.

A query at position p of its sequence sees the keys j < min(len, end(p)),
end(p) = (p // blk + 1) * blk: blk = 1 is the causal mask, blk = 32 that of
decoding in blocks of 32, and blk = 0 stands for no mask.  A query that sees
nothing gets zeros and a log-sum-exp of -inf.

Head size 128, blocks of 32, spans of 256 to 1024 and hidden size 4096 (32
heads of 128) are the decoding settings of the workloads in ``workloads/``;
the other sizes are generic.
"""
from __future__ import annotations

import math

import torch

own = False

PAGE = 64
MAGNITUDES = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
NORM_EPS = 1e-6


# ---------------------------------------------------------------------------
# cases
# ---------------------------------------------------------------------------
def _rope(name, B, lo, hi, H, Hk, D, dtype="bf16", rot=None, interleaved=False, keys=True, norm=True):
    """B sequences of lo to hi tokens; keys: whether the rotated keys come out too."""
    return {"name": name, "op": "rope", "B": B, "lo": lo, "hi": hi, "H": H, "Hk": Hk, "D": D, "dtype": dtype,
            "rot": D if rot is None else rot, "interleaved": interleaved, "keys": keys, "norm": norm}


def _cache(name, B, nq, lo, hi, H, Hk, D, blk=0):
    """B sequences of lo to hi cached tokens, at most nq query tokens each."""
    return {"name": name, "op": "cache", "B": B, "nq": nq, "lo": lo, "hi": hi, "H": H, "Hk": Hk, "D": D, "blk": blk}


def _prompt(name, B, lo, hi, H, Hk, D, blk=0, past=0):
    """B packed sequences of lo to hi tokens, after `past` tokens whose keys are at hand."""
    return {"name": name, "op": "prompt", "B": B, "lo": lo, "hi": hi, "H": H, "Hk": Hk, "D": D, "blk": blk, "past": past}


def listed():
    return [
        # one request's active block in a decoding step: latency
        _rope("rope_block_b1", 1, 32, 32, 32, 32, 128, keys=False),
        # a packed batch of prompts, grouped heads: rotated keys for the prompt's own attention, all into the cache
        _rope("rope_prompts", 24, 150, 1024, 32, 8, 128),
        # float32 activations, another rotation layout over part of the head, odd head size and lengths, no norm
        _rope("rope_f32_partial", 7, 13, 901, 12, 4, 96, "f32", rot=64, interleaved=True, norm=False),
        # one request, one token, a short cache: the smallest call
        _cache("cache_b1_token", 1, 1, 500, 500, 32, 8, 128, blk=1),
        # one request's active block over the whole span (prefix and suffix cached), a head of keys for each of queries
        _cache("cache_b1_block", 1, 32, 1024, 1024, 32, 32, 128),
        # a server's batch in mid-generation: ragged spans from a first token to long ones, partly filled blocks
        _cache("cache_b24_ragged", 24, 32, 1, 4099, 28, 4, 128, blk=32),
        # two requests' next tokens over very long contexts: few rows, a long axis
        _cache("cache_b2_long", 2, 1, 99001, 131072, 32, 8, 128, blk=1),
        # a large batch's blocks over long contexts: the throughput end
        _cache("cache_b64_blocks", 64, 32, 6000, 8192, 32, 8, 128),
        # a short prompt, no mask, of an odd length
        _prompt("prompt_b1_short", 1, 333, 333, 32, 32, 128),
        # packed prompts of very different lengths, the mask of block decoding
        _prompt("prompt_packed", 16, 1, 2048, 32, 8, 128, blk=32),
        # further pieces of prompts whose first part is done, small heads
        _prompt("prompt_chunks", 4, 500, 777, 16, 2, 64, blk=1, past=2000),
        # one long causal prompt: the matrix-core end
        _prompt("prompt_long", 1, 16384, 16384, 16, 4, 128, blk=1),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the ranges above."""
    op = rng.choice(["rope", "cache", "cache", "prompt", "prompt"])
    H, Hk = rng.choice([(32, 32), (32, 8), (28, 4), (16, 2), (12, 4), (8, 8), (40, 8), (5, 1)])
    D = rng.choice([128, 128, 128, 64, 96])
    if op == "rope":
        B = _log_int(rng, 1, 32)
        hi = _log_int(rng, 1, 1024)
        dtype = rng.choice(["bf16", "bf16", "f32"])
        rot = rng.choice([D, D, D // 2])
        c = _rope("", B, rng.choice([hi, (hi + 1) // 2, 1]), hi, H, Hk, D, dtype, rot, rng.random() < 0.3, rng.random() < 0.5,
                  rng.random() < 0.8)
    elif op == "cache":
        nq = rng.choice([1, 1, 4, 17, 32, 32, 64])
        hi = _log_int(rng, 1, 131072)
        B = _log_int(rng, 1, 64)
        while B > 1 and (B * hi * Hk > 64 * 8192 * 8 or B * hi * H * nq > 64 * 8192 * 32 * 32):
            B = (B + 1) // 2
        while nq > 1 and hi * H * nq > 64 * 8192 * 32 * 32:
            nq = (nq + 1) // 2
        c = _cache("", B, nq, rng.choice([hi, (hi + 1) // 2, 1]), hi, H, Hk, D, rng.choice([0, 0, 1, 32]))
    else:
        hi = _log_int(rng, 1, 8192)
        past = rng.choice([0, 0, 0, _log_int(rng, 1, 4096)])
        B = _log_int(rng, 1, 32)
        while B > 1 and 1.0 * B * H * hi * (hi + past) > 16 * 16384.0 ** 2 / 2:
            B = (B + 1) // 2
        while 1.0 * B * H * hi * (hi + past) > 16 * 16384.0 ** 2 / 2:
            hi = (hi + 1) // 2
        c = _prompt("", B, rng.choice([hi, (hi + 1) // 2, 1]), hi, H, Hk, D, rng.choice([0, 0, 1, 1, 32, 48]), past)
    del c["name"]
    return c


def _lens(case):
    """Tokens of each sequence: lo..hi, spread evenly, in a mixed order."""
    n = case["hi"] - case["lo"] + 1
    if case["B"] == 1:
        return [case["hi"]]
    step = (n - 1) / (case["B"] - 1)
    return [case["lo"] + int(round(step * ((7 * b) % case["B"] if case["B"] % 7 else (5 * b) % case["B"] if case["B"] % 5 else b)))
            for b in range(case["B"])]


def _queries(case, lens):
    """Query tokens of each sequence over the cache: nq, with blocks that have fewer left among them."""
    nq = case["nq"]
    return [max(1, nq - (5 * b) % nq) if b % 3 == 2 else nq for b in range(case["B"])]


def _seen(first, n, length, blk):
    """Sum over n queries from position `first` of the keys each sees."""
    if blk == 0:
        return n * length
    return sum(min(length, max(0, ((first + i) // blk + 1) * blk)) for i in range(n))


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------
class State:
    pass


def _gen(seed, dev):
    g = torch.Generator(device=dev)
    g.manual_seed((int(seed) * 0x9E3779B97F4A7C15 + 0x4B17) & ((1 << 63) - 1))
    return g


def _normal(shape, g, dev):
    return torch.empty(shape, dtype=torch.float32, device=dev).normal_(generator=g)


def _cumulated(counts, dev):
    t = torch.zeros(len(counts) + 1, dtype=torch.int32)
    t[1:] = torch.tensor(counts).cumsum(0)
    return t.to(dev)


def _scale_bytes(D):
    return (D // 32 + 3) // 4 * 4


def tile_bytes(D):
    return PAGE * (D + 2 * _scale_bytes(D))


def _scales(x):
    """e of groups x [..., 32]: the smallest power of two with amax <= 7 * 2^e."""
    bits = x.abs().amax(dim=-1).view(torch.int32)
    return (((bits + 0x1FFFFF) >> 23) - 129).clamp_(min=-126)


def _power(e):
    """2^e for whole e from -126 to 127, exactly."""
    return ((e + 127) << 23).view(torch.float32)


def _codes(y):
    """E2M1 codes (0..15) of values y already divided by their scale."""
    a = y.abs()
    c = ((a > 0.25).to(torch.uint8) + (a >= 0.75).to(torch.uint8) + (a > 1.25).to(torch.uint8) + (a >= 1.75).to(torch.uint8)
         + (a > 2.5).to(torch.uint8) + (a >= 3.5).to(torch.uint8) + (a > 5.0).to(torch.uint8))
    return c + torch.signbit(y).to(torch.uint8) * 8


def _pages_of(x):
    """The codes and scales of one operand's pages, x [pages, 64, Hk, D]: [pages, Hk, 32 D] and [pages, Hk, 64 S]."""
    P, _, Hk, D = x.shape
    G, S = D // 32, _scale_bytes(D)
    xg = x.view(P, PAGE, Hk, G, 32).permute(0, 2, 3, 1, 4).contiguous()            # [P, Hk, G, 64, 32]
    e = _scales(xg)
    c = _codes(xg * _power(-e).unsqueeze(-1))
    codes = c[..., 0::2] | (c[..., 1::2] << 4)
    scales = torch.full((P, Hk, PAGE, S), 127, dtype=torch.uint8, device=x.device)
    scales[..., :G] = (e + 127).to(torch.uint8).permute(0, 1, 3, 2)
    return codes.reshape(P, Hk, -1), scales.view(P, Hk, -1)


def _filled_cache(case, lens, g, dev):
    """A cache of the sequences' keys and values, their pages in a mixed order
    among pages of others.  Past a sequence's end its last page holds what an
    earlier user of the page left there: any bytes."""
    Hk, D = case["Hk"], case["D"]
    need = [-(-n // PAGE) for n in lens]
    total = sum(need) + 3
    cache = torch.empty((total, Hk, tile_bytes(D)), dtype=torch.uint8, device=dev)
    # keys with a few strong channels, as models have them
    channel = 1.0 + 2.0 * (torch.rand((Hk, D), generator=g, device=dev) < 0.03).float()
    step = max(1, int(6e7) // (PAGE * Hk * D))
    kc = 32 * D
    for first in range(0, total, step):
        n = min(step, total - first)
        k = _normal((n, PAGE, Hk, D), g, dev) * channel
        v = _normal((n, PAGE, Hk, D), g, dev)
        kcodes, kscales = _pages_of(k)
        vcodes, vscales = _pages_of(v)
        cache[first:first + n] = torch.cat([kcodes, vcodes, kscales, vscales], dim=2)
    order = torch.randperm(total, generator=g, device=dev).to(torch.int32)
    width = max(need)
    table = torch.full((case["B"], width), 0, dtype=torch.int32, device=dev)
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n]
        at += n
        tail = lens[b] % PAGE
        if tail:
            tile = cache[table[b, n - 1].long()]                                    # [Hk, tile]
            junk = torch.randint(0, 256, tile.shape, generator=g, device=dev, dtype=torch.uint8)
            codes = torch.arange(2 * kc, device=dev)
            scales = torch.arange(2 * PAGE * _scale_bytes(D), device=dev)
            token = torch.cat([codes // 16 % PAGE, scales // _scale_bytes(D) % PAGE])
            cache[table[b, n - 1].long()] = torch.where(token >= tail, junk, tile)
    return cache, table


def prepare(case, seed):
    dev = torch.device("cuda", torch.cuda.current_device())
    g = _gen(seed, dev)
    s = State()
    s.op = case["op"]
    s.H, s.Hk, s.D = H, Hk, D = case["H"], case["Hk"], case["D"]
    lens = _lens(case)
    if s.op == "rope":
        T = sum(lens)
        dt = torch.float32 if case["dtype"] == "f32" else torch.bfloat16
        # the projection's output holds the three side by side
        qkv = (_normal((T, (H + 2 * Hk) * D), g, dev) * (0.5 + torch.rand((T, 1), generator=g, device=dev))).to(dt)
        s.q = qkv[:, :H * D].view(T, H, D)
        s.k = qkv[:, H * D:(H + Hk) * D].view(T, Hk, D)
        s.v = qkv[:, (H + Hk) * D:].view(T, Hk, D)
        s.q_weight = 1.0 + 0.2 * _normal((D,), g, dev) if case["norm"] else None
        s.k_weight = 1.0 + 0.2 * _normal((D,), g, dev) if case["norm"] else None
        s.interleaved, rot = case["interleaved"], case["rot"]
        angle = torch.outer(torch.arange(max(lens) + 256, device=dev).double(),
                            10000.0 ** (-torch.arange(0, rot, 2, device=dev).double() / rot))
        s.cos_sin = torch.cat([angle.cos(), angle.sin()], dim=1).float()            # [positions, rot]
        start = torch.randint(0, 256, (case["B"],), generator=g, device=dev).tolist()
        s.positions = torch.cat([torch.arange(a, a + n, device=dev) for a, n in zip(start, lens)]).to(torch.int32)
        # each sequence's tokens go to pages of its own
        need = [-(-n // PAGE) for n in lens]
        pages = torch.randperm(sum(need) + 2, generator=g, device=dev)
        first = [sum(need[:b]) for b in range(len(need))]
        s.slots = torch.cat([(pages[f:f + m].view(m, 1) * PAGE + torch.arange(PAGE, device=dev)).view(-1)[:n]
                             for f, m, n in zip(first, need, lens)]).to(torch.int32)
        s.cache = torch.zeros((sum(need) + 2, Hk, tile_bytes(D)), dtype=torch.uint8, device=dev)
        s.q_out = torch.empty((T, H, D), dtype=dt, device=dev)
        s.k_out = torch.empty((T, Hk, D), dtype=dt, device=dev) if case["keys"] else None
        # what 4 bits hold, in torch's narrowest type that holds it exactly
        s.k_read = torch.empty((T, Hk, D), dtype=torch.float8_e5m2, device=dev)
        s.v_read = torch.empty((T, Hk, D), dtype=torch.float8_e5m2, device=dev)
        return s
    if s.op == "cache":
        counts = _queries(case, lens)
        s.cache, s.page_table = _filled_cache(case, lens, g, dev)
        s.kv_len = torch.tensor(lens, dtype=torch.int32).to(dev)
        s.max_q, s.blk = max(counts), case["blk"]
    else:
        counts = lens
        past = [case["past"] - (case["past"] // 3) * (b % 3) // 2 for b in range(case["B"])]
        s.cu_k = _cumulated([n + p for n, p in zip(lens, past)], dev)
        s.max_q, s.max_k, s.blk = max(lens), max(n + p for n, p in zip(lens, past)), case["blk"]
        Tk = sum(lens) + sum(past)
        s.k = _normal((Tk, Hk, D), g, dev).to(torch.bfloat16)
        s.v = _normal((Tk, Hk, D), g, dev).to(torch.bfloat16)
    T = sum(counts)
    s.cu_q = _cumulated(counts, dev)
    # heads that look about and heads that look at few places
    sharp = 0.5 + 3.0 * torch.rand((1, H, 1), generator=g, device=dev)
    s.q = (_normal((T, H, D), g, dev) * sharp).to(torch.bfloat16)
    s.out = torch.empty((T, H, D), dtype=torch.bfloat16, device=dev)
    s.lse = torch.empty((T, H), dtype=torch.float32, device=dev)
    return s


# ---------------------------------------------------------------------------
# plain forms, 32 bits
# ---------------------------------------------------------------------------
def _rotate(x, cos, sin, interleaved):
    """x [T, h, D]; cos, sin [T, rot / 2]."""
    half = cos.shape[1]
    cos, sin = cos.unsqueeze(1), sin.unsqueeze(1)
    part, rest = x[..., :2 * half], x[..., 2 * half:]
    if interleaved:
        a, b = part[..., 0::2], part[..., 1::2]
        turned = torch.stack([a * cos - b * sin, b * cos + a * sin], dim=-1).flatten(-2)
    else:
        a, b = part[..., :half], part[..., half:]
        turned = torch.cat([a * cos - b * sin, b * cos + a * sin], dim=-1)
    return torch.cat([turned, rest], dim=-1)


def _norm(x, weight):
    if weight is None:
        return x
    return x * torch.rsqrt(x.square().mean(dim=-1, keepdim=True) + NORM_EPS) * weight


def _held(x):
    """The values that the cache holds for x [T, Hk, D]."""
    T, Hk, D = x.shape
    xg = x.view(T, Hk, D // 32, 32)
    e = _scales(xg).unsqueeze(-1)
    code = _codes(xg * _power(-e))
    table = torch.tensor(MAGNITUDES + tuple(-m for m in MAGNITUDES), device=x.device)
    return (table[code.int()] * _power(e)).view(T, Hk, D)


def _plain_rope(s):
    cs = s.cos_sin[s.positions]
    half = cs.shape[1] // 2
    q = _rotate(_norm(s.q.float(), s.q_weight), cs[:, :half], cs[:, half:], s.interleaved)
    k = _rotate(_norm(s.k.float(), s.k_weight), cs[:, :half], cs[:, half:], s.interleaved)
    out = {"q": q.to(s.q_out.dtype), "cache_k": _held(k.contiguous()).to(torch.float8_e5m2),
           "cache_v": _held(s.v.float().contiguous()).to(torch.float8_e5m2)}
    if s.k_out is not None:
        out["k"] = k.to(s.q_out.dtype)
    return out


def _padded(x, cu, width):
    """Packed rows x [T, ...] as [B, width, ...] (past an end: any row), and which are rows."""
    at = torch.arange(width, device=x.device)
    n = cu[1:] - cu[:-1]
    rows = (cu[:-1].view(-1, 1) + at).clamp_(max=max(0, x.shape[0] - 1))
    return x[rows], at < n.view(-1, 1)


def _softmax_rows(scores, v):
    """scores [B, Hk, rows, keys] (-inf where unseen), v [B, Hk, keys, D]: outputs and log-sum-exps."""
    top = scores.amax(dim=-1, keepdim=True)
    scores = scores.sub_(top.clamp(min=-3e38)).exp_()
    total = scores.sum(dim=-1, keepdim=True)
    out = torch.matmul(scores, v) / torch.where(total > 0, total, torch.ones_like(total))
    return out, (top + total.log()).squeeze(-1)


def _attend(s, k, v, kv_len):
    """k, v [B, Hk, keys, D] float32, zeros past kv_len."""
    B, Hk, S, D = k.shape
    q, row = _padded(s.q, s.cu_q, s.max_q)                                          # [B, nq, H, D]
    nq, R = s.max_q, s.H // Hk
    qg = q.float().view(B, nq, Hk, R, D).permute(0, 2, 3, 1, 4).reshape(B, Hk, R * nq, D)
    scores = torch.matmul(qg, k.transpose(2, 3).contiguous()).mul_(1.0 / math.sqrt(D)).view(B, Hk, R, nq, S)
    keys = torch.arange(S, device=k.device)
    end = kv_len.view(B, 1).expand(B, nq)
    if s.blk:
        n = (s.cu_q[1:] - s.cu_q[:-1]).view(B, 1)
        p = kv_len.view(B, 1) - n + torch.arange(nq, device=k.device)
        end = torch.minimum(end, (torch.div(p, s.blk, rounding_mode="floor") + 1) * s.blk)
    scores.masked_fill_((keys >= end.unsqueeze(-1)).view(B, 1, 1, nq, S), -math.inf)
    out, lse = _softmax_rows(scores.view(B, Hk, R * nq, S), v)
    out = out.view(B, Hk, R, nq, D).permute(0, 3, 1, 2, 4).reshape(B, nq, s.H, D)
    lse = lse.view(B, Hk, R, nq).permute(0, 3, 1, 2).reshape(B, nq, s.H)
    return {"out": out[row].to(torch.bfloat16), "lse": lse[row]}


def _plain_values(tiles, at, scales_at, D):
    """One operand of tiles [B, pages, Hk, tile bytes] as float32 [B, Hk, keys, D]."""
    B, P, Hk, _ = tiles.shape
    G, S = D // 32, _scale_bytes(D)
    codes = tiles[..., at:at + 32 * D]
    e = tiles[..., scales_at:scales_at + PAGE * S].view(B, P, Hk, PAGE, S)[..., :G].int() - 127
    one = torch.tensor(MAGNITUDES + tuple(-m for m in MAGNITUDES), device=tiles.device)
    pair = torch.stack([one.repeat(16), one.repeat_interleave(16)], dim=1)          # [256, 2]: low and high nibble
    x = pair[codes.int()].view(B, P, Hk, G, PAGE, 32)
    x = x.mul_(_power(e).permute(0, 1, 2, 4, 3).unsqueeze(-1))
    return x.permute(0, 2, 1, 4, 3, 5).reshape(B, Hk, P * PAGE, D)


def _plain_cache(s):
    tiles = s.cache[s.page_table]                                                   # [B, pages, Hk, tile]
    D = s.D
    there = torch.arange(tiles.shape[1] * PAGE, device=tiles.device) < s.kv_len.view(-1, 1)
    there = there.view(there.shape[0], 1, there.shape[1], 1)
    k = _plain_values(tiles, 0, 64 * D, D).masked_fill_(~there, 0.0)
    v = _plain_values(tiles, 32 * D, 64 * D + PAGE * _scale_bytes(D), D).masked_fill_(~there, 0.0)
    return _attend(s, k, v, s.kv_len)


def _plain_prompt(s):
    k, there = _padded(s.k, s.cu_k, s.max_k)
    v, _ = _padded(s.v, s.cu_k, s.max_k)
    there = there.unsqueeze(-1).unsqueeze(-1)
    k = k.float().masked_fill_(~there, 0.0).permute(0, 2, 1, 3)
    v = v.float().masked_fill_(~there, 0.0).permute(0, 2, 1, 3).contiguous()
    return _attend(s, k, v, s.cu_k[1:] - s.cu_k[:-1])


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------
def _own(s):
    import paper_2606_02955_amd as fd
    if s.op == "rope":
        fd.fdllm_qk_norm_rope(s.q, s.k, s.v, s.positions, s.cos_sin, s.q_out, k_out=s.k_out, q_weight=s.q_weight,
                              k_weight=s.k_weight, eps=NORM_EPS, interleaved=s.interleaved, cache=s.cache, slots=s.slots)
        fd.fdllm_cache_read(s.cache, s.slots, s.k_read, s.v_read)
        out = {"q": s.q_out, "cache_k": s.k_read, "cache_v": s.v_read}
        if s.k_out is not None:
            out["k"] = s.k_out
        return out
    if s.op == "cache":
        fd.fdllm_cache_attention(s.q, s.cache, s.page_table, s.kv_len, s.cu_q, s.out, s.max_q, lse=s.lse, blk=s.blk)
    else:
        fd.fdllm_prompt_attention(s.q, s.k, s.v, s.cu_q, s.cu_k, s.out, s.max_q, lse=s.lse, blk=s.blk)
    return {"out": s.out, "lse": s.lse}


def run(s):
    if own:
        return _own(s)
    return {"rope": _plain_rope, "cache": _plain_cache, "prompt": _plain_prompt}[s.op](s)


def work(case):
    lens = _lens(case)
    H, Hk, D = case["H"], case["Hk"], case["D"]
    if case["op"] == "rope":
        T = sum(lens)
        e = 4.0 if case["dtype"] == "f32" else 2.0
        read = T * (H + 2 * Hk) * D * e + 8.0 * T
        table = 4.0 * case["rot"] * min(T, max(lens) + 256)
        written = T * H * D * e + (T * Hk * D * e if case["keys"] else 0.0)
        # the cache's bytes, and what it holds in a byte a value
        held = T * Hk * (D + 2.0 * (D // 32)) + 2.0 * T * Hk * D
        return {"bytes": read + table + written + held, "flops": 10.0 * T * (H + Hk) * D}
    if case["op"] == "cache":
        counts = _queries(case, lens)
        T = sum(counts)
        seen = sum(_seen(n - c, c, n, case["blk"]) for n, c in zip(lens, counts))
        kv = sum(lens) * Hk * (D + 2.0 * (D // 32))
        return {"bytes": kv + T * H * (4.0 * D + 4.0), "flops": 4.0 * D * H * seen}
    past = [case["past"] - (case["past"] // 3) * (b % 3) // 2 for b in range(case["B"])]
    T, Tk = sum(lens), sum(lens) + sum(past)
    seen = sum(_seen(p, n, n + p, case["blk"]) for n, p in zip(lens, past))
    return {"bytes": T * H * (4.0 * D + 4.0) + 4.0 * Tk * Hk * D, "flops": 4.0 * D * H * seen}


# ---------------------------------------------------------------------------
# the definition in 64 bits: a sequence and a head at a time
# ---------------------------------------------------------------------------
def _exact_held(x):
    """x [T, Hk, D] float64 through the cache's format: nearest of all 16 values, ties to the even code."""
    T, Hk, D = x.shape
    out = torch.empty_like(x)
    values = torch.tensor(MAGNITUDES, dtype=torch.float64, device=x.device)
    for g in range(D // 32):
        part = x[:, :, 32 * g:32 * g + 32]
        top = part.abs().amax(dim=2, keepdim=True)
        e = torch.ceil(torch.log2(top.clamp(min=1e-30) / 7.0)).clamp(min=-126.0)
        unit = torch.exp2(e)
        a = (part / unit).abs()
        best = torch.zeros_like(a)
        gap = a.clone()
        for c in range(1, 8):
            d = (a - values[c]).abs()
            nearer = (d < gap) | ((d == gap) & (c % 2 == 0))
            best = torch.where(nearer, values[c], best)
            gap = torch.where(nearer, d, gap)
        out[:, :, 32 * g:32 * g + 32] = torch.copysign(best, part) * unit
    return out


def _exact_turn(x, weight, s):
    x = x.double()
    if weight is not None:
        x = x / (x.pow(2).sum(dim=-1, keepdim=True) / x.shape[-1] + NORM_EPS).sqrt() * weight.double()
    half = s.cos_sin.shape[1] // 2
    where = s.positions.long()
    z = torch.complex(s.cos_sin[where, :half].double(), s.cos_sin[where, half:].double()).unsqueeze(1)
    i = torch.arange(half, device=x.device)
    first, second = (2 * i, 2 * i + 1) if s.interleaved else (i, i + half)
    turned = torch.complex(x[..., first], x[..., second]) * z
    out = x.clone()
    out[..., first] = turned.real
    out[..., second] = turned.imag
    return out


def _exact_cached(s, b, h, length, at, scales_at):
    """One operand of one sequence and head from the cache, float64 [length, D]."""
    D, S = s.D, _scale_bytes(s.D)
    j = torch.arange(length, device=s.cache.device)
    page, token = s.page_table[b].long()[j // PAGE].view(-1, 1), (j % PAGE).view(-1, 1)
    d = torch.arange(D, device=s.cache.device).view(1, -1)
    byte = s.cache[page, h, at + d // 32 * (16 * PAGE) + token * 16 + d % 32 // 2].long()
    code = torch.where(d % 2 == 1, byte >> 4, byte & 15)
    scale = s.cache[page, h, scales_at + token * S + d // 32].double() - 127.0
    value = torch.tensor(MAGNITUDES, dtype=torch.float64, device=s.cache.device)[code & 7]
    return torch.where(code >= 8, -value, value) * torch.exp2(scale)


def exact(case, seed):
    s = prepare(case, seed)
    H, Hk, D = s.H, s.Hk, s.D
    if s.op == "rope":
        k = _exact_turn(s.k, s.k_weight, s)
        out = {"q": _exact_turn(s.q, s.q_weight, s), "cache_k": _exact_held(k), "cache_v": _exact_held(s.v.double())}
        if s.k_out is not None:
            out["k"] = k
        return out
    T = s.q.shape[0]
    out = torch.zeros((T, H, D), dtype=torch.float64, device=s.q.device)
    lse = torch.full((T, H), -math.inf, dtype=torch.float64, device=s.q.device)
    cu_q = s.cu_q.tolist()
    cu_k = s.cu_k.tolist() if s.op == "prompt" else None
    kv_len = s.kv_len.tolist() if s.op == "cache" else [b - a for a, b in zip(cu_k, cu_k[1:])]
    for b, length in enumerate(kv_len):
        n = cu_q[b + 1] - cu_q[b]
        for h in range(Hk):
            if s.op == "cache":
                k = _exact_cached(s, b, h, length, 0, 64 * D)
                v = _exact_cached(s, b, h, length, 32 * D, 64 * D + PAGE * _scale_bytes(D))
            else:
                k, v = (x[cu_k[b]:cu_k[b + 1], h].double() for x in (s.k, s.v))
            for hq in range(h * (H // Hk), (h + 1) * (H // Hk)):
                for first in range(0, n, 2048):
                    m = min(2048, n - first)
                    rows = slice(cu_q[b] + first, cu_q[b] + first + m)
                    x = s.q[rows, hq].double() @ k.t() / math.sqrt(D)
                    if s.blk:
                        p = length - n + first + torch.arange(m, device=x.device)
                        end = (torch.floor(p.double() / s.blk) + 1) * s.blk
                        x = torch.where(torch.arange(length, device=x.device) < end.view(-1, 1), x, -math.inf)
                    z = torch.logsumexp(x, dim=1)
                    lse[rows, hq] = z
                    out[rows, hq] = torch.exp(x - torch.where(z > -math.inf, z, 0.0).view(-1, 1)) @ v
    return {"out": out, "lse": lse}
