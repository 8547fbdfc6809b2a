"""Decoding with drafted tokens around the 4-bit cache: operators, cases, plain forms.

A drafter (a block decoder with its per-position marginals, or a small model)
proposes tokens, a chain of them or a tree; one call of the target model over
all of them says which stand.  Five operators, each through the public entry
points of ``paper_2606_02955_amd``:

* ``layout``: from the parents of a tree's nodes, who sees whom (a bit mask of
  each node's ancestors and itself), each node's position and its cache slot.
* ``attention``: the nodes' queries over the 4-bit cache, each over the context
  and its own ancestors.
* ``draft``: a chain's tokens against the target's and the drafter's
  probabilities, from given uniform numbers.
* ``tree``: a tree's tokens against a draw from the target at every node.
* ``keep``: the cache entries of the path that stands move to their places
  behind the context, in all layers.

Request b has n nodes, the rows ``cu_q[b]..cu_q[b + 1]`` of everything packed;
node i is token i of them, node 0 the token that the last step ended with.  The
cache holds ``kv_len[b]`` of its tokens, the n nodes last.

* Layout: A_i = {i} and the ancestors of i (parents are earlier nodes, -1: none).
  Bit j % 64 of word j / 64 of row i says whether j is in A_i; position =
  kv_len - n + |A_i| - 1; slot = that of the cache's token kv_len - n + i.
* Attention: node i sees the first kv_len - n keys and those of A_i.
* Probabilities: p = softmax(logits / temperature), temperature 0 all of it on
  the highest logit, the lowest index among equals.  A logit of -inf is a token
  that cannot be.  A draw with u from weights w takes the lowest v for which
  w_0 + ... + w_v > u (w_0 + w_1 + ...).
* Draft: row i judges the draft ids[i + 1].  It stands when those before it do
  and u_i q(draft) < p(draft), q the drafter's probabilities of row i, or 1 for a
  drafter without any.  Then one more token is drawn, from the last row's p when
  all stand, from max(p - q, 0) of the row whose draft fell otherwise (with
  temperature 0: from p, the drafter's are not looked at).
* Tree: y_i is drawn from row i's p with u_i; from node 0 on, y_i is the next
  token and its child with that token, the lowest of several, the next node.
* Tokens are packed as the rows are: those that stand and the one drawn last,
  then -1; beside them the logarithm of the target's probability (0 there).

The cache's format is that of ``perf/operators.py``: 64 tokens to a page, a tile
of a page and a head: key codes, value codes ([D / 32][64 tokens][16 bytes], two
E2M1 codes a byte), key scales, value scales ([64 tokens][D / 32 rounded up to a
multiple of 4], 127 + e).

Vocabularies of 126464 and 32000 and heads of 64 and 128 are those of the
workloads in ``workloads/``; the other sizes are generic.
"""
from __future__ import annotations

import math
import random

import torch

own = False

PAGE = 64
MAGNITUDES = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


# ---------------------------------------------------------------------------
# cases
# ---------------------------------------------------------------------------
def _layout(name, B, n_lo, n_hi, length):
    """B trees of n_lo to n_hi nodes behind contexts of up to `length` tokens."""
    return {"name": name, "op": "layout", "B": B, "n_lo": n_lo, "n_hi": n_hi, "length": length}


def _attention(name, B, n_lo, n_hi, lo, hi, H, Hk, D):
    """B trees of n_lo to n_hi nodes over lo to hi cached tokens before them."""
    return {"name": name, "op": "attention", "B": B, "n_lo": n_lo, "n_hi": n_hi, "lo": lo, "hi": hi, "H": H, "Hk": Hk, "D": D}


def _draft(name, B, n_lo, n_hi, V, dtype="bf16", marginals=True, greedy=0.0, kept=0):
    """B chains of n_lo to n_hi rows (a draft fewer).  marginals: whether the
    drafter has probabilities; greedy: share of requests at temperature 0; kept:
    tokens that a filter left of each row (0: all)."""
    return {"name": name, "op": "draft", "B": B, "n_lo": n_lo, "n_hi": n_hi, "V": V, "dtype": dtype, "marginals": marginals,
            "greedy": greedy, "kept": kept}


def _tree(name, B, n_lo, n_hi, V, dtype="bf16", greedy=0.0, kept=0):
    return {"name": name, "op": "tree", "B": B, "n_lo": n_lo, "n_hi": n_hi, "V": V, "dtype": dtype, "greedy": greedy,
            "kept": kept}


def _keep(name, B, n_lo, n_hi, most, layers, Hk, D):
    """Paths of up to `most` nodes out of trees of n_lo to n_hi."""
    return {"name": name, "op": "keep", "B": B, "n_lo": n_lo, "n_hi": n_hi, "most": most, "layers": layers, "Hk": Hk, "D": D}


def listed():
    return [
        # one request's tree, once a step: latency
        _layout("layout_b1", 1, 26, 26, 1000),
        # a server's batch of large trees, words of the mask more than one
        _layout("layout_b64_wide", 64, 100, 250, 8192),
        # one request, a small tree, a short context: the smallest attention call, once a layer
        _attention("attention_b1_short", 1, 16, 16, 500, 500, 32, 8, 128),
        # a batch in mid-generation: contexts from nothing to long ones, trees of one node to 61, grouped heads
        _attention("attention_b24_ragged", 24, 1, 61, 0, 4099, 28, 4, 128),
        # two requests' trees behind very long contexts: few rows, a long axis
        _attention("attention_b2_long", 2, 25, 26, 99001, 131072, 16, 2, 64),
        # a large batch of trees over long contexts: the throughput end
        _attention("attention_b64", 64, 30, 32, 6000, 8192, 32, 8, 128),
        # one request's chain of four drafts with the drafter's marginals: latency
        _draft("draft_b1", 1, 5, 5, 126464),
        # a batch of blocks drafted by a block decoder, ragged, some requests greedy
        _draft("draft_b48_blocks", 48, 3, 17, 126464, greedy=0.2),
        # one request's tree
        _tree("tree_b1", 1, 26, 26, 126464),
        # a batch of trees in float32, a vocabulary of odd size, rows filtered to their best tokens
        _tree("tree_b16_f32_filtered", 16, 11, 61, 50021, "f32", greedy=0.2, kept=200),
        # the path of one request, a model of a few layers
        _keep("keep_b1", 1, 26, 26, 5, 4, 4, 64),
        # the paths of a batch, in all layers of a larger model
        _keep("keep_b64_layers", 64, 30, 64, 9, 32, 8, 128),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the ranges above."""
    op = rng.choice(["layout", "attention", "attention", "draft", "draft", "tree", "tree", "keep"])
    B = _log_int(rng, 1, 64)
    n_hi = _log_int(rng, 1, 64)
    n_lo = rng.choice([n_hi, (n_hi + 1) // 2, 1])
    H, Hk = rng.choice([(32, 32), (32, 8), (28, 4), (16, 2), (12, 4), (8, 8), (40, 8), (5, 1)])
    D = rng.choice([128, 128, 64, 96])
    if op == "layout":
        n_hi = _log_int(rng, 1, 250)
        c = _layout("", B, rng.choice([n_hi, (n_hi + 1) // 2, 1]), n_hi, _log_int(rng, 1, 8192))
    elif op == "attention":
        hi = _log_int(rng, 1, 131072)
        while B > 1 and (B * hi * Hk > 64 * 7000 * 8 or B * (hi + n_hi) * H * n_hi > 64 * 7000 * 32 * 31):
            B = (B + 1) // 2
        while n_hi > 1 and (hi + n_hi) * H * n_hi > 64 * 7000 * 32 * 31:
            n_hi = (n_hi + 1) // 2
        c = _attention("", B, min(n_lo, n_hi), n_hi, rng.choice([hi, hi // 2, 0]), hi, H, Hk, D)
    elif op in ("draft", "tree"):
        V = rng.choice([126464, 126464, 32000, _log_int(rng, 1000, 131072)])
        if op == "draft":
            n_hi = _log_int(rng, 1, 33)
        dtype = rng.choice(["bf16", "bf16", "f32"])
        rows = (2 if op == "draft" else 1) * (2 if dtype == "f32" else 1)
        while B > 1 and 1.0 * B * n_hi * V * rows > 900 * 126464:
            B = (B + 1) // 2
        n_lo, greedy, kept = rng.choice([n_hi, (n_hi + 1) // 2, 1]), rng.choice([0.0, 0.3]), rng.choice([0, 0, 50])
        if op == "draft":
            c = _draft("", B, n_lo, n_hi, V, dtype, rng.random() < 0.7, greedy, kept)
        else:
            c = _tree("", B, n_lo, n_hi, V, dtype, greedy, kept)
    else:
        n_hi = max(n_hi, 4)
        c = _keep("", B, rng.choice([n_hi, (n_hi + 1) // 2]), n_hi, rng.randint(2, 9), rng.choice([1, 4, 32]), rng.choice([1, 2, 4, 8]), D)
    del c["name"]
    return c


def _spread(B, lo, hi):
    """B whole numbers of lo..hi, spread evenly, in a mixed order."""
    if B == 1:
        return [hi]
    step = (hi - lo) / (B - 1)
    return [lo + int(round(step * ((7 * b) % B if B % 7 else (5 * b) % B if B % 5 else b))) for b in range(B)]


def _nodes(case):
    return _spread(case["B"], case["n_lo"], case["n_hi"])[::-1]


def _kept_nodes(case):
    """Nodes of each path: they and those that they replace are different ones
    (their places lie before the sources), so that a second pass moves the same."""
    return [max(1, min(case["most"] - (2 * b) % case["most"], (n + 1) // 2)) for b, n in enumerate(_nodes(case))]


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------
class State:
    pass


def _gen(seed, dev):
    g = torch.Generator(device=dev)
    g.manual_seed((int(seed) * 0x9E3779B97F4A7C15 + 0x5D33) & ((1 << 63) - 1))
    return g


def _normal(shape, g, dev):
    return torch.empty(shape, dtype=torch.float32, device=dev).normal_(generator=g)


def _uniform(shape, g, dev):
    return torch.rand(shape, generator=g, device=dev)


def _cumulated(counts, dev):
    t = torch.zeros(len(counts) + 1, dtype=torch.int32)
    t[1:] = torch.tensor(counts).cumsum(0)
    return t.to(dev)


def _parents(counts, seed):
    """A tree for every request: the first node is its root, the others hang on
    recent nodes, some of them in long branches."""
    rng = random.Random(seed * 7919 + 17)
    trees = []
    for n in counts:
        reach = rng.choice([1, 4, 9, 30])
        trees.append([-1] + [rng.randint(max(0, i - reach), i - 1) for i in range(1, n)])
    return trees


def _depths(tree):
    d = []
    for p in tree:
        d.append(0 if p < 0 else d[p] + 1)
    return d


def _table(need, total, B, width, g, dev):
    """A page table: every sequence's pages in a mixed order among those of others."""
    order = torch.randperm(total, generator=g, device=dev).to(torch.int32)
    table = torch.zeros((B, width), dtype=torch.int32, device=dev)
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n]
        at += n
    return table


def _scale_bytes(D):
    return (D // 32 + 3) // 4 * 4


def tile_bytes(D):
    return PAGE * (D + 2 * _scale_bytes(D))


def _some_cache(pages, Hk, D, g, dev):
    """Pages of any keys and values: codes of normal values, scales around theirs."""
    S = _scale_bytes(D)
    cache = torch.empty((pages, Hk, tile_bytes(D)), dtype=torch.uint8, device=dev)
    step = max(1, int(1e8) // (Hk * PAGE * D))
    for first in range(0, pages, step):
        n = min(step, pages - first)
        x = _normal((n, Hk, 2, PAGE * D), g, dev).mul_(2.0)
        a = x.abs()
        c = ((a > 0.25).to(torch.uint8) + (a >= 0.75).to(torch.uint8) + (a > 1.25).to(torch.uint8) + (a >= 1.75).to(torch.uint8)
             + (a > 2.5).to(torch.uint8) + (a >= 3.5).to(torch.uint8) + (a > 5.0).to(torch.uint8))
        c += (x < 0).to(torch.uint8) * 8
        cache[first:first + n, :, :PAGE * D] = (c[..., 0::2] | (c[..., 1::2] << 4)).reshape(n, Hk, -1)
        scales = torch.randint(124, 128, (n, Hk, 2, PAGE, S), generator=g, device=dev, dtype=torch.uint8)
        scales[..., D // 32:] = 127
        cache[first:first + n, :, PAGE * D:] = scales.reshape(n, Hk, -1)
    return cache


def _junk_behind(cache, table, kv_len, D, g, dev):
    """Past a sequence's end its last page holds what an earlier user of the page
    left there: any bytes."""
    S = _scale_bytes(D)
    codes, scales = torch.arange(PAGE * D, device=dev), torch.arange(2 * PAGE * S, device=dev)
    token = torch.cat([codes // 16 % PAGE, scales // S % PAGE])
    for b, n in enumerate(kv_len):
        if n % PAGE:
            page = int(table[b, n // PAGE])
            junk = torch.randint(0, 256, cache[page].shape, generator=g, device=dev, dtype=torch.uint8)
            cache[page] = torch.where(token >= n % PAGE, junk, cache[page])


def _logits(rows, case, g, dev):
    """Rows of logits, float32: a background and a few likely tokens; filtered
    rows have -inf but for their best."""
    V = case["V"]
    x = _normal((rows, V), g, dev).mul_(1.5)
    best = torch.randint(0, V, (rows, 4), generator=g, device=dev)
    height = 6.0 + 8.0 * _uniform((rows, 4), g, dev) + 0.25 * math.log(V)
    x.scatter_add_(1, best, height)
    return x


def _filtered(x, kept):
    if not kept or kept >= x.shape[1]:
        return x
    return x.masked_fill_(x < x.topk(kept, dim=1).values[:, -1:], -math.inf)


def _pick(x, temperature, g, dev):
    """A token of each row, drawn from its softmax."""
    noise = -torch.log(-torch.log(_uniform(x.shape, g, dev).clamp_(1e-7, 1.0 - 1e-7)))
    return (x / temperature.clamp(min=1e-3).view(-1, 1) + noise).argmax(dim=1)


def prepare(case, seed):
    dev = torch.device("cuda", torch.cuda.current_device())
    g = _gen(seed, dev)
    s = State()
    s.op, B = case["op"], case["B"]
    s.counts = counts = _nodes(case)
    s.cu_q, s.max_q, T = _cumulated(counts, dev), max(counts), sum(counts)
    s.ws = None
    trees = _parents(counts, seed)
    s.depth = max(max(_depths(t)) for t in trees)
    s.parents = torch.tensor([p for t in trees for p in t], dtype=torch.int32).to(dev)
    if s.op in ("layout", "attention", "keep"):
        if s.op == "attention":
            context = _spread(B, case["lo"], case["hi"])
        else:
            context = [((2 * b + 1) * case.get("length", 200) // (2 * B)) for b in range(B)]
        lens = [c + n for c, n in zip(context, counts)]
        s.kv_len = torch.tensor(lens, dtype=torch.int32).to(dev)
        need = [-(-n // PAGE) for n in lens]
        s.page_table = _table(need, sum(need) + 3, B, max(need), g, dev)
    if s.op in ("layout", "attention"):
        words = -(-s.max_q // 64)
        s.masks = torch.empty((T, words), dtype=torch.int64, device=dev)
        s.positions = torch.empty((T,), dtype=torch.int32, device=dev)
        s.slots = torch.empty((T,), dtype=torch.int32, device=dev)
    if s.op == "attention":
        # the step's layout, made before the first layer
        s.masks.copy_(torch.tensor(_mask_words(trees, words), dtype=torch.int64))
        s.H, s.Hk, s.D = H, Hk, D = case["H"], case["Hk"], case["D"]
        s.cache = _some_cache(sum(need) + 3, Hk, D, g, dev)
        _junk_behind(s.cache, s.page_table, lens, D, g, dev)
        # heads that look about and heads that look at few places
        sharp = 0.2 + 1.0 * _uniform((1, H, 1), g, dev)
        s.q = (_normal((T, H, D), g, dev) * sharp).to(torch.bfloat16)
        s.out = torch.empty((T, H, D), dtype=torch.bfloat16, device=dev)
        s.lse = torch.empty((T, H), dtype=torch.float32, device=dev)
    elif s.op == "keep":
        s.Hk, s.D = Hk, D = case["Hk"], case["D"]
        pages = s.pages = sum(need) + 3
        s.cache = torch.randint(0, 256, (case["layers"], pages, Hk, tile_bytes(D)), generator=g, device=dev, dtype=torch.uint8)
        rng, path = random.Random(seed * 31 + 5), []
        s.n_path = torch.tensor(_kept_nodes(case), dtype=torch.int32).to(dev)
        for n, m in zip(counts, _kept_nodes(case)):
            path += [0] + sorted(rng.sample(range(m, n), m - 1)) + [-1] * (n - m)
        s.path = torch.tensor(path, dtype=torch.int32).to(dev)
        s.kv_out = torch.empty((B,), dtype=torch.int32, device=dev)
    elif s.op in ("draft", "tree"):
        dt = torch.float32 if case["dtype"] == "f32" else torch.bfloat16
        V = case["V"]
        s.temperature = 0.6 + 0.6 * _uniform((B,), g, dev)
        s.temperature[_uniform((B,), g, dev) < case["greedy"]] = 0.0
        row = torch.repeat_interleave(torch.arange(B, device=dev), torch.tensor(counts, device=dev))
        s.logits = torch.empty((T, V), dtype=dt, device=dev)
        s.draft = torch.empty((T, V), dtype=dt, device=dev) if case.get("marginals") else None
        picked = torch.empty((T,), dtype=torch.int64, device=dev)   # what a drafter puts behind each row
        step = max(1, int(1e8) // V)
        for first in range(0, T, step):
            rows = slice(first, min(T, first + step))
            x = _logits(rows.stop - first, case, g, dev)
            near = x + 0.5 * _normal(x.shape, g, dev)
            s.logits[rows] = _filtered(x, case["kept"]).to(dt)
            near = _filtered(near, case["kept"]).to(dt)
            if s.draft is not None:
                s.draft[rows] = near
            picked[rows] = _pick(near.float(), s.temperature[row[rows]], g, dev)
        s.ids = torch.randint(0, V, (T,), generator=g, device=dev)
        first = s.cu_q[row].long()
        at = torch.arange(T, device=dev)
        before = at - 1 if s.op == "draft" else first + s.parents
        s.ids = torch.where(at > first, picked[before.clamp(min=0)], s.ids).to(torch.int32)
        s.u = _uniform((T,), g, dev)
        s.u_draw = _uniform((B,), g, dev)
        s.tokens = torch.empty((T,), dtype=torch.int32, device=dev)
        s.n_tokens = torch.empty((B,), dtype=torch.int32, device=dev)
        s.path = torch.empty((T,), dtype=torch.int32, device=dev)
        s.logp = torch.empty((T,), dtype=torch.float32, device=dev)
    return s


def _mask_words(trees, words):
    """Rows of 64-bit words, as signed numbers, of every tree's ancestors."""
    rows = []
    for tree in trees:
        seen = []
        for i, p in enumerate(tree):
            seen.append((1 << i) | (seen[p] if p >= 0 else 0))
        for m in seen:
            w = [(m >> (64 * k)) & ((1 << 64) - 1) for k in range(words)]
            rows.append([v - (1 << 64) if v >> 63 else v for v in w])
    return rows


# ---------------------------------------------------------------------------
# plain forms
# ---------------------------------------------------------------------------
def _requests(cu, T):
    """The request of each row, and its number in it."""
    at = torch.arange(T, device=cu.device)
    b = (at.view(-1, 1) >= cu[1:].view(1, -1)).sum(dim=1)
    return b, at - cu[b]


def _plain_layout(s):
    T, words = s.masks.shape
    b, i = _requests(s.cu_q, T)
    first = s.cu_q[b].long()
    parent = s.parents.long()
    bits = torch.zeros((T, words), dtype=torch.int64, device=s.cu_q.device)
    one = torch.ones((), dtype=torch.int64, device=s.cu_q.device)
    word = torch.arange(words, device=s.cu_q.device)
    node, depth = i.long(), torch.zeros_like(i)
    for step in range(s.depth + 1):
        there = node >= 0
        bit = torch.bitwise_left_shift(one, node.clamp(min=0) % 64)
        hit = there.view(-1, 1) & (word.view(1, -1) == (node.clamp(min=0) // 64).view(-1, 1))
        bits |= torch.where(hit, bit.view(-1, 1), torch.zeros_like(bits))
        node = torch.where(there, parent[first + node.clamp(min=0)], node)
        depth += (node >= 0).to(depth.dtype)
    context = (s.kv_len - (s.cu_q[1:] - s.cu_q[:-1]))[b].long()
    token = context + i
    slots = s.page_table[b, token // PAGE].long() * PAGE + token % PAGE
    return {"masks": bits, "positions": (context + depth).to(torch.int32), "slots": slots.to(torch.int32)}


def _plain_values(tiles, at, scales_at, D):
    """One operand of tiles [B, pages, Hk, tile bytes] as float32 [B, Hk, keys, D]."""
    B, P, Hk, _ = tiles.shape
    G, S = D // 32, _scale_bytes(D)
    codes = tiles[..., at:at + 32 * D]
    e = tiles[..., scales_at:scales_at + PAGE * S].view(B, P, Hk, PAGE, S)[..., :G].int()
    one = torch.tensor(MAGNITUDES + tuple(-m for m in MAGNITUDES), device=tiles.device)
    pair = torch.stack([one.repeat(16), one.repeat_interleave(16)], dim=1)          # [256, 2]: low and high nibble
    x = pair[codes.int()].view(B, P, Hk, G, PAGE, 32)
    x = x.mul_((e << 23).view(torch.float32).permute(0, 1, 2, 4, 3).unsqueeze(-1))
    return x.permute(0, 2, 1, 4, 3, 5).reshape(B, Hk, P * PAGE, D)


def _plain_attention(s):
    B, D, H, Hk = len(s.counts), s.D, s.H, s.Hk
    dev, nq, R = s.q.device, s.max_q, H // Hk
    tiles = s.cache[s.page_table]                                                   # [B, pages, Hk, tile]
    S = tiles.shape[1] * PAGE
    keys = torch.arange(S, device=dev)
    there = (keys < s.kv_len.view(-1, 1)).view(B, 1, S, 1)
    k = _plain_values(tiles, 0, PAGE * D, D).masked_fill_(~there, 0.0)
    v = _plain_values(tiles, 32 * D, PAGE * D + PAGE * _scale_bytes(D), D).masked_fill_(~there, 0.0)
    n = s.cu_q[1:] - s.cu_q[:-1]
    at = torch.arange(nq, device=dev)
    rows = (s.cu_q[:-1].view(-1, 1) + at).clamp_(max=s.q.shape[0] - 1)
    row = at < n.view(-1, 1)
    q = s.q[rows].float().view(B, nq, Hk, R, D).permute(0, 2, 3, 1, 4).reshape(B, Hk, R * nq, D)
    scores = torch.matmul(q, k.transpose(2, 3).contiguous()).mul_(1.0 / math.sqrt(D)).view(B, Hk, R, nq, S)
    node = keys.view(1, -1) - (s.kv_len - n).view(-1, 1)                            # [B, S]
    words = s.masks[rows]                                                           # [B, nq, words]
    word = (node.clamp(min=0) // 64).clamp(max=words.shape[2] - 1)
    bits = torch.gather(words, 2, word.view(B, 1, S).expand(B, nq, S))
    bits = torch.bitwise_right_shift(bits, (node.clamp(min=0) % 64).view(B, 1, S)) & 1
    seen = (node.view(B, 1, S) < 0) | ((bits == 1) & (node < n.view(-1, 1)).view(B, 1, S))
    scores.masked_fill_(~seen.view(B, 1, 1, nq, S), -math.inf)
    top = scores.amax(dim=-1, keepdim=True)
    scores = scores.sub_(top.clamp(min=-3e38)).exp_()
    total = scores.sum(dim=-1, keepdim=True)
    out = torch.matmul(scores.view(B, Hk, R * nq, S), v).view(B, Hk, R, nq, D) / torch.where(total > 0, total, torch.ones_like(total))
    lse = (top + total.log()).squeeze(-1)
    out = out.permute(0, 3, 1, 2, 4).reshape(B, nq, H, D)
    lse = lse.permute(0, 3, 1, 2).reshape(B, nq, H)
    return {"out": out[row].to(torch.bfloat16), "lse": lse[row]}


def _weights(logits, temperature):
    """Probabilities [rows, V] in 64 bits, and the logarithms of what they were divided by."""
    x = logits.double()
    t = temperature.double().view(-1, 1)
    best = torch.zeros_like(x).scatter_(1, x.argmax(dim=1, keepdim=True), 1.0)
    x = x / torch.where(t > 0, t, torch.ones_like(t))
    x = torch.exp(x - x.amax(dim=1, keepdim=True))
    x = x / x.sum(dim=1, keepdim=True)
    return torch.where(t > 0, x, best)


def _take(w, u):
    """The lowest index up to which the weights add up to more than u of all."""
    c = w.cumsum(dim=1)
    v = (c <= u.double().view(-1, 1) * c[:, -1:]).sum(dim=1)
    last = w.shape[1] - 1 - (w.flip(1) > 0).to(torch.uint8).argmax(dim=1)
    return torch.minimum(v, last)


def _plain_draft(s):
    T, V = s.logits.shape
    b, i = _requests(s.cu_q, T)
    n = (s.cu_q[1:] - s.cu_q[:-1]).long()
    first = s.cu_q[:-1].long()
    step = max(1, int(5e7) // V)
    follows = torch.cat([s.ids[1:], s.ids[:1]]).long()
    pp, qq = torch.empty((T,), dtype=torch.float64, device=s.u.device), torch.ones((T,), dtype=torch.float64, device=s.u.device)
    for at in range(0, T, step):
        rows = slice(at, min(T, at + step))
        t = s.temperature[b[rows]]
        pp[rows] = _weights(s.logits[rows], t).gather(1, follows[rows].view(-1, 1)).view(-1)
        if s.draft is not None:
            qq[rows] = _weights(s.draft[rows], t).gather(1, follows[rows].view(-1, 1)).view(-1)
    greedy = s.temperature[b] == 0
    stands = torch.where(greedy, pp > 0, s.u.double() * qq < pp)
    fell = torch.where(stands | (i >= n[b] - 1), torch.full_like(b, T), i.long())
    m = torch.full((len(n),), T, dtype=torch.int64, device=b.device).scatter_reduce_(0, b, fell, "amin")
    m = torch.minimum(m, n - 1)                                                     # drafts that stand
    where = first + m
    p = _weights(s.logits[where], s.temperature)
    if s.draft is not None:
        q = _weights(s.draft[where], s.temperature)
    else:
        q = torch.zeros_like(p).scatter_(1, follows[where].view(-1, 1), 1.0)
    rest = ((m < n - 1) & (s.temperature > 0)).view(-1, 1)
    w = torch.where(rest, (p - q).clamp(min=0.0), p)
    last = _take(w, s.u_draw)
    k = m[b]
    tokens = torch.where(i < k, follows, torch.where(i == k, last[b], torch.full_like(follows, -1)))
    p_last = p.gather(1, last.view(-1, 1)).view(-1)
    logp = torch.where(i < k, pp, torch.where(i == k, p_last[b], torch.ones_like(pp))).log()
    return {"tokens": tokens.to(torch.int32), "n": (m + 1).to(torch.int32), "logp": logp.float()}


def _plain_tree(s):
    T, V = s.logits.shape
    b, i = _requests(s.cu_q, T)
    first = s.cu_q[b].long()
    step = max(1, int(5e7) // V)
    y, py = torch.empty((T,), dtype=torch.int64, device=b.device), torch.empty((T,), dtype=torch.float64, device=b.device)
    for at in range(0, T, step):
        rows = slice(at, min(T, at + step))
        p = _weights(s.logits[rows], s.temperature[b[rows]])
        y[rows] = _take(p, s.u[rows])
        py[rows] = p.gather(1, y[rows].view(-1, 1)).view(-1)
    # the lowest child of each node that has its token
    at = torch.arange(T, device=b.device)
    up = (first + s.parents).clamp(min=0)
    match = (s.parents >= 0) & (s.ids == y[up])
    child = torch.full((T + 1,), T, dtype=torch.int64, device=b.device)
    child.scatter_reduce_(0, torch.where(match, up, torch.full_like(up, T)), at, "amin")
    child[T] = T
    path = torch.full((T,), -1, dtype=torch.int64, device=b.device)
    tokens, logp = torch.full_like(path, -1), torch.zeros_like(py)
    B = len(s.counts)
    node, n = s.cu_q[:-1].long(), torch.zeros((B,), dtype=torch.int64, device=b.device)
    pad = lambda x, fill: torch.cat([x, torch.full((1,), fill, dtype=x.dtype, device=x.device)])
    path, tokens, logp, y, py = pad(path, -1), pad(tokens, -1), pad(logp, 0.0), pad(y, -1), pad(py, 1.0)
    start = s.cu_q[:-1].long()
    for step in range(s.depth + 1):
        there = node < T
        at = torch.where(there, start + step, torch.full_like(node, T))
        path[at] = torch.where(there, node - start, torch.full_like(node, -1))
        tokens[at] = torch.where(there, y[node], torch.full_like(node, -1))
        logp[at] = torch.where(there, py[node].log(), torch.zeros_like(py[node]))
        n += there.long()
        node = child[node]
    return {"path": path[:T].to(torch.int32), "tokens": tokens[:T].to(torch.int32), "n": n.to(torch.int32), "logp": logp[:T].float()}


def _entry_bytes(D, token):
    """Where a tile holds the tokens' [N] codes and scales: [N, bytes]."""
    S, G = _scale_bytes(D), D // 32
    dev = token.device
    codes = (torch.arange(2 * G, device=dev) * (16 * PAGE)).view(-1, 1) + torch.arange(16, device=dev)
    scales = (PAGE * D + torch.arange(2, device=dev) * (PAGE * S)).view(-1, 1) + torch.arange(S, device=dev)
    at = torch.cat([codes.view(-1), scales.view(-1)])
    each = torch.cat([torch.full((2 * G * 16,), 16, device=dev), torch.full((2 * S,), S, device=dev)])
    return at.view(1, -1) + token.view(-1, 1) * each.view(1, -1)


def _plain_keep(s):
    T = s.path.shape[0]
    b, i = _requests(s.cu_q, T)
    n = s.cu_q[1:] - s.cu_q[:-1]
    context = (s.kv_len - n)[b].long()
    moved = i < s.n_path[b]
    to = context + i
    source = torch.where(moved, context + s.path, to)
    page0, page1 = s.page_table[b, source // PAGE].long(), s.page_table[b, to // PAGE].long()
    at0, at1 = _entry_bytes(s.D, source % PAGE), _entry_bytes(s.D, to % PAGE)
    layer = torch.arange(s.cache.shape[0], device=b.device).view(-1, 1, 1, 1)
    head = torch.arange(s.Hk, device=b.device).view(1, 1, -1, 1)
    held = s.cache[layer, page0.view(1, -1, 1, 1), head, at0.view(1, T, 1, -1)]
    s.cache[layer, page1.view(1, -1, 1, 1), head, at1.view(1, T, 1, -1)] = held
    return {"cache": s.cache, "kv_len": s.kv_len - n + s.n_path}


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------
def _own(s):
    import paper_2606_02955_amd as fd
    if s.op == "layout":
        fd.fdllm_tree_layout(s.parents, s.kv_len, s.cu_q, s.max_q, s.masks, positions=s.positions, page_table=s.page_table,
                             slots=s.slots)
        return {"masks": s.masks, "positions": s.positions, "slots": s.slots}
    if s.op == "attention":
        s.ws = fd.fdllm_tree_attention(s.q, s.cache, s.page_table, s.kv_len, s.cu_q, s.masks, s.out, s.max_q, lse=s.lse,
                                       workspace=s.ws)
        return {"out": s.out, "lse": s.lse}
    if s.op == "draft":
        s.ws = fd.fdllm_verify_draft(s.logits, s.ids, s.cu_q, s.max_q, s.u, s.u_draw, s.tokens, s.n_tokens, draft=s.draft,
                                     temperature=s.temperature, logp=s.logp, workspace=s.ws)
        return {"tokens": s.tokens, "n": s.n_tokens, "logp": s.logp}
    if s.op == "tree":
        s.ws = fd.fdllm_verify_tree(s.logits, s.ids, s.parents, s.cu_q, s.max_q, s.u, s.path, s.tokens, s.n_tokens,
                                    temperature=s.temperature, logp=s.logp, workspace=s.ws)
        return {"path": s.path, "tokens": s.tokens, "n": s.n_tokens, "logp": s.logp}
    fd.fdllm_cache_keep(s.cache, s.page_table, s.kv_len, s.cu_q, s.path, s.n_path, s.max_q, s.kv_out)
    return {"cache": s.cache, "kv_len": s.kv_out}


def run(s):
    if own:
        return _own(s)
    return {"layout": _plain_layout, "attention": _plain_attention, "draft": _plain_draft, "tree": _plain_tree,
            "keep": _plain_keep}[s.op](s)


def work(case):
    counts = _nodes(case)
    T, B = sum(counts), case["B"]
    if case["op"] == "layout":
        words = -(-max(counts) // 64)
        return {"bytes": 4.0 * T + 8.0 * B + 4.0 * B + T * (8.0 * words + 8.0), "flops": 1.0 * T}
    if case["op"] == "attention":
        H, Hk, D = case["H"], case["Hk"], case["D"]
        context = _spread(B, case["lo"], case["hi"])
        seen = sum(n * (c + 1.0) for n, c in zip(counts, context))
        kv = sum(c + n for n, c in zip(counts, context)) * Hk * (D + 2.0 * (D // 32))
        return {"bytes": kv + T * H * (4.0 * D + 4.0) + 8.0 * T, "flops": 4.0 * D * H * seen}
    if case["op"] == "keep":
        moved = sum(m - 1 for m in _kept_nodes(case))
        entry = case["layers"] * case["Hk"] * (case["D"] + 2.0 * _scale_bytes(case["D"]))
        return {"bytes": 2.0 * moved * entry + 12.0 * B + 4.0 * moved, "flops": 0.0}
    rows = T + (T - B if case.get("marginals") else 0)
    e = 4.0 if case["dtype"] == "f32" else 2.0
    return {"bytes": rows * case["V"] * e + 24.0 * T, "flops": 3.0 * rows * case["V"]}


# ---------------------------------------------------------------------------
# the definition in 64 bits: a request at a time
# ---------------------------------------------------------------------------
def _ancestors(tree, i):
    seen = []
    while i >= 0:
        seen.append(i)
        i = tree[i]
    return seen


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


def _exact_attention(s):
    H, Hk, D = s.H, s.Hk, s.D
    out = torch.zeros((s.q.shape[0], H, D), dtype=torch.float64, device=s.q.device)
    lse = torch.full((s.q.shape[0], H), -math.inf, dtype=torch.float64, device=s.q.device)
    cu, lens, parents = s.cu_q.tolist(), s.kv_len.tolist(), s.parents.tolist()
    for b, length in enumerate(lens):
        tree = parents[cu[b]:cu[b + 1]]
        n, rows = len(tree), slice(cu[b], cu[b + 1])
        hidden = torch.zeros((n, length), dtype=torch.bool)
        for i in range(n):
            hidden[i, length - n:] = True
            hidden[i, [length - n + j for j in _ancestors(tree, i)]] = False
        hidden = hidden.to(s.q.device)
        for h in range(Hk):
            k = _exact_cached(s, b, h, length, 0, PAGE * D)
            v = _exact_cached(s, b, h, length, 32 * D, PAGE * D + PAGE * _scale_bytes(D))
            for hq in range(h * (H // Hk), (h + 1) * (H // Hk)):
                x = (s.q[rows, hq].double() @ k.t() / math.sqrt(D)).masked_fill_(hidden, -math.inf)
                z = torch.logsumexp(x, dim=1)
                lse[rows, hq] = z
                out[rows, hq] = torch.exp(x - z.view(-1, 1)) @ v
    return {"out": out, "lse": lse}


def _exact_row(logits, temperature):
    """log p of one row, float64."""
    x = logits.double()
    if temperature == 0.0:
        first = int((x == x.max()).nonzero()[0])
        return torch.full_like(x, -math.inf).index_fill_(0, torch.tensor([first], device=x.device), 0.0)
    return torch.log_softmax(x / temperature, dim=0)


def _exact_draw(w, u):
    c = torch.cumsum(w, 0)
    return int(torch.searchsorted(c, c[-1:] * u, right=True).clamp(max=int((w > 0).nonzero()[-1]))[0])


def _exact_draft(s):
    cu, ids, u, u_draw = s.cu_q.tolist(), s.ids.tolist(), s.u.tolist(), s.u_draw.tolist()
    tokens, counts, logps = [], [], []
    for b, t in enumerate(s.temperature.double().tolist()):
        got, lp = [], []
        for r in range(cu[b], cu[b + 1]):
            p = _exact_row(s.logits[r], t)
            w = p.exp()
            if r + 1 < cu[b + 1]:
                x = ids[r + 1]
                q = _exact_row(s.draft[r], t).exp() if s.draft is not None else None
                qx = 1.0 if q is None else float(q[x])
                if (float(w[x]) > 0.0) if t == 0.0 else (u[r] * qx < float(w[x])):
                    got.append(x)
                    lp.append(float(p[x]))
                    continue
                if t != 0.0:
                    if q is None:
                        w[x] = 0.0
                    else:
                        w = (w - q).clamp(min=0.0)
            y = _exact_draw(w, u_draw[b])
            got.append(y)
            lp.append(float(p[y]))
            break
        n = cu[b + 1] - cu[b]
        counts.append(len(got))
        tokens += got + [-1] * (n - len(got))
        logps += lp + [0.0] * (n - len(lp))
    dev = s.logits.device
    return {"tokens": torch.tensor(tokens, dtype=torch.int32, device=dev), "n": torch.tensor(counts, dtype=torch.int32, device=dev),
            "logp": torch.tensor(logps, dtype=torch.float64, device=dev)}


def _exact_tree(s):
    cu, ids, u, parents = s.cu_q.tolist(), s.ids.tolist(), s.u.tolist(), s.parents.tolist()
    paths, tokens, counts, logps = [], [], [], []
    for b, t in enumerate(s.temperature.double().tolist()):
        node, path, got, lp = 0, [], [], []
        n = cu[b + 1] - cu[b]
        while node is not None:
            r = cu[b] + node
            p = _exact_row(s.logits[r], t)
            y = _exact_draw(p.exp(), u[r])
            path.append(node)
            got.append(y)
            lp.append(float(p[y]))
            node = next((c for c in range(node + 1, n) if parents[cu[b] + c] == node and ids[cu[b] + c] == y), None)
        counts.append(len(got))
        paths += path + [-1] * (n - len(path))
        tokens += got + [-1] * (n - len(got))
        logps += lp + [0.0] * (n - len(lp))
    dev = s.logits.device
    return {"path": torch.tensor(paths, dtype=torch.int32, device=dev), "tokens": torch.tensor(tokens, dtype=torch.int32, device=dev),
            "n": torch.tensor(counts, dtype=torch.int32, device=dev), "logp": torch.tensor(logps, dtype=torch.float64, device=dev)}


def _exact_keep(s):
    D, S = s.D, _scale_bytes(s.D)
    old = s.cache.cpu()
    new = old.clone()
    cu, lens, table, path, kept = (x.tolist() for x in (s.cu_q, s.kv_len, s.page_table, s.path, s.n_path))
    for b, length in enumerate(lens):
        n = cu[b + 1] - cu[b]
        for i in range(kept[b]):
            (p0, t0), (p1, t1) = (divmod(length - n + j, PAGE) for j in (path[cu[b] + i], i))
            for at, each in [(g * 16 * PAGE, 16) for g in range(2 * D // 32)] + [(PAGE * D, S), (PAGE * (D + S), S)]:
                new[:, table[b][p1], :, at + t1 * each:at + (t1 + 1) * each] = \
                    old[:, table[b][p0], :, at + t0 * each:at + (t0 + 1) * each]
    kv = [length - (cu[b + 1] - cu[b]) + kept[b] for b, length in enumerate(lens)]
    return {"cache": new.to(s.cache.device), "kv_len": torch.tensor(kv, dtype=torch.int32, device=s.cache.device)}


def _exact_layout(s):
    cu, lens, table, parents = s.cu_q.tolist(), s.kv_len.tolist(), s.page_table.tolist(), s.parents.tolist()
    words = s.masks.shape[1]
    masks = torch.zeros(s.masks.shape, dtype=torch.int64)
    positions, slots = [], []
    for b, length in enumerate(lens):
        tree = parents[cu[b]:cu[b + 1]]
        for i in range(len(tree)):
            seen = _ancestors(tree, i)
            for w in range(words):
                value = sum(1 << (j % 64) for j in seen if j // 64 == w)
                masks[cu[b] + i, w] = value if value < 1 << 63 else value - (1 << 64)
            positions.append(length - len(tree) + len(seen) - 1)
            token = length - len(tree) + i
            slots.append(table[b][token // PAGE] * PAGE + token % PAGE)
    dev = s.cu_q.device
    return {"masks": masks.to(dev), "positions": torch.tensor(positions, dtype=torch.int32, device=dev),
            "slots": torch.tensor(slots, dtype=torch.int32, device=dev)}


def exact(case, seed):
    s = prepare(case, seed)
    return {"layout": _exact_layout, "attention": _exact_attention, "draft": _exact_draft, "tree": _exact_tree,
            "keep": _exact_keep}[s.op](s)
