"""GPU parity of decoding with drafted tokens against the float64 oracle.

Bounds.  Masks, positions, slots, tokens, paths, counts and cache bytes are
equal.  A token drawn may differ from the oracle's only where its number lies
within the two sides' summation errors of a border: terms are off by 4e-13, sums of
V <= 2^17 doubles by less, so 1e-11 of the whole; the inputs below have none that
near (asserted).  The logarithm of a probability is formed in 64 bits and rounded
once: half a step of float32, 2^-24 of it, plus 1e-11.  Attention as in
test_gpu_attention.py.
"""
import numpy as np
import pytest
import torch

from oracle import attention as oa
from oracle import drafts as od
from test_gpu_attention import _check, _fill, _i32, _normal, _np

pytestmark = pytest.mark.gpu
DEV = "cuda"


def _cu(counts):
    return np.concatenate([[0], np.cumsum(counts)])


def _tree(n, seed, reach=4):
    g = np.random.default_rng(seed)
    return np.array([-1] + [int(g.integers(max(0, i - reach), i)) for i in range(1, n)], dtype=np.int64)[:n]


def _words(sets, words):
    out = np.zeros((len(sets), words), dtype=np.uint64)
    for i, s in enumerate(sets):
        for j in s:
            out[i, j // 64] |= np.uint64(1) << np.uint64(j % 64)
    return out


def _masks(words):
    return torch.tensor(words.view(np.int64), device=DEV)


# ---------------------------------------------------------------------------
# layout
# ---------------------------------------------------------------------------
@pytest.mark.parametrize("counts,reach,words_more", [
    ([1], 1, 0), ([2, 0, 1], 1, 1), ([64], 4, 0), ([65], 64, 0), ([63, 64, 1, 65, 128, 129], 7, 0), ([250], 1, 0),
    ([256, 257, 3], 30, 0), ([320, 5], 1, 3), ([1024], 1, 0), ([1024, 1000], 900, 0), ([3] * 100, 2, 0)])
def test_layout(gpu, counts, reach, words_more):
    T, cu, B = sum(counts), _cu(counts), len(counts)
    g = np.random.default_rng(T)
    parents = np.concatenate([_tree(n, 7 * b + n, reach) for b, n in enumerate(counts)])
    context = g.integers(0, 300, B)
    lens = context + np.array(counts)
    table = g.permutation(B * 21).reshape(B, 21)
    words = -(-max(counts) // 64) + words_more
    masks = torch.full((T, words), 77, dtype=torch.int64, device=DEV)
    pos, slots = (torch.full((T,), 77, dtype=torch.int32, device=DEV) for _ in range(2))
    gpu.fdllm_tree_layout(_i32(parents), _i32(lens), _i32(cu), max(counts), masks, positions=pos, page_table=_i32(table),
                          slots=slots)
    torch.cuda.synchronize()
    got = masks.cpu().numpy().view(np.uint64)
    for b, n in enumerate(counts):
        rows = slice(cu[b], cu[b + 1])
        sets = [od.ancestors(parents[rows], i) for i in range(n)]
        assert np.array_equal(got[rows], _words(sets, words))
        assert pos[rows].tolist() == [context[b] + len(s) - 1 for s in sets]
        assert slots[rows].tolist() == [table[b, (context[b] + i) // 64] * 64 + (context[b] + i) % 64 for i in range(n)]


def test_layout_of_unusual_trees(gpu):
    # parents that are no earlier nodes, several roots, rows of no request, tables without a page, lengths below the nodes'
    parents = np.array([9, 0, 1, 5, -7, 2, 0, 1, 2, 3, 0, 0, 1 << 30, -1, 13])
    cu, lens, max_q = np.array([0, 6, 4, 13, 15]), [6, 50, 130, 1], 8
    table = np.array([[3, 9, 9], [9, 9, 9], [1, -1, 0], [2, 9, 9]])
    masks = torch.full((15, 1), 77, dtype=torch.int64, device=DEV)
    pos, slots = (torch.full((15,), 77, dtype=torch.int32, device=DEV) for _ in range(2))
    gpu.fdllm_tree_layout(_i32(parents), _i32(lens), _i32(cu), max_q, masks, positions=pos, page_table=_i32(table), slots=slots)
    torch.cuda.synchronize()
    # request 1 runs backwards, request 2 has 9 rows: more than max_q
    assert (masks[6:13] == 77).all() and (pos[6:13] == 77).all() and (slots[6:13] == 77).all()
    for rows, n, length, page in ((slice(0, 6), 6, 6, 3), (slice(13, 15), 2, 1, 2)):
        sets = [od.ancestors(parents[rows], i) for i in range(n)]
        assert np.array_equal(masks[rows].cpu().numpy().view(np.uint64), _words(sets, 1))
        assert pos[rows].tolist() == [length - n + len(s) - 1 for s in sets]
        assert slots[rows].tolist() == [page * 64 + length - n + i if length - n + i >= 0 else -1 for i in range(n)]
    # a page that is none, and a table that ends
    gpu.fdllm_tree_layout(_i32(np.full(8, -1)), _i32([132]), _i32([0, 8]), 8, masks[:8], slots=slots[:8], page_table=_i32([[1, -1]]))
    torch.cuda.synchronize()
    assert slots[:8].tolist() == [-1] * 8
    gpu.fdllm_tree_layout(_i32(np.full(8, -1)), _i32([132]), _i32([0, 8]), 8, masks[:8], slots=slots[:8],
                          page_table=_i32([[1, -1, 5]]))
    torch.cuda.synchronize()
    assert slots[:8].tolist() == [-1] * 4 + [320 + i for i in range(4)] and masks[:8, 0].tolist() == [1 << i for i in range(8)]


# ---------------------------------------------------------------------------
# attention
# ---------------------------------------------------------------------------
ATTENTION_CASES = [
    # D, H, Hk, [(nodes, context)], any mask instead of a tree's
    (128, 8, 8, [(1, 0)], False),
    (128, 8, 2, [(4, 500)], False),                                       # 16 rows
    (64, 4, 1, [(3, 60), (4, 61), (1, 0), (2, 700)], False),              # nodes across a page's end
    (96, 6, 2, [(5, 130), (0, 40), (3, 3)], True),
    (128, 2, 2, [(32, 1000), (17, 47), (31, 64)], False),                 # 32 rows
    (128, 8, 4, [(32, 225), (9, 63)], True),                              # two waves by two
    (64, 4, 2, [(26, 480), (1, 1023)], False),
    (96, 4, 2, [(61, 190), (60, 4)], True),
    (128, 8, 2, [(61, 450), (1, 64), (17, 0)], False),                    # 128 rows a workgroup, several groups
    (64, 8, 1, [(130, 333), (65, 31), (64, 0), (129, 2)], True),          # words of the mask more than one
    (128, 5, 1, [(70, 65), (2, 130)], False),
    (64, 4, 1, [(16, 20000)], True),                                      # divided items
    (96, 16, 16, [(40, 3000)], False),
    (128, 4, 4, [(26, 2022)], False),
    (64, 40, 8, [(32, 20)] * 33, False),
    (64, 1, 1, [(1 + i % 5, 7 * i) for i in range(200)], True),           # more requests than a wave has lanes
]


def _run_tree(gpu, D, H, Hk, reqs, any_mask, seed, junk_words=0, stride_more=0):
    g = np.random.default_rng(seed)
    lens = [c + n for n, c in reqs]
    need = [-(-n // 64) for n in lens]
    total = sum(need) + 2
    cache = torch.randint(0, 256, (total, Hk, oa.tile_bytes(D)), dtype=torch.uint8, device=DEV)
    order = g.permutation(total)
    table = np.full((len(reqs), max(need) + 1), 1 << 30)
    at, kv, seen, rows = 0, [], [], []
    words = -(-max(n for n, _ in reqs) // 64) + junk_words
    for b, m in enumerate(need):
        table[b, :m] = order[at:at + m]
        kv.append(_fill(cache, order[at:at + m], lens[b], Hk, D, seed + b))
        at += m
        n = reqs[b][0]
        parents = _tree(n, seed + b)
        bits = g.random((n, n)) < 0.4 if any_mask else \
            np.array([[j in od.ancestors(parents, i) for j in range(n)] for i in range(n)], dtype=bool).reshape(n, n)
        if any_mask and n > 1:
            bits[n // 2] = False                                          # without a context: a row that sees nothing
        w = g.integers(0, 1 << 63, (n, words), dtype=np.uint64) * np.uint64(2) + np.uint64(1)   # any bits from n on
        for j in range(n):
            one = np.uint64(1) << np.uint64(j % 64)
            w[:, j // 64] = np.where(bits[:, j], w[:, j // 64] | one, w[:, j // 64] & ~one)
        rows.append(w)
        seen.append(np.concatenate([np.ones((n, reqs[b][1]), dtype=bool), bits], axis=1))
    cu = _cu([n for n, _ in reqs])
    T = int(cu[-1])
    wide = _normal((T, H * D + stride_more), seed, torch.bfloat16, 2.0)
    q = wide[:, :H * D].view(T, H, D)
    masks = _masks(np.concatenate(rows))
    out = torch.full((T, H, D), float("nan"), dtype=torch.bfloat16, device=DEV)
    lse = torch.full((T, H), float("nan"), device=DEV)
    args = (q, cache, _i32(table), _i32(lens), _i32(cu), masks, out, max(n for n, _ in reqs))
    ws = gpu.fdllm_tree_attention(*args, lse=lse)
    return args, kv, seen, cu, out, lse, ws


@pytest.mark.parametrize("D,H,Hk,reqs,any_mask", ATTENTION_CASES)
def test_tree_attention(gpu, D, H, Hk, reqs, any_mask):
    args, kv, seen, cu, out, lse, _ = _run_tree(gpu, D, H, Hk, reqs, any_mask, 13 * D + H, junk_words=H % 2,
                                                stride_more=8 * (H % 3))
    torch.cuda.synchronize()
    parts = [od.attend(_np(args[0][cu[b]:cu[b + 1]].float()), *kv[b], D ** -0.5, seen[b]) for b in range(len(reqs))]
    _check(out, lse, [np.concatenate(x) for x in zip(*parts)], D)


@pytest.mark.parametrize("D,H,Hk,n,context", [(128, 8, 2, 4, 90), (64, 8, 4, 20, 300), (96, 4, 1, 40, 3000), (128, 16, 4, 130, 64)])
def test_a_chain_is_the_causal_mask(gpu, D, H, Hk, n, context):
    args, kv, seen, cu, out, lse, ws = _run_tree(gpu, D, H, Hk, [(n, context)], False, 3)
    q, cache, table, kv_len, cu_q, masks, _, max_q = args
    gpu.fdllm_tree_layout(_i32(np.arange(-1, n - 1)), kv_len, cu_q, n, masks)
    gpu.fdllm_tree_attention(*args, lse=lse, workspace=ws)
    out2, lse2 = torch.empty_like(out), torch.empty_like(lse)
    gpu.fdllm_cache_attention(q, cache, table, kv_len, cu_q, out2, max_q, lse=lse2, blk=1)
    torch.cuda.synchronize()
    # (they divide the keys by other rules, so that both are held to the oracle's bounds; where both
    # give equal shares they agree bit for bit)
    want = oa.attend(_np(q.float()), *kv[0], D ** -0.5, 1, context)
    _check(out, lse, want, D)
    _check(out2, lse2, want, D)
    if context == 3000:
        assert torch.equal(out, out2) and torch.equal(lse, lse2)


def test_tree_attention_of_unusual_requests(gpu):
    # more nodes than cached tokens, a request out of order, one with more than max_q rows, pages that are not there
    D, H, Hk = 64, 2, 1
    cache = torch.randint(0, 256, (5, Hk, oa.tile_bytes(D)), dtype=torch.uint8, device=DEV)
    k, v = _fill(cache, [2], 3, Hk, D, 1)
    k2, v2 = _fill(cache, [0, 4], 100, Hk, D, 2)
    table, lens = np.array([[2, 1 << 30], [0, 4], [0, 4], [-1, 4]]), [3, 100, 100, 100]
    cu, T = [0, 5, 3, 12, 16], 16
    q = _normal((T, H, D), 3, torch.bfloat16, 2.0)
    masks = torch.full((T, 1), -1, dtype=torch.int64, device=DEV)
    out = torch.full((T, H, D), 7.0, dtype=torch.bfloat16, device=DEV)
    lse = torch.full((T, H), 7.0, device=DEV)
    gpu.fdllm_tree_attention(q, cache, _i32(table), _i32(lens), _i32(cu), masks, out, 6, lse=lse)
    torch.cuda.synchronize()
    assert (out[5:12] == 7).all() and (lse[5:12] == 7).all()
    _check(out[:5], lse[:5], od.attend(_np(q[:5].float()), k, v, D ** -0.5, np.ones((5, 3), dtype=bool)), D)
    seen = np.ones((4, 100), dtype=bool)
    seen[:, :64] = False
    _check(out[12:], lse[12:], od.attend(_np(q[12:].float()), k2, v2, D ** -0.5, seen), D)
    # a table of no pages, and lengths below zero: nothing is seen
    empty = torch.empty((4, 0), dtype=torch.int32, device=DEV)
    for t, kv in ((empty, lens), (_i32(table), [-9, -1 << 31, 0, -1])):
        gpu.fdllm_tree_attention(q, cache, t, _i32(kv), _i32([0, 5, 5, 12, 16]), masks, out, 7, lse=lse)
        torch.cuda.synchronize()
        assert (out == 0).all() and torch.isneginf(lse).all()


# ---------------------------------------------------------------------------
# verification
# ---------------------------------------------------------------------------
def _logits(T, V, seed, dtype, peak=8.0, filtered=0):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((T, V), generator=g) * 1.5
    best = torch.randint(0, V, (T, 3), generator=g)
    x.scatter_add_(1, best, peak * torch.rand((T, 3), generator=g) + 2.0)
    if filtered:
        x[x < x.topk(min(filtered, V), dim=1).values[:, -1:]] = -float("inf")
    return x.to(dtype)


def _numbers(n, seed):
    return np.random.default_rng(seed).random(n).astype(np.float32)


def _f32(x):
    return torch.tensor(np.asarray(x, dtype=np.float32), device=DEV)


def _strided(x, more):
    """x on the GPU with rows that lie `more` elements further apart, behind other elements."""
    T, V = x.shape
    wide = torch.full((T * (V + more) + 3,), 9.0, dtype=x.dtype, device=DEV)
    view = wide[3:].view(T, V + more)[:, :V] if more else wide[3:3 + T * V].view(T, V)
    view.copy_(x)
    return view


def _check_logp(got, want):
    got, want = _np(got), np.asarray(want)
    assert (np.abs(got - want) <= 2.0 ** -24 * np.abs(want) * 1.001 + 1e-11).all(), np.abs(got - want).max()


def _verify_draft(gpu, counts, V, logits, draft, ids, temperature, u, u_draw, max_q=None, cu=None, workspace=None):
    T, cu = len(ids), _cu(counts) if cu is None else cu
    tokens = torch.full((T,), 77, dtype=torch.int32, device=DEV)
    n_tokens = torch.full((len(cu) - 1,), 77, dtype=torch.int32, device=DEV)
    logp = torch.full((T,), 77.0, device=DEV)
    ws = gpu.fdllm_verify_draft(logits, _i32(ids), _i32(cu), max_q or max(counts), _f32(u), _f32(u_draw), tokens, n_tokens,
                                draft=draft, temperature=None if temperature is None else _f32(temperature), logp=logp,
                                workspace=workspace)
    torch.cuda.synchronize()
    return tokens, n_tokens, logp, ws


def _check_draft(counts, logits, draft, ids, temperature, u, u_draw, got):
    tokens, n_tokens, logp = got
    cu = _cu(counts)
    x, d = _np(logits.float()), None if draft is None else _np(draft.float())
    most = 0
    for b, n in enumerate(counts):
        rows = slice(cu[b], cu[b + 1])
        if n == 0:
            assert n_tokens[b] == 0
            continue
        t = 1.0 if temperature is None else float(np.float32(temperature[b]))
        want, lp, near = od.verify_draft(x[rows], ids[rows], None if d is None else d[rows], t, u[rows], u_draw[b])
        assert near > 1e-11
        assert n_tokens[b] == len(want)
        assert tokens[rows].tolist() == want + [-1] * (n - len(want))
        _check_logp(logp[rows], lp + [0.0] * (n - len(lp)))
        most = max(most, len(want))
    return most


DRAFT_CASES = [
    # counts, V, dtype, drafter's logits, filtered, temperatures, elements between rows
    ([1], 5, torch.bfloat16, True, 0, None, 0),
    ([4], 1, torch.float32, True, 0, None, 0),                            # a vocabulary of one
    ([5, 1, 3, 0, 2], 1000, torch.bfloat16, True, 0, [1.0, 0.5, 0.0, 1.0, 2.0], 0),
    ([5, 1, 3, 0, 2], 1001, torch.bfloat16, False, 0, [1.0, 0.5, 0.0, 1.0, 2.0], 5),
    ([9] * 12, 2047, torch.bfloat16, True, 0, None, 1),
    ([9] * 12, 2048, torch.float32, True, 20, None, 0),
    ([9] * 12, 2049, torch.float32, False, 20, None, 3),
    ([3, 17, 2], 32003, torch.bfloat16, True, 0, [0.7, 0.9, 1.1], 0),
    ([33], 4099, torch.bfloat16, True, 0, [0.3], 0),
    ([5], 126464, torch.bfloat16, True, 0, [0.8], 0),
    ([4], 140000, torch.float32, True, 0, [0.8], 0),                      # chunks more than a wave has lanes
    ([3, 2], 300001, torch.bfloat16, False, 0, [1.5, 0.0], 0),
    ([2] * 300, 130, torch.bfloat16, True, 0, None, 0),
    ([64] * 5, 700, torch.float32, True, 300, [1e-3, 1e4, 1.0, 0.0, 0.2], 0),
]


@pytest.mark.parametrize("counts,V,dtype,marginals,filtered,temperature,more", DRAFT_CASES)
def test_verify_draft(gpu, counts, V, dtype, marginals, filtered, temperature, more):
    T, B, seed = sum(counts), len(counts), sum(counts) + V
    x = _logits(T, V, seed, dtype, filtered=filtered)
    g = torch.Generator().manual_seed(seed + 1)
    d = (x.float() + 0.7 * torch.randn((T, V), generator=g)).to(dtype) if marginals else None
    t = np.repeat(np.ones(B) if temperature is None else np.maximum(temperature, 1e-3), counts)
    # drafts drawn from the drafter: most of a chain stands
    from_ = (d if d is not None else x).float() / torch.tensor(t, dtype=torch.float32).view(-1, 1)
    noise = -torch.log(-torch.log(torch.rand((T, V), generator=g).clamp(1e-7, 1 - 1e-7)))
    ids = np.concatenate([[0], (from_ + noise).argmax(1).numpy()[:-1]])
    if T > 6:
        ids[4] = V if T % 2 else -1                                       # no token
    u, u_draw = _numbers(T, seed + 2), _numbers(B, seed + 3)
    logits, draft = _strided(x, more), None if d is None else _strided(d, 2 * more)
    got = _verify_draft(gpu, counts, V, logits, draft, ids, temperature, u, u_draw)
    _check_draft(counts, logits, draft, ids, temperature, u, u_draw, got[:3])
    again = _verify_draft(gpu, counts, V, logits, draft, ids, temperature, u, u_draw, workspace=got[3])
    for a, b in zip(got[:3], again[:3]):
        assert torch.equal(a, b)


def test_verify_draft_all_stand_and_none(gpu):
    # the drafter's logits are the target's: everything stands; then a drafter sure of what cannot be
    V, counts = 3001, [6, 6]
    x = _logits(12, V, 3, torch.bfloat16).to(DEV)
    ids = np.concatenate([[0], x.float().argmax(1).cpu().numpy()[:-1]])
    u, u_draw = np.full(12, 1.0 - 2.0 ** -24, dtype=np.float32), _numbers(2, 5)
    got = _verify_draft(gpu, counts, V, x, x, ids, None, u, u_draw)
    assert got[1].tolist() == [6, 6]
    _check_draft(counts, x, x, ids, None, u, u_draw, got[:3])
    d = torch.full_like(x, -float("inf"))
    for r in range(12):
        x[r, 7] = -float("inf")
        d[r, 7] = 0.0
    ids[:] = 7
    for draft in (d, None):
        got = _verify_draft(gpu, counts, V, x, draft, ids, None, np.zeros(12), u_draw)
        assert got[1].tolist() == [1, 1]
        _check_draft(counts, x, draft, ids, None, np.zeros(12, dtype=np.float32), u_draw, got[:3])


def test_verify_draft_unusual_rows_and_numbers(gpu):
    V = 500
    x = _logits(18, V, 9, torch.float32)
    x[3] = -float("inf")                         # no token can be: nothing stands, -1 is drawn
    x[6, :] = -float("inf")
    x[6, 499] = -3.0                             # one token
    x[9] = 2.0                                   # all alike
    x[12] = x[12] * 0 + torch.tensor([0.0, -3e38] * (V // 2))
    d = x.clone()
    d[1] = -float("inf")                         # a drafter's row without tokens: the draft falls
    counts = [3, 3, 3, 3, 3, 3]
    ids = np.concatenate([[0], x.argmax(1).numpy()[:-1]])
    nan = float("nan")
    u_draw = np.array([0.5, 0.2, 1.0, -4.0, nan, np.inf], dtype=np.float32)
    u = np.array([0.1, 0.2, nan, 0.5, 0.1, 0.1, -1.0, 0.0, 0.1] + [0.0] * 9, dtype=np.float32)
    x, d = x.to(DEV), d.to(DEV)
    for draft in (d, None):
        for temperature in (None, [1.0, 0.5, np.inf, 1e-30, nan, -2.0]):
            got = _verify_draft(gpu, counts, V, x, draft, ids, temperature, u, u_draw)
            assert got[1][1] == 1 and got[0][3] == -1 and got[2][3] == 0
            _check_draft(counts, x, draft, ids, temperature, u, u_draw, got[:3])


def test_verify_draft_leaves_other_rows(gpu):
    V = 800
    x = _logits(20, V, 4, torch.bfloat16).to(DEV)
    ids = np.concatenate([[0], x.float().argmax(1).cpu().numpy()[:-1]])
    u, u_draw = _numbers(20, 1), _numbers(4, 2)
    cu = np.array([12, 16, 3, 11, 11])           # 12..16, one that runs backwards, 8 rows (more than max_q), none
    got = _verify_draft(gpu, None, V, x, None, ids, None, u, u_draw, max_q=5, cu=cu)
    assert got[1].tolist()[1:] == [0, 0, 0]
    want, lp, near = od.verify_draft(_np(x[12:16].float()), ids[12:16], None, 1.0, u[12:16], u_draw[0])
    assert got[1][0] == len(want) and got[0][12:16].tolist() == want + [-1] * (4 - len(want))
    out = np.r_[0:12, 16:20]
    assert (got[0][out] == 77).all() and (got[2][out] == 77).all()


def test_verify_draft_without_rows(gpu):
    empty = torch.empty((0, 100), dtype=torch.bfloat16, device=DEV)
    got = _verify_draft(gpu, [0, 0], 100, empty, None, np.zeros(0), None, np.zeros(0), np.zeros(2), max_q=4)
    assert got[1].tolist() == [0, 0]


TREE_CASES = [
    ([1], 5, torch.bfloat16, 0, None, 0),
    ([4], 1, torch.float32, 0, None, 0),
    ([20, 1, 7, 0, 2], 1000, torch.bfloat16, 0, [1.0, 0.5, 0.0, 1.0, 2.0], 0),
    ([64, 3], 2049, torch.float32, 30, [0.9, 0.0], 3),
    ([26], 126464, torch.bfloat16, 0, [0.8], 0),
    ([9], 140001, torch.bfloat16, 0, [1.0], 1),
    ([3] * 200, 77, torch.bfloat16, 0, None, 0),
    ([1000], 63, torch.float32, 0, None, 0),
]


def _verify_tree(gpu, cu, max_q, logits, ids, parents, temperature, u, workspace=None):
    T = len(ids)
    path, tokens = (torch.full((T,), 77, dtype=torch.int32, device=DEV) for _ in range(2))
    n_tokens = torch.full((len(cu) - 1,), 77, dtype=torch.int32, device=DEV)
    logp = torch.full((T,), 77.0, device=DEV)
    ws = gpu.fdllm_verify_tree(logits, _i32(ids), _i32(parents), _i32(cu), max_q, _f32(u), path, tokens, n_tokens,
                               temperature=None if temperature is None else _f32(temperature), logp=logp, workspace=workspace)
    torch.cuda.synchronize()
    return path, tokens, n_tokens, logp, ws


def _check_tree(cu, logits, ids, parents, temperature, u, got):
    path, tokens, n_tokens, logp = got
    x = _np(logits.float())
    for b in range(len(cu) - 1):
        rows, n = slice(cu[b], cu[b + 1]), cu[b + 1] - cu[b]
        if n == 0:
            assert n_tokens[b] == 0
            continue
        t = 1.0 if temperature is None else float(np.float32(temperature[b]))
        want, toks, lp, near = od.verify_tree(x[rows], ids[rows], parents[rows], t, u[rows])
        assert near > 1e-11
        fill = [-1] * (n - len(want))
        assert n_tokens[b] == len(want) and path[rows].tolist() == want + fill and tokens[rows].tolist() == toks + fill
        _check_logp(logp[rows], lp + [0.0] * len(fill))


@pytest.mark.parametrize("counts,V,dtype,filtered,temperature,more", TREE_CASES)
def test_verify_tree(gpu, counts, V, dtype, filtered, temperature, more):
    T, B, seed, cu = sum(counts), len(counts), sum(counts) + V, _cu(counts)
    x = _logits(T, V, seed, dtype, peak=12.0, filtered=filtered)
    parents = np.concatenate([_tree(n, seed + b) for b, n in enumerate(counts)])
    u = _numbers(T, seed + 2)
    # nodes hold likely tokens of their parents', several children the same
    g = np.random.default_rng(seed)
    likely = x.float().topk(min(3, V), dim=1).indices.numpy()
    ids = g.integers(0, V, T)
    for b in range(B):
        for i in range(1, counts[b]):
            ids[cu[b] + i] = likely[cu[b] + parents[cu[b] + i], g.integers(0, likely.shape[1])]
    logits = _strided(x, more)
    got = _verify_tree(gpu, cu, max(counts), logits, ids, parents, temperature, u)
    _check_tree(cu, logits, ids, parents, temperature, u, got[:4])
    again = _verify_tree(gpu, cu, max(counts), logits, ids, parents, temperature, u, workspace=got[4])
    for a, b in zip(got[:4], again[:4]):
        assert torch.equal(a, b)


def test_verify_tree_walks_to_the_end(gpu):
    # greedy chains: every node's token is its only child's; then the lowest of equal children
    V, n = 900, 150
    x = _logits(n, V, 1, torch.bfloat16).to(DEV)
    best = x.float().argmax(1).cpu().numpy()
    ids, parents = np.concatenate([[5], best[:-1]]), np.arange(-1, n - 1)
    got = _verify_tree(gpu, [0, n], n, x, ids, parents, [0.0], np.zeros(n))
    assert got[2][0] == n and got[0].tolist() == list(range(n)) and got[1].tolist() == best.tolist()
    parents[:] = 0
    ids[:] = best[0]
    got = _verify_tree(gpu, [0, n], n, x, ids, parents, [0.0], np.zeros(n))
    assert got[2][0] == 2 and got[0][:3].tolist() == [0, 1, -1]
    # parents that are no earlier nodes hang on nothing; ids that are no tokens match nothing
    parents[1:] = [1 << 30, 2, 3, -5] + [0] * (n - 5)
    ids[5] = -1
    got = _verify_tree(gpu, [0, n], n, x, ids, parents, [0.0], np.zeros(n))
    assert got[2][0] == 2 and got[0][1] == 6
    x[0] = -float("inf")
    for t in ([0.0], None):
        got = _verify_tree(gpu, [0, n], n, x, np.full(n, -1), np.where(np.arange(n) == 0, -1, 0), t, np.zeros(n))
        assert got[2][0] == 1 and got[1][0] == -1 and got[3][0] == 0


def _mixed_rows(T, V, seed, dtype=torch.bfloat16):
    """Rows of many kinds: far from 0, zeros, nothing near 0, -inf in between and at the end."""
    x = _logits(T, V, seed, torch.float32)
    x[1::8] += 200.0
    x[2::8] *= 30.0
    x[3::8, ::7] = 0.0
    x[4::8] *= 1e-6
    x[5::8, V // 2:] = -float("inf")
    x[6::8, 1000:] = -float("inf")
    return x.to(dtype)


@pytest.mark.parametrize("B", [9, 11])
def test_many_rows_of_bfloat16(gpu, B):
    # rows almost enough, and enough, for the terms to be looked up in a table; temperatures that allow it and not
    V, n = 126464, 10
    T, cu, parents = n * B, _cu([n] * B), np.tile(_tree(n, 5), B)
    x = _mixed_rows(T, V, 3)
    temperature = [1.0, 0.2, 0.19, 0.0, 3.0, 1e-3, 1.0, 1.0, 50.0, 0.7, 1.0][:B]
    likely = x.float().topk(2, dim=1).indices.numpy()
    ids = np.zeros(T, dtype=np.int64)
    for b in range(B):
        for i in range(1, n):
            ids[cu[b] + i] = likely[cu[b] + parents[cu[b] + i], i % 2]
    u, logits = _numbers(T, 8), _strided(x, 1)
    _check_tree(cu, logits, ids, parents, temperature, u, _verify_tree(gpu, cu, n, logits, ids, parents, temperature, u)[:4])


def test_many_requests_with_a_drafter(gpu):
    # requests and rows enough for every variant: the table, the sums of p - q apart
    V, counts = 126464, [2 + b % 3 for b in range(44)]
    T = sum(counts)
    x = _mixed_rows(T, V, 4)
    g = torch.Generator().manual_seed(6)
    d = (x.float() + 0.5 * torch.randn((T, V), generator=g)).to(torch.bfloat16)
    ids = np.concatenate([[0], d.float().topk(2, dim=1).indices[:, 1].numpy()[:-1]])
    temperature = [(1.0, 0.0, 0.5, 2.0, 0.1)[b % 5] for b in range(44)]
    u, u_draw = _numbers(T, 1), _numbers(44, 2)
    logits, draft = x.to(DEV), _strided(d, 3)
    got = _verify_draft(gpu, counts, V, logits, draft, ids, temperature, u, u_draw)
    _check_draft(counts, logits, draft, ids, temperature, u, u_draw, got[:3])


def test_equal_logits_take_the_lowest(gpu):
    V = 5000
    x = torch.zeros((2, V), dtype=torch.bfloat16, device=DEV)
    x[:, [17, 3000, 4999]] = 3.0
    got = _verify_tree(gpu, [0, 1, 2], 1, x, np.zeros(2), np.full(2, -1), [0.0, 1.0], np.zeros(2))
    assert got[1].tolist() == [17, 0]
    # all alike: u = 1/4 is a border, where the weights are not more than u of all before the next token
    x[:] = 1.0
    u = np.nextafter(np.float32(0.25), [0.0, 1.0]).astype(np.float32)      # (in 64 bits: 1/4 both)
    got = _verify_tree(gpu, [0, 1, 2], 1, x, np.zeros(2), np.full(2, -1), None, u)
    assert u.tolist() == [0.25, 0.25] and got[1].tolist() == [V // 4, V // 4]
    u = np.float32(0.25) + np.float32([-2.0 ** -26, 2.0 ** -25])           # and the floats beside it
    got = _verify_tree(gpu, [0, 1, 2], 1, x, np.zeros(2), np.full(2, -1), None, u)
    assert got[1].tolist() == [V // 4 - 1, V // 4]


def test_requests_do_not_change_each_other(gpu):
    V, n = 9001, 6
    x = _logits(40 * n, V, 2, torch.bfloat16).to(DEV)
    d = _logits(40 * n, V, 3, torch.bfloat16).to(DEV)
    ids = np.concatenate([[0], x.float().argmax(1).cpu().numpy()[:-1]])
    u, u_draw = _numbers(40 * n, 1), _numbers(40, 2)
    cu = _cu([n] * 40)
    whole = _verify_draft(gpu, [n] * 40, V, x, d, ids, None, u, u_draw)
    parents = np.tile(np.arange(-1, n - 1), 40)
    tree = _verify_tree(gpu, cu, n, x, ids, parents, None, u)
    for b in (0, 17, 39):
        rows = slice(cu[b], cu[b + 1])
        one = _verify_draft(gpu, [n], V, x[rows], d[rows], ids[rows], None, u[rows], u_draw[b:b + 1])
        for a, w in zip((one[0], one[2], one[1]), (whole[0][rows], whole[2][rows], whole[1][b:b + 1])):
            assert torch.equal(a, w)
        one = _verify_tree(gpu, [0, n], n, x[rows], ids[rows], parents[rows], None, u[rows])
        for a, w in zip((one[0], one[1], one[3], one[2]), (tree[0][rows], tree[1][rows], tree[3][rows], tree[2][b:b + 1])):
            assert torch.equal(a, w)


def test_draws_follow_the_probabilities(gpu):
    # 4096 requests with evenly spaced numbers: each token as often as its probability says, give or take one
    V, B = 40, 4096
    row = _logits(1, V, 8, torch.float32, peak=3.0)
    x = row.expand(B, V).contiguous().to(DEV)
    u = ((np.arange(B) + 0.5) / B).astype(np.float32)
    got = _verify_tree(gpu, np.arange(B + 1), 1, x, np.zeros(B), np.full(B, -1), None, u)
    count = np.bincount(got[1].cpu().numpy(), minlength=V)
    assert (np.abs(count - B * od.softmax(_np(row)[0], 1.0)) <= 1.0).all()


# ---------------------------------------------------------------------------
# what is kept
# ---------------------------------------------------------------------------
@pytest.mark.parametrize("D,Hk,layers,pages,reqs", [
    (64, 1, None, 3, [(5, 20, [0, 2, 3, 4])]),                            # sources that are places of others
    (128, 2, 3, 8, [(40, 50, [0, 1, 7, 8, 39]), (3, 0, [0, 2]), (0, 10, []), (30, 60, [])]),
    (96, 3, 2, 8, [(64, 63, [0] + list(range(2, 64))), (10, 64, [0, 9])]),
    (32, 1, 1, 4, [(100, 3, list(range(0, 100, 2)))]),
    (256, 2, 2, 4, [(9, 60, [0, 3, 5, 6, 8])]),
    (160, 1, 5, 6, [(20, 55, [3, 4, 5, 19]), (20, 50, [0])]),             # the root replaced too
])
def test_cache_keep(gpu, D, Hk, layers, pages, reqs):
    g = np.random.default_rng(D)
    shape = ((layers,) if layers else ()) + (pages, Hk, oa.tile_bytes(D))
    raw = g.integers(0, 256, shape, dtype=np.uint8)
    cache = torch.tensor(raw, device=DEV)
    counts, lens = [r[0] for r in reqs], [r[0] + r[1] for r in reqs]
    need = [-(-n // 64) for n in lens]
    table = np.full((len(reqs), max(need) + 1), -1)
    order = g.permutation(pages)
    at = 0
    for b, m in enumerate(need):
        table[b, :m] = order[at:at + m]
        at += m
    assert at <= pages
    cu = _cu(counts)
    path = np.full(cu[-1], -1)
    for b, r in enumerate(reqs):
        path[cu[b]:cu[b] + len(r[2])] = r[2]
    kept = [len(r[2]) for r in reqs]
    kv_out = torch.full((len(reqs),), 77, dtype=torch.int32, device=DEV)
    gpu.fdllm_cache_keep(cache, _i32(table), _i32(lens), _i32(cu), _i32(path), _i32(kept), max(counts), kv_out=kv_out)
    torch.cuda.synchronize()
    want = raw.reshape((layers or 1,) + raw.shape[-3:]).copy()
    new = [od.keep(want, D, table[b], lens[b], counts[b], path[cu[b]:cu[b + 1]], kept[b]) for b in range(len(reqs))]
    assert np.array_equal(cache.cpu().numpy().reshape(want.shape), want) and kv_out.tolist() == new
    assert not np.array_equal(want.reshape(raw.shape), raw)


def test_cache_keep_moves_nothing_that_is_not_there(gpu):
    D, pages = 64, 4
    g = np.random.default_rng(1)
    raw = g.integers(0, 256, (pages, 1, oa.tile_bytes(D)), dtype=np.uint8)
    # entries before their place or no nodes; pages that are none; a count that cannot be; counts out of order
    cu, lens = np.array([0, 6, 12, 16, 14]), [6, 70, 10, 20]
    path = np.array([3, 1, 1, 6, -1, 5, 0, 2, 3, 4, 5, -1, 0, 1, 2, 3])
    table, kept = np.array([[0, 1], [2, 1 << 20], [3, 1], [3, 1]]), [6, 5, 5, 1]
    cache = torch.tensor(raw, device=DEV)
    kv_out = torch.full((4,), 77, dtype=torch.int32, device=DEV)
    gpu.fdllm_cache_keep(cache, _i32(table), _i32(lens), _i32(cu), _i32(path), _i32(kept), 6, kv_out=kv_out)
    torch.cuda.synchronize()
    want = raw[None].copy()
    new = [od.keep(want, D, table[b], lens[b], 6, path[cu[b]:cu[b] + 6], kept[b]) for b in range(2)]
    assert np.array_equal(cache.cpu().numpy(), want[0]) and kv_out.tolist() == new + [10, 20]
    # no lengths wanted, no pages, no tokens
    gpu.fdllm_cache_keep(cache, _i32(table), _i32(lens), _i32(cu), _i32(path), _i32([0] * 4), 6)
    gpu.fdllm_cache_keep(cache[:0], _i32(table), _i32(lens), _i32(cu), _i32(path), _i32(kept), 6, kv_out=kv_out)
    torch.cuda.synchronize()
    assert np.array_equal(cache.cpu().numpy(), want[0])
