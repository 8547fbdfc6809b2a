"""The attention operators where a call is unusual: counts in another order,
launches of other shapes than small calls have, positions and values at the end
of their types.  Bounds as in test_gpu_attention.py."""
import numpy as np
import pytest
import torch

from oracle import attention as oa
from test_gpu_attention import _check, _i32, _normal, _np, _run_cache, _want

pytestmark = pytest.mark.gpu
DEV = "cuda"


def _prompt(gpu, q, k, v, cu_q, cu_k, max_q, blk=0):
    out = torch.full(q.shape, float("nan"), dtype=torch.bfloat16, device=DEV)
    lse = torch.full(q.shape[:2], float("nan"), device=DEV)
    ws = gpu.fdllm_prompt_attention(q, k, v, _i32(cu_q), _i32(cu_k), out, max_q, lse=lse, blk=blk)
    torch.cuda.synchronize()
    return out, lse, ws


@pytest.mark.parametrize("H,blk", [(4, 0), (1, 0), (5, 1)])
def test_sequences_in_another_order_with_divided_keys(gpu, H, blk):
    # the middle sequence's counts run backwards: it is left out, and the last lies
    # before the first
    D, Hk, L = 64, 1, 4000
    q = _normal((128, H, D), 1, torch.bfloat16, 2.0)
    k, v = (_normal((2 * L, Hk, D), 2 + i, torch.bfloat16) for i in range(2))
    out, lse, ws = _prompt(gpu, q, k, v, [64, 128, 0, 64], [L, 2 * L, 0, L], 64, blk)
    assert ws is not None                                  # the keys are divided
    for rows, keys in ((slice(64, 128), slice(L, 2 * L)), (slice(0, 64), slice(0, L))):
        want = oa.attend(_np(q[rows].float()), _np(k[keys].float()), _np(v[keys].float()), D ** -0.5, blk, L - 64)
        _check(out[rows], lse[rows], want, D)


def test_tokens_in_several_sequences_with_divided_keys(gpu):
    # four sequences are the same tokens over the same keys: more row tiles than a
    # call has room for where no token is in two
    D, H, L = 64, 16, 4000
    q = _normal((64, H, D), 5, torch.bfloat16, 2.0)
    k, v = (_normal((L, 1, D), 6 + i, torch.bfloat16) for i in range(2))
    out, lse, ws = _prompt(gpu, q, k, v, [0, 64, 0, 64, 0, 64, 0, 64], [0, L, 0, L, 0, L, 0, L], 64)
    assert ws is not None
    _check(out, lse, oa.attend(_np(q.float()), _np(k.float()), _np(v.float()), D ** -0.5, 0, 0), D)


def _cache_of(gpu, k, v):
    """A cache of one sequence's keys and values, [T, Hk, D] float32, and its page table."""
    T, Hk, D = k.shape
    cache = gpu.new_cache(-(-T // 64), Hk, D)
    gpu.fdllm_qk_norm_rope(k, k, v, _i32(np.zeros(T)), None, torch.empty_like(k), cache=cache, slots=_i32(range(T)))
    return cache, torch.arange(cache.shape[0], dtype=torch.int32, device=DEV).view(1, -1)


@pytest.mark.parametrize("D,H,Hk,n,T", [
    (64, 4, 1, 1, 300), (128, 1, 1, 32, 300), (128, 2, 1, 30, 300),        # whole items: 16 rows, 32 rows, two waves by two
    (96, 4, 1, 32, 100), (128, 4, 1, 32, 3000), (64, 2, 2, 1, 9000)])      # four waves of rows; divided items
def test_nan_over_the_cache_is_not_an_empty_row(gpu, D, H, Hk, n, T):
    k, v = (_normal((T, Hk, D), i) for i in range(2))
    q = _normal((n, H, D), 3, torch.bfloat16)

    def run(q, k, blk):
        cache, table = _cache_of(gpu, k, v)
        out, lse = torch.empty_like(q), torch.empty((n, H), device=DEV)
        gpu.fdllm_cache_attention(q, cache, table, _i32([T]), _i32([0, n]), out, n, lse=lse, blk=blk)
        torch.cuda.synchronize()
        return out, lse

    clean, clean_lse = run(q, k, 1)
    bad_q = q.clone()
    bad_q[n // 2, H - 1, 7] = float("nan")
    out, lse = run(bad_q, k, 1)
    hit = torch.zeros((n, H), dtype=torch.bool, device=DEV)
    hit[n // 2, H - 1] = True
    assert out[hit].isnan().all() and lse[hit].isnan().all()
    assert torch.equal(out[~hit], clean[~hit]) and torch.equal(lse[~hit], clean_lse[~hit])
    # a key that the later half of the tokens sees
    bad_k = k.clone()
    bad_k[T - 1 - (n - 1) // 2, 0, 9] = float("nan")
    out, lse = run(q, bad_k, 1)
    hit = torch.zeros((n, H), dtype=torch.bool, device=DEV)
    hit[n - 1 - (n - 1) // 2:, :H // Hk] = True
    assert out[hit].isnan().all() and lse[hit].isnan().all()
    assert torch.equal(out[~hit], clean[~hit]) and torch.equal(lse[~hit], clean_lse[~hit])


@pytest.mark.parametrize("D,H,n,T", [(128, 2, 100, 100), (64, 3, 5, 3000), (96, 1, 70, 2000)])
def test_nan_in_a_prompt_is_not_an_empty_row(gpu, D, H, n, T):
    q = _normal((n, H, D), 1, torch.bfloat16)
    k, v = (_normal((T, 1, D), 2 + i, torch.bfloat16) for i in range(2))
    clean, clean_lse, _ = _prompt(gpu, q, k, v, [0, n], [0, T], n, 1)
    bad_q = q.clone()
    bad_q[n // 2, H - 1, 7] = float("nan")
    out, lse, _ = _prompt(gpu, bad_q, k, v, [0, n], [0, T], n, 1)
    hit = torch.zeros((n, H), dtype=torch.bool, device=DEV)
    hit[n // 2, H - 1] = True
    assert out[hit].isnan().all() and lse[hit].isnan().all()
    assert torch.equal(out[~hit], clean[~hit]) and torch.equal(lse[~hit], clean_lse[~hit])
    bad_k = k.clone()
    bad_k[T - 1 - (n - 1) // 2, 0, 9] = float("nan")
    out, lse, _ = _prompt(gpu, q, bad_k, v, [0, n], [0, T], n, 1)
    hit = torch.zeros((n, H), dtype=torch.bool, device=DEV)
    hit[n - 1 - (n - 1) // 2:] = True
    assert out[hit].isnan().all() and lse[hit].isnan().all()
    assert torch.equal(out[~hit], clean[~hit]) and torch.equal(lse[~hit], clean_lse[~hit])


@pytest.mark.parametrize("blk", [1, 32, 1 << 30])
def test_query_positions_at_the_end_of_their_type(gpu, blk):
    # positions past every key see all of them, also where counting on would leave 32 bits
    D, H, n, T = 64, 2, 8, 150
    k, v = (_normal((T, 1, D), i) for i in range(2))
    cache, table = _cache_of(gpu, k, v)
    q = _normal((2 * n, H, D), 2, torch.bfloat16)
    out, lse = torch.empty_like(q), torch.empty((2 * n, H), device=DEV)
    held = [torch.empty((T, 1, D), dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    gpu.fdllm_cache_read(cache, _i32(range(T)), *held)
    for start in ((2 ** 31 - 1, 2 ** 31 - 5), (-2 ** 31, 2 ** 31 - 8)):
        gpu.fdllm_cache_attention(q, cache, table.expand(2, -1).contiguous(), _i32([T, T]), _i32([0, n, 2 * n]), out, n,
                                  lse=lse, blk=blk, q_start=_i32(start))
        torch.cuda.synchronize()
        for rows, s in zip((slice(0, n), slice(n, 2 * n)), start):
            want = oa.attend(_np(q[rows].float()), _np(held[0].float()), _np(held[1].float()), D ** -0.5, blk, s)
            _check(out[rows], lse[rows], want, D)


def test_prompt_with_many_row_tiles(gpu):
    # 65536 tokens of 32 heads on one key head: 16384 row tiles; some of the rows
    D, H, T = 64, 32, 65536
    q = _normal((T, H, D), 1, torch.bfloat16)
    k, v = (_normal((T, 1, D), 2 + i, torch.bfloat16) for i in range(2))
    out, lse, _ = _prompt(gpu, q, k, v, [0, T], [0, T], T, 1)
    assert not out.isnan().any() and not lse.isnan().any()
    kn, vn = _np(k.float()), _np(v.float())
    for t in (0, 1, 127, 40000, 65532, 65535):
        _check(out[t:t + 1], lse[t:t + 1], oa.attend(_np(q[t:t + 1].float()), kn, vn, D ** -0.5, 1, t), D)


def test_prompt_with_room_for_more_queries_than_there_are(gpu):
    D, H = 64, 4
    q = _normal((133, H, D), 1, torch.bfloat16)
    k, v = (_normal((133, 2, D), 2 + i, torch.bfloat16) for i in range(2))
    out, lse, _ = _prompt(gpu, q, k, v, [0, 100, 133], [0, 100, 133], 100, 1)
    more, more_lse, _ = _prompt(gpu, q, k, v, [0, 100, 133], [0, 100, 133], 1 << 30, 1)
    assert torch.equal(out, more) and torch.equal(lse, more_lse)


def _ragged(B, n, longest, seed):
    """B sequences of at most n queries and `longest` cached tokens, some without either."""
    g = np.random.default_rng(seed)
    seqs = [(int(g.integers(1, n + 1)), int(g.integers(1, longest + 1))) for _ in range(B)]
    for i in range(0, B, 17):
        seqs[i] = (0, seqs[i][1])
    for i in range(5, B, 23):
        seqs[i] = (seqs[i][0], 0)
    seqs[1] = (n, longest)
    return seqs


@pytest.mark.parametrize("D,H,Hk,blk,B,n,longest", [
    (64, 1, 1, 1, 1100, 1, 200),         # 8 waves, 512 threads: up to three sequences a thread
    (64, 2, 2, 0, 600, 1, 400),
    (64, 4, 4, 32, 520, 20, 130),        # tiles of 32 rows
    (64, 8, 1, 1, 300, 8, 500),          # two waves of rows: 256 threads, up to two sequences a thread
    (64, 8, 1, 0, 300, 16, 500),         # four waves of rows
    (96, 6, 1, 32, 100, 8, 700),         # more sequences than a wave has lanes, one a thread
    (128, 8, 1, 0, 65, 16, 300),
    (64, 5, 1, 1, 256, 40, 200)])        # several groups of rows, a sequence a thread
def test_cache_attention_of_many_sequences(gpu, D, H, Hk, blk, B, n, longest):
    q, kv, cu, out, lse, _, _ = _run_cache(gpu, D, H, Hk, blk, _ragged(B, n, longest, B + n), B)
    torch.cuda.synchronize()
    _check(out, lse, _want(q, kv, cu, blk, D), D)
