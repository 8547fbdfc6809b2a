"""Decoding with drafted tokens where offsets pass 32 bits: rows of logits far apart,
caches of more than 4 GiB.  Bounds as in test_gpu_drafts.py."""
import numpy as np
import pytest
import torch

from oracle import attention as oa
from oracle import drafts as od
from test_gpu_attention import _check, _fill, _i32, _normal, _np
from test_gpu_drafts import _check_draft, _check_tree, _cu, _logits, _masks, _numbers, _tree, _verify_draft, _verify_tree, _words

pytestmark = pytest.mark.gpu
DEV = "cuda"


def _far(x, stride):
    """x on the GPU with rows `stride` elements apart."""
    T, V = x.shape
    rows = torch.empty((T - 1) * stride + V, dtype=x.dtype, device=DEV).as_strided((T, V), (stride, 1))
    rows.copy_(x)
    return rows


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_rows_far_apart(gpu, dtype):
    V, counts = 5003, [3, 2]
    cu, x = _cu(counts), _logits(5, V, 1, dtype)
    logits = _far(x, (1 << 30) + 3)              # the last row begins beyond 2^32 elements
    ids = np.concatenate([[0], x.float().argmax(1).numpy()[:-1]])
    u, u_draw = _numbers(5, 2), _numbers(2, 3)
    _check_draft(counts, x, None, ids, None, u, u_draw, _verify_draft(gpu, counts, V, logits, None, ids, None, u, u_draw)[:3])
    near = _logits(5, V, 4, dtype)
    got = _verify_draft(gpu, counts, V, near.to(DEV), logits, ids, None, u, u_draw)
    _check_draft(counts, near, x, ids, None, u, u_draw, got[:3])
    parents = np.array([-1, 0, 1, -1, 0])
    _check_tree(cu, x, ids, parents, None, u, _verify_tree(gpu, cu, 3, logits, ids, parents, None, u)[:4])


def test_large_caches(gpu):
    D, H, Hk, n, context = 64, 4, 2, 9, 60
    tile = oa.tile_bytes(D)
    pages = (5 << 30) // (Hk * tile)             # the last ones lie beyond 2^32 bytes
    cache = torch.empty((pages, Hk, tile), dtype=torch.uint8, device=DEV)
    own = [pages - 1, pages - 7]
    k, v = _fill(cache, own, n + context, Hk, D, 1)
    parents = _tree(n, 2)
    sets = [od.ancestors(parents, i) for i in range(n)]
    q = _normal((n, H, D), 3, torch.bfloat16, 2.0)
    out = torch.full((n, H, D), float("nan"), dtype=torch.bfloat16, device=DEV)
    lse = torch.full((n, H), float("nan"), device=DEV)
    for width in (2, 200):                       # items whole, and divided
        table = np.full((1, width), -1)
        table[0, :2] = own
        gpu.fdllm_tree_attention(q, cache, _i32(table), _i32([n + context]), _i32([0, n]), _masks(_words(sets, 1)), out, n, lse=lse)
        torch.cuda.synchronize()
        seen = np.concatenate([np.ones((n, context), dtype=bool), [[j in s for j in range(n)] for s in sets]], axis=1)
        _check(out, lse, od.attend(_np(q.float()), k, v, D ** -0.5, seen), D)
    # layers of one page each, the last ones beyond 2^32 bytes too
    path = np.array([0, 2, 5, 8] + [-1] * 5)
    want = cache[own].cpu().numpy()[None].copy()
    new = od.keep(want, D, np.array([0, 1]), n + context, n, path, 4)
    kv_out = torch.zeros(1, dtype=torch.int32, device=DEV)
    args = (_i32([n + context]), _i32([0, n]), _i32(path), _i32([4]), n)
    before = cache[own].clone()
    gpu.fdllm_cache_keep(cache, _i32(table), *args, kv_out=kv_out)
    torch.cuda.synchronize()
    assert np.array_equal(cache[own].cpu().numpy(), want[0]) and kv_out.tolist() == [new]
    layers = cache[:pages // 2 * 2].view(pages // 2, 2, Hk, tile)
    layers[0], layers[-1] = before, before
    gpu.fdllm_cache_keep(layers, _i32([[0, 1]]), *args)
    torch.cuda.synchronize()
    for layer in (0, -1):
        assert np.array_equal(layers[layer].cpu().numpy(), want[0])
