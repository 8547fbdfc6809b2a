"""Norm and rotation where a workgroup takes several heads one after another, as
calls of a few thousand tokens do: bit for bit what small calls of the same
tokens give (a head a workgroup there), a sample of them against the float64
oracle.  With 33 heads of queries, keys and values a workgroup takes 2 heads from
3841 tokens on, 4 from 7265 and 8 from 13089 (above a head size of 128 from half
as many)."""
import numpy as np
import pytest
import torch

from oracle import attention as oa
from test_gpu_attention import _expected_rows, _i32, _normal, _np

pytestmark = pytest.mark.gpu
DEV = "cuda"

CASES = [
    # T, H, Hk, D, rot, interleaved, norm, dtype, in place
    (4000, 27, 3, 128, 128, False, True, torch.bfloat16, False),      # 2 heads: 26 is the last of q, 27 the first of k
    (8001, 27, 3, 96, 96, True, True, torch.bfloat16, False),         # 4
    (14000, 27, 3, 128, 128, False, True, torch.bfloat16, False),     # 8: one workgroup has q, k and v, the last one head
    (14017, 27, 3, 128, 64, True, True, torch.float32, True),
    (13999, 28, 4, 64, 64, False, True, torch.bfloat16, True),
    (7000, 27, 3, 160, 128, False, True, torch.bfloat16, False),      # 16 lanes a row
    (6999, 27, 3, 256, 256, True, False, torch.float32, True),
    (14000, 27, 3, 32, 0, False, True, torch.bfloat16, False),
]


@pytest.mark.parametrize("T,H,Hk,D,rot,inter,norm,dtype,in_place", CASES)
def test_several_heads_a_workgroup(gpu, T, H, Hk, D, rot, inter, norm, dtype, in_place):
    wide = _normal((T, (H + 2 * Hk) * D), D + T, dtype, 1.5)
    q, k, v = (wide[:, a * D:b * D].view(T, b - a, D) for a, b in ((0, H), (H, H + Hk), (H + Hk, H + 2 * Hk)))
    if in_place:
        q, k = q.contiguous(), k.contiguous()
    qw, kw = (_normal((D,), i) if norm else None for i in (5, 6))
    angle = torch.rand((50, max(rot // 2, 1)), generator=torch.Generator().manual_seed(T)) * 6.28
    cs = torch.cat([angle.cos(), angle.sin()], 1).contiguous().to(DEV) if rot else None
    rng = np.random.default_rng(T)
    pos = rng.integers(0, 50, T)
    pages = T // 64 + 2
    slots = rng.permutation(pages * 64)[:T]
    slots[rng.integers(0, T, 5)] = -1
    pos32, slots32 = _i32(pos), _i32(slots)

    def call(rows, q, k, q_out, k_out, cache):
        gpu.fdllm_qk_norm_rope(q[rows], k[rows], v[rows], pos32[rows], cs, q_out[rows], k_out=k_out[rows], q_weight=qw,
                               k_weight=kw, interleaved=inter, cache=cache, slots=slots32[rows])

    small_q, small_k = (torch.full((T, h, D), 7.0, dtype=dtype, device=DEV) for h in (H, Hk))
    small_cache, cache = gpu.new_cache(pages, Hk, D), gpu.new_cache(pages, Hk, D)
    for first in range(0, T, 512):
        call(slice(first, min(first + 512, T)), q, k, small_q, small_k, small_cache)
    sample = rng.integers(0, T, 12)
    want_q = _expected_rows(q[sample], qw, 1e-6, cs, pos[sample], rot, inter)
    want_k = _expected_rows(k[sample], kw, 1e-6, cs, pos[sample], rot, inter)
    q_out, k_out = (q, k) if in_place else (torch.full((T, h, D), 9.0, dtype=dtype, device=DEV) for h in (H, Hk))
    call(slice(0, T), q, k, q_out, k_out, cache)
    torch.cuda.synchronize()
    assert torch.equal(q_out, small_q) and torch.equal(k_out, small_k) and torch.equal(cache, small_cache)
    rounding = 2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -24
    for got, want in ((q_out[sample], want_q), (k_out[sample], want_k)):
        err = np.abs(_np(got) - want)
        assert (err <= rounding * np.abs(want) * 1.001 + 2e-6 * np.abs(want).max(-1, keepdims=True)).all()
    raw, vn = cache.cpu().numpy(), _np(v[sample])
    for i, t in enumerate(sample):
        if slots[t] < 0:
            continue
        for h in range(Hk):
            held = np.concatenate([oa.value_of(*oa.quantise_group(g)) for g in vn[i, h].reshape(-1, 32)])
            assert np.array_equal(oa.get(raw[slots[t] // 64, h], D, True, slots[t] % 64), held)
