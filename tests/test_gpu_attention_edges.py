"""The attention operators where a call is unusual: counts in another order,
launches of other shapes than small calls have, positions and values at the end
of their types.  Bounds as in test_gpu_attention.py."""
import numpy as np
import pytest
import torch

from oracle import attention as oa
from test_gpu_attention import _check, _i32, _normal, _np

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
