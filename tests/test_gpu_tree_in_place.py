"""Tree attention whose results take the place of its queries: the same bits as
beside them, for whole and divided items, and rows of no request stay as they are."""
import pytest
import torch

from test_gpu_drafts import _run_tree

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("D,H,Hk,reqs", [
    (128, 8, 2, [(4, 500)]), (64, 4, 1, [(16, 20000), (9, 3)]), (96, 6, 2, [(61, 190), (60, 4), (1, 0)]),
    (64, 16, 2, [(130, 9001), (26, 40)]), (128, 28, 4, [(40, 3000)] * 6), (64, 1, 1, [(1 + i % 5, 7 * i) for i in range(100)])])
def test_out_is_q(gpu, D, H, Hk, reqs):
    args, _, _, cu, out, lse, ws = _run_tree(gpu, D, H, Hk, reqs, True, D + H)
    q, cache, table, kv_len, cu_q, masks, _, max_q = args
    for _ in range(3):
        held, lse2 = q.clone(), torch.full_like(lse, float("nan"))
        gpu.fdllm_tree_attention(held, cache, table, kv_len, cu_q, masks, held, max_q, lse=lse2, workspace=ws)
        torch.cuda.synchronize()
        assert torch.equal(held, out) and torch.equal(lse2, lse)
    # the last request's rows belong to none
    held = q.clone()
    short = cu_q.clone()
    short[-1] = short[-2]
    gpu.fdllm_tree_attention(held, cache, table, kv_len, short, masks, held, max_q)
    torch.cuda.synchronize()
    assert torch.equal(held[cu[-2]:], q[cu[-2]:])
    with pytest.raises(Exception, match="invalid"):
        gpu.fdllm_tree_attention(q, cache, table, kv_len, cu_q, masks, q, max_q, lse=q.view(torch.float32).view(-1)[:lse.numel()].view_as(lse))
