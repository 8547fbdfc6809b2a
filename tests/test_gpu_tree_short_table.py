"""Trees whose tokens go past the end of the page table: nodes stay where the length
says they are, as in the layout and where entries move, and what has no page is
seen by nobody.  Bounds as in test_gpu_attention.py."""
import numpy as np
import pytest
import torch

from oracle import drafts as od
from test_gpu_drafts import DEV, _check, _i32, _np, _run_tree, _tree

pytestmark = pytest.mark.gpu

CASES = [
    # D, H, Hk, [(nodes, context)], any mask instead of a tree's, columns of the table
    (64, 4, 2, [(10, 60)], False, 1),                                     # nodes 4 on have no page
    (128, 8, 2, [(10, 60), (3, 10), (40, 100)], True, 1),                 # the last has only a part of its context
    (96, 6, 2, [(40, 100), (61, 60), (5, 130)], False, 2),
    (128, 8, 2, [(61, 450), (130, 333), (17, 0)], True, 6),               # words of the mask more than one
    (128, 4, 4, [(26, 2022)], False, 31),                                 # no node has a page
    (64, 4, 1, [(16, 20000)], True, 300),                                 # divided items
    (64, 16, 2, [(26, 9001), (25, 8965)], False, 141),                    # 9024 of 9027 tokens, and all but none
    (64, 1, 1, [(1 + i % 5, 61 + i) for i in range(100)], True, 1),       # more requests than a wave has lanes
]


@pytest.mark.parametrize("D,H,Hk,reqs,any_mask,width", CASES)
def test_nodes_past_the_table(gpu, D, H, Hk, reqs, any_mask, width):
    args, kv, seen, cu, out, lse, _ = _run_tree(gpu, D, H, Hk, reqs, any_mask, 7 * D + width)
    q, cache, table, kv_len, cu_q, masks, _, max_q = args
    # a table that ends, and one whose other pages are none
    ends = table[:, :width].contiguous()
    none = table.clone()
    none[:, width:] = -1
    keys = 64 * width
    parts = [od.attend(_np(q[cu[b]:cu[b + 1]].float()), kv[b][0][:keys], kv[b][1][:keys], D ** -0.5, seen[b][:, :keys])
             for b in range(len(reqs))]
    want = [np.concatenate(x) for x in zip(*parts)]
    for t in (none, ends):
        out.fill_(float("nan"))
        lse.fill_(float("nan"))
        gpu.fdllm_tree_attention(q, cache, t, kv_len, cu_q, masks, out, max_q, lse=lse)
        torch.cuda.synchronize()
        _check(out, lse, want, D)


def test_the_longest_lengths(gpu):
    # lengths up to the largest number: all of the table is context
    D, H, Hk, n, width = 64, 4, 2, 9, 2
    args, kv, seen, cu, out, lse, _ = _run_tree(gpu, D, H, Hk, [(n, 128 - n)], False, 5)
    q, cache, table, _, cu_q, masks, _, max_q = args
    want = od.attend(_np(q.float()), *kv[0], D ** -0.5, np.ones((n, 128), dtype=bool))
    for length in (128 + n, (1 << 31) - 1):
        gpu.fdllm_tree_attention(q, cache, table[:, :width].contiguous(), _i32([length]), cu_q, masks, out, max_q, lse=lse)
        torch.cuda.synchronize()
        _check(out, lse, want, D)


def test_layout_and_attention_agree(gpu):
    # a node whose slot the layout does not know has no key; the others see theirs and the context's alone
    D, H, Hk, n, context, width = 64, 2, 1, 12, 59, 1
    args, kv, seen, cu, out, lse, _ = _run_tree(gpu, D, H, Hk, [(n, context)], False, 8)
    q, cache, table, kv_len, cu_q, masks, _, max_q = args
    parents, short = _tree(n, 8), table[:, :width].contiguous()
    pos, slots = (torch.full((n,), 77, dtype=torch.int32, device=DEV) for _ in range(2))
    own = torch.empty_like(masks)
    gpu.fdllm_tree_layout(_i32(parents), kv_len, cu_q, n, own, positions=pos, page_table=short, slots=slots)
    gpu.fdllm_tree_attention(q, cache, short, kv_len, cu_q, own, out, n, lse=lse)
    torch.cuda.synchronize()
    stored = [s >= 0 for s in slots.tolist()]
    assert stored == [i < 64 - context for i in range(n)]
    sees = np.zeros((n, 64), dtype=bool)
    sees[:, :context] = True
    for i in range(n):
        for j in od.ancestors(parents, i):
            if stored[j]:
                sees[i, context + j] = True
    _check(out, lse, od.attend(_np(q.float()), kv[0][0][:64], kv[0][1][:64], D ** -0.5, sees), D)
