"""Calls of so many rows that the terms of bfloat16 logits come out of a table, over
more requests than a wave has lanes: the tokens are the oracle's, and the same as in
calls of few rows; logarithms of probabilities agree within the bound of both,
2^-24 of themselves and 1e-11 each.  Bounds as in test_gpu_drafts.py."""
import numpy as np
import pytest
import torch

from test_gpu_drafts import (DEV, _check_draft, _check_tree, _cu, _logits, _np, _numbers, _strided, _tree, _verify_draft,
                             _verify_tree)

pytestmark = pytest.mark.gpu

# the table is taken from 6144 chunks of 2048 logits on, of both sides
V, CHUNKS = 9001, 5


def _near(a, b):
    a, b = _np(a).astype(np.float64), _np(b).astype(np.float64)
    assert (np.abs(a - b) <= 2.0 ** -23 * np.abs(b) * 1.001 + 2e-11).all()


def test_trees(gpu):
    B, n = 210, 6
    T, cu = B * n, _cu([n] * B)
    assert T * CHUNKS >= 6144
    x = _logits(T, V, 21, torch.bfloat16, peak=12.0)
    x[::50] = -float("inf")                       # (rows that cannot have any token)
    x[7::50, ::3] = 0.0                           # patterns that the table does not have
    parents = np.concatenate([_tree(n, b) for b in range(B)])
    g, likely = np.random.default_rng(4), x.float().topk(3, dim=1).indices.numpy()
    ids = np.array([likely[cu[i // n] + max(parents[i], 0), g.integers(0, 3)] for i in range(T)])
    temperature = [(1.0, 0.5, 0.0, 0.15, 1.0, 2.0)[b % 6] for b in range(B)]
    u, logits = _numbers(T, 5), _strided(x, 1)
    whole = _verify_tree(gpu, cu, n, logits, ids, parents, temperature, u)
    _check_tree(cu, logits, ids, parents, temperature, u, whole[:4])
    for b in (0, 1, 64, 65, 137, 209):
        rows = slice(cu[b], cu[b + 1])
        one = _verify_tree(gpu, [0, n], n, logits[rows], ids[rows], parents[rows], temperature[b:b + 1], u[rows])
        assert torch.equal(one[0], whole[0][rows]) and torch.equal(one[1], whole[1][rows])
        assert torch.equal(one[2], whole[2][b:b + 1])
        _near(one[3], whole[3][rows])


@pytest.mark.parametrize("marginals", [True, False])
def test_chains(gpu, marginals):
    # 1 to 5 rows a request, and one in eleven without any
    counts = [0 if b % 11 == 10 else 1 + b % 5 for b in range(230 if marginals else 500)]
    B, T, cu = len(counts), sum(counts), _cu(counts)
    assert (2 * T if marginals else T) * CHUNKS >= 6144
    x = _logits(T, V, 22, torch.bfloat16)
    d = (x.float() + 0.6 * torch.randn((T, V), generator=torch.Generator().manual_seed(23))).to(torch.bfloat16)
    ids = np.concatenate([[0], (d if marginals else x).float().argmax(1).numpy()[:-1]])
    temperature = [(1.0, 1.0, 0.7, 0.0, 1.3)[b // 5 % 5] for b in range(B)]
    u, u_draw = _numbers(T, 24), _numbers(B, 25)
    logits, draft = x.to(DEV), _strided(d, 3) if marginals else None
    whole = _verify_draft(gpu, counts, V, logits, draft, ids, temperature, u, u_draw)
    _check_draft(counts, logits, draft, ids, temperature, u, u_draw, whole[:3])
    for b in (0, 4, 63, 64, 150, B - 1):
        rows = slice(cu[b], cu[b + 1])
        if counts[b] == 0:
            continue
        one = _verify_draft(gpu, [counts[b]], V, logits[rows], draft[rows] if marginals else None, ids[rows], temperature[b:b + 1],
                            u[rows], u_draw[b:b + 1])
        assert torch.equal(one[0], whole[0][rows]) and torch.equal(one[1], whole[1][b:b + 1])
        _near(one[2], whole[2][rows])


@pytest.mark.parametrize("alike", [1.0, 0.3, -3.0, 0.0])
def test_equal_logits(gpu, alike):
    # 4096 rows of 8192 equal logits: the numbers beside a border, and the middle of a token's share
    B, V = 4096, 8192
    x = torch.full((B, V), alike, dtype=torch.bfloat16, device=DEV)
    k = np.random.default_rng(3).integers(1, V, B)
    for off, want in ((2.0 ** -24, k), (-2.0 ** -24, k - 1), (0.5 / V, k)):
        u = (k / V + off).astype(np.float32)
        assert (np.abs(u.astype(np.float64) - k / V) > 1e-9).all()
        got = _verify_tree(gpu, np.arange(B + 1), 1, x, np.zeros(B), np.full(B, -1), None, u)
        # (numbers above 1/2 are a step of 2^-24 apart, so that the offset is a whole one)
        assert got[1].tolist() == want.tolist()
        _near(got[3], torch.full((B,), -float(np.log(V))))
