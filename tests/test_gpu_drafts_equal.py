"""Chains whose drafter has the target's probabilities, or nearly: where p - q is
positive nowhere the token comes from p, whatever the roundings of p and q are, and
where it is small the borders are as far off as it is smaller.

Bounds as in test_gpu_drafts.py; and for a draw from max(p - q, 0), whose weights sum
to S: p and q are each off by 1.2e-12 of themselves at most (three terms of 3.9e-13),
p is taken less by 1.9e-12 of itself, so a sum of differences is off by 4.3e-12, and a
border, a sum by another one, by twice that over S: less than 9e-12 / S.
"""
import numpy as np
import pytest
import torch

from oracle import drafts as od
from oracle import drafts as od
from test_gpu_drafts import DEV, _check_draft, _cu, _logits, _numbers, _verify_draft

pytestmark = pytest.mark.gpu


def _falls(counts, V, what, x):
    """Drafts of which every request's first falls: no token, or one that cannot be."""
    ids = np.concatenate([[0], x.float().argmax(1).numpy()[:-1]])
    ids[_cu(counts)[:-1] + 1] = {"below": -1, "beyond": V, "impossible": 5}[what]
    return ids


@pytest.mark.parametrize("what", ["below", "beyond", "impossible"])
@pytest.mark.parametrize("B", [3, 40])                # max(p - q, 0) in the decision, and apart
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_the_same_rows(gpu, dtype, B, what):
    V, counts = 1000, [3] * B
    x = _logits(3 * B, V, B, dtype)
    x[:, 5] = -float("inf")
    ids = _falls(counts, V, what, x)
    u, u_draw = _numbers(3 * B, 1), _numbers(B, 2)
    t = [(1.0, 0.7, 1.9)[b % 3] for b in range(B)]
    logits = x.to(DEV)
    for draft in (logits, logits.clone()):
        got = _verify_draft(gpu, counts, V, logits, draft, ids, t, u, u_draw)
        assert got[1].tolist() == [1] * B
        _check_draft(counts, logits, draft, ids, t, u, u_draw, got[:3])


def _sixteenths(T, V, seed):
    """Odd sixteenths from -8 to 8: exact in bfloat16, plus 4 too, and never 0."""
    g = torch.Generator().manual_seed(seed)
    return (2.0 * torch.randint(-64, 64, (T, V), generator=g) + 1.0) / 16.0


@pytest.mark.parametrize("dtype,V,B", [(torch.float32, 3000, 3), (torch.bfloat16, 3000, 40),
                                       (torch.bfloat16, 126464, 40)])   # the last looks its terms up
def test_rows_of_the_same_probabilities(gpu, dtype, V, B):
    # the drafter's logits are the target's and a constant: equal probabilities, formed from other terms
    counts = [2] * B
    x = _sixteenths(2 * B, V, V + B)
    d = x + 4.0
    assert torch.equal(x.to(dtype).float(), x) and torch.equal(d.to(dtype).float(), d)
    ids, u, u_draw = _falls(counts, V, "below", x), _numbers(2 * B, 3), _numbers(B, 4)
    logits, draft = x.to(dtype).to(DEV), d.to(dtype).to(DEV)
    got = _verify_draft(gpu, counts, V, logits, draft, ids, None, u, u_draw)
    assert got[1].tolist() == [1] * B
    _check_draft(counts, logits, draft, ids, None, u, u_draw, got[:3])


@pytest.mark.parametrize("apart", [1e-2, 1e-4, 1e-6])
@pytest.mark.parametrize("B", [8, 40])
def test_drafters_near_the_target(gpu, B, apart):
    # the draw is from small differences: tokens in the middle of their share of the numbers
    V, counts = 1000, [2] * B
    x = _logits(2 * B, V, 11, torch.float32)
    g = torch.Generator().manual_seed(12)
    d = x + apart * torch.randn((2 * B, V), generator=g)
    ids, u = _falls(counts, V, "below", x), _numbers(2 * B, 5)
    u_draw, want = np.zeros(B, dtype=np.float32), []
    for b in range(B):
        p, q = od.softmax(x[2 * b].double().numpy(), 1.0), od.softmax(d[2 * b].double().numpy(), 1.0)
        w = np.maximum(p - q, 0.0)
        c = np.cumsum(w)
        v = int(np.argsort(w)[-1 - b % 8])
        u_draw[b] = (c[v] - 0.5 * w[v]) / c[-1]
        token, near = od.draw(w, u_draw[b])
        assert token == v and near > 9e-12 / c[-1]
        want.append(v)
    got = _verify_draft(gpu, counts, V, x.to(DEV), d.to(DEV), ids, None, u, u_draw)
    assert got[1].tolist() == [1] * B and got[0].tolist()[::2] == want
