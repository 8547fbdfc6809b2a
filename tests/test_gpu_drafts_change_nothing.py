"""A greedy generation with trees of drafts gives the tokens of one without: behind
the same cache the model is called with one token after another, and every token
that a step with drafts gave is the highest logit's there too, up to roundings.

Bound.  The two calls differ by what test_gpu_drafted_generation.py allows for two
layers, 2^-6 of the hidden state; a logit is its product with a row of the head, so
it differs by 2^-6 times both norms at most, and so does the highest."""
import pytest
import torch

from test_gpu_drafted_generation import _session

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("width,depth,seed", [(3, 4, 11), (2, 1, 12), (8, 6, 13)])
def test_tokens_without_drafts(gpu, width, depth, seed):
    cfg, s, roots, g = _session(seed, room=2 * (1 + width * depth))
    _, one, _, _ = _session(seed, room=2 * (1 + width * depth))
    head, b, stood, sure = s.model.head, torch.arange(s.B, device="cuda"), 0, 0
    norm = head.float().norm(dim=1).max()
    alone = torch.full((1,), -1, dtype=torch.int32, device="cuda")
    for step in range(6):
        one.stack.copy_(s.stack)
        one.done = s.done.clone()
        r = {}
        tokens, count = s.drafted_step(roots, width, depth, 0.0, g, record=r)
        n = tokens.shape[1]
        m = int(count.max())
        previous = roots
        for i in range(m):
            hidden, _, _ = one.tree_hidden(previous.view(-1, 1), alone)
            logits = (hidden.float() @ head.float().t())
            bound = 2.0 ** -6 * hidden.float().norm(dim=1) * norm
            live = i < count
            # the logits of the drafted call at the node that the walk passed here
            node = r["path"].view(s.B, n)[:, i].clamp(min=0).long()
            with_drafts = r["logits"].float().view(s.B, n, -1)[b, node]
            # (those are rounded to bfloat16)
            off = (logits - with_drafts).abs() - 2.0 ** -9 * logits.abs() * 1.01
            assert (off.amax(dim=1) <= bound)[live].all()
            token = tokens[:, i].clamp(min=0).long()
            assert torch.equal(with_drafts[b, token][live], with_drafts.amax(dim=1)[live])
            best = logits.topk(2, dim=1)
            clear = live & (best.values[:, 0] - best.values[:, 1] > 2 * bound + 2.0 ** -8 * best.values[:, 0].abs())
            assert torch.equal(token[clear], best.indices[clear, 0])
            sure += int(clear.sum())
            previous = torch.where(live, tokens[:, i], previous)
            one.done = one.done + 1
        stood += int(count.sum()) - s.B
        roots = tokens[b, count.long() - 1]
    assert stood > 0 and sure > 0
