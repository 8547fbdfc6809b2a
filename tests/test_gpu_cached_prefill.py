"""The generation's model call over the packed prompts, against the same call with
plain attention in float32."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def _plain(q, k, v, cu_q, cu_k, out, max_q):
    R = q.shape[1] // k.shape[1]
    at = cu_q.tolist()
    assert at == cu_k.tolist() and max_q == max(b - a for a, b in zip(at, at[1:]))
    for a, b in zip(at, at[1:]):
        for h in range(q.shape[1]):
            w = torch.softmax(q[a:b, h].float() @ k[a:b, h // R].float().t() * q.shape[2] ** -0.5, dim=-1)
            out[a:b, h] = (w @ v[a:b, h // R].float()).to(torch.bfloat16)


def test_prefill_matches_plain_attention(gpu, monkeypatch):
    from workloads import cached_generation as cg
    lens = (70, 1, 129)
    cfg = cg.Config(layers=2, hidden=256, heads=8, kv_heads=2, head_dim=64, vocab=1000)
    model = cg.Model(cfg, max(lens) + 32, seed=4)
    g = torch.Generator(device="cuda").manual_seed(9)
    tokens = torch.randint(0, cfg.vocab, (sum(lens),), generator=g, device="cuda")
    session, plain = cg.Session(model, lens, 32), cg.Session(model, lens, 32)
    got = session.prefill(tokens).float()
    with monkeypatch.context() as m:
        m.setattr(cg.fd, "fdllm_prompt_attention", _plain)
        want = plain.prefill(tokens).float()
    # the two differ by the attention's rounding of its weights and results to 8
    # bits, 2^-8 each of values of order one, through two layers and their
    # bfloat16 products
    assert (got - want).norm() / want.norm() < 4 * 2.0 ** -8
    # the first layer's entries do not depend on the attention
    assert torch.equal(session.caches[0], plain.caches[0])
    assert session.caches[1].any()
