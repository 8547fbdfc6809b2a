"""The attention operators, the LM head and the selector together: a small
model's generation over 4-bit caches, against the same model with plain
attention over what the caches hold."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def _plain(session, layer, q, kv_len):
    """Attention over the cache's values in float32, a sequence at a time."""
    import paper_2606_02955_amd as fd
    c = session.model.cfg
    out = torch.empty_like(q)
    for b in range(session.B):
        n = int(kv_len[b])
        at = torch.arange(n, device=q.device)
        slots = session.slots(torch.full_like(at, b), at)
        k, v = (torch.empty((n, c.kv_heads, c.head_dim), dtype=torch.bfloat16, device=q.device) for _ in range(2))
        fd.fdllm_cache_read(session.caches[layer], slots, k, v)
        rows = slice(b * c.block, (b + 1) * c.block)
        for h in range(c.heads):
            kh, vh = k[:, h * c.kv_heads // c.heads].float(), v[:, h * c.kv_heads // c.heads].float()
            w = torch.softmax(q[rows, h].float() @ kh.t() * c.head_dim ** -0.5, dim=-1)
            out[rows, h] = (w @ vh).to(torch.bfloat16)
    return out


def _session(seed, layers=2, lens=(70, 1, 129), gen=64):
    from workloads import cached_generation as cg
    cfg = cg.Config(layers=layers, hidden=256, heads=8, kv_heads=2, head_dim=64, vocab=1000)
    model = cg.Model(cfg, max(lens) + gen, seed=seed)
    session = cg.Session(model, lens, gen)
    g = torch.Generator(device="cuda").manual_seed(seed + 1)
    session.prefill(torch.randint(0, cfg.vocab, (sum(lens),), generator=g, device="cuda"))
    return cfg, session


def test_block_call_matches_plain_attention(gpu):
    cfg, s = _session(3)
    tokens = torch.full((s.B, cfg.block), cfg.vocab, device="cuda")
    got = s.block_hidden(tokens).float()
    want = s.block_hidden(tokens, attention=_plain).float()
    # the two differ by the attention's rounding of its weights and results to 8
    # bits, 2^-8 each of values of order one, through two layers and their
    # bfloat16 products
    assert (got - want).norm() / want.norm() < 4 * 2.0 ** -8


def test_generation_finishes_and_repeats(gpu):
    runs = []
    for _ in range(2):
        cfg, s = _session(5)
        x, steps = s.generate()
        assert x.shape == (3, 64) and (x >= 0).all() and (x < cfg.vocab).all()
        assert 2 <= steps <= 64
        runs.append((x, steps))
    assert runs[0][1] == runs[1][1] and torch.equal(runs[0][0], runs[1][0])


def test_command(gpu, capsys):
    from workloads import cached_generation as cg
    tokens = cg.main(["--batch", "2", "--prompt", "96", "--blocks", "1", "--layers", "1"])
    assert tokens.shape == (2, 32)
    assert "generated 64 tokens" in capsys.readouterr().out
