"""Drafted tokens in a run: tree layout, rotation into the cache, tree attention,
verification and kept entries (or a chain's attention and verification) around a
small model, each step held against the float64 oracle on what the model gave it."""
import numpy as np
import pytest
import torch

from oracle import drafts as od

pytestmark = pytest.mark.gpu


def _session(seed, lens=(70, 1, 129, 62), gen=64, room=64):
    from workloads import cached_generation as cg
    cfg = cg.Config(layers=2, hidden=256, heads=8, kv_heads=2, head_dim=64, vocab=1000)
    model = cg.Model(cfg, max(lens) + gen + room, seed=seed)
    s = cg.Session(model, lens, gen, room)
    g = torch.Generator(device="cuda").manual_seed(seed + 1)
    prompt = torch.randint(0, cfg.vocab, (sum(lens),), generator=g, device="cuda")
    s.prefill(prompt)
    s.done = torch.tensor(lens, device="cuda") - 1
    return cfg, s, prompt[torch.tensor(lens, device="cuda").cumsum(0) - 1].to(torch.int32), g


def _plain(session, layer, q, kv_len, masks):
    """Tree attention over the cache's values in float32, a sequence at a time."""
    import paper_2606_02955_amd as fd
    c = session.model.cfg
    n = q.shape[0] // session.B
    out = torch.empty_like(q)
    bits = (masks[:, :1] >> torch.arange(n, device=q.device)) & 1       # (fewer than 64 nodes)
    for b in range(session.B):
        length = int(kv_len[b])
        at = torch.arange(length, device=q.device)
        slots = session.slots(torch.full_like(at, b), at)
        k, v = (torch.empty((length, c.kv_heads, c.head_dim), dtype=torch.bfloat16, device=q.device) for _ in range(2))
        fd.fdllm_cache_read(session.caches[layer], slots, k, v)
        rows = slice(b * n, (b + 1) * n)
        seen = torch.cat([torch.ones((n, length - n), device=q.device), bits[rows].float()], dim=1) > 0
        for h in range(c.heads):
            kh, vh = k[:, h * c.kv_heads // c.heads].float(), v[:, h * c.kv_heads // c.heads].float()
            x = (q[rows, h].float() @ kh.t() * c.head_dim ** -0.5).masked_fill(~seen, -float("inf"))
            out[rows, h] = (torch.softmax(x, dim=-1) @ vh).to(torch.bfloat16)
    return out


def test_tree_call_matches_plain_attention(gpu):
    cfg, s, roots, g = _session(3)
    ids, parents, _ = s.drafts(roots, 3, 4, 0.0)
    got, _, _ = s.tree_hidden(ids, parents)
    want, _, _ = s.tree_hidden(ids, parents, attention=_plain)
    # the two differ by the attention's rounding of its weights and results to 8
    # bits, 2^-8 each of values of order one, through two layers and their
    # bfloat16 products
    assert (got.float() - want.float()).norm() / want.float().norm() < 4 * 2.0 ** -8


def _near(seen, near):
    """A border nearer than both sides' errors: such a step says nothing."""
    assert near > 1e-11, seen


@pytest.mark.parametrize("temperature", [0.0, 0.7])
def test_tree_steps(gpu, temperature):
    cfg, s, roots, g = _session(5)
    stood = 0
    for step in range(6):
        r = {}
        before = s.done.clone()
        tokens, count = s.drafted_step(roots, 3, 3, temperature, g, record=r)
        n = r["ids"].shape[1]
        x, u = r["logits"].double().cpu().numpy().reshape(s.B, n, -1), r["u"].cpu().numpy().reshape(s.B, n)
        for b in range(s.B):
            path, want, _, near = od.verify_tree(x[b], r["ids"][b].cpu().numpy(), r["parents"].cpu().numpy(), temperature, u[b])
            _near((step, b), near)
            m = len(path)
            assert int(count[b]) == m and tokens[b].tolist() == want + [-1] * (n - m)
            assert r["path"].view(s.B, n)[b].tolist() == path + [-1] * (n - m)
            assert int(s.done[b]) == int(before[b]) + m
            stood += m - 1
            # the kept entries, in all layers; nothing else of the cache moved
            raw, old = s.stack.cpu().numpy(), r["stack"].cpu().numpy()
            want_raw = old.copy()
            for other in range(s.B):
                p = r["path"].view(s.B, n)[other].cpu().numpy()
                od.keep(want_raw, cfg.head_dim, s.table[other].cpu().numpy(), int(r["kv_len"][other]), n, p, int(count[other]))
            assert np.array_equal(raw, want_raw)
        roots = tokens[torch.arange(s.B, device="cuda"), count.long() - 1]
    assert stood > 0        # (drafts did stand, so that entries did move)


@pytest.mark.parametrize("temperature", [0.0, 0.7])
def test_chain_steps(gpu, temperature):
    cfg, s, roots, g = _session(6)
    for step in range(4):
        r = {}
        before = s.done.clone()
        tokens, count = s.drafted_step(roots, 1, 4, temperature, g, record=r)
        n = r["ids"].shape[1]
        x, d = (r[k].double().cpu().numpy().reshape(s.B, n, -1) for k in ("logits", "marginals"))
        u, ud = r["u"].cpu().numpy().reshape(s.B, n), r["u_draw"].cpu().numpy()
        for b in range(s.B):
            want, _, near = od.verify_draft(x[b], r["ids"][b].cpu().numpy(), d[b], temperature, u[b], ud[b])
            _near((step, b), near)
            assert int(count[b]) == len(want) and tokens[b].tolist() == want + [-1] * (n - len(want))
            assert int(s.done[b]) == int(before[b]) + len(want)
        roots = tokens[torch.arange(s.B, device="cuda"), count.long() - 1]


@pytest.mark.parametrize("width,depth,temperature", [(3, 4, 0.0), (2, 5, 0.8), (1, 4, 0.8)])
def test_generation_finishes_and_repeats(gpu, width, depth, temperature):
    runs = []
    for _ in range(2):
        cfg, s, roots, g = _session(7, gen=32)
        x, steps = s.generate_drafted(roots, width, depth, temperature, g)
        assert x.shape == (4, 32) and (x >= 0).all() and (x < cfg.vocab).all()
        assert 32 / (1 + depth) <= steps <= 32
        runs.append((x, steps))
    assert runs[0][1] == runs[1][1] and torch.equal(runs[0][0], runs[1][0])


def test_command(gpu, capsys):
    from workloads import cached_generation as cg
    tokens = cg.main(["--batch", "2", "--prompt", "96", "--blocks", "1", "--layers", "1", "--drafted", "2x3"])
    assert tokens.shape == (2, 32)
    assert "generated 64 tokens" in capsys.readouterr().out
