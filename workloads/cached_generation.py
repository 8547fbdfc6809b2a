"""A masked-diffusion generation with a model in the loop: the attention
operators, the LM head and the commit selector as a serving program calls them.

The model is a small transformer with random weights.  A batch of prompts of
different lengths goes through it once, packed: every layer norms and rotates
its heads, fills its 4-bit cache and attends over the prompts
(``fdllm_qk_norm_rope``, ``fdllm_prompt_attention``).  Then each sequence's
blocks are decoded one after another.  A step runs the model on the active
blocks alone: their keys and values replace those at their positions in the
cache and their queries attend over everything cached
(``fdllm_qk_norm_rope``, ``fdllm_cache_attention``), and the last hidden states
go into ``fdllm_lmhead_decode_step``, which reveals the tokens it commits to.

The same model also generates one token after another, with drafts: a step runs it
on a tree of drafted tokens behind what is cached (``fdllm_tree_layout``,
``fdllm_tree_attention``), ``fdllm_verify_tree`` says which of them stand and
``fdllm_cache_keep`` moves their cache entries into place; a chain of drafts needs
no tree and is held against the drafter's probabilities (``fdllm_verify_draft``).

    python -m workloads.cached_generation --batch 4 --blocks 2
    python -m workloads.cached_generation --batch 4 --blocks 2 --drafted 3x4
"""
from __future__ import annotations

import argparse
import dataclasses
import time

import torch

import paper_2606_02955_amd as fd


@dataclasses.dataclass
class Config:
    layers: int = 4
    hidden: int = 1024
    heads: int = 16
    kv_heads: int = 4
    head_dim: int = 64
    vocab: int = 32000
    block: int = 32          # tokens decoded at a time
    eps: float = 1e-6
    theta: float = 10000.0


def _rms(x, weight, eps):
    f = x.float()
    return (f * torch.rsqrt(f.square().mean(-1, keepdim=True) + eps) * weight).to(torch.bfloat16)


class Model:
    """Random weights of one architecture; embedding row `vocab` is the mask token's."""

    def __init__(self, cfg: Config, max_positions: int, seed: int = 0, device="cuda"):
        g = torch.Generator(device=device).manual_seed(seed)

        def normal(*shape, scale):
            return (torch.randn(shape, generator=g, device=device) * scale).to(torch.bfloat16)

        c, self.cfg, self.device = cfg, cfg, torch.device(device)
        d, wide = c.hidden, (c.heads + 2 * c.kv_heads) * c.head_dim
        self.embed = normal(c.vocab + 1, d, scale=1.0)
        self.qkv = [normal(wide, d, scale=d ** -0.5) for _ in range(c.layers)]
        self.proj = [normal(d, c.heads * c.head_dim, scale=(c.heads * c.head_dim) ** -0.5) for _ in range(c.layers)]
        self.up = [normal(4 * d, d, scale=d ** -0.5) for _ in range(c.layers)]
        self.down = [normal(d, 4 * d, scale=0.5 * d ** -0.5) for _ in range(c.layers)]
        self.norms = [torch.ones(d, device=device) for _ in range(2 * c.layers + 1)]
        self.q_norm = [1.0 + 0.1 * torch.randn(c.head_dim, generator=g, device=device) for _ in range(c.layers)]
        self.k_norm = [1.0 + 0.1 * torch.randn(c.head_dim, generator=g, device=device) for _ in range(c.layers)]
        self.head = normal(c.vocab, d, scale=4.0 * d ** -0.5)
        angle = torch.outer(torch.arange(max_positions, device=device).double(),
                            c.theta ** (-torch.arange(0, c.head_dim, 2, device=device).double() / c.head_dim))
        self.cos_sin = torch.cat([angle.cos(), angle.sin()], 1).float()

    def forward(self, tokens, attend):
        """Hidden states [T, d] of packed tokens; attend(layer, q, k, v) is a layer's attention."""
        c = self.cfg
        h = self.embed[tokens]
        for i in range(c.layers):
            qkv = _rms(h, self.norms[2 * i], c.eps) @ self.qkv[i].t()
            heads = qkv.view(len(tokens), -1, c.head_dim)      # the three side by side: no copy is made
            q, k, v = heads.split([c.heads, c.kv_heads, c.kv_heads], dim=1)
            h = h + attend(i, q, k, v).view(len(tokens), -1) @ self.proj[i].t()
            up = _rms(h, self.norms[2 * i + 1], c.eps) @ self.up[i].t()
            h = h + torch.nn.functional.gelu(up.float()).to(torch.bfloat16) @ self.down[i].t()
        return _rms(h, self.norms[-1], c.eps)


class Session:
    """A batch in generation: its pages, caches and places (room: for tokens beyond
    those to be generated, of trees of drafts)."""

    def __init__(self, model: Model, prompt_lens, gen_len: int, room: int = 0):
        c, dev = model.cfg, model.device
        self.model, self.lens, self.B = model, list(prompt_lens), len(prompt_lens)
        if gen_len % c.block:
            raise ValueError("gen_len must be a multiple of the block")
        self.gen_len = gen_len
        width = -(-(max(self.lens) + gen_len + room) // fd.CACHE_PAGE)
        # pages in a mixed order, as an allocator that has been running hands them out
        order = torch.randperm(self.B * width, generator=torch.Generator().manual_seed(1)).to(torch.int32)
        self.table = order.view(self.B, width).to(dev)
        # the layers' caches one behind the other
        self.stack = fd.new_cache(c.layers * self.B * width, c.kv_heads, c.head_dim, dev).unflatten(0, (c.layers, -1))
        self.caches = list(self.stack.unbind(0))
        self.done = torch.tensor(self.lens, device=dev)          # tokens before the active block
        self.block_at = torch.arange(c.block, device=dev)
        self.block_cu = (torch.arange(self.B + 1, device=dev) * c.block).to(torch.int32)
        self.workspace = None

    def slots(self, b, position):
        """Cache slots of positions of sequences b (both [T])."""
        return (self.table[b, position // fd.CACHE_PAGE] * fd.CACHE_PAGE + position % fd.CACHE_PAGE).to(torch.int32)

    def _rope(self, layer, q, k, v, positions, slots, keys):
        m = self.model
        q_out = torch.empty(q.shape, dtype=torch.bfloat16, device=q.device)
        k_out = torch.empty(k.shape, dtype=torch.bfloat16, device=q.device) if keys else None
        fd.fdllm_qk_norm_rope(q, k, v, positions, m.cos_sin, q_out, k_out=k_out, q_weight=m.q_norm[layer],
                              k_weight=m.k_norm[layer], eps=m.cfg.eps, cache=self.caches[layer], slots=slots)
        return q_out, k_out

    def prefill(self, tokens):
        """The model call over the packed prompts: fills the caches."""
        dev = self.model.device
        lens = torch.tensor(self.lens, device=dev)
        cu = torch.zeros(self.B + 1, dtype=torch.int32, device=dev)
        cu[1:] = lens.cumsum(0)
        b = torch.repeat_interleave(torch.arange(self.B, device=dev), lens)
        position = torch.arange(len(tokens), device=dev) - cu[b]
        slots, pos32 = self.slots(b, position), position.to(torch.int32)

        def attend(layer, q, k, v):
            q_out, k_out = self._rope(layer, q, k, v, pos32, slots, keys=True)
            out = torch.empty_like(q_out)
            fd.fdllm_prompt_attention(q_out, k_out, v, cu, cu, out, max(self.lens))
            return out

        return self.model.forward(tokens, attend)

    def block_hidden(self, tokens, attention=None):
        """The model call on the active blocks, tokens [B, block]: hidden states [B, block, d]."""
        c, dev = self.model.cfg, self.model.device
        position = (self.done.view(-1, 1) + self.block_at).view(-1)
        b = torch.arange(self.B, device=dev).repeat_interleave(c.block)
        slots, pos32 = self.slots(b, position), position.to(torch.int32)
        kv_len = (self.done + c.block).to(torch.int32)

        def attend(layer, q, k, v):
            q_out, _ = self._rope(layer, q, k, v, pos32, slots, keys=False)
            if attention is not None:
                return attention(self, layer, q_out, kv_len)
            out = torch.empty_like(q_out)
            self.workspace = fd.fdllm_cache_attention(q_out, self.caches[layer], self.table, kv_len, self.block_cu, out,
                                                      c.block, workspace=self.workspace)
            return out

        return self.model.forward(tokens.reshape(-1), attend).view(self.B, c.block, -1)

    def generate(self, selector="profile", param=1.0):
        """Decodes gen_len tokens a sequence; returns them and the steps taken."""
        c, dev = self.model.cfg, self.model.device
        B, n = self.B, c.block
        out = torch.empty((B, self.gen_len), dtype=torch.int32, device=dev)
        start, end = torch.zeros(B, dtype=torch.int32, device=dev), torch.full((B,), n, dtype=torch.int32, device=dev)
        steps, lm_ws = 0, None
        for block in range(self.gen_len // n):
            x = torch.full((B, n), -1, dtype=torch.int32, device=dev)
            mask = torch.ones((B, n), dtype=torch.uint8, device=dev)
            while True:
                tokens = torch.where(mask.bool(), c.vocab, x.long())
                hidden = self.block_hidden(tokens)
                lm_ws = fd.fdllm_lmhead_decode_step(hidden, self.model.head, mask, start, end, x, selector, param,
                                                    workspace=lm_ws)
                steps += 1
                if not bool(mask.any()):
                    break
            # the block's final tokens into the cache, before the next one reads it
            self.block_hidden(x.long())
            out[:, block * n:(block + 1) * n] = x
            self.done += n
        return out, steps

    # ---- with drafts ----
    def _need_room(self, tokens: int, positions: int):
        """Refuses sequences of more tokens than they have pages for, or at positions
        beyond the model's: their keys would be nowhere and their results anything."""
        pages, last = self.table.shape[1] * fd.CACHE_PAGE, len(self.model.cos_sin)
        if tokens > pages or positions > last:
            raise ValueError(f"no room for the drafts: {tokens} tokens and {positions} positions are needed, a sequence's "
                             f"pages hold {pages} (Session's room) and the model has {last}")

    def drafts(self, roots, width: int, depth: int, temperature: float, generator=None):
        """A drafter that only knows the token before: `width` branches of `depth`
        tokens behind each root (their likeliest, or one drawn for a chain).
        Returns ids [B, nodes], parents [nodes] and the drafter's logits of every
        node of a chain."""
        m, dev = self.model, self.model.device
        n = 1 + width * depth
        ids = torch.empty((self.B, n), dtype=torch.int32, device=dev)
        parents = torch.tensor([-1] + [0 if i < width else i + 1 - width for i in range(n - 1)], dtype=torch.int32)
        ids[:, 0] = roots
        logits = torch.zeros((self.B, n, m.cfg.vocab), dtype=torch.bfloat16, device=dev) if width == 1 else None
        for level in range(depth):
            before = ids[:, :1] if level == 0 else ids[:, 1 + (level - 1) * width:1 + level * width]
            x = _rms(m.embed[before.long()], m.norms[-1], m.cfg.eps) @ m.head.t()          # [B, nodes before, vocab]
            if width == 1:
                logits[:, level] = x[:, 0]
                if temperature > 0:
                    p = torch.softmax(x[:, 0].float() / temperature, dim=-1)
                    ids[:, 1 + level] = torch.multinomial(p, 1, generator=generator).view(-1).to(torch.int32)
                    continue
            best = x.topk(width if level == 0 else 1, dim=-1).indices.reshape(self.B, width)
            ids[:, 1 + level * width:1 + (level + 1) * width] = best.to(torch.int32)
        return ids, parents.to(dev), logits

    def tree_hidden(self, ids, parents, attention=None):
        """The model call on trees behind what is cached, ids [B, n], parents [n] of
        all of them: hidden states [B * n, d]; the nodes' keys and values go into
        the cache behind the others, in the nodes' order."""
        dev, n = self.model.device, ids.shape[1]
        level = []      # of each node
        for i, p in enumerate(parents.tolist()):
            level.append(level[p] + 1 if 0 <= p < i else 0)
        done = int(self.done.max())
        self._need_room(done + n, done + max(level) + 1)
        T = self.B * n
        cu = (torch.arange(self.B + 1, device=dev) * n).to(torch.int32)
        kv_len = (self.done + n).to(torch.int32)
        masks = torch.empty((T, -(-n // 64)), dtype=torch.int64, device=dev)
        position, slots = (torch.empty(T, dtype=torch.int32, device=dev) for _ in range(2))
        fd.fdllm_tree_layout(parents.repeat(self.B), kv_len, cu, n, masks, positions=position, page_table=self.table,
                             slots=slots)

        def attend(layer, q, k, v):
            q_out, _ = self._rope(layer, q, k, v, position, slots, keys=False)
            if attention is not None:
                return attention(self, layer, q_out, kv_len, masks)
            out = torch.empty_like(q_out)
            fd.fdllm_tree_attention(q_out, self.caches[layer], self.table, kv_len, cu, masks, out, n)
            return out

        return self.model.forward(ids.reshape(-1).long(), attend), kv_len, cu

    def drafted_step(self, roots, width: int, depth: int, temperature: float, generator=None, record=None):
        """One call of the model on drafts behind `roots` [B]: tokens [B, nodes] that
        follow, -1 behind the last, and how many.  record: a dict that gets what the
        step worked on."""
        dev, B = self.model.device, self.B
        ids, parents, marginals = self.drafts(roots, width, depth, temperature, generator)
        n = ids.shape[1]
        T = B * n
        hidden, kv_len, cu = self.tree_hidden(ids, parents)
        logits = hidden @ self.model.head.t()
        tokens, path = (torch.empty(T, dtype=torch.int32, device=dev) for _ in range(2))
        count = torch.empty(B, dtype=torch.int32, device=dev)
        warmth = torch.full((B,), temperature, device=dev)
        u, u_draw = (torch.rand(k, generator=generator, device=dev) for k in (T, B))
        done = torch.empty(B, dtype=torch.int32, device=dev)
        if width == 1:      # what stands of a chain lies in place
            fd.fdllm_verify_draft(logits, ids.view(-1), cu, n, u, u_draw, tokens, count, draft=marginals.view(T, -1),
                                  temperature=warmth)
            done = kv_len - n + count
        else:
            fd.fdllm_verify_tree(logits, ids.view(-1), parents.repeat(B), cu, n, u, path, tokens, count, temperature=warmth)
            if record is not None:
                record["stack"] = self.stack.clone()
            fd.fdllm_cache_keep(self.stack, self.table, kv_len, cu, path, count, n, done)
        if record is not None:
            record.update(ids=ids, parents=parents, marginals=marginals, logits=logits, u=u, u_draw=u_draw, path=path,
                          kv_len=kv_len)
        self.done = done.long()
        return tokens.view(B, n), count

    def generate_drafted(self, last, width: int = 3, depth: int = 4, temperature: float = 0.0, generator=None):
        """gen_len tokens a sequence behind its prompt, whose last tokens are `last`
        [B]; returns them and the steps taken.  Sequences need pages for a step's nodes
        behind their last token but one, and where there are several, of which one that has
        its tokens goes on beside the others, behind depth + 1 more."""
        dev = self.model.device
        n = 1 + width * depth
        most = max(self.lens) + self.gen_len - 2 + (depth + 1 if self.B > 1 else 0)    # cached before a step
        self._need_room(most + n, most + depth + 1)
        out = torch.full((self.B, self.gen_len + n), -1, dtype=torch.int32, device=dev)
        at, steps = torch.zeros(self.B, dtype=torch.long, device=dev), 0
        start = torch.tensor(self.lens, device=dev) - 1     # the last prompt token is the first root
        self.done, roots = start.clone(), last.to(torch.int32)
        b = torch.arange(self.B, device=dev)
        while int(at.min()) < self.gen_len:
            tokens, count = self.drafted_step(roots, width, depth, temperature, generator)
            where = (at.view(-1, 1) + torch.arange(n, device=dev)).clamp(max=out.shape[1] - 1)
            # a sequence that has its tokens stays where it is
            live = at < self.gen_len
            keep = live.view(-1, 1) & (torch.arange(n, device=dev) < count.view(-1, 1))
            out.scatter_(1, where, torch.where(keep, tokens, out.gather(1, where)))
            roots = torch.where(live, tokens[b, count.long() - 1], roots)
            at += torch.where(live, count.long(), torch.zeros_like(at))
            self.done = start + at
            steps += 1
        return out[:, :self.gen_len], steps


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.split("\n\n")[0])
    ap.add_argument("--batch", type=int, default=4)
    ap.add_argument("--prompt", type=int, default=512, help="the longest prompt's tokens")
    ap.add_argument("--blocks", type=int, default=2, help="blocks of 32 tokens to generate")
    ap.add_argument("--layers", type=int, default=4)
    ap.add_argument("--drafted", metavar="WxD", help="generate with drafts, W branches of D tokens each (1xD: a chain)")
    ap.add_argument("--temperature", type=float, default=0.0, help="of a generation with drafts")
    ap.add_argument("--seed", type=int, default=0)
    a = ap.parse_args(argv)
    width, depth = 0, 0
    if a.drafted:
        width, _, depth = (int(x) if x.isdigit() else 0 for x in a.drafted.partition("x"))
        if not (width and depth and 1 + width * depth <= fd.MAX_TREE):
            ap.error(f"--drafted {a.drafted}: WxD, with 1 + W * D at most {fd.MAX_TREE}")
    cfg = Config(layers=a.layers)
    lens = [max(1, a.prompt * (a.batch - b) // a.batch) for b in range(a.batch)]
    gen_len = a.blocks * cfg.block
    room = 2 * (1 + width * depth) if a.drafted else 0
    model = Model(cfg, max(lens) + gen_len + room, seed=a.seed)
    session = Session(model, lens, gen_len, room)
    g = torch.Generator(device="cuda").manual_seed(a.seed + 1)
    prompt = torch.randint(0, cfg.vocab, (sum(lens),), generator=g, device="cuda")
    torch.cuda.synchronize()
    t = time.perf_counter()
    session.prefill(prompt)
    torch.cuda.synchronize()
    print(f"prompts: {sum(lens)} tokens of {a.batch} sequences in {(time.perf_counter() - t) * 1e3:.1f} ms")
    t = time.perf_counter()
    if a.drafted:
        last = prompt[torch.tensor(lens, device="cuda").cumsum(0) - 1]
        tokens, steps = session.generate_drafted(last, width, depth, a.temperature, g)
    else:
        tokens, steps = session.generate()
    torch.cuda.synchronize()
    dt = time.perf_counter() - t
    print(f"generated {tokens.numel()} tokens in {steps} steps, {dt * 1e3:.1f} ms, {dt / steps * 1e3:.2f} ms a step")
    held = sum(x.numel() for x in session.caches)
    wide = sum(4 * x.shape[0] * x.shape[1] * fd.CACHE_PAGE * cfg.head_dim for x in session.caches)
    print(f"caches: {held / 2 ** 20:.1f} MiB in 4 bits ({wide / 2 ** 20:.1f} MiB in bfloat16)")
    return tokens


if __name__ == "__main__":
    main()
