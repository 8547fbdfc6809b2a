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

    python -m workloads.cached_generation --batch 4 --blocks 2
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
    """A batch in generation: its pages, caches and places."""

    def __init__(self, model: Model, prompt_lens, gen_len: int):
        c, dev = model.cfg, model.device
        self.model, self.lens, self.B = model, list(prompt_lens), len(prompt_lens)
        if gen_len % c.block:
            raise ValueError("gen_len must be a multiple of the block")
        self.gen_len = gen_len
        width = -(-(max(self.lens) + gen_len) // fd.CACHE_PAGE)
        # pages in a mixed order, as an allocator that has been running hands them out
        order = torch.randperm(self.B * width, generator=torch.Generator().manual_seed(1)).to(torch.int32)
        self.table = order.view(self.B, width).to(dev)
        self.caches = [fd.new_cache(self.B * width, c.kv_heads, c.head_dim, dev) for _ in range(c.layers)]
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


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.split("\n\n")[0])
    ap.add_argument("--batch", type=int, default=4)
    ap.add_argument("--prompt", type=int, default=512, help="the longest prompt's tokens")
    ap.add_argument("--blocks", type=int, default=2, help="blocks of 32 tokens to generate")
    ap.add_argument("--layers", type=int, default=4)
    ap.add_argument("--seed", type=int, default=0)
    a = ap.parse_args(argv)
    cfg = Config(layers=a.layers)
    lens = [max(1, a.prompt * (a.batch - b) // a.batch) for b in range(a.batch)]
    gen_len = a.blocks * cfg.block
    model = Model(cfg, max(lens) + gen_len, seed=a.seed)
    session = Session(model, lens, gen_len)
    g = torch.Generator(device="cuda").manual_seed(a.seed + 1)
    prompt = torch.randint(0, cfg.vocab, (sum(lens),), generator=g, device="cuda")
    torch.cuda.synchronize()
    t = time.perf_counter()
    session.prefill(prompt)
    torch.cuda.synchronize()
    print(f"prompts: {sum(lens)} tokens of {a.batch} sequences in {(time.perf_counter() - t) * 1e3:.1f} ms")
    t = time.perf_counter()
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
