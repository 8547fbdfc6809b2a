"""The calls for drafted tokens captured into a HIP graph and replayed with eager
work between, on a stream of their own, and two at once with workspaces of their
own: every result is the eager call's bit for bit."""
import numpy as np
import pytest
import torch

from oracle import attention as oa
from test_gpu_drafts import DEV, _cu, _f32, _i32, _logits, _masks, _numbers, _tree, _words
from oracle import drafts as od

pytestmark = pytest.mark.gpu


class Step:
    """A step's calls on fixed inputs: trees over a cache, their logits, a chain's."""

    def __init__(self, fd, counts, contexts, V, seed, D=64, H=4, Hk=2, layers=2):
        self.fd, self.counts, self.max_q = fd, counts, max(counts)
        B, T = len(counts), sum(counts)
        lens = [n + c for n, c in zip(counts, contexts)]
        pages = sum(-(-n // 64) for n in lens)
        width = max(-(-n // 64) for n in lens)
        table, at = np.zeros((B, width)), 0
        for b, n in enumerate(lens):
            table[b, :-(-n // 64)] = np.arange(at, at - (-n // 64))
            at += -(-n // 64)
        g = torch.Generator().manual_seed(seed)
        raw = torch.randint(0, 256, (layers, pages, Hk, oa.tile_bytes(D)), generator=g, dtype=torch.uint8)
        raw[..., 64 * D:] = torch.randint(124, 128, raw[..., 64 * D:].shape, generator=g, dtype=torch.uint8)
        self.stack0 = raw.to(DEV)
        self.stack = self.stack0.clone()
        self.table, self.kv, self.cu = _i32(table), _i32(lens), _i32(_cu(counts))
        self.parents = _i32(np.concatenate([_tree(n, seed + b) for b, n in enumerate(counts)]))
        self.q = torch.randn((T, H, D), generator=g).to(torch.bfloat16).to(DEV)
        self.logits = _logits(T, V, seed, torch.bfloat16).to(DEV)
        self.draft = (self.logits.float() + 0.5 * torch.randn((T, V), generator=g).to(DEV)).to(torch.bfloat16)
        self.ids = self.logits.float().argmax(1).to(torch.int32).roll(1)
        self.u, self.ud = _f32(_numbers(T, seed)), _f32(_numbers(B, seed + 1))
        self.temperature = _f32([0.8 if b % 3 else 0.0 for b in range(B)])
        i32 = lambda n: torch.empty(n, dtype=torch.int32, device=DEV)
        self.outs = dict(masks=torch.empty((T, -(-self.max_q // 64)), dtype=torch.int64, device=DEV), pos=i32(T), slots=i32(T),
                         out=torch.empty_like(self.q), lse=torch.empty((T, H), device=DEV), path=i32(T), tokens=i32(T), n=i32(B),
                         logp=torch.empty(T, device=DEV), kv_out=i32(B), chain=i32(T), n_chain=i32(B),
                         chain_logp=torch.empty(T, device=DEV))
        need = lambda n: torch.empty(max(n, 16), dtype=torch.uint8, device=DEV)
        self.ws = [need(fd.fdllm_cache_attention_workspace_size(B, H, Hk, D, self.max_q, width)),
                   need(fd.fdllm_verify_tree_workspace_size(T, B, V)), need(fd.fdllm_verify_draft_workspace_size(T, B, V, True))]

    def run(self):
        fd, o = self.fd, self.outs
        self.stack.copy_(self.stack0)
        fd.fdllm_tree_layout(self.parents, self.kv, self.cu, self.max_q, o["masks"], positions=o["pos"], page_table=self.table,
                             slots=o["slots"])
        fd.fdllm_tree_attention(self.q, self.stack[1], self.table, self.kv, self.cu, o["masks"], o["out"], self.max_q,
                                lse=o["lse"], workspace=self.ws[0])
        fd.fdllm_verify_tree(self.logits, self.ids, self.parents, self.cu, self.max_q, self.u, o["path"], o["tokens"], o["n"],
                             temperature=self.temperature, logp=o["logp"], workspace=self.ws[1])
        fd.fdllm_cache_keep(self.stack, self.table, self.kv, self.cu, o["path"], o["n"], self.max_q, kv_out=o["kv_out"])
        fd.fdllm_verify_draft(self.logits, self.ids, self.cu, self.max_q, self.u, self.ud, o["chain"], o["n_chain"],
                              draft=self.draft, temperature=self.temperature, logp=o["chain_logp"], workspace=self.ws[2])

    def results(self):
        return {k: v.clone() for k, v in dict(self.outs, stack=self.stack).items()}

    def spoil(self, value):
        for t in self.outs.values():
            t.fill_(value)
        for w in self.ws:
            w.fill_(value)


def _same(a, b):
    for k in a:
        assert torch.equal(a[k].view(torch.uint8) if a[k].dim() else a[k], b[k].view(torch.uint8) if b[k].dim() else b[k]), k


STEPS = [([9, 1, 30, 64], [100, 0, 700, 5], 5000), ([16], [500], 126464), ([3, 70], [9000, 40], 3001),
         ([5] * 40, [64 * (b % 4) for b in range(40)], 20000)]


@pytest.mark.parametrize("counts,contexts,V", STEPS)
def test_graph_replays(gpu, counts, contexts, V):
    s = Step(gpu, counts, contexts, V, 3)
    s.run()
    torch.cuda.synchronize()
    want = s.results()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        s.run()
    for r in range(3):
        s.spoil(7 + r)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        _same(want, s.results())
    # other inputs in the same places
    s.u.copy_(1.0 - s.u - 2.0 ** -24)
    graph.replay()
    torch.cuda.synchronize()
    got = s.results()
    s.run()
    torch.cuda.synchronize()
    _same(got, s.results())


def test_another_stream_and_two_at_once(gpu):
    a, b = Step(gpu, [40, 7], [3000, 10], 30000, 1), Step(gpu, [12] * 5, [77] * 5, 30000, 2)
    for s in (a, b):
        s.run()
    torch.cuda.synchronize()
    want = [s.results() for s in (a, b)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    for s in (a, b):
        s.spoil(5)
    torch.cuda.synchronize()
    for _ in range(3):
        for s, stream in zip((a, b), streams):
            with torch.cuda.stream(stream):
                s.run()
    torch.cuda.synchronize()
    for s, w in zip((a, b), want):
        _same(w, s.results())


def test_two_graphs_share_a_workspace(gpu):
    # replayed one after another: what one leaves in it means nothing to the other
    a, b = Step(gpu, [40, 7], [3000, 10], 30000, 1), Step(gpu, [12] * 5, [77] * 5, 3000, 2)
    b.ws = [x if x.numel() >= y.numel() else y for x, y in zip(a.ws, b.ws)]
    a.ws = b.ws
    for s in (a, b):
        s.run()
    torch.cuda.synchronize()
    want, graphs = [s.results() for s in (a, b)], []
    for s in (a, b):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            s.run()
        graphs.append(g)
    for r in range(3):
        for s, g in zip((a, b), graphs):
            s.outs["tokens"].fill_(r)
            g.replay()
    torch.cuda.synchronize()
    for s, w in zip((a, b), want):
        _same(w, s.results())
