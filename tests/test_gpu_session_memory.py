"""A generation session holds its layers' caches once, while it is made too."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def test_caches_are_allocated_once(gpu):
    from workloads import cached_generation as cg
    cfg = cg.Config(layers=4, hidden=128, heads=4, kv_heads=2, head_dim=64, vocab=100)
    model = cg.Model(cfg, 32, seed=0)
    lens = [1 << 16] * 4
    torch.cuda.synchronize()
    torch.cuda.reset_peak_memory_stats()
    before = torch.cuda.memory_allocated()
    s = cg.Session(model, lens, 0)
    torch.cuda.synchronize()
    peak = torch.cuda.max_memory_allocated() - before
    caches = s.stack.numel()
    assert caches == cfg.layers * 4 * 1024 * cfg.kv_heads * gpu.fdllm_cache_tile_bytes(cfg.head_dim)
    assert s.stack.shape[0] == cfg.layers and [c.data_ptr() for c in s.caches] == [c.data_ptr() for c in s.stack]
    assert peak < 1.1 * caches          # (the table and the places are less than 1 in 1000 of them)
    assert not s.stack.any()
