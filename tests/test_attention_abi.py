"""Argument checks of the attention entry points, on the host: each bad call gets
its status and enqueues nothing."""
import ctypes
import os
import re

import pytest
import torch

import paper_2606_02955_amd as fd
from oracle import attention as oa

HEADER = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "fdllm.h")


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(fd.LIB_PATH) or not os.path.exists(fd.BINDING_PATH):
        from paper_2606_02955_amd import build
        build.build()
    return fd.load()


P = ctypes.c_void_p(0x1000)      # never dereferenced: checks fail first
ODD = ctypes.c_void_p(0x1004)


def test_constants_agree_with_header():
    text = open(HEADER).read()
    assert int(re.search(r"#define FDLLM_CACHE_PAGE (\d+)", text).group(1)) == fd.CACHE_PAGE == oa.PAGE
    assert f"FDLLM_OUT_BF16 = {fd.OUT_BF16}, FDLLM_OUT_E5M2 = {fd.OUT_E5M2}" in text


@pytest.mark.parametrize("D", [32, 64, 96, 128, 160, 256])
def test_tile_bytes(lib, D):
    assert fd.fdllm_cache_tile_bytes(D) == oa.tile_bytes(D)


@pytest.mark.parametrize("D", [0, 16, 48, 288, -32])
def test_tile_bytes_refuses(lib, D):
    with pytest.raises(fd.FdllmError) as e:
        fd.fdllm_cache_tile_bytes(D)
    assert e.value.status == fd.ERR_SIZE
    assert lib.fdllm_cache_tile_bytes(64, None) == fd.ERR_INVALID_ARG


def _rope(lib, **kw):
    a = dict(q=P, qs=256, k=P, ks=128, v=P, vs=128, dt=0, T=4, H=4, Hk=2, D=64, qw=P, kw=P, eps=1e-6, pos=P, cs=P, n_pos=8,
             rot=64, inter=0, qo=P, ko=P, cache=P, pages=2, slots=P)
    a.update(kw)
    return lib.fdllm_qk_norm_rope(*a.values(), None)


@pytest.mark.parametrize("kw,status", [
    (dict(dt=2), fd.ERR_UNSUPPORTED_DTYPE), (dict(dt=-1), fd.ERR_UNSUPPORTED_DTYPE),
    (dict(T=-1), fd.ERR_INVALID_ARG), (dict(H=0), fd.ERR_INVALID_ARG), (dict(Hk=0), fd.ERR_INVALID_ARG),
    (dict(pages=-1), fd.ERR_INVALID_ARG), (dict(n_pos=-1), fd.ERR_INVALID_ARG),
    (dict(D=48), fd.ERR_SIZE), (dict(D=288), fd.ERR_SIZE), (dict(D=0), fd.ERR_SIZE),
    (dict(rot=72), fd.ERR_SIZE), (dict(rot=24), fd.ERR_SIZE), (dict(rot=-16), fd.ERR_SIZE),
    (dict(pages=1 << 26), fd.ERR_SIZE), (dict(H=1 << 15, qs=1 << 21), fd.ERR_SIZE), (dict(T=1 << 28), fd.ERR_SIZE),
    (dict(eps=-1.0), fd.ERR_INVALID_ARG), (dict(eps=float("nan")), fd.ERR_INVALID_ARG),
    (dict(q=None), fd.ERR_INVALID_ARG), (dict(k=None), fd.ERR_INVALID_ARG), (dict(qo=None), fd.ERR_INVALID_ARG),
    (dict(pos=None), fd.ERR_INVALID_ARG), (dict(cs=None), fd.ERR_INVALID_ARG),
    (dict(ko=None, cache=None), fd.ERR_INVALID_ARG), (dict(v=None), fd.ERR_INVALID_ARG), (dict(slots=None), fd.ERR_INVALID_ARG),
    (dict(qs=255), fd.ERR_INVALID_ARG), (dict(qs=260), fd.ERR_INVALID_ARG), (dict(ks=120), fd.ERR_INVALID_ARG),
    (dict(vs=132), fd.ERR_INVALID_ARG), (dict(dt=1, qs=258), fd.ERR_INVALID_ARG),
    (dict(q=ODD), fd.ERR_INVALID_ARG), (dict(ko=ODD), fd.ERR_INVALID_ARG), (dict(cache=ODD), fd.ERR_INVALID_ARG),
    (dict(qw=ODD), fd.ERR_INVALID_ARG), (dict(T=0), fd.OK)])
def test_rope_refuses(lib, kw, status):
    assert _rope(lib, **kw) == status


@pytest.mark.parametrize("kw,status", [
    (dict(out=2), fd.ERR_UNSUPPORTED_DTYPE), (dict(T=-1), fd.ERR_INVALID_ARG), (dict(Hk=0), fd.ERR_INVALID_ARG),
    (dict(D=40), fd.ERR_SIZE), (dict(cache=None), fd.ERR_INVALID_ARG), (dict(pages=0), fd.ERR_INVALID_ARG),
    (dict(slots=None), fd.ERR_INVALID_ARG), (dict(k=None, v=None), fd.ERR_INVALID_ARG), (dict(k=ODD), fd.ERR_INVALID_ARG),
    (dict(T=0), fd.OK)])
def test_cache_read_refuses(lib, kw, status):
    a = dict(cache=P, pages=2, Hk=2, D=64, slots=P, T=3, out=0, k=P, v=P)
    a.update(kw)
    assert lib.fdllm_cache_read(*a.values(), None) == status


@pytest.mark.parametrize("kw,status", [
    (dict(T=-1), fd.ERR_INVALID_ARG), (dict(B=-1), fd.ERR_INVALID_ARG), (dict(max_q=-1), fd.ERR_INVALID_ARG),
    (dict(blk=-1), fd.ERR_INVALID_ARG), (dict(scale=0.0), fd.ERR_INVALID_ARG), (dict(scale=float("nan")), fd.ERR_INVALID_ARG),
    (dict(scale=float("inf")), fd.ERR_INVALID_ARG), (dict(width=-1), fd.ERR_INVALID_ARG),
    (dict(D=32), fd.ERR_SIZE), (dict(D=256), fd.ERR_SIZE), (dict(H=5), fd.ERR_SIZE), (dict(B=70000), fd.ERR_SIZE),
    (dict(pages=1 << 26), fd.ERR_SIZE), (dict(width=1 << 26), fd.ERR_SIZE), (dict(B=60000, width=1 << 20), fd.ERR_SIZE),
    (dict(q=None), fd.ERR_INVALID_ARG), (dict(cu=None), fd.ERR_INVALID_ARG), (dict(kv=None), fd.ERR_INVALID_ARG),
    (dict(out=None), fd.ERR_INVALID_ARG), (dict(table=None), fd.ERR_INVALID_ARG), (dict(cache=None), fd.ERR_INVALID_ARG),
    (dict(pages=0), fd.ERR_INVALID_ARG), (dict(qs=100), fd.ERR_INVALID_ARG), (dict(qs=260), fd.ERR_INVALID_ARG),
    (dict(q=ODD), fd.ERR_INVALID_ARG), (dict(out=ODD), fd.ERR_INVALID_ARG), (dict(ws=None), fd.ERR_WORKSPACE),
    (dict(wsb=8), fd.ERR_WORKSPACE), (dict(T=0), fd.OK), (dict(B=0), fd.OK), (dict(max_q=0), fd.OK)])
def test_cache_attention_refuses(lib, kw, status):
    a = dict(q=P, qs=256, T=6, cu=P, B=2, max_q=4, H=4, Hk=2, D=64, cache=P, pages=3, table=P, width=2, kv=P, qstart=None,
             scale=0.1, blk=0, out=P, lse=None, ws=P, wsb=1 << 30)
    a.update(kw)
    assert lib.fdllm_cache_attention(*a.values(), None) == status


@pytest.mark.parametrize("kw,status", [
    (dict(T=-1), fd.ERR_INVALID_ARG), (dict(Tk=-1), fd.ERR_INVALID_ARG), (dict(blk=-2), fd.ERR_INVALID_ARG),
    (dict(scale=-1.0), fd.ERR_INVALID_ARG), (dict(D=32), fd.ERR_SIZE), (dict(H=5), fd.ERR_SIZE),
    (dict(q=None), fd.ERR_INVALID_ARG), (dict(k=None), fd.ERR_INVALID_ARG), (dict(v=None), fd.ERR_INVALID_ARG),
    (dict(cuq=None), fd.ERR_INVALID_ARG), (dict(cuk=None), fd.ERR_INVALID_ARG), (dict(out=None), fd.ERR_INVALID_ARG),
    (dict(qs=252), fd.ERR_INVALID_ARG), (dict(ks=130), fd.ERR_INVALID_ARG), (dict(vs=64), fd.ERR_INVALID_ARG),
    (dict(v=ODD), fd.ERR_INVALID_ARG), (dict(Tk=1 << 20, ws=None), fd.ERR_WORKSPACE), (dict(Tk=1 << 20, wsb=64), fd.ERR_WORKSPACE),
    (dict(T=0), fd.OK), (dict(B=0), fd.OK), (dict(max_q=0), fd.OK)])
def test_prompt_attention_refuses(lib, kw, status):
    a = dict(q=P, qs=256, k=P, ks=128, v=P, vs=128, T=6, Tk=9, cuq=P, cuk=P, B=2, max_q=4, H=4, Hk=2, D=64, scale=0.1, blk=0,
             out=P, lse=None, ws=P, wsb=1 << 40)
    a.update(kw)
    assert lib.fdllm_prompt_attention(*a.values(), None) == status


def test_workspace_sizes(lib):
    assert fd.fdllm_cache_attention_workspace_size(2, 8, 2, 128, 1, 100) > 0
    assert fd.fdllm_prompt_attention_workspace_size(64, 1 << 16, 1 << 16, 32, 8, 128, 1024) == 0     # row tiles fill the chip
    assert fd.fdllm_prompt_attention_workspace_size(1, 1, 1 << 16, 4, 1, 128, 1) > 0
    # 64 groups of rows of 8 heads are an item a workgroup only where the sequence has all max_q queries
    assert fd.fdllm_cache_attention_workspace_size(1, 32, 8, 128, 2048, 10) > 0
    assert fd.fdllm_cache_attention_workspace_size(1, 32, 8, 128, 2048, 1) == 0                       # no item has two pages
    n = ctypes.c_size_t(0)
    assert lib.fdllm_cache_attention_workspace_size(2, 8, 2, 128, 1, 100, None) == fd.ERR_INVALID_ARG
    assert lib.fdllm_cache_attention_workspace_size(2, 8, 3, 128, 1, 100, ctypes.byref(n)) == fd.ERR_SIZE
    assert lib.fdllm_prompt_attention_workspace_size(-1, 8, 8, 2, 2, 128, 1, 0, ctypes.byref(n)) == fd.ERR_INVALID_ARG
    assert lib.fdllm_prompt_attention_workspace_size(1, 8, 8, 2, 2, 80, 1, 0, ctypes.byref(n)) == fd.ERR_SIZE


def test_binding_refuses(lib):
    q = torch.zeros(4, 4, 64, dtype=torch.bfloat16)
    cu = torch.tensor([0, 4], dtype=torch.int32)
    with pytest.raises(ValueError):
        fd.fdllm_prompt_attention(q, q, q, cu, cu, q, 4)          # not on the GPU
    with pytest.raises(ValueError):
        fd.fdllm_prompt_attention(q, q, q[:, :, :32], cu, cu, q, 4)
    with pytest.raises(ValueError):
        fd.fdllm_cache_read(torch.zeros(2, 2, 100, dtype=torch.uint8), None)


@pytest.mark.parametrize("call", ["rope", "read", "cache", "prompt"])
def test_binding_refuses_what_is_no_tensor_or_has_no_heads(lib, call):
    q, cu = torch.zeros(4, 4, 64, dtype=torch.bfloat16), torch.tensor([0, 4], dtype=torch.int32)
    n = fd._native()
    for bad in (None, 3, torch.zeros(4, 64, dtype=torch.bfloat16)):
        with pytest.raises(ValueError):
            if call == "rope":
                n.qk_norm_rope(bad, q, q, cu, None, q, q, None, None, 1e-6, False, None, None, 0)
            elif call == "read":
                n.cache_read(bad, cu, q, None, 0)
            elif call == "cache":
                n.cache_attention(bad, q, cu, cu, cu, q, 4, None, None, 0, None, None, 0)
            else:
                n.prompt_attention(bad, q, q, cu, cu, q, 4, None, None, 0, None, 0)
    with pytest.raises(TypeError):
        n.cache_read(q, cu)
