"""What the attention calls refuse for its size: a launch that would not fit is
refused before anything is enqueued, and nothing smaller is."""
import ctypes
import os

import pytest

import paper_2606_02955_amd as fd


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(fd.LIB_PATH):
        from paper_2606_02955_amd import build
        build.build()
    return fd.load()


P = ctypes.c_void_p(0x1000)      # never dereferenced: checks fail first


def _cache_status(lib, B, H, Hk, max_q, width, call):
    if not call:
        n = ctypes.c_size_t(0)
        return lib.fdllm_cache_attention_workspace_size(B, H, Hk, 64, max_q, width, ctypes.byref(n))
    return lib.fdllm_cache_attention(P, H * 64, 6, P, B, max_q, H, Hk, 64, P, 3, P, width, P, None, 0.1, 0, P, None, P,
                                     1 << 60, None)


@pytest.mark.parametrize("B,H,Hk,max_q,width,ok", [
    (1, 32, 32, 1 << 23, 2, False),        # the join's 2^23 workgroups of 512
    (1, 32, 32, (1 << 23) - 128, 2, True),
    (1, 32, 32, 1 << 23, 1, True),         # tables of one page: no join
])
def test_cache_attention_join_has_room(lib, B, H, Hk, max_q, width, ok):
    assert _cache_status(lib, B, H, Hk, max_q, width, False) == (fd.OK if ok else fd.ERR_SIZE)
    if not ok:
        assert _cache_status(lib, B, H, Hk, max_q, width, True) == fd.ERR_SIZE


def _prompt_status(lib, B, T, H, Hk, max_q, call, k_stride=None):
    if not call:
        n = ctypes.c_size_t(0)
        return lib.fdllm_prompt_attention_workspace_size(B, T, T, H, Hk, 64, max_q, 1, ctypes.byref(n))
    stride = k_stride or Hk * 64
    return lib.fdllm_prompt_attention(P, H * 64, P, stride, P, stride, T, T, P, P, B, max_q, H, Hk, 64, 0.1, 1, P, None, P,
                                      1 << 60, None)


@pytest.mark.parametrize("B,H,Hk,ok", [
    (1 << 19, 32, 32, False),              # a workgroup of 256 for every sequence and key head: 2^32 threads
    ((1 << 19) - 1, 32, 32, True),
    (1 << 24, 1, 1, False),
    ((1 << 24) - 1, 1, 1, True),
])
def test_prompt_attention_has_room(lib, B, H, Hk, ok):
    assert _prompt_status(lib, B, 1 << 20, H, Hk, 4, False) == (fd.OK if ok else fd.ERR_SIZE)
    if not ok:
        assert _prompt_status(lib, B, 1 << 20, H, Hk, 4, True) == fd.ERR_SIZE


def test_prompt_attention_strides(lib):
    assert _prompt_status(lib, 1, 64, 4, 4, 64, True, k_stride=16776960) == fd.ERR_SIZE


@pytest.mark.parametrize("T,H,Hk,max_q,ok", [
    (65536, 32, 1, 65536, True),           # 16384 row tiles
    (262140, 32, 1, 262140, True),         # 65535
    (262141, 32, 1, 262141, False),
    (100, 32, 1, 1 << 30, True),           # no sequence is longer than all tokens
])
def test_prompt_attention_row_tiles(lib, T, H, Hk, max_q, ok):
    assert _prompt_status(lib, 1, T, H, Hk, max_q, False) == (fd.OK if ok else fd.ERR_SIZE)
    if not ok:
        assert _prompt_status(lib, 1, T, H, Hk, max_q, True) == fd.ERR_SIZE


def test_room_for_more_queries_than_there_are_costs_no_workspace(lib):
    size = fd.fdllm_prompt_attention_workspace_size
    for B, T, Tk, H, Hk, blk in ((3, 700, 700, 5, 1, 1), (1, 40, 6000, 8, 2, 0), (4, 2000, 2000, 32, 8, 1)):
        assert size(B, T, Tk, H, Hk, 128, 1 << 30, blk) == size(B, T, Tk, H, Hk, 128, T, blk)
