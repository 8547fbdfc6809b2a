"""Results of the calls for drafted tokens that share memory with an input, the
workspace or another result are refused, wherever they begin in it; memory beside
them is not.  On the host: refused calls enqueue nothing, and the rule itself is
compiled for the host (csrc/attn_work.h)."""
import ctypes
import os
import subprocess

import pytest
import torch

import paper_2606_02955_amd as fd

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2606_02955_amd", "csrc")
K = 1 << 16


def at(address):
    return ctypes.c_void_p(address)


@pytest.fixture(scope="module")
def lib():
    if torch.cuda.is_available():
        pytest.skip("addresses of nothing: for machines without a GPU")
    if not os.path.exists(fd.LIB_PATH) or not os.path.exists(fd.BINDING_PATH):
        from paper_2606_02955_amd import build
        build.build()
    return fd.load()


# every argument in 64 KiB of its own
def _layout(lib, **kw):
    a = dict(parents=at(K), T=8, cu=at(2 * K), B=2, max_q=6, kv=at(3 * K), table=at(4 * K), width=3, masks=at(5 * K), words=2,
             pos=at(6 * K), slots=at(7 * K))
    a.update(kw)
    return lib.fdllm_tree_layout(*a.values(), None)


def _attention(lib, **kw):
    a = dict(q=at(K), qs=384, T=8, cu=at(2 * K), B=2, max_q=6, H=4, Hk=2, D=64, cache=at(3 * K), pages=3, table=at(4 * K), width=3,
             kv=at(5 * K), masks=at(6 * K), words=2, scale=0.1, out=at(7 * K), lse=at(8 * K), ws=at(1 << 32), bytes=1 << 40)
    a.update(kw)
    return lib.fdllm_tree_attention(*a.values(), None)


def _draft(lib, **kw):
    a = dict(logits=at(K), stride=120, draft=at(2 * K), dstride=100, dt=1, T=6, V=100, ids=at(3 * K), cu=at(4 * K), B=2, max_q=4,
             temp=at(5 * K), u=at(6 * K), ud=at(7 * K), tokens=at(8 * K), n=at(9 * K), logp=at(10 * K), ws=at(1 << 32), bytes=1 << 40)
    a.update(kw)
    return lib.fdllm_verify_draft(*a.values(), None)


def _tree(lib, **kw):
    a = dict(logits=at(K), stride=120, dt=1, T=6, V=100, ids=at(2 * K), parents=at(3 * K), cu=at(4 * K), B=2, max_q=4, temp=at(5 * K),
             u=at(6 * K), path=at(7 * K), tokens=at(8 * K), n=at(9 * K), logp=at(10 * K), ws=at(1 << 32), bytes=1 << 40)
    a.update(kw)
    return lib.fdllm_verify_tree(*a.values(), None)


def _keep(lib, **kw):
    a = dict(cache=at(1 << 32), layers=2, pages=3, Hk=2, D=64, table=at(K), width=2, kv=at(2 * K), cu=at(3 * K), T=6, B=2, max_q=4,
             path=at(4 * K), n=at(5 * K), out=at(6 * K))
    a.update(kw)
    return lib.fdllm_cache_keep(*a.values(), None)


TILE = 64 * (64 + 2 * 4)
OVERLAPS = [
    # a call, a result at an address in something else: its second element, its last byte, and from before it into it
    (_layout, dict(masks=at(K + 8)), "parents"), (_layout, dict(pos=at(K + 4 * 7)), "the last parent"),
    (_layout, dict(slots=at(2 * K + 8)), "cu_q"), (_layout, dict(pos=at(3 * K + 4)), "kv_len"),
    (_layout, dict(slots=at(4 * K + 20)), "the table"), (_layout, dict(masks=at(4 * K - 120)), "into the table"),
    (_layout, dict(pos=at(5 * K + 124)), "the masks' last word"), (_layout, dict(slots=at(6 * K - 28)), "into the positions"),
    (_attention, dict(out=at(K + 16)), "q, a little further on"), (_attention, dict(out=at(K + 2 * (7 * 384) + 496)), "q's last row"),
    (_attention, dict(out=at(K)), "q whose rows lie apart"), (_attention, dict(lse=at(K + 4)), "q"),
    (_attention, dict(out=at(2 * K), cu=at(2 * K + 32)), "cu_q"), (_attention, dict(out=at(3 * K + 6 * TILE - 16)), "the cache's end"),
    (_attention, dict(lse=at(3 * K + 64)), "the cache"), (_attention, dict(lse=at(4 * K + 20)), "the table"),
    (_attention, dict(lse=at(5 * K + 4)), "kv_len"), (_attention, dict(out=at(6 * K + 112)), "the masks"),
    (_attention, dict(out=at(7 * K), lse=at(7 * K + 4092)), "out"), (_attention, dict(width=200, out=at((1 << 32) + 4096)), "the workspace"),
    (_draft, dict(tokens=at(K + 4)), "logits"), (_draft, dict(logp=at(K + 480 * 5 + 396)), "the last row of logits"),
    (_draft, dict(n=at(2 * K + 2396)), "draft_logits"), (_draft, dict(tokens=at(3 * K + 4)), "ids"),
    (_draft, dict(tokens=at(3 * K - 4)), "into ids"), (_draft, dict(n=at(4 * K + 8)), "cu_q"), (_draft, dict(n=at(5 * K + 4)), "temperature"),
    (_draft, dict(logp=at(6 * K + 20)), "u"), (_draft, dict(n=at(7 * K - 4)), "into u_draw"), (_draft, dict(tokens=at(9 * K - 20)), "into n"),
    (_draft, dict(logp=at(8 * K + 12)), "tokens"), (_draft, dict(tokens=at((1 << 32) + 16)), "the workspace"),
    (_draft, dict(T=0, tokens=at(K), n=at(4 * K + 4)), "cu_q, without rows"),
    (_tree, dict(path=at(K + 480)), "logits"), (_tree, dict(tokens=at(2 * K + 20)), "ids"), (_tree, dict(path=at(3 * K + 4)), "parents"),
    (_tree, dict(logp=at(4 * K + 8)), "cu_q"), (_tree, dict(n=at(5 * K + 4)), "temperature"), (_tree, dict(tokens=at(6 * K - 20)), "into u"),
    (_tree, dict(path=at(8 * K + 4)), "tokens"), (_tree, dict(n=at((1 << 32) + 200)), "the workspace"),
    (_keep, dict(out=at(K + 12)), "the table"), (_keep, dict(out=at(2 * K + 4)), "kv_len"), (_keep, dict(out=at(3 * K + 8)), "cu_q"),
    (_keep, dict(out=at(4 * K + 20)), "path"), (_keep, dict(out=at(5 * K - 4)), "into n_path"),
    (_keep, dict(out=at((1 << 32) + 12 * TILE - 4)), "the cache's end"), (_keep, dict(path=at((1 << 32) + 16)), "path in the cache"),
    (_keep, dict(kv=at((1 << 32) - 4)), "kv_len into the cache"),
]


@pytest.mark.parametrize("call,kw,what", OVERLAPS)
def test_overlaps_are_refused(lib, call, kw, what):
    assert call(lib, **kw) == fd.ERR_INVALID_ARG


BESIDE = [
    # ends where something begins, or begins where it ends
    (_layout, dict(pos=at(K - 32), slots=at(K + 32))), (_layout, dict(masks=at(4 * K - 128), pos=at(4 * K + 24))),
    (_attention, dict(out=at(3 * K - 4096), lse=at(3 * K + 6 * TILE))), (_attention, dict(qs=256, out=at(K))),     # q itself
    (_attention, dict(T=1, out=at(K))),
    (_attention, dict(width=2, lse=at((1 << 32) + 4096))),          # (a call that needs no workspace)
    (_draft, dict(tokens=at(3 * K + 24), n=at(4 * K - 8), logp=at(4 * K + 12))), (_draft, dict(n=at(K + 400))),    # between two rows
    (_draft, dict(n=at(K + 480 * 5 + 400))), (_draft, dict(logp=None)), (_draft, dict(draft=at(K), dstride=120)),
    (_tree, dict(path=at(8 * K - 24), logp=at(8 * K + 24))), (_keep, dict(out=at((1 << 32) + 12 * TILE))), (_keep, dict(out=None)),
    (_keep, dict(pages=0, out=at(1 << 32))),
]


@pytest.mark.parametrize("call,kw", BESIDE)
def test_memory_beside_it_is_not(lib, call, kw):
    # past the checks there is no GPU to launch on
    assert call(lib, **kw) == fd.ERR_HIP


SHIM = r"""
#include "attn_work.h"
using namespace fdllm;
extern "C" int meet(uintptr_t r, size_t bytes, uintptr_t p, size_t row, size_t stride, long long rows) {
  return !apart({Span((const void*)r, bytes)}, {Span((const void*)p, row, stride, rows)});
}
"""


def test_the_rule_itself(tmp_path):
    src, so = tmp_path / "shim.cpp", tmp_path / "shim.so"
    src.write_text(SHIM)
    subprocess.run(["g++", "-O1", "-std=c++17", "-shared", "-fPIC", "-I", CSRC, str(src), "-o", str(so)], check=True)
    meet = ctypes.CDLL(str(so)).meet
    meet.argtypes = [ctypes.c_size_t] * 5 + [ctypes.c_longlong]
    for p, row, stride, rows in ((100, 7, 10, 5), (100, 10, 10, 3), (100, 1, 25, 2), (100, 5, 9, 1), (100, 0, 4, 3), (100, 4, 4, 0),
                                 (0, 7, 10, 5)):
        held = {p + k * stride + i for k in range(rows) for i in range(row)} if p else set()
        for r in range(80, 170):
            for n in (0, 1, 2, 3, 4, 12, 40):
                assert bool(meet(r, n, p, row, stride, rows)) == bool(held & set(range(r, r + n))), (p, row, stride, rows, r, n)
    # the largest rows that the calls take
    far = 1 << 40
    assert meet(far + ((1 << 60) - 8), 4, far, 8, 1 << 59, 2) == 0 and meet(far + (1 << 59) + 4, 4, far, 8, 1 << 59, 2) == 1
