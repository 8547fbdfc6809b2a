"""Argument checks of the calls for drafted tokens, on the host: each bad call gets
its status and enqueues nothing; and the binding's refusals of tensors."""
import ctypes
import os
import re

import pytest
import torch

import paper_2606_02955_amd as fd

HEADER = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "fdllm.h")
P = ctypes.c_void_p(0x1000)      # never dereferenced: checks fail first
ODD = ctypes.c_void_p(0x1004)
ODD1 = ctypes.c_void_p(0x1001)
Q, R = ctypes.c_void_p(0x2000), ctypes.c_void_p(0x3000)


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(fd.LIB_PATH) or not os.path.exists(fd.BINDING_PATH):
        from paper_2606_02955_amd import build
        build.build()
    return fd.load()


def test_constants_agree_with_header():
    assert int(re.search(r"#define FDLLM_MAX_TREE (\d+)", open(HEADER).read()).group(1)) == fd.MAX_TREE


def _layout(lib, **kw):
    a = dict(parents=P, T=4, cu=P, B=2, max_q=3, kv=P, table=P, width=2, masks=P, words=1, pos=P, slots=P)
    a.update(kw)
    return lib.fdllm_tree_layout(*a.values(), None)


@pytest.mark.parametrize("kw,status", [
    (dict(T=-1), fd.ERR_INVALID_ARG), (dict(B=-1), fd.ERR_INVALID_ARG), (dict(max_q=-1), fd.ERR_INVALID_ARG),
    (dict(width=-1), fd.ERR_INVALID_ARG), (dict(words=-1), fd.ERR_INVALID_ARG), (dict(words=0), fd.ERR_INVALID_ARG),
    (dict(max_q=65), fd.ERR_INVALID_ARG), (dict(max_q=1025, words=100), fd.ERR_SIZE), (dict(words=(1 << 16) + 1), fd.ERR_SIZE),
    (dict(B=65536), fd.ERR_SIZE), (dict(parents=None), fd.ERR_INVALID_ARG), (dict(cu=None), fd.ERR_INVALID_ARG),
    (dict(kv=None), fd.ERR_INVALID_ARG), (dict(masks=None), fd.ERR_INVALID_ARG), (dict(masks=ODD), fd.ERR_INVALID_ARG),
    (dict(table=None), fd.ERR_INVALID_ARG), (dict(T=0), fd.OK), (dict(B=0), fd.OK), (dict(max_q=0), fd.OK)])
def test_layout_refuses(lib, kw, status):
    assert _layout(lib, **kw) == status


def _attention(lib, **kw):
    a = dict(q=P, qs=256, T=4, cu=P, B=2, max_q=3, H=4, Hk=2, D=64, cache=P, pages=3, table=P, width=2, kv=P, masks=P, words=1,
             scale=0.1, out=P, lse=P, ws=P, bytes=1 << 40)
    a.update(kw)
    return lib.fdllm_tree_attention(*a.values(), None)


@pytest.mark.parametrize("kw,status", [
    (dict(T=-1), fd.ERR_INVALID_ARG), (dict(B=-1), fd.ERR_INVALID_ARG), (dict(max_q=-1), fd.ERR_INVALID_ARG),
    (dict(H=0), fd.ERR_INVALID_ARG), (dict(Hk=0), fd.ERR_INVALID_ARG), (dict(pages=-1), fd.ERR_INVALID_ARG),
    (dict(width=-1), fd.ERR_INVALID_ARG), (dict(words=-1), fd.ERR_INVALID_ARG), (dict(words=0), fd.ERR_INVALID_ARG),
    (dict(max_q=65), fd.ERR_INVALID_ARG), (dict(masks=None), fd.ERR_INVALID_ARG), (dict(masks=ODD), fd.ERR_INVALID_ARG),
    (dict(scale=0.0), fd.ERR_INVALID_ARG), (dict(scale=float("nan")), fd.ERR_INVALID_ARG),
    (dict(D=32), fd.ERR_SIZE), (dict(D=160), fd.ERR_SIZE), (dict(Hk=3), fd.ERR_SIZE), (dict(B=65536), fd.ERR_SIZE),
    (dict(width=1 << 26), fd.ERR_SIZE), (dict(q=None), fd.ERR_INVALID_ARG), (dict(cu=None), fd.ERR_INVALID_ARG),
    (dict(kv=None), fd.ERR_INVALID_ARG), (dict(cache=None), fd.ERR_INVALID_ARG), (dict(table=None), fd.ERR_INVALID_ARG),
    (dict(out=None), fd.ERR_INVALID_ARG), (dict(q=ODD), fd.ERR_INVALID_ARG), (dict(qs=252), fd.ERR_INVALID_ARG),
    (dict(qs=260), fd.ERR_INVALID_ARG), (dict(ws=None, width=200), fd.ERR_WORKSPACE), (dict(bytes=1, width=200), fd.ERR_WORKSPACE),
    (dict(T=0), fd.OK), (dict(B=0), fd.OK), (dict(max_q=0), fd.OK)])
def test_attention_refuses(lib, kw, status):
    assert _attention(lib, **kw) == status


def _draft(lib, **kw):
    a = dict(logits=P, stride=100, draft=P, dstride=100, dt=0, T=6, V=100, ids=P, cu=P, B=2, max_q=4, temp=P, u=P, ud=P, tokens=Q,
             n=P, logp=P, ws=P, bytes=1 << 40)
    a.update(kw)
    return lib.fdllm_verify_draft(*a.values(), None)


def _tree(lib, **kw):
    a = dict(logits=P, stride=100, dt=0, T=6, V=100, ids=P, parents=P, cu=P, B=2, max_q=4, temp=P, u=P, path=R, tokens=Q, n=P,
             logp=P, ws=P, bytes=1 << 40)
    a.update(kw)
    return lib.fdllm_verify_tree(*a.values(), None)


@pytest.mark.parametrize("call", [_draft, _tree])
@pytest.mark.parametrize("kw,status", [
    (dict(T=-1), fd.ERR_INVALID_ARG), (dict(B=-1), fd.ERR_INVALID_ARG), (dict(max_q=-1), fd.ERR_INVALID_ARG),
    (dict(dt=2), fd.ERR_UNSUPPORTED_DTYPE), (dict(dt=-1), fd.ERR_UNSUPPORTED_DTYPE), (dict(V=0), fd.ERR_SIZE),
    (dict(V=(1 << 30) + 1, stride=1 << 31), fd.ERR_SIZE), (dict(B=65536), fd.ERR_SIZE), (dict(max_q=1025), fd.ERR_SIZE),
    (dict(stride=99), fd.ERR_INVALID_ARG), (dict(stride=1 << 60), fd.ERR_SIZE), (dict(cu=None), fd.ERR_INVALID_ARG),
    (dict(n=None), fd.ERR_INVALID_ARG), (dict(logits=None), fd.ERR_INVALID_ARG), (dict(logits=ODD1), fd.ERR_INVALID_ARG),
    (dict(logits=ctypes.c_void_p(0x1002), dt=1), fd.ERR_INVALID_ARG), (dict(ids=None), fd.ERR_INVALID_ARG),
    (dict(u=None), fd.ERR_INVALID_ARG), (dict(tokens=P), fd.ERR_INVALID_ARG), (dict(tokens=None), fd.ERR_INVALID_ARG), (dict(ws=ODD), fd.ERR_INVALID_ARG),
    (dict(ws=None), fd.ERR_WORKSPACE), (dict(bytes=95), fd.ERR_WORKSPACE), (dict(B=0), fd.OK)])
def test_verify_refuses(lib, call, kw, status):
    assert call(lib, **kw) == status


@pytest.mark.parametrize("call,kw,status", [
    (_draft, dict(dstride=99), fd.ERR_INVALID_ARG), (_draft, dict(draft=ODD1), fd.ERR_INVALID_ARG),
    (_draft, dict(ud=None), fd.ERR_INVALID_ARG), (_tree, dict(parents=None), fd.ERR_INVALID_ARG),
    (_tree, dict(path=None), fd.ERR_INVALID_ARG), (_tree, dict(path=P), fd.ERR_INVALID_ARG),
    (_tree, dict(path=Q), fd.ERR_INVALID_ARG)])
def test_verify_refuses_more(lib, call, kw, status):
    assert call(lib, **kw) == status


S = ctypes.c_void_p(0x4000)


@pytest.mark.parametrize("call,kw", [
    (_draft, dict(n=P)), (_draft, dict(n=Q)), (_draft, dict(n=R, logp=P)), (_draft, dict(n=R, logp=R)),
    (_draft, dict(n=R, logp=S, ud=S)), (_draft, dict(n=R, logp=S, temp=S)), (_draft, dict(n=R, logp=S, ws=S)),
    (_draft, dict(n=R, logp=None, cu=Q)), (_tree, dict(n=P)), (_tree, dict(n=R)), (_tree, dict(n=S, logp=P)),
    (_tree, dict(n=S, logp=None, cu=R)), (_tree, dict(n=S, logp=None, ws=Q)),
    (_layout, dict(masks=P)), (_layout, dict(masks=Q, pos=P)), (_layout, dict(masks=Q, pos=R, slots=P)),
    (_layout, dict(masks=Q, pos=R, slots=R)), (_layout, dict(masks=Q, pos=None, slots=S, table=S))])
def test_results_in_the_place_of_inputs_are_refused(lib, call, kw):
    assert call(lib, **kw) == fd.ERR_INVALID_ARG


def test_verify_workspace_sizes(lib):
    for args in ((0, 0, 1), (7, 2, 126464), (1, 1, 1)):
        one = fd.fdllm_verify_draft_workspace_size(*args, False)
        assert fd.fdllm_verify_draft_workspace_size(*args, True) >= one >= 0 and fd.fdllm_verify_tree_workspace_size(*args) >= 0
    n = ctypes.c_size_t(0)
    assert lib.fdllm_verify_draft_workspace_size(1, 1, 1, 0, None) == fd.ERR_INVALID_ARG
    assert lib.fdllm_verify_draft_workspace_size(-1, 1, 1, 0, ctypes.byref(n)) == fd.ERR_INVALID_ARG
    assert lib.fdllm_verify_draft_workspace_size(1, 1, 0, 0, ctypes.byref(n)) == fd.ERR_SIZE
    assert lib.fdllm_verify_tree_workspace_size(1, 1, 1, None) == fd.ERR_INVALID_ARG
    assert lib.fdllm_verify_tree_workspace_size(1, -1, 1, ctypes.byref(n)) == fd.ERR_INVALID_ARG
    assert lib.fdllm_verify_tree_workspace_size(1, 65536, 1, ctypes.byref(n)) == fd.ERR_SIZE


def _keep(lib, **kw):
    a = dict(cache=P, layers=2, pages=3, Hk=2, D=64, table=P, width=2, kv=P, cu=P, T=6, B=2, max_q=4, path=P, n=P,
             out=ctypes.c_void_p(0x2000))
    a.update(kw)
    return lib.fdllm_cache_keep(*a.values(), None)


@pytest.mark.parametrize("kw,status", [
    (dict(layers=-1), fd.ERR_INVALID_ARG), (dict(pages=-1), fd.ERR_INVALID_ARG), (dict(Hk=0), fd.ERR_INVALID_ARG),
    (dict(width=-1), fd.ERR_INVALID_ARG), (dict(T=-1), fd.ERR_INVALID_ARG), (dict(B=-1), fd.ERR_INVALID_ARG),
    (dict(max_q=-1), fd.ERR_INVALID_ARG), (dict(D=48), fd.ERR_SIZE), (dict(D=288), fd.ERR_SIZE), (dict(D=0), fd.ERR_SIZE),
    (dict(layers=1 << 23), fd.ERR_SIZE), (dict(B=65536), fd.ERR_SIZE), (dict(max_q=1025), fd.ERR_SIZE),
    (dict(pages=1 << 26), fd.ERR_SIZE), (dict(kv=None), fd.ERR_INVALID_ARG), (dict(cu=None), fd.ERR_INVALID_ARG),
    (dict(n=None), fd.ERR_INVALID_ARG), (dict(path=None), fd.ERR_INVALID_ARG), (dict(cache=None), fd.ERR_INVALID_ARG),
    (dict(cache=ODD), fd.ERR_INVALID_ARG), (dict(table=None), fd.ERR_INVALID_ARG), (dict(out=P), fd.ERR_INVALID_ARG),
    (dict(n=R, out=R), fd.ERR_INVALID_ARG), (dict(cu=R, out=R), fd.ERR_INVALID_ARG),
    (dict(path=R, out=R), fd.ERR_INVALID_ARG), (dict(table=R, out=R), fd.ERR_INVALID_ARG), (dict(B=0), fd.OK)])
def test_keep_refuses(lib, kw, status):
    assert _keep(lib, **kw) == status


@pytest.mark.parametrize("drafted", ["3", "0x4", "3x0", "x", "3x4x5", "-1x2", "32x32"])
def test_command_refuses(drafted, capsys):
    from workloads import cached_generation
    with pytest.raises(SystemExit):
        cached_generation.main([f"--drafted={drafted}"])
    assert "WxD" in capsys.readouterr().err


# ---- tensors ----
def _i(*shape):
    return torch.zeros(shape, dtype=torch.int32)


def test_binding_refuses_tensors(lib):
    f, m, l = torch.zeros(4), torch.zeros((4, 1), dtype=torch.int64), torch.zeros((4, 9), dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="GPU"):
        fd.fdllm_tree_layout(_i(4), _i(2), _i(3), 4, m)
    with pytest.raises(ValueError, match="parents must be"):
        fd.fdllm_tree_layout(_i(2, 2), _i(2), _i(3), 4, m)
    with pytest.raises(ValueError, match="GPU"):
        fd.fdllm_verify_draft(l, _i(4), _i(3), 4, f, torch.zeros(2), _i(4), _i(2))
    with pytest.raises(ValueError, match="bfloat16 or float32"):
        fd.fdllm_verify_tree(l.half(), _i(4), _i(4), _i(3), 4, f, _i(4), _i(4), _i(2))
    with pytest.raises(ValueError, match="vocabulary"):
        fd.fdllm_verify_tree(f, _i(4), _i(4), _i(3), 4, f, _i(4), _i(4), _i(2))
    with pytest.raises(ValueError, match="no cache has tiles"):
        fd.fdllm_cache_keep(torch.zeros((2, 1, 100), dtype=torch.uint8), _i(1, 1), _i(1), _i(2), _i(4), _i(1), 4)
    with pytest.raises(ValueError, match="cache must be"):
        fd.fdllm_cache_keep(torch.zeros((2, 100), dtype=torch.uint8), _i(1, 1), _i(1), _i(2), _i(4), _i(1), 4)
    with pytest.raises(ValueError, match="must be a tensor"):
        fd._native().cache_keep(None, _i(1, 1), _i(1), _i(2), _i(4), _i(1), 4, None, 0)
    with pytest.raises(TypeError, match="arguments wanted"):
        fd._native().verify_tree(l)
