"""What the attention calls refuse of tensors on the GPU: wrong types, shapes,
strides and devices end in an error that names the argument, before any launch."""
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda"
T, H, HK, D, PAGES = 6, 4, 2, 64, 3


def _args(gpu, call):
    bf, i32, f32 = torch.bfloat16, torch.int32, torch.float32

    def t(*shape, dtype=bf):
        return torch.zeros(shape, dtype=dtype, device=DEV)

    cache = gpu.new_cache(PAGES, HK, D)
    cu = torch.tensor([0, 2, T], dtype=i32, device=DEV)
    if call == "fdllm_qk_norm_rope":
        return dict(q=t(T, H, D), k=t(T, HK, D), v=t(T, HK, D), positions=t(T, dtype=i32), cos_sin=t(8, D, dtype=f32),
                    q_out=t(T, H, D), k_out=t(T, HK, D), q_weight=t(D, dtype=f32), k_weight=t(D, dtype=f32), eps=1e-6,
                    interleaved=False, cache=cache, slots=torch.arange(T, dtype=i32, device=DEV))
    if call == "fdllm_cache_read":
        return dict(cache=cache, slots=t(T, dtype=i32), k_out=t(T, HK, D), v_out=t(T, HK, D))
    if call == "fdllm_cache_attention":
        return dict(q=t(T, H, D), cache=cache, page_table=t(2, PAGES, dtype=i32), kv_len=t(2, dtype=i32), cu_q=cu,
                    out=t(T, H, D), max_q=4, lse=t(T, H, dtype=f32), scale=None, blk=0, q_start=t(2, dtype=i32),
                    workspace=None)
    return dict(q=t(T, H, D), k=t(T, HK, D), v=t(T, HK, D), cu_q=cu, cu_k=cu.clone(), out=t(T, H, D), max_q=4,
                lse=t(T, H, dtype=f32), scale=None, blk=0, workspace=None)


CALLS = ["fdllm_qk_norm_rope", "fdllm_cache_read", "fdllm_cache_attention", "fdllm_prompt_attention"]
TENSORS = {
    "fdllm_qk_norm_rope": ["q", "k", "v", "positions", "cos_sin", "q_out", "k_out", "q_weight", "k_weight", "cache", "slots"],
    "fdllm_cache_read": ["cache", "slots", "k_out", "v_out"],
    "fdllm_cache_attention": ["q", "cache", "page_table", "kv_len", "cu_q", "out", "lse", "q_start"],
    "fdllm_prompt_attention": ["q", "k", "v", "cu_q", "cu_k", "out", "lse"],
}
EACH = [(c, n) for c in CALLS for n in TENSORS[c]]
# whose heads are read where they lie: strides between tokens are allowed
STRIDED = {"q", "k", "v"}


def _refused(gpu, call, args, match):
    with pytest.raises(ValueError, match=match):
        getattr(gpu, call)(**args)
    torch.cuda.synchronize()


@pytest.mark.parametrize("call", CALLS)
def test_the_arguments_as_they_are_pass(gpu, call):
    getattr(gpu, call)(**_args(gpu, call))
    torch.cuda.synchronize()


@pytest.mark.parametrize("call,name", EACH)
def test_wrong_type(gpu, call, name):
    a = _args(gpu, call)
    a[name] = a[name].to(torch.float64)
    _refused(gpu, call, a, "must be|is read as")


@pytest.mark.parametrize("call,name", EACH)
def test_wrong_shape(gpu, call, name):
    a = _args(gpu, call)
    x = a[name]
    # (whose last axis may have any length: one axis more)
    a[name] = x.unsqueeze(0) if name in ("q", "cos_sin", "page_table") else torch.cat([x, x], dim=-1)
    _refused(gpu, call, a, "must (have shape|be )|no cache has heads")


@pytest.mark.parametrize("call,name", EACH)
def test_not_on_the_gpu(gpu, call, name):
    a = _args(gpu, call)
    a[name] = a[name].cpu()
    _refused(gpu, call, a, "must be a GPU tensor")


@pytest.mark.parametrize("call,name", [(c, n) for c, n in EACH if n not in STRIDED])
def test_not_contiguous(gpu, call, name):
    a = _args(gpu, call)
    x = a[name]
    a[name] = torch.stack([x, x], dim=-1)[..., 0]
    assert a[name].shape == x.shape and not a[name].is_contiguous()
    _refused(gpu, call, a, f"{name} must be contiguous")


@pytest.mark.parametrize("call,name", [(c, n) for c, n in EACH if n in STRIDED])
def test_heads_apart(gpu, call, name):
    for wide in (lambda x: torch.stack([x, x], dim=2).flatten(1, 2)[:, ::2], lambda x: torch.stack([x, x], dim=3)[..., 0]):
        a = _args(gpu, call)
        shape = a[name].shape
        a[name] = wide(a[name])
        assert a[name].shape == shape
        _refused(gpu, call, a, f"{name}: the heads of a token must lie side by side")


@pytest.mark.parametrize("call,name", [(c, n) for c, n in EACH if n in STRIDED])
def test_tokens_at_the_same_place(gpu, call, name):
    a = _args(gpu, call)
    a[name] = a[name][:1].expand(T, -1, -1)
    with pytest.raises(gpu.FdllmError) as e:
        getattr(gpu, call)(**a)
    assert e.value.status == gpu.ERR_INVALID_ARG


@pytest.mark.parametrize("call", ["fdllm_cache_attention", "fdllm_prompt_attention"])
def test_workspaces(gpu, call):
    a = _args(gpu, call)
    if call == "fdllm_prompt_attention":          # one that needs a workspace: few rows, many keys
        a["k"], a["v"] = (torch.zeros((5000, HK, D), dtype=torch.bfloat16, device=DEV) for _ in range(2))
        a["cu_k"] = torch.tensor([0, 2500, 5000], dtype=torch.int32, device=DEV)
    ws = getattr(gpu, call)(**a)
    assert ws is not None and ws.is_cuda
    assert getattr(gpu, call)(**{**a, "workspace": ws}) is ws
    with pytest.raises(gpu.FdllmError) as e:
        getattr(gpu, call)(**{**a, "workspace": ws[:-16]})
    assert e.value.status == gpu.ERR_WORKSPACE
    with pytest.raises(gpu.FdllmError) as e:
        getattr(gpu, call)(**{**a, "workspace": torch.cat([ws, ws])[1:]})
    assert e.value.status == gpu.ERR_INVALID_ARG
    for bad in (ws.cpu(), torch.stack([ws, ws], 1)[:, 0]):
        _refused(gpu, call, {**a, "workspace": bad}, "workspace must be a contiguous GPU tensor")
    _refused(gpu, call, {**a, "workspace": 3}, "workspace must be a tensor")


@pytest.mark.parametrize("call,name,bad", [
    ("fdllm_cache_attention", "max_q", 1 << 40), ("fdllm_cache_attention", "max_q", 1.5),
    ("fdllm_prompt_attention", "max_q", None), ("fdllm_cache_attention", "blk", "1"), ("fdllm_prompt_attention", "blk", 1 << 31),
    ("fdllm_cache_attention", "scale", "x"), ("fdllm_qk_norm_rope", "eps", None)])
def test_numbers(gpu, call, name, bad):
    _refused(gpu, call, {**_args(gpu, call), name: bad}, f"{name} (must be a|does not fit)")


def test_what_is_neither_true_nor_false(gpu):
    class Neither:
        def __bool__(self):
            raise TypeError("neither")

    a = _args(gpu, "fdllm_qk_norm_rope")
    before = a["q_out"].fill_(3.0).clone()
    _refused(gpu, "fdllm_qk_norm_rope", {**a, "interleaved": Neither()}, "interleaved must be true or false")
    assert torch.equal(a["q_out"], before)


@pytest.mark.parametrize("name", ["v", "slots"])
def test_what_a_cache_needs(gpu, name):
    _refused(gpu, "fdllm_qk_norm_rope", {**_args(gpu, "fdllm_qk_norm_rope"), name: None}, "v and slots must be given")


def test_reading_into_nothing(gpu):
    a = _args(gpu, "fdllm_cache_read")
    _refused(gpu, "fdllm_cache_read", {**a, "k_out": None, "v_out": None}, "k_out or v_out must be given")
    _refused(gpu, "fdllm_cache_read", {**a, "v_out": a["v_out"].to(torch.float8_e5m2)}, "v_out must be BFloat16")
