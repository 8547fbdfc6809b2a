"""GPU parity of the attention operators against the float64 oracle.

Bounds.  A float32 sum of n products errs by at most n 2^-24 of the sum of
magnitudes; a head's norm and rotation stay within 2e-6 of the row's largest
element.  An attention output in bfloat16 is off by its own rounding (2^-8 of
it), by that of the weights (2^-8 of the attention of |v|), and by the scores'
float32 error d = D 2^-24 max_j sum_d |q_d k_jd| scale, which moves every
weight by 2 d at most; the log-sum-exp by d and its own rounding.  4-bit codes
are equal to the oracle's wherever the value is not within float32's error of
a threshold, and exactly equal for values, which are not computed on the way.
"""
import math

import numpy as np
import pytest
import torch

from oracle import attention as oa

pytestmark = pytest.mark.gpu
DEV = "cuda"


def _np(t):
    return t.detach().double().cpu().numpy()


def _normal(shape, seed, dtype=torch.float32, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=g) * scale).to(dtype).to(DEV)


def _i32(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device=DEV)


# ---------------------------------------------------------------------------
# norm and rotation into the cache
# ---------------------------------------------------------------------------
ROPE_CASES = [
    # T, H, Hk, D, rot, interleaved, norm, dtype, fused projection, keys out
    (1, 1, 1, 32, 32, False, True, torch.bfloat16, False, True),
    (5, 4, 2, 64, 64, False, True, torch.bfloat16, True, True),
    (33, 3, 1, 128, 128, False, True, torch.bfloat16, True, False),
    (40, 2, 2, 128, 64, True, True, torch.bfloat16, False, True),
    (7, 6, 3, 96, 48, False, False, torch.bfloat16, True, True),
    (9, 2, 1, 96, 96, True, True, torch.float32, True, True),
    (65, 5, 1, 64, 16, False, True, torch.float32, False, True),
    (4, 2, 2, 160, 128, False, True, torch.bfloat16, True, True),
    (17, 1, 1, 256, 256, False, True, torch.float32, False, True),
    (6, 2, 1, 224, 0, False, True, torch.bfloat16, False, True),
    (130, 9, 1, 32, 32, True, False, torch.float32, True, False),
]


def _rope_inputs(T, H, Hk, D, rot, norm, dtype, fused, seed):
    if fused:
        qkv = _normal((T, (H + 2 * Hk) * D + 16), seed, dtype, 1.5)
        q, k, v = (qkv[:, a * D:b * D].view(T, b - a, D) for a, b in ((0, H), (H, H + Hk), (H + Hk, H + 2 * Hk)))
    else:
        q, k, v = (_normal((T, h, D), seed + i, dtype, 1.5) for i, h in enumerate((H, Hk, Hk)))
    qw = _normal((D,), seed + 5) if norm else None
    kw = _normal((D,), seed + 6) if norm else None
    ang = torch.rand((50, max(rot // 2, 1)), generator=torch.Generator().manual_seed(seed)) * 6.28
    cs = torch.cat([ang.cos(), ang.sin()], 1).contiguous().to(DEV) if rot else None
    pos = np.random.default_rng(seed).integers(0, 50, T)
    return q, k, v, qw, kw, cs, pos


def _expected_rows(x, w, eps, cs, pos, rot, inter):
    x, w = _np(x), None if w is None else _np(w)
    cs = np.zeros((50, 0)) if cs is None else _np(cs)
    half = rot // 2
    return np.array([[oa.norm_rope(r, w, eps, cs[p, :half], cs[p, half:], inter) for r in rows]
                     for rows, p in zip(x, pos)])


def _near_threshold(x, held_unit):
    """Whether |x| / unit is within float32's error of a rounding threshold."""
    a = np.abs(x) / held_unit
    gaps = np.abs(a[..., None] - np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0]))
    return gaps.min(-1) < 1e-4


@pytest.mark.parametrize("T,H,Hk,D,rot,inter,norm,dtype,fused,keys", ROPE_CASES)
def test_norm_rope_and_cache(gpu, T, H, Hk, D, rot, inter, norm, dtype, fused, keys):
    q, k, v, qw, kw, cs, pos = _rope_inputs(T, H, Hk, D, rot, norm, dtype, fused, 7 * T + D)
    pages = T // 64 + 3
    slots = np.random.default_rng(T).permutation(pages * 64)[:T]
    cache = gpu.new_cache(pages, Hk, D)
    q_out = torch.full((T, H, D), 7.0, dtype=dtype, device=DEV)
    k_out = torch.full((T, Hk, D), 7.0, dtype=dtype, device=DEV) if keys else None
    gpu.fdllm_qk_norm_rope(q, k, v, _i32(pos), cs, q_out, k_out=k_out, q_weight=qw, k_weight=kw, eps=1e-5,
                           interleaved=inter, cache=cache, slots=_i32(slots))
    torch.cuda.synchronize()
    eq = _expected_rows(q, qw, 1e-5, cs, pos, rot, inter)
    ek = _expected_rows(k, kw, 1e-5, cs, pos, rot, inter)
    rounding = 2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -24
    for got, want in ((q_out, eq), (k_out, ek)):
        if got is not None:
            err = np.abs(_np(got) - want)
            assert (err <= rounding * np.abs(want) * 1.001 + 2e-6 * np.abs(want).max(-1, keepdims=True)).all()
    raw = cache.cpu().numpy()
    written = np.zeros((pages, 64), dtype=bool)
    for t, s in enumerate(slots):
        written[s // 64, s % 64] = True
        for h in range(Hk):
            tile = raw[s // 64, h]
            assert np.array_equal(oa.get(tile, D, True, s % 64),
                                  np.concatenate([oa.value_of(*oa.quantise_group(g)) for g in _np(v)[t, h].reshape(-1, 32)]))
            held = oa.get(tile, D, False, s % 64)
            for g in range(D // 32):
                x = ek[t, h, 32 * g:32 * g + 32]
                byte, codes = oa.quantise_group(x)
                same = held[32 * g:32 * g + 32] == oa.value_of(byte, codes)
                top = np.abs(x).max() / 2.0 ** (byte - 127)
                at_edge = min(abs(top - 7.0), abs(top - 3.5)) < 1e-4      # of the scale's choice
                assert (same | _near_threshold(x, 2.0 ** (byte - 127)) | at_edge).all()
    # nothing else was written
    clean = np.zeros_like(raw)
    for p, tok in np.argwhere(written):
        for at in list(range(0, 64 * D // 2, 64 * 16)) + list(range(64 * D // 2, 64 * D, 64 * 16)):
            clean[p, :, at + tok * 16:at + tok * 16 + 16] = 1
        S = oa.scale_stride(D)
        for base in (64 * D, 64 * D + 64 * S):
            clean[p, :, base + tok * S:base + tok * S + D // 32] = 1
    assert (raw[clean == 0] == 0).all()
    # the reader, in both of its types, agrees with the bytes
    for dt in (torch.bfloat16, torch.float8_e5m2):
        kr, vr = (torch.empty((T, Hk, D), dtype=dt, device=DEV) for _ in range(2))
        gpu.fdllm_cache_read(cache, _i32(slots), kr, vr)
        torch.cuda.synchronize()
        for t, s in enumerate(slots):
            for h in range(Hk):
                assert np.array_equal(_np(kr.float())[t, h], oa.get(raw[s // 64, h], D, False, s % 64))
                assert np.array_equal(_np(vr.float())[t, h], oa.get(raw[s // 64, h], D, True, s % 64))
            if t > 20:
                break


def test_rope_in_place_and_unknown_tokens(gpu):
    T, H, Hk, D = 12, 4, 2, 64
    q, k, v, qw, kw, cs, pos = _rope_inputs(T, H, Hk, D, D, True, torch.bfloat16, False, 3)
    pos[[2, 5]] = (-1, 50)                     # outside the table
    slots = np.arange(T) + 60
    slots[[3, 7, 8]] = (-1, 3 * 64, 1 << 30)   # stored nowhere
    cache = gpu.new_cache(3, Hk, D)
    want_q = torch.empty_like(q)
    want_k = torch.empty_like(k)
    gpu.fdllm_qk_norm_rope(q, k, v, _i32(pos), cs, want_q, k_out=want_k, q_weight=qw, k_weight=kw)
    gpu.fdllm_qk_norm_rope(q, k, v, _i32(pos), cs, q, k_out=k, q_weight=qw, k_weight=kw, cache=cache, slots=_i32(slots))
    torch.cuda.synchronize()
    assert torch.equal(q, want_q) and torch.equal(k, want_k)
    assert (q[[2, 5]] == 0).all() and (k[[2, 5]] == 0).all() and (q[3] != 0).any()
    kr, vr = (torch.full((T, Hk, D), 9.0, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    gpu.fdllm_cache_read(cache, _i32(slots), kr, vr)
    torch.cuda.synchronize()
    for t in range(T):
        stored = t not in (2, 3, 5, 7, 8)
        assert ((vr[t] != 0).any() and (kr[t] != 0).any()) if stored else ((vr[t] == 0).all() and (kr[t] == 0).all())


def test_special_values_in_the_cache(gpu):
    D = 64
    rows = np.zeros((10, D))
    rows[1] = 1e-44                             # subnormal: below the smallest scale
    rows[2, :7] = (6.0, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5)
    rows[2, 7:9] = (5.0, -5.0)
    rows[3, 0], rows[3, 1] = 7.0, 6.9           # 6 at scale 1; the float after 7 takes scale 2
    rows[4, 0] = np.nextafter(np.float32(7.0), np.float32(8.0))
    rows[5, 3] = np.nan
    rows[6, 40] = -np.inf
    rows[7] = 3.0e38
    rows[8, ::2] = -0.0
    rows[9] = np.linspace(-3, 3, D)
    v = torch.tensor(rows, dtype=torch.float32, device=DEV).view(10, 1, D)
    q = torch.zeros((10, 1, D), device=DEV)
    cache = gpu.new_cache(1, 1, D)
    slots = _i32(range(10, 20))
    gpu.fdllm_qk_norm_rope(q, q, v, _i32(np.zeros(10)), None, torch.empty_like(q), cache=cache, slots=slots)
    out = torch.empty((10, 1, D), dtype=torch.bfloat16, device=DEV)
    gpu.fdllm_cache_read(cache, slots, None, out)
    torch.cuda.synchronize()
    tile = cache.cpu().numpy()[0, 0]
    for t in range(10):
        want = np.concatenate([oa.value_of(*oa.quantise_group(g)) for g in _np(v)[t, 0].reshape(-1, 32)])
        assert np.array_equal(oa.get(tile, D, True, 10 + t), want, equal_nan=True), t
        if t != 1:                              # (bfloat16 keeps subnormals; the unpacking instruction may not)
            with np.errstate(over="ignore"):    # 2^128, to which the largest elements round, is no bfloat16
                assert np.array_equal(_np(out.float())[t, 0], want.astype(np.float32), equal_nan=True), t


# ---------------------------------------------------------------------------
# attention
# ---------------------------------------------------------------------------
def _check(out, lse, want, D):
    eo, el, av, sabs = want
    got, gl = _np(out.float()), _np(lse)
    d = D * 2.0 ** -24 * sabs
    bound = 2.0 ** -8 * np.abs(eo) * 1.01 + (2.0 ** -8 * 1.01 + 2 * d[..., None] + 2e-6) * av + 1e-37
    assert np.isfinite(got).all()
    assert (np.abs(got - eo) <= bound).all(), float((np.abs(got - eo) / bound).max())
    empty = np.isneginf(el)
    assert np.array_equal(np.isneginf(gl), empty) and (got[empty] == 0).all()
    assert (np.abs(gl[~empty] - el[~empty]) <= (d + 4e-7 * (1 + np.abs(el)))[~empty]).all()


def _fill(cache, pages, length, Hk, D, seed, junk=True):
    """Random entries in a sequence's pages: codes and scales, with any bytes
    (NaN scales among them) behind its end.  Returns keys and values."""
    g = np.random.default_rng(seed)
    S = oa.scale_stride(D)
    k, v = np.zeros((length, Hk, D)), np.zeros((length, Hk, D))
    for i, page in enumerate(pages):
        n = min(64, length - 64 * i)
        raw = g.integers(0, 256, (Hk, oa.tile_bytes(D)), dtype=np.uint8) if junk else np.zeros((Hk, oa.tile_bytes(D)), np.uint8)
        scales = raw[:, 64 * D:].reshape(Hk, 2, 64, S)
        if junk:
            scales[:, :, n:] = g.choice([0, 1, 254, 255], scales[:, :, n:].shape)
        scales[:, :, :n] = g.integers(124, 128, scales[:, :, :n].shape)
        raw[:, :64 * D] = g.integers(0, 256, (Hk, 64 * D))
        raw[:, 64 * D:] = scales.reshape(Hk, -1)
        cache[page] = torch.tensor(raw, device=DEV)
        codes = raw[:, :64 * D].reshape(Hk, 2, D // 32, 64, 16)
        c = np.stack([codes & 15, codes >> 4], -1).reshape(Hk, 2, D // 32, 64, 32).astype(np.int64)
        vals = np.where(c >= 8, -1.0, 1.0) * oa.MAGNITUDES[c & 7]
        vals = vals * 2.0 ** (scales[..., :D // 32].transpose(0, 1, 3, 2).astype(np.float64) - 127.0)[..., None]
        vals = vals.transpose(1, 3, 0, 2, 4).reshape(2, 64, Hk, D)
        k[64 * i:64 * i + n], v[64 * i:64 * i + n] = vals[0, :n], vals[1, :n]
    return k, v


CACHE_CASES = [
    # D, H, Hk, blk, [(queries, cached tokens)]
    (128, 8, 8, 0, [(1, 1)]),
    (128, 4, 1, 1, [(1, 63), (1, 64), (1, 65), (1, 0), (1, 700)]),      # up to 16 rows: single tokens
    (64, 16, 1, 0, [(1, 129), (1, 2000)]),                               # 16 rows exactly
    (96, 6, 2, 1, [(3, 200), (1, 2), (5, 131), (0, 50)]),
    (64, 17, 1, 0, [(1, 300), (1, 5)]),                                  # 17 rows: 32-row tiles, pages dealt to eight waves
    (128, 2, 2, 0, [(32, 1024), (7, 90), (32, 1)]),
    (128, 2, 2, 32, [(32, 97), (20, 40), (32, 33), (9, 9)]),
    (96, 3, 3, 1, [(30, 333), (32, 12)]),                                # more queries than keys: rows that see nothing
    (128, 8, 4, 1, [(32, 257), (31, 64)]),                               # 64 rows: two waves by two
    (64, 4, 2, 32, [(20, 500), (3, 1000), (0, 0)]),
    (96, 4, 2, 0, [(32, 190)]),
    (128, 8, 2, 0, [(32, 450), (1, 64), (17, 0)]),                       # 128 rows a workgroup
    (64, 8, 1, 1, [(40, 333), (33, 20)]),                                # several groups of rows
    (96, 7, 1, 48, [(50, 100), (64, 64)]),
    (128, 5, 1, 0, [(70, 65), (2, 130), (70, 1)]),
    (64, 4, 1, 0, [(1, 20000)]),
    (128, 4, 4, 1, [(1, 2048)]),                                         # one sequence: items whole up to four pages a set
    (128, 4, 4, 1, [(1, 2049)]),
    (96, 8, 2, 32, [(8, 1500)]),
    (64, 7, 1, 0, [(8, 500)]),
    (64, 40, 8, 0, [(32, 20)] * 33),                                     # more items of one page than workgroups
    (64, 1, 1, 1, [(1, 1 + 7 * i) for i in range(300)]),                 # more sequences than a wave has lanes
]


def _run_cache(gpu, D, H, Hk, blk, seqs, seed, q_start=None, width_more=1, stride_more=0, workspace=None):
    need = [-(-n // 64) for _, n in seqs]
    total = sum(need) + 2
    cache = torch.randint(0, 256, (total, Hk, oa.tile_bytes(D)), dtype=torch.uint8, device=DEV)
    order = np.random.default_rng(seed).permutation(total)
    table = np.full((len(seqs), max(need) + width_more), 1 << 30)         # entries past an end say nothing
    at, kv = 0, []
    for b, m in enumerate(need):
        table[b, :m] = order[at:at + m]
        kv.append(_fill(cache, order[at:at + m], seqs[b][1], Hk, D, seed + b))
        at += m
    T = sum(n for n, _ in seqs)
    wide = _normal((T, H * D + stride_more), seed, torch.bfloat16, 2.0)
    q = wide[:, :H * D].view(T, H, D)
    cu = np.concatenate([[0], np.cumsum([n for n, _ in seqs])])
    out = torch.full((T, H, D), float("nan"), dtype=torch.bfloat16, device=DEV)
    lse = torch.full((T, H), float("nan"), device=DEV)
    ws = gpu.fdllm_cache_attention(q, cache, _i32(table), _i32([n for _, n in seqs]), _i32(cu), out,
                                   max(n for n, _ in seqs), lse=lse, blk=blk,
                                   q_start=None if q_start is None else _i32(q_start), workspace=workspace)
    return q, kv, cu, out, lse, ws, (cache, table)


def _want(q, kv, cu, blk, D, starts=None):
    parts = []
    for b, (k, v) in enumerate(kv):
        n = cu[b + 1] - cu[b]
        start = len(k) - n if starts is None else starts[b]
        parts.append(oa.attend(_np(q[cu[b]:cu[b + 1]].float()), k, v, D ** -0.5, blk, start))
    return [np.concatenate(x) for x in zip(*parts)]


@pytest.mark.parametrize("D,H,Hk,blk,seqs", CACHE_CASES)
def test_cache_attention(gpu, D, H, Hk, blk, seqs):
    q, kv, cu, out, lse, _, _ = _run_cache(gpu, D, H, Hk, blk, seqs, 11 * D + H, stride_more=8 * (H % 3))
    torch.cuda.synchronize()
    _check(out, lse, _want(q, kv, cu, blk, D), D)


def test_cache_attention_query_positions(gpu):
    # a block in the middle of its sequence: the suffix is cached too
    seqs, starts = [(32, 300), (8, 200), (5, 70)], [64, -3, 1000]
    for blk in (0, 1, 32):
        q, kv, cu, out, lse, _, _ = _run_cache(gpu, 128, 4, 2, blk, seqs, 5, q_start=starts)
        torch.cuda.synchronize()
        _check(out, lse, _want(q, kv, cu, blk, 128, starts), 128)


def test_cache_attention_pages_outside_the_cache(gpu):
    # tokens of a page that is not there count as unseen
    D, H, Hk, seqs = 64, 4, 2, [(3, 200), (2, 100)]
    q, kv, cu, out, lse, ws, (cache, table) = _run_cache(gpu, D, H, Hk, 0, seqs, 9)
    table[0, 1], table[1, 0], table[1, 1] = -1, len(cache), 1 << 30
    gpu.fdllm_cache_attention(q, cache, _i32(table), _i32([200, 100]), _i32(cu), out, 3, lse=lse, workspace=ws)
    torch.cuda.synchronize()
    keep = np.r_[0:64, 128:200]
    _check(out, lse, _want(q, [(kv[0][0][keep], kv[0][1][keep]), (kv[1][0][:0], kv[1][1][:0])], cu, 0, D), D)


def test_cache_attention_left_out_sequences_and_lengths(gpu):
    D, H, Hk, seqs = 64, 2, 1, [(2, 100), (3, 100), (2, 64)]
    q, kv, cu, out, lse, ws, (cache, table) = _run_cache(gpu, D, H, Hk, 0, seqs, 4)
    width = table.shape[1]
    # more tokens than the table has pages for, and fewer than none
    table[0, 2] = table[0, 0]
    k, v = _fill(cache, table[0, :2], 128, Hk, D, 6)      # entries in every slot
    gpu.fdllm_cache_attention(q, cache, _i32(table), _i32([1 << 30, -5, 64]), _i32(cu), out, 3, lse=lse, workspace=ws)
    torch.cuda.synchronize()
    assert np.isneginf(_np(lse)[2:5]).all() and (out[2:5] == 0).all()
    assert width == 3
    want = oa.attend(_np(q[:2].float()), np.concatenate([k, k[:64]]), np.concatenate([v, v[:64]]), D ** -0.5, 0, 0)
    _check(out[:2], lse[:2], want, D)
    # counts that are none: the rows stay as they are
    out.fill_(3.0)
    bad = cu.copy()
    bad[1], bad[2] = 5, 2                                 # the second sequence runs backwards, the first has 5 > max_q
    gpu.fdllm_cache_attention(q, cache, _i32(table), _i32([100, 100, 64]), _i32(bad), out, 3, lse=lse, workspace=ws)
    torch.cuda.synchronize()
    assert (out[:2] == 3.0).all()


def test_cache_attention_fewer_queries_than_room(gpu):
    # one sequence with a few of the max_q queries that the call has room for: as
    # many items at max_q as workgroups, so a whole item's share is less than one
    for n, max_q in ((100, 8192), (129, 8192), (5, 8192)):
        q, kv, cu, out, lse, _, (cache, table) = _run_cache(gpu, 64, 8, 8, 1, [(n, 300)], n)
        out.fill_(float("nan"))
        lse.fill_(float("nan"))
        gpu.fdllm_cache_attention(q, cache, _i32(table), _i32([300]), _i32(cu), out, max_q, lse=lse, blk=1)
        torch.cuda.synchronize()
        _check(out, lse, _want(q, kv, cu, 1, 64), 64)


def test_cache_attention_one_page_each(gpu):
    # items of one page are never divided, however many sequences: no workspace
    seqs = [(n, m) for n, m in zip([1, 32, 7, 0, 20] * 9, [64, 5, 1, 64, 0, 33, 63] * 7)]
    q, kv, cu, out, lse, ws, _ = _run_cache(gpu, 128, 8, 2, 1, seqs, 21, width_more=0)
    torch.cuda.synchronize()
    assert ws is None
    _check(out, lse, _want(q, kv, cu, 1, 128), 128)


def test_cache_attention_repeats_bit_for_bit(gpu):
    for D, H, Hk, n in ((128, 8, 2, 32), (64, 4, 1, 1)):
        seqs = [(n, 5000), (n, 77), (n, 1300)]
        q, kv, cu, out, lse, ws, (cache, table) = _run_cache(gpu, D, H, Hk, 0, seqs, 8)
        ref, refl = out.clone(), lse.clone()
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        for i in range(3):
            out.fill_(float("nan"))
            ws.random_(0, 256)                            # scratch needs no initialisation
            torch.cuda.synchronize()
            with torch.cuda.stream(side):
                gpu.fdllm_cache_attention(q, cache, _i32(table), _i32([m for _, m in seqs]), _i32(cu), out, n, lse=lse,
                                          workspace=ws)
            torch.cuda.synchronize()
            assert torch.equal(out, ref) and torch.equal(lse, refl)


def test_cache_beyond_four_gigabytes(gpu):
    D, Hk = 128, 8
    pages = (1 << 32) // (Hk * oa.tile_bytes(D)) + 200
    cache = torch.zeros((pages, Hk, oa.tile_bytes(D)), dtype=torch.uint8, device=DEV)
    T = 130
    slots = torch.arange(pages * 64 - T, pages * 64, dtype=torch.int32, device=DEV)
    x = [_normal((T, Hk, D), i, torch.bfloat16) for i in range(3)]
    gpu.fdllm_qk_norm_rope(x[0], x[1], x[2], _i32(np.zeros(T)), None, torch.empty_like(x[0]), cache=cache, slots=slots)
    k, v = (torch.empty_like(x[1]) for _ in range(2))
    gpu.fdllm_cache_read(cache, slots, k, v)
    first = int(slots[0]) // 64
    table = torch.arange(first, pages, dtype=torch.int32, device=DEV).view(1, -1)
    skip = int(slots[0]) % 64
    out, lse = torch.empty((1, Hk, D), dtype=torch.bfloat16, device=DEV), torch.empty((1, Hk), device=DEV)
    gpu.fdllm_cache_attention(x[0][:1], cache, table, _i32([skip + T]), _i32([0, 1]), out, 1, lse=lse)
    torch.cuda.synchronize()
    zeros = np.zeros((skip, Hk, D))                        # the page's earlier slots hold zeros
    want = oa.attend(_np(x[0][:1].float()), np.concatenate([zeros, _np(k.float())]), np.concatenate([zeros, _np(v.float())]),
                     D ** -0.5, 0, 0)
    _check(out, lse, want, D)


PROMPT_CASES = [
    # D, H, Hk, blk, [(queries, keys)]
    (128, 1, 1, 0, [(1, 1)]),
    (128, 4, 4, 1, [(130, 130), (1, 1), (64, 64)]),
    (64, 8, 2, 1, [(33, 33), (0, 0), (200, 200)]),
    (96, 6, 2, 32, [(65, 65), (31, 95), (128, 128)]),
    (128, 8, 1, 48, [(100, 100), (7, 300)]),
    (64, 3, 3, 0, [(129, 40), (5, 0), (1, 64)]),                          # rows without keys
    (96, 5, 1, 1, [(70, 20), (20, 70)]),                                  # queries before the first key
    (128, 2, 1, 1, [(3, 4000)]),                                          # few rows, a long axis: keys divided
    (64, 2, 2, 0, [(40, 3000), (1, 1), (2, 1025)]),
    (96, 3, 1, 32, [(10, 2500)]),
    (128, 40, 8, 1, [(9, 9)] * 20),
    (64, 4, 2, 32, [(1, 1), (150, 150), (9, 9), (40, 40), (0, 0)]),       # ragged: one sequence after another
    (96, 2, 1, 1, [(1, 1), (3, 2600), (170, 170)]),                       # and with divided keys
    (128, 1, 1, 0, [(20, 3000)] * 3),                                     # more keys than an XCD's cache holds
]


@pytest.mark.parametrize("D,H,Hk,blk,seqs", PROMPT_CASES)
def test_prompt_attention(gpu, D, H, Hk, blk, seqs):
    T, Tk = sum(n for n, _ in seqs), sum(m for _, m in seqs)
    wide = _normal((T, H * D + 24), 3 * D + H, torch.bfloat16, 2.0)
    q = wide[:, :H * D].view(T, H, D)
    # the keys lie among others; rows outside every sequence hold NaN
    lead = 5
    kv = torch.full((Tk + lead + 70, 2 * Hk * D), float("nan"), dtype=torch.bfloat16, device=DEV)
    kv[lead:lead + Tk] = _normal((Tk, 2 * Hk * D), D, torch.bfloat16)
    k, v = kv[:, :Hk * D].view(-1, Hk, D), kv[:, Hk * D:].view(-1, Hk, D)
    cu_q = np.concatenate([[0], np.cumsum([n for n, _ in seqs])])
    cu_k = lead + np.concatenate([[0], np.cumsum([m for _, m in seqs])])
    out = torch.full((T, H, D), float("nan"), dtype=torch.bfloat16, device=DEV)
    lse = torch.full((T, H), float("nan"), device=DEV)
    gpu.fdllm_prompt_attention(q, k, v, _i32(cu_q), _i32(cu_k), out, max(n for n, _ in seqs), lse=lse, blk=blk)
    torch.cuda.synchronize()
    keys = [(_np(k[a:b].float()), _np(v[a:b].float())) for a, b in zip(cu_k, cu_k[1:])]
    _check(out, lse, _want(q, keys, cu_q, blk, D), D)


def test_prompt_attention_left_out_sequences(gpu):
    q, k, v = (_normal((100, 2, 64), i, torch.bfloat16) for i in range(3))
    out = torch.full((100, 2, 64), 3.0, dtype=torch.bfloat16, device=DEV)
    good = _i32([0, 10, 60, 100])
    gpu.fdllm_prompt_attention(q, k, v, _i32([0, 10, 200, 100]), good, out, 50)      # a count past the tensor
    torch.cuda.synchronize()
    assert (out[10:] == 3.0).all() and torch.isfinite(out[:10].float()).all() and (out[:10] != 3.0).any()
    out.fill_(3.0)
    gpu.fdllm_prompt_attention(q, k, v, good, good, out, 40)                          # the second has 50 rows
    torch.cuda.synchronize()
    assert (out[10:60] == 3.0).all() and (out[60:] != 3.0).any()


def test_prompt_attention_repeats_bit_for_bit(gpu):
    for T, Tk in ((300, 300), (4, 5000)):
        q = _normal((T, 4, 128), 1, torch.bfloat16)
        k, v = (_normal((Tk, 2, 128), 2 + i, torch.bfloat16) for i in range(2))
        outs = []
        for _ in range(3):
            out, lse = torch.empty_like(q), torch.empty((T, 4), device=DEV)
            gpu.fdllm_prompt_attention(q, k, v, _i32([0, T]), _i32([0, Tk]), out, T, lse=lse, blk=1)
            outs.append((out, lse))
        torch.cuda.synchronize()
        assert all(torch.equal(a, outs[0][0]) and torch.equal(b, outs[0][1]) for a, b in outs)


def test_capture_into_a_graph(gpu):
    """A decoding step's calls captured: replays with new inputs equal the eager calls."""
    B, n, H, Hk, D, L = 3, 8, 4, 2, 128, 500
    T = B * n
    pages = -(-L // 64)
    cs = torch.rand((L, D), device=DEV)
    table = torch.arange(B * pages, dtype=torch.int32, device=DEV).view(B, pages)
    kv_len, cu = _i32([L, 100, 1]), _i32(np.arange(B + 1) * n)
    pos = _i32(np.tile(np.arange(n), B))
    slots = _i32(np.concatenate([b * pages * 64 + np.arange(n) for b in range(B)]))
    x = [_normal((T, h, D), i, torch.bfloat16) for i, h in enumerate((H, Hk, Hk))]
    cache = gpu.new_cache(B * pages, Hk, D)
    g = torch.Generator(device=DEV).manual_seed(0)
    cache[..., :64 * D] = torch.randint(0, 256, cache[..., :64 * D].shape, dtype=torch.uint8, device=DEV, generator=g)
    cache[..., 64 * D:] = 126
    q_out, out, lse = torch.empty_like(x[0]), torch.empty_like(x[0]), torch.empty((T, H), device=DEV)
    own = torch.empty_like(x[0])
    ws = torch.empty(gpu.fdllm_cache_attention_workspace_size(B, H, Hk, D, n, pages), dtype=torch.uint8, device=DEV)
    need = gpu.fdllm_prompt_attention_workspace_size(B, T, T, H, Hk, D, n)
    ws2 = torch.empty(max(need, 16), dtype=torch.uint8, device=DEV)

    def step():
        gpu.fdllm_qk_norm_rope(x[0], x[1], x[2], pos, cs, q_out, cache=cache, slots=slots)
        gpu.fdllm_cache_attention(q_out, cache, table, kv_len, cu, out, n, lse=lse, workspace=ws)
        gpu.fdllm_prompt_attention(q_out, x[1], x[2], cu, cu, own, n, workspace=ws2)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(3):
        for j, t in enumerate(x):
            t.copy_(_normal(t.shape, 50 + 3 * i + j, torch.bfloat16))
        kv_len.copy_(_i32([L - i, 64 * (i + 1), 1 + i]))
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (q_out, out, lse, own, cache)]
        step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, (q_out, out, lse, own, cache)))
