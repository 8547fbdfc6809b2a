// qk_rope.hip -- the heads of queries and keys before attention: RMS norm and
// rotation by position in one pass over them, with the keys and values written
// into the 4-bit cache on the way; and what the cache holds, read back.
//
// A head's row x of D elements becomes y = x rsqrt(mean x^2 + eps) w, then the
// pairs (y_a, y_b) of the first `rot` elements (y_a cos - y_b sin, y_b cos +
// y_a sin) with the angles of the token's position; all in float32, rounded
// once where it is stored.
#include <hip/hip_runtime.h>

#include <stdint.h>

#include "attn_common.h"
#include "fdllm.h"

namespace fdllm {

struct RopeArgs {
  const void* q;
  const void* k;
  const void* v;
  long long q_stride, k_stride, v_stride;   // elements from token to token
  int T, H, Hk, D;
  const float* q_weight;
  const float* k_weight;
  float eps;
  const int32_t* positions;
  const float* cos_sin;   // [n_pos, rot]: cosines, then sines
  int n_pos, rot;
  void* q_out;
  void* k_out;
  uint8_t* cache;
  int n_pages;
  const int32_t* slots;
  int heads_per_wg;
};

constexpr int kRopeThreads = 256;
constexpr int kRopeMaxD = 256;

// Eight elements as they lie in memory, and as floats.
template <typename Elem>
struct Octet;
template <>
struct Octet<float> {
  f32x4 a, b;
  __device__ __forceinline__ void load(const float* p) { a = *(const f32x4*)p, b = *(const f32x4*)(p + 4); }
  __device__ __forceinline__ void to(float* x) const {
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = a[i], x[4 + i] = b[i];
  }
};
template <>
struct Octet<__bf16> {
  bf16x8 a;
  __device__ __forceinline__ void load(const __bf16* p) { a = *(const bf16x8*)p; }
  __device__ __forceinline__ void to(float* x) const {
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = (float)a[i];
  }
};
__device__ __forceinline__ void load8(const float* p, float* x) {
  Octet<float> o;
  o.load(p);
  o.to(x);
}
__device__ __forceinline__ void store8(float* p, const float* x) {
  *(f32x4*)p = f32x4{x[0], x[1], x[2], x[3]};
  *(f32x4*)(p + 4) = f32x4{x[4], x[5], x[6], x[7]};
}
__device__ __forceinline__ void store8(__bf16* p, const float* x) {
  bf16x8 a;
#pragma unroll
  for (int i = 0; i < 8; ++i) a[i] = (__bf16)x[i];
  *(bf16x8*)p = a;
}

// Four neighbouring lanes hold a group of 32, eight each: codes and scale of
// the group.  The largest magnitude is taken of the bits as whole numbers, so
// a NaN counts as the largest of all: such a group, or one with an infinity,
// gets the scale byte 255 and reads back as NaN.
__device__ __forceinline__ uint32_t quantise8(const float* x, uint32_t* scale_byte) {
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(x[i]) & 0x7fffffffu);
  top = max(top, (uint32_t)dpp<kDppXor1>((int)top));
  top = max(top, (uint32_t)dpp<kDppXor2>((int)top));
  if (top >= 0x7f800000u) {
    *scale_byte = 255;
    return 0;
  }
  // the smallest e with top <= 7 * 2^e = 1.75 * 2^(e + 2): the exponent of top,
  // one more where its fraction is over 1.75, less 2.  (With 7, not 6 as the
  // largest code, the root mean square error of normal values is the least:
  // 11.2% of theirs against 11.5% at 6 and 11.5% at 8.)
  int byte = (int)((top + 0x1fffffu) >> 23) - 2;
  byte = byte < 1 ? 1 : byte;
  *scale_byte = (uint32_t)byte;
  const float s = scale_of((uint32_t)byte);
  uint32_t c = 0;
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[0], x[1], s, 0);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[2], x[3], s, 1);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[4], x[5], s, 2);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[6], x[7], s, 3);
  return c;
}

// Elements [8 o, 8 o + 8) of a token's head into its tile.
__device__ __forceinline__ void write_octet(uint8_t* tile, int D, bool value, int token, int o, const float* x) {
  uint32_t byte;
  const uint32_t codes = quantise8(x, &byte);
  const int g = o / 4;
  *(uint32_t*)(tile + (value ? codes_bytes(D) : 0) + (g * kPage + token) * kCodeBytes + (o % 4) * 4) = codes;
  if (o % 4 == 0) tile[(value ? v_scales_at(D) : k_scales_at(D)) + token * scale_stride(D) + g] = (uint8_t)byte;
}

// Bound by memory: 14088 tokens of 32 + 8 + 8 heads of 128 in bfloat16, keys out
// and into the cache, 76 us for 333 MB, 4.4 TB/s (an elementwise copy reaches 6.2);
// its waves wait for memory two thirds of the time.
//
// A workgroup takes 256 / lanes tokens of a few heads; `lanes` (8 up to D =
// 128, 16 beyond) share a row.  A lane holds two octets of its row that rotate
// against each other, with the cosines and sines and the norm's weights, which
// it keeps over the heads; the next head's row is on its way meanwhile.  Keys
// reach the cache through LDS, where they change hands from octets that rotate
// together to octets that share a scale.
template <typename Elem, bool Interleaved>
__global__ void __launch_bounds__(kRopeThreads)
k_rope(const RopeArgs a) {
  __shared__ float s_row[kRopeThreads * 16];
  const int D = a.D, rot = a.rot;
  const int lanes = D <= 128 ? 8 : 16;
  const int j = threadIdx.x % lanes;
  const int tokens = kRopeThreads / lanes;
  const int local = threadIdx.x / lanes;
  const int t = blockIdx.x * tokens + local;
  const bool live = t < a.T;
  const int tc = live ? t : a.T - 1;
  const int octets = D / 8, ro = rot / 16;   // octets of a row; pairs of them that rotate
  const bool mine = j < octets / 2;
  int oa, ob;
  if (Interleaved || j >= ro) {
    const int r = Interleaved ? j : j - ro;
    oa = (Interleaved ? 0 : 2 * ro) + 2 * r;
    ob = oa + 1;
  } else {
    oa = j;
    ob = j + ro;
  }
  if (!mine) oa = ob = 0;
  const bool turn = mine && j < ro;

  const int pos = a.positions[tc];
  const bool known = rot == 0 || (pos >= 0 && pos < a.n_pos);
  const int slot = a.cache ? a.slots[tc] : -1;
  const bool kept = live && known && slot >= 0 && slot / kPage < a.n_pages;
  float cs[8], sn[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) cs[i] = 1.0f, sn[i] = 0.0f;
  if (turn && known) {
    const float* row = a.cos_sin + (size_t)pos * rot + 8 * j;
    load8(row, cs);
    load8(row + rot / 2, sn);
  }

  const int heads = a.H + a.Hk + (a.cache ? a.Hk : 0);
  const int first = blockIdx.y * a.heads_per_wg;
  const int last = min(first + a.heads_per_wg, heads);
  // consecutive octets, of values and of keys on their way to the cache: lanes
  // 4 i .. 4 i + 3 hold the groups 2 i and 2 i + 1
  const int va = (j / 4) * 8 + j % 4, vb = va + 4;
  const int la = va < octets ? va : 0, lb = vb < octets ? vb : 0;
  const size_t page_of_slot = kept ? slot / kPage : 0;
  const int in_page = kept ? slot % kPage : 0;
  const Elem* qrow = (const Elem*)a.q + (size_t)tc * a.q_stride;
  const Elem* krow = (const Elem*)a.k + (size_t)tc * a.k_stride;
  const Elem* vrow = (const Elem*)a.v + (size_t)tc * a.v_stride;
  Octet<Elem> na, nb;   // the next head's
  const auto fetch = [&](int hh) {
    const bool is_q = hh < a.H, is_v = hh >= a.H + a.Hk;
    const Elem* src = is_q ? qrow + (size_t)hh * D
                    : is_v ? vrow + (size_t)(hh - a.H - a.Hk) * D : krow + (size_t)(hh - a.H) * D;
    na.load(src + 8 * (is_v ? la : oa));
    nb.load(src + 8 * (is_v ? lb : ob));
  };
  float wa[8], wb[8];
  const float* w = nullptr;   // the weights that wa and wb hold
  fetch(first);
  for (int hh = first; hh < last; ++hh) {
    const bool is_q = hh < a.H, is_v = hh >= a.H + a.Hk;
    const int h = is_q ? hh : is_v ? hh - a.H - a.Hk : hh - a.H;
    float xa[8], xb[8];
    na.to(xa);
    nb.to(xb);
    if (hh + 1 < last) fetch(hh + 1);
    uint8_t* tile = a.cache + (page_of_slot * a.Hk + h) * tile_bytes(D);
    if (is_v) {
      if (kept && va < octets) write_octet(tile, D, true, in_page, va, xa);
      if (kept && vb < octets) write_octet(tile, D, true, in_page, vb, xb);
      continue;
    }
    const float* weight = is_q ? a.q_weight : a.k_weight;
    if (weight) {
      if (weight != w) {
        load8(weight + 8 * oa, wa);
        load8(weight + 8 * ob, wb);
        w = weight;
      }
      float ss = 0.0f;
#pragma unroll
      for (int i = 0; i < 8; ++i) ss = __builtin_fmaf(xa[i], xa[i], __builtin_fmaf(xb[i], xb[i], ss));
      ss = mine ? ss : 0.0f;
      ss += partner_f32<0>(ss);
      ss += partner_f32<1>(ss);
      ss += partner_f32<2>(ss);
      if (lanes == 16) ss += partner_f32<3>(ss);
      const float r = 1.0f / __builtin_sqrtf(ss / (float)D + a.eps);
#pragma unroll
      for (int i = 0; i < 8; ++i) xa[i] = xa[i] * r * wa[i], xb[i] = xb[i] * r * wb[i];
    }
    if (turn) {
      if (Interleaved) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float u = xa[2 * i], v = xa[2 * i + 1], y = xb[2 * i], z = xb[2 * i + 1];
          xa[2 * i] = u * cs[i] - v * sn[i], xa[2 * i + 1] = v * cs[i] + u * sn[i];
          xb[2 * i] = y * cs[4 + i] - z * sn[4 + i], xb[2 * i + 1] = z * cs[4 + i] + y * sn[4 + i];
        }
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float u = xa[i], v = xb[i];
          xa[i] = u * cs[i] - v * sn[i], xb[i] = v * cs[i] + u * sn[i];
        }
      }
    }
    if (!known) {
#pragma unroll
      for (int i = 0; i < 8; ++i) xa[i] = xb[i] = 0.0f;
    }
    Elem* out = is_q ? (Elem*)a.q_out + ((size_t)tc * a.H + h) * D
                     : a.k_out ? (Elem*)a.k_out + ((size_t)tc * a.Hk + h) * D : nullptr;
    if (live && mine && out) {
      store8(out + 8 * oa, xa);
      store8(out + 8 * ob, xb);
    }
    if (!is_q && a.cache) {
      float* row = s_row + local * 16 * lanes;
      if (mine) {
        store8(row + 8 * oa, xa);
        store8(row + 8 * ob, xb);
      }
      __builtin_amdgcn_wave_barrier();   // the lanes of a row are in one wave
      float ya[8], yb[8];
      load8(row + 8 * la, ya);
      load8(row + 8 * lb, yb);
      __builtin_amdgcn_wave_barrier();
      if (kept && va < octets) write_octet(tile, D, false, in_page, va, ya);
      if (kept && vb < octets) write_octet(tile, D, false, in_page, vb, yb);
    }
  }
}

// ---------------------------------------------------------------------------
// what the cache holds: a thread per sixteen elements of a token's head (14088
// tokens of 8 heads 12.7 us for 44 MB)
// ---------------------------------------------------------------------------
__device__ __forceinline__ void store_held(__bf16* p, const bf16x2* x, bool nan) {
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    u32x4 o;
#pragma unroll
    for (int i = 0; i < 4; ++i) o[i] = nan ? 0x7fc07fc0u : __builtin_bit_cast(uint32_t, x[4 * k + i]);
    *(u32x4*)(p + 8 * k) = o;
  }
}
__device__ __forceinline__ void store_held(uint8_t* p, const bf16x2* x, bool nan) {
  u32x4 o;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    int w = 0;
    w = __builtin_amdgcn_cvt_pk_bf8_f32((float)x[2 * i][0], (float)x[2 * i][1], w, false);
    w = __builtin_amdgcn_cvt_pk_bf8_f32((float)x[2 * i + 1][0], (float)x[2 * i + 1][1], w, true);
    o[i] = nan ? 0x7f7f7f7fu : (uint32_t)w;
  }
  *(u32x4*)p = o;
}

template <typename Out>
__global__ void __launch_bounds__(256)
k_cache_read(const uint8_t* __restrict__ cache, int n_pages, int Hk, int D, const int32_t* __restrict__ slots,
             long long n, Out* __restrict__ k_out, Out* __restrict__ v_out) {
  const int pieces = D / 16;
  for (long long i = blockIdx.x * 256ll + threadIdx.x; i < n; i += gridDim.x * 256ll) {
    const int o = (int)(i % pieces);
    const long long th = i / pieces;
    const int h = (int)(th % Hk);
    const int slot = slots[th / Hk];
    const bool there = slot >= 0 && slot / kPage < n_pages;
    const int token = there ? slot % kPage : 0;
    const uint8_t* tile = cache + ((size_t)(there ? slot / kPage : 0) * Hk + h) * tile_bytes(D);
#pragma unroll
    for (int kv = 0; kv < 2; ++kv) {
      Out* out = kv ? v_out : k_out;
      if (!out) continue;
      const uint32_t byte = tile[(kv ? v_scales_at(D) : k_scales_at(D)) + token * scale_stride(D) + o / 2];
      u32x2 c = *(const u32x2*)(tile + kv * codes_bytes(D) + (o / 2 * kPage + token) * kCodeBytes + o % 2 * 8);
      const float s = scale_of(there && byte != 255 ? byte : kUnitScale);
      bf16x2 x[8];
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const uint32_t ck = there ? c[k] : 0u;
        x[4 * k + 0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(ck, s, 0);
        x[4 * k + 1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(ck, s, 1);
        x[4 * k + 2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(ck, s, 2);
        x[4 * k + 3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(ck, s, 3);
      }
      store_held(out + 16 * i, x, there && byte == 255);
    }
  }
}

static bool aligned16(const void* p) { return ((uintptr_t)p & 15) == 0; }

}  // namespace fdllm

using namespace fdllm;

extern "C" {

fdllm_status fdllm_cache_tile_bytes(int D, size_t* bytes) {
  if (!bytes) return FDLLM_ERR_INVALID_ARG;
  if (D < 32 || D > kRopeMaxD || D % 32) return FDLLM_ERR_SIZE;
  *bytes = (size_t)tile_bytes(D);
  return FDLLM_OK;
}

fdllm_status fdllm_qk_norm_rope(const void* q, int64_t q_stride, const void* k, int64_t k_stride, const void* v,
                                int64_t v_stride, fdllm_dtype dtype, int T, int H, int Hk, int D,
                                const float* q_weight, const float* k_weight, float eps,
                                const int32_t* positions, const float* cos_sin, int n_pos, int rot,
                                int interleaved, void* q_out, void* k_out, uint8_t* cache, int n_pages,
                                const int32_t* slots, fdllm_stream stream) {
  if (dtype != FDLLM_BF16 && dtype != FDLLM_F32) return FDLLM_ERR_UNSUPPORTED_DTYPE;
  if (T < 0 || H < 1 || Hk < 1 || n_pages < 0 || n_pos < 0) return FDLLM_ERR_INVALID_ARG;
  if (D < 32 || D > kRopeMaxD || D % 32 || rot < 0 || rot > D || rot % 16) return FDLLM_ERR_SIZE;
  // a launch has at most 2^32 threads along the tokens, 65535 workgroups along the heads
  if (H > (1 << 14) || Hk > (1 << 14) || T > (1 << 27) || n_pages > INT32_MAX / kPage) return FDLLM_ERR_SIZE;
  if (!(eps >= 0.0f)) return FDLLM_ERR_INVALID_ARG;
  if (T == 0) return FDLLM_OK;
  if (!q || !k || !positions || !q_out || (rot > 0 && !cos_sin) || (!k_out && !cache)) return FDLLM_ERR_INVALID_ARG;
  if (cache && (!v || !slots)) return FDLLM_ERR_INVALID_ARG;
  const int64_t per16 = dtype == FDLLM_BF16 ? 8 : 4;   // elements in 16 bytes
  if (q_stride < (int64_t)H * D || k_stride < (int64_t)Hk * D || q_stride % per16 || k_stride % per16)
    return FDLLM_ERR_INVALID_ARG;
  if (cache && (v_stride < (int64_t)Hk * D || v_stride % per16)) return FDLLM_ERR_INVALID_ARG;
  for (const void* p : {q, k, cache ? v : nullptr, (const void*)q_weight, (const void*)k_weight, (const void*)cos_sin,
                        (const void*)q_out, (const void*)k_out, (const void*)cache})
    if (!aligned16(p)) return FDLLM_ERR_INVALID_ARG;

  RopeArgs a{q, k, v, q_stride, k_stride, v_stride, T, H, Hk, D, q_weight, k_weight, eps, positions, cos_sin,
             n_pos, rot, q_out, k_out, cache, n_pages, slots, 1};
  const int tokens = kRopeThreads / (D <= 128 ? 8 : 16);
  const int heads = H + Hk + (cache ? Hk : 0);
  const long long chunks = (T + tokens - 1) / tokens;
  // A workgroup takes several heads, which saves loads of angles and weights and has
  // the next head's row under way, as long as 2048 workgroups are left.  32 + 8 + 8
  // heads of 128 in bfloat16, with 1, 2, 4 and 8 heads a workgroup: 256 tokens 4.0,
  // 4.9, 7.2 and 11.8 us (this rule: 1), 4096 tokens 21.4, 19.0, 18.5 and 19.8 (2),
  // 8192 39.0, 33.4, 32.2 and 34.0 (4), 14088 109, 90, 84 and 76 (8).
  while (a.heads_per_wg < 8 && chunks * ((heads + 2 * a.heads_per_wg - 1) / (2 * a.heads_per_wg)) >= 2048)
    a.heads_per_wg *= 2;
  const dim3 grid((unsigned)chunks, (unsigned)((heads + a.heads_per_wg - 1) / a.heads_per_wg));
  hipStream_t st = (hipStream_t)stream;
  if (dtype == FDLLM_BF16) {
    if (interleaved) hipLaunchKernelGGL((k_rope<__bf16, true>), grid, dim3(kRopeThreads), 0, st, a);
    else hipLaunchKernelGGL((k_rope<__bf16, false>), grid, dim3(kRopeThreads), 0, st, a);
  } else {
    if (interleaved) hipLaunchKernelGGL((k_rope<float, true>), grid, dim3(kRopeThreads), 0, st, a);
    else hipLaunchKernelGGL((k_rope<float, false>), grid, dim3(kRopeThreads), 0, st, a);
  }
  return hipGetLastError() == hipSuccess ? FDLLM_OK : FDLLM_ERR_HIP;
}

fdllm_status fdllm_cache_read(const uint8_t* cache, int n_pages, int Hk, int D, const int32_t* slots, int T,
                              fdllm_cache_out out_type, void* k_out, void* v_out, fdllm_stream stream) {
  if (out_type != FDLLM_OUT_BF16 && out_type != FDLLM_OUT_E5M2) return FDLLM_ERR_UNSUPPORTED_DTYPE;
  if (T < 0 || Hk < 1 || n_pages < 0) return FDLLM_ERR_INVALID_ARG;
  if (D < 32 || D > kRopeMaxD || D % 32 || Hk > (1 << 15)) return FDLLM_ERR_SIZE;
  if (T == 0) return FDLLM_OK;
  if (!cache || n_pages < 1 || !slots || (!k_out && !v_out)) return FDLLM_ERR_INVALID_ARG;
  if (!aligned16(cache) || !aligned16(k_out) || !aligned16(v_out)) return FDLLM_ERR_INVALID_ARG;
  const long long n = (long long)T * Hk * (D / 16);
  const long long blocks = (n + 255) / 256;
  const dim3 grid((unsigned)(blocks < 8192 ? blocks : 8192));
  hipStream_t st = (hipStream_t)stream;
  if (out_type == FDLLM_OUT_BF16)
    hipLaunchKernelGGL(k_cache_read<__bf16>, grid, dim3(256), 0, st, cache, n_pages, Hk, D, slots, n, (__bf16*)k_out,
                       (__bf16*)v_out);
  else
    hipLaunchKernelGGL(k_cache_read<uint8_t>, grid, dim3(256), 0, st, cache, n_pages, Hk, D, slots, n,
                       (uint8_t*)k_out, (uint8_t*)v_out);
  return hipGetLastError() == hipSuccess ? FDLLM_OK : FDLLM_ERR_HIP;
}

}  // extern "C"
