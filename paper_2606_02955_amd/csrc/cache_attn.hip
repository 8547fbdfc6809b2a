// cache_attn.hip -- attention of a few query tokens per sequence over the
// 4-bit cache on gfx950.
//
//   s_ij = scale q_i . k_j,  m_i = max_j s_ij,  l_i = sum_j exp(s_ij - m_i),
//   out_i = sum_j exp(s_ij - m_i) v_j / l_i,    lse_i = m_i + log l_i
//
// over the keys j that query i sees, in one pass over the cache with running
// m and l.  The query tokens of a sequence times the query heads that share a
// key head are the rows of one product; a (sequence, key head, group of rows)
// is an item, a page of its cache a unit of work.
//
// K: the scaled matrix instruction takes the cache's 4-bit codes and their
// scales as they lie in memory; no key is ever unpacked.  Its other operand
// must have at most 8 bits, so a query is the sum of two E4M3 numbers: a
// bfloat16's 8 significant bits are 4 and 4 of theirs, exactly, down to 2^-16
// of the row's largest element.
// V: unpacked to bfloat16 (exact: a code has two significant bits, its scale
// none) into LDS and read back transposed as the second product's operand.
#include <hip/hip_runtime.h>

#include <stdint.h>

#include <type_traits>

#include "attn_common.h"
#include "fdllm.h"

namespace fdllm {

constexpr int kCaThreads = 256;
constexpr int kCaWaves = kCaThreads / kWave;
constexpr int kHalf = kPage / 2;            // keys whose values are in LDS at a time
constexpr int kCaRowFloats = 2;             // m and l beside a row's partial sums

struct CacheAttnArgs {
  const uint16_t* q;
  long long q_stride;
  int T;
  const uint8_t* cache;
  int n_pages;
  const int32_t* table;
  int table_w;
  const int32_t* kv_len;
  const int32_t* cu_q;
  const int32_t* q_start;
  int B, H, Hk, R, max_q, blk;
  float c;                    // scale * log2 e
  uint16_t* out;
  float* lse;
  float* part;                // [workgroups][2][rows][D + 2]
};

// A sequence as the plan sees it: its query rows, pages and groups of rows.
struct Seq {
  int first, n, len, groups, pages;
};

template <int Rows>
__device__ __forceinline__ Seq sequence(const CacheAttnArgs& a, int b) {
  Seq s;
  s.n = packed_rows(a.cu_q, b, a.T, a.max_q, &s.first);
  const int most = a.table_w * kPage;
  s.len = min(max(a.kv_len[b], 0), most);
  s.groups = (s.n * a.R + Rows - 1) / Rows;
  s.pages = max(1, (s.len + kPage - 1) / kPage);   // one at least: a row without keys gets its zeros
  return s;
}

// Units of all sequences, and the sequence and offset at which unit `u` lies.
template <int Rows>
__device__ __forceinline__ int total_units(const CacheAttnArgs& a, int* s_sum) {
  int n = 0;
  for (int b = threadIdx.x; b < a.B; b += kCaThreads) {
    const Seq s = sequence<Rows>(a, b);
    n += s.groups * s.pages;
  }
#pragma unroll
  for (int x = 1; x < kWave; x <<= 1) n += __shfl_xor(n, x);
  __syncthreads();
  if (threadIdx.x % kWave == 0) s_sum[threadIdx.x / kWave] = n;
  __syncthreads();
  n = 0;
#pragma unroll
  for (int w = 0; w < kCaWaves; ++w) n += s_sum[w];
  return n * a.Hk;
}

// Units before sequence b0 (all of a.B: total_units).
template <int Rows>
__device__ __forceinline__ int units_before(const CacheAttnArgs& a, int b0, int* s_sum) {
  CacheAttnArgs c = a;
  c.B = b0;
  return total_units<Rows>(c, s_sum);
}

// First unit of workgroup g's share.
__device__ __forceinline__ int share_begin(int g, int groups, int units) {
  return (int)((long long)g * units / groups);
}
// The workgroup whose share holds unit u.
__device__ __forceinline__ int share_of(int u, int groups, int units) {
  int g = (int)(((long long)u * groups) / units);
  while (g + 1 < groups && share_begin(g + 1, groups, units) <= u) ++g;
  while (share_begin(g, groups, units) > u) --g;
  return g;
}

// --- queries as pairs of E4M3 ---------------------------------------------
struct PairScale {
  float mul;        // 2^-e: the row's largest magnitude comes to lie in (128, 256]
  int hi, lo;       // scale bytes of the two parts
};

__device__ __forceinline__ PairScale pair_scale(float top) {
  int e = (int)(__float_as_uint(top) >> 23) - 127 - 7;
  e = e < -100 ? -100 : e;
  PairScale p;
  p.mul = scale_of((uint32_t)(127 - e));
  p.hi = 127 + e;
  p.lo = 127 + e - 4;
  return p;
}

// Four elements: hi = E4M3(x), lo = E4M3(16 (x - hi)).
__device__ __forceinline__ void split4(const float* x, int* hi, int* lo) {
  int h = 0, l = 0;
  h = __builtin_amdgcn_cvt_pk_fp8_f32(x[0], x[1], h, false);
  h = __builtin_amdgcn_cvt_pk_fp8_f32(x[2], x[3], h, true);
  const auto a = __builtin_amdgcn_cvt_pk_f32_fp8(h, false);
  const auto b = __builtin_amdgcn_cvt_pk_f32_fp8(h, true);
  l = __builtin_amdgcn_cvt_pk_fp8_f32((x[0] - a[0]) * 16.0f, (x[1] - a[1]) * 16.0f, l, false);
  l = __builtin_amdgcn_cvt_pk_fp8_f32((x[2] - b[0]) * 16.0f, (x[3] - b[1]) * 16.0f, l, true);
  *hi = h;
  *lo = l;
}

// ---------------------------------------------------------------------------
// NG: groups of 32 elements of a head.  MT: rows of a wave's tile, 16 or 32.
// WR: waves that hold different rows of an item; the 4 / WR sets of them take
// different pages.
// ---------------------------------------------------------------------------
template <int NG, int MT, int WR>
struct CaShape {
  static constexpr int D = NG * kGroup;
  static constexpr int WK = kCaWaves / WR;
  static constexpr int Rows = MT * WR;
  static constexpr int RowBytes = 2 * D + 32;              // of a key's values in LDS
  static constexpr int HalfBytes = kHalf * RowBytes;
  static constexpr int Buffers = WR > 1 ? 2 : 1;
  static constexpr int ValueBytes = WK * Buffers * HalfBytes;
  static constexpr int JoinBytes = WK > 1 ? (WK / 2) * Rows * (D + 4) * 4 : 0;
  static constexpr int LdsBytes = ValueBytes > JoinBytes ? ValueBytes : JoinBytes;
  static constexpr int DT = MT == 32 ? NG : 2 * NG;        // tiles of D of the second product
  static constexpr int OR = MT == 32 ? 16 : 4;             // registers of one
  static constexpr int QS = MT == 32 ? (NG + 1) / 2 : 1;   // steps of the first product
};

template <int NG, int MT, int WR>
__global__ void __launch_bounds__(kCaThreads, 2)
k_cache_attn(const CacheAttnArgs a) {
  typedef CaShape<NG, MT, WR> S;
  constexpr int D = S::D;
  constexpr int SPT = kPage / MT;     // subtiles of MT keys in a page
  typedef typename std::conditional<MT == 32, f32x16, f32x4>::type Acc;
  __shared__ __align__(16) uint8_t s_mem[S::LdsBytes];
  __shared__ int s_sum[kCaWaves];
  __shared__ float s_ml[kCaWaves][MT][2];

  const int tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave;
  const int wr = wave % WR, wk = wave / WR;   // its rows, its pages
  const int col = lane % MT, part = lane / MT;

  // this workgroup's share of the units
  const int units = total_units<S::Rows>(a, s_sum);
  if (units == 0) return;
  const int u_begin = share_begin(blockIdx.x, gridDim.x, units);
  const int u_end = share_begin(blockIdx.x + 1, gridDim.x, units);
  if (u_begin >= u_end) return;

  // the sequence of its first unit: 256 at a time, then by steps
  int b = 0, before = 0;
  for (int chunk = kCaThreads; chunk < a.B; chunk += kCaThreads) {
    const int n = units_before<S::Rows>(a, chunk, s_sum);
    if (n > u_begin) break;
    b = chunk;
    before = n;
  }
  Seq seq = sequence<S::Rows>(a, b);
  while (before + seq.groups * seq.pages * a.Hk <= u_begin) {
    before += seq.groups * seq.pages * a.Hk;
    seq = sequence<S::Rows>(a, ++b);
  }

  int u = u_begin;
  int slot = 0;                       // of the next partial result
  while (u < u_end) {
    while (u >= before + seq.groups * seq.pages * a.Hk) {
      before += seq.groups * seq.pages * a.Hk;
      seq = sequence<S::Rows>(a, ++b);
    }
    const int item = (u - before) / seq.pages;
    const int page0 = (u - before) % seq.pages;
    const int page1 = min(seq.pages, page0 + (u_end - u));
    const int h = item % a.Hk, group = item / a.Hk;
    u += page1 - page0;

    // ---- the item's rows ----
    const int r = (group * WR + wr) * MT + col;             // row of this lane
    const bool row_ok = r < seq.n * a.R;
    const int tok = row_ok ? r / a.R : 0, head = h * a.R + (row_ok ? r % a.R : 0);
    const int start = a.q_start ? a.q_start[b] : seq.len - seq.n;
    const int end = row_ok ? visible_end(start + tok, a.blk, seq.len) : 0;
    i32x8 qh[S::QS], ql[S::QS];
    PairScale ps;
    {
      const uint16_t* qrow = a.q + (size_t)(seq.first + tok) * a.q_stride + (size_t)head * D;
      float top = 0.0f;
      bf16x8 x[S::QS][4];
#pragma unroll
      for (int s = 0; s < S::QS; ++s)
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          // the 8-bit operand's element order: 16 from each half of the step
          const int span = MT == 32 ? 64 : 128;
          const int d = s * span + (k / 2) * (span / 2) + part * 16 + (k % 2) * 8;
          bf16x8 v = {};
          if (row_ok && d < D) v = *(const bf16x8*)(qrow + d);
          x[s][k] = v;
#pragma unroll
          for (int i = 0; i < 8; ++i) top = fmaxf(top, __builtin_fabsf((float)v[i]));
        }
      top = max_row<MT>(top);
      ps = pair_scale(top);
#pragma unroll
      for (int s = 0; s < S::QS; ++s)
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          float y[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) y[i] = (float)x[s][k / 2][(k % 2) * 4 + i] * ps.mul;
          int hi, lo;
          split4(y, &hi, &lo);
          qh[s][k] = hi;
          ql[s][k] = lo;
        }
    }

    Acc o[S::DT];
#pragma unroll
    for (int t = 0; t < S::DT; ++t) o[t] = Acc{};
    float m = kNegInf, l = 0.0f;

    // ---- the pages ----
    int buf = 0;
    for (int pg = page0 + wk;; pg += S::WK) {
      // sets of waves without a page left go along while others' barriers run
      const bool active = pg < page1;
      if (WR == 1 ? !active : pg - wk >= page1) break;
      const int32_t page = active && pg * kPage < seq.len ? a.table[(size_t)b * a.table_w + pg] : -1;
      const bool there = page >= 0 && page < a.n_pages;
      const uint8_t* tile = a.cache + ((size_t)(there ? page : 0) * a.Hk + h) * tile_bytes(D);
      const int base = pg * kPage;
      const int limit = there ? seq.len - base : 0;          // keys of the page that exist

      // scores
      Acc sc[SPT];
#pragma unroll
      for (int s = 0; s < SPT; ++s) {
        const int key = s * MT + col;
        uint32_t ks = *(const uint32_t*)(tile + k_scales_at(D) + key * scale_stride(D));
        if (NG == 3) ks = (ks & 0x00ffffffu) | 0x7f000000u;
        if (NG == 2) ks = (ks & 0x0000ffffu) | 0x7f7f0000u;
        const int kb = (int)(ks >> (8 * part));
        sc[s] = Acc{};
#pragma unroll
        for (int t = 0; t < S::QS; ++t) {
          const int g = MT == 32 ? 2 * t + part : part;
          i32x8 k = {};
          if (g < NG) {
            const u32x4 c = *(const u32x4*)(tile + (g * kPage + key) * kCodeBytes);
#pragma unroll
            for (int i = 0; i < 4; ++i) k[i] = (int)c[i];
          }
          if constexpr (MT == 32) {
            // byte 0 of the shifted scales is group `part`, byte 2 group 2 + part
            if (t == 0) {
              sc[s] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(k, qh[t], sc[s], 4, 0, 0, kb, 0, ps.hi);
              sc[s] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(k, ql[t], sc[s], 4, 0, 0, kb, 0, ps.lo);
            } else {
              sc[s] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(k, qh[t], sc[s], 4, 0, 2, kb, 0, ps.hi);
              sc[s] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(k, ql[t], sc[s], 4, 0, 2, kb, 0, ps.lo);
            }
          } else {
            sc[s] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(k, qh[t], sc[s], 4, 0, 0, kb, 0, ps.hi);
            sc[s] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(k, ql[t], sc[s], 4, 0, 0, kb, 0, ps.lo);
          }
        }
      }
      // keys that a row does not see
      const int seen = there ? end - base : 0;
#pragma unroll
      for (int s = 0; s < SPT; ++s)
#pragma unroll
        for (int i = 0; i < S::OR; ++i) {
          const int key = s * MT + (MT == 32 ? i % 4 + 8 * (i / 4) + 4 * part : 4 * part + i);
          sc[s][i] = key < seen ? sc[s][i] : kNegInf;
        }
      // running maximum and sum
      float top = kNegInf;
#pragma unroll
      for (int s = 0; s < SPT; ++s)
#pragma unroll
        for (int i = 0; i < S::OR; ++i) top = fmaxf(top, sc[s][i]);
      top = max_row<MT>(top);
      const float mn = fmaxf(m, top);
      const float ref = fmaxf(mn * a.c, kRefFloor);          // finite while nothing was seen
      const float alpha = __builtin_amdgcn_exp2f(m * a.c - ref);
      m = mn;
      float sum = 0.0f;
      uint32_t p[SPT][S::OR / 2];
#pragma unroll
      for (int s = 0; s < SPT; ++s)
#pragma unroll
        for (int i = 0; i < S::OR; i += 2) {
          const float x = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[s][i], a.c, -ref));
          const float y = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[s][i + 1], a.c, -ref));
          sum += x + y;
          p[s][i / 2] = pack_bf16(x, y);   // weights in (0, 1] to 8 bits, as the values they meet
        }
      l = l * alpha + sum;
#pragma unroll
      for (int t = 0; t < S::DT; ++t)
#pragma unroll
        for (int i = 0; i < S::OR; ++i) o[t][i] *= alpha;

      // values, half a page at a time
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        uint8_t* lds = s_mem + (wk * S::Buffers + buf) * S::HalfBytes;
        if (S::Buffers > 1) buf ^= 1;
        // unpack: 32 keys x NG groups, a lane each
        for (int w = wr * kWave + lane; w < kHalf * NG; w += WR * kWave) {
          const int key = w % kHalf, g = w / kHalf;
          const int kp = half * kHalf + key;
          u32x4 c = *(const u32x4*)(tile + codes_bytes(D) + (g * kPage + kp) * kCodeBytes);
          const uint32_t byte = tile[v_scales_at(D) + kp * scale_stride(D) + g];
          const bool ok = kp < limit;
          const float sv = scale_of(ok ? byte : kUnitScale);
          u32x4* dst = (u32x4*)(lds + key * S::RowBytes + g * 64);
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const uint32_t ci = ok ? c[i] : 0u;
            u32x4 y;
            y[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(ci, sv, 0));
            y[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(ci, sv, 1));
            y[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(ci, sv, 2));
            y[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(ci, sv, 3));
            dst[i] = y;
          }
        }
        if (WR > 1) __syncthreads();
        else __builtin_amdgcn_wave_barrier();
        // a group of 16 lanes reads four keys by 16 elements, transposed
        const int quad = (lane % 16) / 4, four = lane % 4;
        if constexpr (MT == 32) {
          const uint8_t* base_p = lds + (4 * part + quad) * S::RowBytes + (16 * ((lane / 16) % 2) + 4 * four) * 2;
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            u32x4 pk;
#pragma unroll
            for (int i = 0; i < 4; ++i) pk[i] = p[half][4 * k + i];
            const bf16x8 pf = __builtin_bit_cast(bf16x8, pk);
#pragma unroll
            for (int t = 0; t < S::DT; ++t) {
              const i16x4 v0 = read_transposed(base_p + (16 * k) * S::RowBytes + t * 64);
              const i16x4 v1 = read_transposed(base_p + (16 * k + 8) * S::RowBytes + t * 64);
              const bf16x8 vf = __builtin_bit_cast(bf16x8, __builtin_shufflevector(v0, v1, 0, 1, 2, 3, 4, 5, 6, 7));
              o[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf, pf, o[t], 0, 0, 0);
            }
          }
        } else {
          const uint8_t* base_p = lds + (4 * part + quad) * S::RowBytes + (4 * four) * 2;
          u32x4 pk;
          pk[0] = p[2 * half][0], pk[1] = p[2 * half][1], pk[2] = p[2 * half + 1][0], pk[3] = p[2 * half + 1][1];
          const bf16x8 pf = __builtin_bit_cast(bf16x8, pk);
#pragma unroll
          for (int t = 0; t < S::DT; ++t) {
            const i16x4 v0 = read_transposed(base_p + t * 32);
            const i16x4 v1 = read_transposed(base_p + 16 * S::RowBytes + t * 32);
            const bf16x8 vf = __builtin_bit_cast(bf16x8, __builtin_shufflevector(v0, v1, 0, 1, 2, 3, 4, 5, 6, 7));
            o[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pf, o[t], 0, 0, 0);
          }
        }
        __builtin_amdgcn_wave_barrier();
      }
    }
    l = sum_row<MT>(l);

    // ---- the sets of waves join, two by two ----
    if constexpr (S::WK > 1) {
#pragma unroll
      for (int n = S::WK / 2; n >= 1; n /= 2) {
        __syncthreads();
        float* mem = (float*)s_mem;
        if (wk >= n && wk < 2 * n) {
          float* mine = mem + ((wk - n) * WR + wr) * MT * (D + 4);
          if (part == 0) s_ml[wave][col][0] = m, s_ml[wave][col][1] = l;
#pragma unroll
          for (int t = 0; t < S::DT; ++t)
#pragma unroll
            for (int i = 0; i < S::OR; i += 4) {
              const int d = MT == 32 ? t * 32 + 2 * i + 4 * part : t * 16 + 4 * part;
              *(f32x4*)(mine + col * (D + 4) + d) = f32x4{o[t][i], o[t][i + 1], o[t][i + 2], o[t][i + 3]};
            }
        }
        __syncthreads();
        if (wk < n) {
          const int other = (wk + n) * WR + wr;
          const float* theirs = mem + (wk * WR + wr) * MT * (D + 4);
          const float m2 = s_ml[other][col][0], l2 = s_ml[other][col][1];
          const float mn = fmaxf(m, m2);
          const float ref = fmaxf(mn * a.c, kRefFloor);
          const float f1 = __builtin_amdgcn_exp2f(m * a.c - ref), f2 = __builtin_amdgcn_exp2f(m2 * a.c - ref);
          m = mn;
          l = l * f1 + l2 * f2;
#pragma unroll
          for (int t = 0; t < S::DT; ++t)
#pragma unroll
            for (int i = 0; i < S::OR; i += 4) {
              const int d = MT == 32 ? t * 32 + 2 * i + 4 * part : t * 16 + 4 * part;
              const f32x4 x = *(const f32x4*)(theirs + col * (D + 4) + d);
#pragma unroll
              for (int k = 0; k < 4; ++k) o[t][i + k] = o[t][i + k] * f1 + x[k] * f2;
            }
        }
      }
      __syncthreads();
    }

    // ---- results: final where the item is whole, a partial sum otherwise ----
    if (wk == 0) {
      if (page0 == 0 && page1 == seq.pages) {
        if (row_ok) {
          const float inv = l > 0.0f ? 1.0f / l : 0.0f;
          const size_t at = (size_t)(seq.first + tok) * a.H + head;
#pragma unroll
          for (int t = 0; t < S::DT; ++t)
#pragma unroll
            for (int i = 0; i < S::OR; i += 4) {
              const int d = MT == 32 ? t * 32 + 2 * i + 4 * part : t * 16 + 4 * part;
              *(u32x2*)(a.out + at * D + d) = u32x2{pack_bf16(o[t][i] * inv, o[t][i + 1] * inv),
                                                    pack_bf16(o[t][i + 2] * inv, o[t][i + 3] * inv)};
            }
          if (a.lse && part == 0)
            a.lse[at] = l > 0.0f ? (m * a.c + __builtin_amdgcn_logf(l)) * kLn2 : kNegInf;
        }
      } else {
        float* mine = a.part + (((size_t)blockIdx.x * 2 + slot) * S::Rows + wr * MT + col) * (D + kCaRowFloats);
#pragma unroll
        for (int t = 0; t < S::DT; ++t)
#pragma unroll
          for (int i = 0; i < S::OR; i += 2) {
            const int d = MT == 32 ? t * 32 + i % 4 + 8 * (i / 4) + 4 * part : t * 16 + 4 * part + i;
            *(float2*)(mine + d) = float2{o[t][i], o[t][i + 1]};
          }
        if (part == 0) *(float2*)(mine + D) = float2{m, l};
      }
    }
    slot = 1;
  }
}

// Joins the partial results of an item that several workgroups share, in the
// order of its pages.  One workgroup per (item of the widest sequence).
template <int NG, int Rows>
__global__ void __launch_bounds__(kCaThreads)
k_cache_join(const CacheAttnArgs a, int wgs) {
  constexpr int D = NG * kGroup;
  __shared__ int s_sum[kCaWaves];
  const int b = blockIdx.y;
  const Seq seq = sequence<Rows>(a, b);
  if ((int)blockIdx.x >= seq.groups * a.Hk) return;
  const int units = total_units<Rows>(a, s_sum);
  const int u0 = units_before<Rows>(a, b, s_sum) + (int)blockIdx.x * seq.pages;
  const int g0 = share_of(u0, wgs, units), g1 = share_of(u0 + seq.pages - 1, wgs, units);
  if (g0 == g1) return;
  const int h = blockIdx.x % a.Hk, group = blockIdx.x / a.Hk;
  // rows by quarter waves: 16 lanes of NG * 2 elements
  const int lane = threadIdx.x % 16;
  for (int x = threadIdx.x / 16; x < Rows; x += kCaThreads / 16) {
    const int r = group * Rows + x;
    if (r >= seq.n * a.R) break;
    float acc[2 * NG];
#pragma unroll
    for (int i = 0; i < 2 * NG; ++i) acc[i] = 0.0f;
    float m = kNegInf, l = 0.0f;
    for (int g = g0; g <= g1; ++g) {
      const int begin = share_begin(g, wgs, units);
      if (begin == share_begin(g + 1, wgs, units)) continue;
      // an item that begins inside a share is that workgroup's second result
      const int slot = begin < u0 ? 1 : 0;
      const float* p = a.part + (((size_t)g * 2 + slot) * Rows + x) * (D + kCaRowFloats);
      const float m2 = p[D], l2 = p[D + 1];
      const float mn = fmaxf(m, m2);
      const float ref = fmaxf(mn * a.c, kRefFloor);
      const float f1 = __builtin_amdgcn_exp2f(m * a.c - ref), f2 = __builtin_amdgcn_exp2f(m2 * a.c - ref);
      m = mn;
      l = l * f1 + l2 * f2;
#pragma unroll
      for (int i = 0; i < NG; ++i) {
        const float2 v = *(const float2*)(p + 32 * i + 2 * lane);
        acc[2 * i] = acc[2 * i] * f1 + v.x * f2;
        acc[2 * i + 1] = acc[2 * i + 1] * f1 + v.y * f2;
      }
    }
    const int tok = r / a.R, head = h * a.R + r % a.R;
    const size_t at = (size_t)(seq.first + tok) * a.H + head;
    const float inv = l > 0.0f ? 1.0f / l : 0.0f;
#pragma unroll
    for (int i = 0; i < NG; ++i)
      *(uint32_t*)(a.out + at * D + 32 * i + 2 * lane) = pack_bf16(acc[2 * i] * inv, acc[2 * i + 1] * inv);
    if (a.lse && lane == 0) a.lse[at] = l > 0.0f ? (m * a.c + __builtin_amdgcn_logf(l)) * kLn2 : kNegInf;
  }
}

// ---------------------------------------------------------------------------
// host side
// ---------------------------------------------------------------------------
struct CaPlan {
  int mt, wr;        // variant
  int wgs;           // workgroups
  int items;         // items of a sequence with max_q query tokens
  size_t bytes;      // of partial results
};

static bool ca_sizes_ok(int B, int H, int Hk, int D, int max_q, int table_w, int n_pages) {
  if (D != 64 && D != 96 && D != 128) return false;
  if (H % Hk || H > (1 << 15) || B > 65535) return false;
  if (table_w > INT32_MAX / kPage || n_pages > INT32_MAX / kPage) return false;
  const long long rows = (long long)max_q * (H / Hk);
  const long long groups = (rows + 15) / 16;
  if (rows > (1 << 24) || groups * Hk > INT32_MAX / 2) return false;
  // units of work are counted in 32 bits
  const double units = (double)B * (table_w > 1 ? table_w : 1) * (double)groups * Hk;
  return units < 2.0e9;
}

static CaPlan ca_plan(int B, int H, int Hk, int D, int max_q, int table_w) {
  CaPlan p{};
  const long long rows = (long long)max_q * (H / Hk);
  p.mt = rows <= 16 ? 16 : 32;
  p.wr = rows <= 32 ? 1 : rows <= 64 ? 2 : 4;
  const int per = p.mt * p.wr;
  const long long groups = (rows + per - 1) / per;
  p.items = (int)(groups * Hk);
  const int wk = kCaWaves / p.wr;
  // shares of at least one page for each set of waves, two workgroups a CU
  const long long most = (long long)B * p.items * ((table_w + wk - 1) / wk);
  p.wgs = (int)(most < 512 ? most : 512);
  if (p.wgs < 1) p.wgs = 1;
  p.bytes = (size_t)p.wgs * 2 * per * (D + kCaRowFloats) * sizeof(float);
  return p;
}

template <int NG>
static void ca_launch(const CacheAttnArgs& a, const CaPlan& p, hipStream_t st) {
  const dim3 grid((unsigned)p.wgs), block(kCaThreads), join((unsigned)p.items, (unsigned)a.B);
  if (p.mt == 16) {
    hipLaunchKernelGGL((k_cache_attn<NG, 16, 1>), grid, block, 0, st, a);
    hipLaunchKernelGGL((k_cache_join<NG, 16>), join, block, 0, st, a, p.wgs);
  } else if (p.wr == 1) {
    hipLaunchKernelGGL((k_cache_attn<NG, 32, 1>), grid, block, 0, st, a);
    hipLaunchKernelGGL((k_cache_join<NG, 32>), join, block, 0, st, a, p.wgs);
  } else if (p.wr == 2) {
    hipLaunchKernelGGL((k_cache_attn<NG, 32, 2>), grid, block, 0, st, a);
    hipLaunchKernelGGL((k_cache_join<NG, 64>), join, block, 0, st, a, p.wgs);
  } else {
    hipLaunchKernelGGL((k_cache_attn<NG, 32, 4>), grid, block, 0, st, a);
    hipLaunchKernelGGL((k_cache_join<NG, 128>), join, block, 0, st, a, p.wgs);
  }
}

}  // namespace fdllm

using namespace fdllm;

extern "C" {

fdllm_status fdllm_cache_attention_workspace_size(int B, int H, int Hk, int D, int max_q, int table_width,
                                                  size_t* bytes) {
  if (!bytes || B < 0 || H < 1 || Hk < 1 || max_q < 0 || table_width < 0) return FDLLM_ERR_INVALID_ARG;
  if (!ca_sizes_ok(B, H, Hk, D, max_q, table_width, 0)) return FDLLM_ERR_SIZE;
  *bytes = ca_plan(B, H, Hk, D, max_q, table_width).bytes;
  return FDLLM_OK;
}

fdllm_status fdllm_cache_attention(const void* q, int64_t q_stride, int T, const int32_t* cu_q, int B, int max_q,
                                   int H, int Hk, int D, const uint8_t* cache, int n_pages,
                                   const int32_t* page_table, int table_width, const int32_t* kv_len,
                                   const int32_t* q_start, float scale, int blk, void* out, float* lse,
                                   void* workspace, size_t workspace_bytes, fdllm_stream stream) {
  if (T < 0 || B < 0 || max_q < 0 || H < 1 || Hk < 1 || n_pages < 0 || table_width < 0 || blk < 0)
    return FDLLM_ERR_INVALID_ARG;
  if (!(scale > 0.0f) || scale > 3.0e38f) return FDLLM_ERR_INVALID_ARG;
  if (!ca_sizes_ok(B, H, Hk, D, max_q, table_width, n_pages)) return FDLLM_ERR_SIZE;
  if (T == 0 || B == 0 || max_q == 0) return FDLLM_OK;
  if (!q || !cu_q || !kv_len || !out || (table_width > 0 && !page_table) || !cache || n_pages < 1) return FDLLM_ERR_INVALID_ARG;
  if (q_stride < (int64_t)H * D || q_stride % 8) return FDLLM_ERR_INVALID_ARG;
  for (const void* p : {q, (const void*)cache, (const void*)out, (const void*)workspace})
    if ((uintptr_t)p & 15) return FDLLM_ERR_INVALID_ARG;
  const CaPlan p = ca_plan(B, H, Hk, D, max_q, table_width);
  if (!workspace || workspace_bytes < p.bytes) return FDLLM_ERR_WORKSPACE;
  const CacheAttnArgs a{(const uint16_t*)q, q_stride, T, cache, n_pages, page_table, table_width, kv_len, cu_q,
                        q_start, B, H, Hk, H / Hk, max_q, blk, scale * kLog2e, (uint16_t*)out, lse,
                        (float*)workspace};
  hipStream_t st = (hipStream_t)stream;
  if (D == 64) ca_launch<2>(a, p, st);
  else if (D == 96) ca_launch<3>(a, p, st);
  else ca_launch<4>(a, p, st);
  return hipGetLastError() == hipSuccess ? FDLLM_OK : FDLLM_ERR_HIP;
}

}  // extern "C"
