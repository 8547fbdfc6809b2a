// attn_common.h -- what the attention kernels share: the layout of the 4-bit
// cache, the rule of which keys a query sees, matrix-core operand types and
// the wave-level pieces of an online softmax over transposed scores.
// Internal to libfdllm.so.
#ifndef FDLLM_ATTN_COMMON_H
#define FDLLM_ATTN_COMMON_H

#include <hip/hip_runtime.h>

#include <stdint.h>

#include "attn_work.h"
#include "fdllm.h"
#include "pass_common.h"

namespace fdllm {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short i16x2 __attribute__((ext_vector_type(2)));
typedef short i16x4 __attribute__((ext_vector_type(4)));
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

// ---------------------------------------------------------------------------
// the 4-bit cache: [n_pages][kv heads] tiles of one page (64 tokens) of one
// head: key codes, value codes, key scales, value scales (fdllm.h).
// ---------------------------------------------------------------------------
constexpr int kPage = FDLLM_CACHE_PAGE;
constexpr int kGroup = 32;               // elements that share a scale
constexpr int kCodeBytes = kGroup / 2;   // a group of one token
constexpr int kUnitScale = 127;          // scale byte of 2^0

__host__ __device__ constexpr int scale_stride(int D) { return (D / kGroup + 3) / 4 * 4; }
__host__ __device__ constexpr int codes_bytes(int D) { return kPage * D / 2; }
__host__ __device__ constexpr int scales_bytes(int D) { return kPage * scale_stride(D); }
__host__ __device__ constexpr int tile_bytes(int D) { return 2 * (codes_bytes(D) + scales_bytes(D)); }
__host__ __device__ constexpr int k_scales_at(int D) { return 2 * codes_bytes(D); }
__host__ __device__ constexpr int v_scales_at(int D) { return 2 * codes_bytes(D) + scales_bytes(D); }

// 2^(byte - 127) as a float (byte 0, which no writer leaves, gives 0).
__device__ __forceinline__ float scale_of(uint32_t byte) { return __int_as_float((int)(byte << 23)); }

// ---------------------------------------------------------------------------
// which keys a query sees: j < min(len, end(p)), end(p) = (floor(p / blk) + 1) blk
// (blk 0: no mask).  p may be negative (more queries than keys): nothing then.
// ---------------------------------------------------------------------------
__device__ __forceinline__ int visible_end(int p, int blk, int len) {
  if (blk == 0) return len;
  if (p < 0) return 0;
  const long long e = ((long long)(p / blk) + 1) * blk;
  return e < len ? (int)e : len;
}

// ---------------------------------------------------------------------------
// wave-level pieces.  Scores are formed transposed, S^T = K Q^T: a lane holds
// one query row (its column) and the keys lie along its registers, so the
// softmax runs inside the lane but for the last exchange between the lanes
// that share a row, and exp(S^T) is the second product's operand as it stands.
// ---------------------------------------------------------------------------
__device__ __forceinline__ float max_halves(float v) {   // lanes l and l ^ 32
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float sum_halves(float v) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
__device__ __forceinline__ float max_quarters(float v) {   // lanes l, l ^ 16, l ^ 32, l ^ 48
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return max_halves(fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1])));
}
__device__ __forceinline__ float sum_quarters(float v) {
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return sum_halves(__uint_as_float(r[0]) + __uint_as_float(r[1]));
}
template <int MT>
__device__ __forceinline__ float max_row(float v) {
  if constexpr (MT == 32) return max_halves(v);
  else return max_quarters(v);
}
template <int MT>
__device__ __forceinline__ float sum_row(float v) {
  if constexpr (MT == 32) return sum_halves(v);
  else return sum_quarters(v);
}

// The sum over a wave, in a scalar register.
__device__ __forceinline__ int wave_sum(int v) {
  v += partner_i32<0>(v);
  v += partner_i32<1>(v);
  v += partner_i32<2>(v);
  v += partner_i32<3>(v);
  v += partner_i32<4>(v);
  return __builtin_amdgcn_readlane(v, 0) + __builtin_amdgcn_readlane(v, 32);
}

__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
  bf16x2 p;
  p[0] = (__bf16)a;
  p[1] = (__bf16)b;
  return __builtin_bit_cast(uint32_t, p);
}

// Four rows by sixteen columns of 16-bit values in LDS, read transposed: each
// group of 16 lanes gives the address of (row i / 4, columns 4 (i % 4)..) and
// lane i receives column i of the four rows.
__device__ __forceinline__ i16x4 read_transposed(const uint8_t* p) {
  return __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) i16x4*)p);
}

// ---------------------------------------------------------------------------
// outputs.  A wave's tile of MT rows by D lies transposed in its registers: lane
// (col, part) holds row col, and quad q of its registers the four elements from
// quad_element on.  Partial sums are stored as they lie, a quad of all lanes at
// a time: [tile][quads][64 lanes][4].
// ---------------------------------------------------------------------------
template <int MT>
__device__ __forceinline__ int quad_element(int q, int part) {
  return MT == 32 ? (q / 4) * 32 + (q % 4) * 8 + 4 * part : q * 16 + 4 * part;
}
__host__ __device__ constexpr int quads_of(int MT, int NG) { return MT == 32 ? 4 * NG : 2 * NG; }

// Rows of bfloat16 in LDS on their way out, 16-byte pieces exchanged by the
// row's number, so that 16 lanes that hold an element of 16 rows meet all banks.
template <int NG>
struct OutRows {
  static constexpr int RowBytes = NG == 2 ? 128 : 256;
  __device__ static int at(int row, int d) {
    const int swap = NG == 2 ? row / 2 % 8 : row % 16;
    return row * RowBytes + 16 * ((d / 8) ^ swap) + 2 * (d % 8);
  }
};

constexpr float kLn2 = 0.69314718055994530942f;

// The reciprocal and the logarithm of a row's sum l of weights 2^(x - ref): 0 and
// -inf where no key was seen.  Told by the bits, since the build leaves NaN out of
// comparisons' account: a row with a NaN gets NaN, not what stands for no keys.
__device__ __forceinline__ float inverse_sum(float l) { return __float_as_uint(l) ? 1.0f / l : 0.0f; }
__device__ __forceinline__ float log_sum(float ref, float l) {
  return __float_as_uint(l) ? (ref + __builtin_amdgcn_logf(l)) * kLn2 : kNegInf;
}

}  // namespace fdllm

#endif  // FDLLM_ATTN_COMMON_H
