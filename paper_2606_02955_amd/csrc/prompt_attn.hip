// prompt_attn.hip -- attention of whole packed sequences on gfx950:
// out_i = sum_j softmax_j(scale q_i . k_j) v_j over the keys j that query i
// sees, bfloat16 operands, float32 scores, sums and softmax statistics, in one
// pass over the keys with a running maximum and sum.
//
// The query tokens of a sequence times the query heads that share a key head
// are the rows of one product; a workgroup takes 128 of them, a wave 32, over
// tiles of 64 keys staged in LDS.
#include <hip/hip_runtime.h>

#include <stdint.h>

#include <atomic>

#include "attn_common.h"
#include "fdllm.h"

namespace fdllm {

constexpr int kPaThreads = 256;
constexpr int kPaWaves = kPaThreads / kWave;
constexpr int kPaRows = kPaWaves * 32;
constexpr int kPaKeys = 64;
constexpr int kPaSplitTiles = 4;   // tiles of keys that a part of a split row tile has at least

struct PromptArgs {
  const uint16_t* q;
  const uint16_t* k;
  const uint16_t* v;
  long long q_stride, k_stride, v_stride;
  int T, Tk;
  const int32_t* cu_q;
  const int32_t* cu_k;
  int B, H, Hk, R, max_q, blk;
  float c;
  uint16_t* out;
  float* lse;
  int tiles, splits;   // row tiles of max_q tokens; workgroups for the keys of one
  float* part_ml;      // [(b, h), tile, split][rows][2]: reference and sum of a partial result
  float* part;         // [(b, h), tile, split][rows][D]
};

// A tile of rows: 128 of a sequence's query tokens times the heads of a key head.
struct PaTile {
  int first, firstk, n, len, rows;
  int far;      // the most keys that any row sees
  int parts;    // into which its keys are divided
};

__device__ __forceinline__ PaTile pa_tile(const PromptArgs& a, int b, int tile) {
  PaTile t;
  t.n = packed_rows(a.cu_q, b, a.T, a.max_q, &t.first);
  t.len = packed_rows(a.cu_k, b, a.Tk, INT32_MAX, &t.firstk);
  t.rows = t.n * a.R;
  t.far = 0;
  t.parts = 1;
  if (tile * kPaRows >= t.rows) return t;
  const int last = min(t.rows, (tile + 1) * kPaRows) - 1;
  t.far = visible_end(t.len - t.n + last / a.R, a.blk, t.len);
  const int nt = (t.far + kPaKeys - 1) / kPaKeys;
  t.parts = max(1, min(a.splits, (nt + kPaSplitTiles - 1) / kPaSplitTiles));
  return t;
}

// LDS rows of keys and values, with room behind each so that 16 lanes of a
// 16-byte read (keys), or of a transposed read (values), meet no bank twice.
template <int NG>
struct PaShape {
  static constexpr int D = NG * 32;
  static constexpr int KRow = 2 * D + 16, VRow = 2 * D + 32;
  static constexpr int Buffer = kPaKeys * (KRow + VRow);
  static constexpr int LdsBytes = 2 * Buffer;
  static constexpr int Loads = kPaKeys * D * 2 / 16 / kPaThreads;   // 16-byte loads a thread, per operand
};

template <int NG>
__global__ void __launch_bounds__(kPaThreads, 2)
k_prompt_attn(const PromptArgs a) {
  typedef PaShape<NG> S;
  constexpr int D = S::D;
  extern __shared__ __align__(16) uint8_t s_mem[];

  const int tid = threadIdx.x, lane = tid % kWave, wave = __builtin_amdgcn_readfirstlane(tid / kWave);
  const int col = lane % 32, part = lane / 32;
  const int b = blockIdx.x / a.Hk, h = blockIdx.x % a.Hk;
  const int tile = a.tiles - 1 - blockIdx.y;   // the rows that see most keys first
  const PaTile pt = pa_tile(a, b, tile);
  if (tile * kPaRows >= pt.rows || (int)blockIdx.z >= pt.parts) return;
  const int nt = (pt.far + kPaKeys - 1) / kPaKeys;
  const int t0 = (int)((long long)nt * blockIdx.z / pt.parts), t1 = (int)((long long)nt * (blockIdx.z + 1) / pt.parts);

  const int r = tile * kPaRows + wave * 32 + col;
  const bool row_ok = r < pt.rows;
  const int tok = row_ok ? r / a.R : 0, head = h * a.R + (row_ok ? r % a.R : 0);
  const int end = row_ok ? visible_end(pt.len - pt.n + tok, a.blk, pt.len) : 0;
  int all_see = row_ok ? end : INT32_MAX;   // keys that every row of the wave sees
#pragma unroll
  for (int x = 1; x < 32; x <<= 1) all_see = min(all_see, __shfl_xor(all_see, x));
  all_see = __builtin_amdgcn_readfirstlane(all_see);

  bf16x8 qf[2 * NG];
#pragma unroll
  for (int t = 0; t < 2 * NG; ++t) {
    qf[t] = bf16x8{};
    if (row_ok)
      qf[t] = *(const bf16x8*)(a.q + (size_t)(pt.first + tok) * a.q_stride + (size_t)head * D + 16 * t + 8 * part);
  }
  f32x16 o[NG];
#pragma unroll
  for (int t = 0; t < NG; ++t) o[t] = f32x16{};
  float ref = kRefFloor, l = 0.0f;   // weights are 2^(c s - ref), l their sum

  // staging: registers first, LDS when the other buffer is free
  const uint16_t* kbase = a.k + (size_t)pt.firstk * a.k_stride + (size_t)h * D;
  const uint16_t* vbase = a.v + (size_t)pt.firstk * a.v_stride + (size_t)h * D;
  u32x4 kr[S::Loads], vr[S::Loads];
  const auto fetch = [&](int t) {
    const int base = t * kPaKeys;
#pragma unroll
    for (int i = 0; i < S::Loads; ++i) {
      const int x = i * kPaThreads + tid, key = x / (D / 8), d = x % (D / 8);
      kr[i] = u32x4{};
      vr[i] = u32x4{};
      if (base + key < pt.len) {   // past the end of the sequence: zeros
        kr[i] = *(const u32x4*)(kbase + (size_t)(base + key) * a.k_stride + 8 * d);
        vr[i] = *(const u32x4*)(vbase + (size_t)(base + key) * a.v_stride + 8 * d);
      }
    }
  };
  const auto stage = [&](int buf) {
    uint8_t* sk = s_mem + buf * S::Buffer;
    uint8_t* sv = sk + kPaKeys * S::KRow;
#pragma unroll
    for (int i = 0; i < S::Loads; ++i) {
      const int x = i * kPaThreads + tid, key = x / (D / 8), d = x % (D / 8);
      *(u32x4*)(sk + key * S::KRow + 16 * d) = kr[i];
      *(u32x4*)(sv + key * S::VRow + 16 * d) = vr[i];
    }
  };
  if (t0 < t1) {
    fetch(t0);
    stage(0);
  }
  __syncthreads();

  for (int t = t0; t < t1; ++t) {
    const int base = t * kPaKeys;
    const uint8_t* sk = s_mem + ((t - t0) & 1) * S::Buffer;
    const uint8_t* sv = sk + kPaKeys * S::KRow;
    if (t + 1 < t1) fetch(t + 1);
    f32x16 s[2];
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      s[x] = f32x16{};
#pragma unroll
      for (int k = 0; k < 2 * NG; ++k) {
        const bf16x8 kf = *(const bf16x8*)(sk + (32 * x + col) * S::KRow + 32 * k + 16 * part);
        s[x] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf, qf[k], s[x], 0, 0, 0);
      }
    }
    if (base + kPaKeys > all_see) {   // keys that a row does not see
#pragma unroll
      for (int x = 0; x < 2; ++x)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const int key = base + 32 * x + i % 4 + 8 * (i / 4) + 4 * part;
          s[x][i] = key < end ? s[x][i] : kNegInf;
        }
    }
    // the running reference follows the maximum where that has grown by more
    // than 2^8: weights up to 256 lose nothing in floating point, and the sums
    // are rescaled a few times instead of with every tile
    float top = kNegInf;
#pragma unroll
    for (int x = 0; x < 2; ++x)
#pragma unroll
      for (int i = 0; i < 16; ++i) top = fmaxf(top, s[x][i]);
    top = max_halves(top) * a.c;
    if (__any(top > ref + 8.0f)) {
      const float to = fmaxf(ref, top);
      const float f = __builtin_amdgcn_exp2f(ref - to);
      ref = to;
      l *= f;
#pragma unroll
      for (int x = 0; x < NG; ++x)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[x][i] *= f;
    }
    float sum = 0.0f;
    uint32_t p[2][8];
#pragma unroll
    for (int x = 0; x < 2; ++x)
#pragma unroll
      for (int i = 0; i < 16; i += 2) {
        const float y = __builtin_amdgcn_exp2f(__builtin_fmaf(s[x][i], a.c, -ref));
        const float z = __builtin_amdgcn_exp2f(__builtin_fmaf(s[x][i + 1], a.c, -ref));
        sum += y + z;
        p[x][i / 2] = pack_bf16(y, z);   // to 8 bits, as the values they meet
      }
    l += sum;
    const uint8_t* vp =
        sv + (4 * part + (lane % 16) / 4) * S::VRow + (16 * ((lane / 16) % 2) + 4 * (lane % 4)) * 2;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      u32x4 pk;
#pragma unroll
      for (int i = 0; i < 4; ++i) pk[i] = p[k / 2][4 * (k % 2) + i];
      const bf16x8 pf = __builtin_bit_cast(bf16x8, pk);
#pragma unroll
      for (int x = 0; x < NG; ++x) {
        const i16x4 v0 = read_transposed(vp + (16 * k) * S::VRow + x * 64);
        const i16x4 v1 = read_transposed(vp + (16 * k + 8) * S::VRow + x * 64);
        const bf16x8 vf = __builtin_bit_cast(bf16x8, __builtin_shufflevector(v0, v1, 0, 1, 2, 3, 4, 5, 6, 7));
        o[x] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf, pf, o[x], 0, 0, 0);
      }
    }
    if (t + 1 < t1) stage((t + 1 - t0) & 1);
    __syncthreads();
  }
  l = sum_halves(l);

  if (pt.parts == 1) {
    if (!row_ok) return;
    const float inv = l > 0.0f ? 1.0f / l : 0.0f;
    const size_t at = (size_t)(pt.first + tok) * a.H + head;
#pragma unroll
    for (int t = 0; t < NG; ++t)
#pragma unroll
      for (int i = 0; i < 16; i += 4)
        *(u32x2*)(a.out + at * D + t * 32 + 2 * i + 4 * part) =
            u32x2{pack_bf16(o[t][i] * inv, o[t][i + 1] * inv), pack_bf16(o[t][i + 2] * inv, o[t][i + 3] * inv)};
    if (a.lse && part == 0) a.lse[at] = l > 0.0f ? (ref + __builtin_amdgcn_logf(l)) * kLn2 : kNegInf;
  } else {
    const size_t row =
        (((size_t)blockIdx.x * a.tiles + tile) * a.splits + blockIdx.z) * kPaRows + wave * 32 + col;
#pragma unroll
    for (int t = 0; t < NG; ++t)
#pragma unroll
      for (int i = 0; i < 16; i += 4)
        *(f32x4*)(a.part + row * D + t * 32 + 2 * i + 4 * part) = f32x4{o[t][i], o[t][i + 1], o[t][i + 2], o[t][i + 3]};
    if (part == 0) *(float2*)(a.part_ml + row * 2) = float2{ref, l};
  }
}

// Joins the parts of a row tile in the order of their keys: 16 rows a
// workgroup, 16 lanes a row.
template <int NG>
__global__ void __launch_bounds__(256)
k_prompt_join(const PromptArgs a) {
  constexpr int D = NG * 32, Groups = kPaRows / 16;
  const int b = blockIdx.x / a.Hk, h = blockIdx.x % a.Hk;
  const int tile = blockIdx.y / Groups;
  const int x = (blockIdx.y % Groups) * 16 + threadIdx.x / 16, lane = threadIdx.x % 16;
  const PaTile pt = pa_tile(a, b, tile);
  const int r = tile * kPaRows + x;
  if (r >= pt.rows || pt.parts == 1) return;
  const size_t row = (((size_t)blockIdx.x * a.tiles + tile) * a.splits) * kPaRows + x;
  float ref = kRefFloor;
  for (int z = 0; z < pt.parts; ++z) ref = fmaxf(ref, a.part_ml[(row + (size_t)z * kPaRows) * 2]);
  float acc[2 * NG], l = 0.0f;
#pragma unroll
  for (int i = 0; i < 2 * NG; ++i) acc[i] = 0.0f;
#pragma unroll 4
  for (int z = 0; z < pt.parts; ++z) {
    const size_t at = row + (size_t)z * kPaRows;
    const float2 ml = *(const float2*)(a.part_ml + at * 2);
    const float f = __builtin_amdgcn_exp2f(ml.x - ref);
    l += f * ml.y;
#pragma unroll
    for (int i = 0; i < NG; ++i) {
      const float2 v = *(const float2*)(a.part + at * D + 32 * i + 2 * lane);
      acc[2 * i] += f * v.x;
      acc[2 * i + 1] += f * v.y;
    }
  }
  const int tok = r / a.R, head = h * a.R + r % a.R;
  const size_t at = (size_t)(pt.first + tok) * a.H + head;
  const float inv = l > 0.0f ? 1.0f / l : 0.0f;
#pragma unroll
  for (int i = 0; i < NG; ++i)
    *(uint32_t*)(a.out + at * D + 32 * i + 2 * lane) = pack_bf16(acc[2 * i] * inv, acc[2 * i + 1] * inv);
  if (a.lse && lane == 0) a.lse[at] = l > 0.0f ? (ref + __builtin_amdgcn_logf(l)) * kLn2 : kNegInf;
}

// ---------------------------------------------------------------------------
// host side
// ---------------------------------------------------------------------------
struct PaPlan {
  int tiles, splits;
  size_t at_part, bytes;
};

static bool pa_sizes_ok(int B, int H, int Hk, int D, int max_q) {
  if ((D != 64 && D != 96 && D != 128) || H % Hk || H > (1 << 15)) return false;
  return (long long)B * Hk <= INT32_MAX && (long long)max_q * (H / Hk) <= 65535ll / (kPaRows / 16) * kPaRows;
}

// Row tiles alone where they fill the chip; otherwise their keys are divided
// too, two workgroups a CU in all.
static PaPlan pa_plan(int B, int Tk, int H, int Hk, int D, int max_q) {
  PaPlan p{};
  p.tiles = (int)(((long long)max_q * (H / Hk) + kPaRows - 1) / kPaRows);
  const long long base = (long long)B * Hk * p.tiles;
  p.splits = 1;
  if (base > 0 && base < 256) {
    const long long most = (Tk + kPaKeys * kPaSplitTiles - 1) / (kPaKeys * kPaSplitTiles);
    const long long want = 512 / base;
    p.splits = (int)(want < most ? want : most);
    if (p.splits < 1) p.splits = 1;
  }
  if (p.splits > 1) {
    const size_t rows = (size_t)base * p.splits * kPaRows;
    p.at_part = align256(rows * 8);
    p.bytes = p.at_part + rows * D * sizeof(float);
  }
  return p;
}

// The kernel's LDS is above the default limit; the limit is raised once per
// device and kernel, before the first launch there.
constexpr int kPaMaxDevices = 64;

template <int NG>
static hipError_t pa_launch(const PromptArgs& a, hipStream_t st) {
  typedef PaShape<NG> S;
  static std::atomic<bool> allowed[kPaMaxDevices];
  int dev = 0;
  hipError_t e = hipGetDevice(&dev);
  if (e != hipSuccess) return e;
  if (dev < 0 || dev >= kPaMaxDevices || !allowed[dev].load(std::memory_order_acquire)) {
    e = hipFuncSetAttribute((const void*)k_prompt_attn<NG>, hipFuncAttributeMaxDynamicSharedMemorySize, S::LdsBytes);
    if (e != hipSuccess) return e;
    if (dev >= 0 && dev < kPaMaxDevices) allowed[dev].store(true, std::memory_order_release);
  }
  const unsigned bh = (unsigned)(a.B * a.Hk);
  hipLaunchKernelGGL(k_prompt_attn<NG>, dim3(bh, (unsigned)a.tiles, (unsigned)a.splits), dim3(kPaThreads), S::LdsBytes,
                     st, a);
  if (a.splits > 1)
    hipLaunchKernelGGL(k_prompt_join<NG>, dim3(bh, (unsigned)(a.tiles * (kPaRows / 16))), dim3(256), 0, st, a);
  return hipGetLastError();
}

}  // namespace fdllm

using namespace fdllm;

extern "C" {

fdllm_status fdllm_prompt_attention_workspace_size(int B, int Tk, int H, int Hk, int D, int max_q, size_t* bytes) {
  if (!bytes || B < 0 || Tk < 0 || H < 1 || Hk < 1 || max_q < 0) return FDLLM_ERR_INVALID_ARG;
  if (!pa_sizes_ok(B, H, Hk, D, max_q)) return FDLLM_ERR_SIZE;
  *bytes = pa_plan(B, Tk, H, Hk, D, max_q).bytes;
  return FDLLM_OK;
}

fdllm_status fdllm_prompt_attention(const void* q, int64_t q_stride, const void* k, int64_t k_stride, const void* v,
                                    int64_t v_stride, int T, int Tk, const int32_t* cu_q, const int32_t* cu_k, int B,
                                    int max_q, int H, int Hk, int D, float scale, int blk, void* out, float* lse,
                                    void* workspace, size_t workspace_bytes, fdllm_stream stream) {
  if (T < 0 || Tk < 0 || B < 0 || max_q < 0 || H < 1 || Hk < 1 || blk < 0) return FDLLM_ERR_INVALID_ARG;
  if (!(scale > 0.0f) || scale > 3.0e38f) return FDLLM_ERR_INVALID_ARG;
  if (!pa_sizes_ok(B, H, Hk, D, max_q)) return FDLLM_ERR_SIZE;
  if (T == 0 || B == 0 || max_q == 0) return FDLLM_OK;
  if (!q || !cu_q || !cu_k || !out || (Tk > 0 && (!k || !v))) return FDLLM_ERR_INVALID_ARG;
  if (q_stride < (int64_t)H * D || k_stride < (int64_t)Hk * D || v_stride < (int64_t)Hk * D || q_stride % 8 ||
      k_stride % 8 || v_stride % 8)
    return FDLLM_ERR_INVALID_ARG;
  for (const void* p : {q, k, v, (const void*)out, (const void*)workspace})
    if ((uintptr_t)p & 15) return FDLLM_ERR_INVALID_ARG;
  const PaPlan p = pa_plan(B, Tk, H, Hk, D, max_q);
  if (p.bytes && (!workspace || workspace_bytes < p.bytes)) return FDLLM_ERR_WORKSPACE;
  char* ws = (char*)workspace;
  const PromptArgs a{(const uint16_t*)q, (const uint16_t*)k, (const uint16_t*)v, q_stride, k_stride, v_stride, T, Tk,
                     cu_q, cu_k, B, H, Hk, H / Hk, max_q, blk, scale * kLog2e, (uint16_t*)out, lse, p.tiles, p.splits,
                     (float*)ws, (float*)(ws + p.at_part)};
  hipStream_t st = (hipStream_t)stream;
  const hipError_t e = D == 64 ? pa_launch<2>(a, st) : D == 96 ? pa_launch<3>(a, st) : pa_launch<4>(a, st);
  return e == hipSuccess ? FDLLM_OK : FDLLM_ERR_HIP;
}

}  // extern "C"
