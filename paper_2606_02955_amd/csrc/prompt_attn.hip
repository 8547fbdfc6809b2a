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

#include "attn_common.h"
#include "fdllm.h"

namespace fdllm {

constexpr int kPaThreads = 256;
constexpr int kPaWaves = kPaThreads / kWave;
constexpr int kPaRows = kPaWaves * 32;
constexpr int kPaKeys = 64;

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
};

template <int NG>
__global__ void __launch_bounds__(kPaThreads, 2)
k_prompt_attn(const PromptArgs a) {
  constexpr int D = NG * 32;
  constexpr int RowBytes = 2 * D + 32;
  constexpr int Loads = kPaKeys * D * 2 / 16 / kPaThreads;   // 16-byte loads a thread, per operand
  __shared__ __align__(16) uint8_t s_k[kPaKeys * RowBytes];
  __shared__ __align__(16) uint8_t s_v[kPaKeys * RowBytes];

  const int tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave;
  const int col = lane % 32, part = lane / 32;
  const int b = blockIdx.x / a.Hk, h = blockIdx.x % a.Hk;
  const int tile = gridDim.y - 1 - blockIdx.y;   // the rows that see most keys first
  int first, firstk;
  const int n = packed_rows(a.cu_q, b, a.T, a.max_q, &first);
  const int len = packed_rows(a.cu_k, b, a.Tk, INT32_MAX, &firstk);
  const int rows = n * a.R;
  if (tile * kPaRows >= rows) return;

  const int r = tile * kPaRows + wave * 32 + col;
  const bool row_ok = r < rows;
  const int tok = row_ok ? r / a.R : 0, head = h * a.R + (row_ok ? r % a.R : 0);
  const int end = row_ok ? visible_end(len - n + tok, a.blk, len) : 0;
  const int last_row = min(rows, (tile + 1) * kPaRows) - 1;
  const int far = visible_end(len - n + last_row / a.R, a.blk, len);   // the most any row sees

  bf16x8 qf[2 * NG];
#pragma unroll
  for (int t = 0; t < 2 * NG; ++t) {
    bf16x8 x = {};
    if (row_ok)
      x = *(const bf16x8*)(a.q + (size_t)(first + tok) * a.q_stride + (size_t)head * D + 16 * t + 8 * part);
    qf[t] = x;
  }
  f32x16 o[NG];
#pragma unroll
  for (int t = 0; t < NG; ++t) o[t] = f32x16{};
  float m = kNegInf, l = 0.0f;

  for (int base = 0; base < far; base += kPaKeys) {
    __syncthreads();
#pragma unroll
    for (int i = 0; i < Loads; ++i) {
      const int x = i * kPaThreads + tid, key = x / (D / 8), d = x % (D / 8);
      u32x4 kx = {}, vx = {};
      if (base + key < len) {   // past the end of the sequence: zeros
        kx = *(const u32x4*)(a.k + (size_t)(firstk + base + key) * a.k_stride + (size_t)h * D + 8 * d);
        vx = *(const u32x4*)(a.v + (size_t)(firstk + base + key) * a.v_stride + (size_t)h * D + 8 * d);
      }
      *(u32x4*)(s_k + key * RowBytes + 16 * d) = kx;
      *(u32x4*)(s_v + key * RowBytes + 16 * d) = vx;
    }
    __syncthreads();
    f32x16 s[2];
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      s[x] = f32x16{};
#pragma unroll
      for (int t = 0; t < 2 * NG; ++t) {
        const bf16x8 kf = *(const bf16x8*)(s_k + (32 * x + col) * RowBytes + 32 * t + 16 * part);
        s[x] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf, qf[t], s[x], 0, 0, 0);
      }
    }
#pragma unroll
    for (int x = 0; x < 2; ++x)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int key = base + 32 * x + i % 4 + 8 * (i / 4) + 4 * part;
        s[x][i] = key < end ? s[x][i] : kNegInf;
      }
    float top = kNegInf;
#pragma unroll
    for (int x = 0; x < 2; ++x)
#pragma unroll
      for (int i = 0; i < 16; ++i) top = fmaxf(top, s[x][i]);
    top = max_halves(top);
    const float mn = fmaxf(m, top);
    const float ref = fmaxf(mn * a.c, kRefFloor);   // finite while nothing was seen
    const float alpha = __builtin_amdgcn_exp2f(m * a.c - ref);
    m = mn;
    float sum = 0.0f;
    uint32_t p[2][8];
#pragma unroll
    for (int x = 0; x < 2; ++x)
#pragma unroll
      for (int i = 0; i < 16; i += 2) {
        const float y = __builtin_amdgcn_exp2f(__builtin_fmaf(s[x][i], a.c, -ref));
        const float z = __builtin_amdgcn_exp2f(__builtin_fmaf(s[x][i + 1], a.c, -ref));
        sum += y + z;
        p[x][i / 2] = pack_bf16(y, z);
      }
    l = l * alpha + sum;
#pragma unroll
    for (int t = 0; t < NG; ++t)
#pragma unroll
      for (int i = 0; i < 16; ++i) o[t][i] *= alpha;
    const uint8_t* vp = s_v + (4 * part + (lane % 16) / 4) * RowBytes + (16 * ((lane / 16) % 2) + 4 * (lane % 4)) * 2;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      u32x4 pk;
#pragma unroll
      for (int i = 0; i < 4; ++i) pk[i] = p[k / 2][4 * (k % 2) + i];
      const bf16x8 pf = __builtin_bit_cast(bf16x8, pk);
#pragma unroll
      for (int t = 0; t < NG; ++t) {
        const i16x4 v0 = read_transposed(vp + (16 * k) * RowBytes + t * 64);
        const i16x4 v1 = read_transposed(vp + (16 * k + 8) * RowBytes + t * 64);
        const bf16x8 vf = __builtin_bit_cast(bf16x8, __builtin_shufflevector(v0, v1, 0, 1, 2, 3, 4, 5, 6, 7));
        o[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf, pf, o[t], 0, 0, 0);
      }
    }
  }
  l = sum_halves(l);
  if (row_ok) {
    const float inv = l > 0.0f ? 1.0f / l : 0.0f;
    const size_t at = (size_t)(first + tok) * a.H + head;
#pragma unroll
    for (int t = 0; t < NG; ++t)
#pragma unroll
      for (int i = 0; i < 16; i += 4)
        *(u32x2*)(a.out + at * D + t * 32 + 2 * i + 4 * part) =
            u32x2{pack_bf16(o[t][i] * inv, o[t][i + 1] * inv), pack_bf16(o[t][i + 2] * inv, o[t][i + 3] * inv)};
    if (a.lse && part == 0) a.lse[at] = l > 0.0f ? (m * a.c + __builtin_amdgcn_logf(l)) * kLn2 : kNegInf;
  }
}

template <int NG>
static void pa_launch(const PromptArgs& a, hipStream_t st) {
  const long long tiles = ((long long)a.max_q * a.R + kPaRows - 1) / kPaRows;
  hipLaunchKernelGGL(k_prompt_attn<NG>, dim3((unsigned)(a.B * a.Hk), (unsigned)tiles), dim3(kPaThreads), 0, st, a);
}

}  // namespace fdllm

using namespace fdllm;

extern "C" {

fdllm_status fdllm_prompt_attention(const void* q, int64_t q_stride, const void* k, int64_t k_stride, const void* v,
                                    int64_t v_stride, int T, int Tk, const int32_t* cu_q, const int32_t* cu_k, int B,
                                    int max_q, int H, int Hk, int D, float scale, int blk, void* out, float* lse,
                                    fdllm_stream stream) {
  if (T < 0 || Tk < 0 || B < 0 || max_q < 0 || H < 1 || Hk < 1 || blk < 0) return FDLLM_ERR_INVALID_ARG;
  if (!(scale > 0.0f) || scale > 3.0e38f) return FDLLM_ERR_INVALID_ARG;
  if ((D != 64 && D != 96 && D != 128) || H % Hk || H > (1 << 15)) return FDLLM_ERR_SIZE;
  if ((long long)B * Hk > INT32_MAX || (long long)max_q * (H / Hk) > 65535ll * kPaRows) return FDLLM_ERR_SIZE;
  if (T == 0 || B == 0 || max_q == 0) return FDLLM_OK;
  if (!q || !cu_q || !cu_k || !out || (Tk > 0 && (!k || !v))) return FDLLM_ERR_INVALID_ARG;
  if (q_stride < (int64_t)H * D || k_stride < (int64_t)Hk * D || v_stride < (int64_t)Hk * D || q_stride % 8 ||
      k_stride % 8 || v_stride % 8)
    return FDLLM_ERR_INVALID_ARG;
  for (const void* p : {q, k, v, (const void*)out})
    if ((uintptr_t)p & 15) return FDLLM_ERR_INVALID_ARG;
  const PromptArgs a{(const uint16_t*)q, (const uint16_t*)k, (const uint16_t*)v, q_stride, k_stride, v_stride, T, Tk,
                     cu_q, cu_k, B, H, Hk, H / Hk, max_q, blk, scale * kLog2e, (uint16_t*)out, lse};
  hipStream_t st = (hipStream_t)stream;
  if (D == 64) pa_launch<2>(a, st);
  else if (D == 96) pa_launch<3>(a, st);
  else pa_launch<4>(a, st);
  return hipGetLastError() == hipSuccess ? FDLLM_OK : FDLLM_ERR_HIP;
}

}  // extern "C"
