// prompt_attn.hip -- attention of whole packed sequences on gfx950:
// out_i = sum_j softmax_j(scale q_i . k_j) v_j over the keys j that query i
// sees, bfloat16 operands, float32 scores, sums and softmax statistics, in one
// pass over the keys with a running maximum and sum.
//
// The query tokens of a sequence times the query heads that share a key head
// are the rows of one product; a workgroup takes 128 of them, a wave 32, over
// tiles of 64 keys staged in LDS: 32 rows a wave read each key's operand once for
// 32 columns, and 64 KiB of LDS and 256 registers let two workgroups share a CU.
//
// Bound by the matrix cores: one causal prompt of 16384 tokens, 16 heads of 128
// over 4, 962 to 1000 us, 1.10 to 1.14 PFLOP/s (a 16384^3 library product of normal
// values reaches 1.36 to 1.38 in the same runs).  Short prompts by the starts and ends of the workgroups: 16384 tokens in
// prompts of equal length take 88 us and 14 more for every 64 keys.
#include <hip/hip_runtime.h>

#include <stdint.h>

#include <atomic>
#include <type_traits>

#include "attn_common.h"
#include "fdllm.h"

namespace fdllm {

constexpr int kPaThreads = 256;
constexpr int kPaWaves = kPaThreads / kWave;
static_assert(kPaRows == kPaWaves * 32, "a wave 32 rows");
constexpr int kPaKeys = 64;
constexpr int kPaSplitTiles = 4;   // tiles of keys that a part of a split row tile has at least
constexpr int kPaWholeTiles = 8;   // and those up to which none is split: joining costs a launch and 4 us
constexpr int kPaSlots = 512;      // workgroups that the chip runs at once
constexpr int kPaMaxParts = 1536;  // that a call may have room for

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
  int tiles, splits;   // row tiles of the longest sequence; most parts that the keys of one are divided into
  int share;           // tiles of keys that a part is to have
  int places;          // row tiles that there is room for, where keys are divided
  int by_sequence;     // order of the workgroups (pa_by_sequence)
  float* part_ml;      // [place, h, split, wave][32][2]: reference and sum of a row's partial result
  float* part;         // [place, h, split, wave] tiles of partial sums (attn_common.h)
};

// A tile of rows: 128 of a sequence's query tokens times the heads of a key head.
struct PaTile {
  int first, firstk, n, len, rows;
  int far;      // the most keys that any row sees
  int parts;    // into which its keys are divided
  int place;    // among the row tiles of all sequences, where parts > 1
};

__device__ __forceinline__ PaTile pa_tile(const PromptArgs& a, int b, int tile) {
  PaTile t;
  // first of all, so that its loads are under way beside the others: a lane counts
  // the row tiles of every 64th sequence before
  int before = 0;
  if (a.splits > 1 && b > 0)
    before = wave_sum(pa_tiles_before(a.cu_q, b, a.T, a.max_q, a.R, threadIdx.x % kWave, kWave));
  t.n = packed_rows(a.cu_q, b, a.T, a.max_q, &t.first);
  t.len = packed_rows(a.cu_k, b, a.Tk, INT32_MAX, &t.firstk);
  t.rows = t.n * a.R;
  t.far = 0;
  t.parts = 1;
  t.place = 0;
  if (tile * kPaRows >= t.rows) return t;
  const int last = min(t.rows, (tile + 1) * kPaRows) - 1;
  t.far = visible_end(t.len - t.n + last / a.R, a.blk, t.len);
  const int nt = (t.far + kPaKeys - 1) / kPaKeys;
  t.parts = nt <= max(kPaWholeTiles, 2 * a.share) ? 1 : min(a.splits, (nt + a.share - 1) / a.share);
  if (t.parts > 1) {
    t.place = before + tile;
    if (t.place >= a.places) t.parts = 1;   // tokens in several sequences: more row tiles than room
  }
  return t;
}

// A tile's rows in LDS lie RowBytes apart, two buffers each of keys and values.
// Within a row the 16-byte pieces are exchanged by the row's number, so that 16
// lanes meet all banks when they read a piece of 16 rows (keys), and 32 when they read 64 bytes of
// four rows transposed (values); the loads that write LDS fetch the piece that
// belongs where they write.
template <int NG>
struct PaShape {
  static constexpr int D = NG * 32;
  static constexpr int RowBytes = NG == 2 ? 128 : 256;
  static constexpr int Pieces = RowBytes / 16;
  static constexpr int Tile = kPaKeys * RowBytes;
  static constexpr int LdsBytes = 4 * Tile;
  static constexpr int RowsPerLoad = kWave / Pieces;                    // of a wave's load of 1 KiB
  static constexpr int Loads = kPaKeys / kPaWaves / RowsPerLoad;        // a wave, per operand and tile
  __device__ static int swap_k(int row) { return NG == 2 ? row / 2 % 8 : row % 16; }
  __device__ static int swap_v(int row) { return NG == 2 ? row / 2 % 2 * 4 : row % 4 * 4; }
};

typedef __attribute__((address_space(3))) void* pa_lds_t;

// Rows [first, first + rows) of one head of a packed operand as a resource:
// what is beyond reads as zero.
__device__ __forceinline__ i32x4 pa_rows(const uint16_t* p, int rows, long long stride, int D) {
  const uint64_t at = (uint64_t)p;
  i32x4 r;
  r[0] = __builtin_amdgcn_readfirstlane((int)(uint32_t)at);
  r[1] = __builtin_amdgcn_readfirstlane((int)((uint32_t)(at >> 32) & 0xffffu));
  r[2] = __builtin_amdgcn_readfirstlane(rows > 0 ? (int)((uint32_t)(rows - 1) * (uint32_t)(2 * stride) + 2u * D) : 0);
  r[3] = 0x00020000;
  return r;
}

// 16 bytes a lane from rsrc + voff to LDS byte lds + 16 lane.  As inline
// assembly, since the compiler would wait for it before every later LDS read;
// pa_arrive is what waits.  The wait states are the ones that the compiler does
// not put in here: one after the write of m0, five (with the two moves) after a
// vector instruction that wrote a word of rsrc.
__device__ __forceinline__ void pa_dma(i32x4 rsrc, uint32_t lds, uint32_t voff) {
  uint32_t keep;
  asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %1\n\ts_nop 2\n\tbuffer_load_dwordx4 %2, %3, 0 offen lds\n\t"
               "s_mov_b32 m0, %0"
               : "=&s"(keep) : "s"(lds), "v"(voff), "s"(rsrc) : "memory");
}

#define PA_FENCE() __builtin_amdgcn_sched_barrier(0)

// All of this wave's loads to LDS have landed, then everybody's.
__device__ __forceinline__ void pa_arrive() { asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

template <int NG>
__global__ void __launch_bounds__(kPaThreads, 2)
k_prompt_attn(const PromptArgs a) {
  typedef PaShape<NG> S;
  constexpr int D = S::D;
  extern __shared__ __align__(1024) uint8_t s_mem[];

  const int tid = threadIdx.x, lane = tid % kWave, wave = __builtin_amdgcn_readfirstlane(tid / kWave);
  const int col = lane % 32, part = lane / 32;
  const int outer = blockIdx.x / a.Hk, h = blockIdx.x % a.Hk;
  const int b = a.by_sequence ? blockIdx.y : outer;
  const int tile = a.tiles - 1 - (a.by_sequence ? outer : blockIdx.y);   // the rows that see most keys first
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
  float ref = kRefFloor, l = 0.0f, l2 = 0.0f;   // weights are 2^(c s - ref), l and l2 their sums

  // ---- loads to LDS ----
  const uint32_t lds0 = (uint32_t)(uintptr_t)(pa_lds_t)s_mem;
  const uint16_t* kbase = a.k + (size_t)pt.firstk * a.k_stride + (size_t)h * D;
  const uint16_t* vbase = a.v + (size_t)pt.firstk * a.v_stride + (size_t)h * D;
  uint32_t k_at[S::Loads], v_at[S::Loads];
#pragma unroll
  for (int i = 0; i < S::Loads; ++i) {
    const int row = (wave * S::Loads + i) * S::RowsPerLoad + lane / S::Pieces, piece = lane % S::Pieces;
    const int pk = piece ^ S::swap_k(row), pv = piece ^ S::swap_v(row);
    // pieces that a row has no elements for are out of the resource's range
    k_at[i] = 8 * pk < D ? (uint32_t)(row * 2 * a.k_stride) + 16u * pk : 0x7ffffff0u;
    v_at[i] = 8 * pv < D ? (uint32_t)(row * 2 * a.v_stride) + 16u * pv : 0x7ffffff0u;
  }
  const auto load = [&](const uint16_t* base, long long stride, const uint32_t* at, int t, int lds) {
    const i32x4 rsrc = pa_rows(base + (size_t)t * kPaKeys * stride, min(pt.len - t * kPaKeys, kPaKeys), stride, D);
#pragma unroll
    for (int i = 0; i < S::Loads; ++i)
      pa_dma(rsrc, lds0 + (uint32_t)(lds + (wave * S::Loads + i) * 1024), at[i]);
  };
  const auto load_k = [&](int t, int buf) { load(kbase, a.k_stride, k_at, t, buf * S::Tile); };
  const auto load_v = [&](int t, int buf) { load(vbase, a.v_stride, v_at, t, (2 + buf) * S::Tile); };

  // ---- reads from LDS ----
  const uint8_t* k_from[2 * NG];
  const uint8_t* v_from[NG];
#pragma unroll
  for (int k = 0; k < 2 * NG; ++k)
    k_from[k] = s_mem + col * S::RowBytes + 16 * ((2 * k + part) ^ S::swap_k(col));
  {
    const int row = 4 * part + (lane % 16) / 4, piece = 2 * ((lane / 16) % 2) + (lane % 4) / 2;
#pragma unroll
    for (int x = 0; x < NG; ++x)
      v_from[x] = s_mem + 2 * S::Tile + row * S::RowBytes + 16 * ((4 * x + piece) ^ S::swap_v(row)) + 8 * (lane % 2);
  }

  const auto key_operand = [&](int i, int buf) {   // of product i of a tile's scores
    return *(const bf16x8*)(k_from[i % (2 * NG)] + buf * S::Tile + (i / (2 * NG)) * 32 * S::RowBytes);
  };
  const auto value_operand = [&](int i, int buf) {   // of product i of a tile's outputs
    const uint8_t* at = v_from[i % NG] + buf * S::Tile + 16 * (i / NG) * S::RowBytes;
    const i16x4 v0 = read_transposed(at);
    const i16x4 v1 = read_transposed(at + 8 * S::RowBytes);
    return __builtin_bit_cast(bf16x8, __builtin_shufflevector(v0, v1, 0, 1, 2, 3, 4, 5, 6, 7));
  };
  f32x16 s[2], sn[2];   // S^T of a tile and of the next
  // keys that a row does not see
  const auto hide = [&](f32x16* to, int t) {
    const int base = t * kPaKeys;
    if (base + kPaKeys > all_see) {
#pragma unroll
      for (int x = 0; x < 2; ++x)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const int key = base + 32 * x + i % 4 + 8 * (i / 4) + 4 * part;
          to[x][i] = key < end ? to[x][i] : kNegInf;
        }
    }
  };
  const auto largest = [&](const f32x16* of) {
    float top = kNegInf;
#pragma unroll
    for (int x = 0; x < 2; ++x)
#pragma unroll
      for (int i = 0; i < 16; ++i) top = fmaxf(top, of[x][i]);
    return max_halves(top) * a.c;
  };
  // The running reference follows the maximum where that has grown by more than
  // 2^8: weights up to 256 lose nothing in floating point, and the sums are
  // rescaled a few times instead of with every tile.
  const auto follow = [&](float top) {
    if (__any(top > ref + 8.0f)) {
      const float to = fmaxf(ref, top);
      const float f = __builtin_amdgcn_exp2f(ref - to);
      ref = to;
      l *= f;
      l2 *= f;
#pragma unroll
      for (int x = 0; x < NG; ++x)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[x][i] *= f;
    }
  };
  // Pair i of a tile's 16 pairs of weights; four pairs make the operand of one
  // product of outputs and NG - 1 more.  Rounded to bfloat16, the type of the values
  // that they meet (the sums take them unrounded): an output is off by 0.0021 to
  // 0.0022 relative, 0.0017 in 32 bits rounded once; in two pieces they would
  // double the products of the outputs.
  u32x4 p[4];
  const auto weigh = [&](const f32x16* of, int i) {
    const float y = __builtin_amdgcn_exp2f(__builtin_fmaf(of[i / 8][2 * (i % 8)], a.c, -ref));
    const float z = __builtin_amdgcn_exp2f(__builtin_fmaf(of[i / 8][2 * (i % 8) + 1], a.c, -ref));
    l += y;
    l2 += z;
    p[i / 4][i % 4] = pack_bf16(y, z);
  };
  const auto output = [&](bf16x8 v, int i) {
    o[i % NG] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v, __builtin_bit_cast(bf16x8, p[i / NG]), o[i % NG], 0, 0, 0);
  };

  // One tile: the next one's scores are formed while this one's weights are,
  // then this one's outputs beside the next one's maximum.  The workgroup meets
  // once a tile, between the two: what a tile reads after the meeting has had a
  // whole tile's time to land, and what it read before may be written over.
  // The fences keep the order within: a product of the matrix cores, then what
  // the vector units do meanwhile, with LDS reads two products ahead.
  bf16x8 kf[3], vf[3];
  const auto step = [&](int t, f32x16* s, f32x16* sn, auto buf_) {
    constexpr int buf = decltype(buf_)::value, NP = 4 * NG;
    PA_FENCE();
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      if (i + 2 < NP) kf[(i + 2) % 3] = key_operand(i + 2, buf ^ 1);
      const int x = i / (2 * NG);
      sn[x] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[i % 3], qf[i % (2 * NG)], i % (2 * NG) ? sn[x] : f32x16{}, 0, 0,
                                                      0);
      PA_FENCE();
      // twelve of the sixteen pairs of weights
#pragma unroll
      for (int w = i * 12 / NP; w < (i + 1) * 12 / NP; ++w) weigh(s, w);
      PA_FENCE();
    }
    // (the weights stay on this side of the branch)
    asm volatile("" : "+v"(p[0]), "+v"(p[1]), "+v"(p[2]), "+v"(l), "+v"(l2));
    hide(sn, t + 1);
    pa_arrive();
    if (t + 3 < t1) load_k(t + 3, buf ^ 1);
    load_v(t + 1, buf ^ 1);
    __builtin_amdgcn_s_setprio(1);
    vf[0] = value_operand(0, buf);
    vf[1] = value_operand(1, buf);
    PA_FENCE();
#pragma unroll
    for (int w = 12; w < 16; ++w) weigh(s, w);
    float top = kNegInf;
    PA_FENCE();
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      if (i + 2 < NP) vf[(i + 2) % 3] = value_operand(i + 2, buf);
      else kf[i + 2 - NP] = key_operand(i + 2 - NP, buf);   // of the tile after next
      output(vf[i % 3], i);
      PA_FENCE();
#pragma unroll
      for (int m = i * 16 / NP; m < (i + 1) * 16 / NP; ++m)
        top = fmaxf(fmaxf(top, sn[m / 8][2 * (m % 8)]), sn[m / 8][2 * (m % 8) + 1]);
      PA_FENCE();
    }
    __builtin_amdgcn_s_setprio(0);
    follow(max_halves(top) * a.c);
  };
  const auto last = [&](const f32x16* s, int buf) {
#pragma unroll
    for (int i = 0; i < 16; ++i) weigh(s, i);
    pa_arrive();
#pragma unroll
    for (int i = 0; i < 4 * NG; ++i) output(value_operand(i, buf), i);
  };

  if (t0 < t1) {
    load_k(t0, 0);
    if (t0 + 1 < t1) load_k(t0 + 1, 1);
    pa_arrive();
#pragma unroll
    for (int x = 0; x < 2; ++x) s[x] = f32x16{};
#pragma unroll
    for (int i = 0; i < 4 * NG; ++i)
      s[i / (2 * NG)] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(key_operand(i, 0), qf[i % (2 * NG)], s[i / (2 * NG)], 0,
                                                                0, 0);
    hide(s, t0);
    follow(largest(s));
    kf[0] = key_operand(0, 1);
    kf[1] = key_operand(1, 1);
    pa_arrive();   // everybody has read the first keys
    if (t0 + 2 < t1) load_k(t0 + 2, 0);
    load_v(t0, 0);
    int t = t0;
    typedef std::integral_constant<int, 0> Even;
    typedef std::integral_constant<int, 1> Odd;
    for (; t + 2 < t1; t += 2) {
      step(t, s, sn, Even{});
      step(t + 1, sn, s, Odd{});
    }
    if (t + 1 < t1) {
      step(t, s, sn, Even{});
      last(sn, 1);
    } else {
      last(s, 0);
    }
  }
  l = sum_halves(l + l2);

  constexpr int Quads = quads_of(32, NG);
  if (pt.parts == 1) {
    // through LDS (where the keys were: nobody reads them any more), so that a
    // row leaves in one piece
    const float inv = inverse_sum(l);
    uint8_t* lds = s_mem + wave * 32 * OutRows<NG>::RowBytes;
#pragma unroll
    for (int q = 0; q < Quads; ++q) {
      const int x = q / 4, i = 4 * (q % 4);
      *(u32x2*)(lds + OutRows<NG>::at(col, quad_element<32>(q, part))) =
          u32x2{pack_bf16(o[x][i] * inv, o[x][i + 1] * inv), pack_bf16(o[x][i + 2] * inv, o[x][i + 3] * inv)};
    }
    __builtin_amdgcn_wave_barrier();
    if (row_ok && a.lse && part == 0)
      a.lse[(size_t)(pt.first + tok) * a.H + head] = log_sum(ref, l);
#pragma unroll
    for (int j = 0; j < 32 * (D / 8) / kWave; ++j) {
      const int x = j * kWave + lane, row = x / (D / 8), d = 8 * (x % (D / 8)), rr = tile * kPaRows + wave * 32 + row;
      if (rr < pt.rows) {
        const size_t at = (size_t)(pt.first + rr / a.R) * a.H + h * a.R + rr % a.R;
        *(u32x4*)(a.out + at * D + d) = *(const u32x4*)(lds + OutRows<NG>::at(row, d));
      }
    }
  } else {
    const size_t part_tile = (((size_t)pt.place * a.Hk + h) * a.splits + blockIdx.z) * kPaWaves + wave;
#pragma unroll
    for (int q = 0; q < Quads; ++q) {
      const int x = q / 4, i = 4 * (q % 4);
      *(f32x4*)(a.part + ((part_tile * Quads + q) * kWave + lane) * 4) =
          f32x4{o[x][i], o[x][i + 1], o[x][i + 2], o[x][i + 3]};
    }
    if (part == 0) *(float2*)(a.part_ml + (part_tile * 32 + col) * 2) = float2{ref, l};
  }
}

// Joins the parts of a row tile in the order of their keys: a workgroup for the
// 32 rows of a wave, as they lay in its registers, a few quads a wave.
template <int NG>
__global__ void __launch_bounds__(kPaThreads)
k_prompt_join(const PromptArgs a) {
  constexpr int D = NG * 32, Quads = quads_of(32, NG), QPer = Quads / kPaWaves;
  __shared__ __align__(16) uint8_t s_out[32 * OutRows<NG>::RowBytes];
  const int b = blockIdx.x / a.Hk, h = blockIdx.x % a.Hk;
  const int tile = blockIdx.y / kPaWaves, wr = blockIdx.y % kPaWaves;
  const PaTile pt = pa_tile(a, b, tile);
  const int r0 = tile * kPaRows + wr * 32;
  if (r0 >= pt.rows || pt.parts == 1) return;
  const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int col = lane % 32, part = lane / 32;
  const size_t first = (((size_t)pt.place * a.Hk + h) * a.splits) * kPaWaves + wr;
  f32x4 acc[QPer];
#pragma unroll
  for (int i = 0; i < QPer; ++i) acc[i] = f32x4{};
  float ref = kRefFloor, l = 0.0f;
  constexpr int Ahead = 4;   // parts under way at once
  for (int z = 0; z < pt.parts; z += Ahead) {
    float2 ml[Ahead];
    f32x4 v[Ahead][QPer];
#pragma unroll
    for (int k = 0; k < Ahead; ++k) {
      const size_t at = first + (size_t)min(z + k, pt.parts - 1) * kPaWaves;
      ml[k] = *(const float2*)(a.part_ml + (at * 32 + col) * 2);
#pragma unroll
      for (int i = 0; i < QPer; ++i)
        v[k][i] = *(const f32x4*)(a.part + ((at * Quads + wave * QPer + i) * kWave + lane) * 4);
    }
    float to = ref;
#pragma unroll
    for (int k = 0; k < Ahead; ++k) to = fmaxf(to, ml[k].x);
    const float f0 = __builtin_amdgcn_exp2f(ref - to);
    ref = to;
    l *= f0;
#pragma unroll
    for (int i = 0; i < QPer; ++i) acc[i] *= f0;
#pragma unroll
    for (int k = 0; k < Ahead; ++k) {
      const float f = z + k < pt.parts ? __builtin_amdgcn_exp2f(ml[k].x - ref) : 0.0f;
      l += f * ml[k].y;
#pragma unroll
      for (int i = 0; i < QPer; ++i) acc[i] += v[k][i] * f;
    }
  }
  const float inv = inverse_sum(l);
#pragma unroll
  for (int i = 0; i < QPer; ++i)
    *(u32x2*)(s_out + OutRows<NG>::at(col, quad_element<32>(wave * QPer + i, part))) =
        u32x2{pack_bf16(acc[i][0] * inv, acc[i][1] * inv), pack_bf16(acc[i][2] * inv, acc[i][3] * inv)};
  if (wave == 0 && part == 0 && a.lse && r0 + col < pt.rows)
    a.lse[(size_t)(pt.first + (r0 + col) / a.R) * a.H + h * a.R + (r0 + col) % a.R] =
        log_sum(ref, l);
  __syncthreads();
  for (int x = threadIdx.x; x < 32 * (D / 8); x += kPaThreads) {
    const int row = x / (D / 8), d = 8 * (x % (D / 8)), r = r0 + row;
    if (r >= pt.rows) break;
    const size_t at = (size_t)(pt.first + r / a.R) * a.H + h * a.R + r % a.R;
    *(u32x4*)(a.out + at * D + d) = *(const u32x4*)(s_out + OutRows<NG>::at(row, d));
  }
}

// ---------------------------------------------------------------------------
// host side
// ---------------------------------------------------------------------------
struct PaPlan {
  int tiles, splits, share, places;
  size_t at_part, bytes;
};

// a tile's rows are addressed by 32-bit byte offsets
constexpr int64_t kPaMaxStride = INT32_MAX / (2 * kPaKeys) - 256;

// Row tiles of a sequence of n query tokens.
static long long pa_tiles(int n, int R) { return ((long long)n * R + kPaRows - 1) / kPaRows; }

static bool pa_sizes_ok(int B, int T, int H, int Hk, int D, int max_q) {
  if ((D != 64 && D != 96 && D != 128) || H % Hk || H > (1 << 15)) return false;
  if ((long long)B * Hk >= (1ll << 32) / kPaThreads) return false;   // threads along a launch's first axis
  // workgroups along its second; the join has kPaWaves times as many, but keys are
  // divided only where there are few row tiles (kPaMaxParts)
  return pa_tiles(max_q < T ? max_q : T, H / Hk) <= 65535;
}

// A row tile's keys are divided where the longest tile would run on while the
// rest of the chip is done: where it has more than twice the keys that fall to
// one of the workgroups that run at once, as far as the host knows them (it
// knows the sums of the lengths, not the lengths).  Three causal sequences
// of 1, 1937 and 3873 tokens with 5 heads on one: 61 us whole, 52 divided (67 and
// 71 without a mask); three of 20 tokens behind 3000: 48 and 14; 13 of 570 tokens:
// 18 whole, 31 divided, so what is merely uneven stays whole.
static PaPlan pa_plan(int B, int T, int Tk, int H, int Hk, int D, int max_q, int blk) {
  PaPlan p{};
  const int R = H / Hk;
  if (max_q > T) max_q = T;   // no sequence is longer than all of them
  p.tiles = (int)pa_tiles(max_q, R);
  p.splits = 1;
  p.share = kPaSplitTiles;
  if (B < 1 || p.tiles < 1) return p;
  const long long places = pa_places(B, T, R);
  const long long past = Tk > T ? (Tk - T) / B : 0;
  const long long keys = Tk / B - (blk && T < Tk + B ? T / B / 2 : 0);   // of a row, in the middle
  const long long units = ((long long)T * R + kPaRows - 1) / kPaRows * Hk * (keys / kPaKeys + 1);
  const long long longest = ((blk ? max_q + past : Tk < max_q + past ? Tk : max_q + past) + kPaKeys - 1) / kPaKeys;
  const long long share = units / kPaSlots;
  p.share = (int)(share > kPaSplitTiles ? share : kPaSplitTiles);
  if (longest <= kPaWholeTiles || longest <= 2ll * p.share) return p;
  const long long room = kPaMaxParts / (places * Hk), want = (longest + p.share - 1) / p.share;
  p.splits = (int)(room < want ? room : want);
  if (p.splits < 2) {
    p.splits = 1;
    return p;
  }
  p.places = (int)places;
  const size_t rows = (size_t)places * Hk * p.splits * kPaRows;
  p.at_part = align256(rows * 8);
  p.bytes = p.at_part + rows * D * sizeof(float);
  return p;
}

// Workgroups run the longest row tiles of all sequences first, so that none is
// left over in the end; but one sequence after another
// - where many of those would be tiles that a shorter sequence does not have:
//   workgroups are handed out in turn, and empty ones between the others leave
//   the work to some of the CUs (four prompts of 1 to 4096 tokens 382 us by tile,
//   230 by sequence; eight of 1 to 1024 53 and 45; six of 100 to 900 37 and 38);
// - where the keys and values that an XCD's workgroups then have in use (a
//   head's; from eight heads on it works on every eighth) exceed its cache (128
//   prompts of 128 tokens, 8 heads, 8.4 MB: 107 us by tile, 98 by sequence).
// Four of 500 to 777 tokens behind 2000, 2.7 MB: 40.4 us by tile, 42.8 by sequence.
constexpr long long kPaCacheBytes = 4 << 20;

static bool pa_by_sequence(int B, int T, int Tk, int Hk, int D, int max_q, int tiles) {
  // (what the grid has room for: 2^32 threads along the tiles, 65535 sequences)
  if (B < 2 || B > 65535 || (long long)tiles * Hk > (1ll << 32) / kPaThreads - 1) return false;
  return 4ll * T < 3ll * B * max_q || 4ll * Tk * D * ((Hk + 7) / 8) > kPaCacheBytes;
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
  const dim3 grid = a.by_sequence ? dim3((unsigned)(a.tiles * a.Hk), (unsigned)a.B, (unsigned)a.splits)
                                  : dim3(bh, (unsigned)a.tiles, (unsigned)a.splits);
  hipLaunchKernelGGL(k_prompt_attn<NG>, grid, dim3(kPaThreads), S::LdsBytes, st, a);
  if (a.splits > 1)
    hipLaunchKernelGGL(k_prompt_join<NG>, dim3(bh, (unsigned)(a.tiles * kPaWaves)), dim3(kPaThreads), 0, st, a);
  return hipGetLastError();
}

}  // namespace fdllm

using namespace fdllm;

extern "C" {

fdllm_status fdllm_prompt_attention_workspace_size(int B, int T, int Tk, int H, int Hk, int D, int max_q, int blk,
                                                   size_t* bytes) {
  if (!bytes || B < 0 || T < 0 || Tk < 0 || blk < 0 || H < 1 || Hk < 1 || max_q < 0) return FDLLM_ERR_INVALID_ARG;
  if (!pa_sizes_ok(B, T, H, Hk, D, max_q)) return FDLLM_ERR_SIZE;
  *bytes = pa_plan(B, T, Tk, H, Hk, D, max_q, blk).bytes;
  return FDLLM_OK;
}

fdllm_status fdllm_prompt_attention(const void* q, int64_t q_stride, const void* k, int64_t k_stride, const void* v,
                                    int64_t v_stride, int T, int Tk, const int32_t* cu_q, const int32_t* cu_k, int B,
                                    int max_q, int H, int Hk, int D, float scale, int blk, void* out, float* lse,
                                    void* workspace, size_t workspace_bytes, fdllm_stream stream) {
  if (T < 0 || Tk < 0 || B < 0 || max_q < 0 || H < 1 || Hk < 1 || blk < 0) return FDLLM_ERR_INVALID_ARG;
  if (!(scale > 0.0f) || scale > 3.0e38f) return FDLLM_ERR_INVALID_ARG;
  if (!pa_sizes_ok(B, T, H, Hk, D, max_q)) return FDLLM_ERR_SIZE;
  if (T == 0 || B == 0 || max_q == 0) return FDLLM_OK;
  if (!q || !cu_q || !cu_k || !out || (Tk > 0 && (!k || !v))) return FDLLM_ERR_INVALID_ARG;
  if (q_stride < (int64_t)H * D || k_stride < (int64_t)Hk * D || v_stride < (int64_t)Hk * D || q_stride % 8 ||
      k_stride % 8 || v_stride % 8)
    return FDLLM_ERR_INVALID_ARG;
  if (k_stride > kPaMaxStride || v_stride > kPaMaxStride) return FDLLM_ERR_SIZE;
  for (const void* p : {q, k, v, (const void*)out, (const void*)workspace})
    if ((uintptr_t)p & 15) return FDLLM_ERR_INVALID_ARG;
  const PaPlan p = pa_plan(B, T, Tk, H, Hk, D, max_q, blk);
  if (p.bytes && (!workspace || workspace_bytes < p.bytes)) return FDLLM_ERR_WORKSPACE;
  char* ws = (char*)workspace;
  const PromptArgs a{(const uint16_t*)q, (const uint16_t*)k, (const uint16_t*)v, q_stride, k_stride, v_stride, T, Tk,
                     cu_q, cu_k, B, H, Hk, H / Hk, max_q, blk, scale * kLog2e, (uint16_t*)out, lse, p.tiles, p.splits,
                     p.share, p.places, pa_by_sequence(B, T, Tk, Hk, D, max_q, p.tiles), (float*)ws,
                     (float*)(ws + p.at_part)};
  hipStream_t st = (hipStream_t)stream;
  const hipError_t e = D == 64 ? pa_launch<2>(a, st) : D == 96 ? pa_launch<3>(a, st) : pa_launch<4>(a, st);
  return e == hipSuccess ? FDLLM_OK : FDLLM_ERR_HIP;
}

}  // extern "C"
