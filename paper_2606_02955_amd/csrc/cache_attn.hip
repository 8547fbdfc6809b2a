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
// Keys and values are unpacked to bfloat16 (exact: a code has two significant
// bits, its scale none): the keys in registers, as the first product's operand,
// the values into LDS, to be read back transposed as the second's.
//
// Each workgroup takes an equal share of all units, whatever the sequences'
// lengths; an item that lies in several shares is joined afterwards, in the
// order of its pages.
//
// Tiles of 16 rows are bound by the read: two tokens over 99001 to 131072 keys
// (8 heads of keys of 128) 43 us for 250 MB, 5.8 TB/s.  Tiles of 32 by the
// instructions: 64 blocks of 32 tokens, four heads a key head, over 6000 to 8192
// keys 247 us, 0.81 PFLOP/s, the matrix cores busy half of the time and the
// vector units 58%, since a wave's scores, softmax and outputs follow one
// another; to form the next page's scores beside this page's softmax takes more
// registers than a wave has (measured with spills in the starts and ends: 300).
#include <hip/hip_runtime.h>

#include <stdint.h>

#include <atomic>
#include <type_traits>

#include "attn_common.h"
#include "fdllm.h"

namespace fdllm {

constexpr int kCaMaxWaves = 8;

// keeps instructions on their side: the order of the loop below is the one written
#define CA_FENCE() __builtin_amdgcn_sched_barrier(0)

// What an item costs beside its pages (its queries, the way to its first page,
// its results), in pages: half as many units before its pages and half behind
// stand for that, so that a share of many short items takes no longer than one
// of a few long ones.  (Ragged spans of 1 to 4099 tokens, 24 blocks of 32
// queries: 63 us at 0, 44 at 3 or 4.)
constexpr int kItemEnds = 2, kItemUnits = 2 * kItemEnds;

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
  int32_t* plan;              // units of all sequences, then those before each (null: no item is split)
  float* part_ml;             // [workgroups][2][WR][MT][2]: reference and sum of a row's partial result
  float* part;                // [workgroups][2][WR] tiles of partial sums (attn_common.h)
  const unsigned long long* masks;   // of a tree: [T][mask_w]
  int mask_w;
  int whole;                  // of a tree: items of a sequence, where a workgroup takes one whole (0: equal shares)
};

// A sequence as the plan sees it: its query rows, pages and groups of rows.
struct Seq {
  int first, n, len, groups, pages;
  int given;     // the length as it was given: what the table has no page for counts for a tree's places
  // Tokens before a tree's nodes.  (Formed where it is used: kept, it cost two trees
  // over 99001 to 131072 keys 0.9 us of 49.3.)
  __device__ __forceinline__ int context() const { return given - n; }
  __device__ __forceinline__ int units(int Hk) const { return groups * Hk * (pages + kItemUnits); }
};

template <int Rows>
__device__ __forceinline__ Seq sequence(const CacheAttnArgs& a, int b) {
  Seq s;
  s.n = packed_rows(a.cu_q, b, a.T, a.max_q, &s.first);
  const int most = a.table_w * kPage;
  s.given = max(a.kv_len[b], 0);
  s.len = min(s.given, most);
  s.groups = (s.n * a.R + Rows - 1) / Rows;
  s.pages = max(1, (s.len + kPage - 1) / kPage);   // one at least: a row without keys gets its zeros
  return s;
}

// Which of the 64 keys from `base` on a node of a tree sees, a bit each: those
// before the nodes, which begin at key `context`, and of the n nodes those in its
// words of the mask, of which the first is at hand.  (base and context meet in 32
// bits: context is negative only where there are fewer keys than nodes.)
__device__ __forceinline__ unsigned long long tree_window(const unsigned long long* words, unsigned long long word0,
                                                          int n, int base, int context) {
  const int f = base - context;   // the node at the first of them
  const auto word = [&](int w) { return w == 0 ? word0 : w * 64 < n ? words[w] : 0ull; };
  unsigned long long seen;
  if (f < 0) {
    seen = f <= -64 ? ~0ull : word(0) << -f | ((1ull << -f) - 1);
  } else {
    seen = word(f / 64) >> (f % 64);
    if (f % 64) seen |= word(f / 64 + 1) << (64 - f % 64);
  }
  const int left = n - f;         // nodes from the first key on
  return left <= 0 ? 0ull : left < 64 ? seen & ((1ull << left) - 1) : seen;
}

// The units are shared out evenly: share g begins at unit g * q + min(g, r), q
// and r the units by the number of shares.  Only trailing shares are empty.
struct Shares {
  int q, r;
  __device__ __forceinline__ Shares(int units, int n) : q(units / n), r(units % n) {}
  __device__ __forceinline__ int begin(int g) const { return g * q + min(g, r); }
  __device__ __forceinline__ int of(int u) const {
    const int wide = r * (q + 1);   // units in the shares that are one longer
    return u < wide ? u / (q + 1) : r + (u - wide) / q;
  }
};

// ---------------------------------------------------------------------------
// NG: groups of 32 elements of a head.  MT: rows of a wave's tile, 16 or 32.
// WR: waves that hold different rows of an item; the sets of WR waves take
// different pages.
// ---------------------------------------------------------------------------
template <int NG, int MT, int WR>
struct CaShape {
  static constexpr int D = NG * kGroup;
  static constexpr int Waves = WR == 1 ? 8 : 4;
  static constexpr int Threads = Waves * kWave;
  static constexpr int WK = Waves / WR;
  static constexpr int Rows = MT * WR;
  // A key's values in LDS.  The 16-byte pieces of a row are exchanged by the
  // row's number: 16 lanes that write the same piece of 16 rows, and 32 lanes
  // that read 32 or 64 bytes of 8 or 4 rows transposed, meet every bank.
  static constexpr int RowBytes = NG == 2 ? 128 : 256;
  __device__ static int swap(int row) {
    return 4 * (NG == 2 ? row / 2 % 2 : row % 4) ^ (2 * (row / 4 % 2) + row / 8 % 2);
  }
  static constexpr int PageBytes = kPage * RowBytes;
  static constexpr int Buffers = WR > 1 ? 2 : 1;
  static constexpr int ValueBytes = WK * Buffers * PageBytes;
  // Sums of a wave's rows on their way to be added to others': 16-byte pieces,
  // exchanged by the row's number as above.
  static constexpr int JoinRow = NG == 2 ? 256 : 512;
  __device__ static int join_at(int wave, int row, int d) {
    return (wave * MT + row) * JoinRow + 16 * ((d / 4) ^ (row % 16));
  }
  static constexpr int JoinBytes = WK > 1 ? Waves * MT * JoinRow : 4 * MT * OutRows<NG>::RowBytes;
  static constexpr int LdsBytes = ValueBytes > JoinBytes ? ValueBytes : JoinBytes;
  static constexpr int DT = MT == 32 ? NG : 2 * NG;        // tiles of D of the second product
  static constexpr int OR = MT == 32 ? 16 : 4;             // registers of one
  static constexpr int SPT = kPage / MT;                   // subtiles of MT keys in a page
  static constexpr int Steps = MT == 32 ? 2 * NG : NG;     // steps of the first product
  static constexpr int VPer = (NG + WR - 1) / WR;          // groups of values a wave unpacks
};

// Where in a head's row the first product's operand of step s begins for a
// lane: any order of the elements will do that is the same for both operands,
// and this one lets a lane take its keys' codes in 16-byte pieces.
template <int NG, int MT>
__device__ __forceinline__ int element_of(int s, int part) {
  if constexpr (MT == 32) {   // halves take the groups of a pair; an odd last group is halved
    if (NG % 2 == 0 || s < 4 * (NG / 2)) return 32 * (2 * (s / 4) + part) + 8 * (s % 4);
    return 32 * (NG - 1) + 16 * part + 8 * (s % 4);
  } else if constexpr (NG == 4) {   // a group a quarter
    return 32 * part + 8 * s;
  } else if constexpr (NG == 2) {   // half a group
    return 32 * (part / 2) + 16 * (part % 2) + 8 * s;
  } else {
    return 32 * s + 8 * part;
  }
}

// Codes and scales of one page for one lane: addresses are a uniform base and a
// 32-bit offset of the lane's.
template <int NG, int MT, int WR>
struct PageRegs {
  typedef CaShape<NG, MT, WR> S;
  uint32_t k[S::SPT][S::Steps];   // eight codes a step
  uint32_t ks[S::SPT];            // scales of the lane's key of a subtile
  u32x4 v[S::VPer];               // 32 codes of the values of key `lane`, a group each
  uint32_t vs;                    // and its scales

  __device__ __forceinline__ static const uint8_t* tile_of(const CacheAttnArgs& a, int page, int h) {
    const bool there = page >= 0 && page < a.n_pages;
    return a.cache + ((size_t)(there ? page : 0) * a.Hk + h) * tile_bytes(S::D);
  }
  __device__ __forceinline__ void load_k(const uint8_t* tile, int lane) {
    const uint32_t col = (uint32_t)lane % MT, part = (uint32_t)lane / MT;
    constexpr uint32_t kGroupBytes = kPage * kCodeBytes;
#pragma unroll
    for (int x = 0; x < S::SPT; ++x) {
      const uint8_t* codes = tile + x * MT * kCodeBytes;
      ks[x] = *(const uint32_t*)(tile + k_scales_at(S::D) + x * MT * scale_stride(S::D) + col * scale_stride(S::D));
      if constexpr (MT == 32 || NG == 4) {
        const uint32_t at = col * kCodeBytes + part * kGroupBytes;
#pragma unroll
        for (int i = 0; i < S::Steps / 4; ++i) {
          const u32x4 c = *(const u32x4*)(codes + i * 2 * kGroupBytes + at);
#pragma unroll
          for (int j = 0; j < 4; ++j) k[x][4 * i + j] = c[j];
        }
        if constexpr (S::Steps % 4 != 0) {
          const u32x2 c = *(const u32x2*)(codes + (NG - 1) * kGroupBytes + (col * kCodeBytes + 8 * part));
          k[x][S::Steps - 2] = c[0];
          k[x][S::Steps - 1] = c[1];
        }
      } else if constexpr (NG == 2) {
        const u32x2 c = *(const u32x2*)(codes + (col * kCodeBytes + (part / 2) * kGroupBytes + 8 * (part % 2)));
        k[x][0] = c[0];
        k[x][1] = c[1];
      } else {
#pragma unroll
        for (int s = 0; s < S::Steps; ++s)
          k[x][s] = *(const uint32_t*)(codes + s * kGroupBytes + (col * kCodeBytes + 4 * part));
      }
    }
  }
  __device__ __forceinline__ void load_v(const uint8_t* tile, int lane, int wr) {
    static_assert(kPage == kWave, "a lane a key");
    vs = *(const uint32_t*)(tile + v_scales_at(S::D) + (uint32_t)lane * scale_stride(S::D));
#pragma unroll
    for (int i = 0; i < S::VPer; ++i) {
      const int g = min(i * WR + wr, NG - 1);
      v[i] = *(const u32x4*)(tile + codes_bytes(S::D) + g * kPage * kCodeBytes + (uint32_t)lane * kCodeBytes);
    }
  }
};

__device__ __forceinline__ u32x4 unpack8(uint32_t c, float s) {
  u32x4 y;
  y[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, s, 0));
  y[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, s, 1));
  y[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, s, 2));
  y[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, s, 3));
  return y;
}

// Tree: what a row sees is told by its words of the mask (fdllm_tree_attention), at
// the pages with nodes alone: 64 trees of 30 to 32 nodes over 6000 to 8192 keys, 32
// heads over 8 of 128, 250 us, 0.92 PFLOP/s, bound as blocks are.
// Whole: a workgroup takes one item instead of an equal share of all.
template <int NG, int MT, int WR, bool Tree, bool Whole>
__global__ void __launch_bounds__((CaShape<NG, MT, WR>::Threads), 2)
k_cache_attn(const CacheAttnArgs a) {
  typedef CaShape<NG, MT, WR> S;
  constexpr int D = S::D, SPT = S::SPT, WK = S::WK;
  typedef typename std::conditional<MT == 32, f32x16, f32x4>::type Acc;
  extern __shared__ __align__(16) uint8_t s_mem[];
  __shared__ int s_sum[kCaMaxWaves], s_at[2];
  __shared__ float s_ml[S::Waves][MT][2];

  const int tid = threadIdx.x, lane = tid % kWave, wave = __builtin_amdgcn_readfirstlane(tid / kWave);
  const int wr = wave % WR, wk = wave / WR;   // its rows, its pages
  const int col = lane % MT, part = lane / MT;

  // Units of all sequences, this workgroup's share of them, and the sequence of
  // its first: a lane (of all waves, from 65 sequences on) counts a few
  // neighbouring sequences, a scan adds up.
  const bool apart = Whole || a.B <= kWave;   // every wave by itself
  const int who = apart ? lane : tid, per = apart ? 1 : (a.B + S::Threads - 1) / S::Threads;
  const int b0 = who * per, b1 = min(b0 + per, a.B);
  int mine = 0;
  for (int i = b0; i < b1; ++i) mine += sequence<S::Rows>(a, i).units(a.Hk);
  int incl = mine;
#pragma unroll
  for (int x = 1; x < kWave; x <<= 1) {
    const int y = __shfl_up(incl, x);
    if (lane >= x) incl += y;
  }
  int units = __builtin_amdgcn_readlane(incl, kWave - 1);
  if (!apart) {
    if (lane == kWave - 1) s_sum[wave] = incl;
    __syncthreads();
    units = 0;
#pragma unroll
    for (int w = 0; w < S::Waves; ++w) {
      if (w == wave) incl += units;
      units += s_sum[w];
    }
  }
  if (!Whole && units == 0) return;
  const Shares shares(Whole ? 1 : units, gridDim.x);
  int u_begin = shares.begin(blockIdx.x), u_end = shares.begin(blockIdx.x + 1);
  if (!Whole && a.plan && blockIdx.x == 0 && tid == 0) a.plan[0] = units;
  if (!Whole && u_begin >= u_end) return;
  int b, before;
  const bool here = u_begin >= incl - mine && u_begin < incl;
  if constexpr (Whole) {
    b = blockIdx.x / a.whole;
    before = 0;
    const Seq its = sequence<S::Rows>(a, b);
    const int item = blockIdx.x % a.whole, each = its.pages + kItemUnits;
    if (item >= its.groups * a.Hk) return;
    u_begin = item * each;
    u_end = u_begin + each;
  } else if (apart) {
    b = __ffsll((unsigned long long)__ballot(here)) - 1;
    before = __builtin_amdgcn_readlane(incl - mine, b);
  } else {
    if (here) {
      int i = b0, n = incl - mine;
      for (;; ++i) {
        const int k = sequence<S::Rows>(a, i).units(a.Hk);
        if (u_begin < n + k) break;
        n += k;
      }
      s_at[0] = i;
      s_at[1] = n;
    }
    __syncthreads();
    b = __builtin_amdgcn_readfirstlane(s_at[0]);
    before = __builtin_amdgcn_readfirstlane(s_at[1]);
  }
  Seq seq = sequence<S::Rows>(a, b);

  // Where a lane reads its part of a page's values: a group of 16 lanes reads
  // four keys by 16 elements, transposed.
  int v_at[S::DT];
  {
    const int row = 4 * part + (lane % 16) / 4, piece = (MT == 32 ? 2 * ((lane / 16) % 2) : 0) + (lane % 4) / 2;
#pragma unroll
    for (int t = 0; t < S::DT; ++t)
      v_at[t] = row * S::RowBytes + 16 * ((piece + t * MT / 8) ^ S::swap(row)) + 8 * (lane % 2);
  }

  int u = u_begin;
  int slot = 0;                       // of the next partial result
  int buf = 0;                        // of values in LDS; goes on from item to item, so that one barrier a page will do
  while (u < u_end) {
    while (u >= before + seq.units(a.Hk)) {
      before += seq.units(a.Hk);
      seq = sequence<S::Rows>(a, ++b);
    }
    const int each = seq.pages + kItemUnits, item = (u - before) / each;
    const int at = u - before - item * each, upto = min(each, at + (u_end - u));
    if (!Whole && a.plan && u == before && tid == 0) a.plan[1 + b] = before;   // for the join
    u += upto - at;
    const int page0 = max(0, at - kItemEnds), page1 = min(seq.pages, upto - kItemEnds);
    if (page1 <= page0) continue;
    const int h = item % a.Hk, group = item / a.Hk;

    // ---- the item's rows ----
    const int r = (group * WR + wr) * MT + col;             // row of this lane
    const bool row_ok = r < seq.n * a.R;
    const int tok = row_ok ? r / a.R : 0, head = h * a.R + (row_ok ? r % a.R : 0);
    int end = 0, all_see;                                   // keys that every row of the wave sees
    if constexpr (Tree) {
      all_see = seq.context();
    } else {
      const int start = a.q_start ? a.q_start[b] : seq.len - seq.n;
      const int pos = start > INT32_MAX - tok ? INT32_MAX : start + tok;
      end = row_ok ? visible_end(pos, a.blk, seq.len) : 0;
      all_see = row_ok ? end : INT32_MAX;
#pragma unroll
      for (int x = 1; x < MT; x <<= 1) all_see = min(all_see, __shfl_xor(all_see, x));
      all_see = __builtin_amdgcn_readfirstlane(all_see);
    }
    Acc o[S::DT];
#pragma unroll
    for (int t = 0; t < S::DT; ++t) o[t] = Acc{};
    float ref = kRefFloor, l = 0.0f, l2 = 0.0f;   // weights are 2^(c s - ref), l and l2 their sums

    // A wave behind a request's last rows only unpacks values and keeps step (24
    // requests of 40 nodes, 7 heads a key head, over 3000 keys 78 -> 72 us).
    const bool idle = Tree && WR > 1 && (group * WR + wr) * MT >= seq.n * a.R;

    // ---- the pages ----
    const int32_t* table = a.table + (size_t)b * a.table_w;
    // of a page whose tokens all lie past the sequence's end the table says nothing
    // The pages' numbers, 64 at a time, a lane each: a load for every page would
    // have to be waited for behind the page before.
    int ids_at = page0, ids = -1;
    const auto load_ids = [&]() {
      const int pg = ids_at + lane;
      ids = pg < page1 && pg * kPage < seq.len ? table[pg] : -1;
      // waited for here, so that nobody waits behind the branch
      asm volatile("s_waitcnt vmcnt(0)" : "+v"(ids));
    };
    const auto page_id = [&](int pg) {
      if (pg - ids_at >= kWave) {
        ids_at = pg;
        load_ids();
      }
      return __builtin_amdgcn_readlane(ids, pg - ids_at);
    };
    load_ids();
    PageRegs<NG, MT, WR> next;
    int id = page_id(page0 + wk), next_id = page_id(page0 + wk + WK);
    const uint8_t* tile = next.tile_of(a, id, h);
    next.load_k(tile, lane);
    CA_FENCE();
    next.load_v(tile, lane, wr);   // after the keys here too: the loop waits for its loads in this order
    CA_FENCE();
    bf16x8 q[S::Steps];
    {
      const uint16_t* qrow = a.q + (size_t)(seq.first + tok) * a.q_stride + (size_t)head * D;
#pragma unroll
      for (int s = 0; s < S::Steps; ++s) {
        q[s] = bf16x8{};
        if (row_ok) q[s] = *(const bf16x8*)(qrow + element_of<NG, MT>(s, part));
      }
    }
    unsigned long long word0 = 0;   // of the row's mask (at hand before the loop: in it a load waits for all those under way)
    if (Tree && row_ok) word0 = a.masks[(size_t)(seq.first + tok) * a.mask_w];
    // sets of waves without a page left go along while others' barriers run
    for (int pg = page0 + wk; WR == 1 ? pg < page1 : pg - wk < page1; pg += WK) {
      const int base = pg * kPage;
      const bool there = id >= 0 && id < a.n_pages;
      uint8_t* lds = s_mem + (wk * S::Buffers + buf) * S::PageBytes;
      if (S::Buffers > 1) buf ^= 1;

      // scores: a step's keys are unpacked while the one before is multiplied
      Acc sc[SPT];
      if (!idle) {
#pragma unroll
        for (int x = 0; x < SPT; ++x) {
          bf16x8 kf;
#pragma unroll
          for (int s = 0; s < S::Steps; ++s) {
            const int g = MT == 32 ? (NG % 2 == 0 || s < 4 * (NG / 2) ? 2 * (s / 4) + part : NG - 1)
                                   : NG == 4 ? part : NG == 2 ? part / 2 : s;
            const float ksv = scale_of((next.ks[x] >> (8 * g)) & 255u);
            kf = __builtin_bit_cast(bf16x8, unpack8(next.k[x][s], ksv));
            const Acc from = s ? sc[x] : Acc{};
            if constexpr (MT == 32) sc[x] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf, q[s], from, 0, 0, 0);
            else sc[x] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, q[s], from, 0, 0, 0);
            if (s % 2) CA_FENCE();
          }
        }
      }
      // the registers of what is used are loaded for the next page at once
      id = next_id;
      tile = next.tile_of(a, id, h);
      next.load_k(tile, lane);
      CA_FENCE();

      // values: a lane unpacks 32 elements of a key.  Keys past the end get a
      // scale of next to nothing: their weight is 0, and a code is finite.
#pragma unroll
      for (int i = 0; i < S::VPer; ++i) {
        const int g = i * WR + wr;
        if (NG % WR != 0 && g >= NG) break;
        const float sv = scale_of(there && base + lane < seq.len ? (next.vs >> (8 * g)) & 255u : 1u);
#pragma unroll
        for (int j = 0; j < 4; ++j)
          *(u32x4*)(lds + lane * S::RowBytes + 16 * ((4 * g + j) ^ S::swap(lane))) = unpack8(next.v[i][j], sv);
        CA_FENCE();
      }
      next.load_v(tile, lane, wr);
      next_id = page_id(pg + 2 * WK);
      CA_FENCE();

      if (!idle) {
        // keys that a row does not see
        if (!there || base + kPage > all_see) {
          if constexpr (Tree) {
            unsigned long long seen = 0;
            if (there && row_ok)
              seen = tree_window(a.masks + (size_t)(seq.first + tok) * a.mask_w, word0, seq.n, base, seq.context()) >> (4 * part);
#pragma unroll
            for (int x = 0; x < SPT; ++x)
#pragma unroll
              for (int i = 0; i < S::OR; ++i) {
                const int key = x * MT + (MT == 32 ? i % 4 + 8 * (i / 4) : i);   // less the lane's part, shifted out
                sc[x][i] = (uint32_t)(seen >> (key & 32)) >> (key & 31) & 1u ? sc[x][i] : kNegInf;
              }
          } else {
            const int seen = there ? end - base : 0;
#pragma unroll
            for (int x = 0; x < SPT; ++x)
#pragma unroll
              for (int i = 0; i < S::OR; ++i) {
                const int key = x * MT + (MT == 32 ? i % 4 + 8 * (i / 4) + 4 * part : 4 * part + i);
                sc[x][i] = key < seen ? sc[x][i] : kNegInf;
              }
          }
        }
        // The running reference follows the maximum only where that has grown by
        // more than 2^8: weights up to 256 lose nothing in floating point, and
        // the sums are rescaled a few times instead of with every page.
        float top = kNegInf;
#pragma unroll
        for (int x = 0; x < SPT; ++x)
#pragma unroll
          for (int i = 0; i < S::OR; i += 2) top = fmaxf(fmaxf(top, sc[x][i]), sc[x][i + 1]);
        top = max_row<MT>(top) * a.c;
        if (__any(top > ref + 8.0f)) {
          const float to = fmaxf(ref, top);
          const float f = __builtin_amdgcn_exp2f(ref - to);
          ref = to;
          l *= f;
          l2 *= f;
#pragma unroll
          for (int t = 0; t < S::DT; ++t)
#pragma unroll
            for (int i = 0; i < S::OR; ++i) o[t][i] *= f;
        }
      }
      if (WR > 1) __syncthreads();
      else __builtin_amdgcn_wave_barrier();
      if (idle) continue;

      // outputs: the weights of a step of 16 (32) keys are formed beside the
      // products of the one before.  Rounded to bfloat16, the type of the values
      // that they meet in one product (the sums take them unrounded): over many
      // keys an output is off by 0.0019 to 0.0022 relative, 0.0017 in 32 bits
      // rounded once; in two pieces they would double this product.
      u32x4 p[2];
      const auto weigh = [&](int k, int i) {   // pair i of step k
        const int x = MT == 32 ? k / 2 : 2 * k + i / 2, at = MT == 32 ? 8 * (k % 2) + 2 * i : 2 * (i % 2);
        const float y = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[x][at], a.c, -ref));
        const float z = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[x][at + 1], a.c, -ref));
        l += y;
        l2 += z;
        p[k % 2][i] = pack_bf16(y, z);
      };
      constexpr int KS = MT == 32 ? 4 : 2, NP = KS * S::DT;
      const auto value_operand = [&](int i) {   // of product i: transposed reads, the second 8 (16) keys on
        const int k = i / S::DT, t = i % S::DT;
        const uint8_t* at = lds + k * (MT == 32 ? 16 : 32) * S::RowBytes;
        const i16x4 v0 = read_transposed(at + v_at[t]);
        const i16x4 v1 = read_transposed(at + (MT == 32 ? 8 * S::RowBytes + (v_at[t] ^ 16) : 16 * S::RowBytes + v_at[t]));
        return __builtin_bit_cast(bf16x8, __builtin_shufflevector(v0, v1, 0, 1, 2, 3, 4, 5, 6, 7));
      };
      __builtin_amdgcn_s_setprio(1);
      bf16x8 vf[3];
      vf[0] = value_operand(0);
      vf[1] = value_operand(1);
      CA_FENCE();
#pragma unroll
      for (int i = 0; i < 4; ++i) weigh(0, i);
      CA_FENCE();
#pragma unroll
      for (int i = 0; i < NP; ++i) {
        const int k = i / S::DT, t = i % S::DT;
        if (i + 2 < NP) vf[(i + 2) % 3] = value_operand(i + 2);
        const bf16x8 pf = __builtin_bit_cast(bf16x8, p[k % 2]);
        if constexpr (MT == 32) o[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[i % 3], pf, o[t], 0, 0, 0);
        else o[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf[i % 3], pf, o[t], 0, 0, 0);
        CA_FENCE();
        if (k + 1 < KS) {
#pragma unroll
          for (int w = t * 4 / S::DT; w < (t + 1) * 4 / S::DT; ++w) weigh(k + 1, w);
        }
        CA_FENCE();
      }
      __builtin_amdgcn_s_setprio(0);
    }
    l = sum_row<MT>(l + l2);

    // ---- results: final where the item is whole, a partial sum otherwise ----
    const bool whole = page0 == 0 && page1 == seq.pages;
    const size_t tile0 = ((size_t)blockIdx.x * 2 + slot) * WR;   // of partial results
    constexpr int Quads = quads_of(MT, NG);
    if constexpr (WK > 1) {
      // the sets of waves join: every row's sums brought to one reference, added
      // up out of LDS
      if (part == 0) s_ml[wave][col][0] = ref, s_ml[wave][col][1] = l;
      __syncthreads();
      float to = ref;
#pragma unroll
      for (int w = 0; w < WK; ++w) to = fmaxf(to, s_ml[w * WR + wr][col][0]);
      const float f = __builtin_amdgcn_exp2f(ref - to);
#pragma unroll
      for (int q = 0; q < Quads; ++q) {
        const int i = 4 * q % S::OR, t = 4 * q / S::OR;
        *(f32x4*)(s_mem + S::join_at(wave, col, quad_element<MT>(q, part))) =
            f32x4{o[t][i] * f, o[t][i + 1] * f, o[t][i + 2] * f, o[t][i + 3] * f};
      }
      __syncthreads();
      const auto joined = [&](int w0, int row, int d) {
        f32x4 v = *(const f32x4*)(s_mem + S::join_at(w0, row, d));
#pragma unroll
        for (int w = 1; w < WK; ++w) v += *(const f32x4*)(s_mem + S::join_at(w * WR + w0, row, d));
        return v;
      };
      const auto joined_ml = [&](int w0, int row) {
        float m = kRefFloor, n = 0.0f;
#pragma unroll
        for (int w = 0; w < WK; ++w) m = fmaxf(m, s_ml[w * WR + w0][row][0]);
#pragma unroll
        for (int w = 0; w < WK; ++w)
          n += s_ml[w * WR + w0][row][1] * __builtin_amdgcn_exp2f(s_ml[w * WR + w0][row][0] - m);
        return float2{m, n};
      };
      if (whole) {
        for (int x = tid; x < S::Rows * (D / 4); x += S::Threads) {
          const int row = x / (D / 4), d = 4 * (x % (D / 4)), rr = group * S::Rows + row;
          if (rr >= seq.n * a.R) break;
          const f32x4 v = joined(row / MT, row % MT, d);
          const float2 ml = joined_ml(row / MT, row % MT);
          const float inv = inverse_sum(ml.y);
          const size_t to_row = (size_t)(seq.first + rr / a.R) * a.H + h * a.R + rr % a.R;
          *(u32x2*)(a.out + to_row * D + d) = u32x2{pack_bf16(v[0] * inv, v[1] * inv), pack_bf16(v[2] * inv, v[3] * inv)};
          if (a.lse && d == 0) a.lse[to_row] = log_sum(ml.x, ml.y);
        }
      } else {
        for (int x = wave; x < WR * Quads; x += S::Waves) {
          const int w0 = x / Quads, q = x % Quads;
          *(f32x4*)(a.part + ((tile0 * Quads + x) * kWave + lane) * 4) = joined(w0, col, quad_element<MT>(q, part));
          if (q == 0 && part == 0) *(float2*)(a.part_ml + ((tile0 + w0) * MT + col) * 2) = joined_ml(w0, col);
        }
      }
      __syncthreads();
    } else if (whole) {
      // through LDS, so that a row leaves in one piece
      __syncthreads();
      const float inv = inverse_sum(l);
      uint8_t* lds = s_mem + wave * MT * OutRows<NG>::RowBytes;
#pragma unroll
      for (int q = 0; q < Quads; ++q) {
        const int i = 4 * q % S::OR, t = 4 * q / S::OR;
        *(u32x2*)(lds + OutRows<NG>::at(col, quad_element<MT>(q, part))) =
            u32x2{pack_bf16(o[t][i] * inv, o[t][i + 1] * inv), pack_bf16(o[t][i + 2] * inv, o[t][i + 3] * inv)};
      }
      __builtin_amdgcn_wave_barrier();
      const size_t at = (size_t)(seq.first + tok) * a.H + head;
      if (row_ok && a.lse && part == 0) a.lse[at] = log_sum(ref, l);
      for (int x = lane; x < MT * (D / 8); x += kWave) {
        const int row = x / (D / 8), d = 8 * (x % (D / 8)), rr = (group * WR + wr) * MT + row;
        if (rr >= seq.n * a.R) break;
        const size_t to_row = (size_t)(seq.first + rr / a.R) * a.H + h * a.R + rr % a.R;
        *(u32x4*)(a.out + to_row * D + d) = *(const u32x4*)(lds + OutRows<NG>::at(row, d));
      }
      __syncthreads();
    } else {
#pragma unroll
      for (int q = 0; q < Quads; ++q) {
        const int i = 4 * q % S::OR, t = 4 * q / S::OR;
        *(f32x4*)(a.part + (((tile0 + wr) * Quads + q) * kWave + lane) * 4) =
            f32x4{o[t][i], o[t][i + 1], o[t][i + 2], o[t][i + 3]};
      }
      if (part == 0) *(float2*)(a.part_ml + ((tile0 + wr) * MT + col) * 2) = float2{ref, l};
    }
    slot = 1;
  }
}

// Joins the partial results of an item that several workgroups share, always
// in the same order.  A workgroup takes the MT rows of a wave's tile, as they
// lay in its registers.  Where items lie in many shares, Split sets of its
// waves divide the parts (a part costs a round trip to memory, so as many as
// possible are under way at once), and a workgroup takes 32 of a head's elements;
// where they lie in two or so, every wave has quads of its own.
constexpr int kCaJoinWaves = 8;

template <int NG, int MT, int WR, int Split>
__global__ void __launch_bounds__(kCaJoinWaves* kWave)
k_cache_join(const CacheAttnArgs a, int wgs) {
  constexpr int D = NG * kGroup, Quads = quads_of(MT, NG), Rows = MT * WR;
  constexpr int Own = Split > 1 ? quads_of(MT, 1) : Quads;   // quads of the workgroup, from q0 on
  constexpr int Sets = kCaJoinWaves / Split;              // of waves, by quads
  constexpr int QPer = (Own + Sets - 1) / Sets;
  const int q0 = Split > 1 ? blockIdx.z * Own : 0;
  __shared__ __align__(16) uint8_t s_out[MT * OutRows<NG>::RowBytes];
  __shared__ f32x4 s_acc[Split > 1 ? Sets * (Split - 1) : 1][QPer][kWave];
  __shared__ float s_ml[kCaJoinWaves][MT][2];
  const int b = blockIdx.y;
  const int item = blockIdx.x / WR, wr = blockIdx.x % WR;
  const Seq seq = sequence<Rows>(a, b);
  if (item >= seq.groups * a.Hk) return;
  const int h = item % a.Hk, group = item / a.Hk;
  const int r0 = (group * WR + wr) * MT;                  // the tile's first row
  if (r0 >= seq.n * a.R) return;
  const Shares shares(a.plan[0], wgs);
  const int u0 = a.plan[1 + b] + item * (seq.pages + kItemUnits);
  const int g0 = shares.of(u0 + kItemEnds), g1 = shares.of(u0 + kItemEnds + seq.pages - 1);
  if (g0 == g1) return;
  const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int col = lane % MT, part = lane / MT;
  const int sp = wave % Split, set = wave / Split;
  // it is its first share's second result where that holds pages of the item before
  const int first = (g0 * 2 + (shares.begin(g0) < u0 - kItemEnds ? 1 : 0)) * WR + wr;
  const auto tile_of = [&](int g) { return (size_t)(g == g0 ? first : g * 2 * WR + wr); };
  f32x4 acc[QPer];
#pragma unroll
  for (int i = 0; i < QPer; ++i) acc[i] = f32x4{};
  float ref = kRefFloor, l = 0.0f;
  constexpr int Ahead = 4;
  struct Parts {
    float2 ml[Ahead];
    f32x4 v[Ahead][QPer];
  };
  const auto load = [&](int g, Parts& p) {
#pragma unroll
    for (int k = 0; k < Ahead; ++k) {
      const size_t tile = tile_of(min(g + k, g1));
      p.ml[k] = *(const float2*)(a.part_ml + (tile * MT + col) * 2);
#pragma unroll
      for (int i = 0; i < QPer; ++i)
        p.v[k][i] = *(const f32x4*)(a.part + ((tile * Quads + q0 + min(set * QPer + i, Own - 1)) * kWave + lane) * 4);
    }
  };
  Parts p, next;   // in many shares the next ones are under way
  if constexpr (Split > 1) load(g0 + sp * Ahead, next);
  for (int g = g0 + sp * Ahead; g <= g1; g += Split * Ahead) {
    if constexpr (Split > 1) {
      p = next;
      if (g + Split * Ahead <= g1) load(g + Split * Ahead, next);
    } else {
      load(g, p);
    }
    float to = ref;
#pragma unroll
    for (int k = 0; k < Ahead; ++k) to = fmaxf(to, p.ml[k].x);
    const float f0 = __builtin_amdgcn_exp2f(ref - to);
    ref = to;
    l *= f0;
#pragma unroll
    for (int i = 0; i < QPer; ++i) acc[i] *= f0;
#pragma unroll
    for (int k = 0; k < Ahead; ++k) {
      const float f = g + k <= g1 ? __builtin_amdgcn_exp2f(p.ml[k].x - ref) : 0.0f;
      l += f * p.ml[k].y;
#pragma unroll
      for (int i = 0; i < QPer; ++i) acc[i] += p.v[k][i] * f;
    }
  }
  if constexpr (Split > 1) {
    if (part == 0) s_ml[wave][col][0] = ref, s_ml[wave][col][1] = l;
    if (sp > 0) {
#pragma unroll
      for (int i = 0; i < QPer; ++i) s_acc[set * (Split - 1) + sp - 1][i][lane] = acc[i];
    }
    __syncthreads();
    float to = kRefFloor;
#pragma unroll
    for (int w = 0; w < Split; ++w) to = fmaxf(to, s_ml[set * Split + w][col][0]);
    const float f0 = __builtin_amdgcn_exp2f(ref - to);
    l *= f0;
#pragma unroll
    for (int i = 0; i < QPer; ++i) acc[i] *= f0;
#pragma unroll
    for (int w = 1; w < Split; ++w) {   // (of use to the first wave of a set)
      const float f = __builtin_amdgcn_exp2f(s_ml[set * Split + w][col][0] - to);
      l += f * s_ml[set * Split + w][col][1];
#pragma unroll
      for (int i = 0; i < QPer; ++i) acc[i] += s_acc[set * (Split - 1) + w - 1][i][lane] * f;
    }
    ref = to;
  }
  // out through LDS, so that a row leaves in one piece
  const float inv = inverse_sum(l);
  if (sp == 0) {
#pragma unroll
    for (int i = 0; i < QPer; ++i) {
      const int q = set * QPer + i;
      if (q < Own)
        *(u32x2*)(s_out + OutRows<NG>::at(col, quad_element<MT>(q0 + q, part))) =
            u32x2{pack_bf16(acc[i][0] * inv, acc[i][1] * inv), pack_bf16(acc[i][2] * inv, acc[i][3] * inv)};
    }
    const int r = r0 + col;
    if (set == 0 && q0 == 0 && part == 0 && a.lse && r < seq.n * a.R)
      a.lse[(size_t)(seq.first + r / a.R) * a.H + h * a.R + r % a.R] =
          log_sum(ref, l);
  }
  __syncthreads();
  constexpr int Pieces = (Split > 1 ? kGroup : D) / 8;   // of 16 bytes a row
  const int d0 = Split > 1 ? blockIdx.z * kGroup : 0;
  for (int x = threadIdx.x; x < MT * Pieces; x += kCaJoinWaves * kWave) {
    const int row = x / Pieces, d = d0 + 8 * (x % Pieces), r = r0 + row;
    if (r >= seq.n * a.R) break;
    const size_t at = (size_t)(seq.first + r / a.R) * a.H + h * a.R + r % a.R;
    *(u32x4*)(a.out + at * D + d) = *(const u32x4*)(s_out + OutRows<NG>::at(row, d));
  }
}

// ---------------------------------------------------------------------------
// host side
// ---------------------------------------------------------------------------
// Pages a set of waves up to which items stay whole, where there is one sequence:
// without parts there is no join, which costs as much as two or three pages.
// Counted by the width of the page table, all that the host knows of a length.  (32 heads, one token: 12.6 us divided and 9.3 whole at 1024 keys,
// two pages a set; 13.3 and 12.7 at 2048, four; 15.6 and 20.3 at 4096, eight.
// A block of 32: 14.6 and 12.3, 16.0 and 16.5, 22.0 and 24.9.)
constexpr int kCaWholePages = 4;

struct CaPlan {
  int mt, wr;        // variant
  int wgs;           // workgroups
  int items;         // items of a sequence with max_q query tokens
  bool join, split;  // whether items may lie in several shares; in many
  size_t at_ml, at_part, bytes;
};

static bool ca_sizes_ok(int B, int H, int Hk, int D, int max_q, int table_w, int n_pages) {
  if (D != 64 && D != 96 && D != 128) return false;
  if (H % Hk || H > (1 << 15) || B > 65535) return false;
  if (table_w > INT32_MAX / kPage || n_pages > INT32_MAX / kPage) return false;
  const long long rows = (long long)max_q * (H / Hk);
  const long long groups = (rows + 15) / 16;
  if (rows > (1 << 24) || groups * Hk > INT32_MAX / 2) return false;
  // units of work are counted in 32 bits
  const double units = (double)B * (table_w + 1.0 + kItemUnits) * (double)groups * Hk;
  return units < 2.0e9;
}

static CaPlan ca_plan(int B, int H, int Hk, int D, int max_q, int table_w, int most_wr = 4) {
  CaPlan p{};
  const long long rows = (long long)max_q * (H / Hk);
  p.mt = rows <= 16 ? 16 : 32;
  p.wr = rows <= 32 ? 1 : rows <= 64 ? 2 : most_wr;
  const int per = p.mt * p.wr;
  const long long groups = (rows + per - 1) / per;
  p.items = (int)(groups * Hk);
  const int waves = p.wr == 1 ? 8 : 4, wk = waves / p.wr;
  // shares of at least one page for each set of waves, eight waves a CU
  const long long items = (long long)B * p.items, most = items * ((table_w + wk - 1) / wk);
  const int fill = 256 * 8 / waves;
  p.wgs = (int)(most < fill ? (most < 1 ? 1 : most) : fill);
  if (B == 1 && groups == 1 && items <= fill && table_w <= kCaWholePages * wk) p.wgs = (int)items;
  // None is split where there is one share, where an item has no more than a
  // page, or where one sequence of one group of rows has an item a share.  (With
  // more groups it may have fewer items than max_q stands for, and shares that
  // begin inside one.)
  p.join = p.wgs > 1 && table_w > 1 && !(B == 1 && groups == 1 && p.wgs == items);
  p.split = p.wgs >= 4 * items;
  if (!p.join) return p;
  const size_t rows_out = (size_t)p.wgs * 2 * per;
  p.at_ml = align256(((size_t)B + 1) * 4);
  p.at_part = p.at_ml + align256(rows_out * 8);
  p.bytes = p.at_part + rows_out * D * sizeof(float);
  return p;
}

// Trees: items stay whole, a workgroup each, where the chip holds all of them at
// once, or half of them and their pages are few: no shares to find, no join, and
// eight sets of waves to a group of 32 rows, though the keys are read once a group
// then.  The fewer the items, the fewer pages: divided ones fill the chip.  (32 heads
// over 8 of 128; us divided and whole.  16 items: 500 keys 14.5 and 9.8, 2000 17.2 and
// 15.3, 3000 19.0 and 19.2, 4000 20.5 and 23.3.  64 items: 4000 25.2 and 23.6, 8000 29.6
// and 39.3.  128: 4000 29.2 and 25.2, 6000 33.0 and 32.5.  256: 1000 24.8 and 12.9, 8000
// 54.6 and 46.1.  512, twice what the chip holds: 500 27.5 and 20.2, 2000 40.3 and 32.9,
// 3000 47.0 and 42.4.  768: 200 20.6 and 24.8.  Heads of 64 and 96 go by these and by
// how many items the chip holds.)  Keys are counted by the table's width, all that the
// host knows of a length: 16 nodes over 500 keys take 9.6 us with a table of 9 pages and
// 13.0 with one of 64 to 2048, divided for lengths that are not there.
// Divided items of heads of 64 have 64 rows rather than 128, two sets of waves (16
// heads over 2, us with 128 rows and with 64: 2 x 26 nodes over 99000 to 131000 keys
// 50.8 and 49.2, 2 x 16 over 8000 18.7 and 15.8, 64 x 32 over 8000 96.9 and 92.9; heads
// of 96 and 128 lose by it, 64 blocks 261 and 302).
static CaPlan ca_tree_plan(int B, int H, int Hk, int D, int max_q, int table_w, int* whole) {
  const long long rows = (long long)max_q * (H / Hk);
  const int mt = rows <= 16 ? 16 : 32;
  const long long items = (rows + mt - 1) / mt * Hk, all = B * items;
  const int held = D == 64 ? 512 : 256;   // by LDS: two workgroups a CU, or one
  *whole = 0;
  const long long most = all <= held ? 32 + (all < 256 ? all : 256) / 2 : all <= 2 * held ? 64 : 0;
  if (table_w > most) {
    const CaPlan wide = ca_plan(B, H, Hk, D, max_q, table_w), narrow = ca_plan(B, H, Hk, D, max_q, table_w, D == 64 ? 2 : 4);
    return narrow.bytes <= wide.bytes ? narrow : wide;   // (the workspace is asked for by the wide plan)
  }
  CaPlan p{};
  p.mt = mt, p.wr = 1;
  p.items = *whole = (int)items;
  p.wgs = (int)all;
  return p;
}

// The join's workgroups, one a wave's rows of an item, in what a launch has room
// for: 2^32 threads.
static bool ca_join_ok(const CaPlan& p) {
  return !p.join || (long long)p.items * p.wr < (1ll << 32) / (kCaJoinWaves * kWave);
}

// The attention kernels' LDS is above the default limit; the limit is raised
// once per device and kernel, before the first launch there.
constexpr int kCaMaxDevices = 64;

template <int NG, int MT, int WR, bool Tree, bool Whole = false>
static hipError_t ca_launch_one(const CacheAttnArgs& a, const CaPlan& p, hipStream_t st) {
  typedef CaShape<NG, MT, WR> S;
  static std::atomic<bool> allowed[kCaMaxDevices];
  int dev = 0;
  hipError_t e = hipGetDevice(&dev);
  if (e != hipSuccess) return e;
  if (dev < 0 || dev >= kCaMaxDevices || !allowed[dev].load(std::memory_order_acquire)) {
    e = hipFuncSetAttribute((const void*)k_cache_attn<NG, MT, WR, Tree, Whole>, hipFuncAttributeMaxDynamicSharedMemorySize,
                            S::LdsBytes);
    if (e != hipSuccess) return e;
    if (dev >= 0 && dev < kCaMaxDevices) allowed[dev].store(true, std::memory_order_release);
  }
  hipLaunchKernelGGL((k_cache_attn<NG, MT, WR, Tree, Whole>), dim3((unsigned)p.wgs), dim3(S::Threads), S::LdsBytes, st, a);
  const dim3 join((unsigned)(p.items * WR), (unsigned)a.B, p.split ? NG : 1), threads(kCaJoinWaves * kWave);
  if (p.join && p.split) hipLaunchKernelGGL((k_cache_join<NG, MT, WR, 4>), join, threads, 0, st, a, p.wgs);
  else if (p.join) hipLaunchKernelGGL((k_cache_join<NG, MT, WR, 1>), join, threads, 0, st, a, p.wgs);
  return hipGetLastError();
}

template <int NG, bool Tree>
static hipError_t ca_launch(const CacheAttnArgs& a, const CaPlan& p, hipStream_t st) {
  if constexpr (Tree) {
    if (a.whole) return p.mt == 16 ? ca_launch_one<NG, 16, 1, true, true>(a, p, st) : ca_launch_one<NG, 32, 1, true, true>(a, p, st);
  }
  if (p.mt == 16) return ca_launch_one<NG, 16, 1, Tree>(a, p, st);
  if (p.wr == 1) return ca_launch_one<NG, 32, 1, Tree>(a, p, st);
  if (p.wr == 2) return ca_launch_one<NG, 32, 2, Tree>(a, p, st);
  return ca_launch_one<NG, 32, 4, Tree>(a, p, st);
}

// Both calls: of a (masks, q_start, blk) either the masks or the others count.
template <bool Tree>
static fdllm_status ca_call(CacheAttnArgs a, int D, float scale, void* workspace, size_t workspace_bytes, fdllm_stream stream) {
  if (a.T < 0 || a.B < 0 || a.max_q < 0 || a.H < 1 || a.Hk < 1 || a.n_pages < 0 || a.table_w < 0 || a.blk < 0 || a.mask_w < 0)
    return FDLLM_ERR_INVALID_ARG;
  if (!(scale > 0.0f) || scale > 3.0e38f) return FDLLM_ERR_INVALID_ARG;
  if (!ca_sizes_ok(a.B, a.H, a.Hk, D, a.max_q, a.table_w, a.n_pages)) return FDLLM_ERR_SIZE;
  if (Tree && a.mask_w < (a.max_q + 63) / 64) return FDLLM_ERR_INVALID_ARG;
  if (a.T == 0 || a.B == 0 || a.max_q == 0) return FDLLM_OK;
  if (!a.q || !a.cu_q || !a.kv_len || !a.out || (a.table_w > 0 && !a.table) || !a.cache || a.n_pages < 1)
    return FDLLM_ERR_INVALID_ARG;
  if (Tree && (!a.masks || (uintptr_t)a.masks & 7)) return FDLLM_ERR_INVALID_ARG;
  if (a.q_stride < (int64_t)a.H * D || a.q_stride % 8) return FDLLM_ERR_INVALID_ARG;
  for (const void* p : {(const void*)a.q, (const void*)a.cache, (const void*)a.out, (const void*)workspace})
    if ((uintptr_t)p & 15) return FDLLM_ERR_INVALID_ARG;
  const CaPlan p = Tree ? ca_tree_plan(a.B, a.H, a.Hk, D, a.max_q, a.table_w, &a.whole)
                        : ca_plan(a.B, a.H, a.Hk, D, a.max_q, a.table_w);
  if (!ca_join_ok(p)) return FDLLM_ERR_SIZE;
  if (p.bytes && (!workspace || workspace_bytes < p.bytes)) return FDLLM_ERR_WORKSPACE;
  if constexpr (Tree) {
    // (out may be q itself: a workgroup has read an item's rows of q before it writes them,
    // and of an item that several have, it writes the join's scratch)
    const size_t row = (size_t)a.H * D * 2, counts = (size_t)a.B * 4;
    const bool itself = a.out == a.q && (a.T == 1 || (size_t)a.q_stride * 2 == row);
    size_t tile = 0;
    fdllm_cache_tile_bytes(D, &tile);
    if (!apart({{a.out, a.T * row}, {a.lse, (size_t)a.T * a.H * 4}},
               {{itself ? nullptr : a.q, row, (size_t)a.q_stride * 2, a.T}, {a.cache, (size_t)a.n_pages * a.Hk * tile},
                {a.table, counts * a.table_w}, {a.kv_len, counts}, {a.cu_q, counts + 4}, {a.masks, (size_t)a.T * 8 * a.mask_w},
                {workspace, p.bytes}}))
      return FDLLM_ERR_INVALID_ARG;
  }
  char* ws = (char*)workspace;
  a.R = a.H / a.Hk;
  a.c = scale * kLog2e;
  a.plan = p.join ? (int32_t*)ws : nullptr;
  a.part_ml = (float*)(ws + p.at_ml);
  a.part = (float*)(ws + p.at_part);
  hipStream_t st = (hipStream_t)stream;
  const hipError_t e = D == 64 ? ca_launch<2, Tree>(a, p, st) : D == 96 ? ca_launch<3, Tree>(a, p, st) : ca_launch<4, Tree>(a, p, st);
  return e == hipSuccess ? FDLLM_OK : FDLLM_ERR_HIP;
}

}  // namespace fdllm

using namespace fdllm;

extern "C" {

fdllm_status fdllm_cache_attention_workspace_size(int B, int H, int Hk, int D, int max_q, int table_width,
                                                  size_t* bytes) {
  if (!bytes || B < 0 || H < 1 || Hk < 1 || max_q < 0 || table_width < 0) return FDLLM_ERR_INVALID_ARG;
  if (!ca_sizes_ok(B, H, Hk, D, max_q, table_width, 0)) return FDLLM_ERR_SIZE;
  const CaPlan p = ca_plan(B, H, Hk, D, max_q, table_width);
  if (!ca_join_ok(p)) return FDLLM_ERR_SIZE;
  *bytes = p.bytes;
  return FDLLM_OK;
}

fdllm_status fdllm_cache_attention(const void* q, int64_t q_stride, int T, const int32_t* cu_q, int B, int max_q,
                                   int H, int Hk, int D, const uint8_t* cache, int n_pages,
                                   const int32_t* page_table, int table_width, const int32_t* kv_len,
                                   const int32_t* q_start, float scale, int blk, void* out, float* lse,
                                   void* workspace, size_t workspace_bytes, fdllm_stream stream) {
  CacheAttnArgs a{};
  a.q = (const uint16_t*)q, a.q_stride = q_stride, a.T = T, a.cache = cache, a.n_pages = n_pages, a.table = page_table;
  a.table_w = table_width, a.kv_len = kv_len, a.cu_q = cu_q, a.q_start = q_start, a.B = B, a.H = H, a.Hk = Hk;
  a.max_q = max_q, a.blk = blk, a.out = (uint16_t*)out, a.lse = lse;
  return ca_call<false>(a, D, scale, workspace, workspace_bytes, stream);
}

fdllm_status fdllm_tree_attention(const void* q, int64_t q_stride, int T, const int32_t* cu_q, int B, int max_q,
                                  int H, int Hk, int D, const uint8_t* cache, int n_pages,
                                  const int32_t* page_table, int table_width, const int32_t* kv_len,
                                  const uint64_t* masks, int mask_words, float scale, void* out, float* lse,
                                  void* workspace, size_t workspace_bytes, fdllm_stream stream) {
  CacheAttnArgs a{};
  a.q = (const uint16_t*)q, a.q_stride = q_stride, a.T = T, a.cache = cache, a.n_pages = n_pages, a.table = page_table;
  a.table_w = table_width, a.kv_len = kv_len, a.cu_q = cu_q, a.B = B, a.H = H, a.Hk = Hk, a.max_q = max_q;
  a.masks = (const unsigned long long*)masks, a.mask_w = mask_words, a.out = (uint16_t*)out, a.lse = lse;
  return ca_call<true>(a, D, scale, workspace, workspace_bytes, stream);
}

}  // extern "C"
