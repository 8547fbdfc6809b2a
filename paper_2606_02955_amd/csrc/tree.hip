// tree.hip -- around the attention of drafted trees on gfx950 (fdllm.h): who sees
// whom, positions and slots from the nodes' parents before the first layer, and
// the cache entries of what stands moved to their places behind the last.
#include <hip/hip_runtime.h>

#include <stdint.h>

#include "attn_common.h"
#include "fdllm.h"

namespace fdllm {

constexpr int kTlWords = 4;   // words of the masks at a time

struct LayoutArgs {
  const int32_t* parents;
  int T;
  const int32_t* cu_q;
  int B, max_q;
  const int32_t* kv_len;
  const int32_t* table;   // may be null
  int table_w;
  unsigned long long* masks;
  int words;
  int32_t* positions;     // may be null
  int32_t* slots;         // may be null
};

// The slot of a sequence's token, -1 without a page.
__device__ __forceinline__ int slot_of(const int32_t* table, int table_w, int b, int token) {
  if (token < 0 || token / kPage >= table_w) return -1;
  const int page = table[(size_t)b * table_w + token / kPage];
  return page >= 0 && page <= INT32_MAX / kPage - 1 ? page * kPage + token % kPage : -1;
}

// A workgroup a request, a thread a node.  A node's set of ancestors doubles its
// reach each round: with A_k(i) the first 2^k of the chain i, parent(i), ... and
// j_k(i) the node behind them, A_k+1(i) = A_k(i) or A_k(j_k(i)), so a chain of n
// takes log2 n rounds.  Latency-bound: 26 nodes 2.8 us, 64 trees of 100 to 250 5.4.
__global__ void __launch_bounds__(FDLLM_MAX_TREE)
k_tree_layout(const LayoutArgs a) {
  __shared__ unsigned long long s_set[kTlWords][FDLLM_MAX_TREE];
  __shared__ int16_t s_jump[FDLLM_MAX_TREE];
  const int b = blockIdx.x, i = threadIdx.x;
  int first;
  const int n = packed_rows(a.cu_q, b, a.T, a.max_q, &first);
  if (n == 0) return;
  const bool node = i < n;
  int parent = node ? a.parents[first + i] : -1;
  if (parent < -1 || parent >= i) parent = -1;
  const int context = max(a.kv_len[b], 0) - n;
  int seen = 0;
  for (int w0 = 0; w0 < a.words; w0 += kTlWords) {
    unsigned long long set[kTlWords];
#pragma unroll
    for (int w = 0; w < kTlWords; ++w) set[w] = i / 64 == w0 + w ? 1ull << (i % 64) : 0ull;
    int jump = parent;
    // (words behind the last node's have nothing)
    while (w0 * 64 < n && __syncthreads_or(jump >= 0)) {
      if (node) {
#pragma unroll
        for (int w = 0; w < kTlWords; ++w) s_set[w][i] = set[w];
        s_jump[i] = (int16_t)jump;
      }
      __syncthreads();
      if (jump >= 0) {
#pragma unroll
        for (int w = 0; w < kTlWords; ++w) set[w] |= s_set[w][jump];
        jump = s_jump[jump];
      }
    }
    if (node) {
#pragma unroll
      for (int w = 0; w < kTlWords; ++w) {
        if (w0 + w >= a.words) break;
        seen += __popcll(set[w]);
        a.masks[(size_t)(first + i) * a.words + w0 + w] = set[w];
      }
    }
  }
  if (!node) return;
  if (a.positions) a.positions[first + i] = context + seen - 1;
  if (a.slots) a.slots[first + i] = slot_of(a.table, a.table_w, b, context + i);
}

// ---------------------------------------------------------------------------
// A wave takes a request's path in a tile (a head of a layer).  An entry is D / 16
// pieces of 16 bytes and two of the scales; the lanes take as many entries at a time
// as they have pieces for.  A source never lies before its place (path[i] >= i), so
// the entries of one time are read before any of them is written, and no later one
// reads what was written.  Bound by whole cache lines: the pieces of an entry lie a
// page of tokens apart, and one of 16 bytes costs 128 (64 paths in 256 tiles: 9 MB
// moved, 60 read and 14 written, 16.4 us with the launch; 17.0 with two tiles a wave
// under way, 17.4 with four, 18.5 with eight).
// ---------------------------------------------------------------------------
constexpr int kCkThreads = 256;

struct KeepArgs {
  uint8_t* cache;
  int tiles, n_pages, Hk, D;    // tiles: layers times heads
  const int32_t* table;
  int table_w;
  const int32_t* kv_len;
  const int32_t* cu_q;
  int T, B, max_q;
  const int32_t* path;
  const int32_t* n_path;
  int32_t* kv_out;              // may be null
};

// ScaleBytes: of a token's scales of one operand.
template <int ScaleBytes>
__global__ void __launch_bounds__(kCkThreads)
k_cache_keep(const KeepArgs a) {
  const int b = blockIdx.y, lane = threadIdx.x % kWave;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave) + blockIdx.x * (kCkThreads / kWave);
  int first;
  const int n = packed_rows(a.cu_q, b, a.T, a.max_q, &first);
  const int len = a.kv_len[b], kept = a.n_path[b];
  const bool moves = kept >= 0 && kept <= n;
  if (a.kv_out && wave == 0 && lane == 0) a.kv_out[b] = moves ? len - n + kept : len;
  if (!moves || a.tiles == 0) return;
  const int codes = a.D / 16, pieces = codes + 2, each = kWave / pieces;
  const int entry = lane / pieces, piece = lane % pieces;
  const bool scale = piece >= codes;
  const size_t tile = tile_bytes(a.D);
  // where a token's piece lies in a tile
  const int at = scale ? k_scales_at(a.D) + (piece - codes) * scales_bytes(a.D) : piece * kPage * kCodeBytes;
  const int step = scale ? ScaleBytes : kCodeBytes;
  for (int i0 = 0; i0 < kept; i0 += each) {
    const int i = i0 + entry;
    int from = -1, to = -1;
    if (entry < each && i < kept) {
      const int j = a.path[first + i];
      if (j > i && j < n) {
        const long long context = (long long)len - n;
        if (context + i >= 0) {
          from = slot_of(a.table, a.table_w, b, (int)(context + j));
          to = slot_of(a.table, a.table_w, b, (int)(context + i));
        }
      }
    }
    const bool ok = from >= 0 && to >= 0 && from / kPage < a.n_pages && to / kPage < a.n_pages;
    if (!__any(ok)) continue;
    const uint8_t* src = a.cache + (size_t)(ok ? from / kPage : 0) * a.Hk * tile + at + (ok ? from % kPage : 0) * step;
    uint8_t* dst = a.cache + (size_t)(ok ? to / kPage : 0) * a.Hk * tile + at + (ok ? to % kPage : 0) * step;
    for (int t = wave; t < a.tiles; t += gridDim.x * (kCkThreads / kWave)) {
      const size_t tile_at = ((size_t)(t / a.Hk) * a.n_pages * a.Hk + t % a.Hk) * tile;
      u32x4 v;
      if (ok) {
        const uint8_t* p = src + tile_at;
        if (!scale) v = *(const u32x4*)p;
        else if constexpr (ScaleBytes == 4) v[0] = *(const uint32_t*)p;
        else v[0] = ((const uint32_t*)p)[0], v[1] = ((const uint32_t*)p)[1];
      }
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");   // all lanes' reads, then all writes
      if (ok) {
        uint8_t* p = dst + tile_at;
        if (!scale) *(u32x4*)p = v;
        else if constexpr (ScaleBytes == 4) *(uint32_t*)p = v[0];
        else ((uint32_t*)p)[0] = v[0], ((uint32_t*)p)[1] = v[1];
      }
    }
  }
}

}  // namespace fdllm

using namespace fdllm;

extern "C" {

fdllm_status fdllm_tree_layout(const int32_t* parents, int T, const int32_t* cu_q, int B, int max_q,
                               const int32_t* kv_len, const int32_t* page_table, int table_width, uint64_t* masks,
                               int mask_words, int32_t* positions, int32_t* slots, fdllm_stream stream) {
  if (T < 0 || B < 0 || max_q < 0 || table_width < 0 || mask_words < 0) return FDLLM_ERR_INVALID_ARG;
  if (B > 65535 || max_q > FDLLM_MAX_TREE || mask_words > (1 << 16)) return FDLLM_ERR_SIZE;
  if (mask_words < (max_q + 63) / 64) return FDLLM_ERR_INVALID_ARG;
  if (T == 0 || B == 0 || max_q == 0) return FDLLM_OK;
  if (!parents || !cu_q || !kv_len || !masks || (slots && table_width > 0 && !page_table)) return FDLLM_ERR_INVALID_ARG;
  if ((uintptr_t)masks & 7) return FDLLM_ERR_INVALID_ARG;
  const size_t rows = (size_t)T * 4, counts = (size_t)B * 4;
  if (!apart({{masks, 2 * rows * mask_words}, {positions, rows}, {slots, rows}},
             {{parents, rows}, {cu_q, counts + 4}, {kv_len, counts}, {page_table, counts * table_width}}))
    return FDLLM_ERR_INVALID_ARG;
  const LayoutArgs a{parents, T, cu_q, B, max_q, kv_len, page_table, table_width, (unsigned long long*)masks, mask_words,
                     positions, slots};
  const unsigned threads = (unsigned)((max_q + kWave - 1) / kWave * kWave);
  hipLaunchKernelGGL(k_tree_layout, dim3((unsigned)B), dim3(threads), 0, (hipStream_t)stream, a);
  return hipGetLastError() == hipSuccess ? FDLLM_OK : FDLLM_ERR_HIP;
}

fdllm_status fdllm_cache_keep(uint8_t* cache, int layers, int n_pages, int Hk, int D, const int32_t* page_table,
                              int table_width, const int32_t* kv_len, const int32_t* cu_q, int T, int B, int max_q,
                              const int32_t* path, const int32_t* n_path, int32_t* kv_out, fdllm_stream stream) {
  if (layers < 0 || n_pages < 0 || Hk < 1 || table_width < 0 || T < 0 || B < 0 || max_q < 0) return FDLLM_ERR_INVALID_ARG;
  size_t tile = 0;
  if (fdllm_cache_tile_bytes(D, &tile) != FDLLM_OK) return FDLLM_ERR_SIZE;
  if ((long long)layers * Hk >= (1 << 24) || B > 65535 || max_q > FDLLM_MAX_TREE || n_pages > INT32_MAX / kPage) return FDLLM_ERR_SIZE;
  if (B == 0) return FDLLM_OK;
  const size_t counts = (size_t)B * 4;
  if (!kv_len || !cu_q || !n_path ||
      !apart({{kv_out, counts}, {cache, (size_t)layers * n_pages * Hk * tile}},
             {{kv_len, counts}, {cu_q, counts + 4}, {n_path, counts}, {page_table, counts * table_width}, {path, (size_t)T * 4}}))
    return FDLLM_ERR_INVALID_ARG;
  const int tiles = n_pages > 0 && table_width > 0 && T > 0 ? layers * Hk : 0;
  if (tiles && (!cache || !page_table || !path || ((uintptr_t)cache & 15))) return FDLLM_ERR_INVALID_ARG;
  const KeepArgs a{cache, tiles, n_pages, Hk, D, page_table, tiles ? table_width : 0, kv_len, cu_q, T, B, max_q, path, n_path, kv_out};
  const int per = kCkThreads / kWave;
  const dim3 grid((unsigned)(tiles ? (tiles + per - 1) / per : 1), (unsigned)B);
  if (scale_stride(D) == 4) hipLaunchKernelGGL(k_cache_keep<4>, grid, dim3(kCkThreads), 0, (hipStream_t)stream, a);
  else hipLaunchKernelGGL(k_cache_keep<8>, grid, dim3(kCkThreads), 0, (hipStream_t)stream, a);
  return hipGetLastError() == hipSuccess ? FDLLM_OK : FDLLM_ERR_HIP;
}

}  // extern "C"
