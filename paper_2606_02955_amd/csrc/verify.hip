// verify.hip -- drafted tokens against a target's probabilities on gfx950: a
// chain with the drafter's probabilities, and a tree by draws at its nodes
// (fdllm.h).
//
//   p_v = 2^((x_v - M) c) / Z,  c = log2(e) / temperature,  Z = sum_v 2^((x_v - M) c)
//   chain:  draft x of row i stands when u_i q_i(x) < p_i(x)
//   drawn:  the lowest v with w_0 + .. + w_v > u (w_0 + w_1 + ..), w = p or max(p - q, 0)
//
// A token is a whole number: a sum that is off by d moves each of V borders by d,
// and a draw goes wrong with a probability of up to 2 V d.  So terms and sums
// are formed in 64 bits.  Sums are kept by chunk of a row; a draw finds its chunk
// in them and looks at that chunk alone again.
//
// One pass over all rows (k_vf_sums), then a chain's decision with the sums of
// max(p - q, 0) of the one row that needs them (k_vd_decide) and its draw
// (k_vd_draw), or the draws at a tree's nodes (k_vt_draw) and its walk
// (k_vt_walk).
#include <hip/hip_runtime.h>

#include <stdint.h>

#include "attn_work.h"
#include "fdllm.h"
#include "pass_common.h"

namespace fdllm {

typedef u32x4 u32x4_a2 __attribute__((aligned(2)));   // rows may begin at any element
typedef u32x4 u32x4_a4 __attribute__((aligned(4)));

constexpr int kVfThreads = 256, kVfWaves = kVfThreads / kWave;
constexpr int kVfLane = 32;                   // logits of a lane
constexpr int kVfChunk = kVfLane * kWave;     // and of a chunk

struct VfArgs {
  const char* logits;
  long long stride;          // bytes of a row
  const char* draft;         // may be null
  long long draft_stride;
  int T, V, B, max_q, chunks;
  const int32_t* ids;
  const int32_t* parents;    // of a tree
  const int32_t* cu_q;
  const float* temperature;  // may be null
  const float* u;
  const float* u_draw;
  int32_t* path;
  int32_t* tokens;
  int32_t* n_tokens;
  float* logp;               // may be null
  struct VfPart* part;       // [sides][T][chunks]
  double* rest;              // [B][chunks]: sums of max(p - q, 0)
  struct VfChoice* choice;   // [B]
  int32_t* drawn;            // [T]: a tree's tokens
  float* drawn_lp;           // [T]
};

// A chunk of a row: its maximum, and the sum of 2^((x - m) c), or with
// temperature 0 the first place of the maximum.
struct __align__(16) VfPart {
  double s;
  float m;
  int first;
};

struct VfStats {   // of a row; Z 0: no token at all
  double Z;
  float M;
  int first;
};

// What was decided for a chain: the row to draw from, and from what.
struct __align__(16) VfChoice {
  VfStats p, q;
  int row;     // -1: nothing to draw
  int rest;    // from max(p - q, 0)
};

// ---------------------------------------------------------------------------
// 2^t, t <= 0, in 64 bits: t in steps of 1/128, a table of 2^(j/128) in LDS and
// the cubic of the remainder: Taylor's, with as much of the fourth term in the
// square's as leaves the least error (x^4 - a x^2 is smallest over |x| <= 1/2 for a =
// (sqrt 2 - 1) / 2), off by 3.9e-13 at most.  2^0 is 1 exactly, so that equal logits
// have borders where the definition has them.  About 15 instructions and a read of
// LDS; the library's takes three times as many.
// ---------------------------------------------------------------------------
constexpr int kVfSteps = 128;
constexpr double kVfCut = -1000.0 * kVfSteps;     // 2^-1000 and less count as nothing
constexpr double kVfRound = 6755399441055744.0;   // 1.5 * 2^52: adding it rounds to a whole number

__device__ __forceinline__ void fill_table(double* table) {
  if (threadIdx.x < kVfSteps) table[threadIdx.x] = exp2((double)threadIdx.x / kVfSteps);
}

// The factors of 2^((x - M) c) = scale * poly, for d = x - M.
__device__ __forceinline__ double exp2_steps(double d, double c, const double* table) {
  const double k = __builtin_fma(d, c, kVfRound);
  const double f = __builtin_fma(d, c, -(k - kVfRound));
  const int lo = (int)(uint32_t)__double_as_longlong(k);
  const double t = *(const double*)((const char*)table + ((lo << 3) & (kVfSteps - 1) * 8));
  const long long bits = __double_as_longlong(t);
  const int hi = (int)(bits >> 32) + ((lo & ~(kVfSteps - 1)) << 13);   // the whole powers of two
  const double scale = __longlong_as_double(((long long)hi << 32) | (uint32_t)bits);
  double p = __builtin_fma(f, 0x1.c6b08d704a0bfp-26, 0x1.ebfbf049a8568p-17);
  p = __builtin_fma(f, p, 0x1.62e42fefa39efp-8);
  p = __builtin_fma(f, p, 1.0);
  return scale * p;
}
// A weight: nothing at all below the cut (c in steps, lowest = cut / c).
__device__ __forceinline__ double weight_of(float x, float M, double c, double lowest, const double* table) {
  const double d = (double)x - (double)M;
  return d > lowest ? exp2_steps(d, c, table) : 0.0;
}

// The request's temperature: c in steps; false for 0.
__device__ __forceinline__ bool scale_for(const VfArgs& a, int b, double* c) {
  uint32_t bits = a.temperature ? __float_as_uint(a.temperature[b]) : __float_as_uint(1.0f);
  if (bits == 0 || bits > 0x7f800000u) return false;           // 0, negative, NaN
  bits = min(bits, 0x7f7fffffu);
  *c = 1.44269504088896340736 * kVfSteps / (double)__uint_as_float(bits);
  return true;
}

// A number in [0, 1).
__device__ __forceinline__ double number_of(float u) {
  return (double)__int_as_float(min(max(__float_as_int(u), 0), 0x3f7fffff));
}

// ---------------------------------------------------------------------------
// a lane's logits of a chunk: vectors of 16 bytes, a wave's side by side
// ---------------------------------------------------------------------------
template <bool F32>
struct VfRow {
  static constexpr int Bytes = F32 ? 4 : 2, Per = 16 / Bytes, Vecs = kVfLane / Per;
  u32x4 v[Vecs];

  __device__ static int index(int chunk, int j, int lane) { return chunk * kVfChunk + (j * kWave + lane) * Per; }
  __device__ __forceinline__ float at(int j, int e) const {
    if constexpr (F32) return __uint_as_float(v[j][e]);
    else return __uint_as_float(e % 2 ? v[j][e / 2] & 0xffff0000u : v[j][e / 2] << 16);
  }
  __device__ __forceinline__ void load(const char* row, int V, int chunk, int lane) {
    typedef typename std::conditional<F32, u32x4_a4, u32x4_a2>::type Vec;
    if ((chunk + 1) * kVfChunk <= V) {
      const char* p = row + (size_t)chunk * kVfChunk * Bytes;
#pragma unroll
      for (int j = 0; j < Vecs; ++j) v[j] = *(const Vec*)(p + (uint32_t)(j * kWave + lane) * 16u);
      return;
    }
#pragma unroll
    for (int j = 0; j < Vecs; ++j) {   // the row's last: past its end nothing can be
      const int i = index(chunk, j, lane);
      if (i + Per <= V) {
        v[j] = *(const Vec*)(row + (size_t)i * Bytes);
      } else {
        const uint32_t none = F32 ? 0xff800000u : 0xff80ff80u;
        v[j] = u32x4{none, none, none, none};
#pragma unroll
        for (int e = 0; e < Per; ++e) {
          if (i + e >= V) continue;
          if constexpr (F32) {
            v[j][e] = *(const uint32_t*)(row + (size_t)(i + e) * 4);
          } else {
            const uint32_t h = *(const uint16_t*)(row + (size_t)(i + e) * 2);
            v[j][e / 2] = e % 2 ? (v[j][e / 2] & 0xffffu) | h << 16 : (v[j][e / 2] & 0xffff0000u) | h;
          }
        }
      }
    }
  }
};

template <bool F32>
__device__ __forceinline__ float logit_at(const char* row, int v) {
  if constexpr (F32) return *(const float*)(row + (size_t)v * 4);
  else return __uint_as_float((uint32_t)*(const uint16_t*)(row + (size_t)v * 2) << 16);
}

// ---------------------------------------------------------------------------
// the pass over all rows.  A wave takes every so-and-so-many-th chunk of one.
// ---------------------------------------------------------------------------
template <bool F32>
__global__ void __launch_bounds__(kVfThreads)
k_vf_sums(const VfArgs a, int sides) {
  typedef VfRow<F32> Row;
  __shared__ double s_table[kVfSteps];
  const int b = blockIdx.z, i = blockIdx.y / sides, side = blockIdx.y % sides;
  int first;
  const int n = packed_rows(a.cu_q, b, a.T, a.max_q, &first);
  if (i >= n - side) return;   // (the drafter's last row is not read)
  double c = 0.0;
  const bool warm = scale_for(a, b, &c);
  if (!warm && side) return;
  fill_table(s_table);
  __syncthreads();
  const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const char* row = side ? a.draft + (size_t)(first + i) * a.draft_stride : a.logits + (size_t)(first + i) * a.stride;
  VfPart* part = a.part + ((size_t)side * a.T + first + i) * a.chunks;
  const int step = gridDim.x * kVfWaves;
  int ch = blockIdx.x * kVfWaves + wave;
  if (ch >= a.chunks) return;
  const double lowest = kVfCut / c;
  Row next;
  next.load(row, a.V, ch, lane);
  for (; ch < a.chunks; ch += step) {
    const Row x = next;
    if (ch + step < a.chunks) next.load(row, a.V, ch + step, lane);
    float m = kNegInf;
#pragma unroll
    for (int j = 0; j < Row::Vecs; ++j)
#pragma unroll
      for (int e = 0; e < Row::Per; ++e) m = fmaxf(m, x.at(j, e));
    m = wave_max(m);
    double s = 0.0;
    int at = 0;
    if (!warm) {
      at = INT32_MAX;
#pragma unroll
      for (int j = Row::Vecs - 1; j >= 0; --j)
#pragma unroll
        for (int e = Row::Per - 1; e >= 0; --e)
          if (x.at(j, e) == m) at = Row::index(ch, j, lane) + e;
      at = wave_min(at);
    } else if (m > kNegInf) {
      const double M = m;
      double s1 = 0.0;
#pragma unroll
      for (int j = 0; j < Row::Vecs; ++j)
#pragma unroll
        for (int e = 0; e < Row::Per; e += 2) {
          s += exp2_steps(fmax((double)x.at(j, e) - M, lowest), c, s_table);
          s1 += exp2_steps(fmax((double)x.at(j, e + 1) - M, lowest), c, s_table);
        }
      s = wave_sum_f64(s + s1);
    }
    if (lane == 0) part[ch] = VfPart{s, m, at};
  }
}

// ---------------------------------------------------------------------------
// wave-level pieces of what follows
// ---------------------------------------------------------------------------
// A chunk's sum brought to the row's maximum M.
__device__ __forceinline__ double part_weight(const VfPart& p, float M, double c) {
  const double d = (double)p.m - (double)M;
  return d * c > kVfCut ? p.s * exp2(d * c * (1.0 / kVfSteps)) : 0.0;   // (-inf: 0)
}

__device__ __forceinline__ VfStats row_stats(const VfPart* part, int chunks, bool warm, double c, int lane) {
  VfStats r{0.0, kNegInf, 0};
  for (int ch = lane; ch < chunks; ch += kWave) r.M = fmaxf(r.M, part[ch].m);
  r.M = wave_max(r.M);
  if (!(r.M > kNegInf)) return r;
  if (warm) {
    for (int ch = lane; ch < chunks; ch += kWave) r.Z += part_weight(part[ch], r.M, c);
    r.Z = wave_sum_f64(r.Z);
  } else {
    int at = INT32_MAX;
    for (int ch = lane; ch < chunks; ch += kWave)
      if (part[ch].m == r.M) at = min(at, part[ch].first);
    at = wave_min(at);
    r.first = at < INT32_MAX ? at : -1;
    r.Z = 1.0;
  }
  return r;
}

// p of one token.
template <bool F32>
__device__ __forceinline__ double probability(const char* row, int v, const VfStats& r, double c) {
  const double d = ((double)logit_at<F32>(row, v) - (double)r.M) * c;
  return d > kVfCut ? exp2(d * (1.0 / kVfSteps)) / r.Z : 0.0;
}
template <bool F32>
__device__ __forceinline__ float log_probability(const char* row, int v, const VfStats& r, double c) {
  const double d = ((double)logit_at<F32>(row, v) - (double)r.M) * c;
  return (float)(d * (0.69314718055994530942 / kVfSteps) - log(r.Z));
}

// The weights that a token is drawn from: 2^((x - M) c) of a row, without the
// token `without`, or, where there is a row q, max(p - q, 0).
template <bool F32>
struct VfWeights {
  const char* p;
  const char* q;
  VfStats sp, sq;
  double c, ip, iq, lowest;
  int without;

  __device__ VfWeights(const char* p_, const VfStats& sp_, const char* q_, const VfStats& sq_, double c_, int without_)
      : p(p_), q(q_), sp(sp_), sq(sq_), c(c_), ip(1.0 / sp_.Z), iq(q_ ? 1.0 / sq_.Z : 0.0), lowest(kVfCut / c_),
        without(without_) {}

  __device__ __forceinline__ void of_chunk(int V, int ch, int lane, const double* table, double (&w)[kVfLane]) const {
    typedef VfRow<F32> Row;
    Row x, y;
    x.load(p, V, ch, lane);
    if (q) y.load(q, V, ch, lane);
#pragma unroll
    for (int j = 0; j < Row::Vecs; ++j)
#pragma unroll
      for (int e = 0; e < Row::Per; ++e) w[j * Row::Per + e] = weight_of(x.at(j, e), sp.M, c, lowest, table);
    if (q) {
#pragma unroll
      for (int j = 0; j < Row::Vecs; ++j)
#pragma unroll
        for (int e = 0; e < Row::Per; ++e) {
          double& v = w[j * Row::Per + e];
          v = fmax(v * ip - weight_of(y.at(j, e), sq.M, c, lowest, table) * iq, 0.0);
        }
    } else if (without >= 0) {
#pragma unroll
      for (int j = 0; j < Row::Vecs; ++j)
#pragma unroll
        for (int e = 0; e < Row::Per; ++e)
          if (Row::index(ch, j, lane) + e == without) w[j * Row::Per + e] = 0.0;
    }
  }
  __device__ double sum_of_chunk(int V, int ch, int lane, const double* table) const {
    double w[kVfLane], s = 0.0;
    of_chunk(V, ch, lane, table, w);
#pragma unroll
    for (int i = 0; i < kVfLane; ++i) s += w[i];
    return wave_sum_f64(s);
  }
};

// Inclusive sums over the lanes.
__device__ __forceinline__ double wave_scan_f64(double v, int lane) {
#pragma unroll
  for (int x = 1; x < kWave; x <<= 1) {
    const double y = __shfl_up(v, x);
    if (lane >= x) v += y;
  }
  return v;
}

// The token drawn with number u, -1 where all weights are 0; sum_of(chunk): a
// chunk's sum, the same in every lane that asks for it.
template <bool F32, typename F>
__device__ int draw_token(const VfWeights<F32>& weights, int V, int chunks, const double* table, double u, int lane,
                          F&& sum_of) {
  typedef VfRow<F32> Row;
  const int per = (chunks + kWave - 1) / kWave, c0 = lane * per, c1 = min(c0 + per, chunks);
  double mine = 0.0;
  for (int ch = c0; ch < c1; ++ch) mine += sum_of(ch);
  const double incl = wave_scan_f64(mine, lane);
  const double total = readlane_f64(incl, kWave - 1);
  if (!(total > 0.0)) return -1;
  const double target = u * total;
  const unsigned long long some = __ballot(mine > 0.0), over = __ballot(incl > target) & some;
  if (!some) return -1;
  const int L = over ? __ffsll(over) - 1 : 63 - __clzll(some);
  double before = readlane_f64(incl - mine, L);
  int ch = -1;
  for (int k = L * per; k < min((L + 1) * per, chunks); ++k) {   // of the lane's chunks the first beyond, or its last
    const double s = sum_of(k);
    if (!(s > 0.0)) continue;
    ch = k;
    if (before + s > target) break;
    if (k + 1 < min((L + 1) * per, chunks)) before += s;
  }
  ch = __builtin_amdgcn_readfirstlane(ch);
  if (ch < 0) return -1;
  double w[kVfLane], from[Row::Vecs];
  weights.of_chunk(V, ch, lane, table, w);
  // sums before each vector of the lane
#pragma unroll
  for (int j = 0; j < Row::Vecs; ++j) {
    double s = 0.0;
#pragma unroll
    for (int e = 0; e < Row::Per; ++e) s += w[j * Row::Per + e];
    const double in = wave_scan_f64(s, lane);
    from[j] = before + (in - s);
    before += readlane_f64(in, kWave - 1);
  }
  int best = INT32_MAX, last = -1;
#pragma unroll
  for (int j = 0; j < Row::Vecs; ++j) {
    double s = from[j];
#pragma unroll
    for (int e = 0; e < Row::Per; ++e) {
      const double x = w[j * Row::Per + e];
      const int at = Row::index(ch, j, lane) + e;
      s += x;
      if (x > 0.0 && at < V) {
        last = at;
        if (s > target) best = min(best, at);
      }
    }
  }
  best = wave_min(best);
  // the chunk's sum was formed in another order: past its end by a rounding, its last
  return best != INT32_MAX ? best : -wave_min(-last);
}

// ---------------------------------------------------------------------------
// a chain: which drafts stand, and the sums of max(p - q, 0) where one fell.
// Every workgroup of a request decides by itself; the first writes it down.
// ---------------------------------------------------------------------------
template <bool F32>
__global__ void __launch_bounds__(kVfThreads)
k_vd_decide(const VfArgs a) {
  __shared__ double s_table[kVfSteps];
  __shared__ VfChoice s_choice;
  __shared__ int s_fell[kVfWaves];
  const int b = blockIdx.y;
  const int tid = threadIdx.x, lane = tid % kWave, wave = __builtin_amdgcn_readfirstlane(tid / kWave);
  const bool writes = blockIdx.x == 0;
  int first;
  const int n = packed_rows(a.cu_q, b, a.T, a.max_q, &first);
  if (n == 0) {
    if (writes && tid == 0) {
      a.n_tokens[b] = 0;
      if (a.choice) a.choice[b].row = -1;
    }
    return;
  }
  fill_table(s_table);
  double c = 0.0;
  const bool warm = scale_for(a, b, &c);
  const bool with_q = warm && a.draft;
  const VfPart* p_part = a.part + (size_t)first * a.chunks;
  const VfPart* q_part = a.part + ((size_t)a.T + first) * a.chunks;

  // a wave a draft, those after one that fell for nothing
  int fell = n - 1;
  for (int i = wave; i < fell; i += kVfWaves) {
    const VfStats sp = row_stats(p_part + (size_t)i * a.chunks, a.chunks, warm, c, lane);
    VfStats sq{1.0, 0.0, 0};
    if (with_q) sq = row_stats(q_part + (size_t)i * a.chunks, a.chunks, warm, c, lane);
    const int x = a.ids[first + i + 1];
    const char* row = a.logits + (size_t)(first + i) * a.stride;
    bool stands = x >= 0 && x < a.V && sp.Z > 0.0 && sq.Z > 0.0;
    if (stands && warm) {
      const double p = probability<F32>(row, x, sp, c);
      double q = 1.0;
      if (with_q) q = probability<F32>(a.draft + (size_t)(first + i) * a.draft_stride, x, sq, c);
      stands = number_of(a.u[first + i]) * q < p;
    } else if (stands) {
      stands = x == sp.first;
    }
    if (!stands) fell = i;
    else if (writes && a.logp && lane == 0) a.logp[first + i] = warm ? log_probability<F32>(row, x, sp, c) : 0.0f;
  }
  if (lane == 0) s_fell[wave] = fell;
  __syncthreads();
  int m = n - 1;
#pragma unroll
  for (int w = 0; w < kVfWaves; ++w) m = min(m, s_fell[w]);
  if (wave == 0) {
    VfChoice r{};
    r.p = row_stats(p_part + (size_t)m * a.chunks, a.chunks, warm, c, lane);
    r.q = VfStats{0.0, kNegInf, 0};
    if (with_q && m < n - 1) r.q = row_stats(q_part + (size_t)m * a.chunks, a.chunks, warm, c, lane);
    r.row = first + m;
    r.rest = warm && m < n - 1 && (!a.draft || r.q.Z > 0.0);
    if (lane == 0) {
      s_choice = r;
      if (writes) {
        if (a.choice) a.choice[b] = r;
        a.n_tokens[b] = m + 1;
      }
    }
  }
  __syncthreads();
  if (writes) {
    for (int i = tid; i < n; i += kVfThreads) {
      if (i < m) a.tokens[first + i] = a.ids[first + i + 1];
      else if (i > m) {
        a.tokens[first + i] = -1;
        if (a.logp) a.logp[first + i] = 0.0f;
      }
    }
  }
  const VfChoice r = s_choice;
  if (!r.rest || !a.draft || !(r.p.Z > 0.0)) return;
  const VfWeights<F32> weights(a.logits + (size_t)r.row * a.stride, r.p, a.draft + (size_t)r.row * a.draft_stride, r.q, c, -1);
  for (int ch = blockIdx.x * kVfWaves + wave; ch < a.chunks; ch += gridDim.x * kVfWaves) {
    const double s = weights.sum_of_chunk(a.V, ch, lane, s_table);
    if (lane == 0) a.rest[(size_t)b * a.chunks + ch] = s;
  }
}

// The token after the drafts that stand: a wave a request.
template <bool F32>
__global__ void __launch_bounds__(kVfSteps)
k_vd_draw(const VfArgs a) {
  __shared__ double s_table[kVfSteps];
  fill_table(s_table);
  __syncthreads();
  if (threadIdx.x >= kWave) return;
  const int b = blockIdx.x, lane = threadIdx.x;
  const VfChoice r = a.choice[b];
  if (r.row < 0) return;
  double c = 0.0;
  const bool warm = scale_for(a, b, &c);
  const char* row = a.logits + (size_t)r.row * a.stride;
  const VfPart* part = a.part + (size_t)r.row * a.chunks;
  int y = -1;
  if (!(r.p.Z > 0.0)) {
    // no token can be
  } else if (!warm) {
    y = r.p.first;
  } else {
    const double u = number_of(a.u_draw[b]);
    if (r.rest && a.draft) {
      const VfWeights<F32> w(row, r.p, a.draft + (size_t)r.row * a.draft_stride, r.q, c, -1);
      const double* rest = a.rest + (size_t)b * a.chunks;
      y = draw_token(w, a.V, a.chunks, s_table, u, lane, [&](int ch) { return rest[ch]; });
    } else if (r.rest) {
      // all but the draft: its chunk's sum without it
      const int x = a.ids[r.row + 1];
      const VfWeights<F32> w(row, r.p, nullptr, r.q, c, x >= 0 && x < a.V ? x : -1);
      const int its = w.without >= 0 ? x / kVfChunk : -1;
      const double other = its >= 0 ? w.sum_of_chunk(a.V, its, lane, s_table) : 0.0;
      y = draw_token(w, a.V, a.chunks, s_table, u, lane,
                     [&](int ch) { return ch == its ? other : part_weight(part[ch], r.p.M, c); });
    }
    if (y < 0) {
      const VfWeights<F32> w(row, r.p, nullptr, r.q, c, -1);
      y = draw_token(w, a.V, a.chunks, s_table, u, lane, [&](int ch) { return part_weight(part[ch], r.p.M, c); });
    }
  }
  if (lane == 0) {
    a.tokens[r.row] = y;
    if (a.logp) a.logp[r.row] = warm && y >= 0 ? log_probability<F32>(row, y, r.p, c) : 0.0f;
  }
}

// ---------------------------------------------------------------------------
// a tree: a draw at every node, a wave each; then the walk, a workgroup a request
// ---------------------------------------------------------------------------
template <bool F32>
__global__ void __launch_bounds__(kVfThreads)
k_vt_draw(const VfArgs a) {
  __shared__ double s_table[kVfSteps];
  const int b = blockIdx.y, lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  int first;
  const int n = packed_rows(a.cu_q, b, a.T, a.max_q, &first);
  if ((int)blockIdx.x * kVfWaves >= n) return;
  fill_table(s_table);
  __syncthreads();
  const int i = blockIdx.x * kVfWaves + wave;
  if (i >= n) return;
  double c = 0.0;
  const bool warm = scale_for(a, b, &c);
  const int r = first + i;
  const char* row = a.logits + (size_t)r * a.stride;
  const VfPart* part = a.part + (size_t)r * a.chunks;
  const VfStats sp = row_stats(part, a.chunks, warm, c, lane);
  int y = -1;
  float lp = 0.0f;
  if (sp.Z > 0.0 && warm) {
    const VfWeights<F32> w(row, sp, nullptr, sp, c, -1);
    y = draw_token(w, a.V, a.chunks, s_table, number_of(a.u[r]), lane,
                   [&](int ch) { return part_weight(part[ch], sp.M, c); });
    if (y >= 0) lp = log_probability<F32>(row, y, sp, c);
  } else if (sp.Z > 0.0) {
    y = sp.first;
  }
  if (lane == 0) {
    a.drawn[r] = y;
    a.drawn_lp[r] = lp;
  }
}

__global__ void __launch_bounds__(kVfThreads)
k_vt_walk(const VfArgs a) {
  __shared__ int s_y[FDLLM_MAX_TREE], s_child[FDLLM_MAX_TREE], s_path[FDLLM_MAX_TREE], s_len;
  const int b = blockIdx.x, tid = threadIdx.x;
  int first;
  const int n = packed_rows(a.cu_q, b, a.T, a.max_q, &first);
  if (n == 0) {
    if (tid == 0) a.n_tokens[b] = 0;
    return;
  }
  for (int i = tid; i < n; i += kVfThreads) {
    s_y[i] = a.drawn[first + i];
    s_child[i] = INT32_MAX;
  }
  __syncthreads();
  for (int i = tid; i < n; i += kVfThreads) {
    const int p = a.parents[first + i];
    if (p >= 0 && p < i && s_y[p] >= 0 && a.ids[first + i] == s_y[p]) atomicMin(&s_child[p], i);   // the lowest, in any order
  }
  __syncthreads();
  if (tid == 0) {
    int len = 0;
    for (int i = 0; i < n; i = s_child[i]) s_path[len++] = i;   // children come after their parents
    s_len = len;
    a.n_tokens[b] = len;
  }
  __syncthreads();
  const int len = s_len;
  for (int i = tid; i < n; i += kVfThreads) {
    const int node = i < len ? s_path[i] : -1;
    a.path[first + i] = node;
    a.tokens[first + i] = node >= 0 ? s_y[node] : -1;
    if (a.logp) a.logp[first + i] = node >= 0 ? a.drawn_lp[first + node] : 0.0f;
  }
}

// ---------------------------------------------------------------------------
// host side
// ---------------------------------------------------------------------------
struct VfPlan {
  int chunks;
  size_t at_rest, at_choice, at_drawn, at_lp, bytes;
};

static bool vf_sizes_ok(int T, int B, int V) { return V >= 1 && V <= (1 << 30) && B <= 65535; }

static VfPlan vf_plan(int T, int B, int V, bool tree, bool marginals) {
  VfPlan p{};
  p.chunks = (V + kVfChunk - 1) / kVfChunk;
  size_t at = align256((size_t)(marginals ? 2 : 1) * T * p.chunks * sizeof(VfPart));
  const auto take = [&](size_t n) {
    const size_t here = at;
    at += align256(n);
    return here;
  };
  if (tree) {
    p.at_drawn = take((size_t)T * 4);
    p.at_lp = take((size_t)T * 4);
  } else {
    p.at_choice = take((size_t)B * sizeof(VfChoice));
    if (marginals) p.at_rest = take((size_t)B * p.chunks * sizeof(double));
  }
  p.bytes = at;
  return p;
}

// Workgroups a row: eight a CU in all, no more than a wave a chunk.
static int vf_parts(long long rows, int chunks) {
  const long long want = (256 * 8 + rows - 1) / (rows < 1 ? 1 : rows), most = (chunks + kVfWaves - 1) / kVfWaves;
  return (int)(want < 1 ? 1 : want < most ? want : most);
}

static fdllm_status vf_check(const void* logits, int64_t stride, fdllm_dtype dtype, int T, int V, const int32_t* cu_q, int B,
                             int max_q, const int32_t* n_tokens) {
  if (T < 0 || B < 0 || max_q < 0) return FDLLM_ERR_INVALID_ARG;
  if (dtype != FDLLM_BF16 && dtype != FDLLM_F32) return FDLLM_ERR_UNSUPPORTED_DTYPE;
  if (!vf_sizes_ok(T, B, V) || max_q > FDLLM_MAX_TREE) return FDLLM_ERR_SIZE;
  if (stride < V) return FDLLM_ERR_INVALID_ARG;
  if ((double)stride * T > 1.0e18) return FDLLM_ERR_SIZE;   // offsets fit 64 bits
  if (B > 0 && (!cu_q || !n_tokens)) return FDLLM_ERR_INVALID_ARG;
  if (T > 0 && !logits) return FDLLM_ERR_INVALID_ARG;
  if ((uintptr_t)logits & (dtype == FDLLM_F32 ? 3 : 1)) return FDLLM_ERR_INVALID_ARG;
  return FDLLM_OK;
}

template <bool F32>
static void vf_sums(const VfArgs& a, int sides, hipStream_t st) {
  if (a.T == 0 || a.max_q == 0) return;
  const int rows = a.max_q < a.T ? a.max_q : a.T;   // of a request
  hipLaunchKernelGGL((k_vf_sums<F32>), dim3((unsigned)vf_parts((long long)a.T * sides, a.chunks), (unsigned)(rows * sides), (unsigned)a.B),
                     dim3(kVfThreads), 0, st, a, sides);
}

template <bool F32>
static hipError_t vd_launch(const VfArgs& a, hipStream_t st) {
  vf_sums<F32>(a, a.draft ? 2 : 1, st);
  const int parts = a.draft ? vf_parts(a.B, a.chunks) : 1;
  hipLaunchKernelGGL((k_vd_decide<F32>), dim3((unsigned)parts, (unsigned)a.B), dim3(kVfThreads), 0, st, a);
  hipLaunchKernelGGL((k_vd_draw<F32>), dim3((unsigned)a.B), dim3(kVfSteps), 0, st, a);
  return hipGetLastError();
}

template <bool F32>
static hipError_t vt_launch(const VfArgs& a, hipStream_t st) {
  vf_sums<F32>(a, 1, st);
  const int rows = a.max_q < a.T ? a.max_q : a.T;
  if (rows > 0)
    hipLaunchKernelGGL((k_vt_draw<F32>), dim3((unsigned)((rows + kVfWaves - 1) / kVfWaves), (unsigned)a.B), dim3(kVfThreads), 0, st, a);
  hipLaunchKernelGGL(k_vt_walk, dim3((unsigned)a.B), dim3(kVfThreads), 0, st, a);
  return hipGetLastError();
}

}  // namespace fdllm

using namespace fdllm;

extern "C" {

fdllm_status fdllm_verify_draft_workspace_size(int T, int B, int V, int with_draft_logits, size_t* bytes) {
  if (!bytes || T < 0 || B < 0) return FDLLM_ERR_INVALID_ARG;
  if (!vf_sizes_ok(T, B, V)) return FDLLM_ERR_SIZE;
  *bytes = vf_plan(T, B, V, false, with_draft_logits != 0).bytes;
  return FDLLM_OK;
}

fdllm_status fdllm_verify_tree_workspace_size(int T, int B, int V, size_t* bytes) {
  if (!bytes || T < 0 || B < 0) return FDLLM_ERR_INVALID_ARG;
  if (!vf_sizes_ok(T, B, V)) return FDLLM_ERR_SIZE;
  *bytes = vf_plan(T, B, V, true, false).bytes;
  return FDLLM_OK;
}

fdllm_status fdllm_verify_draft(const void* logits, int64_t logits_stride, const void* draft_logits, int64_t draft_stride,
                                fdllm_dtype dtype, int T, int V, const int32_t* ids, const int32_t* cu_q, int B, int max_q,
                                const float* temperature, const float* u, const float* u_draw, int32_t* tokens,
                                int32_t* n_tokens, float* logp, void* workspace, size_t workspace_bytes,
                                fdllm_stream stream) {
  fdllm_status ok = vf_check(logits, logits_stride, dtype, T, V, cu_q, B, max_q, n_tokens);
  if (ok == FDLLM_OK && draft_logits) ok = vf_check(draft_logits, draft_stride, dtype, T, V, cu_q, B, max_q, n_tokens);
  if (ok != FDLLM_OK) return ok;
  if (B == 0) return FDLLM_OK;
  if (T > 0 && (!ids || !u || !u_draw || !tokens)) return FDLLM_ERR_INVALID_ARG;
  const VfPlan p = vf_plan(T, B, V, false, draft_logits != nullptr);
  if ((uintptr_t)workspace & 15) return FDLLM_ERR_INVALID_ARG;
  if (!workspace || workspace_bytes < p.bytes) return FDLLM_ERR_WORKSPACE;
  char* ws = (char*)workspace;
  const int es = dtype == FDLLM_F32 ? 4 : 2;
  VfArgs a{};
  a.logits = (const char*)logits, a.stride = logits_stride * es;
  a.draft = (const char*)draft_logits, a.draft_stride = draft_stride * es;
  a.T = T, a.V = V, a.B = B, a.max_q = max_q, a.chunks = p.chunks;
  a.ids = ids, a.cu_q = cu_q, a.temperature = temperature, a.u = u, a.u_draw = u_draw;
  a.tokens = tokens, a.n_tokens = n_tokens, a.logp = logp;
  a.part = (VfPart*)ws, a.rest = (double*)(ws + p.at_rest), a.choice = (VfChoice*)(ws + p.at_choice);
  const hipError_t e = dtype == FDLLM_F32 ? vd_launch<true>(a, (hipStream_t)stream) : vd_launch<false>(a, (hipStream_t)stream);
  return e == hipSuccess ? FDLLM_OK : FDLLM_ERR_HIP;
}

fdllm_status fdllm_verify_tree(const void* logits, int64_t logits_stride, fdllm_dtype dtype, int T, int V,
                               const int32_t* ids, const int32_t* parents, const int32_t* cu_q, int B, int max_q,
                               const float* temperature, const float* u, int32_t* path, int32_t* tokens,
                               int32_t* n_tokens, float* logp, void* workspace, size_t workspace_bytes,
                               fdllm_stream stream) {
  const fdllm_status ok = vf_check(logits, logits_stride, dtype, T, V, cu_q, B, max_q, n_tokens);
  if (ok != FDLLM_OK) return ok;
  if (B == 0) return FDLLM_OK;
  if (T > 0 && (!ids || !parents || !u || !path || !tokens)) return FDLLM_ERR_INVALID_ARG;
  const VfPlan p = vf_plan(T, B, V, true, false);
  if ((uintptr_t)workspace & 15) return FDLLM_ERR_INVALID_ARG;
  if (p.bytes && (!workspace || workspace_bytes < p.bytes)) return FDLLM_ERR_WORKSPACE;
  char* ws = (char*)workspace;
  const int es = dtype == FDLLM_F32 ? 4 : 2;
  VfArgs a{};
  a.logits = (const char*)logits, a.stride = logits_stride * es;
  a.T = T, a.V = V, a.B = B, a.max_q = max_q, a.chunks = p.chunks;
  a.ids = ids, a.parents = parents, a.cu_q = cu_q, a.temperature = temperature, a.u = u;
  a.path = path, a.tokens = tokens, a.n_tokens = n_tokens, a.logp = logp;
  a.part = (VfPart*)ws, a.drawn = (int32_t*)(ws + p.at_drawn), a.drawn_lp = (float*)(ws + p.at_lp);
  const hipError_t e = dtype == FDLLM_F32 ? vt_launch<true>(a, (hipStream_t)stream) : vt_launch<false>(a, (hipStream_t)stream);
  return e == hipSuccess ? FDLLM_OK : FDLLM_ERR_HIP;
}

}  // extern "C"
