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
// One pass over all rows (k_vf_sums); then a chain's decision, with the draw where
// there are no drafter's logits (k_vd_decide), otherwise with the sums of max(p - q,
// 0) of the row that needs them (apart for many requests: k_vd_rest) and the draw
// behind it (k_vd_draw); or the draws at a tree's nodes and its walk (k_vt_draw,
// k_vt_walk).
#include <hip/hip_runtime.h>

#include <stdint.h>

#include "attn_work.h"
#include "fdllm.h"
#include "pass_common.h"

namespace fdllm {

// Rows may begin at any element: 16 bytes of one promise no more alignment than
// that.  (A type passed as a template's argument would lose its alignment.)
template <bool F32>
struct VfVec;
template <>
struct VfVec<false> {
  typedef u32x4 type __attribute__((aligned(2)));
};
template <>
struct VfVec<true> {
  typedef u32x4 type __attribute__((aligned(4)));
};
static_assert(alignof(VfVec<false>::type) == 2 && alignof(VfVec<true>::type) == 4, "alignment of a row");
template <bool F32>
__device__ __forceinline__ u32x4 load_16(const char* p) {
  return *(const typename VfVec<F32>::type*)p;
}

constexpr int kVfThreads = 256, kVfWaves = kVfThreads / kWave;
constexpr int kVtThreads = 512;               // of the pass with a table
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
  double* rest;              // [B][pieces]: sums of max(p - q, 0)
  struct VfChoice* choice;   // [B]
  bool together;             // the decision forms rest as well
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
// (sqrt 2 - 1) / 2), off by 3.9e-13 at most.  2^0 is 1 exactly, so that a row of
// equal logits has its borders where the definition has them (not where terms are
// looked up, below: those are of logits less 0, not less the highest, and no whole
// numbers).  About 15 instructions and a read of LDS; the library's takes three times
// as many.
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
  const int lo = __double2loint(k);
  const double t = *(const double*)((const char*)table + ((lo << 3) & (kVfSteps - 1) * 8));
  const int hi = __double2hiint(t) + ((lo & ~(kVfSteps - 1)) << 13);   // the whole powers of two
  const double scale = __hiloint2double(hi, __double2loint(t));
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

// A request's temperature: c in steps; false for 0.
__device__ __forceinline__ uint32_t temperature_of(const VfArgs& a, int b) {
  return a.temperature ? __float_as_uint(a.temperature[b]) : __float_as_uint(1.0f);
}
__device__ __forceinline__ bool scale_for(uint32_t bits, double* c) {
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
// Bfloat16 logits are few: between 2^-18 and 64 there are 6144, both signs taken
// together.  Where a workgroup has many of one temperature it looks 2^(x c) up
// (7 vector instructions a logit for 23, all counted), without a reference: for 64 c <= 480 all
// terms and sums are numbers of 64 bits.  Entries lie by the bits of a logit with its
// sign moved to the end, so that two are told from one word at a time.
// ---------------------------------------------------------------------------
constexpr int kVtLow = 109 << 8, kVtHigh = 133 << 8, kVtEntries = kVtHigh - kVtLow;   // exponents -18 to 5
constexpr double kVtMost = 480.0 / 64.0 * kVfSteps;   // c in steps, at most
typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ void fill_lookup(double* lookup, double c, const double* table, int threads) {
  for (int i = threadIdx.x; i < kVtEntries; i += threads) {
    const uint32_t turned = i + kVtLow;
    lookup[i] = exp2_steps((double)__uint_as_float((turned >> 1 | (turned & 1) << 15) << 16), c, table);
  }
}
// Two logits' places in the table; beyond its end where they are not in it.
__device__ __forceinline__ u16x2 places_of(uint32_t word) {
  const u16x2 w = __builtin_bit_cast(u16x2, word);
  return w * (unsigned short)2 + ((w >> 15) - (unsigned short)kVtLow);
}

template <bool F32>
__device__ __forceinline__ float logit_at(const char* row, int v) {
  if constexpr (F32) return *(const float*)(row + (size_t)v * 4);
  else return __uint_as_float((uint32_t)*(const uint16_t*)(row + (size_t)v * 2) << 16);
}

// 16 bytes of a row from element i on, past whose end nothing can be (-inf): the
// last 16 that the row has, shifted, so that all lanes load at once.
template <bool F32>
__device__ __forceinline__ u32x4 load_end(const char* row, int V, int i) {
  constexpr int Bits = F32 ? 32 : 16, Per = 128 / Bits;
  constexpr unsigned long long none = F32 ? 0xff800000ff800000ull : 0xff80ff80ff80ff80ull;
  unsigned long long lo = none, hi = none;
  if (V >= Per) {
    const int from = min(i, V - Per);
    const u32x4 v = load_16<F32>(row + (size_t)from * (Bits / 8));
    lo = v[0] | (unsigned long long)v[1] << 32;
    hi = v[2] | (unsigned long long)v[3] << 32;
    const int past = min(i - from, Per) * Bits;   // bits to be dropped
    if (past >= 64) {
      lo = past == 128 ? none : past == 64 ? hi : hi >> (past - 64) | none << (128 - past);
      hi = none;
    } else if (past > 0) {
      lo = lo >> past | hi << (64 - past);
      hi = hi >> past | none << (64 - past);
    }
  } else {
#pragma unroll 1
    for (int e = V - 1; e >= i; --e) {
      hi = hi << Bits | lo >> (64 - Bits);
      lo = lo << Bits | __float_as_uint(logit_at<F32>(row, e)) >> (32 - Bits);
    }
  }
  return u32x4{(uint32_t)lo, (uint32_t)(lo >> 32), (uint32_t)hi, (uint32_t)(hi >> 32)};
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
    if ((chunk + 1) * kVfChunk <= V) {
      const char* p = row + (size_t)chunk * kVfChunk * Bytes;
#pragma unroll
      for (int j = 0; j < Vecs; ++j) v[j] = __builtin_nontemporal_load((const typename VfVec<F32>::type*)(p + (uint32_t)(j * kWave + lane) * 16u));
      return;
    }
#pragma unroll
    for (int j = 0; j < Vecs; ++j) {   // the row's last chunk
      const int first = index(chunk, j, 0);
      if (first + kWave * Per <= V) {
        v[j] = load_16<F32>(row + ((size_t)first + lane * Per) * Bytes);
      } else if (first < V) {
        v[j] = load_end<F32>(row, V, first + lane * Per);
      } else {
        const uint32_t none = F32 ? 0xff800000u : 0xff80ff80u;
        v[j] = u32x4{none, none, none, none};
      }
    }
  }
};

// ---------------------------------------------------------------------------
// the pass over all rows.  The units of work are chunks: of a request those of
// its rows, then those of its drafter's.  Every workgroup takes an equal share,
// whatever the requests' lengths, its waves one chunk after another in turn, the
// next one's loads under way.  Bound by HBM where chunks are many: 48 chains of 3 to
// 17 rows with their drafter's, 231 MB of bfloat16, 43 us in the middle and
// 37.4 at best, 5.4 and 6.2 TB/s (95 -> 69 us for the call by the table of terms and
// nontemporal loads, 5 of it the latter); 16 float trees of 11 to 61 rows of 50021,
// filtered, 23.5 us, 4.9 TB/s, with 3.4 chunks a wave; by starting and the loads' latency
// where few: 26 rows of 126464 6.5 us.  (A second chunk under way, workgroups of 1024,
// three a CU: no gain, or spills.)
// ---------------------------------------------------------------------------
struct VfRequest {
  int first, n, rows;   // rows: of both sides
  bool warm;
  double c;
};
struct VfLoaded {   // what has to be loaded for it (first, so that other things are done meanwhile)
  int32_t cu[2];
  uint32_t temperature;
};
__device__ __forceinline__ VfLoaded load_request(const VfArgs& a, int b) {
  return VfLoaded{{a.cu_q[b], a.cu_q[b + 1]}, temperature_of(a, b)};
}
__device__ __forceinline__ VfRequest request_of(const VfArgs& a, const VfLoaded& l) {
  VfRequest r;
  r.n = packed_rows(l.cu, 0, a.T, a.max_q, &r.first);
  r.c = 0.0;
  r.warm = scale_for(l.temperature, &r.c);
  r.rows = r.n + (a.draft && r.warm ? max(r.n - 1, 0) : 0);   // (the drafter's last row is not read)
  return r;
}
__device__ __forceinline__ VfRequest request_of(const VfArgs& a, int b) { return request_of(a, load_request(a, b)); }

// Lookup: terms of bfloat16 logits out of a table.
template <bool F32, bool Lookup>
__global__ void __launch_bounds__(Lookup ? kVtThreads : kVfThreads, Lookup ? 4 : 1)
k_vf_sums(const VfArgs a) {
  typedef VfRow<F32> Row;
  constexpr int Threads = Lookup ? kVtThreads : kVfThreads, Waves = Threads / kWave;
  __shared__ double s_table[kVfSteps];
  __shared__ double s_lookup[Lookup ? kVtEntries : 1];
  __shared__ int s_sum[Waves], s_at[2];
  const int tid = threadIdx.x, lane = tid % kWave, wave = __builtin_amdgcn_readfirstlane(tid / kWave);

  // all units, this workgroup's, and the request of its first (a lane, from 65
  // requests on a thread, counts a few neighbouring requests; a scan adds up)
  const bool apart = a.B <= kWave;
  const int who = apart ? lane : tid, per = apart ? 1 : (a.B + Threads - 1) / Threads;
  const int b0 = min(who * per, a.B), b1 = min(b0 + per, a.B);
  const VfLoaded loaded = load_request(a, min(b0, a.B - 1));
  fill_table(s_table);
  int mine = b0 < b1 ? request_of(a, loaded).rows * a.chunks : 0;
  for (int i = b0 + 1; i < b1; ++i) mine += request_of(a, i).rows * a.chunks;
  int incl = mine;
#pragma unroll
  for (int x = 1; x < kWave; x <<= 1) {
    const int y = __shfl_up(incl, x);
    if (lane >= x) incl += y;
  }
  int units = __builtin_amdgcn_readlane(incl, kWave - 1);
  if (lane == kWave - 1) s_sum[wave] = incl;
  __syncthreads();
  if (!apart) {
    units = 0;
#pragma unroll
    for (int w = 0; w < Waves; ++w) {
      if (w == wave) incl += units;
      units += s_sum[w];
    }
  }
  const int q = units / gridDim.x, r = units % gridDim.x, g = blockIdx.x;
  int u = g * q + min(g, r);
  const int u_end = u + q + (g < r ? 1 : 0);
  if (u >= u_end) return;
  int b, before;
  const bool here = u >= incl - mine && u < incl;
  if (apart) {
    b = __ffsll((unsigned long long)__ballot(here)) - 1;
    before = __builtin_amdgcn_readlane(incl - mine, b);
  } else {
    if (here) {
      int i = b0, n = incl - mine;
      for (;; ++i) {
        const int k = request_of(a, i).rows * a.chunks;
        if (u < n + k) break;
        n += k;
      }
      s_at[0] = i;
      s_at[1] = n;
    }
    __syncthreads();
    b = __builtin_amdgcn_readfirstlane(s_at[0]);
    before = __builtin_amdgcn_readfirstlane(s_at[1]);
  }

  double filled = 0.0;   // the lookup's c
  for (; u < u_end; ++b) {
    const VfRequest rq = request_of(a, b);
    const bool looks_up = Lookup && rq.warm && rq.c <= kVtMost;
    const int behind = before + rq.rows * a.chunks, upto = min(u_end, behind);
    const double lowest = kVfCut / rq.c;
    const auto row_of = [&](int v, int* ch, size_t* place) {
      const int at = v - before, i = at / a.chunks;
      *ch = at - i * a.chunks;
      const bool drafter = i >= rq.n;
      const int t = rq.first + (drafter ? i - rq.n : i);
      *place = ((size_t)(drafter ? a.T : 0) + t) * a.chunks + *ch;
      return drafter ? a.draft + (size_t)t * a.draft_stride : a.logits + (size_t)t * a.stride;
    };
    int v = u + wave, ch_next = 0;
    size_t place_next = 0;
    Row next;
    if (v < upto) {
      const char* row = row_of(v, &ch_next, &place_next);
      next.load(row, a.V, ch_next, lane);
    }
    if (looks_up && rq.rows > 0 && rq.c != filled) {
      __syncthreads();
      fill_lookup(s_lookup, rq.c, s_table, Threads);
      filled = rq.c;
      __syncthreads();
    }
    for (; v < upto; v += Waves) {
      const Row x = next;
      const int ch = ch_next;
      const size_t place = place_next;
      if (v + Waves < upto) {
        const char* row = row_of(v + Waves, &ch_next, &place_next);
        next.load(row, a.V, ch_next, lane);
      }
      if constexpr (Lookup) {
        if (looks_up) {
          u16x2 at[Row::Vecs][4], most = 0;
#pragma unroll
          for (int j = 0; j < Row::Vecs; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              at[j][e] = places_of(x.v[j][e]);
              most = __builtin_elementwise_max(most, at[j][e]);
            }
          if (!__any(max(most[0], most[1]) >= kVtEntries)) {
            double s = 0.0, s1 = 0.0;
#pragma unroll
            for (int j = 0; j < Row::Vecs; ++j)
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                const uint32_t two = __builtin_bit_cast(uint32_t, at[j][e]);
                s += s_lookup[two & 0xffffu];
                s1 += s_lookup[two >> 16];
              }
            s = wave_sum_f64(s + s1);
            if (lane == 0) a.part[place] = VfPart{s, 0.0f, 0};
            continue;
          }
        }
      }
      float m = kNegInf, some = -kNegInf;   // the least of the vectors' maxima tells whether one is empty
      float most[Row::Vecs];
#pragma unroll
      for (int j = 0; j < Row::Vecs; ++j) {
        most[j] = x.at(j, 0);
#pragma unroll
        for (int e = 1; e < Row::Per; ++e) most[j] = fmaxf(most[j], x.at(j, e));
        m = fmaxf(m, most[j]);
        some = fminf(some, most[j]);
      }
      m = wave_max(m);
      double s = 0.0;
      int at = 0;
      if (!rq.warm) {
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
        const auto add = [&](int j) {
#pragma unroll
          for (int e = 0; e < Row::Per; e += 2) {
            s += exp2_steps(fmax((double)x.at(j, e) - M, lowest), rq.c, s_table);
            s1 += exp2_steps(fmax((double)x.at(j, e + 1) - M, lowest), rq.c, s_table);
          }
        };
        if (!__any(some == kNegInf)) {
#pragma unroll
          for (int j = 0; j < Row::Vecs; ++j) add(j);
        } else {   // a filter has left few tokens: vectors without any are passed over
#pragma unroll
          for (int j = 0; j < Row::Vecs; ++j)
            if (__any(most[j] > kNegInf)) add(j);
        }
        s = wave_sum_f64(s + s1);
      }
      if (lane == 0) a.part[place] = VfPart{s, m, at};
    }
    u = upto;
    before = behind;
  }
}

// ---------------------------------------------------------------------------
// pieces of what follows
// ---------------------------------------------------------------------------
// A chunk's sum brought to the row's reference M.
__device__ __forceinline__ double part_weight(const VfPart& p, float M, double c, const double* table) {
  const double d = (double)p.m - (double)M;
  return d * c > kVfCut ? p.s * exp2_steps(d, c, table) : 0.0;   // (-inf: 0)
}

// By a wave.
__device__ __forceinline__ VfStats row_stats(const VfPart* part, int chunks, bool warm, double c, int lane,
                                             const double* table) {
  VfStats r{0.0, kNegInf, 0};
  for (int ch = lane; ch < chunks; ch += kWave) r.M = fmaxf(r.M, part[ch].m);
  r.M = wave_max(r.M);
  if (!(r.M > kNegInf)) return r;
  if (warm) {
    for (int ch = lane; ch < chunks; ch += kWave) r.Z += part_weight(part[ch], r.M, c, table);
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

// p of one token, and its logarithm.
__device__ __forceinline__ double probability(float x, const VfStats& r, double c, const double* table) {
  const double d = (double)x - (double)r.M;
  return d * c > kVfCut ? exp2_steps(d, c, table) / r.Z : 0.0;
}
__device__ __forceinline__ double exponent(float x, const VfStats& r, double c) {
  return ((double)x - (double)r.M) * c * (0.69314718055994530942 / kVfSteps);
}
__device__ __forceinline__ float log_probability(float x, const VfStats& r, double c) {
  return (float)(exponent(x, r, c) - log(r.Z));
}

// Eight logits from an element on, a thread's of a piece that is looked at again.
constexpr int kVfEight = 8;
template <bool F32>
struct VfEight {
  u32x4 v[F32 ? 2 : 1];
  __device__ __forceinline__ float at(int e) const {
    if constexpr (F32) return __uint_as_float(v[e / 4][e % 4]);
    else return __uint_as_float(e % 2 ? v[0][e / 2] & 0xffff0000u : v[0][e / 2] << 16);
  }
  __device__ __forceinline__ void load(const char* row, int V, int at) {
    if (at + kVfEight <= V) {
      if constexpr (F32) {
        v[0] = load_16<true>(row + (size_t)at * 4);
        v[1] = load_16<true>(row + (size_t)at * 4 + 16);
      } else {
        v[0] = load_16<false>(row + (size_t)at * 2);
      }
    } else {
      v[0] = load_end<F32>(row, V, at);
      if constexpr (F32) v[1] = load_end<F32>(row, V, at + 4);
    }
  }
};

// The weights that a token is drawn from: 2^((x - M) c) of a row, without the
// token `without`, or, where there is a row q, max(p - q, 0).  Of that p and q are
// each off by 1.2e-12 of themselves at most (three terms meet in them) and their
// products are rounded: where they are equal the difference is what that leaves, of
// either sign.  So p is taken less by kVfEqual of itself, and equal ones have none.
constexpr double kVfEqual = 0x1p-39;   // 1.8e-12
template <bool F32>
struct VfWeights {
  const char* p;
  const char* q;
  VfStats sp, sq;
  double c, ip, iq, lowest;
  int without;

  __device__ VfWeights(const char* p_, const VfStats& sp_, const char* q_, const VfStats& sq_, double c_, int without_)
      : p(p_), q(q_), sp(sp_), sq(sq_), c(c_), ip(q_ ? (1.0 - kVfEqual) / sp_.Z : 1.0), iq(q_ ? 1.0 / sq_.Z : 0.0), lowest(kVfCut / c_),
        without(without_) {}

  __device__ __forceinline__ void load(int V, int at, VfEight<F32>& x, VfEight<F32>& y) const {
    x.load(p, V, at);
    if (q) y.load(q, V, at);
  }
  // of eight tokens from their logits in both rows
  __device__ __forceinline__ void of(int at, const VfEight<F32>& x, const VfEight<F32>& y, const double* table,
                                     double (&w)[kVfEight]) const {
#pragma unroll
    for (int e = 0; e < kVfEight; ++e) w[e] = weight_of(x.at(e), sp.M, c, lowest, table);
    if (q) {
#pragma unroll
      for (int e = 0; e < kVfEight; ++e) w[e] = fmax(w[e] * ip - weight_of(y.at(e), sq.M, c, lowest, table) * iq, 0.0);
    }
    if (without >= 0) {
#pragma unroll
      for (int e = 0; e < kVfEight; ++e)
        if (at + e == without) w[e] = 0.0;
    }
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

struct VfDrawn {
  int token;   // -1: all weights are 0
  float x;     // its logit
};
template <int Waves>
struct VfDrawScratch {
  double total[Waves];
  int best[Waves], last[Waves];
  VfDrawn drawn;
};

// A row in pieces, sum_of(piece) the sum of one's weights, the same for every lane
// that asks.  A lane has neighbouring pieces, of which it keeps the first few sums.
constexpr int kVfOwn = 4;
struct VfOwn {
  double sum[kVfOwn];
};
template <typename F>
__device__ __forceinline__ VfOwn own_sums(int pieces, F&& sum_of) {
  const int lane = threadIdx.x % kWave, per = (pieces + kWave - 1) / kWave, c0 = lane * per, c1 = min(c0 + per, pieces);
  VfOwn own;
#pragma unroll
  for (int i = 0; i < kVfOwn; ++i) own.sum[i] = c0 + i < c1 ? sum_of(c0 + i) : 0.0;
  return own;
}

// The token drawn with number u, by a workgroup; all threads get it.  A piece is
// `each` tokens, at most eight a thread.
template <bool F32, int Waves, typename F>
__device__ VfDrawn draw_token(const VfWeights<F32>& weights, int V, int pieces, int each, const double* table, double u,
                              VfDrawScratch<Waves>* s, const VfOwn& own, F&& sum_of) {
  const int tid = threadIdx.x, lane = tid % kWave, wave = __builtin_amdgcn_readfirstlane(tid / kWave);
  // the piece, by every wave for itself: a lane adds up neighbouring pieces
  const int per = (pieces + kWave - 1) / kWave, c0 = min(lane * per, pieces), c1 = min(c0 + per, pieces);
  double mine = 0.0;
#pragma unroll
  for (int i = 0; i < kVfOwn; ++i) mine += own.sum[i];
  for (int k = c0 + kVfOwn; k < c1; ++k) mine += sum_of(k);
  const double incl = wave_scan_f64(mine, lane);
  const double total = readlane_f64(incl, kWave - 1);
  const double target = u * total;
  const unsigned long long some = __ballot(mine > 0.0), over = __ballot(incl > target) & some;
  if (!some) return VfDrawn{-1, 0.0f};
  const int L = over ? __ffsll(over) - 1 : 63 - __clzll(some);
  // of the lane's pieces the first beyond, or the last with any
  double before = readlane_f64(incl - mine, L), held = 0.0;
  int piece = -1;
  bool found = false;
  const auto look = [&](int k, double w) {
    if (found || !(w > 0.0)) return;
    before += held;
    held = w;
    piece = k;
    found = before + w > target;
  };
#pragma unroll
  for (int i = 0; i < kVfOwn; ++i) look(L * per + i, readlane_f64(own.sum[i], L));
  for (int k = L * per + kVfOwn; k < min((L + 1) * per, pieces) && !found; ++k) look(k, sum_of(k));
  piece = __builtin_amdgcn_readfirstlane(piece);
  if (piece < 0 || piece >= pieces) return VfDrawn{-1, 0.0f};

  // its tokens
  const int at = piece * each + tid * kVfEight;
  VfEight<F32> x, y;
  double w[kVfEight], sum = 0.0;
#pragma unroll
  for (int e = 0; e < kVfEight; ++e) w[e] = 0.0;
  if (tid * kVfEight < each) {
    weights.load(V, at, x, y);
    weights.of(at, x, y, table, w);
#pragma unroll
    for (int e = 0; e < kVfEight; ++e) sum += w[e];
  }
  const double in = wave_scan_f64(sum, lane);
  if (lane == kWave - 1) s->total[wave] = in;
  __syncthreads();
  double from = before + (in - sum);
#pragma unroll
  for (int k = 0; k < Waves; ++k)
    if (k < wave) from += s->total[k];
  int best = INT32_MAX, last = -1;
#pragma unroll
  for (int e = 0; e < kVfEight; ++e) {
    from += w[e];
    if (w[e] > 0.0 && at + e < V) {
      last = at + e;
      if (from > target) best = min(best, at + e);
    }
  }
  const int wave_best = wave_min(best), wave_last = -wave_min(-last);
  if (lane == 0) s->best[wave] = wave_best, s->last[wave] = wave_last;
  __syncthreads();
  int token = INT32_MAX, end = -1;
#pragma unroll
  for (int k = 0; k < Waves; ++k) {
    token = min(token, s->best[k]);
    end = max(end, s->last[k]);
  }
  // the piece's sum was formed in another order: past its end by a rounding, its last
  if (token == INT32_MAX) token = end;
  if (token < 0) return VfDrawn{-1, 0.0f};
#pragma unroll
  for (int e = 0; e < kVfEight; ++e)
    if (tid * kVfEight < each && at + e == token) s->drawn = VfDrawn{token, x.at(e)};
  __syncthreads();
  return s->drawn;
}

// ---------------------------------------------------------------------------
// a chain: which drafts stand, the sums of max(p - q, 0) by piece where one fell,
// and the draw.  Every workgroup of a request decides by itself, a wave a draft;
// the first writes it down.  (One launch, the last workgroup of a request to be
// done drawing, took longer than two: to tell it that the others' sums are written
// is to write an XCD's cache back, 48 chains 66 -> 114 to 165 us.)  Chains of loads
// that wait for one another: one chain of five rows of 126464 4.5 us, 48 6.8.
// ---------------------------------------------------------------------------
constexpr int kVdThreads = 1024, kVdWaves = kVdThreads / kWave;
constexpr int kVdPiece = kWave * kVfEight, kVdPieces = kVfChunk / kVdPiece;   // pieces of a chunk

// A wave's pieces of a row: k0, k0 + step, ...
template <bool F32>
__device__ __forceinline__ void rest_sums(const VfWeights<F32>& weights, int V, int k0, int end, int step, double* rest,
                                          const double* table, int lane) {
  constexpr int Ahead = 2;   // pieces under way
  for (; k0 < end; k0 += Ahead * step) {
    VfEight<F32> x[Ahead], y[Ahead];
#pragma unroll
    for (int i = 0; i < Ahead; ++i)
      if (k0 + i * step < end) weights.load(V, (k0 + i * step) * kVdPiece + lane * kVfEight, x[i], y[i]);
#pragma unroll
    for (int i = 0; i < Ahead; ++i) {
      const int k = k0 + i * step;
      if (k >= end) break;
      double w[kVfEight], s = 0.0;
      weights.of(k * kVdPiece + lane * kVfEight, x[i], y[i], table, w);
#pragma unroll
      for (int e = 0; e < kVfEight; ++e) s += w[e];
      s = wave_sum_f64(s);
      if (lane == 0) rest[k] = s;
    }
  }
}

// The token after the drafts that stand, by a workgroup.  of_rest: own sums of max(p - q, 0).
template <bool F32, int Waves>
__device__ void draw_next(const VfArgs& a, int b, const VfChoice& r, bool warm, double c, float u_draw, const VfOwn& of_rest,
                          const double* table, VfDrawScratch<Waves>* scratch) {
  const int tid = threadIdx.x, lane = tid % kWave, wave = __builtin_amdgcn_readfirstlane(tid / kWave);
  const char* row = a.logits + (size_t)r.row * a.stride;
  const VfPart* part = a.part + (size_t)r.row * a.chunks;
  VfDrawn y{-1, 0.0f};
  if (!(r.p.Z > 0.0)) {
    // no token can be
  } else if (!warm) {
    y.token = r.p.first;
  } else {
    const double u = number_of(u_draw);
    if (r.rest && a.draft) {
      const VfWeights<F32> w(row, r.p, a.draft + (size_t)r.row * a.draft_stride, r.q, c, -1);
      const int pieces = a.chunks * kVdPieces;
      const double* rest = a.rest + (size_t)b * pieces;
      y = draw_token(w, a.V, pieces, kVdPiece, table, u, scratch, of_rest, [&](int k) { return rest[k]; });
    } else if (r.rest) {
      // all but the draft: its chunk's sum without it
      const int x = a.ids[r.row + 1];
      const VfWeights<F32> w(row, r.p, nullptr, r.q, c, x >= 0 && x < a.V ? x : -1);
      const int its = w.without >= 0 ? x / kVfChunk : -1;
      double other = 0.0;
      if (its >= 0) {
        if (tid * kVfEight < kVfChunk) {
          VfEight<F32> l;
          double v[kVfEight];
          w.load(a.V, its * kVfChunk + tid * kVfEight, l, l);
          w.of(its * kVfChunk + tid * kVfEight, l, l, table, v);
#pragma unroll
          for (int e = 0; e < kVfEight; ++e) other += v[e];
        }
        other = wave_sum_f64(other);
        if (lane == 0) scratch->total[wave] = other;
        __syncthreads();
        other = 0.0;
#pragma unroll
        for (int k = 0; k < Waves; ++k) other += scratch->total[k];
        __syncthreads();
      }
      const auto sum_of = [&](int ch) { return ch == its ? other : part_weight(part[ch], r.p.M, c, table); };
      y = draw_token(w, a.V, a.chunks, kVfChunk, table, u, scratch, own_sums(a.chunks, sum_of), sum_of);
    }
    if (y.token < 0) {
      const VfWeights<F32> w(row, r.p, nullptr, r.q, c, -1);
      __syncthreads();
      const auto sum_of = [&](int ch) { return part_weight(part[ch], r.p.M, c, table); };
      y = draw_token(w, a.V, a.chunks, kVfChunk, table, u, scratch, own_sums(a.chunks, sum_of), sum_of);
    }
  }
  if (tid == 0) {
    a.tokens[r.row] = y.token;
    if (a.logp) a.logp[r.row] = warm && y.token >= 0 ? log_probability(y.x, r.p, c) : 0.0f;
  }
}

template <bool F32>
__global__ void __launch_bounds__(kVdThreads)
k_vd_decide(const VfArgs a) {
  __shared__ double s_table[kVfSteps];
  __shared__ VfChoice s_choice[kVdWaves];
  __shared__ VfDrawScratch<kVdWaves> s_draw;
  __shared__ double s_exponent[FDLLM_MAX_TREE], s_sum[FDLLM_MAX_TREE];   // of the drafts: their logarithms are taken together
  const int b = blockIdx.y;
  const int tid = threadIdx.x, lane = tid % kWave, wave = __builtin_amdgcn_readfirstlane(tid / kWave);
  const bool writes = blockIdx.x == 0;
  const VfLoaded loaded = load_request(a, b);
  fill_table(s_table);
  const VfRequest rq = request_of(a, loaded);
  const int first = rq.first, n = rq.n;
  if (n == 0) {
    if (writes && tid == 0) {
      a.n_tokens[b] = 0;
      a.choice[b].row = -1;
    }
    return;
  }
  __syncthreads();
  const bool warm = rq.warm, with_q = warm && a.draft;
  const double c = rq.c;
  const VfPart* p_part = a.part + (size_t)first * a.chunks;
  const VfPart* q_part = a.part + ((size_t)a.T + first) * a.chunks;

  // each wave goes on to the first of its drafts that falls, or to the last row
  VfChoice r{};
  int fell = n;
  for (int i = wave; i < n; i += kVdWaves) {
    bool stands = i < n - 1;
    const int x = stands ? a.ids[first + i + 1] : -1;
    const bool real = x >= 0 && x < a.V;
    float lx = 0.0f, lq = 0.0f, u = 0.0f;   // (loaded before the sums are waited for)
    if (real && warm) {
      lx = logit_at<F32>(a.logits + (size_t)(first + i) * a.stride, x);
      if (with_q) lq = logit_at<F32>(a.draft + (size_t)(first + i) * a.draft_stride, x);
      u = a.u[first + i];
    }
    r.p = row_stats(p_part + (size_t)i * a.chunks, a.chunks, warm, c, lane, s_table);
    r.q = VfStats{1.0, 0.0, 0};
    if (stands) {
      if (with_q) r.q = row_stats(q_part + (size_t)i * a.chunks, a.chunks, warm, c, lane, s_table);
      stands = real && r.p.Z > 0.0 && r.q.Z > 0.0;
      if (stands && warm) {
        const double q = with_q ? probability(lq, r.q, c, s_table) : 1.0;
        stands = number_of(u) * q < probability(lx, r.p, c, s_table);
        if (lane == 0) s_exponent[i] = exponent(lx, r.p, c), s_sum[i] = r.p.Z;
      } else if (stands) {
        stands = x == r.p.first;
      }
    }
    if (!stands) {
      fell = i;
      break;
    }
  }
  if (lane == 0) {
    r.row = fell;
    s_choice[wave] = r;
  }
  __syncthreads();
  int who = 0;
#pragma unroll
  for (int w = 1; w < kVdWaves; ++w)
    if (s_choice[w].row < s_choice[who].row) who = w;
  r = s_choice[who];
  const int m = r.row;   // drafts that stand
  r.row += first;
  r.rest = warm && m < n - 1 && r.q.Z > 0.0 && r.p.Z > 0.0;
  if (writes) {
    if (tid == 0) {
      a.choice[b] = r;
      a.n_tokens[b] = m + 1;
    }
    for (int i = tid; i < n; i += kVdThreads) {
      if (i == m) continue;   // (the token drawn)
      a.tokens[first + i] = i < m ? a.ids[first + i + 1] : -1;
      if (a.logp) a.logp[first + i] = i < m && warm ? (float)(s_exponent[i] - log(s_sum[i])) : 0.0f;
    }
  }
  if (!a.draft) {
    draw_next<F32>(a, b, r, warm, c, a.u_draw[b], VfOwn{}, s_table, &s_draw);
  } else if (a.together && r.rest) {
    const VfWeights<F32> weights(a.logits + (size_t)r.row * a.stride, r.p, a.draft + (size_t)r.row * a.draft_stride, r.q, c, -1);
    const int pieces = a.chunks * kVdPieces;
    rest_sums(weights, a.V, blockIdx.x + wave * gridDim.x, pieces, gridDim.x * kVdWaves, a.rest + (size_t)b * pieces, s_table, lane);
  }
}

// The same sums apart, where there are many requests: those that a draft fell of,
// in equal shares whatever their number.  48 chains 9.6 us, half of it the terms in
// 64 bits; the rows come out of the caches.
template <bool F32>
__global__ void __launch_bounds__(kVfThreads)
k_vd_rest(const VfArgs a) {
  __shared__ double s_table[kVfSteps];
  const int tid = threadIdx.x, lane = tid % kWave, wave = __builtin_amdgcn_readfirstlane(tid / kWave);
  const auto has_rest = [&](int b) {
    const VfChoice& r = a.choice[b];
    return r.row >= 0 && r.rest;
  };
  fill_table(s_table);
  __syncthreads();
  // (every wave by itself: a lane counts neighbouring requests)
  const int per = (a.B + kWave - 1) / kWave, b0 = min(lane * per, a.B), b1 = min(b0 + per, a.B);
  int mine = 0;
  for (int b = b0; b < b1; ++b) mine += has_rest(b);
  int incl = mine;
#pragma unroll
  for (int x = 1; x < kWave; x <<= 1) {
    const int y = __shfl_up(incl, x);
    if (lane >= x) incl += y;
  }
  const int requests = __builtin_amdgcn_readlane(incl, kWave - 1), pieces = a.chunks * kVdPieces;
  const long long units = (long long)requests * pieces;
  const long long u_begin = units * blockIdx.x / gridDim.x, u_end = units * (blockIdx.x + 1) / gridDim.x;
  for (long long u = u_begin; u < u_end;) {
    const int k = (int)(u / pieces);            // the k-th of them
    const int L = __ffsll((unsigned long long)__ballot(incl > k)) - 1;
    int b = L * per, left = k - __builtin_amdgcn_readlane(incl - mine, L);
    while (b < a.B - 1 && (!has_rest(b) || left-- > 0)) ++b;
    const long long upto = min(u_end, (long long)(k + 1) * pieces);
    const VfChoice r = a.choice[b];
    double c = 0.0;
    scale_for(temperature_of(a, b), &c);
    const VfWeights<F32> weights(a.logits + (size_t)r.row * a.stride, r.p, a.draft + (size_t)r.row * a.draft_stride, r.q, c, -1);
    const int from = (int)(u - (long long)k * pieces), to = (int)(upto - (long long)k * pieces);
    rest_sums(weights, a.V, from + wave, to, kVfWaves, a.rest + (size_t)b * pieces, s_table, lane);
    u = upto;
  }
}

// The draw apart, where there are a drafter's logits: a workgroup a request, three
// trips to memory (4.6 us for one, 5.5 for 48; the call of 48 63.6 -> 62.4 us by loading
// the sums beside the choice).
template <bool F32>
__global__ void __launch_bounds__(kVfThreads)
k_vd_draw(const VfArgs a) {
  __shared__ double s_table[kVfSteps];
  __shared__ VfDrawScratch<kVfWaves> s_draw;
  const int b = blockIdx.x;
  const VfChoice r = a.choice[b];
  const uint32_t temperature = temperature_of(a, b);
  // (loaded beside the choice, which says whether they are wanted; the sums are loaded in any case)
  const float u_draw = a.T > 0 ? a.u_draw[b] : 0.0f;
  const double* rest = a.rest + (size_t)b * a.chunks * kVdPieces;
  const VfOwn own = own_sums(a.chunks * kVdPieces, [&](int k) { return rest[k]; });
  fill_table(s_table);
  if (r.row < 0) return;
  double c = 0.0;
  const bool warm = scale_for(temperature, &c);
  __syncthreads();
  draw_next<F32>(a, b, r, warm, c, u_draw, own, s_table, &s_draw);
}

// ---------------------------------------------------------------------------
// a tree: a draw at every node, a workgroup each (26 nodes 5.0 us, 16 trees of 11
// to 61 6.0: counts, sums, a chunk, one after another); then the walk, a workgroup
// a request (2.0)
// ---------------------------------------------------------------------------
template <bool F32>
__global__ void __launch_bounds__(kVfThreads)
k_vt_draw(const VfArgs a) {
  __shared__ double s_table[kVfSteps];
  __shared__ VfDrawScratch<kVfWaves> s_draw;
  const int b = blockIdx.y, i = blockIdx.x, tid = threadIdx.x, lane = tid % kWave;
  const VfLoaded loaded = load_request(a, b);
  fill_table(s_table);
  const VfRequest rq = request_of(a, loaded);
  if (i >= rq.n) return;
  __syncthreads();
  const int r = rq.first + i;
  const VfPart* part = a.part + (size_t)r * a.chunks;
  const VfStats sp = row_stats(part, a.chunks, rq.warm, rq.c, lane, s_table);
  VfDrawn y{-1, 0.0f};
  if (sp.Z > 0.0 && rq.warm) {
    const VfWeights<F32> w(a.logits + (size_t)r * a.stride, sp, nullptr, sp, rq.c, -1);
    const auto sum_of = [&](int ch) { return part_weight(part[ch], sp.M, rq.c, s_table); };
    y = draw_token(w, a.V, a.chunks, kVfChunk, s_table, number_of(a.u[r]), &s_draw, own_sums(a.chunks, sum_of), sum_of);
  } else if (sp.Z > 0.0) {
    y.token = sp.first;
  }
  if (tid == 0) {
    a.drawn[r] = y.token;
    a.drawn_lp[r] = rq.warm && y.token >= 0 ? log_probability(y.x, sp, rq.c) : 0.0f;
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
  for (int k = tid; k < n; k += kVfThreads) {
    s_y[k] = a.drawn[first + k];
    s_child[k] = INT32_MAX;
  }
  __syncthreads();
  for (int k = tid; k < n; k += kVfThreads) {
    const int p = a.parents[first + k];
    if (p >= 0 && p < k && s_y[p] >= 0 && a.ids[first + k] == s_y[p]) atomicMin(&s_child[p], k);   // the lowest, in any order
  }
  __syncthreads();
  if (tid == 0) {
    int len = 0;
    for (int k = 0; k < n; k = s_child[k]) s_path[len++] = k;   // children come after their parents
    s_len = len;
    a.n_tokens[b] = len;
  }
  __syncthreads();
  const int len = s_len;
  for (int k = tid; k < n; k += kVfThreads) {
    const int node = k < len ? s_path[k] : -1;
    a.path[first + k] = node;
    a.tokens[first + k] = node >= 0 ? s_y[node] : -1;
    if (a.logp) a.logp[first + k] = node >= 0 ? a.drawn_lp[first + node] : 0.0f;
  }
}

// ---------------------------------------------------------------------------
// host side
// ---------------------------------------------------------------------------
struct VfPlan {
  int chunks;
  size_t at_rest, at_choice, at_drawn, at_lp, bytes;
};

static bool vf_sizes_ok(int T, int B, int V) {
  if (V < 1 || V > (1 << 30) || B > 65535) return false;
  return 2.0 * T * ((V + kVfChunk - 1) / kVfChunk) < 2.0e9;   // chunks are counted in 32 bits
}

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
    if (marginals) p.at_rest = take((size_t)B * p.chunks * kVdPieces * sizeof(double));
  }
  p.bytes = at;
  return p;
}

// Workgroups of the pass that the chip holds at a time.
constexpr int kVfFill = 256 * 4, kVtFill = 256 * 2;
// Chunks two waves have from which the table pays (without it and with; 1.1 a wave:
// 15 chains of 10 rows of 32000 25.2 and 27.4 us, 60 trees of 5 19.6 and 22.3; 1.5, 5
// trees of 20 rows of 126464: 21.1 and 21.4; 1.8, 24 chains of 10 rows of 32000: 30.8
// and 29.3; 2.3, 10 of 8 rows of 126464: 32.5 and 30.3; 800 rows of them 75 and 52).
// It is a loss where requests of few chunks and other temperatures are many, for each
// of which it is filled again: calls just below and above the border, trees of two rows
// of 1000 48.6 and 67.5 us, chains of two 75 and 82, trees of four of 9001 25.7 and 27.5.
constexpr int kVtChunks = 3;
// Requests up to which the decision forms the sums of max(p - q, 0): a workgroup a
// CU in all, and a request that needs none leaves its CUs idle (8 drafts of
// 126464: 16 requests 35.4 us together and 39.8 apart, 32 47.4 and 49.2; six, 64
// 64.1 and 62.5; four, 96 72.9 and 61.6).
constexpr int kVdTogether = 32, kVdFill = 256, kVdRestFill = 256 * 4;

static fdllm_status vf_check(const void* logits, int64_t stride, fdllm_dtype dtype, int T, int V, const int32_t* cu_q, int B,
                             int max_q, const int32_t* n_tokens) {
  if (T < 0 || B < 0 || max_q < 0) return FDLLM_ERR_INVALID_ARG;
  if (dtype != FDLLM_BF16 && dtype != FDLLM_F32) return FDLLM_ERR_UNSUPPORTED_DTYPE;
  if (!vf_sizes_ok(T, B, V) || max_q > FDLLM_MAX_TREE) return FDLLM_ERR_SIZE;
  if (2.0 * B * (max_q < T ? max_q : T) * ((V + kVfChunk - 1) / kVfChunk) >= 2.0e9) return FDLLM_ERR_SIZE;
  if (stride < V) return FDLLM_ERR_INVALID_ARG;
  if ((double)stride * T > 1.0e18) return FDLLM_ERR_SIZE;   // offsets fit 64 bits
  if (B > 0 && (!cu_q || !n_tokens)) return FDLLM_ERR_INVALID_ARG;
  if (T > 0 && !logits) return FDLLM_ERR_INVALID_ARG;
  if ((uintptr_t)logits & (dtype == FDLLM_F32 ? 3 : 1)) return FDLLM_ERR_INVALID_ARG;
  return FDLLM_OK;
}

template <bool F32>
static void vf_sums(const VfArgs& a, hipStream_t st) {
  if (a.T == 0 || a.max_q == 0) return;
  const long long chunks = (long long)a.T * (a.draft ? 2 : 1) * a.chunks;
  if constexpr (!F32) {
    if (2 * chunks >= (long long)kVtFill * (kVtThreads / kWave) * kVtChunks) {
      hipLaunchKernelGGL((k_vf_sums<false, true>), dim3(kVtFill), dim3(kVtThreads), 0, st, a);
      return;
    }
  }
  const long long most = (chunks + kVfWaves - 1) / kVfWaves;
  hipLaunchKernelGGL((k_vf_sums<F32, false>), dim3((unsigned)(most < kVfFill ? most : kVfFill)), dim3(kVfThreads), 0, st, a);
}

template <bool F32>
static hipError_t vd_launch(const VfArgs& a, hipStream_t st) {
  vf_sums<F32>(a, st);
  // with a drafter's logits workgroups for all CUs, of four waves with a piece at least (16 of one
  // CU: a chain of nine rows of 126464 19.7 us for 18.5)
  const int most = (a.chunks * kVdPieces + 3) / 4, fill = kVdFill / a.B;
  VfArgs d = a;
  d.together = a.draft && a.B <= kVdTogether;
  const int parts = !d.together ? 1 : fill < most ? fill : most;
  hipLaunchKernelGGL((k_vd_decide<F32>), dim3((unsigned)parts, (unsigned)a.B), dim3(kVdThreads), 0, st, d);
  if (a.draft && !d.together) hipLaunchKernelGGL((k_vd_rest<F32>), dim3(kVdRestFill), dim3(kVfThreads), 0, st, a);
  if (a.draft) hipLaunchKernelGGL((k_vd_draw<F32>), dim3((unsigned)a.B), dim3(kVfThreads), 0, st, a);
  return hipGetLastError();
}

template <bool F32>
static hipError_t vt_launch(const VfArgs& a, hipStream_t st) {
  vf_sums<F32>(a, st);
  const int rows = a.max_q < a.T ? a.max_q : a.T;
  if (rows > 0) hipLaunchKernelGGL((k_vt_draw<F32>), dim3((unsigned)rows, (unsigned)a.B), dim3(kVfThreads), 0, st, a);
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
  const size_t es = dtype == FDLLM_F32 ? 4 : 2, rows = (size_t)T * 4, counts = (size_t)B * 4;
  if (!apart({{tokens, rows}, {n_tokens, counts}, {logp, rows}},
             {{logits, V * es, logits_stride * es, T}, {draft_logits, V * es, draft_stride * es, T}, {ids, rows}, {cu_q, counts + 4},
              {temperature, counts}, {u, rows}, {u_draw, counts}, {workspace, p.bytes}}))
    return FDLLM_ERR_INVALID_ARG;
  char* ws = (char*)workspace;
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
  const size_t es = dtype == FDLLM_F32 ? 4 : 2, rows = (size_t)T * 4, counts = (size_t)B * 4;
  if (!apart({{path, rows}, {tokens, rows}, {n_tokens, counts}, {logp, rows}},
             {{logits, V * es, logits_stride * es, T}, {ids, rows}, {parents, rows}, {cu_q, counts + 4}, {temperature, counts}, {u, rows},
              {workspace, p.bytes}}))
    return FDLLM_ERR_INVALID_ARG;
  char* ws = (char*)workspace;
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
