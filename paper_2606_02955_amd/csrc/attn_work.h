// attn_work.h -- which rows a packed sequence has, and where the row tiles of
// prompts whose keys are divided have their scratch: plain functions of the
// cumulated counts, evaluated on the device (the host does not know them).
// Internal to libfdllm.so; compiled for the host as well, to be tested there.
#ifndef FDLLM_ATTN_WORK_H
#define FDLLM_ATTN_WORK_H

#include <stdint.h>

#include <initializer_list>

#ifndef FDLLM_HD
#ifdef __HIPCC__
#define FDLLM_HD __host__ __device__
#else
#define FDLLM_HD
#endif
#endif

namespace fdllm {

// Rows [s, e) of a packed tensor of T rows, as two cumulated counts give them;
// anything else (or more than `most` rows) counts as a sequence without rows.
inline FDLLM_HD int packed_rows(const int32_t* cu, int b, int T, int most, int* first) {
  const int s = cu[b], e = cu[b + 1];
  *first = s;
  return (s >= 0 && s <= e && e <= T && e - s <= most) ? e - s : 0;
}

// Whether no result of a call lies at an input's address, or another result's
// (null: not there).
inline bool apart(std::initializer_list<const void*> results, std::initializer_list<const void*> inputs) {
  for (const void* const* r = results.begin(); r != results.end(); ++r) {
    if (!*r) continue;
    for (const void* i : inputs)
      if (*r == i) return false;
    for (const void* const* o = results.begin(); o != r; ++o)
      if (*r == *o) return false;
  }
  return true;
}

constexpr int kPaRows = 128;   // rows of a row tile: query tokens times the heads of a key head

// Row tiles that a call of T query tokens has at most, where no token is in two
// sequences.
inline FDLLM_HD long long pa_places(int B, int T, int R) { return (long long)T * R / kPaRows + B + 1; }

// A part of the row tiles of the sequences before b: those of sequences from,
// from + step, ...  All parts together are the place of b's first row tile; no
// two row tiles have the same, whatever the order of the sequences' rows.  (The
// place of a token that is in several sequences may lie beyond pa_places.)
inline FDLLM_HD int pa_tiles_before(const int32_t* cu, int b, int T, int max_q, int R, int from, int step) {
  int tiles = 0;
  for (int i = from; i < b; i += step) {
    int first;
    tiles += (int)(((long long)packed_rows(cu, i, T, max_q, &first) * R + kPaRows - 1) / kPaRows);
  }
  return tiles;
}

}  // namespace fdllm

#endif  // FDLLM_ATTN_WORK_H
