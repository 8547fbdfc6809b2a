// attn_work.h -- which rows a packed sequence has, and where the row tiles of
// prompts whose keys are divided have their scratch: plain functions of the
// cumulated counts, evaluated on the device (the host does not know them); and
// whether a call's results lie apart from its inputs, evaluated on the host.
// Internal to libfdllm.so; compiled for the host as well, to be tested there.
#ifndef FDLLM_ATTN_WORK_H
#define FDLLM_ATTN_WORK_H

#include <stddef.h>
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

// Memory of an argument: `rows` pieces of `bytes`, `stride` bytes from one to the
// next (null: not there).
struct Span {
  uintptr_t p;
  size_t bytes, stride;
  long long rows;
  Span(const void* at, size_t n) : p((uintptr_t)at), bytes(n), stride(n), rows(1) {}
  Span(const void* at, size_t n, size_t step, long long count) : p((uintptr_t)at), bytes(n), stride(step), rows(count) {}
};

// Whether a result, of one piece, shares a byte with it: the first piece that ends
// behind the result's begin is there, and begins before the result's end.
inline bool meets(const Span& result, const Span& s) {
  if (!result.p || !s.p || !result.bytes || !s.bytes || s.rows < 1) return false;
  const uintptr_t begin = result.p, end = result.p + result.bytes;
  uintptr_t at = s.p;
  if (begin >= at + s.bytes && s.rows > 1 && s.stride > 0) {
    const size_t k = (begin - at - s.bytes) / s.stride + 1;
    at += s.stride * (k < (size_t)s.rows ? k : (size_t)s.rows - 1);
  }
  return begin < at + s.bytes && at < end;
}

// Whether no result of a call shares memory with an input, or another result.
inline bool apart(std::initializer_list<Span> results, std::initializer_list<Span> inputs) {
  for (const Span* r = results.begin(); r != results.end(); ++r) {
    for (const Span& i : inputs)
      if (meets(*r, i)) return false;
    for (const Span* o = results.begin(); o != r; ++o)
      if (meets(*r, *o)) return false;
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
