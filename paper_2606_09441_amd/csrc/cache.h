// Device pieces of the page cache's kernels: a sequence's sizes, where its keys
// lie, and the even split of all sequences' work over a launch.
#pragma once

#include "flash.h"

namespace sift {
namespace cache {

using namespace flash;

// A wave-uniform load through the scalar cache (no vector-memory counter, so it
// does not wait for the DMAs in flight).
__device__ __forceinline__ int32_t scalar(const int32_t* p, int64_t i) {
  typedef const __attribute__((address_space(4))) int32_t* ptr;
  return ((ptr)p)[i];
}

struct Seq {
  int32_t len;   // slots
  int32_t row0;  // first new token
  int32_t n;     // new tokens
};

// (any lane may ask for its own b)
__device__ __forceinline__ Seq sequence(const CacheArgs& a, int b) {
  Seq s;
  s.len = min(max(a.lens[b], 0), a.max_pages << a.page_shift);
  if (a.row_ptr == nullptr) {
    s.n = a.rows / a.num_seqs;
    s.row0 = b * s.n;
  } else {
    s.row0 = min(max(a.row_ptr[b], 0), a.rows);
    s.n = max(min(min(a.row_ptr[b + 1], a.rows) - s.row0, a.max_rows), 0);
  }
  return s;
}

__device__ __forceinline__ int64_t wave_sum(int64_t x) {
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) x += __shfl_xor(x, d);
  return x;
}

// The work of all sequences, `cost(Seq)` steps each, one after another.
struct Place {
  int32_t b;     // sequence that holds step x, num_seqs past the end
  int64_t at;    // the sequence's first step
};

template <typename Cost>
__device__ __forceinline__ int64_t total_work(const CacheArgs& a, Cost cost) {
  int64_t sum = 0;
  for (int b = threadIdx.x & 63; b < a.num_seqs; b += 64) sum += cost(sequence(a, b));
  return wave_sum(sum);
}

template <typename Cost>
__device__ __forceinline__ Place find_work(const CacheArgs& a, int64_t x, Cost cost) {
  const int lane = threadIdx.x & 63;
  int64_t before = 0;
  for (int b0 = 0; b0 < a.num_seqs; b0 += 64) {
    const int64_t mine = b0 + lane < a.num_seqs ? cost(sequence(a, b0 + lane)) : 0;
    int64_t upto = mine;  // inclusive scan
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const int64_t y = __shfl_up(upto, d);
      if (lane >= d) upto += y;
    }
    const uint64_t past = __ballot(before + upto > x);
    if (past != 0) {
      const int l = __ffsll(static_cast<unsigned long long>(past)) - 1;
      return Place{b0 + l, before + __shfl(upto - mine, l)};
    }
    before += __shfl(upto, 63);
  }
  return Place{a.num_seqs, before};
}

// The sequence that new token `token` belongs to (num_seqs: none), and its first
// step.
template <typename Cost>
__device__ __forceinline__ Place find_token(const CacheArgs& a, int token, Cost cost) {
  const int lane = threadIdx.x & 63;
  int64_t before = 0;
  for (int b0 = 0; b0 < a.num_seqs; b0 += 64) {
    const bool in = b0 + lane < a.num_seqs;
    const Seq s = sequence(a, min(b0 + lane, a.num_seqs - 1));
    const int64_t mine = in ? cost(s) : 0;
    const uint64_t has = __ballot(in && token >= s.row0 && token < s.row0 + s.n);
    if (has != 0) {
      const int l = __ffsll(static_cast<unsigned long long>(has)) - 1;
      return Place{b0 + l, before + wave_sum(lane < l ? mine : 0)};
    }
    before += wave_sum(mine);
  }
  return Place{a.num_seqs, before};
}

// Steps x of [0, total) go to workgroup share_of(x): workgroup i takes those
// from share(i) to share(i + 1).  groups <= total: every workgroup has some.
__device__ __forceinline__ int64_t share(int64_t i, int64_t total, int64_t groups) {
  return i * total / groups;
}
__device__ __forceinline__ int64_t share_of(int64_t x, int64_t total, int64_t groups) {
  return ((x + 1) * groups - 1) / total;
}

// 16 rows of keys: where, and how many are valid.
struct Rows16 {
  int64_t row;  // of the pool, or of the new tokens
  int32_t n;    // 0 .. 16
};

// Slots slot .. slot + 15 (slot a multiple of 16) of sequence b.  All scalar.
__device__ __forceinline__ Rows16 cached_rows(const CacheArgs& a, int b, int len, int slot) {
  const int pi = min(slot >> a.page_shift, a.max_pages - 1);
  const int in = slot & ((1 << a.page_shift) - 1);
  const int64_t at = static_cast<int64_t>(b) * a.max_pages + pi;
  int n = len - slot;
  if (a.page_lens != nullptr) n = min(n, scalar(a.page_lens, at) - in);
  const int page = min(max(scalar(a.table, at), 0), a.num_pages - 1);
  return Rows16{(static_cast<int64_t>(page) << a.page_shift) + in, min(max(n, 0), 16)};
}

// Scores of a block whose keys' positions are not consecutive.
__device__ __forceinline__ void score_block_at(const ScoreArgs& sc, float slope,
                                               const int (&dist)[16], f32x16& s) {
  if (sc.x != 0.f) cap_scores(sc, s);
  const float c = sc.x != 0.f ? 1.f : sc.c;
#pragma unroll
  for (int v = 0; v < 16; ++v)
    s[v] = fmaf(s[v], c, -slope * fabsf(static_cast<float>(dist[v])));
}

}  // namespace cache
}  // namespace sift
