// Device pieces of the page cache's kernels: a sequence's sizes, where its keys
// lie, and the even split of all sequences' work over a launch.
#pragma once

#include "clamp.h"
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

__device__ __forceinline__ float scalar(const float* p, int64_t i) {
  typedef const __attribute__((address_space(4))) float* ptr;
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
  s.len = within(a.lens[b], a.max_pages << a.page_shift);
  if (a.row_ptr == nullptr) {
    s.n = a.rows / a.num_seqs;
    s.row0 = b * s.n;
  } else {
    s.row0 = within(a.row_ptr[b], a.rows);
    s.n = rows_between(s.row0, a.row_ptr[b + 1], a.rows, a.max_rows);
  }
  return s;
}

__device__ __forceinline__ int wave_sum(int x) {
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) x += __shfl_xor(x, d);
  return uniform(x);
}

__device__ __forceinline__ int lane_value(int x, int lane) {
  return __builtin_amdgcn_readlane(x, lane);
}

// The work of all sequences, cost(Seq) steps each, one after another: fewer than
// 2^31 (checked by the host).  All uniform.
struct Place {
  int32_t b;   // sequence that holds a step, num_seqs past the end
  int32_t at;  // the sequence's first step
};

template <typename Cost>
struct Work {
  const CacheArgs& a;
  const Cost cost;
  // of sequence `lane`, the first 64: their sizes, and their steps with those before
  Seq mine;
  int upto;
  int first, total;  // steps of the first 64, and of all
  __device__ __forceinline__ Work(const CacheArgs& args, Cost c) : a(args), cost(c) {
    const int lane = threadIdx.x & 63;
    mine = sequence(a, min(lane, a.num_seqs - 1));
    upto = scan(lane < a.num_seqs ? cost(mine) : 0);
    first = total = lane_value(upto, 63);
    if (a.num_seqs <= 64) return;
    int sum = 0;
    for (int b = 64 + lane; b < a.num_seqs; b += 64) sum += cost(sequence(a, b));
    total += wave_sum(sum);
  }
  static __device__ __forceinline__ int scan(int x) {  // inclusive
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const int y = __shfl_up(x, d);
      if (lane >= d) x += y;
    }
    return x;
  }
  static __device__ __forceinline__ Place among(int b0, int before, int upto, int x) {
    const int l =
        __ffsll(static_cast<unsigned long long>(__ballot(before + upto > x))) - 1;  // there is one
    return Place{b0 + l, before + (l > 0 ? lane_value(upto, l - 1) : 0)};
  }
  // The place of step x.
  __device__ __forceinline__ Place find(int x) const {
    if (x < first) return among(0, 0, upto, x);
    const int lane = threadIdx.x & 63;
    int before = first;
    for (int b0 = 64; b0 < a.num_seqs; b0 += 64) {
      const int u = scan(b0 + lane < a.num_seqs ? cost(sequence(a, b0 + lane)) : 0);
      const int all = lane_value(u, 63);
      if (x < before + all) return among(b0, before, u, x);
      before += all;
    }
    return Place{a.num_seqs, before};
  }
  // The sequence that new token `token` belongs to, and its first step.
  __device__ __forceinline__ Place find_token(int token) const {
    const int lane = threadIdx.x & 63;
    const auto has = [&](const Seq& s, bool in) {
      return __ballot(in && token >= s.row0 && token < s.row0 + s.n);
    };
    uint64_t m = has(mine, lane < a.num_seqs);
    int before = 0, u = upto, b0 = 0;
    while (m == 0) {
      before += lane_value(u, 63);
      b0 += 64;
      if (b0 >= a.num_seqs) return Place{a.num_seqs, before};
      const Seq s = sequence(a, min(b0 + lane, a.num_seqs - 1));
      const bool in = b0 + lane < a.num_seqs;
      u = scan(in ? cost(s) : 0);
      m = has(s, in);
    }
    const int l = __ffsll(static_cast<unsigned long long>(m)) - 1;
    return Place{b0 + l, before + (l > 0 ? lane_value(u, l - 1) : 0)};
  }
  __device__ __forceinline__ Seq seq(int b) const {
    if (b < 64) return Seq{lane_value(mine.len, b), lane_value(mine.row0, b), lane_value(mine.n, b)};
    if (b >= a.num_seqs) return Seq{0, 0, 0};
    const Seq s = sequence(a, b);
    return Seq{uniform(s.len), uniform(s.row0), uniform(s.n)};
  }
};

// An even split of `total` steps over the workgroups of a launch, or over as many
// as there are steps: workgroup i takes those from at(i) to at(i + 1).
struct Split {
  int total, groups, each, more;  // total = groups * each + more
  __device__ __forceinline__ Split(int total_, int launched)
      : total(total_), groups(min(total_, launched)) {
    each = groups > 0 ? quotient(total, groups) : 0;
    more = total - each * groups;
  }
  static __device__ __forceinline__ int quotient(int x, int y) {
    return uniform(static_cast<int>(static_cast<unsigned>(x) / static_cast<unsigned>(y)));
  }
  // the first `more` workgroups take one step more
  __device__ __forceinline__ int at(int i) const { return i * each + min(i, more); }
  __device__ __forceinline__ int of(int x) const {
    const int big = more * (each + 1);  // steps of the first ones
    return uniform(x < big ? quotient(x, each + 1) : more + quotient(x - big, each));
  }
};

// The units of an attention: kRows rows (new token, query head) of a (sequence, kv
// head) over all its keys, in steps.
struct Narrow {  // four 32-key tiles a step
  static constexpr int kRows = 32;
  static constexpr int kTileKeys = 32, kStepTiles = 4;
  static constexpr int kLead = 0;  // steps of a unit that are none: what beginning it costs
};
struct Wide {    // a 64-key tile a step
  static constexpr int kRows = 128;
  static constexpr int kTileKeys = 64, kStepTiles = 1;
  static constexpr int kLead = 0;
};
// A unit of codes costs about two steps more than its own: its tables, the queries, the
// first tiles' way, the merge of its wavefronts.  Counted in the split, the workgroups with
// several short sequences do not end last: us of 32 sequences of 200 to 16640 slots with
// none / one / two / four 80 / 68 / 68 / 68.4, of 16 such 42 / 36 / 34 / 36, of 20 of 30 to
// 30000 66 / 50 / 46 / -, of 32 of 300 20 / 18 / 21 / 21.5 (so batches of short sequences
// lose a little: two are for the longer calls).
struct NarrowCodes : Narrow {
  static constexpr int kLead = 2;
};
template <typename U>
struct UnitCost {
  int32_t g, hkv;
  __device__ __forceinline__ int blocks(const Seq& s) const {
    return (s.n * g + U::kRows - 1) / U::kRows;
  }
  static __device__ __forceinline__ int cached_tiles(const Seq& s) {
    return (s.len + U::kTileKeys - 1) / U::kTileKeys;
  }
  static __device__ __forceinline__ int tiles(const Seq& s) {
    return cached_tiles(s) + (s.n + U::kTileKeys - 1) / U::kTileKeys;
  }
  static __device__ __forceinline__ int steps(const Seq& s) {
    return U::kLead + (tiles(s) + U::kStepTiles - 1) / U::kStepTiles;
  }
  __device__ __forceinline__ int operator()(const Seq& s) const {
    return hkv * blocks(s) * steps(s);
  }
};

// A workgroup's place in the list of steps.  Workgroups go round-robin over the
// XCDs: where all have work, those of an XCD take neighbouring shares, so that
// units of the same keys meet in its L2.
__device__ __forceinline__ int group_of(const Split& split) {
  if (split.groups < static_cast<int>(gridDim.x) || split.groups % kNumXcd != 0) return blockIdx.x;
  return blockIdx.x % kNumXcd * (split.groups / kNumXcd) + blockIdx.x / kNumXcd;
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
  const int n = a.page_lens != nullptr ? keys_of_page(scalar(a.page_lens, at), in, len - slot)
                                       : within(len - slot, 16);
  const int page = within(scalar(a.table, at), a.num_pages - 1);
  return Rows16{(static_cast<int64_t>(page) << a.page_shift) + in, n};
}

}  // namespace cache
}  // namespace sift
