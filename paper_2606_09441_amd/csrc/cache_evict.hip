// Eviction: of every (sequence, kv head) the keys of least weight leave the
// cache, and the others move into its first slots.
//
// Kept keys that lie in the first n = min(keys, budget) slots stay; the j-th of
// the others moves to the j-th free slot there.  Sources and destinations are
// different slots, so all rows move in parallel and in place, and as few as can
// be.  The order of a cache's slots means nothing; positions move along.

#include <algorithm>

#include "cache.h"
#include "sift_internal.h"

namespace sift {
namespace {

using namespace cache;

constexpr int kThreads = 1024;
constexpr int kSelWaves = kThreads / 64;

// Order of the keys to be kept: 0: no key; 1: a NaN weight; then by weight;
// all ones: protected.
__device__ __forceinline__ uint32_t rank_of(float w, bool safe) {
  if (safe) return 0xffffffffu;
  if (w != w) return 1u;
  const uint32_t u = __builtin_bit_cast(uint32_t, w + 0.f);  // -0 and 0 tie
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// The weight order of one (sequence, kv head)'s slots.
struct Ranks {
  const CacheEvictArgs& p;
  int64_t at0;
  int b, len, page, next;
  __device__ __forceinline__ Ranks(const CacheEvictArgs& args, int head)
      : p(args), at0(static_cast<int64_t>(head) * (args.c.max_pages << args.c.page_shift)),
        b(head / args.c.hkv), page(1 << args.c.page_shift) {
    len = min(max(p.c.lens[b], 0), p.c.max_pages << p.c.page_shift);
    next = p.next_pos != nullptr ? p.next_pos[b] : len;
  }
  __device__ __forceinline__ int pos(int i) const {
    return p.c.key_pos != nullptr ? p.c.key_pos[at0 + i] : i;
  }
  __device__ __forceinline__ bool used(int i) const {
    return p.c.page_lens == nullptr ||
           (i & (page - 1)) <
               p.c.page_lens[static_cast<int64_t>(b) * p.c.max_pages + (i >> p.c.page_shift)];
  }
  __device__ __forceinline__ uint32_t rank(int i) const {
    const int at = pos(i);
    const bool safe =
        at < p.sinks || static_cast<int64_t>(at) >= static_cast<int64_t>(next) - p.recent;
    return used(i) ? rank_of(p.weights[at0 + i], safe) : 0u;
  }
};

// Ranks of the slots i0 + 64 e + lane of a wavefront, in registers (kPer > 0: at
// most that many to a lane), or made again each time they are asked for.
template <int kPer>
struct Held {
  uint32_t r[kPer];
  __device__ __forceinline__ void load(const Ranks& x, int i0, int i1, int lane) {
#pragma unroll
    for (int e = 0; e < kPer; ++e) {
      const int i = i0 + 64 * e + lane;
      const uint32_t y = x.rank(min(i, x.len - 1));  // (no branch: all loads in flight at once)
      r[e] = i < i1 ? y : 0u;
    }
  }
  template <typename F>
  __device__ __forceinline__ void each(const Ranks&, int i0, int i1, int lane, F f) const {
#pragma unroll
    for (int e = 0; e < kPer; ++e)
      if (i0 + 64 * e < i1) f(i0 + 64 * e, r[e]);
  }
};
template <>
struct Held<0> {
  __device__ __forceinline__ void load(const Ranks&, int, int, int) {}
  template <typename F>
  __device__ __forceinline__ void each(const Ranks& x, int i0, int i1, int lane, F f) const {
    for (int i = i0; i < i1; i += 64) f(i, i + lane < i1 ? x.rank(i + lane) : 0u);
  }
};

constexpr int kCopies = 16;  // of the histogram: lanes of one digit rarely meet

// One workgroup selects for a (sequence, kv head); a wavefront takes a sixteenth
// of the slots, consecutive ones.  The n-th largest rank is found by four 8-bit
// digits, each a histogram over the slots that share the digits before; equal
// ranks go to the lowest slots.  Counts of the wavefronts before then give every
// kept and every free slot its number.  Bound by one CU's reading and LDS
// atomics; the ranks stay in registers, since a walk over memory costs a round
// trip for every 1024 slots.
template <int kPer>
__global__ __launch_bounds__(kThreads) void cache_select_kernel(CacheEvictArgs p) {
  __shared__ int hist[256 * kCopies];
  __shared__ int sums[256];
  __shared__ int wave_cnt[kSelWaves][3];
  __shared__ int digit, above;
  const Ranks x(p, blockIdx.x);
  const int slots = p.c.max_pages << p.c.page_shift;
  const int len = x.len;
  const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6);
  const uint64_t before = (uint64_t(1) << lane) - 1;
  const int per = (len + kThreads - 1) / kThreads * 64;  // slots of a wavefront
  const int i0 = min(len, wave * per), i1 = min(len, i0 + per);
  Held<kPer> held;
  if (len > 0) held.load(x, i0, i1, lane);

  uint32_t prefix = 0;  // the digits of the n-th largest rank
  int keep = 0, want = 0;
  for (int shift = 24; shift >= 0; shift -= 8) {
    for (int i = threadIdx.x; i < 256 * kCopies; i += kThreads) hist[i] = 0;
    __syncthreads();
    held.each(x, i0, i1, lane, [&](int, uint32_t r) {
      const bool in = r != 0u && (shift == 24 || (r >> (shift + 8)) == prefix);
      if (in) atomicAdd(&hist[((r >> shift) & 255) * kCopies + lane % kCopies], 1);
    });
    __syncthreads();
    if (threadIdx.x < 256) {
      int c = 0;
#pragma unroll
      for (int e = 0; e < kCopies; ++e) c += hist[threadIdx.x * kCopies + (e + lane) % kCopies];
      sums[threadIdx.x] = c;
    }
    __syncthreads();
    if (wave == 0) {
      // lane l holds digits 255 - 4 l .. 252 - 4 l
      int c[4], mine = 0;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        c[e] = sums[255 - 4 * lane - e];
        mine += c[e];
      }
      int upto = mine;
#pragma unroll
      for (int d = 1; d < 64; d <<= 1) {
        const int y = __shfl_up(upto, d);
        if (lane >= d) upto += y;
      }
      if (shift == 24) keep = want = min(__shfl(upto, 63), p.budget);
      // the first digit from the top where the count reaches what is wanted
      int run = upto - mine;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        if (want > 0 && run < want && run + c[e] >= want) {
          digit = 255 - 4 * lane - e;
          above = run;
        }
        run += c[e];
      }
      if (shift == 24 && lane == 0) wave_cnt[0][0] = keep;
    }
    __syncthreads();
    if (shift == 24) keep = want = wave_cnt[0][0];
    if (want > 0) {
      prefix = prefix << 8 | static_cast<uint32_t>(digit);
      want -= above;
    }
    __syncthreads();
  }
  // kept: ranks above `prefix`, and the first `want` slots of that rank

  int ties = 0;
  if (keep > 0)
    held.each(x, i0, i1, lane, [&](int, uint32_t r) { ties += __popcll(__ballot(r == prefix)); });
  if (lane == 0) wave_cnt[wave][0] = ties;
  __syncthreads();
  int ties_before = 0;
  for (int w = 0; w < wave; ++w) ties_before += wave_cnt[w][0];

  // `f`(first slot of 64, mask of the kept ones), in slot order
  const auto walk = [&](auto f) {
    int seen = ties_before;
    held.each(x, i0, i1, lane, [&](int i, uint32_t r) {
      const bool tie = keep > 0 && r == prefix;  // (prefix is not 0 then: a key's rank)
      const uint64_t mask = __ballot(tie);
      const bool kept =
          keep > 0 && (r > prefix || (tie && seen + __popcll(mask & before) < want));
      seen += __popcll(mask);
      f(i, __ballot(kept));
    });
  };
  // of 64 slots from i on: those before slot `keep`, and those that exist
  const auto low = [&](int i) { return low_bits(keep - i); };
  int moved = 0, free = 0;
  walk([&](int i, uint64_t kept) {
    moved += __popcll(kept & ~low(i));
    free += __popcll(~kept & low(i) & low_bits(i1 - i));
  });
  if (lane == 0) {
    wave_cnt[wave][1] = moved;
    wave_cnt[wave][2] = free;
  }
  __syncthreads();
  moved = free = 0;
  int all_moved = 0;
  for (int w = 0; w < kSelWaves; ++w) {
    if (w < wave) {
      moved += wave_cnt[w][1];
      free += wave_cnt[w][2];
    }
    all_moved += wave_cnt[w][1];
  }
  int32_t* holes = p.moves + x.at0;
  int32_t* from = holes + slots / 2;
  walk([&](int i, uint64_t kept) {
    const uint64_t goes = kept & ~low(i), hole = ~kept & low(i) & low_bits(i1 - i);
    if ((goes >> lane) & 1) from[moved + __popcll(goes & before)] = i + lane;
    if ((hole >> lane) & 1) holes[free + __popcll(hole & before)] = i + lane;
    if (((kept & low(i)) >> lane) & 1) {
      p.weights_out[x.at0 + i + lane] = p.weights[x.at0 + i + lane];
      p.pos_out[x.at0 + i + lane] = x.pos(i + lane);
    }
    moved += __popcll(goes);
    free += __popcll(hole);
  });
  if (threadIdx.x == 0) {
    p.num_moves[blockIdx.x] = all_moved;
    if (blockIdx.x % p.c.hkv == 0) p.lens_out[x.b] = keep;
  }
}

constexpr int kMoveRows = 64;  // rows of a workgroup

// The moves of a (sequence, kv head), kMoveRows of them a workgroup, kRow / 16
// lanes a row; the slots past the kept ones are cleared on the side.
template <int kRow>
__global__ __launch_bounds__(256) void cache_move_kernel(CacheEvictArgs p, int per_head) {
  const CacheArgs& a = p.c;
  constexpr int kLanes = kRow / 16;
  const int slots = a.max_pages << a.page_shift;
  const int64_t head = blockIdx.x / per_head;
  const int j0 = static_cast<int>(blockIdx.x % per_head) * kMoveRows;
  const int n = p.num_moves[head];
  const int b = static_cast<int>(head / a.hkv), kvh = static_cast<int>(head % a.hkv);
  const int64_t at0 = head * slots;
  for (int i = p.lens_out[b] + static_cast<int>(blockIdx.x % per_head) * 256 + threadIdx.x;
       i < slots; i += per_head * 256) {
    p.weights_out[at0 + i] = 0.f;
    p.pos_out[at0 + i] = -1;
  }
  if (j0 >= n) return;
  const int32_t* holes = p.moves + head * slots;
  const int32_t* from = holes + slots / 2;
  const auto row = [&](int slot) {
    const int32_t t = a.table[static_cast<int64_t>(b) * a.max_pages + (slot >> a.page_shift)];
    const int64_t pg = min(max(t, 0), a.num_pages - 1);
    return (((pg << a.page_shift) + (slot & ((1 << a.page_shift) - 1))) * a.hkv + kvh) * kRow;
  };
  const int ch = threadIdx.x % kLanes;
  for (int j = j0 + threadIdx.x / kLanes; j < min(n, j0 + kMoveRows); j += 256 / kLanes) {
    const int hole = holes[j], slot = from[j];
    const int64_t to = row(hole) + 16 * ch, src = row(slot) + 16 * ch;
    if (ch == 0) {
      p.weights_out[at0 + hole] = p.weights[at0 + slot];
      p.pos_out[at0 + hole] = a.key_pos != nullptr ? a.key_pos[at0 + slot] : slot;
    }
    uint8_t* k = static_cast<uint8_t*>(const_cast<void*>(a.k));
    uint8_t* v = static_cast<uint8_t*>(const_cast<void*>(a.v));
    const u32x4 x = *reinterpret_cast<const u32x4*>(k + src);
    const u32x4 y = *reinterpret_cast<const u32x4*>(v + src);
    *reinterpret_cast<u32x4*>(k + to) = x;
    *reinterpret_cast<u32x4*>(v + to) = y;
  }
}

}  // namespace

hipError_t launch_cache_evict(const CacheEvictArgs& a, int row_bytes, hipStream_t stream) {
  const int64_t heads = static_cast<int64_t>(a.c.num_seqs) * a.c.hkv;
  const int64_t slots = static_cast<int64_t>(a.c.max_pages) << a.c.page_shift;
  const int64_t most = std::min<int64_t>(a.budget, slots / 2);  // moves of a head at most
  const int64_t per = std::max<int64_t>(1, (most + kMoveRows - 1) / kMoveRows);
  // grids of fewer than 2^32 threads
  if (heads >= int64_t(1) << 22 || heads * per >= int64_t(1) << 24) return hipErrorInvalidValue;
  const dim3 sel(static_cast<unsigned>(heads)), threads(kThreads);
  // slots in registers, 1024 to a unit; beyond 72 of them from memory
  if (slots <= 4 * kThreads)
    hipLaunchKernelGGL((cache_select_kernel<4>), sel, threads, 0, stream, a);
  else if (slots <= 20 * kThreads)
    hipLaunchKernelGGL((cache_select_kernel<20>), sel, threads, 0, stream, a);
  else if (slots <= 72 * kThreads)
    hipLaunchKernelGGL((cache_select_kernel<72>), sel, threads, 0, stream, a);
  else
    hipLaunchKernelGGL((cache_select_kernel<0>), sel, threads, 0, stream, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const dim3 grid(static_cast<unsigned>(heads * per)), block(256);
  const int n = static_cast<int>(per);
  if (row_bytes == 128)
    hipLaunchKernelGGL((cache_move_kernel<128>), grid, block, 0, stream, a, n);
  else if (row_bytes == 256)
    hipLaunchKernelGGL((cache_move_kernel<256>), grid, block, 0, stream, a, n);
  else
    hipLaunchKernelGGL((cache_move_kernel<512>), grid, block, 0, stream, a, n);
  return hipGetLastError();
}

}  // namespace sift
