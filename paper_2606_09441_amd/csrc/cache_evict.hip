// Eviction: of every (sequence, kv head) the keys of least weight leave the
// cache, and the others move into its first slots.
//
// Kept keys that lie in the first n = min(keys, budget) slots stay; the j-th of
// the others moves to the j-th free slot there.  Sources and destinations are
// different slots, so all rows move in parallel and in place, and as few as can
// be.  The order of a cache's slots means nothing; positions move along.

#include <algorithm>
#include <type_traits>

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
  int b, len, page;
  int late;  // the first position that is protected as recent
  __device__ __forceinline__ Ranks(const CacheEvictArgs& args, int head)
      : p(args), at0(static_cast<int64_t>(head) * (args.c.max_pages << args.c.page_shift)),
        b(head / args.c.hkv), page(1 << args.c.page_shift) {
    len = min(max(p.c.lens[b], 0), p.c.max_pages << p.c.page_shift);
    const int64_t next = p.next_pos != nullptr ? p.next_pos[b] : len;
    late = static_cast<int>(max(next - p.recent, static_cast<int64_t>(-0x7fffffff)));
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
    return used(i) ? rank_of(p.weights[at0 + i], at < p.sinks || at >= late) : 0u;
  }
};

// The numbers that a wavefront has got to: ties seen, rows that move, free slots.
struct Counts {
  int ties, moved, free;
};

// Lists what 64 consecutive slots from i on hold, given the masks of the ranks
// above the n-th and of those equal to it, of which the first `want` are kept.
struct Places {
  const CacheEvictArgs& p;
  const Ranks& x;
  int keep, want;
  __device__ __forceinline__ void list(int i, int lane, uint64_t kept, uint64_t tie,
                                       Counts& c) const {
    const uint64_t before = (uint64_t(1) << lane) - 1;
    int32_t* holes = p.moves + x.at0;
    int32_t* from = holes + (p.c.max_pages << p.c.page_shift) / 2;
    kept |= __ballot(((tie >> lane) & 1) && c.ties + __popcll(tie & before) < want);
    c.ties += __popcll(tie);
    const uint64_t m = low_bits(keep - i), goes = kept & ~m, hole = ~kept & m;
    if ((goes >> lane) & 1) from[c.moved + __popcll(goes & before)] = i + lane;
    if ((hole >> lane) & 1) holes[c.free + __popcll(hole & before)] = i + lane;
    c.moved += __popcll(goes);
    c.free += __popcll(hole);
    // what stays, stays; the free slots among these are written with the moves
    if (i + lane < keep) {
      p.weights_out[x.at0 + i + lane] = p.weights[x.at0 + i + lane];
      p.pos_out[x.at0 + i + lane] = x.pos(i + lane);
    }
  }
};

constexpr int kCopies = 8;       // of the histogram: lanes of one digit rarely meet
constexpr int kHeld = 8;         // ranks of a lane
constexpr int kSelectSlots = kHeld * kThreads;  // longest cache of one workgroup

// One workgroup selects for a (sequence, kv head) of up to kSelectSlots slots,
// the ranks in registers; a wavefront has a sixteenth of the slots, consecutive
// ones.  The n-th largest rank is found by four 8-bit digits, each a histogram
// over the slots that share the digits before; equal ranks go to the lowest
// slots.  Counts of the wavefronts before then give every kept and every free
// slot its number.
__global__ __launch_bounds__(kThreads) void cache_select_kernel(CacheEvictArgs p) {
  __shared__ int hist[256 * kCopies];
  __shared__ int sums[256];
  __shared__ int counts[kSelWaves][4];
  __shared__ int digit, above, found;
  const Ranks x(p, blockIdx.x);
  const int len = x.len;
  const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6);
  const int per = (len + kThreads - 1) / kThreads * 64;  // slots of a wavefront
  const int i0 = min(len, wave * per), i1 = min(len, i0 + per);
  uint32_t r[kHeld];
#pragma unroll
  for (int e = 0; e < kHeld; ++e) {
    const int i = i0 + 64 * e + lane;
    r[e] = len > 0 ? x.rank(min(i, len - 1)) : 0u;
    if (i >= i1) r[e] = 0u;
  }

  uint32_t prefix = 0;  // the digits of the n-th largest rank
  int keep = 0, want = 0;
#pragma unroll 1
  for (int shift = 24; shift >= 0; shift -= 8) {
    for (int i = threadIdx.x; i < 256 * kCopies; i += kThreads) hist[i] = 0;
    __syncthreads();
#pragma unroll
    for (int e = 0; e < kHeld; ++e)
      if (r[e] != 0u && (shift == 24 || (r[e] >> (shift + 8)) == prefix))
        atomicAdd(&hist[((r[e] >> shift) & 255) * kCopies + lane % kCopies], 1);
    __syncthreads();
    if (threadIdx.x < 256) {
      int c = 0;
#pragma unroll
      for (int e = 0; e < kCopies; ++e) c += hist[threadIdx.x * kCopies + (e + lane / 8) % kCopies];
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
      for (int d = 1; d < 64; d <<= 1) {
        const int y = __shfl_up(upto, d);
        if (lane >= d) upto += y;
      }
      if (shift == 24) {
        want = min(__shfl(upto, 63), p.budget);
        if (lane == 0) found = want;
      }
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
    }
    __syncthreads();
    if (shift == 24) keep = want = found;
    if (want > 0) {
      prefix = prefix << 8 | static_cast<uint32_t>(digit);
      want -= above;
    }
  }
  // kept: ranks above `prefix`, and the first `want` slots of that rank

  const auto masks = [&](int e, uint64_t& kept, uint64_t& tie) {
    kept = __ballot(keep > 0 && r[e] > prefix);
    tie = __ballot(keep > 0 && r[e] == prefix);  // (prefix is a key's rank then, not 0)
  };
  // of 64 slots from i on, those before slot `keep`
  const auto low = [&](int i) { return low_bits(keep - i); };
  int n[4] = {0, 0, 0, 0};  // kept and ties, before slot `keep` and from it on
#pragma unroll
  for (int e = 0; e < kHeld; ++e) {
    uint64_t kept, tie;
    masks(e, kept, tie);
    const uint64_t m = low(i0 + 64 * e);
    n[0] += __popcll(kept & m);
    n[1] += __popcll(tie & m);
    n[2] += __popcll(kept & ~m);
    n[3] += __popcll(tie & ~m);
  }
  if (lane < 4) counts[wave][lane] = lane == 0 ? n[0] : lane == 1 ? n[1] : lane == 2 ? n[2] : n[3];
  __syncthreads();
  // of the wavefronts before this one and of all: lanes 0 .. 15 add them up
  int k0 = 0, t0 = 0, k1 = 0, t1 = 0, all_k1 = 0, all_t0 = 0, all_t = 0;
  if (lane < kSelWaves) {
    const int c0 = counts[lane][0], c1 = counts[lane][1], c2 = counts[lane][2],
              c3 = counts[lane][3];
    if (lane < wave) {
      k0 = c0;
      t0 = c1;
      k1 = c2;
      t1 = c3;
    }
    all_k1 = c2;
    all_t0 = c1;
    all_t = c1 + c3;
  }
  for (int d = 8; d > 0; d >>= 1) {
    k0 += __shfl_xor(k0, d);
    t0 += __shfl_xor(t0, d);
    k1 += __shfl_xor(k1, d);
    t1 += __shfl_xor(t1, d);
    all_k1 += __shfl_xor(all_k1, d);
    all_t0 += __shfl_xor(all_t0, d);
    all_t += __shfl_xor(all_t, d);
  }
  const Places at{p, x, keep, want};
  Counts c{uniform(t0 + t1), uniform(k1 + min(want, t0 + t1) - min(want, t0)),
           uniform(min(i0, keep) - k0 - min(want, t0))};
#pragma unroll
  for (int e = 0; e < kHeld; ++e)
    if (i0 + 64 * e < i1) {
      uint64_t kept, tie;
      masks(e, kept, tie);
      at.list(i0 + 64 * e, lane, kept, tie, c);
    }
  if (threadIdx.x == 0) {
    p.num_moves[blockIdx.x] = all_k1 + min(want, all_t) - min(want, all_t0);
    if (blockIdx.x % p.c.hkv == 0) p.lens_out[x.b] = keep;
  }
}

// The same for long caches, the slots dealt over workgroups of kPart: one CU
// needs 0.4 us for every instruction of a walk over 64K slots.  Five launches
// (digits of 10, 11 and 11 bits, counts, lists), each reads the ranks anew; what
// they hand on lies in the handle's scratch.  The histograms are zero between
// calls: a stage clears those that no later one reads.
constexpr int kPart = 2048;
constexpr int kPickWaves = 4;
constexpr int kUnitSlots = kPart / kPickWaves;  // of a wavefront, consecutive ones

__device__ __forceinline__ int* hist_of(const CacheEvictArgs& p, int head, int stage) {
  constexpr int kFrom[3] = {0, 1024, 1024 + 2048};
  return p.hist + static_cast<int64_t>(head) * kEvictHist + kFrom[stage];
}

template <int kStage>
__global__ __launch_bounds__(64 * kPickWaves) void cache_pick_kernel(CacheEvictArgs p, int parts) {
  __shared__ int bins[kStage < 3 ? 2048 : 1];
  __shared__ int tot[kPickWaves], found[2];
  const int head = blockIdx.x / parts, part = blockIdx.x % parts;
  const Ranks x(p, head);
  const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6);
  const int i0 = part * kPart + wave * kUnitSlots + lane;
  uint32_t r[kUnitSlots / 64];
#pragma unroll
  for (int e = 0; e < kUnitSlots / 64; ++e) {
    const int i = i0 + 64 * e;
    r[e] = x.len > 0 ? x.rank(min(i, x.len - 1)) : 0u;
    if (i >= x.len) r[e] = 0u;
  }
  // {digits so far, keys of that prefix still wanted, keys kept}
  int4* state = p.state + 3 * static_cast<int64_t>(head);
  int4 st = kStage >= 2 ? state[kStage == 4 ? 2 : kStage - 2] : int4{0, 0, 0, 0};
  if constexpr (kStage >= 1 && kStage <= 3) {
    // this stage's prefix, from the histogram before: thread t holds kMine bins
    // from the top
    constexpr int kMine = (kStage == 1 ? 1024 : 2048) / (64 * kPickWaves);
    const int* h = hist_of(p, head, kStage - 1);
    const int first = (kStage == 1 ? 1023 : 2047) - kMine * static_cast<int>(threadIdx.x);
    int c[kMine], mine = 0;
#pragma unroll
    for (int e = 0; e < kMine; ++e) {
      c[e] = h[first - e];
      mine += c[e];
    }
    int upto = mine;
    for (int d = 1; d < 64; d <<= 1) {
      const int y = __shfl_up(upto, d);
      if (lane >= d) upto += y;
    }
    if (lane == 63) tot[wave] = upto;
    __syncthreads();
    int all = 0, run = upto - mine;
    for (int w = 0; w < kPickWaves; ++w) {
      if (w < wave) run += tot[w];
      all += tot[w];
    }
    if (kStage == 1) st = int4{0, min(all, p.budget), min(all, p.budget), 0};
#pragma unroll
    for (int e = 0; e < kMine; ++e) {
      if (st.y > 0 && run < st.y && run + c[e] >= st.y) {
        found[0] = first - e;
        found[1] = run;
      }
      run += c[e];
    }
    __syncthreads();
    if (st.y > 0) {
      st.x = static_cast<int>(static_cast<uint32_t>(st.x) << (kStage == 1 ? 10 : 11) |
                              static_cast<uint32_t>(found[0]));
      st.y -= found[1];
    }
    if (part == 0 && threadIdx.x == 0) state[kStage - 1] = st;
  }
  const uint32_t prefix = static_cast<uint32_t>(st.x);
  if constexpr (kStage < 3) {
    for (int i = threadIdx.x; i < 2048; i += 64 * kPickWaves) bins[i] = 0;
    __syncthreads();
    constexpr int kShift = kStage == 0 ? 22 : kStage == 1 ? 11 : 0;
#pragma unroll
    for (int e = 0; e < kUnitSlots / 64; ++e) {
      const bool in = r[e] != 0u && (kStage == 0 || (r[e] >> (kStage == 1 ? 22 : 11)) == prefix);
      if (in) atomicAdd(&bins[(r[e] >> kShift) & (kStage == 0 ? 1023 : 2047)], 1);
    }
    __syncthreads();
    int* h = hist_of(p, head, kStage);
    for (int i = threadIdx.x; i < (kStage == 0 ? 1024 : 2048); i += 64 * kPickWaves)
      if (bins[i] != 0) atomicAdd(&h[i], bins[i]);
    return;
  }
  const int keep = st.z, want = st.y;
  const int unit = part * kPickWaves + wave, units = parts * kPickWaves;
  int4* counts = p.counts + static_cast<int64_t>(head) * units;
  const auto low = [&](int i) { return low_bits(keep - i); };
  const auto masks = [&](int e, uint64_t& kept, uint64_t& tie) {
    kept = __ballot(keep > 0 && r[e] > prefix);
    tie = __ballot(keep > 0 && r[e] == prefix);  // (prefix is a key's rank then, not 0)
  };
  if constexpr (kStage == 3) {
    int4 n{0, 0, 0, 0};  // kept and ties, before slot `keep` and from it on
#pragma unroll
    for (int e = 0; e < kUnitSlots / 64; ++e) {
      uint64_t kept, tie;
      masks(e, kept, tie);
      const uint64_t m = low(i0 - lane + 64 * e);
      n.x += __popcll(kept & m);
      n.y += __popcll(tie & m);
      n.z += __popcll(kept & ~m);
      n.w += __popcll(tie & ~m);
    }
    if (lane == 0) counts[unit] = n;
    if (part == 0)
      for (int i = threadIdx.x; i < 1024 + 2048; i += 64 * kPickWaves) hist_of(p, head, 0)[i] = 0;
  } else {
    // of the units before this one, and of all that the sequence reaches (with those of
    // its capacity the time would grow as the square of that)
    int k0 = 0, t0 = 0, k1 = 0, t1 = 0, all_k1 = 0, all_t0 = 0, all_t = 0;
    const int reached = x.len / kUnitSlots + 1;
    for (int u = lane; u < min(units, reached); u += 64) {
      const int4 n = counts[u];
      if (u < unit) {
        k0 += n.x;
        t0 += n.y;
        k1 += n.z;
        t1 += n.w;
      }
      all_k1 += n.z;
      all_t0 += n.y;
      all_t += n.y + n.w;
    }
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) {
      k0 += __shfl_xor(k0, d);
      t0 += __shfl_xor(t0, d);
      k1 += __shfl_xor(k1, d);
      t1 += __shfl_xor(t1, d);
      all_k1 += __shfl_xor(all_k1, d);
      all_t0 += __shfl_xor(all_t0, d);
      all_t += __shfl_xor(all_t, d);
    }
    // the first `want` ties are kept; those before slot `keep` come first
    const Places at{p, x, keep, want};
    const int first = i0 - lane;
    Counts c{uniform(t0 + t1), uniform(k1 + min(want, t0 + t1) - min(want, t0)),
             uniform(min(first, keep) - k0 - min(want, t0))};
#pragma unroll
    for (int e = 0; e < kUnitSlots / 64; ++e) {
      uint64_t kept, tie;
      masks(e, kept, tie);
      at.list(first + 64 * e, lane, kept, tie, c);
    }
    if (part == 0) {
      for (int i = threadIdx.x; i < 2048; i += 64 * kPickWaves) hist_of(p, head, 2)[i] = 0;
      if (threadIdx.x == 0) {
        p.num_moves[head] = all_k1 + min(want, all_t) - min(want, all_t0);
        if (head % p.c.hkv == 0) p.lens_out[x.b] = keep;
      }
    }
  }
}

constexpr int kMoveRows = 64;    // moves of a workgroup, where that is not too many of them
constexpr int kMoveGroups = 8192;

// The moves of a (sequence, kv head) over per_head workgroups, kRow / 16 lanes a
// row; the slots past the kept ones are cleared on the side.  Bound by HBM.
template <int kRow>
__global__ __launch_bounds__(256) void cache_move_kernel(CacheEvictArgs p, int per_head) {
  const CacheArgs& a = p.c;
  constexpr int kLanes = kRow / 16;
  const int slots = a.max_pages << a.page_shift;
  const int64_t head = blockIdx.x / per_head;
  const int first = static_cast<int>(blockIdx.x % per_head);
  const int n = p.num_moves[head];
  const int b = static_cast<int>(head / a.hkv), kvh = static_cast<int>(head % a.hkv);
  const int64_t at0 = head * slots;
  // (64 bits: a step from the last slots passes 2^31)
  for (int64_t i = p.lens_out[b] + first * 256 + threadIdx.x; i < slots; i += per_head * 256) {
    p.weights_out[at0 + i] = 0.f;
    p.pos_out[at0 + i] = -1;
  }
  const int32_t* holes = p.moves + head * slots;
  const int32_t* from = holes + slots / 2;
  const auto row = [&](int slot) {
    const int32_t t = a.table[static_cast<int64_t>(b) * a.max_pages + (slot >> a.page_shift)];
    const int64_t pg = min(max(t, 0), a.num_pages - 1);
    return (((pg << a.page_shift) + (slot & ((1 << a.page_shift) - 1))) * a.hkv + kvh) * kRow;
  };
  const int ch = threadIdx.x % kLanes;
  constexpr int kAtOnce = 256 / kLanes;
  for (int j = first * kAtOnce + threadIdx.x / kLanes; j < n; j += per_head * kAtOnce) {
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
  const int64_t per = std::max<int64_t>(
      1, std::min((most + kMoveRows - 1) / kMoveRows, (kMoveGroups + heads - 1) / heads));
  // grids of fewer than 2^32 threads
  if (heads >= int64_t(1) << 22 || heads * slots >= int64_t(1) << 33) return hipErrorInvalidValue;
  hipError_t e;
  if (slots <= kSelectSlots) {
    hipLaunchKernelGGL(cache_select_kernel, dim3(static_cast<unsigned>(heads)), dim3(kThreads), 0,
                       stream, a);
    if ((e = hipGetLastError()) != hipSuccess) return e;
  } else {
    const int parts = static_cast<int>((slots + kPart - 1) / kPart);
    const dim3 grid(static_cast<unsigned>(heads * parts)), block(64 * kPickWaves);
    const auto stage = [&](auto k) {
      hipLaunchKernelGGL((cache_pick_kernel<decltype(k)::value>), grid, block, 0, stream, a, parts);
      return hipGetLastError();
    };
    if ((e = stage(std::integral_constant<int, 0>{})) != hipSuccess ||
        (e = stage(std::integral_constant<int, 1>{})) != hipSuccess ||
        (e = stage(std::integral_constant<int, 2>{})) != hipSuccess ||
        (e = stage(std::integral_constant<int, 3>{})) != hipSuccess ||
        (e = stage(std::integral_constant<int, 4>{})) != hipSuccess)
      return e;
  }
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
