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

// One workgroup selects for a (sequence, kv head).  The n-th largest rank is
// found by four 8-bit digits, each a histogram over the slots that share the
// digits before; equal ranks go to the lowest slots.  Wavefront w then walks the
// slots of its own sixteenth in order, so that counts before it give every kept
// and every free slot its number.
__global__ __launch_bounds__(kThreads) void cache_select_kernel(CacheEvictArgs p) {
  const CacheArgs& a = p.c;
  __shared__ int hist[256];
  __shared__ int wave_cnt[kSelWaves][3];
  __shared__ int digit, above;
  const int b = blockIdx.x / a.hkv;
  const int slots = a.max_pages << a.page_shift;
  const int page = 1 << a.page_shift;
  const int len = min(max(a.lens[b], 0), slots);
  const int64_t at0 = static_cast<int64_t>(blockIdx.x) * slots;
  const int next = p.next_pos != nullptr ? p.next_pos[b] : len;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;

  const auto pos_at = [&](int i) { return a.key_pos != nullptr ? a.key_pos[at0 + i] : i; };
  const auto rank = [&](int i) -> uint32_t {
    if (a.page_lens != nullptr &&
        (i & (page - 1)) >= a.page_lens[static_cast<int64_t>(b) * a.max_pages + (i >> a.page_shift)])
      return 0u;
    const int pos = pos_at(i);
    return rank_of(p.weights[at0 + i],
                   pos < p.sinks || static_cast<int64_t>(pos) >= static_cast<int64_t>(next) - p.recent);
  };

  // the digits of the n-th largest rank
  uint32_t prefix = 0;
  int keep = 0, want = 0;
  for (int shift = 24; shift >= 0; shift -= 8) {
    if (threadIdx.x < 256) hist[threadIdx.x] = 0;
    __syncthreads();
    int keys = 0;
    for (int i = threadIdx.x; i < len; i += kThreads) {
      const uint32_t r = rank(i);
      keys += r != 0;
      if (shift == 24 ? r != 0 : (r >> (shift + 8)) == prefix) atomicAdd(&hist[(r >> shift) & 255], 1);
    }
    if (shift == 24) {
#pragma unroll
      for (int d = 32; d > 0; d >>= 1) keys += __shfl_xor(keys, d);
      if (lane == 0) wave_cnt[wave][0] = keys;
    }
    __syncthreads();
    if (shift == 24) {
      int all = 0;
      for (int w = 0; w < kSelWaves; ++w) all += wave_cnt[w][0];
      keep = want = min(all, p.budget);
    }
    // the first digit from the top where the count reaches what is wanted
    if (wave == 0) {
      // lane l holds digits 255 - 4 l .. 252 - 4 l
      int c[4], mine = 0;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        c[e] = hist[255 - 4 * lane - e];
        mine += c[e];
      }
      int upto = mine;
#pragma unroll
      for (int d = 1; d < 64; d <<= 1) {
        const int y = __shfl_up(upto, d);
        if (lane >= d) upto += y;
      }
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
    if (want > 0) {
      prefix = prefix << 8 | static_cast<uint32_t>(digit);
      want -= above;
    }
    __syncthreads();
  }
  // kept: ranks above `prefix`, and the first `want` slots of that rank

  const int per = (len + kSelWaves * 64 - 1) / (kSelWaves * 64) * 64;  // slots of a wavefront
  const int i0 = min(len, wave * per), i1 = min(len, i0 + per);
  int ties = 0;
  if (keep > 0)
    for (int i = i0 + lane; i < i1; i += 64) ties += rank(i) == prefix;
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) ties += __shfl_xor(ties, d);
  if (lane == 0) wave_cnt[wave][0] = ties;
  __syncthreads();
  int ties_before = 0;
  for (int w = 0; w < wave; ++w) ties_before += wave_cnt[w][0];

  // `each`(slot, in range, kept), in slot order
  const auto walk = [&](auto each) {
    int seen = ties_before;
    for (int i = i0 + lane; i - lane < i1; i += 64) {
      const uint32_t r = i < i1 && keep > 0 ? rank(i) : 0u;
      const bool tie = r != 0u && r == prefix;
      const uint64_t mask = __ballot(tie);
      const int place = seen + __popcll(mask & ((uint64_t(1) << lane) - 1));
      each(i, i < i1, r > prefix || (tie && place < want));
      seen += __popcll(mask);
    }
  };
  int moved = 0, free = 0;
  walk([&](int i, bool in, bool kept) {
    moved += __popcll(__ballot(in && kept && i >= keep));
    free += __popcll(__ballot(in && !kept && i < keep));
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
  int32_t* holes = p.moves + at0;
  int32_t* from = holes + slots / 2;
  walk([&](int i, bool in, bool kept) {
    const uint64_t before = (uint64_t(1) << lane) - 1;
    const bool goes = in && kept && i >= keep, hole = in && !kept && i < keep;
    const uint64_t gm = __ballot(goes), hm = __ballot(hole);
    if (goes) from[moved + __popcll(gm & before)] = i;
    if (hole) holes[free + __popcll(hm & before)] = i;
    if (in && kept && i < keep) {
      p.weights_out[at0 + i] = p.weights[at0 + i];
      p.pos_out[at0 + i] = pos_at(i);
    }
    moved += __popcll(gm);
    free += __popcll(hm);
  });
  __syncthreads();
  for (int j = threadIdx.x; j < all_moved; j += kThreads) {
    const int to = holes[j], i = from[j];
    p.weights_out[at0 + to] = p.weights[at0 + i];
    p.pos_out[at0 + to] = pos_at(i);
  }
  for (int i = keep + threadIdx.x; i < slots; i += kThreads) {
    p.weights_out[at0 + i] = 0.f;
    p.pos_out[at0 + i] = -1;
  }
  if (threadIdx.x == 0) {
    p.num_moves[blockIdx.x] = all_moved;
    if (blockIdx.x % a.hkv == 0) p.lens_out[b] = keep;
  }
}

constexpr int kMoveRows = 64;  // rows of a workgroup

// kRow bytes a row: kRow / 16 lanes each.
template <int kRow>
__global__ __launch_bounds__(256) void cache_move_kernel(CacheEvictArgs p, int per_head) {
  const CacheArgs& a = p.c;
  constexpr int kLanes = kRow / 16;
  const int slots = a.max_pages << a.page_shift;
  const int64_t head = blockIdx.x / per_head;
  const int j0 = static_cast<int>(blockIdx.x % per_head) * kMoveRows;
  const int n = p.num_moves[head];
  if (j0 >= n) return;
  const int b = static_cast<int>(head / a.hkv), kvh = static_cast<int>(head % a.hkv);
  const int32_t* holes = p.moves + head * slots;
  const int32_t* from = holes + slots / 2;
  const auto row = [&](int slot) {
    const int32_t t = a.table[static_cast<int64_t>(b) * a.max_pages + (slot >> a.page_shift)];
    const int64_t pg = min(max(t, 0), a.num_pages - 1);
    return (((pg << a.page_shift) + (slot & ((1 << a.page_shift) - 1))) * a.hkv + kvh) * kRow;
  };
  const int ch = threadIdx.x % kLanes;
  for (int j = j0 + threadIdx.x / kLanes; j < min(n, j0 + kMoveRows); j += 256 / kLanes) {
    const int64_t to = row(holes[j]) + 16 * ch, src = row(from[j]) + 16 * ch;
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
  hipLaunchKernelGGL(cache_select_kernel, dim3(static_cast<unsigned>(heads)), dim3(kThreads), 0,
                     stream, a);
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
