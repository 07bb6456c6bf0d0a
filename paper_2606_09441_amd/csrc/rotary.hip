// Rotary positions of q and k (sift_rotate): any frequency table, half or interleaved
// pairs, part of the head, in place or not; the transpose with the angles negative.
//
// HBM bounds it: every number is read once and written once.  A wavefront takes a
// token: each lane one item (two 16-byte chunks of halves, or one of whole pairs) of
// the heads that it goes through, whose angles it forms once.  Where there are few
// tokens their heads are split over several wavefronts.  16640 tokens of 32/8 heads, D =
// 128, bf16: 60 us, 5.7 TB/s (a copy reaches 4.9 to 5.2); 66048 of 48/8 with the
// gradient, two launches: 683 us, 5.5 TB/s; 32 tokens 3.0 us.

#include <algorithm>

#include "rotary.h"

namespace sift {
namespace {

using namespace rotary;

constexpr int kAhead = 4;  // items whose loads a lane has under way
// Wavefronts that a launch of few tokens is split into (us of 40 heads, D = 128, one a
// token / 4096 / 32768: 1 token 2.9 / 2.2 / 2.2, 32 tokens 4.0 / 3.0 / 3.0, 2000 tokens
// 8.5 / 8.4 / 9.7).
constexpr int64_t kRotateWaves = 4096;

// q's heads, then k's, of a token.
template <typename P>
__device__ __forceinline__ P* head_of(P* q, P* k, const RotateArgs& a, int64_t token, int h) {
  return h < a.hq ? q + (token * a.hq + h) * a.d : k + (token * a.hk + (h - a.hq)) * a.d;
}

template <typename T, bool kInterleaved>
__global__ __launch_bounds__(256) void rotate_kernel(RotateArgs a, int parts) {
  using I = Item<T, kInterleaved>;
  constexpr int n = Chunk<T>::kCount;
  const int lane = threadIdx.x & 63;
  const int heads = a.hq + a.hk;
  const int items = a.r.half / I::kAngles;         // of a head
  const int at_once = 64 / items;                  // heads
  const int item = lane % items, sub = lane / items;
  const int gap = a.r.half;                        // between an item's chunks
  const T* const q = static_cast<const T*>(a.q);
  const T* const k = static_cast<const T*>(a.k);
  T* const qo = static_cast<T*>(a.q_out);
  T* const ko = static_cast<T*>(a.k_out);
  const int64_t units = a.tokens * parts;
  for (int64_t u = static_cast<int64_t>(blockIdx.x) * 4 + (threadIdx.x >> 6); u < units;
       u += static_cast<int64_t>(gridDim.x) * 4) {
    const int64_t token = u / parts;
    const int part = static_cast<int>(u - token * parts);
    const int first = part * at_once + sub, step = parts * at_once;
    I it;
    bool made = false;
    for (int h0 = first; h0 < heads && sub < at_once; h0 += kAhead * step) {
      u32x4 x[kAhead][I::kChunks];
#pragma unroll
      for (int i = 0; i < kAhead; ++i) {
        const int h = h0 + i * step;
        if (h >= heads) break;
        const T* p = head_of(q, k, a, token, h) + item * n;
#pragma unroll
        for (int j = 0; j < I::kChunks; ++j) x[i][j] = *reinterpret_cast<const u32x4*>(p + j * gap);
      }
      if (!made) it.angles(a.r, a.positions[token], item);
      made = true;
#pragma unroll
      for (int i = 0; i < kAhead; ++i) {
        const int h = h0 + i * step;
        if (h >= heads) break;
        Chunk<T> y[I::kChunks];
#pragma unroll
        for (int j = 0; j < I::kChunks; ++j) y[j].set(x[i][j]);
        it.apply(y);
        T* p = head_of(qo, ko, a, token, h) + item * n;
#pragma unroll
        for (int j = 0; j < I::kChunks; ++j) *reinterpret_cast<u32x4*>(p + j * gap) = y[j].get();
      }
    }
    // the dims that do not turn
    const int rest = a.d / n - 2 * gap / n;
    if (!a.copy || rest == 0) continue;
    for (int e = part * 64 + lane; e < heads * rest; e += parts * 64) {
      const int h = e / rest, c = 2 * gap + (e - h * rest) * n;
      *reinterpret_cast<u32x4*>(head_of(qo, ko, a, token, h) + c) =
          *reinterpret_cast<const u32x4*>(head_of(q, k, a, token, h) + c);
    }
  }
}

__device__ __forceinline__ float value(float x) { return x; }
__device__ __forceinline__ float value(__bf16 x) { return static_cast<float>(x); }

// Whole chunks whose pairs lie anywhere (a part of the head that is no multiple of them):
// a lane takes a chunk of a head, and the other halves of its pairs from LDS, where the
// head's lanes leave theirs.  16640 tokens of 32/8 heads, 100 of 128 dims turning: 81 us, a
// pair at a time 186; interleaved 63 and 188.
template <typename T, bool kInterleaved>
__global__ __launch_bounds__(256) void rotate_chunks_kernel(RotateArgs a, int parts) {
  constexpr int n = Chunk<T>::kCount;
  __shared__ u32x4 seen[4][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int heads = a.hq + a.hk;
  const int chunks = a.d / n, at_once = 64 / chunks;  // of a head; heads
  const int chunk = lane % chunks, sub = lane / chunks;
  const T* const head = reinterpret_cast<const T*>(&seen[wave][sub * chunks]);
  const T* const q = static_cast<const T*>(a.q);
  const T* const k = static_cast<const T*>(a.k);
  T* const qo = static_cast<T*>(a.q_out);
  T* const ko = static_cast<T*>(a.k_out);
  const int64_t units = a.tokens * parts;
  for (int64_t u = static_cast<int64_t>(blockIdx.x) * 4 + wave; u < units;
       u += static_cast<int64_t>(gridDim.x) * 4) {
    const int64_t token = u / parts;
    const int part = static_cast<int>(u - token * parts);
    const int step = parts * at_once;
    AnyChunk<T, kInterleaved> it;
    it.angles(a.r, a.positions[token], chunk);
    for (int h0 = part * at_once + sub; h0 < heads && sub < at_once; h0 += kAhead * step) {
      u32x4 x[kAhead];
#pragma unroll
      for (int i = 0; i < kAhead; ++i)
        if (h0 + i * step < heads)
          x[i] = *reinterpret_cast<const u32x4*>(head_of(q, k, a, token, h0 + i * step) + chunk * n);
#pragma unroll
      for (int i = 0; i < kAhead; ++i) {
        const int h = h0 + i * step;
        if (h >= heads) break;
        if constexpr (!kInterleaved) seen[wave][lane] = x[i];
        lds_order();
        Chunk<T> y;
        y.set(x[i]);
        it.apply(a.r, y, head);
        lds_order();
        *reinterpret_cast<u32x4*>(head_of(qo, ko, a, token, h) + chunk * n) = y.get();
      }
    }
  }
}

// Any sizes and alignment: a lane takes a pair of all heads that its wavefront goes
// through, then dims that stay.
template <typename T>
__global__ __launch_bounds__(256) void rotate_pairs_kernel(RotateArgs a, int parts) {
  const int lane = threadIdx.x & 63;
  const int heads = a.hq + a.hk;
  const T* const q = static_cast<const T*>(a.q);
  const T* const k = static_cast<const T*>(a.k);
  T* const qo = static_cast<T*>(a.q_out);
  T* const ko = static_cast<T*>(a.k_out);
  const int64_t units = a.tokens * parts;
  for (int64_t u = static_cast<int64_t>(blockIdx.x) * 4 + (threadIdx.x >> 6); u < units;
       u += static_cast<int64_t>(gridDim.x) * 4) {
    const int64_t token = u / parts;
    const int part = static_cast<int>(u - token * parts);
    const int pos = a.positions[token];
    for (int i = lane; i < a.r.half; i += 64) {
      float c, s;
      turn<T>(a.r, pos, i, c, s);
      const int d0 = a.r.interleaved ? 2 * i : i, d1 = a.r.interleaved ? d0 + 1 : a.r.half + i;
      for (int h0 = part; h0 < heads; h0 += kAhead * parts) {
        float x[kAhead], y[kAhead];
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
          if (h0 + j * parts >= heads) break;
          const T* p = head_of(q, k, a, token, h0 + j * parts);
          x[j] = value(p[d0]);
          y[j] = value(p[d1]);
        }
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
          if (h0 + j * parts >= heads) break;
          rotate(c, s, x[j], y[j]);
          T* o = head_of(qo, ko, a, token, h0 + j * parts);
          o[d0] = static_cast<T>(x[j]);
          o[d1] = static_cast<T>(y[j]);
        }
      }
    }
    if (!a.copy) continue;
    for (int h = part; h < heads; h += parts)
      for (int d = 2 * a.r.half + lane; d < a.d; d += 64)
        head_of(qo, ko, a, token, h)[d] = head_of(q, k, a, token, h)[d];
  }
}

bool aligned16(const void* p) { return reinterpret_cast<uintptr_t>(p) % 16 == 0; }

}  // namespace

hipError_t launch_rotate(const RotateArgs& a, bool bf16, hipStream_t stream) {
  const int heads = a.hq + a.hk;
  if (a.tokens == 0) return hipSuccess;
  const bool aligned = aligned16(a.q) && aligned16(a.k) && aligned16(a.q_out) && aligned16(a.k_out);
  const auto launch = [&](auto elem) {
    using T = decltype(elem);
    // wavefronts that a token's heads are split over, `turns` of each at most, and workgroups
    int64_t parts, g;
    const auto split = [&](int64_t turns) {
      parts = std::max<int64_t>(1, std::min(turns, kRotateWaves / a.tokens));
      g = std::min<int64_t>((a.tokens * parts + 3) / 4, 1 << 22);
    };
    if (aligned && by_chunks<T>(a.d) && !by_items<T>(a.r, a.d)) {
      const int at_once = 64 / (a.d / Chunk<T>::kCount);
      split((heads + at_once - 1) / at_once);
      const dim3 grid(static_cast<unsigned>(g)), block(256);
      if (a.r.interleaved)
        hipLaunchKernelGGL((rotate_chunks_kernel<T, true>), grid, block, 0, stream, a,
                           static_cast<int>(parts));
      else
        hipLaunchKernelGGL((rotate_chunks_kernel<T, false>), grid, block, 0, stream, a,
                           static_cast<int>(parts));
      return hipGetLastError();
    }
    if (!aligned || !by_items<T>(a.r, a.d)) {
      split(heads);
      hipLaunchKernelGGL((rotate_pairs_kernel<T>), dim3(static_cast<unsigned>(g)), dim3(256), 0,
                         stream, a, static_cast<int>(parts));
      return hipGetLastError();
    }
    const auto go = [&](auto inter) {
      using I = Item<T, decltype(inter)::value>;
      const int at_once = 64 / (a.r.half / I::kAngles);
      split((heads + at_once - 1) / at_once);
      hipLaunchKernelGGL((rotate_kernel<T, decltype(inter)::value>), dim3(static_cast<unsigned>(g)),
                         dim3(256), 0, stream, a, static_cast<int>(parts));
      return hipGetLastError();
    };
    return a.r.interleaved ? go(std::true_type{}) : go(std::false_type{});
  };
  return bf16 ? launch(__bf16{}) : launch(float{});
}

}  // namespace sift
