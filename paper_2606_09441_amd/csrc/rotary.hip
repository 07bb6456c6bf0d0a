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

// Any sizes and alignment, a pair at a time.
template <typename T>
__global__ __launch_bounds__(256) void rotate_pairs_kernel(RotateArgs a) {
  const int heads = a.hq + a.hk;
  const int half = a.r.half, each = half + (a.copy ? a.d - 2 * half : 0);
  const int64_t n = a.tokens * heads * each;
  for (int64_t e = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x; e < n;
       e += static_cast<int64_t>(gridDim.x) * 256) {
    const int64_t th = e / each;
    const int i = static_cast<int>(e - th * each);
    const int64_t token = th / heads;
    const int h = static_cast<int>(th - token * heads);
    const T* p = head_of(static_cast<const T*>(a.q), static_cast<const T*>(a.k), a, token, h);
    T* o = head_of(static_cast<T*>(a.q_out), static_cast<T*>(a.k_out), a, token, h);
    if (i >= half) {
      o[half + i] = p[half + i];
      continue;
    }
    float c, s;
    turn<T>(a.r, a.positions[token], i, c, s);
    const int d0 = a.r.interleaved ? 2 * i : i, d1 = a.r.interleaved ? 2 * i + 1 : half + i;
    float x = value(p[d0]), y = value(p[d1]);
    rotate(c, s, x, y);
    o[d0] = static_cast<T>(x);
    o[d1] = static_cast<T>(y);
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
    if (!aligned || !by_items<T>(a.r, a.d)) {
      const int64_t n = a.tokens * heads * (a.d - a.r.half);
      const int64_t g = std::min<int64_t>((n + 255) / 256, 65536);
      hipLaunchKernelGGL((rotate_pairs_kernel<T>), dim3(static_cast<unsigned>(g)), dim3(256), 0,
                         stream, a);
      return hipGetLastError();
    }
    const auto go = [&](auto inter) {
      using I = Item<T, decltype(inter)::value>;
      const int at_once = 64 / (a.r.half / I::kAngles);
      const int64_t turns = (heads + at_once - 1) / at_once;
      const int64_t parts =
          std::max<int64_t>(1, std::min(turns, kRotateWaves / std::max<int64_t>(1, a.tokens)));
      const int64_t g = std::min<int64_t>((a.tokens * parts + 3) / 4, 1 << 22);
      hipLaunchKernelGGL((rotate_kernel<T, decltype(inter)::value>), dim3(static_cast<unsigned>(g)),
                         dim3(256), 0, stream, a, static_cast<int>(parts));
      return hipGetLastError();
    };
    return a.r.interleaved ? go(std::true_type{}) : go(std::false_type{});
  };
  return bf16 ? launch(__bf16{}) : launch(float{});
}

}  // namespace sift
