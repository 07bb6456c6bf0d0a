// Device pieces of the rotary positions (rotary.hip, cache_append.hip).
//
// A pair (x, y) of a head's dims turns by the angle a = position * inv_freq[i]:
//   x' = m (x cos a - y sin a),  y' = m (y cos a + x sin a)
// i < half; the pair's dims are i and half + i, or 2 i and 2 i + 1 (interleaved).
// The product of the position and the frequency is formed and taken modulo a turn in
// 64 bits: in 32, an angle of a million radians would be off by a thirtieth of one.
// There are few angles to do: one for the pairs i of all heads of a token.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "sift_internal.h"

namespace sift {
namespace rotary {

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

// Cosine and sine of 2 pi turns.
template <bool kFull>
__device__ __forceinline__ void unit(double turns, float& c, float& s) {
  if constexpr (!kFull) {
    // the hardware's, of a fraction of a turn: off by some 1e-6, where the result is
    // rounded to 8 bits of significand
    const float r = static_cast<float>(__builtin_amdgcn_fract(turns));
    c = __builtin_amdgcn_cosf(r);
    s = __builtin_amdgcn_sinf(r);
  } else {
    // the nearest quarter turn, and Taylor's polynomials of the rest, |y| <= pi / 4:
    // the first terms left out are below y^11 / 11! = 1.8e-9 and y^12 / 12! = 1.2e-10
    const double r = turns - rint(turns);
    const double quarter = rint(4.0 * r);
    const float y = static_cast<float>((r - 0.25 * quarter) * 6.283185307179586);
    const float w = y * y;
    const float sy =
        fmaf(y * w, fmaf(w, fmaf(w, fmaf(w, 1.f / 362880, -1.f / 5040), 1.f / 120), -1.f / 6), y);
    const float cy = fmaf(
        w,
        fmaf(w, fmaf(w, fmaf(w, fmaf(w, -1.f / 3628800, 1.f / 40320), -1.f / 720), 1.f / 24), -0.5f),
        1.f);
    const int q = static_cast<int>(quarter);  // -2 .. 2
    const float a = (q & 1) ? sy : cy, b = (q & 1) ? cy : sy;
    c = (q == 0 || q == -1) ? a : -a;
    s = (q == 0 || q == 1) ? b : -b;
  }
}

// Turns a position that frequency i makes: the constant and the product are each off by
// 2^-53 of themselves at most, as is a position's product.
__device__ __forceinline__ double frequency(const RotaryArgs& r, int i) {
  return static_cast<double>(r.inv_freq[i]) * 0.15915494309189535;  // 1 / (2 pi)
}
// Cosine and sine of a position's angle, times the magnitude; back: of the negative angle.
template <typename T>
__device__ __forceinline__ void turn(const RotaryArgs& r, int position, double frequency, float& c,
                                     float& s) {
  unit<std::is_same<T, float>::value>(static_cast<double>(position) * frequency, c, s);
  c *= r.magnitude;
  s *= r.back ? -r.magnitude : r.magnitude;
}
template <typename T>
__device__ __forceinline__ void turn(const RotaryArgs& r, int position, int i, float& c, float& s) {
  turn<T>(r, position, frequency(r, i), c, s);
}

// 16 bytes as numbers and back, rounded to the nearest.
template <typename T>
struct Chunk {
  static constexpr int kCount = 16 / static_cast<int>(sizeof(T));
  float x[kCount];
  __device__ __forceinline__ void set(u32x4 v) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t w = v[i];
      if constexpr (std::is_same<T, float>::value) {
        x[i] = __builtin_bit_cast(float, w);
      } else {
        x[2 * i] = __builtin_bit_cast(float, w << 16);
        x[2 * i + 1] = __builtin_bit_cast(float, w & 0xffff0000u);
      }
    }
  }
  __device__ __forceinline__ u32x4 get() const {
    u32x4 v;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (std::is_same<T, float>::value)
        v[i] = __builtin_bit_cast(uint32_t, x[i]);
      else
        v[i] = __builtin_bit_cast(
            uint32_t, bf16x2{static_cast<__bf16>(x[2 * i]), static_cast<__bf16>(x[2 * i + 1])});
    }
    return v;
  }
};

__device__ __forceinline__ void rotate(float c, float s, float& x, float& y) {
  const float z = fmaf(x, c, -(y * s));
  y = fmaf(y, c, x * s);
  x = z;
}

// The dims of one item of a head: with halves two chunks, half / kCount apart,
// interleaved one chunk of whole pairs.  `angles` of them, from dim `first` on.
template <typename T, bool kInterleaved>
struct Item {
  static constexpr int kCount = Chunk<T>::kCount;
  static constexpr int kAngles = kInterleaved ? kCount / 2 : kCount;
  static constexpr int kChunks = kInterleaved ? 1 : 2;
  float c[kAngles], s[kAngles];
  __device__ __forceinline__ void angles(const RotaryArgs& r, int position, int item) {
#pragma unroll
    for (int i = 0; i < kAngles; ++i) turn<T>(r, position, item * kAngles + i, c[i], s[i]);
  }
  __device__ __forceinline__ void apply(Chunk<T> (&x)[kChunks]) const {
#pragma unroll
    for (int i = 0; i < kAngles; ++i) {
      if constexpr (kInterleaved)
        rotate(c[i], s[i], x[0].x[2 * i], x[0].x[2 * i + 1]);
      else
        rotate(c[i], s[i], x[0].x[i], x[1].x[i]);
    }
  }
};

// A lane's chunk of a head whose pairs lie anywhere: of each of its dims the cosine, the
// sine with the sign that the other one of its pair takes, and where that one is.
template <typename T, bool kInterleaved>
struct AnyChunk {
  static constexpr int kCount = Chunk<T>::kCount;
  float c[kCount], s[kCount];
  int first;  // dim
  __device__ __forceinline__ void angles(const RotaryArgs& r, int position, int chunk) {
    first = chunk * kCount;
#pragma unroll
    for (int e = 0; e < kCount; ++e) {
      const int d = first + e;
      c[e] = 1.f;
      s[e] = 0.f;
      if (d >= 2 * r.half) continue;  // stays
      if (kInterleaved && (e & 1)) {
        c[e] = c[e - 1];
        s[e] = -s[e - 1];
        continue;
      }
      const bool low = kInterleaved || d < r.half;
      turn<T>(r, position, kInterleaved ? d / 2 : low ? d : d - r.half, c[e], s[e]);
      if (low) s[e] = -s[e];
    }
  }
  // x: the chunk; head: where the head's chunks lie in LDS, as the lanes of this wavefront
  // left them.
  __device__ __forceinline__ void apply(const RotaryArgs& r, Chunk<T>& x, const T* head) const {
    Chunk<T> y;
#pragma unroll
    for (int e = 0; e < kCount; ++e) {
      const int d = first + e;
      float other;
      if constexpr (kInterleaved)
        other = x.x[e ^ 1];
      else
        other = static_cast<float>(head[d < r.half ? d + r.half : d - r.half]);
      y.x[e] = d < 2 * r.half ? fmaf(x.x[e], c[e], other * s[e]) : x.x[e];
    }
    x = y;
  }
};

// Between a wavefront's writes to LDS of its own and its lanes' reads of them, and back: the
// hardware keeps their order, so must the compiler.
__device__ __forceinline__ void lds_order() { asm volatile("" ::: "memory"); }

// Whether rows of D dims go by chunks, pairs wherever they are: whole chunks, a head's in a
// wavefront.
template <typename T>
__host__ __device__ inline bool by_chunks(int d) {
  return d % Chunk<T>::kCount == 0 && d / Chunk<T>::kCount <= 64;
}

// Whether rows of D dims go by items: 16-byte chunks of them hold whole pairs, or whole
// stretches of a half, and a wavefront holds a head's.
template <typename T>
__host__ __device__ inline bool by_items(const RotaryArgs& r, int d) {
  constexpr int n = Chunk<T>::kCount;
  const int part = r.interleaved ? 2 * r.half : r.half;
  return d % n == 0 && part % n == 0 && part / n <= 64;
}

}  // namespace rotary
}  // namespace sift
