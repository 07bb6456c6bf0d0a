// Accumulated attention weights of a cache's keys:
//
//   out[b, kv, i] = decay * weights[b, kv, i]
//                   + sum over b's new rows and kv's query heads of e^(s - lse)
//
// S = Q K^T with the rows on M and the keys on N, so that a lane holds one key's
// scores for 16 rows of a block of 32 and their sum is in-lane but for one
// exchange.  A wavefront keeps 32 keys in registers, read straight from the
// pages, and walks the row blocks of Q, which the workgroup holds in LDS; the
// next 32 keys are on their way meanwhile.  K is read once (for every chunk_rows
// rows) and a key's sum is made by one lane in row order: no atomics.
//
// The exponent is formed as scale * q.k - lse in the natural domain and only
// then multiplied by log2(e): the two are large and nearly equal for the keys
// that count, and their difference is exact there.

#include <algorithm>

#include "cache.h"
#include "sift_internal.h"

namespace sift {
namespace {

using namespace cache;

constexpr int kWaves = 8;
constexpr int kStepKeys = 32 * kWaves;  // a step: 32 keys of each wavefront

struct KeyCost {
  int32_t hkv;
  static __device__ __forceinline__ int steps(const Seq& s) {
    return (s.len + kStepKeys - 1) / kStepKeys;
  }
  __device__ __forceinline__ int operator()(const Seq& s) const { return hkv * steps(s); }
};

template <typename T, int D>
__global__ __launch_bounds__(64 * kWaves, 2) void cache_weights_kernel(CacheWeightArgs p) {
  using G = Tile<T, D>;
  // chunk_rows rows of Q, swizzled as K tiles are, then {lse, slope, position} of each
  extern __shared__ __attribute__((aligned(1024))) uint8_t smem[];
  const CacheArgs& a = p.c;
  const int g = a.hq / a.hkv;
  const KeyCost cost{a.hkv};
  const Split split(total_work(a, cost), p.groups);
  const int group = group_of(split);
  if (group >= split.groups) return;
  int x = split.at(group);
  const int xend = split.at(group + 1);

  const int lane = threadIdx.x & 63;
  const int wave = uniform(threadIdx.x >> 6);
  const int l32 = lane & 31, hf = lane >> 5;
  const int slots = a.max_pages << a.page_shift;
  const int lds0 = static_cast<int>(reinterpret_cast<size_t>((lds_u8*)smem));
  const int qaddr = lds0 + G::lane_k(l32, hf);
  const int lse0 = lds0 + p.chunk_rows * G::kRow;  // three float arrays of chunk_rows
  const int slope0 = lse0 + 4 * p.chunk_rows, pos0 = slope0 + 4 * p.chunk_rows;
  const bool bias = a.sc.slopes != nullptr;

  Place pl = find_work(a, x, cost);
  while (x < xend && pl.b < a.num_seqs) {
    const int b = pl.b;
    const Seq s = sequence(a, b);
    const int len = uniform(s.len), n = uniform(s.n), row0 = uniform(s.row0);
    const int steps = uniform(cost.steps(s));
    const int kvh = Split::quotient(x - pl.at, steps);
    const int s0 = x - pl.at - kvh * steps;
    const int s1 = min(steps, s0 + (xend - x));
    const int64_t at0 = (static_cast<int64_t>(b) * a.hkv + kvh) * slots;
    const int rows = n * g;

    for (int c0 = 0; c0 == 0 || c0 < rows; c0 += p.chunk_rows) {
      const int cn = min(rows - c0, p.chunk_rows);
      const int blocks = (cn + 31) / 32;
      __syncthreads();  // the last chunk is read
      for (int e = threadIdx.x; e < blocks * 32 * G::kChunks; e += 64 * kWaves) {
        const int i = e / G::kChunks, ch = e % G::kChunks, r = c0 + i;
        u32x4 y = u32x4{0u, 0u, 0u, 0u};
        if (i < cn)
          y = *reinterpret_cast<const u32x4*>(
              static_cast<const uint8_t*>(a.q) +
              (static_cast<int64_t>(row0 + r / g) * a.hq + kvh * g + r % g) * G::kRow + 16 * ch);
        *reinterpret_cast<lds_u32x4*>(
            static_cast<size_t>(lds0 + i * G::kRow + 16 * (ch ^ G::swz_k(i)))) = y;
      }
      for (int i = threadIdx.x; i < blocks * 32; i += 64 * kWaves) {
        const int r = c0 + i, tok = row0 + r / g, h = kvh * g + r % g;
        // a row without weight or keys, or none: +inf, its weights are 0
        float l = INFINITY, slope = 0.f;
        int pos = 0;
        if (i < cn) {
          const float f = p.row_weight != nullptr ? p.row_weight[tok] : 1.f;
          const float y = p.lse[static_cast<int64_t>(tok) * a.hq + h];
          if (f != 0.f && y != -INFINITY) l = f == 1.f ? y : y - logf(f);
          if (bias) {
            slope = a.sc.slopes[h];
            pos = a.row_pos != nullptr ? a.row_pos[tok] : len + r / g;
          }
        }
        *reinterpret_cast<lds_float*>(static_cast<size_t>(lse0 + 4 * i)) = l;
        *reinterpret_cast<lds_float*>(static_cast<size_t>(slope0 + 4 * i)) = slope;
        *reinterpret_cast<lds_int*>(static_cast<size_t>(pos0 + 4 * i)) = pos;
      }
      __syncthreads();

      // this lane's key of tile t: row l32
      const auto key_at = [&](int t, bool& valid) {
        const int slot = t * 32 + 16 * (l32 >> 4);
        const Rows16 lo = cached_rows(a, b, len, t * 32), hi = cached_rows(a, b, len, t * 32 + 16);
        const Rows16 r = l32 < 16 ? lo : hi;
        valid = slot < slots && (l32 & 15) < r.n;
        return static_cast<const uint8_t*>(a.k) + ((r.row + (l32 & 15)) * a.hkv + kvh) * G::kRow +
               16 * hf;
      };
      u32x4 kf[G::kSteps], kn[G::kSteps];
      bool valid = false, valid_next = false;
      const auto load = [&](int t, u32x4(&dst)[G::kSteps], bool& ok) {
        const uint8_t* src = key_at(t, ok);
#pragma unroll
        for (int i = 0; i < G::kSteps; ++i) {
          dst[i] = u32x4{0u, 0u, 0u, 0u};
          if (ok) dst[i] = *reinterpret_cast<const u32x4*>(src + 32 * i);
        }
      };
      const int tend = min((len + 31) / 32, s1 * kWaves);
      int t = s0 * kWaves + wave;
      if (t < tend) load(t, kf, valid);
      for (; t < tend; t += kWaves) {
        if (t + kWaves < tend) load(t + kWaves, kn, valid_next);
        const int slot = t * 32 + l32;
        float old = 0.f;
        if (slot < len && hf == 0) {
          if (c0 > 0)
            old = p.out[at0 + slot];
          else if (p.weights != nullptr && p.decay != 0.f)
            old = p.decay * p.weights[at0 + slot];
        }
        int kpos = slot;
        if (bias && a.key_pos != nullptr) kpos = a.key_pos[at0 + min(slot, slots - 1)];
        float sum = 0.f;
        for (int rb = 0; rb < blocks; ++rb) {
          f32x16 sc = f32x16{};
#pragma unroll
          for (int i = 0; i < G::kSteps; ++i)
            sc = dot_step<T>(G::k_frag(qaddr + rb * 32 * G::kRow, 0, i), kf[i], sc);
          const int left = cn - 32 * rb;
          if (a.sc.x != 0.f) cap_scores(a.sc, sc);
          const float c = a.sc.x != 0.f ? 1.f : a.sc.c;
          float part = 0.f;
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            if (8 * j >= left) break;  // the block's rows end before
            const int off = 4 * (32 * rb + 8 * j + 4 * hf);
            const f32x4 l = *reinterpret_cast<const lds_f32x4*>(static_cast<size_t>(lse0 + off));
            f32x4 sl = f32x4{0.f, 0.f, 0.f, 0.f};
            i32x4 ps = i32x4{0, 0, 0, 0};
            if (bias) {
              sl = *reinterpret_cast<const lds_f32x4*>(static_cast<size_t>(slope0 + off));
              ps = *reinterpret_cast<const lds_i32x4*>(static_cast<size_t>(pos0 + off));
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              float y = fmaf(sc[4 * j + e], c, -l[e]);
              if (bias) y = fmaf(-sl[e], fabsf(static_cast<float>(ps[e] - kpos)), y);
              const float w = __builtin_amdgcn_exp2f(y * kLog2e);
              part += l[e] < INFINITY ? w : 0.f;
            }
          }
          sum += part;
        }
        sum = half_sum(sum);
        if (slot < len && hf == 0) p.out[at0 + slot] = valid ? old + sum : 0.f;
#pragma unroll
        for (int i = 0; i < G::kSteps; ++i) kf[i] = kn[i];
        valid = valid_next;
      }
    }
    x += s1 - s0;
    if (x < xend && x - pl.at >= cost(s)) pl = find_work(a, x, cost);
  }
}

}  // namespace

int64_t cache_weights_steps(const CacheArgs& a) {
  return static_cast<int64_t>(a.num_seqs) * a.hkv *
         (((static_cast<int64_t>(a.max_pages) << a.page_shift) + kStepKeys - 1) / kStepKeys);
}

hipError_t launch_cache_weights(CacheWeightArgs a, bool bf16, int head_dim, int cus,
                                hipStream_t stream) {
  const int64_t most = static_cast<int64_t>(std::min(a.c.rows, a.c.max_rows)) * (a.c.hq / a.c.hkv);
  const auto launch = [&](auto elem, auto dim) {
    using T = decltype(elem);
    constexpr int D = decltype(dim)::value;
    constexpr int kRowLds = Tile<T, D>::kRow + 12;
    constexpr int kFit = 144 * 1024 / kRowLds / 32 * 32;  // rows that 144 KB hold
    const int64_t need = std::max<int64_t>(32, (most + 31) / 32 * 32);
    a.chunk_rows = static_cast<int32_t>(std::min<int64_t>(need, kFit));
    const int lds = a.chunk_rows * kRowLds;
    a.groups = cus * (lds <= 72 * 1024 ? 2 : 1);
    hipLaunchKernelGGL((cache_weights_kernel<T, D>), dim3(a.groups), dim3(64 * kWaves), lds,
                       stream, a);
    return hipGetLastError();
  };
  using D64 = std::integral_constant<int, 64>;
  using D128 = std::integral_constant<int, 128>;
  if (bf16) return head_dim == 128 ? launch(__bf16{}, D128{}) : launch(__bf16{}, D64{});
  return head_dim == 128 ? launch(float{}, D128{}) : launch(float{}, D64{});
}

}  // namespace sift
