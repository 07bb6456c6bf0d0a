// Accumulated attention weights of a cache's keys:
//
//   out[b, kv, i] = decay * weights[b, kv, i]
//                   + sum over b's new rows and kv's query heads of e^(s - lse)
//
// S = Q K^T with the rows on M and the keys on N, so that a lane holds one key's
// scores for 16 rows of a block of 32 and their sum is in-lane but for one
// exchange.  A wavefront keeps 32 keys in registers and walks the row blocks of Q,
// which the workgroup holds in LDS; while the VALU makes the weights of a block
// the matrix cores form the scores of the next.  K is read once (for every
// chunk_rows rows) and a key's sum is made by one lane in row order: no atomics.
//  * Few rows (one block or two): HBM bounds it.  K comes by DMA through LDS of
//    the wavefront's own, whole lines at a time, the next tile as soon as the
//    present one is in registers.
//  * Many rows: their Q takes that LDS, and K goes straight to registers.  A score
//    costs the VALU an FMA, a product, an exponential and a sum; 384 rows of 66048
//    keys of 8 kv heads, D = 128 take 88 us, the VALU busy in 52% of the SIMDs' cycles
//    and the MFMAs in 30%.
// The instances of bf16 D = 128 and fp32 D = 64 through LDS, and of fp32 D = 128 from
// registers, spill 40 to 44 bytes of registers a lane.
//
// The exponent is formed as scale * q.k - lse in the natural domain and only then
// multiplied by log2(e): the two are large and nearly equal for the keys that count,
// and their difference is exact there, also for bf16, whose products are exact in
// fp32.  In the log2 domain, an instruction a score less (384 rows of 66048 keys, 8 kv
// heads, D = 128: 84 us instead of 88), rounding lse and the scale put up to 5e-6 on
// the weights of scores near 120, ten times what remains.

#include <algorithm>

#include "cache.h"
#include "sift_internal.h"

namespace sift {
namespace {

using namespace cache;

constexpr int kWaves = 8;
constexpr int kStepTiles = 8;           // tiles of 32 keys of a step
constexpr int kStepKeys = 32 * kStepTiles;
constexpr int kMostBlocks = 32;         // of 32 rows in LDS
// Rows up to which K comes through LDS.  us by registers / through LDS, bf16 D = 128,
// 8 kv heads: 66048 keys, 32 rows 36 / 28, 128 50 / 43, 192 53 / 54, 256 63 / 66; 16
// sequences of 8192 keys 57 / 51, 81 / 75, 92 / 95, 111 / 116.  (One limit for all: at
// D = 64, and for fp32 at D = 64, LDS is still the faster at 320 rows, 61 / 51 and 225 /
// 220; fp32 at D = 128 has no room for it beyond 32.)
constexpr int kFewRows = 192;

struct KeyCost {
  int32_t hkv;
  static __device__ __forceinline__ int steps(const Seq& s) {
    return (s.len + kStepKeys - 1) / kStepKeys;
  }
  __device__ __forceinline__ int operator()(const Seq& s) const { return hkv * steps(s); }
};

template <typename T, int D, bool kDma>
__global__ __launch_bounds__(64 * kWaves, kDma && sizeof(T) * D <= 256 ? 4 : 2) void
cache_weights_kernel(CacheWeightArgs p) {
  using G = Tile<T, D>;
  // LDS of a wavefront's keys: a tile of them, or as many rows as fit in 4 KB
  constexpr int kTurn = kDma ? 32 : 4096 / G::kRow < 32 ? 4096 / G::kRow : 32;
  constexpr int kKeys = kTurn * G::kRow;
  // chunk_rows rows of Q, swizzled as K tiles are, then {lse, slope, position} of
  // each, then the keys of each wavefront
  extern __shared__ __attribute__((aligned(1024))) uint8_t smem[];
  __shared__ int dead[kMostBlocks];  // whether a block has rows that count for nothing
  const CacheArgs& a = p.c;
  const int g = a.hq / a.hkv;
  const KeyCost cost{a.hkv};
  int group, x, xend;
  Place pl;
  Seq s;
  {
    const Work work(a, cost);
    const Split split(work.total, p.groups);
    group = group_of(split);
    if (group >= split.groups) return;
    x = split.at(group);
    xend = split.at(group + 1);
    pl = work.find(x);
    s = work.seq(pl.b);
  }

  const int lane = threadIdx.x & 63;
  const int wave = uniform(threadIdx.x >> 6);
  const int l32 = lane & 31, hf = lane >> 5;
  const int slots = a.max_pages << a.page_shift;
  const int stride = a.hkv * G::kRow;
  const int lds0 = static_cast<int>(reinterpret_cast<size_t>((lds_u8*)smem));
  const int qaddr = lds0 + G::lane_k(l32, hf);
  const int lse0 = lds0 + p.chunk_rows * G::kRow;  // three arrays of chunk_rows
  const int slope0 = lse0 + 4 * p.chunk_rows, pos0 = slope0 + 4 * p.chunk_rows;
  const int kt = lds0 + (p.chunk_rows * (G::kRow + 12) + 1023) / 1024 * 1024 + wave * kKeys;
  const int kaddr = kt + G::lane_k(l32 % kTurn, hf);
  const int koff = G::template dma_lane<false>(lane, stride);
  const bool bias = a.sc.slopes != nullptr;
  const float c = a.sc.x != 0.f ? 1.f : a.sc.c;

  while (x < xend && pl.b < a.num_seqs) {
    const int b = pl.b;
    const int len = s.len, n = s.n, row0 = s.row0;
    const int steps = uniform(cost.steps(s));
    const int kvh = Split::quotient(x - pl.at, steps);
    const int s0 = x - pl.at - kvh * steps;
    const int s1 = min(steps, s0 + (xend - x));
    const int64_t at0 = (static_cast<int64_t>(b) * a.hkv + kvh) * slots;
    const int rows = n * g;

    for (int c0 = 0; c0 == 0 || c0 < rows; c0 += p.chunk_rows) {
      const int cn = min(rows - c0, p.chunk_rows);
      const int blocks = (cn + 31) / 32;

      // A tile's keys: to LDS (kDma) or to registers, with what else a lane needs of
      // its key (lane l32).
      struct Key {
        float old;
        int pos;
        bool valid;
      };
      const auto fetch = [&](int t, u32x4(&dst)[G::kSteps], Key& k) {
        const Rows16 r0 = cached_rows(a, b, len, t * 32), r1 = cached_rows(a, b, len, t * 32 + 16);
        const int slot = t * 32 + l32;
        const Rows16 r = l32 < 16 ? r0 : r1;
        k.valid = (l32 & 15) < r.n;
        if constexpr (kDma) {
          dma_rows<T, D, false>(kt, rows_rsrc(reinterpret_cast<unsigned long long>(a.k) +
                                                  (r0.row * a.hkv + kvh) * G::kRow,
                                              r0.n, stride, G::kRow), koff, stride);
          dma_rows<T, D, false>(kt + 16 * G::kRow,
                                rows_rsrc(reinterpret_cast<unsigned long long>(a.k) +
                                              (r1.row * a.hkv + kvh) * G::kRow,
                                          r1.n, stride, G::kRow), koff, stride);
        } else {
          // whole rows, kDmaRows of them an instruction
          const int row = lane / G::kChunks;
          const uint8_t* src = static_cast<const uint8_t*>(a.k) +
                               ((static_cast<int64_t>(row) * a.hkv) + kvh) * G::kRow +
                               16 * (lane % G::kChunks);
#pragma unroll
          for (int i = 0; i < G::kSteps; ++i) {
            const int at = i * G::kDmaRows % 16;
            const Rows16& x = i * G::kDmaRows < 16 ? r0 : r1;
            dst[i] = u32x4{0u, 0u, 0u, 0u};
            if (at + row < x.n)
              dst[i] = *reinterpret_cast<const u32x4*>(src + (x.row + at) * a.hkv * G::kRow);
          }
        }
        k.old = 0.f;
        if (slot < len && hf == 0) {
          if (c0 > 0)
            k.old = p.out[at0 + slot];
          else if (p.weights != nullptr && p.decay != 0.f)
            k.old = p.decay * p.weights[at0 + slot];
        }
        k.pos = bias && a.key_pos != nullptr ? a.key_pos[at0 + min(slot, slots - 1)] : slot;
      };

      u32x4 kf[G::kSteps], kn[G::kSteps];
      Key key{0.f, 0, false}, next{0.f, 0, false};
      const int tend = min((len + 31) / 32, s1 * kStepTiles);
      int t = s0 * kStepTiles + wave;
      if (t < tend) fetch(t, kn, next);

      __syncthreads();  // the last chunk is read
      if (threadIdx.x < kMostBlocks) dead[threadIdx.x] = 0;
      __syncthreads();
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
        if (l == INFINITY) dead[i / 32] = 1;
        *reinterpret_cast<lds_float*>(static_cast<size_t>(lse0 + 4 * i)) = l;
        *reinterpret_cast<lds_float*>(static_cast<size_t>(slope0 + 4 * i)) = slope;
        *reinterpret_cast<lds_int*>(static_cast<size_t>(pos0 + 4 * i)) = pos;
      }
      __syncthreads();
      for (int e = threadIdx.x; e < blocks * 32 * G::kChunks; e += 64 * kWaves) {
        const int i = e / G::kChunks, ch = e % G::kChunks, r = c0 + i;
        u32x4 y = u32x4{0u, 0u, 0u, 0u};
        if (*reinterpret_cast<const lds_float*>(static_cast<size_t>(lse0 + 4 * i)) != INFINITY)
          y = *reinterpret_cast<const u32x4*>(
              static_cast<const uint8_t*>(a.q) +
              (static_cast<int64_t>(row0 + r / g) * a.hq + kvh * g + r % g) * G::kRow + 16 * ch);
        *reinterpret_cast<lds_u32x4*>(
            static_cast<size_t>(lds0 + i * G::kRow + 16 * (ch ^ G::swz_k(i)))) = y;
      }
      __syncthreads();
      const uint32_t dead_blocks =
          static_cast<uint32_t>(__ballot(lane < kMostBlocks && dead[lane % kMostBlocks] != 0));

      for (; t < tend; t += kWaves) {
        key = next;
        if constexpr (kDma) {
          wait_vm<0>();
#pragma unroll
          for (int i = 0; i < G::kSteps; ++i) kf[i] = G::k_frag(kaddr, 0, i);
          wait_lds();  // the tile is in registers
        } else {
          // from rows to fragments, kTurn rows at a time (LDS keeps a wavefront's order)
#pragma unroll
          for (int z = 0; z < 32 / kTurn; ++z) {
            constexpr int kOnce = kTurn / G::kDmaRows;
#pragma unroll
            for (int i = 0; i < kOnce; ++i) {
              const int r = i * G::kDmaRows + lane / G::kChunks;
              *reinterpret_cast<lds_u32x4*>(static_cast<size_t>(
                  kt + r * G::kRow + 16 * (lane % G::kChunks ^ G::swz_k(r)))) = kn[z * kOnce + i];
            }
            if (l32 / kTurn == z) {
#pragma unroll
              for (int i = 0; i < G::kSteps; ++i) kf[i] = G::k_frag(kaddr, 0, i);
            }
          }
        }
        if (t + kWaves < tend) fetch(t + kWaves, kn, next);

        // Scores of row block rb, transformed; lane's key, registers' rows.
        const auto transform = [&](int rb, f32x16& sc) {
          if (a.sc.x != 0.f) cap_scores(a.sc, sc, 4 * min(4, (cn - 32 * rb + 7) / 8));
          if (bias) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              const int off = 4 * (32 * rb + 8 * j + 4 * hf);
              const f32x4 sl =
                  *reinterpret_cast<const lds_f32x4*>(static_cast<size_t>(slope0 + off));
              const i32x4 ps = *reinterpret_cast<const lds_i32x4*>(static_cast<size_t>(pos0 + off));
#pragma unroll
              for (int e = 0; e < 4; ++e)
                sc[4 * j + e] = fmaf(sc[4 * j + e], c,
                                     -sl[e] * fabsf(static_cast<float>(ps[e] - key.pos)));
            }
          }
        };
        const float cc = bias ? 1.f : c;
        const auto row_lse = [&](int rb, f32x4(&l)[4]) {
#pragma unroll
          for (int j = 0; j < 4; ++j)
            l[j] = *reinterpret_cast<const lds_f32x4*>(
                static_cast<size_t>(lse0 + 4 * (32 * rb + 8 * j + 4 * hf)));
        };
        const auto weight = [&](const f32x16& sc, const f32x4(&l)[4], int v) {
          return __builtin_amdgcn_exp2f(fmaf(sc[v], cc, -l[v >> 2][v & 3]) * kLog2e);
        };
        // The sum of a block's weights, rows that count for nothing left out,
        // whatever the key holds (a log sum that is no number is none of these).
        const auto careful = [&](int rb, const f32x16& sc, const f32x4(&l)[4]) {
          float part[2] = {0.f, 0.f};
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            if (32 * rb + 8 * j >= cn) break;  // the block's rows end before
#pragma unroll
            for (int v = 4 * j; v < 4 * j + 4; ++v) {
              const float w = weight(sc, l, v);
              part[v & 1] += l[j][v & 3] == INFINITY ? 0.f : w;
            }
          }
          return part[0] + part[1];
        };
        const auto scores = [&](int rb) {
          f32x16 sc = f32x16{};
#pragma unroll
          for (int i = 0; i < G::kSteps; ++i)
            sc = dot_step<T>(G::k_frag(qaddr + rb * 32 * G::kRow, 0, i), kf[i], sc);
          return sc;
        };
        float sum = 0.f;
        if constexpr (kDma || !G::kBf16) {
          for (int rb = 0; rb < blocks; ++rb) {
            f32x4 l[4];
            row_lse(rb, l);
            f32x16 sc = scores(rb);
            transform(rb, sc);
            sum += careful(rb, sc, l);
          }
        } else {
          // block rb's weights beside block rb + 1's scores; the fragments three
          // steps ahead and the log sums a block ahead, across the blocks (past the
          // last one the first again, for nothing)
          const auto block_at = [&](int rb) {
            return qaddr + (rb < blocks ? rb : 0) * 32 * G::kRow;
          };
          constexpr int kAhead = 3, kEach = 16 / G::kSteps > 0 ? 16 / G::kSteps : 1;
          u32x4 f[kAhead];
          const auto body = [&](int rb, f32x16& cur, f32x4(&l)[4], f32x16& nxt, f32x4(&ln)[4]) {
            row_lse(rb + 1 < blocks ? rb + 1 : 0, ln);
            if ((dead_blocks >> rb) & 1) {
              sum += careful(rb, cur, l);
              nxt = scores(rb + 1 < blocks ? rb + 1 : 0);
#pragma unroll
              for (int i = 0; i < kAhead; ++i) f[i] = G::k_frag(block_at(rb + 2), 0, i);
            } else {
              float part[2] = {0.f, 0.f};
              const int q1 = block_at(rb + 1), q2 = block_at(rb + 2);
              u32x4 h[kAhead] = {f[0], f[1], f[2]};
              nxt = f32x16{};
#pragma unroll
              for (int i = 0; i < G::kSteps; ++i) {
                nxt = dot_step<T>(h[i % kAhead], kf[i], nxt);
                const int j = i + kAhead;
                h[i % kAhead] = j < G::kSteps ? G::k_frag(q1, 0, j) : G::k_frag(q2, 0, j - G::kSteps);
#pragma unroll
                for (int u = 0; u < kEach; ++u) part[u & 1] += weight(cur, l, i * kEach + u);
                __builtin_amdgcn_sched_barrier(0);
              }
#pragma unroll
              for (int i = 0; i < kAhead; ++i) f[i] = h[(G::kSteps + i) % kAhead];
              sum += part[0] + part[1];
            }
            transform(rb + 1 < blocks ? rb + 1 : 0, nxt);
          };
          if (blocks > 0) {
            f32x16 s0_ = scores(0), s1_;
            f32x4 l0[4], l1[4];
            row_lse(0, l0);
            transform(0, s0_);
#pragma unroll
            for (int i = 0; i < kAhead; ++i) f[i] = G::k_frag(block_at(1), 0, i);
            for (int rb = 0; rb < blocks; rb += 2) {
              body(rb, s0_, l0, s1_, l1);
              if (rb + 1 < blocks) body(rb + 1, s1_, l1, s0_, l0);
            }
          }
        }
        sum = half_sum(sum);
        const int slot = t * 32 + l32;
        if (slot < len && hf == 0) p.out[at0 + slot] = key.valid ? key.old + sum : 0.f;
      }
    }
    x += s1 - s0;
    if (x < xend && x - pl.at >= cost(s)) {
      const Work work(a, cost);
      pl = work.find(x);
      s = work.seq(pl.b);
    }
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
    constexpr int kTileLds = kWaves * 32 * Tile<T, D>::kRow + 1024;
    constexpr int kTurnLds = kWaves * 4096 + 1024;
    constexpr int kFit = std::min((158 * 1024 - kTurnLds) / kRowLds, 32 * kMostBlocks) / 32 * 32;
    const int64_t need = std::max<int64_t>(32, (most + 31) / 32 * 32);
    a.chunk_rows = static_cast<int32_t>(std::min<int64_t>(need, kFit));
    int lds = a.chunk_rows * kRowLds;
    const bool dma = need <= kFewRows && lds + kTileLds <= 158 * 1024;
    lds += dma ? kTileLds : kTurnLds;
    a.groups = cus * (lds <= 79 * 1024 ? 2 : 1);
    if (dma)
      hipLaunchKernelGGL((cache_weights_kernel<T, D, true>), dim3(a.groups), dim3(64 * kWaves), lds,
                         stream, a);
    else
      hipLaunchKernelGGL((cache_weights_kernel<T, D, false>), dim3(a.groups), dim3(64 * kWaves),
                         lds, stream, a);
    return hipGetLastError();
  };
  using D64 = std::integral_constant<int, 64>;
  using D128 = std::integral_constant<int, 128>;
  if (bf16) return head_dim == 128 ? launch(__bf16{}, D128{}) : launch(__bf16{}, D64{});
  return head_dim == 128 ? launch(float{}, D128{}) : launch(float{}, D64{});
}

}  // namespace sift
