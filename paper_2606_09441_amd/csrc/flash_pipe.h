// The software pipeline of the bf16 attention over 64-key tiles: 128 query rows
// of a workgroup, 32 of each of its four wavefronts.  In a step the scores of the
// next tile, S' = K' Q^T, are formed on the matrix cores while the VALU makes the
// weights P of the present one, then O += V^T P^T while it takes the maxima of
// S'.  K runs a tile ahead of V, each has two LDS slots that the DMA fills a step
// before they are read; one barrier a step.  The order inside both halves is laid
// down by hand: left to itself the compiler moves the fragments' reads together
// and runs out of registers.
//
// With a cap the tanh is a polynomial of the product where none of the
// wavefront's tile is large, folded into the exponent's FMA; the exact form
// apart where one is.  The cap keeps the order, so the maxima are the products'.
#pragma once

#include "flash.h"

namespace sift {
namespace flash {

constexpr int kKeys = 64;  // of a tile

// A tile's exponents are z p(z^2) + slope_key (key - d), less the reference, with
// the tanh's p, or (1, 0, ..) where the scores are capped already; without kCap
// p0 alone, the scale.  The key's terms only with kLinear.
struct Form {
  float p0, p1, p2, p3;
  float slope_key, d;
};

template <bool kCap>
__device__ __forceinline__ float capped(const Form& f, float z) {
  if constexpr (!kCap) return z * f.p0;
  const float y = z * z;
  return z * fmaf(y, fmaf(y, fmaf(y, f.p3, f.p2), f.p1), f.p0);
}

// The form of a tile whose products, s0 and s1, have the largest mx and the
// smallest mn.  Large products are capped in place.  Then, where `odd`, whatever
// else sets the tile apart: keys whose bit is not set (bits(): one a key), and the
// bias, slope * dist(key), where kBias.  Returns the bound of the row's scores,
// its largest.
template <bool kCap, bool kBias, typename Bits, typename Dist>
__device__ __forceinline__ float take_tile(const ScoreArgs& sc, f32x16& s0, f32x16& s1, float mx,
                                           float mn, bool odd, Bits bits, int hf, float slope,
                                           Dist dist, Form& f) {
  // Masked scores: -inf, or where z p(z^2) has to stay a number one that no score
  // comes near (|capped score| <= kMaxCap log2(e)).
  constexpr float kOut = kCap ? -1e18f : -INFINITY;
  f = Form{kCap ? sc.b[0] : sc.c, sc.b[1], sc.b[2], sc.b[3], 0.f, 0.f};
  if constexpr (kCap) {
    if (__builtin_amdgcn_ballot_w64(fmaxf(mx, -mn) * sc.x > kTanhSmallBf16)) {
#pragma unroll
      for (int v = 0; v < 16; ++v) {
        s0[v] = cap_any(sc, s0[v]);
        s1[v] = cap_any(sc, s1[v]);
      }
      mx = cap_any(sc, mx);
      f.p0 = 1.f;
      f.p1 = f.p2 = f.p3 = 0.f;
    }
  }
  if (odd) {
    const uint64_t m = bits();
    const uint32_t m0 = static_cast<uint32_t>(m >> (4 * hf));
    const uint32_t m1 = static_cast<uint32_t>(m >> (32 + 4 * hf));
    mx = -INFINITY;
#pragma unroll
    for (int v = 0; v < 16; ++v) {
      float x0 = s0[v], x1 = s1[v];
      if constexpr (kCap || kBias) {
        x0 = capped<kCap>(f, x0);
        x1 = capped<kCap>(f, x1);
      }
      if constexpr (kBias) {
        x0 = fmaf(-slope, dist(key_of(v)), x0);
        x1 = fmaf(-slope, dist(key_of(v) + 32), x1);
      }
      const bool in0 = (m0 >> key_of(v)) & 1u, in1 = (m1 >> key_of(v)) & 1u;
      mx = fmaxf(mx, fmaxf(in0 ? x0 : -INFINITY, in1 ? x1 : -INFINITY));
      s0[v] = in0 ? x0 : kOut;
      s1[v] = in1 ? x1 : kOut;
    }
    if constexpr (kCap || kBias) {  // all of the exponent is in the scores
      f.p0 = 1.f;
      f.p1 = f.p2 = f.p3 = 0.f;
      return half_max(mx);
    }
  }
  mx = half_max(mx);
  return mx > -INFINITY ? capped<kCap>(f, mx) : mx;
}

// Src: what the tiles are.
//   int steps               of the workgroup
//   int mine                of this wavefront: it takes the first ones
//   rows<kV>(i)             this wavefront's 16 rows of step i's K or V tile
//   clean(i, lds)           the V tile that the step is about to use (all
//                           wavefronts): see only_finite
//   take(i, s0, s1, mx, mn, form) -> bound   as take_tile
template <int D, bool kCap, bool kLinear, bool kLse, typename Src>
__device__ __forceinline__ void run_pipe(Src& src, const QFrag<__bf16, D>& q, RowState<D>& st,
                                         uint8_t* smem, int lane, int stride) {
  using T = __bf16;
  using G = Tile<T, D>;
  constexpr int kTile = kKeys * G::kRow;
  constexpr int kSteps = G::kSteps;         // of QK^T: 16 dims each
  static_assert(kSteps == 2 * G::kGroupDmas, "a DMA instruction a step");
  constexpr int kEach = 32 / kSteps;        // present scores that go with one
  constexpr int kPv = 4 * (D / 32);         // matrix instructions of PV
  constexpr int kDone = 32 / kPv;           // next scores that go with one
  const int l32 = lane & 31, hf = lane >> 5;
  // K slots 0 and 1, V slots 0 and 1
  const int lds0 = static_cast<int>(reinterpret_cast<size_t>((lds_u8*)smem));
  const int own = lds0 + uniform(threadIdx.x >> 6) * 16 * G::kRow;  // rows that it brings
  int kaddr = lds0 + G::lane_k(l32, hf);
  int vaddr = lds0 + 2 * kTile + G::lane_v(lane, l32, hf);
  int koff = G::template dma_lane<false>(lane, stride);
  int voff = G::template dma_lane<true>(lane, stride);
  const bf16x2 ones = bf16x2{static_cast<__bf16>(1.f), static_cast<__bf16>(1.f)};

  // The weight of score e (0 .. 31) of a tile, with its neighbour, into pb.
  bf16x8 pb[4];
  const auto weigh = [&](int e, const f32x16& s0, const f32x16& s1, const Form& f, float base,
                         float& sum, float& le) {
    const int i = e >> 3, v = 8 * (i & 1) + (e & 7);
    float p[2];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const float z = i < 2 ? s0[v + u] : s1[v + u];
      float b = -base, pz = f.p0;
      if constexpr (kLinear)
        b = fmaf(f.slope_key, static_cast<float>(key_of(v + u) + (i < 2 ? 0 : 32)), fmaf(-f.slope_key, f.d, -base));
      if constexpr (kCap) {
        const float y = z * z;
        pz = fmaf(y, fmaf(y, fmaf(y, f.p3, f.p2), f.p1), f.p0);
      }
      p[u] = __builtin_amdgcn_exp2f(fmaf(z, pz, b));
    }
    const bf16x2 pp = bf16x2{static_cast<__bf16>(p[0]), static_cast<__bf16>(p[1])};
    pb[i][e & 7] = pp[0];
    pb[i][(e & 7) + 1] = pp[1];
    sum = __builtin_amdgcn_fdot2_f32_bf16(pp, ones, sum, false);
    if constexpr (kLse) le += p[0] + p[1];
  };

  // n0, n1 = K Q^T from K slot `slot`, beside the weights of the tile c0, c1
  // and issue(s), s = 0 .. kSteps - 1
  const auto qk_and_weigh = [&](int slot, f32x16& n0, f32x16& n1, const f32x16& c0,
                                const f32x16& c1, const Form& f, auto issue) {
    const float base = st.base();
    float sum = 0.f, le = 0.f;
    u32x4 x[3][2];
#pragma unroll
    for (int s = 0; s < 3; ++s) {
      x[s][0] = G::k_frag(kaddr + slot, 0, s);
      x[s][1] = G::k_frag(kaddr + slot, 1, s);
    }
    n0 = n1 = f32x16{};
#pragma unroll
    for (int s = 0; s < kSteps; ++s) {
      n0 = dot_step<T>(x[s % 3][0], q.x[s], n0);
      n1 = dot_step<T>(x[s % 3][1], q.x[s], n1);
#pragma unroll
      for (int u = 0; u < kEach; u += 2) weigh(s * kEach + u, c0, c1, f, base, sum, le);
      issue(s);
      if (s + 3 < kSteps) {
        x[s % 3][0] = G::k_frag(kaddr + slot, 0, s + 3);
        x[s % 3][1] = G::k_frag(kaddr + slot, 1, s + 3);
      }
      __builtin_amdgcn_sched_barrier(0);
    }
    st.l += sum;
    st.le += le;
  };
  // O += V^T P^T from V slot `slot`; with(i) goes beside matrix instruction i
  const auto pv_and = [&](int slot, auto with) {
    constexpr int kAhead = 3;
    bf16x8 x[kAhead];
#pragma unroll
    for (int i = 0; i < kAhead; ++i) x[i] = G::v_frag(vaddr + slot, i % (D / 32), i / (D / 32));
#pragma unroll
    for (int i = 0; i < kPv; ++i) {
      const int db = i % (D / 32);
      st.o[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x[i % kAhead], pb[i / (D / 32)], st.o[db],
                                                        0, 0, 0);
      with(i);
      const int j = i + kAhead;
      if (j < kPv) x[j % kAhead] = G::v_frag(vaddr + slot, j % (D / 32), j / (D / 32));
      __builtin_amdgcn_sched_barrier(0);
    }
  };

  // step i: its tile's scores in c0, c1 with form f; leaves the next in n0, n1
  Form f;
  const auto step = [&](int i, f32x16& c0, f32x16& c1, f32x16& n0, f32x16& n1) {
    const int par = i & 1;
    // addresses made anew in every step: kept, each would hold a register
    asm volatile("" : "+v"(kaddr), "+v"(vaddr), "+v"(koff), "+v"(voff));
    // K of step i + 2 and V of step i + 1 (past the last step zeros, from nowhere)
    const i32x4 none = i32x4{0, 0, 0, kBufferWord3};
    const i32x4 krs = i + 2 < src.steps ? src.template rows<false>(i + 2) : none;
    const i32x4 vrs = i + 1 < src.steps ? src.template rows<true>(i + 1) : none;
    const auto issue = [&](int s) {
      if (s < G::kGroupDmas)
        dma_b128(own + par * kTile + s * 1024, G::template dma_off<false>(koff, s, stride), krs);
      else
        dma_b128(own + (2 + (par ^ 1)) * kTile + (s - G::kGroupDmas) * 1024,
                 G::template dma_off<true>(voff, s - G::kGroupDmas, stride), vrs);
    };
    src.clean(i, lds0 + (2 + par) * kTile);
    if (i < src.mine) {
      // (past the last tile a body like the others: its scores go nowhere)
      qk_and_weigh((par ^ 1) * kTile, n0, n1, c0, c1, f, issue);
      float mx = -INFINITY, mn = INFINITY;
      pv_and(par * kTile, [&](int e) {
#pragma unroll
        for (int u = 0; u < kDone; u += 2) {
          const int v = (e * kDone + u) & 15;
          const f32x16& n = e * kDone < 16 ? n0 : n1;
          mx = fmaxf(fmaxf(mx, n[v]), n[v + 1]);
          if constexpr (kCap) mn = fminf(fminf(mn, n[v]), n[v + 1]);
        }
        asm volatile("" : "+v"(mx), "+v"(mn));  // here, not where they are used
      });
      if (i + 1 < src.mine) st.rescale(src.take(i + 1, n0, n1, mx, mn, f));
    } else {
#pragma unroll
      for (int s = 0; s < kSteps; ++s) issue(s);
    }
    wait_vm<0>();
    __syncthreads();
  };

  dma_rows<T, D, false>(own, src.template rows<false>(0), koff, stride);
  dma_rows<T, D, true>(own + 2 * kTile, src.template rows<true>(0), voff, stride);
  if (src.steps > 1) dma_rows<T, D, false>(own + kTile, src.template rows<false>(1), koff, stride);
  wait_vm<0>();
  __syncthreads();
  f32x16 a0{}, a1{}, b0{}, b1{};
  if (src.mine > 0) {
    a0 = qk_block<T, D>(kaddr, 0, q);
    a1 = qk_block<T, D>(kaddr, 1, q);
    float mx = -INFINITY, mn = INFINITY;
#pragma unroll
    for (int v = 0; v < 16; ++v) {
      mx = fmaxf(fmaxf(mx, a0[v]), a1[v]);
      mn = fminf(fminf(mn, a0[v]), a1[v]);
    }
    st.rescale(src.take(0, a0, a1, mx, mn, f));
  }
  __syncthreads();  // K slot 0 is refilled by step 0
  for (int i = 0; i < src.steps; i += 2) {
    step(i, a0, a1, b0, b1);
    if (i + 1 < src.steps) step(i + 1, b0, b1, a0, a1);
  }
}

// A V tile (kKeys rows at LDS address `tile`) that some rows of the workgroup see
// other keys of than others: a weight of 0 times an infinity would be a NaN in
// rows that do not see the key, so the places that are not finite are taken out,
// to be added to the rows that see them at the end.  All wavefronts call this;
// returns whether there were any.
template <typename T, int D>
__device__ __forceinline__ bool clean_tile(int tile) {
  constexpr int kTile = kKeys * Tile<T, D>::kRow;
  bool bad = false;
  for (int i = threadIdx.x; i < kTile / 16; i += 256)
    bad |= not_finite<T>(*reinterpret_cast<const lds_u32x4*>(static_cast<size_t>(tile + 16 * i)));
  if (!__syncthreads_or(bad)) return false;
  for (int i = threadIdx.x; i < kTile / 16; i += 256) {
    lds_u32x4* p = reinterpret_cast<lds_u32x4*>(static_cast<size_t>(tile + 16 * i));
    *p = only_finite<T>(*p);
  }
  __syncthreads();
  return true;
}

// What clean_tile took out of a key's V row (of 32-wide blocks, this lane's dims
// of which start at `row`), for a row that sees the key.
template <typename T, int D>
__device__ __forceinline__ void add_not_finite_row(const T* row, bool sees, f32x16 (&o)[D / 32]) {
#pragma unroll
  for (int db = 0; db < D / 32; ++db)
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const float x = static_cast<float>(row[32 * db + key_of(i)]);
      if (sees && !(fabsf(x) < INFINITY)) o[db][i] += x;
    }
}

}  // namespace flash
}  // namespace sift
