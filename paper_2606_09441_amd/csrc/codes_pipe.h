// The software pipeline of the attention of many rows over 64-key tiles of e4m3 codes:
// that of flash_pipe.h (128 query rows of a workgroup, 32 of each wavefront; the scores of
// the next tile formed beside the weights of the present one, then PV beside the next
// tile's maxima), with codes in LDS.  They become bf16 in registers, once a wavefront: an
// eighth more for the VALU, but half the bytes through LDS, which the four wavefronts
// read the same tiles from, and room for three tiles of K and of V: the DMA of a tile has
// two steps to arrive in.
//
// A tile's four groups of 16 keys have scales of their own.  V's are part of the conversions
// and of the exponents (ValueScale), K's a factor of the exponents; where scores are capped
// or biased K's are multiplied into the scores beside PV.
#pragma once

#include "codes.h"
#include "flash_pipe.h"

namespace sift {
namespace flash {

constexpr int kGroups = kKeys / 16;

// kPages: 1 where a tile lies in one page, else as many as it has groups.
// A tile: this wavefront's 16 rows, and its pages.
template <int kPages>
struct CodeWhere {
  int64_t row;
  int32_t n;
  int32_t page[kPages];
};
template <int kPages>
struct CodeScales {
  float k[kPages], v[kPages];
};
// A tile's V scales.
template <int kPages>
struct ValueScales {
  ValueScale g[kPages];
  __device__ __forceinline__ void set(const CodeScales<kPages>& z) {
#pragma unroll
    for (int i = 0; i < kPages; ++i) g[i].set(z.v[i]);
  }
};

// Src: what the tiles are.
//   int steps               of the workgroup;  int mine: of this wavefront, the first ones
//   where(i)                step i's tile, no rows of it past the last step
//   rows<kV>(where), scales(where): this wavefront's rows of K or V; the tile's scales
//   take(i, s0, s1, mx, mn, form) -> bound   as take_tile, of scaled products; kPlain:
//   mask(i, s0, s1, mx), which only hides what a row does not see, and corrects mx
template <int D, int kPages, bool kCap, bool kPlain, typename Src>
__device__ __forceinline__ void run_code_pipe(Src& src, const CodeQ<D>& q, RowState<D>& st,
                                              int lds0, int lane, int stride) {
  using C = CodeTile<D>;
  static_assert(kPages == 1 || kPages == kGroups, "");
  constexpr int kSame = kGroups / kPages;   // groups of a page
  constexpr int kTile = kKeys * C::kRow;
  constexpr int kSteps = D / 16;            // of QK^T: 16 dims each
  constexpr int kEach = 32 / kSteps;        // present scores that go with one
  constexpr int kPv = 4 * (D / 32);         // matrix instructions of PV
  constexpr int kDone = 32 / kPv;           // next scores that go with one
  constexpr int kDmas = C::kGroupDmas;
  const int l32 = lane & 31, hf = lane >> 5;
  // K slots 0, 1 and 2, then V's
  const int own = lds0 + uniform(threadIdx.x >> 6) * 16 * C::kRow;  // rows that it brings
  int kaddr = lds0 + C::lane_k(l32, hf);
  int vaddr = lds0 + 3 * kTile + C::lane_v(lane, hf);
  const int koff = C::template dma_lane<false>(lane, stride);
  const int voff = C::template dma_lane<true>(lane, stride);
  const bf16x2 ones = bf16x2{static_cast<__bf16>(1.f), static_cast<__bf16>(1.f)};

  Form f;
  float fk[kPages];  // kPlain: K's scales and the scores'
  ValueScales<kPages> w;
  // The bound of a tile's scores from its pages' largest products.
  const auto largest = [&](const float (&m)[kPages]) {
    float x = m[0] * fk[0];
#pragma unroll
    for (int g = 1; g < kPages; ++g) x = fmaxf(x, m[g] * fk[g]);
    return half_max(x);
  };
  // The weight of score e (0 .. 31) of a tile, with its neighbour, into pb.
  bf16x8 pb[kGroups];
  const auto weigh = [&](int e, const f32x16& s0, const f32x16& s1, const Form& f, float p0,
                         float base, float& sum, float& le) {
    const int i = e >> 3, v = 8 * (i & 1) + (e & 7);
    float p[2];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const float z = i < 2 ? s0[v + u] : s1[v + u];
      float pz = p0;
      if constexpr (kCap) {
        const float y = z * z;
        pz = fmaf(y, fmaf(y, fmaf(y, f.p3, f.p2), f.p1), f.p0);
      }
      p[u] = __builtin_amdgcn_exp2f(fmaf(z, pz, -base));
    }
    const bf16x2 pp = bf16x2{static_cast<__bf16>(p[0]), static_cast<__bf16>(p[1])};
    pb[i][e & 7] = pp[0];
    pb[i][(e & 7) + 1] = pp[1];
    sum = __builtin_amdgcn_fdot2_f32_bf16(pp, ones, sum, false);
    le += p[0] + p[1];
  };

  // n0, n1 = K Q^T from K slot `slot`, beside the weights of the tile c0, c1 and issue(s)
  const auto qk_and_weigh = [&](int slot, f32x16& n0, f32x16& n1, const f32x16& c0,
                                const f32x16& c1, const Form& f,
                                const ValueScales<kPages>& w, auto issue) {
    const float base = st.base();
    float sum = 0.f, le = 0.f;
    u32x4 x[2][2];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      x[u][0] = C::k_chunk(kaddr + slot, u);
      x[u][1] = C::k_chunk(kaddr + slot + 32 * C::kRow, u);
    }
    n0 = n1 = f32x16{};
#pragma unroll
    for (int s = 0; s < kSteps; ++s) {
      const u32x4 a = x[(s >> 1) & 1][0], b = x[(s >> 1) & 1][1];
      const int j = 2 * (s & 1);
      n0 = __builtin_amdgcn_mfma_f32_32x32x16_bf16(code_values(u32x2{a[j], a[j + 1]}),
                                                   __builtin_bit_cast(bf16x8, q.x[s]), n0, 0, 0, 0);
      n1 = __builtin_amdgcn_mfma_f32_32x32x16_bf16(code_values(u32x2{b[j], b[j + 1]}),
                                                   __builtin_bit_cast(bf16x8, q.x[s]), n1, 0, 0, 0);
#pragma unroll
      for (int u = 0; u < kEach; u += 2) {
        const int e = s * kEach + u, i = (e >> 3) / kSame;
        weigh(e, c0, c1, f, kPlain ? fk[i] : f.p0, base + w.g[i].lift, sum, le);
        if (e % (8 * kSame) == 8 * kSame - 2) {  // the page's last
          st.l = fmaf(sum, w.g[i].undo, st.l);
          st.le = fmaf(le, w.g[i].undo, st.le);
          sum = le = 0.f;
        }
      }
      issue(s);
      if ((s & 1) && (s >> 1) + 2 < kSteps / 2) {
        x[(s >> 1) & 1][0] = C::k_chunk(kaddr + slot, (s >> 1) + 2);
        x[(s >> 1) & 1][1] = C::k_chunk(kaddr + slot + 32 * C::kRow, (s >> 1) + 2);
      }
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  // O += V^T P^T from V slot `slot`; with(i) goes beside matrix instruction i
  const auto pv_and = [&](int slot, auto with) {
    constexpr int kAhead = 4;
    u32x2 x[kAhead];
#pragma unroll
    for (int i = 0; i < kAhead; ++i) x[i] = C::v_codes(vaddr + slot, i % (D / 32), i / (D / 32));
#pragma unroll
    for (int i = 0; i < kPv; ++i) {
      const int db = i % (D / 32);
      st.o[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
          code_values(x[i % kAhead], w.g[i / (D / 32) / kSame].power), pb[i / (D / 32)], st.o[db],
          0, 0, 0);
      with(i);
      const int j = i + kAhead;
      if (j < kPv) x[j % kAhead] = C::v_codes(vaddr + slot, j % (D / 32), j / (D / 32));
      __builtin_amdgcn_sched_barrier(0);
    }
  };

  // Of steps i + 2 and i + 3; the scales of step i + 1.  Tables and scales are asked for
  // a step before they are used.
  CodeWhere<kPages> in2 = src.where(2), in3 = src.where(3);
  CodeScales<kPages> next;
  // Slots (byte offsets) of K of steps i, i + 1 and i + 2, and of V's.
  int k0 = 0, k1 = kTile, k2 = 2 * kTile, v0 = 0, v1 = kTile, v2 = 2 * kTile;
  // step i: its tile's scores in c0, c1 with form f; leaves the next in n0, n1
  const auto step = [&](int i, f32x16& c0, f32x16& c1, f32x16& n0, f32x16& n1) {
    // addresses made anew in every step: kept, each would hold a register
    asm volatile("" : "+v"(kaddr), "+v"(vaddr));
    // K of step i + 3 and V of step i + 2 (past the last step zeros, from nowhere)
    const i32x4 krs = src.template rows<false>(in3), vrs = src.template rows<true>(in2);
    const auto issue = [&](int s) {
      if (s < kDmas)
        dma_b128(own + k0 + s * 1024, C::template dma_off<false>(koff, s, stride), krs);
      else if (s < 2 * kDmas)
        dma_b128(own + 3 * kTile + v2 + (s - kDmas) * 1024,
                 C::template dma_off<true>(voff, s - kDmas, stride), vrs);
    };
    const CodeScales<kPages> now = next;
    if (i < src.mine) {
      // (past the last tile a body like the others: its scores go nowhere)
      qk_and_weigh(k1, n0, n1, c0, c1, f, w, issue);
      float ks[kPages];
#pragma unroll
      for (int g = 0; g < kPages; ++g) ks[g] = usable_scale(now.k[g]);
      float mx = -INFINITY, mn = INFINITY;
      float mg[kPages];
#pragma unroll
      for (float& m : mg) m = -INFINITY;
      pv_and(v0, [&](int e) {
#pragma unroll
        for (int u = 0; u < kDone; u += 2) {
          const int x = e * kDone + u, v = x & 15;
          f32x16& n = x < 16 ? n0 : n1;
          if constexpr (kPlain) {
            float& m = mg[(x >> 3) / kSame];
            m = fmaxf(fmaxf(m, n[v]), n[v + 1]);
            asm volatile("" : "+v"(m));  // here, not where it is used
          } else {
            n[v] *= ks[(x >> 3) / kSame];
            n[v + 1] *= ks[(x >> 3) / kSame];
            mx = fmaxf(fmaxf(mx, n[v]), n[v + 1]);
            if constexpr (kCap) mn = fminf(fminf(mn, n[v]), n[v + 1]);
          }
        }
        if constexpr (!kPlain) asm volatile("" : "+v"(mx), "+v"(mn));
      });
      if (i + 1 < src.mine) {
        if constexpr (kPlain) {
#pragma unroll
          for (int g = 0; g < kPages; ++g) fk[g] = ks[g] * src.factor();
          src.mask(i + 1, n0, n1, mg);
          st.rescale(largest(mg));
        } else {
          st.rescale(src.take(i + 1, n0, n1, mx, mn, f));
        }
        w.set(now);
      }
    } else {
#pragma unroll
      for (int s = 0; s < 2 * kDmas; ++s) issue(s);
    }
    next = src.scales(in2);
    in2 = in3;
    in3 = src.where(i + 4);
    wait_vm<2 * kDmas>();  // but for those of this step
    __syncthreads();
    const int a = k0, b = v0;
    k0 = k1, k1 = k2, k2 = a;
    v0 = v1, v1 = v2, v2 = b;
  };

  const auto bring_k = [&](int slot, const CodeWhere<kPages>& y) {
    C::template dma_rows<false>(own + slot * kTile, src.template rows<false>(y), koff, stride);
  };
  const auto bring_v = [&](int slot, const CodeWhere<kPages>& y) {
    C::template dma_rows<true>(own + (3 + slot) * kTile, src.template rows<true>(y), voff, stride);
  };
  CodeScales<kPages> first;
  {
    const CodeWhere<kPages> in0 = src.where(0), in1 = src.where(1);
    bring_k(0, in0);
    bring_v(0, in0);
    bring_k(1, in1);
    bring_k(2, in2);
    bring_v(1, in1);
    first = src.scales(in0);
    next = src.scales(in1);
  }
  wait_vm<2 * kDmas>();
  __syncthreads();
  f32x16 a0{}, a1{}, b0{}, b1{};
  if (src.mine > 0) {
    float ks[kPages];
#pragma unroll
    for (int g = 0; g < kPages; ++g) ks[g] = usable_scale(first.k[g]);
    a0 = qk_codes<D>(kaddr, q);
    a1 = qk_codes<D>(kaddr + 32 * C::kRow, q);
    if constexpr (kPlain) {
      float mg[kPages];
#pragma unroll
      for (float& m : mg) m = -INFINITY;
#pragma unroll
      for (int v = 0; v < 16; ++v) {
        float &m0 = mg[(v >> 3) / kSame], &m1 = mg[(2 + (v >> 3)) / kSame];
        m0 = fmaxf(m0, a0[v]);
        m1 = fmaxf(m1, a1[v]);
      }
#pragma unroll
      for (int g = 0; g < kPages; ++g) fk[g] = ks[g] * src.factor();
      src.mask(0, a0, a1, mg);
      st.rescale(largest(mg));
    } else {
      float mx = -INFINITY, mn = INFINITY;
#pragma unroll
      for (int v = 0; v < 16; ++v) {
        a0[v] *= ks[(v >> 3) / kSame];
        a1[v] *= ks[(2 + (v >> 3)) / kSame];
        mx = fmaxf(fmaxf(mx, a0[v]), a1[v]);
        mn = fminf(fminf(mn, a0[v]), a1[v]);
      }
      st.rescale(src.take(0, a0, a1, mx, mn, f));
    }
    w.set(first);
  }
  __syncthreads();  // K slot 0 is refilled by step 0
  for (int i = 0; i < src.steps; i += 2) {
    step(i, a0, a1, b0, b1);
    if (i + 1 < src.steps) step(i + 1, b0, b1, a0, a1);
  }
  wait_vm<0>();  // zeros from nowhere, into LDS that is used again
  __syncthreads();
}

}  // namespace flash
}  // namespace sift
