// Attention of new tokens over a paged cache held in e4m3, with a scale for each page
// and kv head: the units, their split over the workgroups and the merge are those of
// cache_attn.hip.  HBM bounds it, at half the bytes of bf16.
//
// K's scale is a factor of the scores, V's one of the conversion and of the weights, there
// part of the exponent (ValueScale), so that neither costs an operation a key.  Codes become
// bf16 in registers, exactly, on the way from LDS to the matrix instructions; the new tokens' own keys are bf16 tiles, taken last.
// 8 sequences of 131072 slots, 32/8 heads, D = 128: 392 us, 5.5 TB/s of HBM; 32 of 200 to
// 16640 slots 60 us, 4.3 TB/s: ten of them until the first tiles are there and after the
// last, and workgroups that the memory serves unevenly (they end between 42 and 60 us).
// Each wavefront has two tiles of K and of V in LDS, in the room that a bf16 one takes:
// K of the tile after next is fetched as soon as K is read, V likewise.

#include "cache.h"
#include "codes.h"
#include "sift_internal.h"

namespace sift {
namespace {

using namespace cache;

constexpr int kTileKeys = Narrow::kTileKeys;
constexpr int kStepTiles = Narrow::kStepTiles;
constexpr int kRows = Narrow::kRows;

// A tile of cached keys, in one page or two of 16: its rows, as many of them as are
// valid, and the scales.
template <int kPages>
struct CodeRows {
  int64_t row[kPages];
  int32_t n[kPages];
};
template <int kPages>
struct Scales {
  float k[kPages], v[kPages];
};

template <int D, int kPages, bool kCap, bool kBias>
__global__ __launch_bounds__(256, 2) void cache_codes_kernel(CacheAttnArgs p) {
  using T = __bf16;
  using G = Tile<T, D>;       // of the new tokens' keys
  using C = CodeTile<D>;      // of the cached ones
  constexpr int kTile = kTileKeys * G::kRow;
  constexpr int kCodes = kTileKeys * C::kRow;  // half of it
  constexpr int kDmas = 2 * C::kGroupDmas;     // of a K or V tile
  constexpr int kEach = kTileKeys / kPages;    // keys of a page
  __shared__ __attribute__((aligned(1024))) uint8_t smem[4 * 2 * kTile];
  __shared__ float part[4][kRows][3];
  const CacheArgs& a = p.c;
  const int g = a.hq / a.hkv;
  const UnitCost<NarrowCodes> cost{g, a.hkv};
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
  const int stride = a.hkv * C::kRow, stride_new = a.hkv * G::kRow;
  const int lds0 = static_cast<int>(reinterpret_cast<size_t>((lds_u8*)smem));
  const int kt = lds0 + wave * 2 * kTile, vt = kt + kTile;  // this wavefront's tiles
  const int klane = C::lane_k(l32, hf), vlane = C::lane_v(lane, hf);
  const int koff = C::template dma_lane<false>(lane, stride);
  const int voff = C::template dma_lane<true>(lane, stride);
  const float c = kCap || kBias ? 1.f : a.sc.c;  // score_factor

  while (x < xend && pl.b < a.num_seqs) {
    // the unit that holds step x
    const int b = pl.b;
    const int len = s.len, n = s.n, row0 = s.row0;
    const int steps = uniform(cost.steps(s)), blocks = uniform(cost.blocks(s));
    const int unit = Split::quotient(x - pl.at, steps);
    const int s0 = x - pl.at - unit * steps;
    const int s1 = min(steps, s0 + (xend - x));
    const int kvh = unit / blocks, r0 = unit % blocks * kRows;
    const int ct = cost.cached_tiles(s);
    const int tiles = cost.tiles(s);

    const int r = r0 + l32;
    const bool live = r < n * g;
    const int node = live ? r / g : 0;
    const int h = kvh * g + (live ? r % g : 0);
    CodeQ<D> q;
    q.load(static_cast<const T*>(a.q) + (static_cast<int64_t>(row0 + node) * a.hq + h) * D, hf,
           live);
    const float slope = kBias ? a.sc.slopes[h] * kLog2e : 0.f;
    const int my_pos = !kBias ? 0 : a.row_pos != nullptr ? a.row_pos[row0 + node] : len + node;

    const auto rows_of = [&](int t) {
      CodeRows<kPages> y;
#pragma unroll
      for (int i = 0; i < kPages; ++i) {
        const int slot = t * kTileKeys + i * kEach;
        const Rows16 r = cached_rows(a, b, len, slot);
        y.row[i] = r.row;
        y.n[i] = r.n;
        if constexpr (kEach > 16) {  // the same page's next 16
          if (r.n == 16) y.n[i] += cached_rows(a, b, len, slot + 16).n;
        }
      }
      return y;
    };
    const auto scales_of = [&](const CodeRows<kPages>& y) {
      Scales<kPages> z;
#pragma unroll
      for (int i = 0; i < kPages; ++i) {
        const int64_t at = (y.row[i] >> a.page_shift) * a.hkv + kvh;
        z.k[i] = scalar(p.k_scales, at);
        z.v[i] = scalar(p.v_scales, at);
      }
      return z;
    };
    const auto fetch = [&](const CodeRows<kPages>& y, int slot, auto v) {
      constexpr bool kV = decltype(v)::value;
      const void* base = kV ? a.v : a.k;
#pragma unroll
      for (int i = 0; i < kPages; ++i) {
        const i32x4 rs = rows_rsrc(reinterpret_cast<unsigned long long>(base) +
                                       (y.row[i] * a.hkv + kvh) * C::kRow,
                                   y.n[i], stride, C::kRow);
#pragma unroll
        for (int j = 0; j < kEach; j += 16)
          C::template dma_rows<kV>((kV ? vt : kt) + slot * kCodes + (i * kEach + j) * C::kRow, rs,
                                   kV ? voff : koff, stride, j);
      }
    };
    constexpr std::false_type kK{};
    constexpr std::true_type kV{};

    RowState<D> st;
    st.clear();
    // Products sc of the tile that begins with key j0 (of the cache, or of the new ones),
    // of whose keys this row sees `bits`, to the exponents' form, and the reference moved:
    // what is left is c (times K's scales) and the returned offset.
    const auto shape = [&](f32x16& sc, uint32_t bits, bool fresh, int j0, const float (&f)[2]) {
      if constexpr (kCap) cap_scores(a.sc, sc);
      if (__builtin_amdgcn_ballot_w64(bits != ~0u)) mask_block(sc, bits >> (4 * hf));
      float off = 0.f;
      if constexpr (kBias) {
        const auto bias = [&](auto far) {
          off = half_max(largest_bias(sc, slope, far));
          if (off == -INFINITY) off = 0.f;
          add_bias(a.sc, sc, slope, off, far);
        };
        if ((fresh ? a.row_pos : a.key_pos) != nullptr) {
          float dist[16];
#pragma unroll
          for (int v = 0; v < 16; ++v) {
            const int j = j0 + 4 * hf + key_of(v);
            const int pos =
                fresh ? a.row_pos[row0 + min(j, n - 1)]
                      : a.key_pos[((static_cast<int64_t>(b) * a.hkv + kvh) * a.max_pages
                                   << a.page_shift) +
                                  min(j, (a.max_pages << a.page_shift) - 1)];
            dist[v] = fabsf(static_cast<float>(my_pos - pos));
          }
          bias([&](int v) { return dist[v]; });
        } else {
          const float d0 = static_cast<float>(my_pos - (fresh ? len : 0) - j0 - 4 * hf);
          bias([&](int v) { return fabsf(d0 - static_cast<float>(key_of(v))); });
        }
      }
      float m0 = sc[0], m1 = sc[8];
#pragma unroll
      for (int v = 1; v < 8; ++v) {
        m0 = fmaxf(m0, sc[v]);
        m1 = fmaxf(m1, sc[8 + v]);
      }
      st.rescale(half_max(fmaxf(m0 * f[0], m1 * f[1])) + off);
      return off;
    };

    // (of the unit's steps the first kLead are none)
    const int first = max(s0 - NarrowCodes::kLead, 0), last = max(s1 - NarrowCodes::kLead, 0);
    const int tend = min(tiles, last * kStepTiles);
    const int cend = min(ct, tend);
    int t = first * kStepTiles + wave;
    if (t < cend) {
      // Of this tile, the next and the one after; the scales are asked for behind the rows.
      // In the loop, tables and scales are asked for while the weights are made: an answer
      // that is on its way would hold up reads of LDS, which count with it.
      CodeRows<kPages> now = rows_of(t), next = rows_of(min(t + kStepTiles, cend - 1));
      fetch(now, 0, kK);
      fetch(now, 0, kV);
      if (t + kStepTiles < cend) {
        fetch(next, 1, kK);
        fetch(next, 1, kV);
      }
      CodeRows<kPages> after = rows_of(min(t + 2 * kStepTiles, cend - 1));
      Scales<kPages> mine = scales_of(now);
      int slot = 0;
      for (; t < cend; t += kStepTiles, slot ^= 1) {
        const bool one = t + kStepTiles < cend, two = t + 2 * kStepTiles < cend;
        uint32_t bits = static_cast<uint32_t>(low_bits(now.n[0]));
        if constexpr (kPages == 2) bits |= static_cast<uint32_t>(low_bits(now.n[1])) << 16;
        if (one)
          wait_vm<3 * kDmas>();  // K is there, V and the next tile may still be on their way
        else
          wait_vm<kDmas>();
        f32x16 sc = qk_codes<D>(kt + slot * kCodes + klane, q);
        wait_lds();  // K is read
        if (two) fetch(after, slot, kK);
        const CodeRows<kPages> third = rows_of(min(t + 3 * kStepTiles, cend - 1));
        const Scales<kPages> then = scales_of(next);
        float f[2], base[2], undo[2], power[2];
#pragma unroll
        for (int i = 0; i < kPages; ++i) {
          const float ks = usable_scale(mine.k[i]);
          f[i] = ks * c;
          if constexpr (kCap || kBias) {
#pragma unroll
            for (int v = i * kEach / 2; v < (i + 1) * kEach / 2; ++v) sc[v] *= ks;
            f[i] = c;
          }
          ValueScale vs;
          vs.set(mine.v[i]);
          base[i] = vs.lift;
          undo[i] = vs.undo;
          power[i] = vs.power;
        }
        if constexpr (kPages == 1) {
          f[1] = f[0];
          base[1] = base[0];
          undo[1] = undo[0];
          power[1] = power[0];
        }
        const float off = shape(sc, bits, false, t * kTileKeys, f);
#pragma unroll
        for (int i = 0; i < 2; ++i) base[i] += st.base() - off;
        weigh_codes(sc, f, base, undo, st.l, st.le);
        if (two)
          wait_vm<3 * kDmas>();
        else if (one)
          wait_vm<2 * kDmas>();
        else
          wait_vm<0>();
        pv_codes<D>(vt + slot * kCodes + vlane, sc, power, st.o);
        wait_lds();  // V is read
        if (two) fetch(after, slot, kV);
        now = next;
        next = after;
        after = third;
        mine = then;
      }
    }
    // the new tokens' own
    for (; t < tend; t += kStepTiles) {
      const int j0 = (t - ct) * kTileKeys;
      const int koff_new = G::template dma_lane<false>(lane, stride_new);
      const int voff_new = G::template dma_lane<true>(lane, stride_new);
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int64_t at = (static_cast<int64_t>(row0) + j0 + 16 * i) * a.hkv + kvh;
        const int have = min(max(n - j0 - 16 * i, 0), 16);
        dma_rows<T, D, false>(
            kt + i * 16 * G::kRow,
            rows_rsrc(reinterpret_cast<unsigned long long>(p.k_new) + at * G::kRow, have,
                      stride_new, G::kRow),
            koff_new, stride_new);
        dma_rows<T, D, true>(
            vt + i * 16 * G::kRow,
            rows_rsrc(reinterpret_cast<unsigned long long>(p.v_new) + at * G::kRow, have,
                      stride_new, G::kRow),
            voff_new, stride_new);
      }
      uint32_t bits = static_cast<uint32_t>(low_bits(n - j0));
      if (p.tree_mask != nullptr)
        bits &= static_cast<uint32_t>(
            p.tree_mask[static_cast<int64_t>(row0 + node) * p.mask_words + (j0 >> 6)] >>
            (j0 & 32));
      else
        bits &= static_cast<uint32_t>(low_bits(node + 1 - j0));
      wait_vm<0>();
      f32x16 sc = qk_beside_codes<D>(kt, l32, hf, q);
      float f[2] = {c, c};
      const float off = shape(sc, bits, true, j0, f);
      weigh_block<T, true>(sc, c, st.base() - off, st.l, st.le);
      mend_own_tile<T, D>(vt, live ? bits : 0u, lane, st.o);
      pv_block<T, D>(vt + G::lane_v(lane, l32, hf), sc, st.o);
      wait_lds();
    }

    const bool whole = s0 == 0 && s1 == steps;
    merge_waves<D>(st, kt, lds0, 2 * kTile, part, wave, l32, hf,
                   [&](int row, int dim, const float(&o)[4], float top, float l, float le) {
                     const int rr = r0 + row;
                     if (rr >= n * g) return;
                     const int64_t at =
                         static_cast<int64_t>(row0 + rr / g) * a.hq + kvh * g + rr % g;
                     const int64_t slot =
                         (2 * static_cast<int64_t>(group) + (s0 == 0)) * kRows + row;
                     if (whole) {
                       store_row(static_cast<T*>(p.out) + at * D + dim, o, inverse(l));
                       if (dim == 0 && p.lse != nullptr) p.lse[at] = log_sum(top, le);
                     } else {
                       *reinterpret_cast<f32x4*>(p.part_o + slot * D + dim) =
                           f32x4{o[0], o[1], o[2], o[3]};
                       if (dim == 0) p.part_ml[slot] = float4{top, l, le, 0.f};
                     }
                   });
    x += s1 - s0;
    if (x < xend && x - pl.at >= cost(s)) {
      const Work work(a, cost);
      pl = work.find(x);
      s = work.seq(pl.b);
    }
  }
}

}  // namespace

hipError_t launch_cache_codes(const CacheAttnArgs& a, int head_dim, hipStream_t stream) {
  const auto launch = [&](auto dim, auto pages, auto cap, auto bias) {
    hipLaunchKernelGGL((cache_codes_kernel<decltype(dim)::value, decltype(pages)::value,
                                           decltype(cap)::value, decltype(bias)::value>),
                       dim3(a.groups), dim3(256), 0, stream, a);
  };
  const auto of = [&](auto dim, auto pages) {
    const std::true_type yes;
    const std::false_type no;
    if (a.c.sc.x != 0.f)
      a.c.sc.slopes != nullptr ? launch(dim, pages, yes, yes) : launch(dim, pages, yes, no);
    else
      a.c.sc.slopes != nullptr ? launch(dim, pages, no, yes) : launch(dim, pages, no, no);
  };
  const auto with_pages = [&](auto dim) {
    if ((1 << a.c.page_shift) >= kTileKeys)
      of(dim, std::integral_constant<int, 1>{});
    else
      of(dim, std::integral_constant<int, 2>{});
  };
  if (head_dim == 128)
    with_pages(std::integral_constant<int, 128>{});
  else
    with_pages(std::integral_constant<int, 64>{});
  return hipGetLastError();
}

}  // namespace sift
