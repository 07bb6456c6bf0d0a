// The attention of many new tokens over a paged cache held in e4m3: units of 128 rows of
// a (sequence, kv head), as in cache_wide.hip, over the pipeline of codes_pipe.h.  The new
// tokens' own keys, bf16 tiles, are taken last and one at a time.
//
// 64 tokens, 48/8 heads, D = 128 over 66048 slots: 153 us of the call with its merge, 680
// TFLOP/s (another card, both caches in turn: 157, bf16 161).  The vector unit issues in 58%
// of the SIMDs' cycles (12 operations a matrix instruction, four of them conversions), the
// matrix cores are busy in 35%, one or the other in 72%.  Twice the slots cost 116 us more: 34 are a workgroup's start and end
// and the merge of what they share, 33 MB of sums written and read again.  In the others
// the vector unit is what counts: with the exponentials' longer issue (four times the
// others') its operations fill nine tenths of the cycles, and one workgroup on a CU does as
// many tiles as two.  Kernels of their own for tiles in one page keep a scale where four
// would be, and spill less (27 registers a lane, not 39): 158 us, not 170 in one run.
// Capped scores take 186 and biased ones 203: 18.6 vector operations a matrix instruction
// capped, not 12.2, among them K's scale times every score, which plain ones have in their
// factor.

#include "cache.h"
#include "codes_pipe.h"
#include "sift_internal.h"

namespace sift {
namespace {

using namespace cache;

// Cached tiles s0 .. of a unit.
template <int D, int kPages, bool kCap, bool kBias>
struct CodeTiles {
  const CacheAttnArgs& p;
  int b, len, kvh;
  int s0, steps, mine;
  int turn;          // its steps begin with the turn-th, and go round
  int wave, hf;
  float slope;
  int pos;

  // (with a bias the near keys, which set the reference, come first)
  __device__ __forceinline__ int tile(int i) const {
    if constexpr (kBias) return s0 + steps - 1 - i;
    const int j = i + turn;
    return s0 + (j < steps ? j : j - steps);
  }
  // Step i's tile (past the last step none of its rows).
  __device__ __forceinline__ CodeWhere<kPages> where(int i) const {
    const CacheArgs& a = p.c;
    const int slot = tile(min(i, steps - 1)) * kKeys;
    const Rows16 r = cached_rows(a, b, len, slot + 16 * wave);
    CodeWhere<kPages> y;
    y.row = r.row;
    y.n = i < steps ? r.n : 0;
    if constexpr (kPages == 1) {
      y.page[0] = static_cast<int32_t>(r.row >> a.page_shift);
      return y;
    }
#pragma unroll
    for (int g = 0; g < kPages; ++g) {
      const int pi = min((slot + 16 * g) >> a.page_shift, a.max_pages - 1);
      y.page[g] =
          within(scalar(a.table, static_cast<int64_t>(b) * a.max_pages + pi), a.num_pages - 1);
    }
    return y;
  }
  template <bool kV>
  __device__ __forceinline__ i32x4 rows(const CodeWhere<kPages>& y) const {
    using C = CodeTile<D>;
    const CacheArgs& a = p.c;
    return rows_rsrc(reinterpret_cast<unsigned long long>(kV ? a.v : a.k) +
                         (y.row * a.hkv + kvh) * C::kRow,
                     y.n, a.hkv * C::kRow, C::kRow);
  }
  // As they are.
  __device__ __forceinline__ CodeScales<kPages> scales(const CodeWhere<kPages>& y) const {
    CodeScales<kPages> z;
#pragma unroll
    for (int g = 0; g < kPages; ++g) {
      const int64_t at = static_cast<int64_t>(y.page[g]) * p.c.hkv + kvh;
      z.k[g] = scalar(p.k_scales, at);
      z.v[g] = scalar(p.v_scales, at);
    }
    return z;
  }
  // One bit a key of tile t.
  __device__ __forceinline__ uint64_t bits(int t) const {
    const CacheArgs& a = p.c;
    if (a.page_lens == nullptr) return low_bits(len - t * kKeys);
    uint64_t m = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i)
      m |= low_bits(cached_rows(a, b, len, t * kKeys + 16 * i).n) << (16 * i);
    return m;
  }
  __device__ __forceinline__ float factor() const { return p.c.sc.c; }
  __device__ __forceinline__ void mask(int i, f32x16& s0_, f32x16& s1_, float (&mg)[kPages]) const {
    const uint64_t m = bits(tile(i));
    if (m == ~uint64_t(0)) return;
    mask_block(s0_, static_cast<uint32_t>(m >> (4 * hf)));
    mask_block(s1_, static_cast<uint32_t>(m >> (32 + 4 * hf)));
#pragma unroll
    for (float& m : mg) m = -INFINITY;
#pragma unroll
    for (int v = 0; v < 32; ++v) {
      float& m = mg[(v >> 3) * kPages / kGroups];
      m = fmaxf(m, v < 16 ? s0_[v & 15] : s1_[v & 15]);
    }
  }
  __device__ __forceinline__ float take(int i, f32x16& s0_, f32x16& s1_, float mx, float mn,
                                        Form& f) const {
    const CacheArgs& a = p.c;
    const int t = tile(i);
    const uint64_t m = bits(t);
    const int j0 = t * kKeys + 4 * hf;
    const int slots = a.max_pages << a.page_shift;
    const int32_t* table =
        kBias && a.key_pos != nullptr
            ? a.key_pos + (static_cast<int64_t>(b) * a.hkv + kvh) * slots
            : nullptr;
    const float d = static_cast<float>(pos - j0);
    return take_tile<kCap, kBias>(
        a.sc, s0_, s1_, mx, mn, kBias || ~m != 0, [&] { return m; }, hf, slope,
        [&](int key) {
          return fabsf(table != nullptr ? static_cast<float>(pos - table[min(j0 + key, slots - 1)])
                                        : d - static_cast<float>(key));
        },
        f);
  }
};

template <int D, int kPages, bool kCap, bool kBias>
__global__ __launch_bounds__(256, 2) void codes_wide_kernel(CacheAttnArgs p) {
  using T = __bf16;
  using G = Tile<T, D>;
  using C = CodeTile<D>;
  // six tiles of codes; or K and V of a bf16 one
  static_assert(6 * C::kRow >= 2 * G::kRow, "");
  __shared__ __attribute__((aligned(1024))) uint8_t smem[6 * kKeys * C::kRow];
  const CacheArgs& a = p.c;
  const int g = a.hq / a.hkv;
  const UnitCost<Wide> cost{g, a.hkv};
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
  const int run = xend - x;
  const int lds0 = static_cast<int>(reinterpret_cast<size_t>((lds_u8*)smem));

  while (x < xend && pl.b < a.num_seqs) {
    const int b = pl.b;
    const int steps = uniform(cost.steps(s)), blocks = uniform(cost.blocks(s));
    const int unit = Split::quotient(x - pl.at, steps);
    const int s0 = x - pl.at - unit * steps;
    const int s1 = min(steps, s0 + (xend - x));
    const int kvh = unit / blocks, r0 = unit % blocks * Wide::kRows;
    const int r = r0 + 32 * wave + l32;
    const int len = s.len, n = s.n, row0 = s.row0;
    const bool live = r < n * g;
    const int token = live ? r / g : 0;
    const int h = kvh * g + (live ? r % g : 0);
    CodeQ<D> q;
    q.load(static_cast<const T*>(a.q) + (static_cast<int64_t>(row0 + token) * a.hq + h) * D, hf,
           live);
    RowState<D> st;
    st.clear();
    const int ct = uniform(cost.cached_tiles(s));
    const int c1 = min(s1, ct);  // the end of its cached tiles
    const bool any = r0 + 32 * wave < n * g;
    const float slope = kBias ? a.sc.slopes[h] * kLog2e : 0.f;
    const int pos =
        !kBias ? 0 : a.row_pos != nullptr ? a.row_pos[row0 + token] : len + token;
    if (s0 < c1) {
      // The first step is one whose number is a multiple of the runs' length, so that units
      // of the same keys read each tile at about the same time (cache_wide.hip).
      const int over = s0 - Split::quotient(s0, run) * run;
      const int turn = over > 0 ? run - over : 0;
      CodeTiles<D, kPages, kCap, kBias> src{p,      b,
                                    len,    kvh,
                                    s0,     c1 - s0,
                                    any ? c1 - s0 : 0,
                                    turn < c1 - s0 ? turn : 0,
                                    wave,   hf,
                                    slope,  pos};
      run_code_pipe<D, kPages, kCap, !kCap && !kBias>(src, q, st, lds0, lane, a.hkv * C::kRow);
    }
    // the new tokens' own
    bool cleaned = false;
    const int stride = a.hkv * G::kRow;
    const int vt = lds0 + kKeys * G::kRow;
    const auto seen_of = [&](int j0) {  // bits of 64 of them
      const uint64_t seen =
          p.tree_mask != nullptr
              ? p.tree_mask[static_cast<int64_t>(row0 + token) * p.mask_words + (j0 >> 6)]
              : low_bits(token + 1 - j0);
      return seen & low_bits(n - j0);
    };
    for (int t = max(s0, ct); t < s1; ++t) {
      const int j0 = (t - ct) * kKeys;
      const auto rows = [&](const void* base) {
        const int j = j0 + 16 * wave;
        return rows_rsrc(reinterpret_cast<unsigned long long>(base) +
                             ((static_cast<int64_t>(row0) + j) * a.hkv + kvh) * G::kRow,
                         min(max(n - j, 0), 16), stride, G::kRow);
      };
      dma_rows<T, D, false>(lds0 + 16 * wave * G::kRow, rows(p.k_new),
                            G::template dma_lane<false>(lane, stride), stride);
      dma_rows<T, D, true>(vt + 16 * wave * G::kRow, rows(p.v_new),
                           G::template dma_lane<true>(lane, stride), stride);
      wait_vm<0>();
      __syncthreads();
      cleaned |= clean_tile<T, D>(vt);
      if (any) {
        f32x16 z0 = qk_beside_codes<D>(lds0, l32, hf, q);
        f32x16 z1 = qk_beside_codes<D>(lds0 + 32 * G::kRow, l32, hf, q);
        float mx = -INFINITY, mn = INFINITY;
#pragma unroll
        for (int v = 0; v < 16; ++v) {
          mx = fmaxf(fmaxf(mx, z0[v]), z1[v]);
          mn = fminf(fminf(mn, z0[v]), z1[v]);
        }
        const uint64_t m = seen_of(j0);
        const float d = static_cast<float>(pos - len - j0 - 4 * hf);
        Form f;
        st.rescale(take_tile<kCap, kBias>(
            a.sc, z0, z1, mx, mn, true, [&] { return m; }, hf, slope,
            [&](int key) {
              return fabsf(a.row_pos != nullptr
                               ? static_cast<float>(pos - a.row_pos[row0 + min(j0 + 4 * hf + key, n - 1)])
                               : d - static_cast<float>(key));
            },
            f));
        // (the cap is in the scores where there is one: f is then 1)
        weigh_block<T, true>(z0, f.p0, st.base(), st.l, st.le);
        weigh_block<T, true>(z1, f.p0, st.base(), st.l, st.le);
        const int vaddr = vt + G::lane_v(lane, l32, hf);
        pv_block<T, D>(vaddr, z0, st.o);
        pv_block<T, D>(vaddr + 32 * G::kRow, z1, st.o);
      }
      __syncthreads();  // K and V are read
    }
    if (cleaned) {
#pragma unroll 1
      for (int j = 0; j < n; ++j)
        add_not_finite_row<T, D>(static_cast<const T*>(p.v_new) +
                                     (static_cast<int64_t>(row0 + j) * a.hkv + kvh) * D + 4 * hf,
                                 (seen_of(j & ~(kKeys - 1)) >> (j % kKeys)) & 1, st.o);
    }
    if (live) {
      const float l = half_sum(st.l), le = half_sum(st.le);
      const int64_t at = static_cast<int64_t>(row0 + token) * a.hq + h;
      const bool whole = s0 == 0 && s1 == steps;
      const int64_t slot =
          (2 * static_cast<int64_t>(group) + (s0 == 0)) * Wide::kRows + 32 * wave + l32;
      if (hf == 0) {
        if (!whole)
          p.part_ml[slot] = float4{st.m, l, le, 0.f};
        else if (p.lse != nullptr)
          p.lse[at] = log_sum(st.m, le);
      }
      const float inv = inverse(l);
#pragma unroll
      for (int db = 0; db < D / 32; ++db)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int dim = 32 * db + 8 * i + 4 * hf;
          const float o[4] = {st.o[db][4 * i], st.o[db][4 * i + 1], st.o[db][4 * i + 2],
                              st.o[db][4 * i + 3]};
          if (whole)
            store_row(static_cast<T*>(p.out) + at * D + dim, o, inv);
          else
            *reinterpret_cast<f32x4*>(p.part_o + slot * D + dim) = f32x4{o[0], o[1], o[2], o[3]};
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

hipError_t launch_codes_wide(const CacheAttnArgs& a, int head_dim, hipStream_t stream) {
  const auto launch = [&](auto dim, auto pages, auto cap, auto bias) {
    hipLaunchKernelGGL((codes_wide_kernel<decltype(dim)::value, decltype(pages)::value,
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
    if ((1 << a.c.page_shift) >= kKeys)
      of(dim, std::integral_constant<int, 1>{});
    else
      of(dim, std::integral_constant<int, kGroups>{});
  };
  if (head_dim == 128)
    with_pages(std::integral_constant<int, 128>{});
  else
    with_pages(std::integral_constant<int, 64>{});
  return hipGetLastError();
}

}  // namespace sift
