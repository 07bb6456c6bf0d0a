// Attention of every sequence's new tokens (one, a chain, a drafted tree) over
// its paged cache and over each other.
//
// A unit is 32 rows of a (sequence, kv head): row r is new token r / g and query
// head r % g of the g that share the kv head, so that a key is read once for
// all of them.  Its keys are tiles of 32, the cached ones first, then the new
// ones; all cached keys are visible to all rows, of the new ones those of the
// row's mask.  Few rows and long caches: HBM bounds it, so what counts is even
// and continuous reading.
//  * The tiles of all units, four to a step, form one list, cut into equal runs
//    for a fixed number of workgroups, whatever the lengths (which only the
//    device knows).  A unit that one workgroup has whole is written by it; of
//    the others every workgroup leaves its part (not normalised, with reference
//    max and sums), and a second launch merges them in workgroup order.
//  * The four wavefronts of a workgroup take the four tiles of a step, each
//    through LDS of its own (16 KB at bf16, D = 128): no barriers inside a run.
//    K of the next tile is fetched as soon as K is read, V likewise, so that
//    each wavefront always has about a tile's half in flight, 128 KB a CU.

#include <algorithm>

#include "cache.h"
#include "sift_internal.h"

namespace sift {
namespace {

using namespace cache;

constexpr int kTileKeys = Narrow::kTileKeys;
constexpr int kStepTiles = Narrow::kStepTiles;  // a tile for each wavefront
constexpr int kRows = Narrow::kRows;

template <typename T, int D>
__global__ __launch_bounds__(256, sizeof(T) * D > 256 ? 1 : 2) void cache_attn_kernel(CacheAttnArgs p) {
  using G = Tile<T, D>;
  constexpr int kTile = kTileKeys * G::kRow;
  constexpr int kDmas = 2 * G::kGroupDmas;  // of a K or V tile
  __shared__ __attribute__((aligned(1024))) uint8_t smem[4 * 2 * kTile];
  __shared__ float part[4][kRows][3];
  const CacheArgs& a = p.c;
  const int g = a.hq / a.hkv;
  const UnitCost<Narrow> cost{g, a.hkv};
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
  const int stride = a.hkv * G::kRow;
  const int lds0 = static_cast<int>(reinterpret_cast<size_t>((lds_u8*)smem));
  const int kt = lds0 + wave * 2 * kTile, vt = kt + kTile;  // this wavefront's tiles
  const int kaddr = kt + G::lane_k(l32, hf);
  const int vaddr = vt + G::lane_v(lane, l32, hf);
  const int koff = G::template dma_lane<false>(lane, stride);
  const int voff = G::template dma_lane<true>(lane, stride);
  const float c = score_factor(a.sc);

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
    QFrag<T, D> q;
    q.load(static_cast<const T*>(a.q) + (static_cast<int64_t>(row0 + node) * a.hq + h) * D, hf,
           live);
    const float slope = a.sc.slopes != nullptr ? a.sc.slopes[h] * kLog2e : 0.f;
    const int my_pos = a.sc.slopes == nullptr ? 0
                       : a.row_pos != nullptr ? a.row_pos[row0 + node]
                                              : len + node;

    struct TileRows {
      Rows16 r[2];
    };
    const auto rows_of = [&](int t) {
      TileRows x;
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int j = (t - ct) * kTileKeys + 16 * i;
        x.r[i] = t < ct ? cached_rows(a, b, len, t * kTileKeys + 16 * i)
                        : Rows16{static_cast<int64_t>(row0) + j, min(max(n - j, 0), 16)};
      }
      return x;
    };
    const auto fetch = [&](int t, const TileRows& x, auto v) {
      constexpr bool kV = decltype(v)::value;
      const void* base = t < ct ? (kV ? a.v : a.k) : (kV ? p.v_new : p.k_new);
#pragma unroll
      for (int i = 0; i < 2; ++i)
        dma_rows<T, D, kV>((kV ? vt : kt) + i * 16 * G::kRow,
                           rows_rsrc(reinterpret_cast<unsigned long long>(base) +
                                         (x.r[i].row * a.hkv + kvh) * G::kRow,
                                     x.r[i].n, stride, G::kRow),
                           kV ? voff : koff, stride);
    };

    RowState<D> st;
    st.clear();
    const int tend = min(tiles, s1 * kStepTiles);
    int t = s0 * kStepTiles + wave;
    TileRows rows{};
    if (t < tend) {
      rows = rows_of(t);
      fetch(t, rows, std::false_type{});
      fetch(t, rows, std::true_type{});
    }
    for (; t < tend; t += kStepTiles) {
      const bool more = t + kStepTiles < tend;
      // one bit a key: those this row sees
      uint32_t bits = static_cast<uint32_t>(low_bits(rows.r[0].n)) |
                      static_cast<uint32_t>(low_bits(rows.r[1].n)) << 16;
      if (more) rows = rows_of(t + kStepTiles);
      wait_vm<kDmas>();  // K is there, V may still be on its way
      f32x16 sc = qk_block<T, D>(kaddr, 0, q);
      wait_lds();        // K is read
      if (more) fetch(t + kStepTiles, rows, std::false_type{});
      const bool fresh = t >= ct;
      const int j0 = (fresh ? t - ct : t) * kTileKeys;
      if (fresh) {
        if (p.tree_mask != nullptr)
          bits &= static_cast<uint32_t>(
              p.tree_mask[static_cast<int64_t>(row0 + node) * p.mask_words + (j0 >> 6)] >>
              (j0 & 32));
        else
          bits &= static_cast<uint32_t>(low_bits(node + 1 - j0));
      }
      if (a.sc.x != 0.f) cap_scores(a.sc, sc);
      if (__builtin_amdgcn_ballot_w64(bits != ~0u)) mask_block(sc, bits >> (4 * hf));
      float off = 0.f;
      const auto bias = [&](auto far) {
        off = half_max(largest_bias(sc, slope, far));
        if (off == -INFINITY) off = 0.f;
        add_bias(a.sc, sc, slope, off, far);
      };
      if (a.sc.slopes != nullptr && (fresh ? a.row_pos : a.key_pos) != nullptr) {
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
      } else if (a.sc.slopes != nullptr) {
        const float d0 = static_cast<float>(my_pos - (fresh ? len : 0) - j0 - 4 * hf);
        bias([&](int v) { return fabsf(d0 - static_cast<float>(key_of(v))); });
      }
      st.rescale(fmaf(half_max(block_max(sc)), c, off));
      weigh_block<T, true>(sc, c, st.base() - off, st.l, st.le);
      if (more)
        wait_vm<kDmas>();  // V is there, the next K may not be
      else
        wait_vm<0>();
      if (fresh) mend_own_tile<T, D>(vt, live ? bits : 0u, lane, st.o);
      pv_block<T, D>(vaddr, sc, st.o);
      wait_lds();  // V is read
      if (more) fetch(t + kStepTiles, rows, std::true_type{});
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

// Merge of the parts of each (new token, query head), `each` of them a workgroup:
// eight groups of 32 lanes take every eighth part, lane l dims l D / 32 and on.
template <typename U, typename T, int D>
__global__ __launch_bounds__(256) void cache_merge_kernel(CacheAttnArgs p, int each) {
  const CacheArgs& a = p.c;
  constexpr int kDims = D / 32;
  __shared__ float acc[8][D];
  __shared__ float part[8][2];
  const int g = a.hq / a.hkv;
  const UnitCost<U> cost{g, a.hkv};
  const Work work(a, cost);
  const Split split(work.total, p.groups);
  if (split.total == 0) return;
  const int end = min(static_cast<int>(blockIdx.x + 1) * each, a.rows * a.hq);
  for (int item = blockIdx.x * each; item < end; ++item) {
    const int token = item / a.hq, h = item % a.hq;
    const Place pl = work.find_token(token);
    if (pl.b >= a.num_seqs) continue;  // no sequence's
    const Seq s = work.seq(pl.b);
    const int steps = uniform(cost.steps(s));
    const int r = (token - s.row0) * g + h % g;
    const int u0 = uniform(pl.at + (h / g * cost.blocks(s) + r / U::kRows) * steps);
    const int first = split.of(u0);
    const int n = split.of(u0 + steps - 1) - first + 1;
    if (n == 1) continue;  // written already
    // the first part is its workgroup's second, the others their workgroups' first
    const auto slot = [&](int i) {
      return (2 * static_cast<int64_t>(first + i) + (i == 0)) * U::kRows + r % U::kRows;
    };
    float top = -INFINITY;
    for (int i = threadIdx.x & 63; i < n; i += 64) top = fmaxf(top, p.part_ml[slot(i)].x);
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor(top, d));
    const int grp = threadIdx.x >> 5, l32 = threadIdx.x & 31;
    float l = 0.f, le = 0.f, o[kDims] = {};
#pragma unroll 4
    for (int i = grp; i < n; i += 8) {
      const float4 ml = p.part_ml[slot(i)];
      const float* src = p.part_o + slot(i) * D + l32 * kDims;
      const float wt = part_weight(ml.x, top);
      l += ml.y * wt;
      le += ml.z * wt;
#pragma unroll
      for (int e = 0; e < kDims; ++e) o[e] += src[e] * wt;
    }
    __syncthreads();  // the last item's sums are read
#pragma unroll
    for (int e = 0; e < kDims; ++e) acc[grp][l32 * kDims + e] = o[e];
    if (l32 == 0) {
      part[grp][0] = l;
      part[grp][1] = le;
    }
    __syncthreads();
    if (threadIdx.x >= D) continue;
    float y = 0.f;
    l = le = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      y += acc[i][threadIdx.x];
      l += part[i][0];
      le += part[i][1];
    }
    const int64_t at = static_cast<int64_t>(item) * D + threadIdx.x;
    static_cast<T*>(p.out)[at] = static_cast<T>(y * inverse(l));
    if (p.lse != nullptr && threadIdx.x == 0) p.lse[item] = log_sum(top, le);
  }
}

}  // namespace

// bf16 with more than 32 rows of a kv head goes by the wide units, whose 128 rows
// share what the workgroup reads and whose matrix work is pipelined, but whose
// workgroups take longer to start and to end: only where there are so many rows
// times cached keys.  us of narrow / wide, 8 kv heads, D = 128: 48 rows of 65536 keys
// 88 / 65, of 32768 48 / 46; 128 rows of 32768 59 / 54, of 16384 40 / 44; 256 rows of
// 16384 55 / 55, of 4096 29 / 38; 32 rows of 65536 54 / 61.
constexpr int64_t kNarrowMost = int64_t(24) << 20;
// e4m3: the narrow units read half as much, the wide ones turn codes into bf16 for fewer
// rows each.  us of narrow / wide at 48/8 heads: 64 tokens of 16384 slots 61 / 61, of 32768
// 115 / 92; 22 of 32768 50 / 61, of 65536 98 / 98; 32 of 65536 127 / 104; 8 sequences of
// 16384, 12 tokens each 148 / 109; 16 of 2048, 64 each 147 / 171.
constexpr int64_t kNarrowMostCodes = int64_t(48) << 20;

// Workgroups of the merge: as many as are resident at once, since where there are
// many items most have nothing to merge and a workgroup of its own costs more than
// they (us of the call with an item each / with 2048 workgroups: 256 sequences of
// 512 keys, 65536 items 299 / 218, 8192 items 133 / 125; up to 1024 items the same).
constexpr int64_t kMergeGroups = 2048;

bool cache_attn_wide(Pool pool, int64_t rows_of_kv, int64_t keys) {
  const int64_t most = pool == Pool::kE4m3 ? kNarrowMostCodes : kNarrowMost;
  return pool != Pool::kF32 && rows_of_kv > kRows && rows_of_kv >= (most + keys - 1) / keys;
}

int64_t cache_attn_steps(const CacheArgs& a, bool codes) {
  // as if every sequence had the most rows, which row pointers may say whatever they
  // add up to; of the narrow units: the wide ones are no more, and take twice the steps
  // where there are half as many
  const int64_t rows = std::min(a.rows, a.max_rows);
  const int64_t units = static_cast<int64_t>(a.num_seqs) * a.hkv *
                        ((rows * (a.hq / a.hkv) + kRows - 1) / kRows);
  const int64_t keys = (static_cast<int64_t>(a.max_pages) << a.page_shift) + rows + 4 * kTileKeys;
  const int64_t steps = keys / (kTileKeys * kStepTiles) + 1 + (codes ? NarrowCodes::kLead : 0);
  return units >= int64_t(1) << 31 ? units : units * steps;
}

hipError_t launch_cache_attn(const CacheAttnArgs& a, Pool pool, int head_dim, hipStream_t stream) {
  if (a.c.rows == 0) return hipSuccess;
  const int64_t items = static_cast<int64_t>(a.c.rows) * a.c.hq;
  if (items >= int64_t(1) << 24) return hipErrorInvalidValue;  // fewer than 2^32 threads
  const int64_t most = static_cast<int64_t>(std::min(a.c.rows, a.c.max_rows)) * (a.c.hq / a.c.hkv);
  const bool codes = pool == Pool::kE4m3;
  const bool wide = cache_attn_wide(
      pool, most, (static_cast<int64_t>(a.c.max_pages) << a.c.page_shift) * a.c.num_seqs * a.c.hkv);
  const auto launch = [&](auto elem, auto dim) {
    using T = decltype(elem);
    constexpr int D = decltype(dim)::value;
    // no more workgroups than are resident at once: most have nothing to merge where
    // there are many
    const int each = static_cast<int>((items + kMergeGroups - 1) / kMergeGroups);
    const dim3 grid(static_cast<unsigned>((items + each - 1) / each)), block(256);
    if constexpr (Tile<T, D>::kBf16) {
      if (wide) {
        const hipError_t e =
            codes ? launch_codes_wide(a, D, stream) : launch_cache_wide(a, D, stream);
        if (e != hipSuccess) return e;
        hipLaunchKernelGGL((cache_merge_kernel<Wide, T, D>), grid, block, 0, stream, a, each);
        return hipGetLastError();
      }
    }
    hipError_t e;
    if (codes) {
      e = launch_cache_codes(a, D, stream);
    } else {
      hipLaunchKernelGGL((cache_attn_kernel<T, D>), dim3(a.groups), block, 0, stream, a);
      e = hipGetLastError();
    }
    if (e != hipSuccess) return e;
    if (codes)
      hipLaunchKernelGGL((cache_merge_kernel<NarrowCodes, T, D>), grid, block, 0, stream, a, each);
    else
      hipLaunchKernelGGL((cache_merge_kernel<Narrow, T, D>), grid, block, 0, stream, a, each);
    return hipGetLastError();
  };
  using D64 = std::integral_constant<int, 64>;
  using D128 = std::integral_constant<int, 128>;
  if (pool != Pool::kF32)
    return head_dim == 128 ? launch(__bf16{}, D128{}) : launch(__bf16{}, D64{});
  return head_dim == 128 ? launch(float{}, D128{}) : launch(float{}, D64{});
}

}  // namespace sift
