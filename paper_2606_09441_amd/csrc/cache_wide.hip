// The attention of many new tokens over a paged cache (bf16): units of 128 rows of
// a (sequence, kv head), 32 of each wavefront, which share the 64-key tiles of the
// pipeline (flash_pipe.h).  With hundreds of rows to a key (64 drafted tokens, 6
// query heads) the products are what there is to do, not the bytes.  The tiles of all
// units form one list, cut into equal runs, as in cache_attn.hip, whose merge this
// shares.  64 tokens, 48/8 heads, D = 128 over 66048 slots: 143 us, 730 TFLOP/s, the
// MFMAs busy in 37% of the SIMDs' cycles, the VALU in 42%: runs of 48 tiles a
// workgroup, and the instances of D = 128 spill 120 to 148 bytes of registers a lane.

#include "cache.h"
#include "flash_pipe.h"
#include "sift_internal.h"

namespace sift {
namespace {

using namespace cache;

// Steps s0 .. of a unit.
template <int D, bool kCap, bool kBias>
struct CacheTiles {
  using T = __bf16;
  using G = Tile<T, D>;
  const CacheAttnArgs& p;
  int b, len, n, row0, kvh;
  int ct;            // tiles of cached keys
  int s0, steps, mine;
  int turn;          // its steps begin with the turn-th, and go round
  int wave, hf;
  int token;         // this lane's new token in its sequence
  bool live;
  float slope;
  int pos;
  bool cleaned = false;

  // (with a bias the near keys, which set the reference, come first)
  __device__ __forceinline__ int tile(int i) const {
    if constexpr (kBias) return s0 + steps - 1 - i;
    const int j = i + turn;
    return s0 + (j < steps ? j : j - steps);
  }
  template <bool kV>
  __device__ __forceinline__ i32x4 rows(int i) const {
    const CacheArgs& a = p.c;
    const int t = tile(i), j = (t - ct) * kKeys + 16 * wave;
    const Rows16 r = t < ct ? cached_rows(a, b, len, t * kKeys + 16 * wave)
                            : Rows16{static_cast<int64_t>(row0) + j, min(max(n - j, 0), 16)};
    const void* base = t < ct ? (kV ? a.v : a.k) : (kV ? p.v_new : p.k_new);
    return rows_rsrc(
        reinterpret_cast<unsigned long long>(base) + (r.row * a.hkv + kvh) * G::kRow, r.n,
        a.hkv * G::kRow, G::kRow);
  }
  __device__ __forceinline__ void clean(int i, int lds) {
    if (tile(i) >= ct) cleaned |= clean_tile<T, D>(lds);
  }
  // One bit a key of tile t: those this row sees.
  __device__ __forceinline__ uint64_t bits(int t) const {
    const CacheArgs& a = p.c;
    if (t < ct) {
      uint64_t m = low_bits(len - t * kKeys);
      if (a.page_lens != nullptr) {
        m = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i)
          m |= low_bits(cached_rows(a, b, len, t * kKeys + 16 * i).n) << (16 * i);
      }
      return m;
    }
    const int j0 = (t - ct) * kKeys;
    const uint64_t seen =
        p.tree_mask != nullptr
            ? p.tree_mask[static_cast<int64_t>(row0 + token) * p.mask_words + (t - ct)]
            : low_bits(token + 1 - j0);
    return seen & low_bits(n - j0);
  }
  __device__ __forceinline__ float take(int i, f32x16& s0_, f32x16& s1_, float mx, float mn,
                                        Form& f) const {
    const CacheArgs& a = p.c;
    const int t = tile(i);
    const uint64_t m = bits(t);
    const bool fresh = t >= ct;
    const int j0 = (fresh ? t - ct : t) * kKeys + 4 * hf;
    const int32_t* table = nullptr;  // of the keys' positions
    int last = 0;
    if constexpr (kBias) {
      const int slots = a.max_pages << a.page_shift;
      if (fresh && a.row_pos != nullptr) {
        table = a.row_pos + row0;
        last = n - 1;
      } else if (!fresh && a.key_pos != nullptr) {
        table = a.key_pos + (static_cast<int64_t>(b) * a.hkv + kvh) * slots;
        last = slots - 1;
      }
    }
    const float d = static_cast<float>(pos - (fresh ? len : 0) - j0);
    return take_tile<kCap, kBias>(
        a.sc, s0_, s1_, mx, mn, kBias || __builtin_amdgcn_ballot_w64(~m != 0) != 0, [&] { return m; }, hf,
        slope,
        [&](int key) {
          return fabsf(table != nullptr ? static_cast<float>(pos - table[min(j0 + key, last)])
                                        : d - static_cast<float>(key));
        },
        f);
  }
};

template <int D, bool kCap, bool kBias>
__global__ __launch_bounds__(256, 2) void cache_wide_kernel(CacheAttnArgs p) {
  using T = __bf16;
  using G = Tile<T, D>;
  __shared__ __attribute__((aligned(1024))) uint8_t smem[4 * kKeys * G::kRow];
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
    QFrag<T, D> q;
    q.load(static_cast<const T*>(a.q) + (static_cast<int64_t>(row0 + token) * a.hq + h) * D, hf,
           live);
    RowState<D> st;
    st.clear();
    // The first step is one whose number is a multiple of the runs' length: units of the
    // same keys, whose runs do not begin at the same ones, then read each tile at about
    // the same time, so that all but one find it in the L2 (us of the call without /
    // with it: 22 drafted tokens over 66048 slots, 48/8 heads 114 / 103, 64 161 / 160;
    // 8 sequences of 8192 slots, 64 tokens each 204 / 188).
    const int over = s0 - Split::quotient(s0, run) * run;
    const int turn = over > 0 ? run - over : 0;
    CacheTiles<D, kCap, kBias> src{p,
                                   b,
                                   len,
                                   n,
                                   row0,
                                   kvh,
                                   uniform(cost.cached_tiles(s)),
                                   s0,
                                   s1 - s0,
                                   r0 + 32 * wave < n * g ? s1 - s0 : 0,
                                   turn < s1 - s0 ? turn : 0,
                                   wave,
                                   hf,
                                   token,
                                   live,
                                   kBias ? a.sc.slopes[h] * kLog2e : 0.f,
                                   kBias ? (a.row_pos != nullptr ? a.row_pos[row0 + token] : len + token)
                                         : 0};
    run_pipe<D, kCap, false, true>(src, q, st, smem, lane, a.hkv * G::kRow);
    if (src.cleaned) {
#pragma unroll 1
      for (int j = 0; j < n; ++j)
        add_not_finite_row<T, D>(
            static_cast<const T*>(p.v_new) +
                (static_cast<int64_t>(row0 + j) * a.hkv + kvh) * D + 4 * hf,
            (src.bits(src.ct + j / kKeys) >> (j % kKeys)) & 1, st.o);
    }
    if (live) {
      const float l = half_sum(st.l), le = half_sum(st.le);
      const int64_t at = static_cast<int64_t>(row0 + token) * a.hq + h;
      const bool whole = s0 == 0 && s1 == steps;
      const int64_t slot = (2 * static_cast<int64_t>(group) + (s0 == 0)) * Wide::kRows + 32 * wave + l32;
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

hipError_t launch_cache_wide(const CacheAttnArgs& a, int head_dim, hipStream_t stream) {
  const dim3 g(a.groups), b(256);
  const auto launch = [&](auto dim) {
    constexpr int D = decltype(dim)::value;
    if (a.c.sc.x != 0.f) {
      if (a.c.sc.slopes != nullptr)
        hipLaunchKernelGGL((cache_wide_kernel<D, true, true>), g, b, 0, stream, a);
      else
        hipLaunchKernelGGL((cache_wide_kernel<D, true, false>), g, b, 0, stream, a);
    } else if (a.c.sc.slopes != nullptr) {
      hipLaunchKernelGGL((cache_wide_kernel<D, false, true>), g, b, 0, stream, a);
    } else {
      hipLaunchKernelGGL((cache_wide_kernel<D, false, false>), g, b, 0, stream, a);
    }
  };
  if (head_dim == 128)
    launch(std::integral_constant<int, 128>{});
  else
    launch(std::integral_constant<int, 64>{});
  return hipGetLastError();
}

}  // namespace sift
