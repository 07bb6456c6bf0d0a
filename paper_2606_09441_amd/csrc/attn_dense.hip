// Dense attention of a plan's prompts with transformed scores: capped by a
// tanh, biased by distance, under a causal, a document or a prefix mask.
//
//   s(i, j) = cap tanh(scale q_i.k_j / cap) - slope |i - j|
//   out_i   = sum_j exp(s - lse_i) v_j,  lse_i = log sum_j exp(s),  j visible to i
//
// Every mask leaves a row one run of keys: a record of 128 rows of a segment
// (rows r0 .., of one head: a workgroup of four wavefronts) walks the keys
// from `first` to its last row, or to `upto` (the end of the prompt's
// documents under the prefix mask) where that is later; key j is visible to
// row i where j < upto or j <= i.  64-key tiles of K and V go through two LDS
// slots each, brought by DMA while the tile before is computed; one barrier a
// tile.  Only tiles at the diagonal are masked.
//
// Records run longest first, and those of the query heads that share a kv
// head on one XCD (launch_attn_dense), so that its L2 holds their keys.

#include <algorithm>

#include "flash_pipe.h"
#include "sift_internal.h"

namespace sift {
namespace {

using namespace flash;

// Workgroup -> record and head, XCD blockIdx % 8 (see dense_grid).
__device__ __forceinline__ void place(const DenseArgs& a, int& rec, int& h) {
  const int g = a.hq / a.hkv, x = blockIdx.x % kNumXcd, i = blockIdx.x / kNumXcd;
  if (a.hkv % kNumXcd == 0) {
    const int per = a.hkv / kNumXcd * g;
    rec = i / per;
    h = (x + kNumXcd * (i % per / g)) * g + i % g;
  } else if (kNumXcd % a.hkv == 0) {
    const int per = kNumXcd / a.hkv;
    rec = i / g * per + x / a.hkv;
    h = x % a.hkv * g + i % g;
  } else {
    rec = blockIdx.x / a.hq;
    h = blockIdx.x % a.hq;
  }
}

// A workgroup's record and this lane's row.
struct Row {
  int r0, rows, first, upto, kend, tiles;
  int h, kvh;
  int lane, wave, l32, hf;
  int tok;          // row
  bool live;
  // keys before `all` are visible to every row of the record, those before
  // `mine` to every row of this wavefront; those from `last` on to none of it
  int all, mine, last;
  __device__ __forceinline__ void load(const DenseArgs& a, int rec, int head) {
    const int4 r = a.recs[rec];
    r0 = uniform(r.x);
    rows = uniform(r.y);
    first = uniform(r.z);
    upto = uniform(r.w);
    h = uniform(head);
    kvh = h / (a.hq / a.hkv);
    lane = threadIdx.x & 63;
    wave = uniform(threadIdx.x >> 6);
    l32 = lane & 31;
    hf = lane >> 5;
    const int row = wave * 32 + l32;
    live = row < rows;
    tok = r0 + row;
    kend = max(r0 + rows, upto);
    tiles = (kend - first + kKeys - 1) / kKeys;
    all = max(upto, r0 + 1);
    mine = max(upto, r0 + 32 * wave + 1);
    last = 32 * wave >= rows ? first : max(upto, min(r0 + rows, r0 + 32 * wave + 32));
  }
  // Whether rows of the record differ in what they see of the tile from j0 on.
  __device__ __forceinline__ bool mixed(int j0) const { return j0 + kKeys > all && upto < kend; }
  // One bit a key of the tile from j0 on: those this row sees.
  __device__ __forceinline__ uint64_t bits(int j0) const {
    return live ? low_bits(max(upto, tok + 1) - j0) : 0;
  }
};

// This wavefront's 16 rows of a 64-key tile, K or V, to LDS address `slot`; off0:
// dma_lane.
template <typename T, int D, bool kV>
__device__ __forceinline__ i32x4 tile_rows(const DenseArgs& a, const Row& w, int t) {
  using G = Tile<T, D>;
  const int k0 = w.first + t * kKeys + 16 * w.wave;
  return rows_rsrc(reinterpret_cast<unsigned long long>(kV ? a.v : a.k) +
                       (static_cast<int64_t>(k0) * a.hkv + w.kvh) * G::kRow,
                   min(16, w.kend - k0), a.hkv * G::kRow, G::kRow);
}
template <typename T, int D, bool kV>
__device__ __forceinline__ void stage(const DenseArgs& a, const Row& w, int t, int slot, int off0) {
  using G = Tile<T, D>;
  dma_rows<T, D, kV>(slot + w.wave * 16 * G::kRow, tile_rows<T, D, kV>(a, w, t), off0,
                     a.hkv * G::kRow);
}

// Adds what clean_tile took out to the rows that see it.
template <typename T, int D>
__device__ __forceinline__ void add_not_finite(const DenseArgs& a, const Row& w,
                                               f32x16 (&o)[D / 32]) {
  const T* v = static_cast<const T*>(a.v) + static_cast<int64_t>(w.kvh) * D + 4 * w.hf;
#pragma unroll 1
  for (int j = w.first + (w.all - w.first) / kKeys * kKeys; j < w.kend; ++j) {
    add_not_finite_row<T, D>(v + static_cast<int64_t>(j) * a.hkv * D, j < w.upto || j <= w.tok, o);
  }
}

template <typename T, int D, bool kLse>
__device__ __forceinline__ void finish(const DenseArgs& a, const Row& w, const RowState<D>& st) {
  if (!w.live) return;
  const float inv = inverse(half_sum(st.l));
  const int64_t at = static_cast<int64_t>(w.tok) * a.hq + w.h;
  if constexpr (kLse) {
    const float le = half_sum(st.le);
    if (w.hf == 0) a.lse[at] = log_sum(st.m, le);
  }
  T* dst = static_cast<T*>(a.out) + at * D + 4 * w.hf;
#pragma unroll
  for (int db = 0; db < D / 32; ++db)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float o[4] = {st.o[db][4 * i], st.o[db][4 * i + 1], st.o[db][4 * i + 2],
                          st.o[db][4 * i + 3]};
      store_row(dst + 32 * db + 8 * i, o, inv);
    }
}

// fp32: the matrix instructions take 16 times as long as bf16's and bound it, so
// a tile's steps simply follow each other.
template <int D, bool kLse>
__global__ __launch_bounds__(256, D == 64 ? 2 : 1) void attn_dense_f32_kernel(DenseArgs a) {
  using T = float;
  using G = Tile<T, D>;
  constexpr int kTile = kKeys * G::kRow;  // bytes
  // K slots 0 and 1, V slots 0 and 1
  __shared__ __attribute__((aligned(1024))) uint8_t smem[4 * kTile];
  int rec, h;
  place(a, rec, h);
  if (rec >= a.num_recs) return;
  Row w;
  w.load(a, rec, h);
  QFrag<T, D> q;
  q.load(static_cast<const T*>(a.q) + (static_cast<int64_t>(w.tok) * a.hq + w.h) * D, w.hf, w.live);
  const int lds0 = static_cast<int>(reinterpret_cast<size_t>((lds_u8*)smem));
  const int kaddr = lds0 + G::lane_k(w.l32, w.hf);
  const int vaddr = lds0 + 2 * kTile + G::lane_v(w.lane, w.l32, w.hf);
  const float slope = a.sc.slopes != nullptr ? a.sc.slopes[w.h] * kLog2e : 0.f;
  const float c = score_factor(a.sc);
  const int koff = G::template dma_lane<false>(w.lane, a.hkv * G::kRow);
  const int voff = G::template dma_lane<true>(w.lane, a.hkv * G::kRow);
  const auto both = [&](int t) {
    stage<T, D, false>(a, w, t, lds0 + (t & 1) * kTile, koff);
    stage<T, D, true>(a, w, t, lds0 + (2 + (t & 1)) * kTile, voff);
  };
  RowState<D> st;
  st.clear();
  bool cleaned = false;
  both(0);
  for (int t = 0; t < w.tiles; ++t) {
    wait_vm<0>();
    __syncthreads();  // tile t is there, and every wavefront is done with tile t - 1
    if (t + 1 < w.tiles) both(t + 1);
    const int j0 = w.first + t * kKeys;
    const int slot = (t & 1) * kTile;
    const uint64_t bits = w.bits(j0);
    if (w.mixed(j0)) cleaned |= clean_tile<T, D>(lds0 + 2 * kTile + slot);
    if (j0 >= w.last) continue;
    f32x16 s0 = qk_block<T, D>(kaddr + slot, 0, q);
    f32x16 s1 = qk_block<T, D>(kaddr + slot, 1, q);
    const float dist = static_cast<float>(w.tok - j0 - 4 * w.hf);
    if (a.sc.x != 0.f) {
      cap_scores(a.sc, s0);
      cap_scores(a.sc, s1);
    }
    if (j0 + kKeys > w.mine) {
      mask_block(s0, static_cast<uint32_t>(bits >> (4 * w.hf)));
      mask_block(s1, static_cast<uint32_t>(bits >> (32 + 4 * w.hf)));
    }
    float off = 0.f;
    if (a.sc.slopes != nullptr) {
      const auto far0 = [&](int v) { return fabsf(dist - static_cast<float>(key_of(v))); };
      const auto far1 = [&](int v) { return fabsf(dist - static_cast<float>(32 + key_of(v))); };
      off = half_max(fmaxf(largest_bias(s0, slope, far0), largest_bias(s1, slope, far1)));
      if (off == -INFINITY) off = 0.f;
      add_bias(a.sc, s0, slope, off, far0);
      add_bias(a.sc, s1, slope, off, far1);
    }
    st.rescale(fmaf(half_max(fmaxf(block_max(s0), block_max(s1))), c, off));
    weigh_block<T, kLse>(s0, c, st.base() - off, st.l, st.le);
    weigh_block<T, kLse>(s1, c, st.base() - off, st.l, st.le);
    pv_block<T, D>(vaddr + slot, s0, st.o);
    pv_block<T, D>(vaddr + slot + 32 * G::kRow, s1, st.o);
  }
  if (cleaned) add_not_finite<T, D>(a, w, st.o);
  finish<T, D, kLse>(a, w, st);
}

// The record's tiles as the pipeline takes them (flash_pipe.h).  kBias: outside the
// diagonal the distance is linear in the key, so that the bias is one more FMA with
// a constant, folded into the exponent.  The tile's bound then is its largest product
// with its largest bias, of two keys maybe: above the largest score by the range of
// the biases at most.  What it is above, all weights lose, so where that range passes
// kMostAbove (slopes beyond 0.88) the largest score itself is found, an FMA and a
// maximum a score more (16.6K tokens, 32/8 heads, prefix mask: 4.2 -> 4.65 ms, capped
// 5.0 -> 6.2).  With 2^-80 lost a row's weights down to 2^-46 of its largest remain
// normal numbers.
constexpr float kMostAbove = 80.f;
template <int D, bool kCap, bool kBias>
struct DenseTiles {
  using T = __bf16;
  const DenseArgs& a;
  const Row& w;
  float slope;
  int steps, mine;
  int lo;   // this wavefront's rows: lo .. lo + 31
  int mid;  // the last row's own tile
  bool steep;
  bool cleaned = false;
  __device__ __forceinline__ DenseTiles(const DenseArgs& args, const Row& row)
      : a(args), w(row), slope(kBias ? args.sc.slopes[row.h] * kLog2e : 0.f), steps(row.tiles),
        lo(row.r0 + 32 * row.wave) {
    // (with a bias the tiles do not come in order, and every wavefront takes all,
    // some of them masked)
    mine = kBias && w.last > w.first ? steps : (w.last - w.first + kKeys - 1) / kKeys;
    mid = min(steps - 1, (w.r0 + w.rows - 1 - w.first) / kKeys);
    steep = fabsf(slope) * static_cast<float>(kKeys - 1) > kMostAbove;
  }
  // Tile of step i.  With a bias from the last row's own back, then on: the
  // reference, which the near keys set, then hardly moves.
  __device__ __forceinline__ int tile(int i) const { return !kBias ? i : i <= mid ? mid - i : i; }
  template <bool kV>
  __device__ __forceinline__ i32x4 rows(int i) const {
    return tile_rows<T, D, kV>(a, w, tile(i));
  }
  __device__ __forceinline__ void clean(int i, int lds) {
    if (w.mixed(w.first + tile(i) * kKeys)) cleaned |= clean_tile<T, D>(lds);
  }
  __device__ __forceinline__ float take(int i, f32x16& s0, f32x16& s1, float mx, float mn,
                                        Form& f) const {
    const int j0 = w.first + tile(i) * kKeys;
    const bool masked = j0 + kKeys > w.mine;
    const bool around = kBias && j0 + kKeys - 1 > lo && j0 < lo + 31;  // a row inside the tile
    const float d = static_cast<float>(w.tok - j0 - 4 * w.hf);
    mx = take_tile<kCap, kBias>(
        a.sc, s0, s1, mx, mn, masked || around, [&] { return w.bits(j0); }, w.hf, slope,
        [&](int key) { return fabsf(d - static_cast<float>(key)); }, f);
    if constexpr (kBias) {
      if (!masked && !around) {
        const float dist = static_cast<float>(w.tok - j0);
        f.slope_key = j0 < lo ? slope : -slope;
        f.d = d;
        if (steep) {
          mx = -INFINITY;
#pragma unroll
          for (int v = 0; v < 16; ++v)
            mx = fmaxf(mx, fmaxf(fmaf(f.slope_key, static_cast<float>(key_of(v)),
                                      capped<kCap>(f, s0[v])),
                                 fmaf(f.slope_key, static_cast<float>(key_of(v) + 32),
                                      capped<kCap>(f, s1[v]))));
          mx = half_max(fmaf(-f.slope_key, d, mx));
        } else {
          // the distances run from |dist| to |dist - 63|; slopes may be negative
          mx += fmaxf(-slope * fabsf(dist), -slope * fabsf(dist - static_cast<float>(kKeys - 1)));
        }
      }
    }
    return mx;
  }
};

// (D = 128 with bias and log sums: two registers of a lane are spilled)
template <int D, bool kCap, bool kBias, bool kLse>
__global__ __launch_bounds__(256, 2) void attn_dense_bf16_kernel(DenseArgs a) {
  using T = __bf16;
  __shared__ __attribute__((aligned(1024))) uint8_t smem[4 * kKeys * Tile<T, D>::kRow];
  int rec, h;
  place(a, rec, h);
  if (rec >= a.num_recs) return;
  Row w;
  w.load(a, rec, h);
  QFrag<T, D> q;
  q.load(static_cast<const T*>(a.q) + (static_cast<int64_t>(w.tok) * a.hq + w.h) * D, w.hf, w.live);
  RowState<D> st;
  st.clear();
  DenseTiles<D, kCap, kBias> src(a, w);
  run_pipe<D, kCap, kBias, kLse>(src, q, st, smem, w.lane, a.hkv * Tile<T, D>::kRow);
  if (src.cleaned) add_not_finite<T, D>(a, w, st.o);
  finish<T, D, kLse>(a, w, st);
}

// Few records: 32 rows a workgroup (blockIdx.y of the record's four), whose keys its
// wavefronts share out, 32 at a time through LDS of their own, as in cache_attn.hip:
// sixteen times the wavefronts, each with a quarter of the steps.
template <typename T, int D>
__global__ __launch_bounds__(256, sizeof(T) * D > 256 ? 1 : 2) void attn_dense_small_kernel(DenseArgs a) {
  using G = Tile<T, D>;
  constexpr int kOwn = 32;  // keys of a wavefront's tile
  constexpr int kTile = kOwn * G::kRow;
  constexpr int kDmas = 2 * G::kGroupDmas;  // of a K or V tile
  __shared__ __attribute__((aligned(1024))) uint8_t smem[4 * 2 * kTile];
  __shared__ float part[4][32][3];
  int rec, h;
  place(a, rec, h);
  if (rec >= a.num_recs) return;
  const int4 r = a.recs[rec];
  const int r0 = uniform(r.x) + 32 * static_cast<int>(blockIdx.y);
  const int rows = min(32, uniform(r.x) + uniform(r.y) - r0);
  if (rows <= 0) return;
  h = uniform(h);
  const int first = uniform(r.z);
  // keys that all rows of the record see: up to the record's own first (causal),
  // which is before this workgroup's
  const bool prefix = uniform(r.w) > uniform(r.x);
  const int upto = prefix ? uniform(r.w) : r0;
  const int kend = max(r0 + rows, upto);
  const int kvh = h / (a.hq / a.hkv);
  const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6);
  const int l32 = lane & 31, hf = lane >> 5;
  const int tok = r0 + l32;
  const bool live = l32 < rows;
  const int stride = a.hkv * G::kRow;
  QFrag<T, D> q;
  q.load(static_cast<const T*>(a.q) + (static_cast<int64_t>(tok) * a.hq + h) * D, hf, live);
  const int lds0 = static_cast<int>(reinterpret_cast<size_t>((lds_u8*)smem));
  const int kt = lds0 + wave * 2 * kTile, vt = kt + kTile;
  const int kaddr = kt + G::lane_k(l32, hf), vaddr = vt + G::lane_v(lane, l32, hf);
  const int koff = G::template dma_lane<false>(lane, stride);
  const int voff = G::template dma_lane<true>(lane, stride);
  const float slope = a.sc.slopes != nullptr ? a.sc.slopes[h] * kLog2e : 0.f;
  const float c = score_factor(a.sc);
  const int tiles = (kend - first + kOwn - 1) / kOwn;
  const auto fetch = [&](int t, auto v) {
    constexpr bool kV = decltype(v)::value;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int k0 = first + t * kOwn + 16 * i;
      dma_rows<T, D, kV>((kV ? vt : kt) + i * 16 * G::kRow,
                         rows_rsrc(reinterpret_cast<unsigned long long>(kV ? a.v : a.k) +
                                       (static_cast<int64_t>(k0) * a.hkv + kvh) * G::kRow,
                                   min(16, kend - k0), stride, G::kRow),
                         kV ? voff : koff, stride);
    }
  };
  RowState<D> st;
  st.clear();
  int t = wave;
  if (t < tiles) {
    fetch(t, std::false_type{});
    fetch(t, std::true_type{});
  }
  for (; t < tiles; t += 4) {
    const bool more = t + 4 < tiles;
    wait_vm<kDmas>();  // K is there, V may still be on its way
    f32x16 s = qk_block<T, D>(kaddr, 0, q);
    wait_lds();        // K is read
    if (more) fetch(t + 4, std::false_type{});
    const int j0 = first + t * kOwn;
    const uint32_t bits =
        live ? static_cast<uint32_t>(low_bits(max(upto, tok + 1) - j0)) : 0u;
    if (a.sc.x != 0.f) cap_scores(a.sc, s);
    if (__builtin_amdgcn_ballot_w64(bits != ~0u)) mask_block(s, bits >> (4 * hf));
    float off = 0.f;
    if (a.sc.slopes != nullptr) {
      const float dist = static_cast<float>(tok - j0 - 4 * hf);
      const auto far = [&](int v) { return fabsf(dist - static_cast<float>(key_of(v))); };
      off = half_max(largest_bias(s, slope, far));
      if (off == -INFINITY) off = 0.f;
      add_bias(a.sc, s, slope, off, far);
    }
    st.rescale(fmaf(half_max(block_max(s)), c, off));
    weigh_block<T, true>(s, c, st.base() - off, st.l, st.le);
    if (more)
      wait_vm<kDmas>();  // V is there, the next K may not be
    else
      wait_vm<0>();
    if (j0 + kOwn > max(upto, r0 + 1) && upto < kend)
      mend_own_tile<T, D>(vt, bits, lane, st.o);
    pv_block<T, D>(vaddr, s, st.o);
    wait_lds();        // V is read
    if (more) fetch(t + 4, std::true_type{});
  }
  merge_waves<D>(st, kt, lds0, 2 * kTile, part, wave, l32, hf,
                 [&](int row, int dim, const float(&o)[4], float top, float l, float le) {
                   if (row >= rows) return;
                   const int64_t at = static_cast<int64_t>(r0 + row) * a.hq + h;
                   store_row(static_cast<T*>(a.out) + at * D + dim, o, inverse(l));
                   if (dim == 0 && a.lse != nullptr) a.lse[at] = log_sum(top, le);
                 });
}

}  // namespace

// Workgroups of 128 rows up to which those of 32 rows run instead: the card is not
// full, so what counts is how long one takes.  us of 128 / 32 rows (causal, bf16 D =
// 128, then fp32 D = 64): 6 workgroups 11.8 / 8.1, 25.8 / 11.6; 136: 45 / 30, 156 /
// 77; 264: 86 / 73, 315 / 205; but 224 of a short prompt 19.3 / 20.0, 544: 59 / 82,
// 216 / 194.  (One limit for both types, where bf16's lies; fp32's own lies higher.)
constexpr int64_t kDenseFew = 256;

int64_t dense_grid(int32_t num_recs, int32_t hq, int32_t hkv) {
  const int64_t n = num_recs;
  if (hkv % kNumXcd == 0 || kNumXcd % hkv != 0) return n * hq;
  const int64_t per = kNumXcd / hkv;  // XCDs of a kv head, records dealt over them
  return (n + per - 1) / per * (hq / hkv) * kNumXcd;
}

hipError_t launch_attn_dense(const DenseArgs& a, bool bf16, int head_dim, hipStream_t stream) {
  const int64_t grid = dense_grid(a.num_recs, a.hq, a.hkv);
  if (grid == 0) return hipSuccess;
  if (grid >= int64_t(1) << 24) return hipErrorInvalidValue;  // fewer than 2^32 threads
  const dim3 g(static_cast<unsigned>(grid)), b(256);
  const bool small = grid <= kDenseFew;
  using F = std::false_type;
  using Y = std::true_type;
  const auto launch = [&](auto dim) {
    constexpr int D = decltype(dim)::value;
    const auto with = [&](auto cap, auto bias, auto lse) {
      hipLaunchKernelGGL((attn_dense_bf16_kernel<D, decltype(cap)::value, decltype(bias)::value,
                                                 decltype(lse)::value>),
                         g, b, 0, stream, a);
    };
    const auto scored = [&](auto cap, auto bias) {
      if (a.lse != nullptr)
        with(cap, bias, Y{});
      else
        with(cap, bias, F{});
    };
    if (small) {
      const dim3 sub(g.x, kDenseRows / 32);
      if (bf16)
        hipLaunchKernelGGL((attn_dense_small_kernel<__bf16, D>), sub, b, 0, stream, a);
      else
        hipLaunchKernelGGL((attn_dense_small_kernel<float, D>), sub, b, 0, stream, a);
    } else if (!bf16) {
      if (a.lse != nullptr)
        hipLaunchKernelGGL((attn_dense_f32_kernel<D, true>), g, b, 0, stream, a);
      else
        hipLaunchKernelGGL((attn_dense_f32_kernel<D, false>), g, b, 0, stream, a);
    } else if (a.sc.x != 0.f) {
      if (a.sc.slopes != nullptr)
        scored(Y{}, Y{});
      else
        scored(Y{}, F{});
    } else if (a.sc.slopes != nullptr) {
      scored(F{}, Y{});
    } else {
      scored(F{}, F{});
    }
  };
  if (head_dim == 128)
    launch(std::integral_constant<int, 128>{});
  else
    launch(std::integral_constant<int, 64>{});
  return hipGetLastError();
}

}  // namespace sift
