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

#include "flash.h"
#include "sift_internal.h"

namespace sift {
namespace {

using namespace flash;

constexpr int kKeys = 64;   // of a tile

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
__device__ __forceinline__ void stage(const DenseArgs& a, const Row& w, int t, int slot, int off0) {
  using G = Tile<T, D>;
  const int k0 = w.first + t * kKeys + 16 * w.wave;
  const int stride = a.hkv * G::kRow;
  dma_rows<T, D, kV>(
      slot + w.wave * 16 * G::kRow,
      rows_rsrc(reinterpret_cast<unsigned long long>(kV ? a.v : a.k) +
                    (static_cast<int64_t>(k0) * a.hkv + w.kvh) * G::kRow,
                min(16, w.kend - k0), stride, G::kRow),
      off0, stride);
}

// A V tile at LDS address `tile` whose keys some rows of the record see and others
// do not: a weight of 0 times an infinity would be a NaN in rows that do not see
// the key, so the places that are not finite are taken out (and put right at the
// end, see add_not_finite).  All wavefronts call this; returns whether there
// were any.
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

// Adds what clean_tile took out to the rows that see it.
template <typename T, int D>
__device__ __forceinline__ void add_not_finite(const DenseArgs& a, const Row& w,
                                               f32x16 (&o)[D / 32]) {
  const T* v = static_cast<const T*>(a.v) + static_cast<int64_t>(w.kvh) * D + 4 * w.hf;
#pragma unroll 1
  for (int j = w.first + (w.all - w.first) / kKeys * kKeys; j < w.kend; ++j) {
    const T* row = v + static_cast<int64_t>(j) * a.hkv * D;
    const bool sees = j < w.upto || j <= w.tok;
#pragma unroll
    for (int db = 0; db < D / 32; ++db)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const float x = static_cast<float>(row[32 * db + key_of(i)]);
        if (sees && !(fabsf(x) < INFINITY)) o[db][i] += x;
      }
  }
}

template <typename T, int D, bool kLse>
__device__ __forceinline__ void finish(const DenseArgs& a, const Row& w, const RowState<D>& st) {
  if (!w.live) return;
  const float l = half_sum(st.l);
  const float inv = l > 0.f ? 1.f / l : l == l ? 0.f : l;
  const int64_t at = static_cast<int64_t>(w.tok) * a.hq + w.h;
  if constexpr (kLse) {
    const float le = half_sum(st.le);
    if (w.hf == 0) a.lse[at] = le > 0.f ? fmaf(st.m, kLn2, logf(le)) : le == le ? -INFINITY : le;
  }
  T* dst = static_cast<T*>(a.out) + at * D + 4 * w.hf;
#pragma unroll
  for (int db = 0; db < D / 32; ++db)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const f32x4 y = f32x4{st.o[db][4 * i] * inv, st.o[db][4 * i + 1] * inv,
                            st.o[db][4 * i + 2] * inv, st.o[db][4 * i + 3] * inv};
      if constexpr (Tile<T, D>::kBf16)
        *reinterpret_cast<bf16x4*>(dst + 32 * db + 8 * i) =
            bf16x4{static_cast<__bf16>(y[0]), static_cast<__bf16>(y[1]), static_cast<__bf16>(y[2]),
                   static_cast<__bf16>(y[3])};
      else
        *reinterpret_cast<f32x4*>(dst + 32 * db + 8 * i) = y;
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
    score_block(a.sc, slope, dist, s0);
    score_block(a.sc, slope, dist - 32.f, s1);
    if (j0 + kKeys > w.mine) {
      mask_block(s0, static_cast<uint32_t>(bits >> (4 * w.hf)));
      mask_block(s1, static_cast<uint32_t>(bits >> (32 + 4 * w.hf)));
    }
    st.rescale(half_max(fmaxf(block_max(s0), block_max(s1))) * c);
    weigh_block<T, kLse>(s0, c, st.base(), st.l, st.le);
    weigh_block<T, kLse>(s1, c, st.base(), st.l, st.le);
    pv_block<T, D>(vaddr + slot, s0, st.o);
    pv_block<T, D>(vaddr + slot + 32 * G::kRow, s1, st.o);
  }
  if (cleaned) add_not_finite<T, D>(a, w, st.o);
  finish<T, D, kLse>(a, w, st);
}

// bf16, software-pipelined: in step t the scores S(t + 1) = K(t + 1) Q^T are
// formed on the matrix cores while the VALU makes the weights of S(t), then O
// += V(t)^T P(t) while it takes the maxima of S(t + 1); K runs a tile ahead of V.  The order inside both halves is laid down by hand.
//  * kCap: the tanh as a polynomial of the product where none of the wavefront's
//    tile is large, folded into the exponent's FMA; the exact form apart where
//    one is.  The cap keeps the order, so the maxima are those of the products.
//  * kBias: outside the diagonal the distance is linear in the key, so that the
//    bias is one more FMA with a constant, folded into the exponent; the tile's
//    bound stands in for its maximum (its largest product at the smallest
//    distance), which only has to be near and not below.
template <int D, bool kCap, bool kBias, bool kLse>
__global__ __launch_bounds__(256, 2) void attn_dense_bf16_kernel(DenseArgs a) {
  using T = __bf16;
  using G = Tile<T, D>;
  constexpr int kTile = kKeys * G::kRow;
  constexpr int kSteps = G::kSteps;         // of QK^T: 16 dims each
  constexpr int kEach = 32 / kSteps;        // scores of S(t) that go with one
  constexpr int kPv = 4 * (D / 32);         // matrix instructions of PV
  constexpr int kDone = 32 / kPv;           // scores of S(t + 1) that go with one
  __shared__ __attribute__((aligned(1024))) uint8_t smem[4 * kTile];
  int rec, h;
  place(a, rec, h);
  if (rec >= a.num_recs) return;
  Row w;
  w.load(a, rec, h);
  QFrag<T, D> q;
  q.load(static_cast<const T*>(a.q) + (static_cast<int64_t>(w.tok) * a.hq + w.h) * D, w.hf, w.live);
  const int lds0 = static_cast<int>(reinterpret_cast<size_t>((lds_u8*)smem));
  int kaddr = lds0 + G::lane_k(w.l32, w.hf);
  int vaddr = lds0 + 2 * kTile + G::lane_v(w.lane, w.l32, w.hf);
  int koff = G::template dma_lane<false>(w.lane, a.hkv * G::kRow);
  int voff = G::template dma_lane<true>(w.lane, a.hkv * G::kRow);
  const float slope = kBias ? a.sc.slopes[w.h] * kLog2e : 0.f;
  const bf16x2 ones = bf16x2{static_cast<__bf16>(1.f), static_cast<__bf16>(1.f)};

  RowState<D> st;
  st.clear();
  // tiles that this wavefront computes: the first ones (with a bias they do not
  // come in order, and it takes all, some of them masked)
  const int mine = kBias && w.last > w.first ? w.tiles : (w.last - w.first + kKeys - 1) / kKeys;
  bool cleaned = false;

  // A tile's exponents are cap(z) + slope_key key + at, less the reference.  The
  // cap is z p(z^2) with these coefficients: the tanh's where no product of the
  // wavefront's tile is large, (1, 0, ..) where the scores are capped already.
  struct Form {
    float p0, p1, p2, p3;  // without kCap: p0 alone, the scale
    float slope_key, at;
  };
  const int lo = w.r0 + 32 * w.wave;  // this wavefront's rows: lo .. lo + 31
  // Tile t has keys before and after rows of this wavefront.
  const auto around = [&](int t) {
    const int j0 = w.first + t * kKeys;
    return kBias && j0 + kKeys - 1 > lo && j0 < lo + 31;
  };
  const auto masked = [&](int t) { return w.first + (t + 1) * kKeys > w.mine; };
  const auto capped = [&](const Form& f, float z) {
    if constexpr (!kCap) return z * f.p0;
    const float y = z * z;
    return z * fmaf(y, fmaf(y, fmaf(y, f.p3, f.p2), f.p1), f.p0);
  };
  // Masked scores: -inf, or where z p(z^2) has to stay a number one that no score
  // comes near (|capped score| <= kMaxCap log2(e)).
  constexpr float kOut = kCap ? -1e18f : -INFINITY;
  // Tile t's form, given the largest and the smallest product of each row; the
  // scores in place where the tile is odd (a large product, keys around the
  // row, a mask).  Returns the row's bound: its largest product's score at the
  // smallest distance of the tile.
  const auto take = [&](int t, f32x16& s0, f32x16& s1, float mx, float mn, Form& f) {
    const int j0 = w.first + t * kKeys;
    f = Form{kCap ? a.sc.b[0] : a.sc.c, a.sc.b[1], a.sc.b[2], a.sc.b[3], 0.f, 0.f};
    bool large = false;
    if constexpr (kCap) {
      large = __builtin_amdgcn_ballot_w64(fmaxf(mx, -mn) * a.sc.x > kTanhSmallBf16) != 0;
      if (large) {
#pragma unroll
        for (int v = 0; v < 16; ++v) {
          s0[v] = cap_any(a.sc, s0[v]);
          s1[v] = cap_any(a.sc, s1[v]);
        }
        mx = cap_any(a.sc, mx);
        f.p0 = 1.f;
        f.p1 = f.p2 = f.p3 = 0.f;
      }
    }
    if (masked(t) || around(t)) {
      const float d = static_cast<float>(w.tok - j0 - 4 * w.hf);
      const uint64_t bits = w.bits(j0);
      const uint32_t m0 = static_cast<uint32_t>(bits >> (4 * w.hf));
      const uint32_t m1 = static_cast<uint32_t>(bits >> (32 + 4 * w.hf));
      mx = -INFINITY;
#pragma unroll
      for (int v = 0; v < 16; ++v) {
        float x0 = s0[v], x1 = s1[v];
        if constexpr (kCap || kBias) {
          x0 = capped(f, x0);
          x1 = capped(f, x1);
        }
        if constexpr (kBias) {
          x0 = fmaf(-slope, fabsf(d - static_cast<float>(key_of(v))), x0);
          x1 = fmaf(-slope, fabsf(d - static_cast<float>(key_of(v) + 32)), x1);
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
    if (mx > -INFINITY) mx = capped(f, mx);
    if constexpr (kBias) {
      const float dist = static_cast<float>(w.tok - j0);
      f.slope_key = j0 < lo ? slope : -slope;
      f.at = -f.slope_key * (dist - static_cast<float>(4 * w.hf));
      mx -= slope * (j0 < lo ? dist - static_cast<float>(kKeys - 1) : -dist);
    }
    return mx;
  };

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
      if constexpr (kBias)
        b = fmaf(f.slope_key, static_cast<float>(key_of(v + u) + (i < 2 ? 0 : 32)), f.at - base);
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
  const auto qk_and_weigh = [&](int slot, f32x16& n0, f32x16& n1, const f32x16& c0,
                                const f32x16& c1, const Form& f) {
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

  // Tile of step i.  With a bias from the last row's own tile back, then on: the
  // reference, which the near keys set, then hardly moves.
  const int mid = min(w.tiles - 1, (w.r0 + w.rows - 1 - w.first) / kKeys);
  const auto tile = [&](int i) { return !kBias ? i : i <= mid ? mid - i : i; };

  // step i: its tile's scores in c0, c1 with form f; leaves the next in n0, n1
  Form f;
  const auto step = [&](int i, f32x16& c0, f32x16& c1, f32x16& n0, f32x16& n1) {
    const int par = i & 1;
    // addresses made anew in every step: kept, each would hold a register
    asm volatile("" : "+v"(kaddr), "+v"(vaddr), "+v"(koff), "+v"(voff));
    if (i + 1 < w.tiles) stage<T, D, true>(a, w, tile(i + 1), lds0 + (2 + (par ^ 1)) * kTile, voff);
    if (i + 2 < w.tiles) stage<T, D, false>(a, w, tile(i + 2), lds0 + par * kTile, koff);
    if (w.mixed(w.first + tile(i) * kKeys))
      cleaned |= clean_tile<T, D>(lds0 + (2 + par) * kTile);
    if (i < mine) {
      // (past the last tile a body like the others: its scores go nowhere)
      qk_and_weigh((par ^ 1) * kTile, n0, n1, c0, c1, f);
      float mx = -INFINITY, mn = INFINITY;
      pv_and(par * kTile, [&](int e) {
#pragma unroll
        for (int u = 0; u < kDone; u += 2) {
          const int v = (e * kDone + u) & 15;
          const f32x16& n = e * kDone < 16 ? n0 : n1;
          mx = fmaxf(fmaxf(mx, n[v]), n[v + 1]);
          if constexpr (kCap) mn = fminf(fminf(mn, n[v]), n[v + 1]);
        }
      });
      if (i + 1 < mine) st.rescale(take(tile(i + 1), n0, n1, mx, mn, f));
    }
    wait_vm<0>();
    __syncthreads();
  };

  stage<T, D, false>(a, w, tile(0), lds0, koff);
  stage<T, D, true>(a, w, tile(0), lds0 + 2 * kTile, voff);
  if (w.tiles > 1) stage<T, D, false>(a, w, tile(1), lds0 + kTile, koff);
  wait_vm<0>();
  __syncthreads();
  f32x16 a0{}, a1{}, b0{}, b1{};
  if (mine > 0) {
    a0 = qk_block<T, D>(kaddr, 0, q);
    a1 = qk_block<T, D>(kaddr, 1, q);
    float mx = -INFINITY, mn = INFINITY;
#pragma unroll
    for (int v = 0; v < 16; ++v) {
      mx = fmaxf(fmaxf(mx, a0[v]), a1[v]);
      mn = fminf(fminf(mn, a0[v]), a1[v]);
    }
    st.rescale(take(tile(0), a0, a1, mx, mn, f));
  }
  __syncthreads();  // K slot 0 is refilled by step 0
  for (int i = 0; i < w.tiles; i += 2) {
    step(i, a0, a1, b0, b1);
    if (i + 1 < w.tiles) step(i + 1, b0, b1, a0, a1);
  }
  if (cleaned) add_not_finite<T, D>(a, w, st.o);
  finish<T, D, kLse>(a, w, st);
}

}  // namespace

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
    if (!bf16) {
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
