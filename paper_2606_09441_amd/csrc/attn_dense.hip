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
// += V(t)^T P(t) while it caps S(t + 1) and takes its maxima; K runs a tile
// ahead of V.  The order inside both halves is laid down by hand.
//  * kCap: the polynomial of the tanh where no score of the wavefront's tile is
//    large, the exact form apart where one is.
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
  // tiles that this wavefront computes
  const int mine = (w.last - w.first + kKeys - 1) / kKeys;
  bool cleaned = false;

  // The cap on scores of which none is large, or (1, 0, ..) nothing at all.
  struct Poly {
    float a0, a1, a2, a3, a4;
    __device__ __forceinline__ float operator()(float z) const {
      const float y = z * z;
      return z * fmaf(y, fmaf(y, fmaf(y, fmaf(y, a4, a3), a2), a1), a0);
    }
  };
  // A tile's exponents are c s + slope_key key + at, less the reference.
  struct Form {
    float c, slope_key, at;
  };
  const int lo = w.r0 + 32 * w.wave;  // this wavefront's rows: lo .. lo + 31
  // Tile t has keys before and after rows of this wavefront.
  const auto mixed = [&](int t) {
    const int j0 = w.first + t * kKeys;
    return kBias && j0 + kKeys - 1 > lo && j0 < lo + 31;
  };
  const auto masked = [&](int t) { return w.first + (t + 1) * kKeys > w.mine; };
  const auto form = [&](int t) {
    Form f{kCap ? 1.f : a.sc.c, 0.f, 0.f};
    if constexpr (kBias) {
      const int j0 = w.first + t * kKeys;
      const float d = static_cast<float>(w.tok - j0 - 4 * w.hf);
      f.slope_key = j0 < lo ? slope : -slope;
      f.at = -f.slope_key * d;
      if (mixed(t)) f = Form{1.f, 0.f, 0.f};  // odd_tile has the bias in the scores
    }
    return f;
  };
  // The bound of a tile from its largest score.
  const auto bound = [&](int t, const Form& f, float mx) {
    mx = half_max(mx) * f.c;
    if constexpr (kBias) {
      // the smallest distance to a key of the tile
      const int j0 = w.first + t * kKeys;
      if (f.slope_key > 0.f) mx -= slope * static_cast<float>(w.tok - j0 - (kKeys - 1));
      if (f.slope_key < 0.f) mx -= slope * static_cast<float>(j0 - w.tok);
    }
    return mx;
  };
  const auto any_large = [&](const f32x16& s0, const f32x16& s1) {
    if constexpr (!kCap) return false;
    float big = 0.f;
#pragma unroll
    for (int v = 0; v < 16; ++v) big = fmaxf(big, fmaxf(fabsf(s0[v]), fabsf(s1[v])));
    return __builtin_amdgcn_ballot_w64(big * a.sc.x > kTanhSmall) != 0;
  };
  const auto cap_exactly = [&](f32x16& s0, f32x16& s1) {
#pragma unroll
    for (int v = 0; v < 16; ++v) {
      s0[v] = cap_any(a.sc, s0[v]);
      s1[v] = cap_any(a.sc, s1[v]);
    }
  };
  // The bias of tiles that have keys on both sides of a row, and the mask, on
  // tile t's capped scores; returns their maximum.
  const auto odd_tile = [&](int t, f32x16& s0, f32x16& s1) {
    const int j0 = w.first + t * kKeys;
    if (mixed(t)) {
      const float c = kCap ? 1.f : a.sc.c;
      const float d = static_cast<float>(w.tok - j0 - 4 * w.hf);
#pragma unroll
      for (int v = 0; v < 16; ++v) {
        const float e = d - static_cast<float>(key_of(v));
        s0[v] = fmaf(s0[v], c, -slope * fabsf(e));
        s1[v] = fmaf(s1[v], c, -slope * fabsf(e - 32.f));
      }
    }
    if (masked(t)) {
      const uint64_t bits = w.bits(j0);
      mask_block(s0, static_cast<uint32_t>(bits >> (4 * w.hf)));
      mask_block(s1, static_cast<uint32_t>(bits >> (32 + 4 * w.hf)));
    }
    return fmaxf(block_max(s0), block_max(s1));
  };

  // The weight of score e (0 .. 31) of a tile, with its neighbour, into pb.
  bf16x8 pb[4];
  const auto weigh = [&](int e, const f32x16& s0, const f32x16& s1, const Form& f, float base,
                         float& sum, float& le) {
    const int i = e >> 3, v = 8 * (i & 1) + (e & 7);
    float x0 = i < 2 ? s0[v] : s1[v], x1 = i < 2 ? s0[v + 1] : s1[v + 1];
    float b0 = -base, b1 = -base;
    if constexpr (kBias) {
      const int key = key_of(v) + (i < 2 ? 0 : 32);
      b0 = fmaf(f.slope_key, static_cast<float>(key), f.at - base);
      b1 = fmaf(f.slope_key, static_cast<float>(key + 1), f.at - base);
    }
    const float p0 = __builtin_amdgcn_exp2f(fmaf(x0, f.c, b0));
    const float p1 = __builtin_amdgcn_exp2f(fmaf(x1, f.c, b1));
    const bf16x2 pp = bf16x2{static_cast<__bf16>(p0), static_cast<__bf16>(p1)};
    pb[i][e & 7] = pp[0];
    pb[i][(e & 7) + 1] = pp[1];
    sum = __builtin_amdgcn_fdot2_f32_bf16(pp, ones, sum, false);
    if constexpr (kLse) le += p0 + p1;
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

  // step t: S(t) in c0, c1 with form f; leaves S(t + 1) in n0, n1
  Form f;
  const auto step = [&](int t, f32x16& c0, f32x16& c1, f32x16& n0, f32x16& n1) {
    const int par = t & 1;
    // addresses made anew in every step: kept, each would hold a register
    asm volatile("" : "+v"(kaddr), "+v"(vaddr), "+v"(koff), "+v"(voff));
    if (t + 1 < w.tiles) stage<T, D, true>(a, w, t + 1, lds0 + (2 + (par ^ 1)) * kTile, voff);
    if (t + 2 < w.tiles) stage<T, D, false>(a, w, t + 2, lds0 + par * kTile, koff);
    if (w.mixed(w.first + t * kKeys)) cleaned |= clean_tile<T, D>(lds0 + (2 + par) * kTile);
    if (t < mine) {
      // (past the last tile a body like the others: its scores go nowhere)
      const bool more = t + 1 < mine;
      qk_and_weigh((par ^ 1) * kTile, n0, n1, c0, c1, f);
      f = form(t + 1);
      Poly poly{a.sc.a[0], a.sc.a[1], a.sc.a[2], a.sc.a[3], a.sc.a[4]};
      if constexpr (kCap) {
        if (any_large(n0, n1)) {
          cap_exactly(n0, n1);
          poly = Poly{1.f, 0.f, 0.f, 0.f, 0.f};
        }
      }
      float mx = -INFINITY;
      pv_and(par * kTile, [&](int i) {
#pragma unroll
        for (int u = 0; u < kDone; ++u) {
          const int e = i * kDone + u;
          f32x16& n = e < 16 ? n0 : n1;
          if constexpr (kCap) n[e & 15] = poly(n[e & 15]);
          mx = fmaxf(mx, n[e & 15]);
        }
      });
      if (more && (masked(t + 1) || mixed(t + 1))) mx = odd_tile(t + 1, n0, n1);
      st.rescale(more ? bound(t + 1, f, mx) : -INFINITY);
    }
    wait_vm<0>();
    __syncthreads();
  };

  stage<T, D, false>(a, w, 0, lds0, koff);
  stage<T, D, true>(a, w, 0, lds0 + 2 * kTile, voff);
  if (w.tiles > 1) stage<T, D, false>(a, w, 1, lds0 + kTile, koff);
  wait_vm<0>();
  __syncthreads();
  f32x16 a0{}, a1{}, b0{}, b1{};
  if (mine > 0) {
    a0 = qk_block<T, D>(kaddr, 0, q);
    a1 = qk_block<T, D>(kaddr, 1, q);
    f = form(0);
    if constexpr (kCap) cap_exactly(a0, a1);
    st.rescale(bound(0, f, odd_tile(0, a0, a1)));
  }
  __syncthreads();  // K slot 0 is refilled by step 0
  for (int t = 0; t < w.tiles; t += 2) {
    step(t, a0, a1, b0, b1);
    if (t + 1 < w.tiles) step(t + 1, b0, b1, a0, a1);
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
