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

template <typename T, int D, bool kLse>
__global__ __launch_bounds__(256, 2) void attn_dense_kernel(DenseArgs a) {
  using G = Tile<T, D>;
  constexpr int kTile = kKeys * G::kRow;  // bytes
  // K slots 0 and 1, V slots 0 and 1
  __shared__ __attribute__((aligned(1024))) uint8_t smem[4 * kTile];

  // workgroup -> record and head, XCD blockIdx % 8 (see launch_attn_dense)
  int rec, h;
  {
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
  if (rec >= a.num_recs) return;
  const int4 r = a.recs[rec];
  const int r0 = uniform(r.x), rows = uniform(r.y), first = uniform(r.z), upto = uniform(r.w);
  h = uniform(h);
  const int kvh = h / (a.hq / a.hkv);
  const int lane = threadIdx.x & 63;
  const int wave = uniform(threadIdx.x >> 6);
  const int l32 = lane & 31, hf = lane >> 5;
  const int row = wave * 32 + l32;
  const bool live = row < rows;
  const int tok = r0 + row;
  const int stride = a.hkv * G::kRow;

  QFrag<T, D> q;
  q.load(static_cast<const T*>(a.q) + (static_cast<int64_t>(tok) * a.hq + h) * D, hf, live);

  const int lds0 = static_cast<int>(reinterpret_cast<size_t>((lds_u8*)smem));
  const int kaddr = lds0 + G::lane_k(l32, hf);
  const int vaddr = lds0 + 2 * kTile + G::lane_v(lane, l32, hf);
  const int kend = max(r0 + rows, upto);
  const int tiles = (kend - first + kKeys - 1) / kKeys;
  const float slope = a.sc.slopes != nullptr ? a.sc.slopes[h] * kLog2e : 0.f;
  const float c = score_factor(a.sc);

  // this wavefront's 16 rows of tile t, K and V, into slot t % 2
  auto stage = [&](int t) {
    const int k0 = first + t * kKeys + 16 * wave;
    const int64_t off = (static_cast<int64_t>(k0) * a.hkv + kvh) * G::kRow;
    const int n = min(16, kend - k0);
    const int at = lds0 + (t & 1) * kTile + wave * 16 * G::kRow;
    dma_rows<T, D, false>(at, rows_rsrc(reinterpret_cast<unsigned long long>(a.k) + off, n, stride,
                                        G::kRow), lane, stride);
    dma_rows<T, D, true>(at + 2 * kTile, rows_rsrc(reinterpret_cast<unsigned long long>(a.v) + off,
                                                   n, stride, G::kRow), lane, stride);
  };

  RowState<D> st;
  st.clear();
  // keys before `all` are visible to every row of the record, those before
  // `mine` to every row of this wavefront; those from `last` on to none of it
  const int all = max(upto, r0 + 1), mine = max(upto, r0 + 32 * wave + 1);
  const int last = max(upto, min(r0 + rows, r0 + 32 * wave + 32));
  const bool idle = 32 * wave >= rows;

  stage(0);
  for (int t = 0; t < tiles; ++t) {
    wait_vm<0>();
    __syncthreads();  // tile t is there, and every wavefront is done with tile t - 1
    if (t + 1 < tiles) stage(t + 1);
    const int j0 = first + t * kKeys;
    const int slot = (t & 1) * kTile;
    const uint64_t bits = live ? low_bits(max(upto, tok + 1) - j0) : 0;
    if (j0 + kKeys > all && upto < kend) {
      // rows differ in what they see of V
      bool bad = false;
      for (int i = threadIdx.x; i < kTile / 16; i += 256)
        bad |= not_finite<T>(*reinterpret_cast<const lds_u32x4*>(
            static_cast<size_t>(lds0 + 2 * kTile + slot + 16 * i)));
      if (__syncthreads_or(bad)) {
        add_not_finite<T, D>(lds0 + 2 * kTile + slot, kKeys, bits, hf, st.o);
        __syncthreads();
        for (int i = threadIdx.x; i < kTile / 16; i += 256) {
          lds_u32x4* p =
              reinterpret_cast<lds_u32x4*>(static_cast<size_t>(lds0 + 2 * kTile + slot + 16 * i));
          *p = only_finite<T>(*p);
        }
        __syncthreads();
      }
    }
    if (idle || j0 >= last) continue;
    f32x16 s0 = qk_block<T, D>(kaddr + slot, 0, q);
    f32x16 s1 = qk_block<T, D>(kaddr + slot, 1, q);
    const float dist = static_cast<float>(tok - j0 - 4 * hf);
    score_block(a.sc, slope, dist, s0);
    score_block(a.sc, slope, dist - 32.f, s1);
    if (j0 + kKeys > mine) {
      mask_block(s0, static_cast<uint32_t>(bits >> (4 * hf)));
      mask_block(s1, static_cast<uint32_t>(bits >> (32 + 4 * hf)));
    }
    st.rescale(half_max(fmaxf(block_max(s0), block_max(s1))) * c);
    weigh_block<T, kLse>(s0, c, st.base(), st.l, st.le);
    weigh_block<T, kLse>(s1, c, st.base(), st.l, st.le);
    pv_block<T, D>(vaddr + slot, s0, st.o);
    pv_block<T, D>(vaddr + slot + 32 * G::kRow, s1, st.o);
  }

  if (!live) return;
  const float l = half_sum(st.l);
  const float inv = l > 0.f ? 1.f / l : l == l ? 0.f : l;
  const int64_t at = static_cast<int64_t>(tok) * a.hq + h;
  if constexpr (kLse) {
    const float le = half_sum(st.le);
    if (hf == 0) a.lse[at] = le > 0.f ? fmaf(st.m, kLn2, logf(le)) : le == le ? -INFINITY : le;
  }
  T* dst = static_cast<T*>(a.out) + at * D + 4 * hf;
#pragma unroll
  for (int db = 0; db < D / 32; ++db)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const f32x4 y = f32x4{st.o[db][4 * i] * inv, st.o[db][4 * i + 1] * inv,
                            st.o[db][4 * i + 2] * inv, st.o[db][4 * i + 3] * inv};
      if constexpr (G::kBf16)
        *reinterpret_cast<bf16x4*>(dst + 32 * db + 8 * i) =
            bf16x4{static_cast<__bf16>(y[0]), static_cast<__bf16>(y[1]), static_cast<__bf16>(y[2]),
                   static_cast<__bf16>(y[3])};
      else
        *reinterpret_cast<f32x4*>(dst + 32 * db + 8 * i) = y;
    }
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
  const auto launch = [&](auto elem, auto dim) {
    using T = decltype(elem);
    constexpr int D = decltype(dim)::value;
    if (a.lse != nullptr)
      hipLaunchKernelGGL((attn_dense_kernel<T, D, true>), g, b, 0, stream, a);
    else
      hipLaunchKernelGGL((attn_dense_kernel<T, D, false>), g, b, 0, stream, a);
  };
  using D64 = std::integral_constant<int, 64>;
  using D128 = std::integral_constant<int, 128>;
  if (bf16 && head_dim == 128)
    launch(__bf16{}, D128{});
  else if (bf16)
    launch(__bf16{}, D64{});
  else if (head_dim == 128)
    launch(float{}, D128{});
  else
    launch(float{}, D64{});
  return hipGetLastError();
}

}  // namespace sift
