// Tiles of e4m3 codes in LDS, and how lanes read them as bf16 operands: every code, times
// any power of two of a scale's, is a bf16 number, so nothing is lost.  K's scale goes to
// the scores, V's power of two into the conversion, and what is left of V's to the weights.  (The 8-bit matrix instructions, which would take K's codes as
// they are beside queries split in two, add with too few bits: off by 2^-13 of the sum of
// the products' sizes, as measured over 64 of them, where fp32 allows 2^-24 each.)
#pragma once

#include "clamp.h"
#include "flash.h"

namespace sift {
namespace flash {

typedef __attribute__((address_space(3))) u32x2 lds_u32x2;
typedef int i32x2 __attribute__((ext_vector_type(2)));
typedef __attribute__((address_space(3))) i32x2 lds_i32x2;

// Eight codes as bf16, times a power of two.
__device__ __forceinline__ bf16x8 code_values(u32x2 v, float power = 1.f) {
  bf16x8 x;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const uint32_t w = v[i];
    const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, power, false);
    const bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, power, true);
    x[4 * i] = a[0];
    x[4 * i + 1] = a[1];
    x[4 * i + 2] = b[0];
    x[4 * i + 3] = b[1];
  }
  return x;
}

// Rows of D codes, their 16-byte chunks XORed with the row, as Tile's.
template <int D>
struct CodeTile {
  static constexpr int kRow = D;                // bytes of a row: 64 or 128
  static constexpr int kChunks = kRow / 16;
  static constexpr int kDmaRows = 1024 / kRow;  // rows of one DMA instruction
  static constexpr int kGroupDmas = 16 / kDmaRows;
  static constexpr int kPairs = D / 32;         // 32 dims: a chunk of each lane half

  // Sixteen lanes read whole chunks of K, one of a row: eight rows meet all banks.
  static __device__ __forceinline__ int swz_k(int row) {
    return kRow == 128 ? (row >> 1) & 7 : (row >> 1) & 3;
  }
  // Thirty-two lanes read two neighbouring chunks of V rows 0-3 and 8-11 (+ 4, + 16).
  static __device__ __forceinline__ int swz_v(int row) {
    return kRow == 128 ? 2 * ((row >> 1) & 1) + 4 * ((row >> 3) & 1) : 2 * ((row >> 3) & 1);
  }
  template <bool kV>
  static __device__ __forceinline__ int dma_lane(int lane, int stride) {
    const int row = lane / kChunks;
    return row * stride + 16 * ((lane % kChunks) ^ (kV ? swz_v(row) : swz_k(row)));
  }
  template <bool kV>
  static __device__ __forceinline__ int dma_off(int off0, int j, int stride) {
    const int row = j * kDmaRows;
    return (off0 ^ (16 * (kV ? swz_v(row) : swz_k(row)))) + row * stride;
  }
  // DMA of 16 rows into LDS at `lds`, the resource's from row `from` (a multiple of 16) on.
  template <bool kV>
  static __device__ __forceinline__ void dma_rows(int lds, const i32x4& rs, int off0, int stride,
                                                  int from = 0) {
#pragma unroll
    for (int j = 0; j < kGroupDmas; ++j)
      dma_b128(lds + j * 1024, dma_off<kV>(off0, j, stride) + from * stride, rs);
  }

  // A operands of S^T: chunk 2 u + hf of row l32, dims 32 u + 16 hf and on, the first
  // eight for one matrix instruction, the others for the next.
  static __device__ __forceinline__ int lane_k(int l32, int hf) {
    return l32 * kRow + 16 * (hf ^ swz_k(l32));
  }
  static __device__ __forceinline__ u32x4 k_chunk(int addr, int u) {
    return *reinterpret_cast<const lds_u32x4*>(static_cast<size_t>(addr ^ (u << 5)));
  }

  // A operand of O^T += V^T P^T: the transposing read of eight rows of 16 codes, which
  // gives lane i of 16 the i-th codes.  Its rows are the weights' keys of this lane half:
  // 16 st + 4 hf + 0..3, and 8 more.
  static __device__ __forceinline__ int lane_v(int lane, int hf) {
    const int z = (lane & 15) >> 1;
    const int row = 4 * hf + (z & 3) + 8 * (z >> 2);
    return row * kRow + 16 * (((lane >> 4) & 1) ^ swz_v(row)) + 8 * (lane & 1);
  }
  static __device__ __forceinline__ u32x2 v_codes(int addr, int db, int st) {
    const i32x2 v = __builtin_amdgcn_ds_read_tr8_b64_v2i32(reinterpret_cast<lds_i32x2*>(
        static_cast<size_t>((addr ^ (db << 5)) + 16 * st * kRow)));
    return __builtin_bit_cast(u32x2, v);
  }
};

// Q operand for CodeTile's order of the dims: lane holds dims 32 u + 16 hf + 8 j and on
// of its row, for matrix instruction 2 u + j.
template <int D>
struct CodeQ {
  u32x4 x[D / 16];
  __device__ __forceinline__ void load(const __bf16* row, int hf, bool live) {
#pragma unroll
    for (int s = 0; s < D / 16; ++s) {
      x[s] = u32x4{0u, 0u, 0u, 0u};
      if (live)
        x[s] = *reinterpret_cast<const u32x4*>(row + 32 * (s >> 1) + 16 * hf + 8 * (s & 1));
    }
  }
};

// S^T of 32 keys: codes; addr includes lane_k.
template <int D>
__device__ __forceinline__ f32x16 qk_codes(int addr, const CodeQ<D>& q) {
  f32x16 s = f32x16{};
#pragma unroll
  for (int u = 0; u < CodeTile<D>::kPairs; ++u) {
    const u32x4 c = CodeTile<D>::k_chunk(addr, u);
    s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(code_values(u32x2{c[0], c[1]}),
                                                __builtin_bit_cast(bf16x8, q.x[2 * u]), s, 0, 0, 0);
    s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(code_values(u32x2{c[2], c[3]}),
                                                __builtin_bit_cast(bf16x8, q.x[2 * u + 1]), s, 0,
                                                0, 0);
  }
  return s;
}

// The same of a bf16 tile (Tile's layout) at LDS address `tile`.
template <int D>
__device__ __forceinline__ f32x16 qk_beside_codes(int tile, int l32, int hf, const CodeQ<D>& q) {
  using G = Tile<__bf16, D>;
  const int addr = tile + l32 * G::kRow + 16 * ((2 * hf) ^ G::swz_k(l32));
  f32x16 s = f32x16{};
#pragma unroll
  for (int i = 0; i < D / 16; ++i)
    s = dot_step<__bf16>(*reinterpret_cast<const lds_u32x4*>(static_cast<size_t>(
                             addr ^ (16 * (4 * (i >> 1) + (i & 1))))),
                         q.x[i], s);
  return s;
}

// V's scale of a page.  Its power of two goes to the codes, as far as 2^100, where they are
// finite bf16 numbers yet; the rest, from 1 to 2 and with scales above that to 2^20, is a
// factor of the weights, there part of the exponent: 2^(s - (base + lift)).  So the weights
// are of the sizes that they have without a scale: with all of it in the exponent those
// beside a scale of 2^-100 vanished from 2^-26 on, from the sums too, and beside 2^120 they
// came to infinity.
struct ValueScale {
  float power, lift, undo;  // undo: one over the rest
  __device__ __forceinline__ void set(float scale) {
    const uint32_t s = __builtin_bit_cast(uint32_t, usable_scale(scale));
    const uint32_t e = min(s & 0xff800000u, (100u + 127u) << 23);
    power = __builtin_bit_cast(float, e);
    const float rest =  // (times one over the power)
        __builtin_bit_cast(float, s) * __builtin_bit_cast(float, (254u << 23) - e);
    lift = -__builtin_amdgcn_logf(rest);
    undo = __builtin_amdgcn_rcpf(rest);
  }
};

// O^T += V^T P^T over 32 keys at LDS address addr (lane_v included); power: of V's scales,
// of each 16 keys.
template <int D>
__device__ __forceinline__ void pv_codes(int addr, const f32x16& p, const float (&power)[2],
                                         f32x16 (&o)[D / 32]) {
#pragma unroll
  for (int st = 0; st < 2; ++st) {
    bf16x8 b;
#pragma unroll
    for (int i = 0; i < 8; ++i) b[i] = static_cast<__bf16>(p[8 * st + i]);
#pragma unroll
    for (int db = 0; db < D / 32; ++db)
      o[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
          code_values(CodeTile<D>::v_codes(addr, db, st), power[st]), b, o[db], 0, 0, 0);
  }
}

// Weights of 32 keys of two groups of 16, times what is left of their V scales:
// 2^(c_i s - base_i), where base_i holds the lift.  l and le as weigh_block's: sums of the
// weights alone.
__device__ __forceinline__ void weigh_codes(f32x16& s, const float (&c)[2], const float (&base)[2],
                                            const float (&undo)[2], float& l, float& le) {
  const bf16x2 ones = bf16x2{static_cast<__bf16>(1.f), static_cast<__bf16>(1.f)};
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    float sum = 0.f, a = 0.f, b = 0.f;
#pragma unroll
    for (int v = 8 * i; v < 8 * i + 8; v += 2) {
      s[v] = __builtin_amdgcn_exp2f(fmaf(s[v], c[i], -base[i]));
      s[v + 1] = __builtin_amdgcn_exp2f(fmaf(s[v + 1], c[i], -base[i]));
      const bf16x2 p = bf16x2{static_cast<__bf16>(s[v]), static_cast<__bf16>(s[v + 1])};
      sum = __builtin_amdgcn_fdot2_f32_bf16(p, ones, sum, false);
      a += s[v];
      b += s[v + 1];
    }
    l = fmaf(sum, undo[i], l);
    le = fmaf(a + b, undo[i], le);
  }
}

}  // namespace flash
}  // namespace sift
