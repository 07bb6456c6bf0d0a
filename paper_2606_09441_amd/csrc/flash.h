// Device pieces shared by the dense attention (attn_dense.hip) and the page
// cache's kernels (cache_attn.hip, cache_weights.hip), for bf16 and fp32
// inputs of head dimension 64 or 128.
//
// A wavefront owns 32 query rows.  S^T = K Q^T on 32x32 matrix instructions
// (keys on M, queries on N), so lanes l and l ^ 32 hold one query's scores:
// register v of a 32-key block holds key 8 (v / 4) + 4 hf + v % 4, hf = lane /
// 32.  That accumulator is the B operand of O^T += V^T P^T as it stands: for
// bf16 (32x32x16, rounded to bf16) with the keys of a k-step permuted, which
// the transposing LDS read of V follows; for fp32 (32x32x2) register v is the
// operand of the k-step of keys 8 (v / 4) + v % 4 and that + 4.
//
// K and V tiles lie in LDS as unpadded rows whose 16-byte chunks are XORed
// with the row (swz_k, swz_v), so that the operand reads are free of bank
// conflicts; the LDS DMA brings them, 16 bytes a lane, the swizzle applied to
// the global address.  A DMA goes through a buffer resource that ends at the
// last valid row of 16, so rows past it arrive as zeros and nothing outside
// the caller's rows is ever read.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "sift_internal.h"

namespace sift {

namespace flash {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) uint8_t lds_u8;
typedef __attribute__((address_space(3))) bf16x4 lds_bf16x4;
typedef __attribute__((address_space(3))) u32x4 lds_u32x4;
typedef __attribute__((address_space(3))) float lds_float;
typedef __attribute__((address_space(3))) f32x4 lds_f32x4;
typedef __attribute__((address_space(3))) int lds_int;
typedef __attribute__((address_space(3))) i32x4 lds_i32x4;

constexpr int kBufferWord3 = 0x00020000;  // gfx9-family raw buffer resource word 3
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

// The reference max of a row moves only when a tile exceeds it by this much
// (log2 units): weights stay <= 2^8, and their relative precision the same.
constexpr float kLazy = 8.0f;

__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }

__device__ __forceinline__ float half_max(float x) {
  float a = x, b = x;
  asm("s_nop 1\n\tv_permlane32_swap_b32 %0, %1\n\ts_nop 1" : "+v"(a), "+v"(b));
  return fmaxf(a, b);
}

__device__ __forceinline__ float half_sum(float x) {
  float a = x, b = x;
  asm("s_nop 1\n\tv_permlane32_swap_b32 %0, %1\n\ts_nop 1" : "+v"(a), "+v"(b));
  return a + b;
}

// Layout of a tile of rows of D values of T in LDS, and how lanes read it.
template <typename T, int D>
struct Tile {
  static constexpr bool kBf16 = std::is_same<T, __bf16>::value;
  static constexpr int kRow = D * static_cast<int>(sizeof(T));  // bytes of a row: 128, 256, 512
  static constexpr int kChunks = kRow / 16;
  static constexpr int kDmaRows = 1024 / kRow;                  // rows of one DMA instruction
  static constexpr int kGroupDmas = 16 / kDmaRows;              // instructions of 16 rows
  static constexpr int kSteps = kChunks / 2;  // pairs of chunks: a lane half takes one of each
  static constexpr int kBlocks = D / 32;      // 32-wide blocks of the head dimension

  static __device__ __forceinline__ int swz_k(int row) {
    return kRow == 128 ? (row >> 1) & 7 : row & 15;
  }
  static __device__ __forceinline__ int swz_v(int row) {
    if (!kBf16) return 8 * ((row >> 2) & 1);
    return kRow == 128 ? 4 * ((row >> 1) & 1) : 4 * (row & 3);
  }

  // Byte offset (from the first of 16 rows of a head, `stride` bytes apart) of
  // the 16 bytes that this lane brings in DMA instruction j of those rows: the
  // lane's offset for j = 0, its chunk XORed with the swizzle of row j kDmaRows
  // (of whose bits the row inside the instruction has none).
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

  // A operand of S^T: chunk 2 s + hf of row l32 of block kb.  lane_k is the
  // lane's address for s = 0 of block 0.
  static __device__ __forceinline__ int lane_k(int l32, int hf) {
    return l32 * kRow + 16 * (hf ^ swz_k(l32));
  }
  static __device__ __forceinline__ u32x4 k_frag(int addr, int kb, int s) {
    return *reinterpret_cast<const lds_u32x4*>(
        static_cast<size_t>((addr ^ (s << 5)) + kb * 32 * kRow));
  }

  // A operand of O^T += V^T P^T.  bf16: two transposing reads of 4-row blocks,
  // rows z + 4 hf (+ 8), z = (lane & 15) / 4, columns 32 db + 16 ((lane / 16) &
  // 1) + 4 (lane & 3) .. + 3.  fp32: element 32 db + l32 of key 8 (v / 4) +
  // 4 hf + v % 4.
  static __device__ __forceinline__ int lane_v(int lane, int l32, int hf) {
    if (!kBf16) return 4 * hf * kRow + 128 * hf + 4 * l32;
    const int z = (lane & 15) >> 2;
    const int chunk = (2 * ((lane >> 4) & 1) + ((lane & 3) >> 1)) ^ swz_v(z);
    return (z + 4 * hf) * kRow + 16 * chunk + 8 * (lane & 1);
  }
  static __device__ __forceinline__ bf16x8 v_frag(int addr, int db, int st) {
    const int a = (addr ^ (db << 6)) + 16 * st * kRow;
    const bf16x4 x = __builtin_amdgcn_ds_read_tr16_b64_v4bf16(
        reinterpret_cast<lds_bf16x4*>(static_cast<size_t>(a)));
    const bf16x4 y = __builtin_amdgcn_ds_read_tr16_b64_v4bf16(
        reinterpret_cast<lds_bf16x4*>(static_cast<size_t>(a + 8 * kRow)));
    return bf16x8{x[0], x[1], x[2], x[3], y[0], y[1], y[2], y[3]};
  }
  static __device__ __forceinline__ float v_elem(int addr, int db, int v) {
    return *reinterpret_cast<const lds_float*>(
        static_cast<size_t>((addr ^ (db << 7)) + (8 * (v >> 2) + (v & 3)) * kRow));
  }
  // LDS byte address, inside a tile, of element `dim` of row `row` of V.
  static __device__ __forceinline__ int v_at(int row, int dim) {
    const int byte = dim * static_cast<int>(sizeof(T));
    return row * kRow + 16 * ((byte >> 4) ^ swz_v(row)) + (byte & 15);
  }
};

// Global -> LDS, 16 bytes per lane from byte voff of the resource, landing at
// m0 + 16 * lane.  Waited for by hand (wait_vm): the compiler does not see it.
__device__ __forceinline__ void dma_b128(int m0, int voff, const i32x4& rs) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds"
               :
               : "s"(m0), "v"(voff), "s"(rs)
               : "memory", "m0");
}

template <int kLeft>
__device__ __forceinline__ void wait_vm() {
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(kLeft) : "memory");
}

__device__ __forceinline__ void wait_lds() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }

// Resource of `rows` (0 .. 16) rows of one head from address a on, `stride`
// bytes apart.
__device__ __forceinline__ i32x4 rows_rsrc(unsigned long long a, int rows, int stride, int row) {
  return i32x4{uniform(static_cast<int>(static_cast<unsigned>(a))),
               uniform(static_cast<int>((a >> 32) & 0xffff)),
               uniform(rows > 0 ? (rows - 1) * stride + row : 0), kBufferWord3};
}

// DMA of 16 rows into LDS at `lds` (wave-uniform byte address); off0: dma_lane.
template <typename T, int D, bool kV>
__device__ __forceinline__ void dma_rows(int lds, const i32x4& rs, int off0, int stride) {
  using G = Tile<T, D>;
#pragma unroll
  for (int j = 0; j < G::kGroupDmas; ++j)
    dma_b128(lds + j * 1024, G::template dma_off<kV>(off0, j, stride), rs);
}

// Q operand: lane holds chunk 2 s + hf of its row, 16 bytes each.
template <typename T, int D>
struct QFrag {
  u32x4 x[Tile<T, D>::kSteps];
  __device__ __forceinline__ void load(const T* row, int hf, bool live) {
#pragma unroll
    for (int s = 0; s < Tile<T, D>::kSteps; ++s) {
      x[s] = u32x4{0u, 0u, 0u, 0u};
      if (live)
        x[s] = *reinterpret_cast<const u32x4*>(reinterpret_cast<const uint8_t*>(row) + 32 * s +
                                               16 * hf);
    }
  }
};

// acc += A B over one chunk pair (bf16: 16 dims, fp32: 8).
template <typename T>
__device__ __forceinline__ f32x16 dot_step(u32x4 a, u32x4 b, f32x16 acc) {
  if constexpr (std::is_same<T, __bf16>::value) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a),
                                                   __builtin_bit_cast(bf16x8, b), acc, 0, 0, 0);
  } else {
    const f32x4 fa = __builtin_bit_cast(f32x4, a), fb = __builtin_bit_cast(f32x4, b);
#pragma unroll
    for (int i = 0; i < 4; ++i)
      acc = __builtin_amdgcn_mfma_f32_32x32x2f32(fa[i], fb[i], acc, 0, 0, 0);
    return acc;
  }
}

// S^T of one 32-key block (addr: lane_k plus the block's place in LDS).
template <typename T, int D>
__device__ __forceinline__ f32x16 qk_block(int addr, int kb, const QFrag<T, D>& q) {
  f32x16 s = f32x16{};
#pragma unroll
  for (int i = 0; i < Tile<T, D>::kSteps; ++i)
    s = dot_step<T>(Tile<T, D>::k_frag(addr, kb, i), q.x[i], s);
  return s;
}

// O^T += V^T P^T over one 32-key block at LDS address addr (lane_v included).
template <typename T, int D>
__device__ __forceinline__ void pv_block(int addr, const f32x16& p, f32x16 (&o)[D / 32]) {
  if constexpr (std::is_same<T, __bf16>::value) {
#pragma unroll
    for (int st = 0; st < 2; ++st) {
      bf16x8 b;
#pragma unroll
      for (int i = 0; i < 8; ++i) b[i] = static_cast<__bf16>(p[8 * st + i]);
#pragma unroll
      for (int db = 0; db < D / 32; ++db)
        o[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(Tile<T, D>::v_frag(addr, db, st), b, o[db],
                                                        0, 0, 0);
    }
  } else {
#pragma unroll
    for (int v = 0; v < 16; ++v)
#pragma unroll
      for (int db = 0; db < D / 32; ++db)
        o[db] = __builtin_amdgcn_mfma_f32_32x32x2f32(Tile<T, D>::v_elem(addr, db, v), p[v], o[db],
                                                     0, 0, 0);
  }
}

// cap * tanh(x z0), in the unit of sc, for any z0.
__device__ __forceinline__ float cap_any(const ScoreArgs& sc, float z) {
  const float y = z * sc.x;
  const float w = z * z;
  const float small =
      z * fmaf(w, fmaf(w, fmaf(w, fmaf(w, sc.a[4], sc.a[3]), sc.a[2]), sc.a[1]), sc.a[0]);
  // 1 - 2 / (e^2y + 1): exact at both ends of the range, NaN stays NaN
  const float e = __builtin_amdgcn_exp2f(y * (2.f * kLog2e));
  const float large = sc.cap2 - 2.f * sc.cap2 * __builtin_amdgcn_rcpf(e + 1.f);
  return fabsf(y) <= kTanhSmall ? small : large;
}

// The cap applied to a block of products, in the log2 domain.  Where none of
// the wavefront's products is large the polynomial alone serves.  Only the first
// `count` (a multiple of 4) matter.
__device__ __forceinline__ void cap_scores(const ScoreArgs& sc, f32x16& s, int count = 16) {
  float mx = s[0], mn = s[0];
#pragma unroll
  for (int v = 1; v < 15; v += 2) {
    mx = fmaxf(fmaxf(mx, s[v]), s[v + 1]);
    mn = fminf(fminf(mn, s[v]), s[v + 1]);
  }
  const float big = fmaxf(fmaxf(mx, s[15]), -fminf(mn, s[15]));
  // (a NaN is dropped here, and stays one in the polynomial)
  if (__builtin_amdgcn_ballot_w64(big * sc.x > kTanhSmall)) {
#pragma unroll
    for (int v = 0; v < 16; ++v) s[v] = cap_any(sc, s[v]);
  } else {
#pragma unroll
    for (int j = 0; j < 16; j += 4) {
      if (j >= count) break;
#pragma unroll
      for (int v = j; v < j + 4; ++v) {
        const float w = s[v] * s[v];
        s[v] *= fmaf(w, fmaf(w, fmaf(w, fmaf(w, sc.a[4], sc.a[3]), sc.a[2]), sc.a[1]), sc.a[0]);
      }
    }
  }
}

// Key of register v of a 32-key block, less 4 hf.
__device__ __forceinline__ constexpr int key_of(int v) { return 8 * (v >> 2) + (v & 3); }

// The scores of a block are its products, capped where there is a cap, times a
// factor, in the log2 domain, and the bias.
__device__ __forceinline__ float score_factor(const ScoreArgs& sc) {
  return sc.x != 0.f || sc.slopes != nullptr ? 1.f : sc.c;
}
// A bias may be far larger than what a row's scores differ by.  So it is taken
// less the tile's largest bias of a seen key, and the reference too: what is
// rounded then is as small as the difference.  far(v): the distance of register
// v's key.
template <typename Far>
__device__ __forceinline__ float largest_bias(const f32x16& s, float slope, Far far) {
  float a = -INFINITY;
#pragma unroll
  for (int v = 0; v < 16; ++v)
    if (s[v] > -INFINITY) a = fmaxf(a, -slope * far(v));
  return a;
}
template <typename Far>
__device__ __forceinline__ void add_bias(const ScoreArgs& sc, f32x16& s, float slope, float off,
                                         Far far) {
  const float c = sc.x != 0.f ? 1.f : sc.c;
#pragma unroll
  for (int v = 0; v < 16; ++v) s[v] = fmaf(s[v], c, fmaf(-slope, far(v), -off));
}

// Scores of the keys whose bit is not set become -inf.  bits: one a key of the
// block, shifted down by 4 hf.
__device__ __forceinline__ void mask_block(f32x16& s, uint32_t bits) {
#pragma unroll
  for (int v = 0; v < 16; ++v)
    if (!((bits >> key_of(v)) & 1u)) s[v] = -INFINITY;
}

// The low n (0 .. 64) bits.
__device__ __forceinline__ uint64_t low_bits(int n) {
  return n >= 64 ? ~uint64_t(0) : n <= 0 ? uint64_t(0) : (uint64_t(1) << n) - 1;
}

__device__ __forceinline__ float block_max(const f32x16& s) {
  float a = fmaxf(s[0], s[1]), b = fmaxf(s[2], s[3]);
#pragma unroll
  for (int v = 4; v < 16; v += 4) {
    a = fmaxf(a, fmaxf(s[v], s[v + 1]));
    b = fmaxf(b, fmaxf(s[v + 2], s[v + 3]));
  }
  return fmaxf(a, b);
}

// Weights of a block against the row's reference, rounded to what the product
// with V takes.  l gets their sum: numerator and denominator then hold the
// same weights, and a key that has all of a row's weight is returned exactly.
// le (kExact) gets the sum before the rounding, what the log sum is made of.
template <typename T, bool kExact>
__device__ __forceinline__ void weigh_block(f32x16& s, float c, float base, float& l, float& le) {
  const bf16x2 ones = bf16x2{static_cast<__bf16>(1.f), static_cast<__bf16>(1.f)};
  float sum = 0.f, a = 0.f, b = 0.f;
#pragma unroll
  for (int v = 0; v < 16; v += 2) {
    s[v] = __builtin_amdgcn_exp2f(fmaf(s[v], c, -base));
    s[v + 1] = __builtin_amdgcn_exp2f(fmaf(s[v + 1], c, -base));
    if constexpr (std::is_same<T, __bf16>::value) {
      const bf16x2 p = bf16x2{static_cast<__bf16>(s[v]), static_cast<__bf16>(s[v + 1])};
      sum = __builtin_amdgcn_fdot2_f32_bf16(p, ones, sum, false);
    }
    if constexpr (kExact || !std::is_same<T, __bf16>::value) {
      a += s[v];
      b += s[v + 1];
    }
  }
  l += std::is_same<T, __bf16>::value ? sum : a + b;
  le += a + b;
}

// Whether 16 bytes hold an infinity or a NaN.
template <typename T>
__device__ __forceinline__ bool not_finite(u32x4 x) {
  bool bad = false;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (std::is_same<T, __bf16>::value)
      bad |= (x[i] & 0x7f80u) == 0x7f80u || (x[i] & 0x7f800000u) == 0x7f800000u;
    else
      bad |= (x[i] & 0x7f800000u) == 0x7f800000u;
  }
  return bad;
}

// The same 16 bytes with zeros in those places.
template <typename T>
__device__ __forceinline__ u32x4 only_finite(u32x4 x) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (std::is_same<T, __bf16>::value) {
      if ((x[i] & 0x7f80u) == 0x7f80u) x[i] &= 0xffff0000u;
      if ((x[i] & 0x7f800000u) == 0x7f800000u) x[i] &= 0xffffu;
    } else {
      if ((x[i] & 0x7f800000u) == 0x7f800000u) x[i] = 0u;
    }
  }
  return x;
}

template <typename T>
__device__ __forceinline__ float lds_value(int addr) {
  if constexpr (std::is_same<T, __bf16>::value) {
    typedef __attribute__((address_space(3))) uint16_t lds_u16;
    return __builtin_bit_cast(
        float, static_cast<unsigned>(*reinterpret_cast<const lds_u16*>(static_cast<size_t>(addr)))
                   << 16);
  } else {
    return *reinterpret_cast<const lds_float*>(static_cast<size_t>(addr));
  }
}

// Row state of a wavefront: 32 query rows, lanes l and l ^ 32 share one.
template <int D>
struct RowState {
  f32x16 o[D / 32];
  float m;    // reference max, log2 domain; -inf: no key yet
  float l;    // this lane's share of the sum of weights as they are multiplied
  float le;   // and of their sum before rounding, where the log sum is wanted
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int db = 0; db < D / 32; ++db) o[db] = f32x16{};
    m = -INFINITY;
    l = le = 0.f;
  }
  __device__ __forceinline__ float base() const { return m == -INFINITY ? 0.f : m; }
  // Moves the reference where mx exceeds it by more than kLazy, or is the
  // row's first.
  __device__ __forceinline__ void rescale(float mx) {
    const bool grow = mx > m + kLazy || (m == -INFINITY && mx > m);
    if (__builtin_amdgcn_ballot_w64(grow)) {
      // (a row without a reference holds zeros, or what add_not_finite added)
      const float alpha = grow && m != -INFINITY ? __builtin_amdgcn_exp2f(m - mx) : 1.f;
      m = grow ? mx : m;
      l *= alpha;
      le *= alpha;
#pragma unroll
      for (int db = 0; db < D / 32; ++db)
#pragma unroll
        for (int v = 0; v < 16; ++v) o[db][v] *= alpha;
    }
  }
};

// The result of a row: four of its dims, and its log sum; l, le: the sums of its
// weights as they were multiplied, and before their rounding.
template <typename T>
__device__ __forceinline__ void store_row(T* dst, const float (&o)[4], float inv) {
  if constexpr (std::is_same<T, __bf16>::value)
    *reinterpret_cast<bf16x4*>(dst) =
        bf16x4{static_cast<__bf16>(o[0] * inv), static_cast<__bf16>(o[1] * inv),
               static_cast<__bf16>(o[2] * inv), static_cast<__bf16>(o[3] * inv)};
  else
    *reinterpret_cast<f32x4*>(dst) = f32x4{o[0] * inv, o[1] * inv, o[2] * inv, o[3] * inv};
}
__device__ __forceinline__ float inverse(float l) { return l > 0.f ? 1.f / l : l == l ? 0.f : l; }
__device__ __forceinline__ float log_sum(float m, float le) {
  return le > 0.f ? fmaf(m, kLn2, logf(le)) : le == le ? -INFINITY : le;
}
// Weight of a part with reference m in a sum with reference top (>= m).
__device__ __forceinline__ float part_weight(float m, float top) {
  return m == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m - top);  // no key: zeros, or NaN
}

// Merge of four wavefronts that took different keys of the same 32 rows.  Each
// leaves its rows at its own LDS address `mine` (`apart` bytes after the one before,
// the first at lds0) as fp32 rows whose 16-byte chunks are XORed with the row; then
// eight threads a row call f(row, first dim, sums of four dims, reference, l, le).
// All wavefronts call this; the LDS is free again when it returns.
template <int D, typename F>
__device__ __forceinline__ void merge_waves(const RowState<D>& st, int mine, int lds0, int apart,
                                            float (&part)[4][32][3], int wave, int l32, int hf,
                                            F f) {
  constexpr int kChunks = D / 4;
  const float l = half_sum(st.l), le = half_sum(st.le);
  if (hf == 0) {
    part[wave][l32][0] = st.m;
    part[wave][l32][1] = l;
    part[wave][l32][2] = le;
  }
#pragma unroll
  for (int db = 0; db < D / 32; ++db)
#pragma unroll
    for (int i = 0; i < 4; ++i)
      *reinterpret_cast<lds_f32x4*>(static_cast<size_t>(
          mine + l32 * D * 4 + 16 * ((8 * db + 2 * i + hf) ^ (l32 & (kChunks - 1))))) =
          f32x4{st.o[db][4 * i], st.o[db][4 * i + 1], st.o[db][4 * i + 2], st.o[db][4 * i + 3]};
  __syncthreads();
  const int row = threadIdx.x >> 3;
  float top = -INFINITY, wt[4], sl = 0.f, sle = 0.f;
#pragma unroll
  for (int w = 0; w < 4; ++w) top = fmaxf(top, part[w][row][0]);
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    wt[w] = part_weight(part[w][row][0], top);
    sl += part[w][row][1] * wt[w];
    sle += part[w][row][2] * wt[w];
  }
  for (int ch = threadIdx.x & 7; ch < kChunks; ch += 8) {
    float o[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const f32x4 y = *reinterpret_cast<const lds_f32x4*>(static_cast<size_t>(
          lds0 + w * apart + row * D * 4 + 16 * (ch ^ (row & (kChunks - 1)))));
#pragma unroll
      for (int e = 0; e < 4; ++e) o[e] += y[e] * wt[w];
    }
    f(row, 4 * ch, o, top, sl, sle);
  }
  __syncthreads();
}

// V of a tile whose keys are visible to some rows and not to others: a weight
// of 0 times an infinity would be a NaN in rows that do not see the key.  The
// places that are not finite are taken out of the matrix product (`clean`)
// and added to the rows that see them (`bits`: one bit a key of the tile).
template <typename T, int D>
__device__ __forceinline__ void add_not_finite(int tile, int keys, uint64_t bits, int hf,
                                               f32x16 (&o)[D / 32]) {
  for (int key = 0; key < keys; ++key) {
    const bool sees = (bits >> key) & 1;
    for (int db = 0; db < D / 32; ++db)
#pragma unroll
      for (int v = 0; v < 16; ++v) {
        const float x =
            lds_value<T>(tile + Tile<T, D>::v_at(key, 32 * db + 8 * (v >> 2) + 4 * hf + (v & 3)));
        const bool bad = (__builtin_bit_cast(unsigned, x) & 0x7f800000u) == 0x7f800000u;
#pragma unroll
        for (int b = 0; b < D / 32; ++b)
          if (b == db && bad && sees) o[b][v] += x;
      }
  }
}

// The same for a wavefront's own tile of 32 keys at LDS address `tile`.
template <typename T, int D>
__device__ __forceinline__ void mend_own_tile(int tile, uint32_t bits, int lane,
                                              f32x16 (&o)[D / 32]) {
  constexpr int kTile = 32 * Tile<T, D>::kRow;
  bool bad = false;
  for (int i = lane; i < kTile / 16; i += 64)
    bad |= not_finite<T>(*reinterpret_cast<const lds_u32x4*>(static_cast<size_t>(tile + 16 * i)));
  if (!__builtin_amdgcn_ballot_w64(bad)) return;
  add_not_finite<T, D>(tile, 32, bits, lane >> 5, o);
  for (int i = lane; i < kTile / 16; i += 64) {
    lds_u32x4* at = reinterpret_cast<lds_u32x4*>(static_cast<size_t>(tile + 16 * i));
    *at = only_finite<T>(*at);
  }
  wait_lds();
}

}  // namespace flash
}  // namespace sift
