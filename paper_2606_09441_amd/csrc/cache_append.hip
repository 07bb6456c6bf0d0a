// New keys and values of every sequence into its pages (sift_cache_append), the keys
// turned by their positions on the way.  HBM bounds it: every number is read once and
// written once.
//
// Pages of the new keys' own type: a wavefront takes a token, or part of its heads.  65
// thousand rows of 8 heads, D = 128, into bf16 pages: 95 us, 5.6 TB/s.
//
// e4m3 pages hold x / scale, a scale for each page and kv head: a workgroup takes a
// page that new keys enter, of a head.  The scale has to be known before the first code
// is written, so the page's new rows, K and V, stay in registers between the maximum
// and the codes; angles are formed by the lane that turns with them.
//  * A scale is the least power of two that leaves room for what the page holds.  e4m3
//    numbers keep the same relative precision over their whole range, so any other
//    factor would gain nothing; a power of two loses nothing in the division, and keys
//    that a page holds already keep their values when its scale grows, but for those
//    below the smallest normal one.
//  * 16640 rows of 8 heads into empty pages: 26 us of the kernel, of which 21 are the
//    bytes' at a copy's rate and the rest a workgroup's way to its first row (sequence,
//    table) and from its last (maximum, codes); vector unit active in 48% of the cycles.
//    A token of each of 32 sequences: 5.7 us.
//  * The bound of a turned pair is sqrt(2) times its larger half, whatever the angle: the
//    scale depends on no cosine, and is the same for keys moved to other positions.

#include <algorithm>

#include "cache.h"
#include "rotary.h"

namespace sift {
namespace {

using namespace cache;
using rotary::Chunk;

// How many pages the new keys of a sequence enter.
struct PageCost {
  int32_t page_shift, slots, heads;
  __device__ __forceinline__ int end(const Seq& s) const { return s.len + min(s.n, slots - s.len); }
  __device__ __forceinline__ int first(const Seq& s) const { return s.len >> page_shift; }
  __device__ __forceinline__ int pages(const Seq& s) const {
    const int e = end(s);
    return e > s.len ? ((e - 1) >> page_shift) + 1 - first(s) : 0;
  }
  __device__ __forceinline__ int operator()(const Seq& s) const { return heads * pages(s); }
};

__device__ __forceinline__ void write_lens(const CacheAppendArgs& p) {
  if (blockIdx.x != 0 || p.lens_out == nullptr) return;
  const int slots = p.c.max_pages << p.c.page_shift;
  for (int b = threadIdx.x; b < p.c.num_seqs; b += blockDim.x) {
    const Seq s = sequence(p.c, b);
    p.lens_out[b] = s.len + min(s.n, slots - s.len);
  }
}

// How a head's dims turn.
enum Turns { kNone, kHalves, kPairs, kAny, kAnyPairs };

// ---------------------------------------------------------------------------
// pages of the keys' own type
// ---------------------------------------------------------------------------

template <typename T, int kTurns>
__global__ __launch_bounds__(256) void append_kernel(CacheAppendArgs p, int parts) {
  constexpr int n = Chunk<T>::kCount;
  const CacheArgs& a = p.c;
  __shared__ u32x4 others[kTurns == kAny ? 4 : 1][kTurns == kAny ? 64 : 1];
  const int lane = threadIdx.x & 63;
  const int slots = a.max_pages << a.page_shift;
  write_lens(p);
  const Work work(a, PageCost{a.page_shift, slots, 0});
  const int64_t units = static_cast<int64_t>(a.rows) * parts;
  for (int64_t u = static_cast<int64_t>(blockIdx.x) * 4 + uniform(threadIdx.x >> 6); u < units;
       u += static_cast<int64_t>(gridDim.x) * 4) {
    const int token = uniform(static_cast<int>(u / parts));
    const int part = uniform(static_cast<int>(u - static_cast<int64_t>(token) * parts));
    const Place pl = work.find_token(token);
    if (pl.b >= a.num_seqs) continue;  // no sequence's
    const Seq s = work.seq(pl.b);
    const int slot = p.slots != nullptr ? scalar(p.slots, token) : s.len + (token - s.row0);
    if (slot < 0 || slot >= slots) continue;
    const int page =
        scalar(a.table, static_cast<int64_t>(pl.b) * a.max_pages + (slot >> a.page_shift));
    if (page < 0 || page >= a.num_pages) continue;
    const int64_t row =
        (static_cast<int64_t>(page) << a.page_shift) + (slot & ((1 << a.page_shift) - 1));
    const int pos = a.row_pos != nullptr ? scalar(a.row_pos, token) : slot;
    const int64_t head = static_cast<int64_t>(a.hkv) * p.d;  // numbers of a row
    const T* const k = static_cast<const T*>(p.k) + token * head;
    const T* const v = static_cast<const T*>(p.v) + token * head;
    T* const ko = static_cast<T*>(p.k_pages) + row * head;
    T* const vo = static_cast<T*>(p.v_pages) + row * head;
    const int chunks = p.d / n;  // of a head
    if (p.pos_out != nullptr)
      for (int h = part * 64 + lane; h < a.hkv; h += parts * 64)
        p.pos_out[(static_cast<int64_t>(pl.b) * a.hkv + h) * slots + slot] = pos;
    int from = 0;  // chunks of K that turn
    if constexpr (kTurns == kHalves || kTurns == kPairs) {
      using I = rotary::Item<T, kTurns == kPairs>;
      const int items = p.r.half / I::kAngles, at_once = 64 / items;
      const int item = lane % items, sub = lane / items;
      I it;
      if (sub < at_once) {
        it.angles(p.r, pos, item);
#pragma unroll 2
        for (int h = part * at_once + sub; h < a.hkv; h += parts * at_once) {
          const int64_t at = static_cast<int64_t>(h) * p.d + item * n;
          Chunk<T> x[I::kChunks];
#pragma unroll
          for (int j = 0; j < I::kChunks; ++j)
            x[j].set(*reinterpret_cast<const u32x4*>(k + at + j * p.r.half));
          it.apply(x);
#pragma unroll
          for (int j = 0; j < I::kChunks; ++j)
            *reinterpret_cast<u32x4*>(ko + at + j * p.r.half) = x[j].get();
        }
      }
      from = 2 * p.r.half / n;
    }
    if constexpr (kTurns == kAny || kTurns == kAnyPairs) {
      constexpr bool kInterleaved = kTurns == kAnyPairs;
      const int at_once = 64 / chunks;  // heads
      const int chunk = lane % chunks, sub = lane / chunks;
      u32x4* const seen = others[kInterleaved ? 0 : threadIdx.x >> 6];
      rotary::AnyChunk<T, kInterleaved> it;
      it.angles(p.r, pos, chunk);
#pragma unroll 2
      for (int h = part * at_once + sub; h < a.hkv; h += parts * at_once) {
        const int at = h * p.d + chunk * n;
        const u32x4 raw = *reinterpret_cast<const u32x4*>(k + at);
        if constexpr (!kInterleaved) seen[lane] = raw;
        rotary::lds_order();
        Chunk<T> x;
        x.set(raw);
        it.apply(p.r, x, reinterpret_cast<const T*>(seen + sub * chunks));
        rotary::lds_order();
        *reinterpret_cast<u32x4*>(ko + at) = x.get();
      }
      from = chunks;
    }
    // the rest of K, and V
    const int rest = chunks - from;
    for (int e = part * 64 + lane; e < a.hkv * rest; e += parts * 64) {
      const int h = e / rest, at = h * p.d + (from + e - h * rest) * n;
      *reinterpret_cast<u32x4*>(ko + at) =
          *reinterpret_cast<const u32x4*>(k + at);
    }
#pragma unroll 2
    for (int e = part * 64 + lane; e < a.hkv * chunks; e += parts * 64)
      *reinterpret_cast<u32x4*>(vo + e * n) =
          *reinterpret_cast<const u32x4*>(v + e * n);
  }
}

// ---------------------------------------------------------------------------
// e4m3 pages
// ---------------------------------------------------------------------------

constexpr float kRoot2 = 1.4142137f;  // just above sqrt(2)
constexpr int kLeastScale = -100;     // exponent: a page of nothing larger holds zeros to any score

// The larger of two sizes, of finite ones.
__device__ __forceinline__ float larger(float m, float x) {
  const float a = fabsf(x);
  return a < INFINITY ? fmaxf(m, a) : m;
}

// The least power of two, from 2^kLeastScale on, with size <= 448 times it: 448 = 1.75 2^8.
__device__ __forceinline__ float scale_for(float size) {
  const uint32_t u = __builtin_bit_cast(uint32_t, fminf(size, 3.402823e38f));
  const int e = static_cast<int>(u >> 23) - 127 - 8 + ((u & 0x7fffffu) > 0x600000u);
  return __builtin_bit_cast(float, static_cast<uint32_t>(max(e, kLeastScale) + 127) << 23);
}
// The least power of two that is not below x.
__device__ __forceinline__ float power_from(float x) {
  const uint32_t u = __builtin_bit_cast(uint32_t, x);
  return __builtin_bit_cast(float, (u + 0x7fffffu) & 0xff800000u);
}

// Sizes of bf16 numbers as their bits, which order them: the largest of each half of words.
typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ u16x2 larger_bits(u16x2 m, uint32_t w) {
  return __builtin_elementwise_max(m, __builtin_bit_cast(u16x2, w & 0x7fff7fffu));
}
// The larger half as a number; infinity where it is none.
__device__ __forceinline__ float size_of(u16x2 m) {
  const uint32_t u = m[0] > m[1] ? m[0] : m[1];
  return u >= 0x7f80u ? INFINITY : __builtin_bit_cast(float, u << 16);
}

// Eight numbers as codes of `scale` (a power of two), rounded to the nearest; what is
// not finite, or rounds to more than 448, becomes NaN, which e4m3 has in place of
// infinities.
typedef short s16x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ u32x2 encode(const float (&x)[8], float scale) {
  u32x2 v;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    s16x2 w = {0, 0};
    w = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(w, x[4 * i], x[4 * i + 1], scale, false);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(w, x[4 * i + 2], x[4 * i + 3], scale, true);
    v[i] = __builtin_bit_cast(uint32_t, w);
  }
  return v;
}
__device__ __forceinline__ u32x2 encode(u32x4 x, float scale) {  // of bf16
  u32x2 v;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const uint32_t a = x[2 * i], b = x[2 * i + 1];
    s16x2 w = {0, 0};
    w = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(w, __builtin_bit_cast(bf16x2, a), scale, false);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(w, __builtin_bit_cast(bf16x2, b), scale, true);
    v[i] = __builtin_bit_cast(uint32_t, w);
  }
  return v;
}

__device__ __forceinline__ void decode(u32x2 v, float scale, float (&x)[8]) {
  typedef float f32x2 __attribute__((ext_vector_type(2)));
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int w = static_cast<int>(v[i]);
    const f32x2 a = __builtin_amdgcn_cvt_pk_f32_fp8(w, false);
    const f32x2 b = __builtin_amdgcn_cvt_pk_f32_fp8(w, true);
    x[4 * i] = a[0] * scale;
    x[4 * i + 1] = a[1] * scale;
    x[4 * i + 2] = b[0] * scale;
    x[4 * i + 3] = b[1] * scale;
  }
}

// A lane's item of a row: two chunks of eight dims.  Halves: those of a pair of
// stretches, then the rest; else two neighbours.
template <int kTurns>
__device__ __forceinline__ void chunks_of(const RotaryArgs& r, int item, int& a, int& b) {
  a = 2 * item;
  b = a + 1;
  if constexpr (kTurns == kHalves) {
    const int h = r.half / 8;
    if (item < h) {
      a = item;
      b = item + h;
    }
  }
}

// kPasses passes of a workgroup over a page's rows.
template <int D, int kTurns, int kPasses>
__global__ __launch_bounds__(256) void append_codes_kernel(CacheAppendArgs p) {
  using C = Chunk<__bf16>;
  constexpr int kItems = D / 16;  // of a row
  __shared__ float part[2][4];
  __shared__ u32x4 seen[kTurns == kAny ? 256 : 1][2];
  const CacheArgs& a = p.c;
  const int slots = a.max_pages << a.page_shift;
  write_lens(p);
  const PageCost cost{a.page_shift, slots, a.hkv};
  const Work work(a, cost);
  const int item = threadIdx.x % kItems, r0 = threadIdx.x / kItems;
  const int each = blockDim.x / kItems;  // rows of a pass
  const int wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
  int c0, c1;
  chunks_of<kTurns>(p.r, item, c0, c1);
  for (int x = blockIdx.x; x < work.total; x += gridDim.x) {
    const Place pl = work.find(x);
    if (pl.b >= a.num_seqs) return;
    const Seq s = work.seq(pl.b);
    const int u = x - pl.at;
    const int h = u % a.hkv, pi = cost.first(s) + u / a.hkv;
    const int page = scalar(a.table, static_cast<int64_t>(pl.b) * a.max_pages + pi);
    if (page < 0 || page >= a.num_pages) continue;
    const int base = pi << a.page_shift;              // the page's first slot
    const int lo = max(s.len - base, 0);              // its new rows
    const int hi = min(cost.end(s) - base, 1 << a.page_shift);
    const int64_t row = static_cast<int64_t>(page) << a.page_shift;
    const int64_t src = s.row0 + (base - s.len);      // of the page's row 0, were it new

    // the new rows, K and V
    u32x4 kx[kPasses][2], vx[kPasses][2];
#pragma unroll
    for (int i = 0; i < kPasses; ++i) {
      const int r = r0 + i * each;
#pragma unroll
      for (int j = 0; j < 2; ++j) kx[i][j] = vx[i][j] = u32x4{0u, 0u, 0u, 0u};
      if (r < lo || r >= hi) continue;
      const int64_t at = ((src + r) * a.hkv + h) * D;
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const int64_t c = at + 8 * (j ? c1 : c0);
        kx[i][j] = *reinterpret_cast<const u32x4*>(static_cast<const __bf16*>(p.k) + c);
        vx[i][j] = *reinterpret_cast<const u32x4*>(static_cast<const __bf16*>(p.v) + c);
      }
    }
    const int64_t sc = static_cast<int64_t>(page) * a.hkv + h;
    const bool begun = lo > 0;
    float old_k = begun ? p.k_scales[sc] : 0.f, old_v = begun ? p.v_scales[sc] : 0.f;

    // this lane's frequencies, for all its rows
    double freq[8] = {};
    if constexpr (kTurns == kHalves) {
      if (8 * c0 < p.r.half)
#pragma unroll
        for (int e = 0; e < 8; ++e) freq[e] = rotary::frequency(p.r, 8 * c0 + e);
    } else if constexpr (kTurns == kPairs) {
#pragma unroll
      for (int e = 0; e < 8; ++e)  // (8 item + e: the chunks are neighbours)
        freq[e] = rotary::frequency(p.r, min(8 * item + e, p.r.half - 1));
    }

    // their largest sizes
    const float grow = kRoot2 * p.r.magnitude;  // of dims that turn
    float mk, mv;
    {
      u16x2 r = {0, 0}, k = {0, 0}, v = {0, 0};  // of dims that turn, that stay, of V
#pragma unroll
      for (int i = 0; i < kPasses; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            v = larger_bits(v, vx[i][j][e]);
            if (kTurns > kHalves && 4 * (j ? c1 : c0) + e < p.r.half)
              r = larger_bits(r, kx[i][j][e]);
            else
              k = larger_bits(k, kx[i][j][e]);
          }
      mk = size_of(k);
      mv = size_of(v);
      if (kTurns == kHalves && 8 * c0 < p.r.half) mk *= grow;  // all of the item's, or none
      if (kTurns > kHalves) mk = fmaxf(mk, size_of(r) * grow);
    }
    if (__syncthreads_or(mk == INFINITY || mv == INFINITY)) {  // without what is not finite
      float r = 0.f;
      mk = mv = 0.f;
#pragma unroll
      for (int i = 0; i < kPasses; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          C k, v;
          k.set(kx[i][j]);
          v.set(vx[i][j]);
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            mv = larger(mv, v.x[e]);
            if (kTurns != kNone && 4 * (j ? c1 : c0) + e / 2 < p.r.half)
              r = larger(r, k.x[e]);
            else
              mk = larger(mk, k.x[e]);
          }
        }
      if (kTurns != kNone) mk = fmaxf(mk, r * grow);
    }
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) {
      mk = fmaxf(mk, __shfl_xor(mk, d));
      mv = fmaxf(mv, __shfl_xor(mv, d));
    }
    if ((threadIdx.x & 63) == 0) {
      part[0][wave] = mk;
      part[1][wave] = mv;
    }
    __syncthreads();
    for (int w = 0; w < waves; ++w) {
      mk = fmaxf(mk, part[0][w]);
      mv = fmaxf(mv, part[1][w]);
    }
    if (begun) {  // as the attention takes them: what the page holds stays what it was read as
      old_k = usable_scale(old_k);
      old_v = usable_scale(old_v);
    }
    const float new_k = fmaxf(power_from(old_k), scale_for(mk));
    const float new_v = fmaxf(power_from(old_v), scale_for(mv));
    __syncthreads();  // the maxima and the old scales are read
    if (threadIdx.x == 0) {
      p.k_scales[sc] = new_k;
      p.v_scales[sc] = new_v;
    }
    uint8_t* const ko = static_cast<uint8_t*>(p.k_pages);
    uint8_t* const vo = static_cast<uint8_t*>(p.v_pages);
    // rows that the page held
    const auto again = [&](uint8_t* pool, float was, float is) {
      for (int r = r0; r < lo; r += each)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          u32x2* q = reinterpret_cast<u32x2*>(pool + ((row + r) * a.hkv + h) * D + 8 * (j ? c1 : c0));
          float y[8];
          decode(*q, was, y);
          *q = encode(y, is);
        }
    };
    if (begun && new_k != old_k) again(ko, old_k, new_k);
    if (begun && new_v != old_v) again(vo, old_v, new_v);
    // the new ones
#pragma unroll
    for (int i = 0; i < kPasses; ++i) {
      const int r = r0 + i * each;
      if (r < lo || r >= hi) continue;
      const int pos = a.row_pos != nullptr ? a.row_pos[src + r] : base + r;
      C k[2];
#pragma unroll
      for (int j = 0; j < 2; ++j) k[j].set(kx[i][j]);
      if constexpr (kTurns == kHalves) {
        if (8 * c0 < p.r.half)
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            float c, sn;
            rotary::turn<__bf16>(p.r, pos, freq[e], c, sn);
            rotary::rotate(c, sn, k[0].x[e], k[1].x[e]);
          }
      } else if constexpr (kTurns == kPairs) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          if (8 * item + e >= p.r.half) break;
          float c, sn;
          rotary::turn<__bf16>(p.r, pos, freq[e], c, sn);
          C& x = k[e >> 2];
          rotary::rotate(c, sn, x.x[2 * (e & 3)], x.x[2 * (e & 3) + 1]);
        }
      } else if constexpr (kTurns == kAny) {  // halves of no whole chunks
        // (a row's lanes, neighbours in a wavefront, leave it in LDS)
        seen[threadIdx.x][0] = kx[i][0];
        seen[threadIdx.x][1] = kx[i][1];
        rotary::lds_order();
        const __bf16* const kr =
            reinterpret_cast<const __bf16*>(&seen[threadIdx.x - item][0]);
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const int d = 8 * (j ? c1 : c0) + e;
            if (d >= 2 * p.r.half) continue;
            const bool low = d < p.r.half;
            float c, sn;
            rotary::turn<__bf16>(p.r, pos, low ? d : d - p.r.half, c, sn);
            const float other = static_cast<float>(kr[low ? d + p.r.half : d - p.r.half]);
            k[j].x[e] = fmaf(k[j].x[e], c, low ? -(other * sn) : other * sn);
          }
        rotary::lds_order();
      }
      const int64_t at = ((row + r) * a.hkv + h) * D;
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const int64_t c = at + 8 * (j ? c1 : c0);
        *reinterpret_cast<u32x2*>(ko + c) =
            kTurns == kNone ? encode(kx[i][j], new_k) : encode(k[j].x, new_k);
        *reinterpret_cast<u32x2*>(vo + c) = encode(vx[i][j], new_v);
      }
      if (item == 0 && p.pos_out != nullptr)
        p.pos_out[(static_cast<int64_t>(pl.b) * a.hkv + h) * slots + base + r] = pos;
    }
  }
}

__global__ __launch_bounds__(256) void lens_kernel(CacheAppendArgs p) {
  const int b = blockIdx.x * 256 + threadIdx.x;
  if (b >= p.c.num_seqs) return;
  const int slots = p.c.max_pages << p.c.page_shift;
  const Seq s = sequence(p.c, b);
  p.lens_out[b] = s.len + min(s.n, slots - s.len);
}

// Wavefronts that a launch of few tokens is split into (us of 8 heads, D = 128, bf16, one
// a token / 4096 / 32768: 4 tokens 3.5 / 3.2 / 3.2, 400 4.4 / 4.0 / 4.0, 2000 6.4 / 6.4 /
// 6.6).
constexpr int64_t kAppendWaves = 4096;

}  // namespace

int64_t cache_append_units(const CacheAppendArgs& a) {
  const int64_t rows =
      std::min<int64_t>(a.c.rows, static_cast<int64_t>(a.c.max_pages) << a.c.page_shift);
  return static_cast<int64_t>(a.c.num_seqs) * a.c.hkv * ((rows >> a.c.page_shift) + 2);
}

hipError_t launch_cache_append(CacheAppendArgs a, Pool pool, hipStream_t stream) {
  // lens that are read and written are written by a launch of their own
  const bool apart = a.lens_out != nullptr && a.lens_out == a.c.lens;
  int32_t* const lens_out = a.lens_out;
  if (apart) a.lens_out = nullptr;
  const int page = 1 << a.c.page_shift;
  if (pool == Pool::kE4m3) {
    const int threads = std::min(256, page * (a.d / 16));
    const int passes = page * (a.d / 16) / threads;
    const int64_t pages = std::min<int64_t>(a.c.rows / page + 2 * static_cast<int64_t>(a.c.num_seqs),
                                            a.c.rows);
    const int64_t units = std::max<int64_t>(1, std::min<int64_t>(pages * a.c.hkv, 1 << 22));
    const int turns = a.r.half == 0 ? kNone
                      : a.r.interleaved ? kPairs
                      : a.r.half % 8 == 0 ? kHalves
                                          : kAny;
    const auto go = [&](auto dim, auto turn, auto pass) {
      hipLaunchKernelGGL(
          (append_codes_kernel<decltype(dim)::value, decltype(turn)::value, decltype(pass)::value>),
          dim3(static_cast<unsigned>(units)), dim3(threads), 0, stream, a);
    };
    const auto with_passes = [&](auto dim, auto turn) {
      if (passes == 1) go(dim, turn, std::integral_constant<int, 1>{});
      else if (passes == 2) go(dim, turn, std::integral_constant<int, 2>{});
      else go(dim, turn, std::integral_constant<int, 4>{});
    };
    const auto with_turns = [&](auto dim) {
      if (turns == kNone) with_passes(dim, std::integral_constant<int, kNone>{});
      else if (turns == kHalves) with_passes(dim, std::integral_constant<int, kHalves>{});
      else if (turns == kPairs) with_passes(dim, std::integral_constant<int, kPairs>{});
      else with_passes(dim, std::integral_constant<int, kAny>{});
    };
    if (a.d == 128)
      with_turns(std::integral_constant<int, 128>{});
    else
      with_turns(std::integral_constant<int, 64>{});
  } else {
    const auto launch = [&](auto elem_) {
      using T = decltype(elem_);
      const int64_t parts = std::max<int64_t>(
          1, std::min<int64_t>((static_cast<int64_t>(a.c.hkv) * a.d * sizeof(T) + 1023) / 1024,
                               kAppendWaves / std::max<int64_t>(1, a.c.rows)));
      const int64_t g =
          std::max<int64_t>(1, std::min<int64_t>((a.c.rows * parts + 3) / 4, 1 << 22));
      const auto go = [&](auto turn) {
        hipLaunchKernelGGL((append_kernel<T, decltype(turn)::value>),
                           dim3(static_cast<unsigned>(g)), dim3(256), 0, stream, a,
                           static_cast<int>(parts));
      };
      if (a.r.half == 0)
        go(std::integral_constant<int, kNone>{});
      else if (!rotary::by_items<T>(a.r, a.d) && a.r.interleaved)
        go(std::integral_constant<int, kAnyPairs>{});
      else if (!rotary::by_items<T>(a.r, a.d))
        go(std::integral_constant<int, kAny>{});
      else if (a.r.interleaved)
        go(std::integral_constant<int, kPairs>{});
      else
        go(std::integral_constant<int, kHalves>{});
    };
    if (pool == Pool::kBf16)
      launch(__bf16{});
    else
      launch(float{});
  }
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || !apart) return e;
  a.lens_out = lens_out;
  hipLaunchKernelGGL(lens_kernel, dim3((a.c.num_seqs + 255) / 256), dim3(256), 0, stream, a);
  return hipGetLastError();
}

}  // namespace sift
