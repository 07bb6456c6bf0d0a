// C ABI of the page cache (include/sift_serve.h): the handle with its scratch,
// and the host checks of its calls.  The kernels are in cache_attn.hip,
// cache_append.hip, cache_weights.hip and cache_evict.hip.

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <initializer_list>
#include <limits>
#include <new>

#include "rotary_api.h"
#include "score_api.h"
#include "sift.h"
#include "sift_internal.h"
#include "sift_serve.h"

struct sift_cache {
  int device = 0;
  int32_t num_seqs = 0, hq = 0, hkv = 0, head_dim = 0, page = 0, max_pages = 0, max_rows = 0;
  int32_t cus = 0;           // compute units of the device
  void* dev = nullptr;
  float* part_o = nullptr;
  float4* part_ml = nullptr;
  int32_t* moves = nullptr;      // of the eviction (CacheEvictArgs)
  int32_t* num_moves = nullptr;
  int32_t* hist = nullptr;
  int4* state = nullptr;
  int4* counts = nullptr;
  hipStream_t last_stream = nullptr;  // the stream of the last enqueued work
};

namespace {

constexpr int64_t kMost = std::numeric_limits<int32_t>::max() - 255;

bool aligned16(const void* p) { return reinterpret_cast<uintptr_t>(p) % 16 == 0; }

int32_t log2_of(int32_t x) {
  int32_t s = 0;
  while ((1 << s) < x) ++s;
  return s;
}

sift_status check_tensor(const sift_tensor* t, int32_t tokens, int32_t heads, int32_t dim,
                         int32_t dtype) {
  if (t == nullptr) return SIFT_E_NULL;
  if (t->data == nullptr && static_cast<int64_t>(t->tokens) * t->heads * t->head_dim > 0)
    return SIFT_E_NULL;
  if (t->dtype != SIFT_F32 && t->dtype != SIFT_BF16 && t->dtype != SIFT_E4M3)
    return SIFT_E_UNSUPPORTED;
  if (t->tokens != tokens || t->heads != heads || t->head_dim != dim) return SIFT_E_SHAPE;
  if (t->dtype != dtype || !aligned16(t->data)) return SIFT_E_UNSUPPORTED;
  return SIFT_OK;
}

// The cache's own arguments; a's device-side view of them.  codes: the call takes pools
// of e4m3.
sift_status check_kv(const sift_cache* c, const sift_cache_kv* kv, sift::CacheArgs* a,
                     bool codes = false) {
  if (c == nullptr || kv == nullptr || kv->k_pages == nullptr || kv->v_pages == nullptr)
    return SIFT_E_NULL;
  const int32_t rows = kv->k_pages->tokens, dtype = kv->k_pages->dtype;
  if (rows < c->page || rows % c->page != 0) return SIFT_E_SHAPE;
  sift_status st;
  if ((st = check_tensor(kv->k_pages, rows, c->hkv, c->head_dim, dtype)) != SIFT_OK) return st;
  if ((st = check_tensor(kv->v_pages, rows, c->hkv, c->head_dim, dtype)) != SIFT_OK) return st;
  if (kv->page_table == nullptr || kv->lens == nullptr) return SIFT_E_NULL;
  if (dtype == SIFT_E4M3) {
    if (!codes) return SIFT_E_UNSUPPORTED;
    if (kv->k_scales == nullptr || kv->v_scales == nullptr) return SIFT_E_NULL;
  }
  if (!aligned16(kv->key_pos)) return SIFT_E_UNSUPPORTED;
  int dev = -1;
  if (hipGetDevice(&dev) != hipSuccess) return SIFT_E_HIP;
  if (dev != c->device) return SIFT_E_PLAN;
  a->k = kv->k_pages->data;
  a->v = kv->v_pages->data;
  a->table = kv->page_table;
  a->lens = kv->lens;
  a->page_lens = kv->page_lens;
  a->key_pos = kv->key_pos;
  a->num_seqs = c->num_seqs;
  a->max_pages = c->max_pages;
  a->page_shift = log2_of(c->page);
  a->num_pages = rows / c->page;
  a->hq = c->hq;
  a->hkv = c->hkv;
  return SIFT_OK;
}

// The new tokens; dtype: the pools'.
sift_status check_rows(const sift_cache* c, const sift_cache_rows* r, const sift_tensor* q,
                       int32_t dtype, const sift_score* score, double unit, sift::CacheArgs* a) {
  if (q == nullptr) return SIFT_E_NULL;
  const int32_t rows = q->tokens;
  if (rows < 0) return SIFT_E_SHAPE;
  sift_status st;
  if ((st = check_tensor(q, rows, c->hq, c->head_dim, dtype)) != SIFT_OK) return st;
  a->row_ptr = r != nullptr ? r->row_ptr : nullptr;
  a->row_pos = r != nullptr ? r->row_pos : nullptr;
  if (a->row_ptr == nullptr &&
      (rows % c->num_seqs != 0 || rows / c->num_seqs > c->max_rows))
    return SIFT_E_SHAPE;
  if (static_cast<int64_t>(rows) * c->hq >= int64_t(1) << 24) return SIFT_E_CAPACITY;
  a->rows = rows;
  a->max_rows = c->max_rows;
  a->q = q->data;
  return sift::make_score(score, c->head_dim, unit, &a->sc);
}

// Whether [p, p + n) and [q, q + n) share a byte.
bool overlap(const void* p, const void* q, size_t n) {
  const uintptr_t a = reinterpret_cast<uintptr_t>(p), b = reinterpret_cast<uintptr_t>(q);
  return q != nullptr && a < b + n && b < a + n;
}

// The type of a call's other tensors.
int32_t type_beside(int32_t pools) { return pools == SIFT_E4M3 ? SIFT_BF16 : pools; }

sift::Pool pool_of(int32_t pools) {
  return pools == SIFT_E4M3   ? sift::Pool::kE4m3
         : pools == SIFT_BF16 ? sift::Pool::kBf16
                              : sift::Pool::kF32;
}

// Workgroups of the attention: two to a CU (one where its LDS allows no more).
int32_t attn_groups(const sift_cache* c, bool bf16) {
  return c->cus * (!bf16 && c->head_dim == 128 ? 1 : 2);
}

}  // namespace

extern "C" {

sift_status sift_cache_create(int32_t num_seqs, int32_t num_q_heads, int32_t num_kv_heads,
                              int32_t head_dim, int32_t page, int32_t max_pages,
                              int32_t max_rows, sift_cache** cache_out) {
  if (cache_out == nullptr) return SIFT_E_NULL;
  *cache_out = nullptr;
  if (num_seqs < 1 || num_q_heads < 1 || num_kv_heads < 1 || num_q_heads % num_kv_heads != 0 ||
      max_pages < 1 || max_rows < 1)
    return SIFT_E_SHAPE;
  if (head_dim != 64 && head_dim != 128) return SIFT_E_UNSUPPORTED;
  if (page != 16 && page != 32 && page != 64 && page != 128) return SIFT_E_UNSUPPORTED;
  const int64_t g = num_q_heads / num_kv_heads;
  if (static_cast<int64_t>(max_pages) * page > kMost || max_rows * g > kMost ||
      num_seqs > kMost || num_kv_heads > sift::kMostKvHeads)
    return SIFT_E_CAPACITY;
  sift_cache* c = new (std::nothrow) sift_cache();
  if (c == nullptr) return SIFT_E_HIP;
  c->num_seqs = num_seqs;
  c->hq = num_q_heads;
  c->hkv = num_kv_heads;
  c->head_dim = head_dim;
  c->page = page;
  c->max_pages = max_pages;
  c->max_rows = max_rows;
  const auto fail = [c]() {
    if (c->dev != nullptr) (void)hipFree(c->dev);
    delete c;
    return SIFT_E_HIP;
  };
  if (hipGetDevice(&c->device) != hipSuccess ||
      hipDeviceGetAttribute(&c->cus, hipDeviceAttributeMultiprocessorCount, c->device) !=
          hipSuccess)
    return fail();
  // (where bf16 does not go by the wide units, e4m3 does not either)
  const bool wide = sift::cache_attn_wide(
      sift::Pool::kBf16, max_rows * g,
      static_cast<int64_t>(num_seqs) * num_kv_heads * max_pages * page);
  const size_t rows = static_cast<size_t>(2 * 2 * c->cus) *
                      (wide ? sift::kCacheWideRows : sift::kCacheRows);
  const size_t o_bytes = rows * head_dim * sizeof(float);
  const size_t heads = static_cast<size_t>(num_seqs) * num_kv_heads;
  const size_t moves = heads * max_pages * page;
  size_t at = 0;
  const auto place = [&at](size_t n) {
    const size_t off = at;
    at += (n + 255) & ~size_t(255);
    return off;
  };
  const size_t o_o = place(o_bytes), o_ml = place(rows * sizeof(float4));
  const size_t o_moves = place(moves * sizeof(int32_t)), o_num = place(heads * sizeof(int32_t));
  const size_t units = static_cast<size_t>(
      sift::evict_units(static_cast<int64_t>(max_pages) * page));
  const size_t hist_bytes = heads * sift::kEvictHist * sizeof(int32_t);
  const size_t o_hist = place(hist_bytes), o_state = place(heads * 3 * sizeof(int4));
  const size_t o_counts = place(heads * units * sizeof(int4));
  if (hipMalloc(&c->dev, at) != hipSuccess) return fail();
  uint8_t* base = static_cast<uint8_t*>(c->dev);
  c->part_o = reinterpret_cast<float*>(base + o_o);
  c->part_ml = reinterpret_cast<float4*>(base + o_ml);
  c->moves = reinterpret_cast<int32_t*>(base + o_moves);
  c->num_moves = reinterpret_cast<int32_t*>(base + o_num);
  c->hist = reinterpret_cast<int32_t*>(base + o_hist);
  c->state = reinterpret_cast<int4*>(base + o_state);
  c->counts = reinterpret_cast<int4*>(base + o_counts);
  if (hipMemset(c->hist, 0, hist_bytes) != hipSuccess ||
      hipStreamSynchronize(nullptr) != hipSuccess)
    return fail();
  *cache_out = c;
  return SIFT_OK;
}

sift_status sift_cache_destroy(sift_cache* cache) {
  if (cache == nullptr) return SIFT_OK;
  sift_status st = SIFT_OK;
  // the last work may still use the scratch
  if (hipStreamSynchronize(cache->last_stream) != hipSuccess) st = SIFT_E_HIP;
  if (hipFree(cache->dev) != hipSuccess) st = SIFT_E_HIP;
  delete cache;
  return st;
}

sift_status sift_cache_attention(sift_cache* cache, const sift_cache_kv* kv,
                                 const sift_cache_rows* new_rows, const sift_tensor* q,
                                 const sift_tensor* k_new, const sift_tensor* v_new,
                                 const uint64_t* tree_mask, int32_t mask_words,
                                 const sift_score* score, sift_tensor* out, float* lse,
                                 void* stream) {
  sift::CacheAttnArgs a{};
  sift_status st;
  if ((st = check_kv(cache, kv, &a.c, true)) != SIFT_OK) return st;
  const int32_t pools = kv->k_pages->dtype, dtype = type_beside(pools);
  if ((st = check_rows(cache, new_rows, q, dtype, score, sift::kUnitLog2e, &a.c)) != SIFT_OK)
    return st;
  const int32_t rows = q->tokens, d = cache->head_dim;
  if ((st = check_tensor(k_new, rows, cache->hkv, d, dtype)) != SIFT_OK) return st;
  if ((st = check_tensor(v_new, rows, cache->hkv, d, dtype)) != SIFT_OK) return st;
  if ((st = check_tensor(out, rows, cache->hq, d, dtype)) != SIFT_OK) return st;
  if (tree_mask != nullptr && mask_words < (cache->max_rows + 63) / 64) return SIFT_E_CAPACITY;
  if (sift::cache_attn_steps(a.c, pools == SIFT_E4M3) >= int64_t(1) << 31) return SIFT_E_CAPACITY;
  if (rows == 0) return SIFT_OK;
  a.k_new = k_new->data;
  a.v_new = v_new->data;
  a.tree_mask = tree_mask;
  a.mask_words = mask_words;
  a.out = out->data;
  a.lse = lse;
  a.part_o = cache->part_o;
  a.part_ml = cache->part_ml;
  if (pools == SIFT_E4M3) {
    a.k_scales = kv->k_scales;
    a.v_scales = kv->v_scales;
  }
  a.groups = attn_groups(cache, dtype == SIFT_BF16);
  const hipStream_t s = static_cast<hipStream_t>(stream);
  const hipError_t e = sift::launch_cache_attn(a, pool_of(pools), d, s);
  cache->last_stream = s;
  return e == hipSuccess ? SIFT_OK : SIFT_E_HIP;
}

sift_status sift_cache_append(sift_cache* cache, const sift_cache_kv* kv,
                              const sift_cache_rows* new_rows, const sift_tensor* k,
                              const sift_tensor* v, const sift_rotary* rotary,
                              const int32_t* slots, int32_t* pos_out, int32_t* lens_out,
                              void* stream) {
  sift::CacheAppendArgs a{};
  sift_status st;
  if ((st = check_kv(cache, kv, &a.c, true)) != SIFT_OK) return st;
  if (k == nullptr) return SIFT_E_NULL;
  const int32_t rows = k->tokens, dtype = kv->k_pages->dtype;
  if (rows < 0) return SIFT_E_SHAPE;
  for (const sift_tensor* t : {k, v})
    if ((st = check_tensor(t, rows, cache->hkv, cache->head_dim, type_beside(dtype))) != SIFT_OK)
      return st;
  a.c.row_ptr = new_rows != nullptr ? new_rows->row_ptr : nullptr;
  a.c.row_pos = new_rows != nullptr ? new_rows->row_pos : nullptr;
  if (a.c.row_ptr == nullptr && rows % cache->num_seqs != 0) return SIFT_E_SHAPE;
  a.c.rows = a.c.max_rows = rows;
  if (rotary != nullptr && (st = sift::make_rotary(rotary, cache->head_dim, &a.r)) != SIFT_OK)
    return st;
  if (slots != nullptr && (lens_out != nullptr || dtype == SIFT_E4M3)) return SIFT_E_UNSUPPORTED;
  const size_t small = static_cast<size_t>(cache->num_seqs) * 4;
  if (lens_out != kv->lens && overlap(lens_out, kv->lens, small)) return SIFT_E_UNSUPPORTED;
  if (static_cast<int64_t>(rows) * cache->hkv >= int64_t(1) << 31 ||
      sift::cache_append_units(a) >= int64_t(1) << 31)
    return SIFT_E_CAPACITY;
  a.d = cache->head_dim;
  a.k = k->data;
  a.v = v->data;
  a.k_pages = kv->k_pages->data;
  a.v_pages = kv->v_pages->data;
  if (dtype == SIFT_E4M3) {
    a.k_scales = kv->k_scales;
    a.v_scales = kv->v_scales;
  }
  a.slots = slots;
  a.pos_out = pos_out;
  a.lens_out = lens_out;
  const hipStream_t s = static_cast<hipStream_t>(stream);
  const hipError_t e = sift::launch_cache_append(a, pool_of(dtype), s);
  cache->last_stream = s;
  return e == hipSuccess ? SIFT_OK : SIFT_E_HIP;
}

sift_status sift_cache_accumulate(sift_cache* cache, const sift_cache_kv* kv,
                                  const sift_cache_rows* new_rows, const sift_tensor* q,
                                  const float* lse, const float* row_weight,
                                  const sift_score* score, const float* weights, float decay,
                                  float* out, void* stream) {
  sift::CacheWeightArgs a{};
  sift_status st;
  if ((st = check_kv(cache, kv, &a.c)) != SIFT_OK) return st;
  const int32_t dtype = kv->k_pages->dtype;
  if ((st = check_rows(cache, new_rows, q, dtype, score, 1.0, &a.c)) != SIFT_OK) return st;
  if (out == nullptr || (lse == nullptr && q->tokens > 0)) return SIFT_E_NULL;
  if (!std::isfinite(decay)) return SIFT_E_UNSUPPORTED;
  if (sift::cache_weights_steps(a.c) >= int64_t(1) << 31) return SIFT_E_CAPACITY;
  a.lse = lse;
  a.row_weight = row_weight;
  a.weights = weights;
  a.out = out;
  a.decay = decay;
  const hipStream_t s = static_cast<hipStream_t>(stream);
  const hipError_t e =
      sift::launch_cache_weights(a, dtype == SIFT_BF16, cache->head_dim, cache->cus, s);
  cache->last_stream = s;
  return e == hipSuccess ? SIFT_OK : SIFT_E_HIP;
}

sift_status sift_cache_evict(sift_cache* cache, const sift_cache_kv* kv, const float* weights,
                             const int32_t* next_pos, int32_t budget, int32_t sinks,
                             int32_t recent, float* weights_out, int32_t* pos_out,
                             int32_t* lens_out, void* stream) {
  sift::CacheEvictArgs a{};
  sift_status st;
  if ((st = check_kv(cache, kv, &a.c)) != SIFT_OK) return st;
  if (weights == nullptr || weights_out == nullptr || pos_out == nullptr || lens_out == nullptr)
    return SIFT_E_NULL;
  if (budget < 1 || sinks < 0 || recent < 0 || static_cast<int64_t>(sinks) + recent > budget)
    return SIFT_E_SHAPE;
  const int64_t heads = static_cast<int64_t>(cache->num_seqs) * cache->hkv;
  const int64_t slots = static_cast<int64_t>(cache->max_pages) * cache->page;
  const size_t bytes = static_cast<size_t>(heads * slots) * 4;
  if (overlap(weights_out, weights, bytes) || overlap(weights_out, kv->key_pos, bytes) ||
      overlap(pos_out, weights, bytes) || overlap(pos_out, kv->key_pos, bytes) ||
      overlap(pos_out, weights_out, bytes))
    return SIFT_E_UNSUPPORTED;
  const size_t small = static_cast<size_t>(cache->num_seqs) * 4;
  if (overlap(lens_out, kv->lens, small) || overlap(lens_out, next_pos, small))
    return SIFT_E_UNSUPPORTED;
  if (heads >= int64_t(1) << 22 || heads * slots >= int64_t(1) << 33) return SIFT_E_CAPACITY;
  a.weights = weights;
  a.next_pos = next_pos;
  a.budget = budget;
  a.sinks = sinks;
  a.recent = recent;
  a.weights_out = weights_out;
  a.pos_out = pos_out;
  a.lens_out = lens_out;
  a.moves = cache->moves;
  a.num_moves = cache->num_moves;
  a.hist = cache->hist;
  a.state = cache->state;
  a.counts = cache->counts;
  const hipStream_t s = static_cast<hipStream_t>(stream);
  const int row = cache->head_dim * (kv->k_pages->dtype == SIFT_BF16 ? 2 : 4);
  const hipError_t e = sift::launch_cache_evict(a, row, s);
  cache->last_stream = s;
  return e == hipSuccess ? SIFT_OK : SIFT_E_HIP;
}

}  // extern "C"
