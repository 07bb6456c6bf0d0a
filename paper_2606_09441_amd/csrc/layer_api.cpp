// C ABI of the pieces the decoder-layer prefill slice adds around the sparse
// attention: the rotary position embedding (rope.hip; rotary.hip for any table,
// layout and part of the head), the norms and the SwiGLU product (layer_ops.hip).
// The projections are library GEMMs called by the caller.

#include <hip/hip_runtime.h>

#include <cstdint>

#include "layer_api.h"
#include "rotary_api.h"
#include "sift.h"
#include "sift_internal.h"
#include "sift_serve.h"

namespace {
bool aligned16(const void* p) { return reinterpret_cast<uintptr_t>(p) % 16 == 0; }

// Whether two buffers of a and b bytes share one.
bool overlap(const void* p, size_t a, const void* q, size_t b) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(p), y = reinterpret_cast<uintptr_t>(q);
  return a > 0 && b > 0 && x < y + b && y < x + a;
}

// An input of sift_rotate and its output, which is the same buffer or one apart.
sift_status check_turned(const sift_tensor* t, const sift_tensor* out, const sift_tensor* q) {
  if (t == nullptr || out == nullptr) return SIFT_E_NULL;
  if (t->tokens < 0 || t->heads < 1 || t->head_dim < 1) return SIFT_E_SHAPE;
  if (t->tokens > 0 && (t->data == nullptr || out->data == nullptr)) return SIFT_E_NULL;
  if (t->dtype != SIFT_F32 && t->dtype != SIFT_BF16) return SIFT_E_UNSUPPORTED;
  if (t->tokens != q->tokens || t->head_dim != q->head_dim || out->tokens != t->tokens ||
      out->heads != t->heads || out->head_dim != t->head_dim)
    return SIFT_E_SHAPE;
  if (t->dtype != q->dtype || out->dtype != t->dtype) return SIFT_E_UNSUPPORTED;
  return SIFT_OK;
}

size_t bytes_of(const sift_tensor* t) {
  return static_cast<size_t>(t->tokens) * t->heads * t->head_dim * (t->dtype == SIFT_F32 ? 4 : 2);
}
}  // namespace

extern "C" {

sift_status sift_rope(const sift_tensor* q, const sift_tensor* k, const int32_t* positions,
                      const float* inv_freq, void* stream) {
  if (q == nullptr || k == nullptr) return SIFT_E_NULL;
  if (q->tokens > 0 && (q->data == nullptr || k->data == nullptr || positions == nullptr ||
                        inv_freq == nullptr))
    return SIFT_E_NULL;
  if (q->tokens != k->tokens || q->tokens < 0) return SIFT_E_SHAPE;
  if (q->head_dim != k->head_dim || q->heads < 1 || k->heads < 1) return SIFT_E_SHAPE;
  if (q->dtype != SIFT_BF16 || k->dtype != SIFT_BF16) return SIFT_E_UNSUPPORTED;
  if (q->head_dim < 2 || q->head_dim % 2 != 0) return SIFT_E_UNSUPPORTED;
  if (q->tokens == 0) return SIFT_OK;
  const hipError_t e = sift::launch_rope(q->data, q->tokens, q->heads, k->data, k->heads,
                                         q->head_dim, positions, inv_freq,
                                         static_cast<hipStream_t>(stream));
  return e == hipSuccess ? SIFT_OK : SIFT_E_HIP;
}

sift_status sift_rotate(const sift_tensor* q, const sift_tensor* k, const int32_t* positions,
                        const sift_rotary* rotary, int32_t back, sift_tensor* q_out,
                        sift_tensor* k_out, void* stream) {
  if (q == nullptr || rotary == nullptr) return SIFT_E_NULL;
  sift_status st;
  if ((st = check_turned(q, q_out, q)) != SIFT_OK) return st;
  if ((k == nullptr) != (k_out == nullptr)) return SIFT_E_NULL;
  if (k != nullptr && (st = check_turned(k, k_out, q)) != SIFT_OK) return st;
  sift::RotateArgs a{};
  if ((st = sift::make_rotary(rotary, q->head_dim, &a.r)) != SIFT_OK) return st;
  if (q->tokens > 0 && positions == nullptr) return SIFT_E_NULL;
  const int64_t heads = static_cast<int64_t>(q->heads) + (k != nullptr ? k->heads : 0);
  if (heads >= (int64_t(1) << 31) / q->head_dim) return SIFT_E_CAPACITY;  // 32-bit indexes
  const size_t qn = bytes_of(q), kn = k != nullptr ? bytes_of(k) : 0;
  if (q_out->data != q->data && overlap(q->data, qn, q_out->data, qn)) return SIFT_E_UNSUPPORTED;
  if (k != nullptr && ((k_out->data != k->data && overlap(k->data, kn, k_out->data, kn)) ||
                       overlap(k->data, kn, q_out->data, qn) ||
                       overlap(q->data, qn, k_out->data, kn) ||
                       overlap(q_out->data, qn, k_out->data, kn)))
    return SIFT_E_UNSUPPORTED;
  a.r.back = back != 0;
  a.q = q->data;
  a.q_out = q_out->data;
  a.hq = q->heads;
  if (k != nullptr) {
    a.k = k->data;
    a.k_out = k_out->data;
    a.hk = k->heads;
  }
  a.positions = positions;
  a.tokens = q->tokens;
  a.d = q->head_dim;
  a.copy = a.q != a.q_out || a.k != a.k_out;
  const hipError_t e =
      sift::launch_rotate(a, q->dtype == SIFT_BF16, static_cast<hipStream_t>(stream));
  return e == hipSuccess ? SIFT_OK : SIFT_E_HIP;
}

sift_status sift_layer_rms_norm(const void* x, const void* weight, int64_t rows, int32_t width,
                                float eps, void* out, void* stream) {
  if (rows < 0 || width < 1) return SIFT_E_SHAPE;
  if (rows == 0) return SIFT_OK;
  if (x == nullptr || weight == nullptr || out == nullptr) return SIFT_E_NULL;
  if (width % 8 != 0 || width > sift::kMaxNormWidth) return SIFT_E_UNSUPPORTED;
  if (!aligned16(x) || !aligned16(weight) || !aligned16(out)) return SIFT_E_UNSUPPORTED;
  if (rows >= int64_t(1) << 24) return SIFT_E_CAPACITY;  // a grid holds fewer than 2^32 threads
  const hipError_t e = sift::launch_rms_norm(x, weight, rows, width, eps, out,
                                             static_cast<hipStream_t>(stream));
  return e == hipSuccess ? SIFT_OK : SIFT_E_HIP;
}

sift_status sift_layer_silu_mul(const void* gate, const void* up, int64_t count, void* out,
                                void* stream) {
  if (count < 0) return SIFT_E_SHAPE;
  if (count == 0) return SIFT_OK;
  if (gate == nullptr || up == nullptr || out == nullptr) return SIFT_E_NULL;
  if (count % 8 != 0 || !aligned16(gate) || !aligned16(up) || !aligned16(out))
    return SIFT_E_UNSUPPORTED;
  const hipError_t e =
      sift::launch_silu_mul(gate, up, count, out, static_cast<hipStream_t>(stream));
  return e == hipSuccess ? SIFT_OK : SIFT_E_HIP;
}

}  // extern "C"
