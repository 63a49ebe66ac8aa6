// Shared pieces of the serving-cache calls (kvh_append, kvh_attention): argument checks, the requests as the kernels see
// them, conversions.  These sources are compiled with NaN honoured: what a caller's cache holds is not ours to choose.
#pragma once

#include "kvh_common.hpp"

#include <cmath>

namespace kvh {

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

constexpr int kMaxRequests = 65535;
constexpr int64_t kMaxLength = INT32_MAX - 127;  // tokens of a request: the number past a step or tile that begins below it is an int32 too
constexpr int64_t kMaxRowStride = 1 << 20;  // elements: lane offsets inside a tile stay far below 2^31 bytes

inline bool is_aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

inline int check_cache(const kvh_cache* c) {
  if (c == nullptr || c->k == nullptr || c->v == nullptr) return KVH_E_ARG;
  if (c->kind != KVH_CACHE_16 && c->kind != KVH_CACHE_I8 && c->kind != KVH_CACHE_E4M3) return KVH_E_ARG;
  const bool coded = c->kind != KVH_CACHE_16;
  if (coded != (c->k_scale != nullptr) || coded != (c->v_scale != nullptr)) return KVH_E_ARG;
  if (c->head_dim != 64 && c->head_dim != 128) return KVH_E_SHAPE;
  if (c->layers < 1 || c->layers > 32767 || c->pages < 1 || c->heads < 1 || c->heads > 4096) return KVH_E_SHAPE;
  if (c->block_tokens < 1) return KVH_E_ARG;
  if (c->layer_stride < 0 || c->token_stride < (int64_t)c->heads * c->head_dim || c->token_stride >= kMaxRowStride) return KVH_E_ARG;
  if (coded && (c->scale_layer_stride < 0 || c->scale_page_stride < c->heads)) return KVH_E_ARG;
  const int64_t unit = coded ? 16 : 8;
  if (!is_aligned16(c->k) || !is_aligned16(c->v) || c->layer_stride % unit != 0 || c->token_stride % unit != 0) return KVH_E_ALIGN;
  if (coded && (((uintptr_t)c->k_scale | (uintptr_t)c->v_scale) & 3u) != 0) return KVH_E_ALIGN;
  return KVH_OK;
}

inline int check_requests(const kvh_requests* r) {
  if (r == nullptr || r->starts == nullptr || r->lens == nullptr || r->page_table == nullptr) return KVH_E_ARG;
  if (r->n_requests < 1 || r->n_requests > kMaxRequests || r->max_new < 1 || r->n_tokens < 0) return KVH_E_ARG;
  if (r->table_pages < 1 || r->table_stride < 0) return KVH_E_ARG;
  return KVH_OK;
}

inline int check_rows(const kvh_rows* r, int64_t channels, int n_tokens) {
  if ((r->p == nullptr && n_tokens != 0) || r->layer_stride < 0 || r->token_stride < channels) return KVH_E_ARG;
  if (!is_aligned16(r->p) || r->layer_stride % 8 != 0 || r->token_stride % 8 != 0) return KVH_E_ALIGN;
  return KVH_OK;
}

// The requests as the kernels see them.
struct Requests {
  const int32_t* starts;
  const int32_t* lens;
  const int32_t* table;
  int64_t table_stride;
  int32_t table_pages, n, max_new, n_tokens;
  int64_t capacity;  // tokens a row of the table has pages for, and a request may have
  explicit Requests(const kvh_requests& r, int block_tokens)
      : starts(r.starts), lens(r.lens), table(r.page_table), table_stride(r.table_stride), table_pages(r.table_pages), n(r.n_requests),
        max_new(r.max_new), n_tokens(r.n_tokens), capacity((int64_t)r.table_pages * block_tokens < kMaxLength ? (int64_t)r.table_pages * block_tokens : kMaxLength) {}
  Requests() = default;
};

struct Request {
  int32_t start, n, len;
  bool ok;
};

// Whether a request is one that the call can serve: see include/kvh.h.
__device__ __forceinline__ bool request_ok(const Requests& r, int32_t start, int32_t end, int32_t len) {
  return start >= 0 && end >= start && end <= r.n_tokens && end - start <= r.max_new && len >= 0 && len <= r.capacity;
}

// 8 values of 16 bits <-> fp32.
template <int DT>
__device__ __forceinline__ void widen8(const u32x4& w, float (&x)[8]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = t16_to_f32<DT>(w[i] & 0xffffu);
    x[2 * i + 1] = t16_to_f32<DT>(w[i] >> 16);
  }
}

// Two values rounded to nearest even in one instruction; a NaN stays one.
template <int DT>
__device__ __forceinline__ uint32_t narrow2(float a, float b) {
  const f32x2 v = {a, b};
  if constexpr (DT == KVH_F16)
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, f16x2));
  else
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, bf16x2));
}

}  // namespace kvh
