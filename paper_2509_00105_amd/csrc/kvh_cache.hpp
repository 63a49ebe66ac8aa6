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

inline int check_bounds(const kvh_bounds* b) {
  if (b == nullptr || b->codes == nullptr || b->scale == nullptr) return KVH_E_ARG;
  if (b->head_dim != 64 && b->head_dim != 128) return KVH_E_SHAPE;
  if (b->layers < 1 || b->layers > 32767 || b->pages < 1 || b->heads < 1 || b->heads > 4096) return KVH_E_SHAPE;
  if (b->block_tokens < 1) return KVH_E_ARG;
  if (b->layer_stride < 0 || b->page_stride < (int64_t)b->heads * 2 * b->head_dim || b->scale_layer_stride < 0 || b->scale_page_stride < b->heads) return KVH_E_ARG;
  if (!is_aligned16(b->codes) || b->layer_stride % 16 != 0 || b->page_stride % 16 != 0 || (reinterpret_cast<uintptr_t>(b->scale) & 3u) != 0) return KVH_E_ALIGN;
  return KVH_OK;
}
// Whether the bounds are those of such a cache.
inline int check_bounds_of(const kvh_bounds* b, const kvh_cache* c) {
  if (int rc = check_bounds(b)) return rc;
  return b->layers == c->layers && b->pages == c->pages && b->block_tokens == c->block_tokens && b->heads == c->heads && b->head_dim == c->head_dim ? KVH_OK : KVH_E_SHAPE;
}

inline bool heads_fit(int heads, int q_heads) { return heads >= 1 && q_heads >= heads && q_heads % heads == 0 && q_heads <= 65536; }

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

// The two values of lanes 32 apart, and of lanes 16 apart, in both: moves between lanes without LDS.
__device__ __forceinline__ f32x2 apart32(float v) {
  const auto r = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(int, v), __builtin_bit_cast(int, v), false, false);
  return f32x2{__builtin_bit_cast(float, (int)r[0]), __builtin_bit_cast(float, (int)r[1])};
}
__device__ __forceinline__ f32x2 apart16(float v) {
  const auto r = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(int, v), __builtin_bit_cast(int, v), false, false);
  return f32x2{__builtin_bit_cast(float, (int)r[0]), __builtin_bit_cast(float, (int)r[1])};
}
__device__ __forceinline__ float over_halves_max(float v) {  // of the 2 lanes that hold a row of the kernel for many rows
  const f32x2 x = apart32(v);
  return fmaxf(x[0], x[1]);
}
__device__ __forceinline__ float over_halves_sum(float v) {
  const f32x2 x = apart32(v);
  return x[0] + x[1];
}
__device__ __forceinline__ float over_groups_max(float v) {  // of the 4 lanes that hold a row of the kernel for few
  const f32x2 x = apart16(v);
  return over_halves_max(fmaxf(x[0], x[1]));
}
__device__ __forceinline__ float over_groups_sum(float v) {
  const f32x2 x = apart16(v);
  return over_halves_sum(x[0] + x[1]);
}

// Lanes of a row of 16 exchange by moves; rows through scalar registers.
template <int CTRL>
__device__ __forceinline__ uint32_t of_row(uint32_t v) { return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xf, 0xf, true); }  // 0 from past the row
constexpr int kFromAbove = 0x100, kFromBelow = 0x110;  // + n: the lane n above, n below

__device__ __forceinline__ uint32_t wave_max(uint32_t v) {
  v = max(v, of_row<kFromBelow + 1>(v));
  v = max(v, of_row<kFromBelow + 2>(v));
  v = max(v, of_row<kFromBelow + 4>(v));
  v = max(v, of_row<kFromBelow + 8>(v));
  const uint32_t a = __builtin_amdgcn_readlane(v, 15), b = __builtin_amdgcn_readlane(v, 31), c = __builtin_amdgcn_readlane(v, 47), d = __builtin_amdgcn_readlane(v, 63);
  return max(max(a, b), max(c, d));
}
// The sum of the lane's value and those of the lanes above it in its row.
__device__ __forceinline__ uint32_t row_sum_from(uint32_t v) {
  v += of_row<kFromAbove + 1>(v);
  v += of_row<kFromAbove + 2>(v);
  v += of_row<kFromAbove + 4>(v);
  v += of_row<kFromAbove + 8>(v);
  return v;
}

// The sum over the first row's lanes, where the others are of no account.
__device__ __forceinline__ uint32_t row_sum(uint32_t v) { return (uint32_t)__builtin_amdgcn_readlane((int)row_sum_from(v), 0); }

// The sum of the lane's value and those of all lanes below it, and the sum of all.
__device__ __forceinline__ uint32_t wave_sum_to(uint32_t v, uint32_t& all) {
  v += of_row<kFromBelow + 1>(v);
  v += of_row<kFromBelow + 2>(v);
  v += of_row<kFromBelow + 4>(v);
  v += of_row<kFromBelow + 8>(v);
  const uint32_t a = __builtin_amdgcn_readlane(v, 15), b = a + __builtin_amdgcn_readlane(v, 31), c = b + __builtin_amdgcn_readlane(v, 47), lane = threadIdx.x % kWave;
  all = c + __builtin_amdgcn_readlane(v, 63);
  return v + (lane < 16 ? 0 : lane < 32 ? a : lane < 48 ? b : c);
}

// The request that a row of the packed tensors belongs to, one that is not refused; all lanes of a wave ask for the same row.  False where there is none: the next row that
// one has is `next` then, INT32_MAX if none has.
__device__ __forceinline__ bool request_of(const Requests& r, int row, int lane, int& b, Request& rq, int& next) {
  // As long as starts do not fall it is the last one whose start is not past the row.
  int32_t start, end, len;
  if (r.n <= kWave) {  // all of them at once: one trip to memory, not two
    start = INT32_MAX, end = len = 0;
    if (lane < r.n) start = r.starts[lane], end = r.starts[lane + 1], len = r.lens[lane];
    const uint64_t below = __ballot(start <= row);
    b = below == 0 ? 0 : 63 - __builtin_clzll(below);
    start = __builtin_amdgcn_readlane(start, b), end = __builtin_amdgcn_readlane(end, b), len = __builtin_amdgcn_readlane(len, b);
  } else {
    int first = 0, many = r.n;
    while (many > 1) {
      const int step = (many + kWave - 1) / kWave, at = lane * step;
      const uint64_t below = __ballot(at < many && r.starts[first + at] <= row);
      const int k = below == 0 ? 0 : 63 - __builtin_clzll(below);
      first += k * step;
      many = many - k * step < step ? many - k * step : step;
    }
    b = uniform(first);
    start = uniform(r.starts[b]), end = uniform(r.starts[b + 1]), len = uniform(r.lens[b]);
  }
  rq = Request{start, end - start, len, request_ok(r, start, end, len) && start <= row && row < end};
  if (__builtin_expect(rq.ok, 1)) return true;
  // It is refused, or the row is none's, or the start of a refused request behind the row's own has led astray: all are looked at.
  uint32_t after = 0;  // the inverse of the least start past the row
#pragma unroll 1
  for (int b0 = 0; b0 < r.n; b0 += kWave) {
    const int at = b0 + lane;
    start = end = len = 0;
    if (at < r.n) start = r.starts[at], end = r.starts[at + 1], len = r.lens[at];
    const bool has = end > start && request_ok(r, start, end, len);
    const uint64_t who = __ballot(has && start <= row && row < end);
    if (who != 0) {
      const int l = __builtin_ctzll(who);
      b = b0 + l;
      start = __builtin_amdgcn_readlane(start, l);
      rq = Request{start, __builtin_amdgcn_readlane(end, l) - start, __builtin_amdgcn_readlane(len, l), true};
      return true;
    }
    if (has && start > row) after = max(after, ~(uint32_t)start);
  }
  after = wave_max(after);
  next = after == 0 ? INT32_MAX : (int)~after;
  return false;
}
__device__ __forceinline__ bool request_of(const Requests& r, int row, int lane, int& b, Request& rq) {
  int next;
  return request_of(r, row, lane, b, rq, next);
}

// Says which requests are refused; the kernels, of THREADS threads a block, pass over them.
template <int THREADS = kBlockThreads>
__device__ __forceinline__ void tell_refused(const Requests& r, int32_t* status) {
  if (blockIdx.x != 0 || status == nullptr) return;
  for (int b = threadIdx.x; b < r.n; b += THREADS)
    if (!request_ok(r, r.starts[b], r.starts[b + 1], r.lens[b])) status[b] = KVH_DEV_BAD_REQUEST;
}

// Whether a word of values holds an infinity or NaN.
template <int DT, int KIND>
__device__ __forceinline__ bool has_odd(uint32_t w) {
  if constexpr (KIND == KVH_CACHE_E4M3) {
    bool odd = false;
#pragma unroll
    for (int e = 0; e < 4; ++e) odd |= (w >> 8 * e & 0x7fu) == 0x7fu;
    return odd;
  } else if constexpr (KIND == KVH_CACHE_16) {
    constexpr uint32_t kExp = DT == KVH_BF16 ? 0x7f80u : 0x7c00u;
    return (w & kExp) == kExp || (w >> 16 & kExp) == kExp;
  } else {
    return false;
  }
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
