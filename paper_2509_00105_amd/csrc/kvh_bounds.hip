// kvh_bound_keys: the lowest and highest key of each channel, page by page.
//
// Every page that new tokens lie on is read as a whole from the cache, so that nothing is kept from call to call and a call can be repeated: that is 16 tokens for one
// at most, and no more than what was appended where whole pages are new.  Extremes are found two at a time among whole numbers of 16 bits in the values' order.  Memory
// bounds it, or the launch: 32 layers of 8192 tokens, int8: 55 us = 5.5 TB/s (a plain read reaches 6.5); 64 single tokens, bf16: 4.9 us.
#include "kvh_bounds.hpp"

#include <algorithm>

namespace kvh {
namespace {

// ---- bounds -------------------------------------------------------------------------------------------------------
struct BoundParams {
  Requests req;
  const uint8_t* ck;
  const float* sk;
  int64_t c_ls, c_ts, s_ls, s_ps;  // of the cache: elements; floats
  int8_t* codes;
  float* scale;
  int64_t b_ls, b_ps, bs_ls, bs_ps;  // of the bounds
  int pages, block_tokens, heads;
  int32_t* status;
  uint32_t units, strips;  // of a request and layer; of a page
  Divisor by_block, by_strips;
};

typedef int16_t i16x2 __attribute__((ext_vector_type(2)));

// Least and greatest of several values of 16 or 8 bits, two at a time as whole numbers of 16 bits that have their order: a negative number's magnitude is
// inverted, and 8 bits are the upper half.  Infinities and NaN lie outside of all others.
template <int DT, int KIND>
struct Extremes {
  static constexpr bool kHalf = KIND == KVH_CACHE_16;
  static constexpr int kPer = kHalf ? 8 : 16;           // values of 16 bytes
  static constexpr int kWords = kHalf ? 4 : 8;          // pairs
  static constexpr int kFlip = kHalf ? 0x7fff : KIND == KVH_CACHE_I8 ? 0 : 0x7f00;
  static constexpr int kTop = kHalf ? (DT == KVH_BF16 ? 0x7f80 : 0x7c00) : KIND == KVH_CACHE_I8 ? 0x7fff : 0x7f00;  // the first that is no finite number
  i16x2 lo[kWords], hi[kWords];

  __device__ __forceinline__ Extremes() {
#pragma unroll
    for (int i = 0; i < kWords; ++i) lo[i] = i16x2{INT16_MAX, INT16_MAX}, hi[i] = i16x2{INT16_MIN, INT16_MIN};
  }
  static __device__ __forceinline__ i16x2 turn(i16x2 x) { return kFlip == 0 ? x : x ^ (x >> 15 & i16x2{(int16_t)kFlip, (int16_t)kFlip}); }
  __device__ __forceinline__ void take(int i, uint32_t w) {
    const i16x2 x = turn(__builtin_bit_cast(i16x2, w));
    lo[i] = __builtin_elementwise_min(lo[i], x), hi[i] = __builtin_elementwise_max(hi[i], x);
  }
  __device__ __forceinline__ void take(const u32x4& w) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (kHalf) {
        take(i, w[i]);
      } else {  // bytes 0 and 2, 1 and 3
        take(2 * i, (w[i] & 0x00ff00ffu) << 8);
        take(2 * i + 1, w[i] & 0xff00ff00u);
      }
    }
  }
  // Value e of the 16 bytes.
  static __device__ __forceinline__ float value(const i16x2 (&of)[kWords], int e) {
    const int i = kHalf ? e / 2 : e / 4 * 2 + e % 2, half = kHalf ? e % 2 : e / 2 % 2;
    const int16_t x = turn(of[i])[half];
    if constexpr (kHalf)
      return t16_to_f32<DT>((uint16_t)x);
    else if constexpr (KIND == KVH_CACHE_I8)
      return (float)(x >> 8);
    else
      return __builtin_amdgcn_cvt_f32_fp8((int)(uint16_t)x >> 8, 0);
  }
  __device__ __forceinline__ bool odd() const {
    bool is = false;
    if constexpr (KIND != KVH_CACHE_I8) {
#pragma unroll
      for (int i = 0; i < kWords; ++i) is |= hi[i][0] >= kTop || hi[i][1] >= kTop || lo[i][0] < -kTop || lo[i][1] < -kTop;
    }
    return is;
  }
};

// A wave takes 1 KiB of the channels of a page: a lane 16 bytes of each token.
// PAST: keys that are read once, and so many, pass by the caches.
template <int DT, int KIND, int D, bool PAST>
__global__ __launch_bounds__(kBlockThreads) void bound_kernel(BoundParams a) {
  constexpr int kWidth = KIND == KVH_CACHE_16 ? 2 : 1, kPer = 16 / kWidth;
  constexpr int kLanes = D / kPer, kAtOnce = 8;  // lanes of a head; tokens under way
  const int lane = threadIdx.x % kWave;
  const uint32_t u = uniform((int32_t)(blockIdx.x * kWavesPerBlock + threadIdx.x / kWave));
  if (u >= a.units) return;
  const int b = blockIdx.y, layer = blockIdx.z;
  const int32_t start = a.req.starts[b], end = a.req.starts[b + 1], len = a.req.lens[b], n = end - start;
  const bool tells = lane == 0 && a.status != nullptr;
  if (!request_ok(a.req, start, end, len) || len < n) {
    if (tells && u == 0) a.status[b] = KVH_DEV_BAD_REQUEST;
    return;
  }
  if (n == 0) return;
  const uint32_t part = a.by_strips.quotient(u);
  const int strip = (int)(u - part * a.strips);
  const int at = (int)a.by_block.quotient((uint32_t)(len - n)) + (int)part;  // the page's place in the request
  const int64_t first = (int64_t)at * a.block_tokens;
  if (first >= len) return;
  const int rows = len - first < a.block_tokens ? (int)(len - first) : a.block_tokens;
  const int page = uniform(a.req.table[(int64_t)b * a.req.table_stride + at]);
  if (page < 0 || page >= a.pages) {
    if (tells) a.status[b] = KVH_DEV_BAD_REQUEST;
    return;
  }
  const int ch = strip * kWave * kPer + lane * kPer, head = ch / D;
  const bool mine = head < a.heads;
  const uint8_t* src = a.ck + (layer * a.c_ls + (int64_t)page * a.block_tokens * a.c_ts + (mine ? ch : 0)) * kWidth;
  Extremes<DT, KIND> found;
  for (int r0 = 0; r0 < rows; r0 += kAtOnce) {
    u32x4 w[kAtOnce];
#pragma unroll
    for (int i = 0; i < kAtOnce; ++i) {
      const int r = r0 + i < rows ? r0 + i : rows - 1;  // the last one stands for those behind it
      const u32x4* p = reinterpret_cast<const u32x4*>(src + (int64_t)r * a.c_ts * kWidth);
      w[i] = PAST ? __builtin_nontemporal_load(p) : *p;
    }
#pragma unroll
    for (int i = 0; i < kAtOnce; ++i) found.take(w[i]);
  }
  float lo[kPer], hi[kPer];
#pragma unroll
  for (int e = 0; e < kPer; ++e) lo[e] = found.value(found.lo, e), hi[e] = found.value(found.hi, e);
  bool odd = found.odd();
  float most = 0.0f;
#pragma unroll
  for (int e = 0; e < kPer; ++e) most = fmaxf(most, fmaxf(fabsf(lo[e]), fabsf(hi[e])));
#pragma unroll
  for (int d = 1; d < kLanes; d *= 2) most = fmaxf(most, __shfl_xor(most, d));
  const uint64_t lanes = ((uint64_t)1 << kLanes) - 1;
  odd = (__ballot(odd) >> (lane & ~(kLanes - 1)) & lanes) != 0;
  const bool none = odd || most < 0x1p-100f;
  const Around127 around127(none ? 1.0f : most);
  int8_t* to = a.codes + layer * a.b_ls + (int64_t)page * a.b_ps + (int64_t)head * 2 * D + ch % D;
  if (mine) {
    uint32_t low[kPer / 4], high[kPer / 4];
#pragma unroll
    for (int i = 0; i < kPer / 4; ++i) {
      float l[4], h[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        l[e] = none ? 0.0f : around127.down(lo[4 * i + e]);
        h[e] = none ? 0.0f : around127.up(hi[4 * i + e]);
      }
      low[i] = four_codes(l[0], l[1], l[2], l[3]);
      high[i] = four_codes(h[0], h[1], h[2], h[3]);
    }
    if constexpr (kPer == 8) {
      *reinterpret_cast<u32x2*>(to) = u32x2{low[0], low[1]};
      *reinterpret_cast<u32x2*>(to + D) = u32x2{high[0], high[1]};
    } else {
      *reinterpret_cast<u32x4*>(to) = u32x4{low[0], low[1], low[2], low[3]};
      *reinterpret_cast<u32x4*>(to + D) = u32x4{high[0], high[1], high[2], high[3]};
    }
    if (ch % D == 0) {
      float s = odd ? NAN : none ? 0.0f : most / 127.0f;
      if constexpr (KIND != KVH_CACHE_16) {
        s *= a.sk[layer * a.s_ls + (int64_t)page * a.s_ps + head];
        if (!(fabsf(s) < INFINITY)) s = NAN;
      }
      a.scale[layer * a.bs_ls + (int64_t)page * a.bs_ps + head] = s;
    }
  }
}

template <int DT, int KIND, int D>
void launch_past(const BoundParams& a, bool past, dim3 grid, hipStream_t stream) {
  if (past)
    launch_kernel(bound_kernel<DT, KIND, D, true>, grid, dim3(kBlockThreads), 0, stream, a);
  else
    launch_kernel(bound_kernel<DT, KIND, D, false>, grid, dim3(kBlockThreads), 0, stream, a);
}

template <int DT, int KIND>
void launch_dim(const BoundParams& a, int head_dim, bool past, dim3 grid, hipStream_t stream) {
  if (head_dim == 128)
    launch_past<DT, KIND, 128>(a, past, grid, stream);
  else
    launch_past<DT, KIND, 64>(a, past, grid, stream);
}

}  // namespace
}  // namespace kvh

using namespace kvh;

extern "C" int kvh_bound_keys(const kvh_cache* cache, const kvh_requests* requests, kvh_dtype dt, const kvh_bounds* bounds, int32_t* status_dev, void* stream) {
  if (dt != KVH_F16 && dt != KVH_BF16) return KVH_E_ARG;
  if (int rc = check_cache(cache)) return rc;
  if (int rc = check_requests(requests)) return rc;
  if (int rc = check_bounds_of(bounds, cache)) return rc;
  if (requests->n_tokens == 0) return KVH_OK;
  BoundParams a{};
  a.req = Requests(*requests, cache->block_tokens);
  const int most = std::min(requests->max_new, requests->n_tokens);
  a.req.max_new = most;
  a.ck = static_cast<const uint8_t*>(cache->k), a.sk = cache->k_scale;
  a.c_ls = cache->layer_stride, a.c_ts = cache->token_stride, a.s_ls = cache->scale_layer_stride, a.s_ps = cache->scale_page_stride;
  a.codes = bounds->codes, a.scale = bounds->scale;
  a.b_ls = bounds->layer_stride, a.b_ps = bounds->page_stride, a.bs_ls = bounds->scale_layer_stride, a.bs_ps = bounds->scale_page_stride;
  a.pages = cache->pages, a.block_tokens = cache->block_tokens, a.heads = cache->heads;
  a.status = status_dev;
  a.by_block = Divisor((uint32_t)cache->block_tokens);
  const int per = cache->kind == KVH_CACHE_16 ? 512 : 1024;
  a.strips = (uint32_t)((cache->heads * cache->head_dim + per - 1) / per);
  a.by_strips = Divisor(a.strips);
  const int64_t spread = std::min<int64_t>(((int64_t)most + cache->block_tokens - 2) / cache->block_tokens + 1, most);
  const int64_t units = std::min<int64_t>(spread, requests->table_pages) * a.strips;  // pages that `most` tokens touch at most
  if (units >= (int64_t)1 << 31) return KVH_E_SHAPE;
  a.units = (uint32_t)units;
  const dim3 grid((unsigned)((units + kWavesPerBlock - 1) / kWavesPerBlock), (unsigned)requests->n_requests, (unsigned)cache->layers);
  // 32 layers of 8192 tokens, int8: 56 us past the caches, 67 through them; 64 single tokens: the two are alike.
  const bool past = units * requests->n_requests * cache->layers * cache->block_tokens * per >= (int64_t)8 << 20;
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (cache->kind == KVH_CACHE_I8)
    launch_dim<KVH_F16, KVH_CACHE_I8>(a, cache->head_dim, past, grid, s);
  else if (cache->kind == KVH_CACHE_E4M3)
    launch_dim<KVH_F16, KVH_CACHE_E4M3>(a, cache->head_dim, past, grid, s);
  else if (dt == KVH_F16)
    launch_dim<KVH_F16, KVH_CACHE_16>(a, cache->head_dim, past, grid, s);
  else
    launch_dim<KVH_BF16, KVH_CACHE_16>(a, cache->head_dim, past, grid, s);
  KVH_HIP_CHECK_LAUNCH();
  return KVH_OK;
}
