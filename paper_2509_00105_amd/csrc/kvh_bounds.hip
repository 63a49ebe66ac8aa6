// kvh_bound_keys: the lowest and highest key of each channel, page by page.
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

// Values of 16 bytes of the cache.
template <int DT, int KIND, int N>
__device__ __forceinline__ void values(const u32x4& w, float (&x)[N]) {
  if constexpr (KIND == KVH_CACHE_16) {
    widen8<DT>(w, x);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (KIND == KVH_CACHE_I8) {
#pragma unroll
        for (int e = 0; e < 4; ++e) x[4 * i + e] = (float)(int8_t)(w[i] >> 8 * e);
      } else {
        x[4 * i] = __builtin_amdgcn_cvt_f32_fp8((int)w[i], 0);
        x[4 * i + 1] = __builtin_amdgcn_cvt_f32_fp8((int)w[i], 1);
        x[4 * i + 2] = __builtin_amdgcn_cvt_f32_fp8((int)w[i], 2);
        x[4 * i + 3] = __builtin_amdgcn_cvt_f32_fp8((int)w[i], 3);
      }
    }
  }
}

// A wave takes 1 KiB of the channels of a page: a lane 16 bytes of each token.
template <int DT, int KIND, int D>
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
  float lo[kPer], hi[kPer];
#pragma unroll
  for (int e = 0; e < kPer; ++e) lo[e] = INFINITY, hi[e] = -INFINITY;
  bool odd = false;
  for (int r0 = 0; r0 < rows; r0 += kAtOnce) {
    u32x4 w[kAtOnce];
#pragma unroll
    for (int i = 0; i < kAtOnce; ++i) {
      const int r = r0 + i < rows ? r0 + i : rows - 1;  // the last one stands for those behind it
      w[i] = *reinterpret_cast<const u32x4*>(src + (int64_t)r * a.c_ts * kWidth);
    }
#pragma unroll
    for (int i = 0; i < kAtOnce; ++i) {
      float x[kPer];
      values<DT, KIND>(w[i], x);
#pragma unroll
      for (int e = 0; e < 4; ++e) odd |= has_odd<DT, KIND>(w[i][e]);
#pragma unroll
      for (int e = 0; e < kPer; ++e) lo[e] = fminf(lo[e], x[e]), hi[e] = fmaxf(hi[e], x[e]);
    }
  }
  float most = 0.0f;
#pragma unroll
  for (int e = 0; e < kPer; ++e) most = fmaxf(most, fmaxf(fabsf(lo[e]), fabsf(hi[e])));
#pragma unroll
  for (int d = 1; d < kLanes; d *= 2) most = fmaxf(most, __shfl_xor(most, d));
  const uint64_t lanes = ((uint64_t)1 << kLanes) - 1;
  odd = (__ballot(odd) >> (lane & ~(kLanes - 1)) & lanes) != 0;
  const bool none = odd || most < 0x1p-100f;
  const Part127 part127(none ? 1.0f : most);
  int8_t* to = a.codes + layer * a.b_ls + (int64_t)page * a.b_ps + (int64_t)head * 2 * D + ch % D;
  if (mine) {
    uint32_t low[kPer / 4], high[kPer / 4];
#pragma unroll
    for (int i = 0; i < kPer / 4; ++i) {
      float l[4], h[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        l[e] = none ? 0.0f : __builtin_floorf(part127.of(lo[4 * i + e]));
        h[e] = none ? 0.0f : __builtin_ceilf(part127.of(hi[4 * i + e]));
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

template <int DT, int KIND>
void launch_bound_dim(const BoundParams& a, int head_dim, dim3 grid, hipStream_t stream) {
  if (head_dim == 128)
    launch_kernel(bound_kernel<DT, KIND, 128>, grid, dim3(kBlockThreads), 0, stream, a);
  else
    launch_kernel(bound_kernel<DT, KIND, 64>, grid, dim3(kBlockThreads), 0, stream, a);
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
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (cache->kind == KVH_CACHE_I8)
    launch_bound_dim<KVH_F16, KVH_CACHE_I8>(a, cache->head_dim, grid, s);
  else if (cache->kind == KVH_CACHE_E4M3)
    launch_bound_dim<KVH_F16, KVH_CACHE_E4M3>(a, cache->head_dim, grid, s);
  else if (dt == KVH_F16)
    launch_bound_dim<KVH_F16, KVH_CACHE_16>(a, cache->head_dim, grid, s);
  else
    launch_bound_dim<KVH_BF16, KVH_CACHE_16>(a, cache->head_dim, grid, s);
  KVH_HIP_CHECK_LAUNCH();
  return KVH_OK;
}
