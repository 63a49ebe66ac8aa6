// kvh_bound_keys: the lowest and highest key of each channel, page by page.  kvh_select_pages: the pages that a token's queries may find large
// products on, by a score from these bounds.
//
// A key k of the page lies in the box [lowest, highest], so q . k <= sum_d max(q_d lowest_d, q_d highest_d) = q- . lowest + q+ . highest with
// q- = min(q, 0) and q+ = max(q, 0): a matrix product with rows [q-, q+] and columns [lowest, highest] of 2 D bytes, which is how a page's bounds lie in memory.
// Both are int8, so the 16x16x64 products are exact and the same in any order.
#include "kvh_cache.hpp"

#include <algorithm>

namespace kvh {
namespace {

typedef int32_t i32x4 __attribute__((ext_vector_type(4)));

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

__device__ __forceinline__ uint32_t four_codes(float a, float b, float c, float d) {
  return ((uint32_t)(int)a & 0xffu) | ((uint32_t)(int)b & 0xffu) << 8 | ((uint32_t)(int)c & 0xffu) << 16 | (uint32_t)(int)d << 24;
}

// 127 x / a for |x| <= a, rounded once: x has 11 bits at most, so 127/128 of it is exact, and a >= 2^-100.
struct Part127 {
  float by;
  __device__ __forceinline__ explicit Part127(float a) : by(a * (1.0f / 128.0f)) {}
  __device__ __forceinline__ float of(float x) const { return x * (127.0f / 128.0f) / by; }
};

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

// ---- selection ----------------------------------------------------------------------------------------------------
// A page's score as a number whose order is the scores': 0 for a page that is no candidate, kAlways for one that is chosen in any case.
constexpr uint32_t kAlways = 0xffffffffu, kInfinite = 0xff800000u;

__device__ __forceinline__ uint32_t order_of(float score) {
  const uint32_t w = __builtin_bit_cast(uint32_t, score + 0.0f);  // the two zeros are one
  return (w >> 31) != 0 ? ~w : w | 0x80000000u;
}

struct SelectParams {
  Requests req;
  const uint16_t* q;
  int64_t q_ts;
  const int8_t* codes;  // of the layer
  const float* scale;
  int64_t b_ps, bs_ps;
  int pages, block_tokens, heads, group, first, last, count;
  int32_t* out;
  int32_t* status;
  uint32_t* keys;   // [token of this turn][head][table_pages, rounded up to 4]
  int64_t pitch;    // of a token and head
  int token0;       // the turn's first token
  uint32_t tiles;   // of pages, in a row of the table
  Divisor by_block, by_heads, by_tiles;
};

constexpr int kTilePages = 64;  // that a block scores: 16 each wave

// Rows of up to 16 query heads of one token, as the product's rows: lane l holds row l % 16, bytes 64 kk + 16 (l / 16) and on of [q-, q+].
template <int DT, int D>
struct Queries {
  static constexpr int kSums = 2 * D / 64;
  i32x4 code[kSums];
  float size;  // a_u of the lane's row; 0 where it counts as zeros

  __device__ __forceinline__ void load(const uint16_t* row, bool real, int grp) {
    constexpr int kSets = D / 64;  // of 16 channels that the lane holds, for q- and again for q+
    u32x4 raw[kSets][2];
    float most = 0.0f;
    bool odd = false;
#pragma unroll
    for (int i = 0; i < kSets; ++i)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        raw[i][h] = u32x4{0, 0, 0, 0};
        if (real) raw[i][h] = *reinterpret_cast<const u32x4*>(row + i * 64 + grp * 16 + h * 8);
        float x[8];
        widen8<DT>(raw[i][h], x);
#pragma unroll
        for (int e = 0; e < 8; ++e) most = fmaxf(most, fabsf(x[e]));
#pragma unroll
        for (int e = 0; e < 4; ++e) odd |= has_odd<DT, KVH_CACHE_16>(raw[i][h][e]);
      }
    if (odd) most = INFINITY;
    most = fmaxf(most, __shfl_xor(most, 16));
    most = fmaxf(most, __shfl_xor(most, 32));
    const bool none = !(most < INFINITY) || most < 0x1p-100f;
    size = none ? 0.0f : most;
    const Part127 part127(none ? 1.0f : most);
#pragma unroll
    for (int i = 0; i < kSets; ++i) {
      float c[16];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        float x[8];
        widen8<DT>(raw[i][h], x);
#pragma unroll
        for (int e = 0; e < 8; ++e) c[8 * h + e] = none ? 0.0f : __builtin_rintf(part127.of(x[e]));
      }
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        const float *v = c + 4 * w;
        code[i][w] = (int32_t)four_codes(fminf(v[0], 0.0f), fminf(v[1], 0.0f), fminf(v[2], 0.0f), fminf(v[3], 0.0f));
        code[i + kSets][w] = (int32_t)four_codes(fmaxf(v[0], 0.0f), fmaxf(v[1], 0.0f), fmaxf(v[2], 0.0f), fmaxf(v[3], 0.0f));
      }
    }
  }
};

template <int DT, int D>
__global__ __launch_bounds__(kBlockThreads) void score_kernel(SelectParams a) {
  constexpr int kSums = 2 * D / 64;
  const int lane = threadIdx.x % kWave, wave = uniform((int32_t)(threadIdx.x / kWave)), l16 = lane % 16, grp = lane / 16;
  if (a.token0 == 0) tell_refused(a.req, a.status);
  const uint32_t unit = a.by_tiles.quotient(blockIdx.x), tile = blockIdx.x - unit * a.tiles;
  const uint32_t token = a.by_heads.quotient(unit);
  const int head = (int)(unit - token * a.heads), row = a.token0 + (int)token;
  int b;
  Request rq;
  if (!request_of(a.req, row, lane, b, rq)) return;
  const int p = rq.len - rq.n + (row - rq.start);
  if (p < 0) return;
  const int end = (int)a.by_block.quotient((uint32_t)p) + 1;
  const int j0 = (int)tile * kTilePages + wave * 16;
  if (j0 >= end) return;
  const int j = j0 + l16;
  int page = -1;
  if (j < end) page = a.req.table[(int64_t)b * a.req.table_stride + j];
  const bool there = page >= 0 && page < a.pages;
  if (__any(j < end && !there) && lane == 0 && a.status != nullptr) a.status[b] = KVH_DEV_BAD_REQUEST;
  const int8_t* from = a.codes + (int64_t)(there ? page : 0) * a.b_ps + (int64_t)head * 2 * D + grp * 16;
  i32x4 box[kSums];
#pragma unroll
  for (int kk = 0; kk < kSums; ++kk) box[kk] = *reinterpret_cast<const i32x4*>(from + kk * 64);
  const float scale = a.scale[(int64_t)(there ? page : 0) * a.bs_ps + head];
  float best = -INFINITY;
  for (int u0 = 0; u0 < a.group; u0 += 16) {
    Queries<DT, D> q;
    const bool real = u0 + l16 < a.group;
    q.load(a.q + (int64_t)row * a.q_ts + ((int64_t)head * a.group + u0 + (real ? l16 : 0)) * D, real, grp);
    i32x4 dot = {0, 0, 0, 0};
#pragma unroll
    for (int kk = 0; kk < kSums; ++kk) dot = __builtin_amdgcn_mfma_i32_16x16x64_i8(q.code[kk], box[kk], dot, 0, 0, 0);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float size = __shfl(q.size, grp * 4 + i);
      if (u0 + grp * 4 + i < a.group) best = fmaxf(best, (float)dot[i] * size);
    }
  }
  best = fmaxf(best, __shfl_xor(best, 16));
  best = fmaxf(best, __shfl_xor(best, 32));
  if (grp == 0 && j < end) {
    const float score = best * scale;
    uint32_t key = !(score == score) || !(fabsf(scale) < INFINITY) ? kInfinite : order_of(score);
    if (j < a.first || j >= end - a.last) key = kAlways;
    a.keys[((int64_t)token * a.heads + head) * a.pitch + j] = there ? key : 0;
  }
}

// Chooses among `n` keys: those above the threshold, and the first ones of those that are equal to it.
__global__ __launch_bounds__(kBlockThreads) void pick_kernel(SelectParams a) {
  __shared__ uint32_t bins[256];
  __shared__ uint32_t found[2], more[kWavesPerBlock], same[kWavesPerBlock];
  const int lane = threadIdx.x % kWave, wave = uniform((int32_t)(threadIdx.x / kWave));
  const uint32_t token = a.by_heads.quotient(blockIdx.x);
  const int head = (int)(blockIdx.x - token * a.heads), row = a.token0 + (int)token;
  int b;
  Request rq;
  if (!request_of(a.req, row, lane, b, rq)) return;
  const int p = rq.len - rq.n + (row - rq.start);
  const int n = p < 0 ? 0 : (int)a.by_block.quotient((uint32_t)p) + 1;
  const uint32_t* keys = a.keys + ((int64_t)token * a.heads + head) * a.pitch;
  int32_t* out = a.out + ((int64_t)row * a.heads + head) * a.count;
  // The threshold's digits, 8 bits at a time from the top: `want` is how many are still to be chosen among the keys that begin with `top`.
  uint32_t top = 0, want = (uint32_t)a.count;
  if (n > a.count) {
    for (int shift = 24; shift >= 0; shift -= 8) {
      bins[threadIdx.x] = 0;
      __syncthreads();
      for (int j = threadIdx.x; j < n; j += kBlockThreads) {
        const uint32_t key = keys[j];
        if (shift == 24 || key >> (shift + 8) == top) atomicAdd(&bins[key >> shift & 255u], 1u);
      }
      __syncthreads();
      if (wave == 0) {  // the bin of the want-th from above: lane l has bins 4 l .. 4 l + 3
        uint32_t mine[4], sum = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) sum += mine[i] = bins[4 * lane + i];
        uint32_t above = sum;  // of this lane and those behind it
#pragma unroll
        for (int d = 1; d < kWave; d *= 2) {
          const uint32_t x = __shfl_down(above, d);
          if (lane + d < kWave) above += x;
        }
        uint32_t past = above - sum;
#pragma unroll
        for (int i = 3; i >= 0; --i) {
          if (past < want && past + mine[i] >= want) found[0] = 4 * lane + i, found[1] = want - past;
          past += mine[i];
        }
      }
      __syncthreads();
      top = top << 8 | found[0], want = found[1];
    }
  }
  // n <= count: all candidates are above 0.
  const uint32_t least = top;
  if (least == 0) want = 0;  // keys of 0 are no candidates
  const int each = ((n + kWavesPerBlock - 1) / kWavesPerBlock + kWave - 1) / kWave * kWave;  // keys of a wave, one after the other
  const int begin = wave * each, stop = begin + each < n ? begin + each : n;
  uint32_t m = 0, s = 0;
  for (int j = begin; j < stop; j += kWave) {
    const uint32_t key = j + lane < stop ? keys[j + lane] : 0;
    m += __popcll(__ballot(key > least));
    s += __popcll(__ballot(key == least && j + lane < stop));
  }
  if (lane == 0) more[wave] = m, same[wave] = s;
  __syncthreads();
  uint32_t at = 0, equal = 0, total = 0, all_equal = 0;
  for (int w = 0; w < kWavesPerBlock; ++w) {
    if (w == wave) at = total, equal = all_equal;
    total += more[w], all_equal += same[w];
  }
  at += equal < want ? equal : want;
  total += all_equal < want ? all_equal : want;
  const uint64_t before = ((uint64_t)1 << lane) - 1;
  for (int j = begin; j < stop; j += kWave) {
    const uint32_t key = j + lane < stop ? keys[j + lane] : 0;
    const bool is = key == least && j + lane < stop;
    const uint64_t eq = __ballot(is);
    const bool take = key > least || (is && equal + __popcll(eq & before) < want);
    const uint64_t taken = __ballot(take);
    if (take) out[at + __popcll(taken & before)] = j + lane;
    at += __popcll(taken), equal += __popcll(eq);
  }
  for (int i = (int)total + threadIdx.x; i < a.count; i += kBlockThreads) out[i] = -1;
}

constexpr int kMostListed = 4096;
int64_t pitch_of(int table_pages) { return ((int64_t)table_pages + 3) & ~(int64_t)3; }

}  // namespace
}  // namespace kvh

using namespace kvh;

extern "C" {

int kvh_bound_keys(const kvh_cache* cache, const kvh_requests* requests, kvh_dtype dt, const kvh_bounds* bounds, int32_t* status_dev, void* stream) {
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

size_t kvh_select_workspace(int n_requests, int n_tokens, int heads, int table_pages) {
  if (n_requests < 1 || n_requests > kMaxRequests || n_tokens < 1 || heads < 1 || heads > 4096 || table_pages < 1) return 0;
  const size_t token = (size_t)heads * pitch_of(table_pages) * sizeof(uint32_t), most = (size_t)64 << 20;
  return std::max(token, std::min((size_t)n_tokens, most / token) * token);
}

int kvh_select_pages(const kvh_bounds* bounds, int layer, const kvh_requests* requests, kvh_dtype dt, const kvh_rows* q, int q_heads, int first, int last,
                     int count, int32_t* pages_dev, void* workspace_dev, size_t workspace_bytes, int32_t* status_dev, void* stream) {
  if ((dt != KVH_F16 && dt != KVH_BF16) || q == nullptr || (pages_dev == nullptr && requests != nullptr && requests->n_tokens != 0)) return KVH_E_ARG;
  if (int rc = check_bounds(bounds)) return rc;
  if (int rc = check_requests(requests)) return rc;
  if (layer < 0 || layer >= bounds->layers || !heads_fit(bounds->heads, q_heads)) return KVH_E_SHAPE;
  if (int rc = check_rows(q, (int64_t)q_heads * bounds->head_dim, requests->n_tokens)) return rc;
  if (first < 0 || last < 1 || count < 1 || count > kMostListed || first > count - last) return KVH_E_ARG;
  if (!is_aligned16(workspace_dev) || (reinterpret_cast<uintptr_t>(pages_dev) & 3u) != 0) return KVH_E_ALIGN;
  if (requests->n_tokens == 0) return KVH_OK;
  SelectParams a{};
  a.req = Requests(*requests, bounds->block_tokens);
  if (a.req.max_new > a.req.n_tokens) a.req.max_new = a.req.n_tokens;
  a.q = static_cast<const uint16_t*>(q->p), a.q_ts = q->token_stride;
  a.codes = bounds->codes + layer * bounds->layer_stride, a.scale = bounds->scale + layer * bounds->scale_layer_stride;
  a.b_ps = bounds->page_stride, a.bs_ps = bounds->scale_page_stride;
  a.pages = bounds->pages, a.block_tokens = bounds->block_tokens, a.heads = bounds->heads, a.group = q_heads / bounds->heads;
  a.first = first, a.last = last, a.count = count;
  a.out = pages_dev, a.status = status_dev;
  a.keys = static_cast<uint32_t*>(workspace_dev);
  a.pitch = pitch_of(requests->table_pages);
  a.tiles = (uint32_t)((requests->table_pages + kTilePages - 1) / kTilePages);
  a.by_block = Divisor((uint32_t)bounds->block_tokens), a.by_heads = Divisor((uint32_t)bounds->heads), a.by_tiles = Divisor(a.tiles);
  const int64_t token = (int64_t)a.heads * a.pitch * sizeof(uint32_t);
  int64_t turn = workspace_dev == nullptr ? 0 : (int64_t)(workspace_bytes / (size_t)token);
  if (turn < 1) return KVH_E_SIZE;
  if ((int64_t)a.heads * a.tiles >= (int64_t)1 << 31) return KVH_E_SHAPE;
  turn = std::min({turn, (int64_t)requests->n_tokens, (((int64_t)1 << 31) - 1) / ((int64_t)a.heads * a.tiles)});
  hipStream_t s = static_cast<hipStream_t>(stream);
  for (int64_t t0 = 0; t0 < requests->n_tokens; t0 += turn) {
    a.token0 = (int)t0;
    const int64_t units = std::min<int64_t>(turn, requests->n_tokens - t0) * a.heads;
    const dim3 scores((unsigned)(units * a.tiles)), picks((unsigned)units);
    if (dt == KVH_F16 && bounds->head_dim == 128)
      launch_kernel(score_kernel<KVH_F16, 128>, scores, dim3(kBlockThreads), 0, s, a);
    else if (dt == KVH_F16)
      launch_kernel(score_kernel<KVH_F16, 64>, scores, dim3(kBlockThreads), 0, s, a);
    else if (bounds->head_dim == 128)
      launch_kernel(score_kernel<KVH_BF16, 128>, scores, dim3(kBlockThreads), 0, s, a);
    else
      launch_kernel(score_kernel<KVH_BF16, 64>, scores, dim3(kBlockThreads), 0, s, a);
    KVH_HIP_CHECK_LAUNCH();
    hipLaunchKernelGGL(pick_kernel, picks, dim3(kBlockThreads), 0, s, a);
    KVH_HIP_CHECK_LAUNCH();
  }
  return KVH_OK;
}

}  // extern "C"
