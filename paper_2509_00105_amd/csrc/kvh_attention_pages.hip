// kvh_attention_pages: each new token's queries over the pages that are listed for it and a KV head.
//
// The listed pages, one after the other, are a request of their own for the worker of kvh_attention: its page table is the list, looked up in the request's
// table and kept in LDS, its length ends with the last listed page, or at the token's own position where that page is the last.  The query heads of the KV head
// are the rows, 16 a tile.
//
// A token's pages are read once for its own KV head, 2 D bytes of each token at a time (of 16 bits), which memory bounds: 64 requests, 64 pages of 16 each for 8 heads of 128, bf16: 53 us =
// 4.8 TB/s (over all 4096 tokens kvh_attention takes 186), int8 and e4m3: 34 us.  Where tokens of a request read the same pages, an XCD's 4 MiB hold part of a head's: 512 tokens after
// 32768, 64 pages each at random, int8: 107 us, in which 1.07 GB are read through the caches and 0.53 come from behind them (kvh_attention: 396).  The tile has rows for other
// tokens, which have lists of their own: where neighbours choose the same pages, those are read again for each.
#include "kvh_attention_few.hpp"

#include <algorithm>

namespace kvh {
namespace {

struct ListParams {
  const int32_t* list;  // [token][head][count]; it ends at the first entry that is negative, not larger than the one before or past the token's own page
  int count;
  int row_tiles;        // of a head's query rows
  int splits;           // blocks that share a token and head
  int each;             // steps of such a share
  Divisor by_splits, by_row_tiles;
};

template <int DT, int KIND, int D, bool PAGE16>
__global__ __launch_bounds__(kFewThreads, 8 / kFewWaves) void pages_kernel(AttnParams a, ListParams x) {
  __shared__ float lds[kFewWaves * 16 * (D + 4)];
  __shared__ float lds_ml[kFewWaves][16][2];
  __shared__ int32_t entries;
  extern __shared__ int32_t pages[];
  const int lane = threadIdx.x % kWave, wave = uniform((int32_t)(threadIdx.x / kWave));
  tell_refused(a);
  const uint32_t part = x.by_splits.quotient(blockIdx.x), split = blockIdx.x - part * x.splits;
  const uint32_t unit = x.by_row_tiles.quotient(part), row_tile = part - unit * x.row_tiles;
  const uint32_t row = a.by_heads.quotient(unit);
  const int head = (int)(unit - row * a.heads);
  Item it;
  Request rq;
  if (!request_of(a.req, (int)row, lane, it.b, rq)) return;
  const int p = rq.len - rq.n + ((int)row - rq.start);
  const int own = p < 0 ? -1 : (int)a.by_block.quotient((uint32_t)p);
  const int32_t* list = x.list + ((int64_t)row * a.heads + head) * x.count;
  const int32_t* table = a.req.table + (int64_t)it.b * a.req.table_stride;
  if (threadIdx.x == 0) entries = x.count;
  __syncthreads();
  for (int i = threadIdx.x; i < x.count; i += kFewThreads) {
    const int e = list[i], before = i > 0 ? list[i - 1] : -1;
    if (e < 0 || e <= before || e > own)  // (what follows the end is anything: a negative entry may be larger than the one before)
      atomicMin(&entries, i);
    else
      pages[i] = table[e];
  }
  __syncthreads();
  const int n = uniform(entries);
  if (n < x.count && threadIdx.x == 0 && a.status != nullptr && list[n] >= 0) a.status[it.b] = KVH_DEV_BAD_REQUEST;
  int len = n * a.block_tokens;
  if (n > 0 && uniform(list[n - 1]) == own) len -= a.block_tokens - (p - own * a.block_tokens) - 1;
  it.rq.start = (int)row, it.rq.n = 1, it.rq.len = len, it.rq.ok = true;
  it.tile = (int)row_tile, it.tiles = x.row_tiles;
  it.from = (int)split * x.each, it.count = x.each;
  it.last = split == (uint32_t)x.splits - 1, it.split = x.splits > 1;
  it.slot = ((int64_t)row * x.row_tiles + row_tile) * x.splits + split;
  attend<DT, KIND, D, 1, PAGE16>(a, it, [&] { return pages; }, head, wave, lane, lds, lds_ml);
}

// Joins the parts of a query row: a wave a row.
template <int DT, int D>
__global__ __launch_bounds__(kBlockThreads) void join_kernel(AttnParams a, ListParams x) {
  constexpr int kPer = D / 64;
  const int lane = threadIdx.x % kWave, wave = uniform((int32_t)(threadIdx.x / kWave));
  const uint32_t unit = a.by_group.quotient(blockIdx.x * kWavesPerBlock + wave), u = blockIdx.x * kWavesPerBlock + wave - unit * a.group;
  const uint32_t row = a.by_heads.quotient(unit);
  const int head = (int)(unit - row * a.heads);
  if (row >= (uint32_t)a.req.n_tokens) return;
  int b;
  Request rq;
  if (!request_of(a.req, (int)row, lane, b, rq)) return;
  const int p = rq.len - rq.n + ((int)row - rq.start);
  const int32_t first = uniform(x.list[((int64_t)row * a.heads + head) * x.count]);
  const bool blind = p < 0 || first < 0 || first > (int)a.by_block.quotient((uint32_t)p);
  const int64_t slot = ((int64_t)row * x.row_tiles + (u >> 4)) * x.splits, next = (int64_t)a.heads * 16;
  const int64_t at = (slot * a.heads + head) * 16 + (u & 15);
  f32x2 ml = {-INFINITY, 0.0f};
  if (lane < x.splits) ml = *reinterpret_cast<const f32x2*>(a.part_ml + 2 * (at + lane * next));
  float m = ml[0];
#pragma unroll
  for (int d = 1; d < kWave; d *= 2) m = fmaxf(m, __shfl_xor(m, d));
  const float f = lane >= x.splits ? 0.0f : ml[0] == m ? 1.0f : __builtin_amdgcn_exp2f(ml[0] - m);
  float l = f * ml[1];
#pragma unroll
  for (int d = 1; d < kWave; d *= 2) l += __shfl_xor(l, d);
  float y[kPer];
#pragma unroll
  for (int c = 0; c < kPer; ++c) y[c] = 0.0f;
  const float* from = a.part + at * D + lane * kPer;
  for (int s = 0; s < x.splits; ++s) {
    const float by = __shfl(f, s);
#pragma unroll
    for (int c = 0; c < kPer; ++c) y[c] = __builtin_fmaf(by, from[s * next * D + c], y[c]);
  }
  const float by = 1.0f / l;
  uint16_t* to = a.out + (int64_t)row * a.o_ts + ((int64_t)head * a.group + u) * D + lane * kPer;
  if constexpr (kPer == 2)
    *reinterpret_cast<uint32_t*>(to) = blind ? 0u : narrow2<DT>(y[0] * by, y[1] * by);
  else
    *to = blind ? 0 : (uint16_t)narrow2<DT>(y[0] * by, 0.0f);
  if (a.lse != nullptr && lane == 0)
    a.lse[(int64_t)row * ((int64_t)a.heads * a.group) + (int64_t)head * a.group + u] = blind ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * kLn2;
}

// ---- launch -------------------------------------------------------------------------------------------------------
constexpr int kMostListed = 4096, kMostSplits = 64;
// Rules with both sides measured (us, 8 KV heads of 128, 32 query heads, bf16, pages of 16).  Tokens and heads are shared by blocks until there are 256 of these:
// 32 of 64 pages 31 whole and 36 in two, 4 of 256 pages (int8) 17 for 256 blocks and 21 for 512, 16 of 64 pages 21 and 22.  8 steps a block at least (one
// of 256 pages: 16.5, with 4 steps 20.6), and only where that takes 16 from a block's (one of 16 pages, 8 steps: 8.5 whole, 11.2 in two; of 32 pages 10.7
// and 12.4; of 64 pages 12.7 in four, 14.3 in two).
constexpr int kFill = 256, kLeastSteps = 8, kGain = 16;

struct Plan {
  int row_tiles, splits;
  size_t slot;  // bytes of a partial result, of all heads
  int64_t tiles;
};

Plan plan_of(int n_tokens, int heads, int q_heads, int head_dim, int block_tokens, int count) {
  Plan p;
  p.row_tiles = (q_heads / heads + 15) / 16;
  p.tiles = (int64_t)n_tokens * p.row_tiles;
  const int64_t units = p.tiles * heads, steps = ((int64_t)count * block_tokens + kStep - 1) / kStep;
  p.splits = (int)std::max<int64_t>(1, std::min<int64_t>({kFill / units, steps / kLeastSteps, (int64_t)kMostSplits}));
  if (steps - (steps + p.splits - 1) / p.splits < kGain) p.splits = 1;
  p.slot = (size_t)heads * 16 * (head_dim + 2) * sizeof(float);
  return p;
}

template <int DT, int KIND, int D>
void launch_pages(const AttnParams& a, const ListParams& x, dim3 grid, hipStream_t stream) {
  const unsigned lds = (unsigned)x.count * sizeof(int32_t);
  if (a.block_tokens % 16 == 0)
    launch_kernel(pages_kernel<DT, KIND, D, true>, grid, dim3(kFewThreads), lds, stream, a, x);
  else
    launch_kernel(pages_kernel<DT, KIND, D, false>, grid, dim3(kFewThreads), lds, stream, a, x);
}

template <int DT, int D>
void launch_kind(const AttnParams& a, const ListParams& x, int kind, dim3 grid, hipStream_t stream) {
  switch (kind) {
    case KVH_CACHE_16: launch_pages<DT, KVH_CACHE_16, D>(a, x, grid, stream); break;
    case KVH_CACHE_I8: launch_pages<DT, KVH_CACHE_I8, D>(a, x, grid, stream); break;
    default: launch_pages<DT, KVH_CACHE_E4M3, D>(a, x, grid, stream);
  }
  if (x.splits == 1) return;
  const int64_t rows = (int64_t)a.req.n_tokens * a.heads * a.group;
  hipLaunchKernelGGL((join_kernel<DT, D>), dim3((unsigned)((rows + kWavesPerBlock - 1) / kWavesPerBlock)), dim3(kBlockThreads), 0, stream, a, x);
}

}  // namespace
}  // namespace kvh

using namespace kvh;

extern "C" {

size_t kvh_attention_pages_workspace(int n_tokens, int heads, int q_heads, int head_dim, int block_tokens, int count) {
  if (n_tokens < 1 || !heads_fit(heads, q_heads) || (head_dim != 64 && head_dim != 128) || block_tokens < 1 || count < 1 || count > kMostListed) return 0;
  const Plan p = plan_of(n_tokens, heads, q_heads, head_dim, block_tokens, count);
  return p.splits == 1 ? 0 : (size_t)p.tiles * p.splits * p.slot;
}

int kvh_attention_pages(const kvh_cache* cache, int layer, const kvh_requests* requests, kvh_dtype dt, const kvh_rows* q, const kvh_rows* out, int q_heads,
                        const int32_t* pages_dev, int count, float* lse_dev, float scale, void* workspace_dev, size_t workspace_bytes, int32_t* status_dev,
                        void* stream) {
  if ((dt != KVH_F16 && dt != KVH_BF16) || q == nullptr || out == nullptr) return KVH_E_ARG;
  if (int rc = check_cache(cache)) return rc;
  if (int rc = check_requests(requests)) return rc;
  if (pages_dev == nullptr && requests->n_tokens != 0) return KVH_E_ARG;
  if (layer < 0 || layer >= cache->layers || !heads_fit(cache->heads, q_heads)) return KVH_E_SHAPE;
  for (const kvh_rows* r : {q, out})
    if (int rc = check_rows(r, (int64_t)q_heads * cache->head_dim, requests->n_tokens)) return rc;
  if (!std::isfinite(scale) || count < 1 || count > kMostListed) return KVH_E_ARG;
  if ((int64_t)count * cache->block_tokens > kMaxLength) return KVH_E_SHAPE;
  if (!is_aligned16(workspace_dev) || ((reinterpret_cast<uintptr_t>(lse_dev) | reinterpret_cast<uintptr_t>(pages_dev)) & 3u) != 0) return KVH_E_ALIGN;
  if (requests->n_tokens == 0) return KVH_OK;
  AttnParams a{};
  a.req = Requests(*requests, cache->block_tokens);
  if (a.req.max_new > a.req.n_tokens) a.req.max_new = a.req.n_tokens;
  a.q = static_cast<const uint16_t*>(q->p);
  a.out = static_cast<uint16_t*>(out->p);
  a.lse = lse_dev;
  a.q_ts = q->token_stride, a.o_ts = out->token_stride;
  const int width = cache->kind == KVH_CACHE_16 ? 2 : 1;
  a.ck = static_cast<const uint8_t*>(cache->k) + layer * cache->layer_stride * width;
  a.cv = static_cast<const uint8_t*>(cache->v) + layer * cache->layer_stride * width;
  if (cache->k_scale != nullptr) {
    a.sk = cache->k_scale + layer * cache->scale_layer_stride;
    a.sv = cache->v_scale + layer * cache->scale_layer_stride;
  }
  a.c_ts = cache->token_stride, a.s_ps = cache->scale_page_stride;
  a.pages = cache->pages, a.block_tokens = cache->block_tokens, a.heads = cache->heads;
  a.group = q_heads / cache->heads;
  a.scale = scale;
  a.status = status_dev;
  a.by_block = Divisor((uint32_t)cache->block_tokens), a.by_group = Divisor((uint32_t)a.group), a.by_heads = Divisor((uint32_t)a.heads);
  Plan p = plan_of(requests->n_tokens, a.heads, q_heads, cache->head_dim, cache->block_tokens, count);
  const size_t room = workspace_dev == nullptr ? 0 : workspace_bytes / (p.slot * p.tiles);
  if (room < (size_t)p.splits) p.splits = std::max((int)room, 1);
  const int steps = (int)(((int64_t)count * cache->block_tokens + kStep - 1) / kStep);
  ListParams x{};
  x.list = pages_dev, x.count = count, x.row_tiles = p.row_tiles, x.splits = p.splits;
  x.each = (steps + p.splits - 1) / p.splits;
  x.by_splits = Divisor((uint32_t)p.splits), x.by_row_tiles = Divisor((uint32_t)p.row_tiles);
  if (p.splits > 1) {
    a.part = static_cast<float*>(workspace_dev);
    a.part_ml = a.part + (size_t)p.tiles * p.splits * a.heads * 16 * cache->head_dim;
  }
  const int64_t blocks = p.tiles * a.heads * p.splits;
  if (blocks >= (int64_t)1 << 31 || (int64_t)requests->n_tokens * q_heads >= (int64_t)1 << 31) return KVH_E_SHAPE;
  hipStream_t s = static_cast<hipStream_t>(stream);
  const dim3 grid((unsigned)blocks);
  if (dt == KVH_F16) {
    if (cache->head_dim == 128)
      launch_kind<KVH_F16, 128>(a, x, cache->kind, grid, s);
    else
      launch_kind<KVH_F16, 64>(a, x, cache->kind, grid, s);
  } else {
    if (cache->head_dim == 128)
      launch_kind<KVH_BF16, 128>(a, x, cache->kind, grid, s);
    else
      launch_kind<KVH_BF16, 64>(a, x, cache->kind, grid, s);
  }
  KVH_HIP_CHECK_LAUNCH();
  return KVH_OK;
}

}  // extern "C"
