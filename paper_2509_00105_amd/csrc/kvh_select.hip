// kvh_select_pages: the pages that a token's queries may find large products on, by a score from the bounds of the pages' keys.
//
// A key k of the page lies in the box [lowest, highest], so q . k <= sum_d max(q_d lowest_d, q_d highest_d) = q- . lowest + q+ . highest with
// q- = min(q, 0) and q+ = max(q, 0): a matrix product with rows [q-, q+] and columns [lowest, highest] of 2 D bytes, which is how a page's bounds lie in memory.
// Both are int8, so the 16x16x64 products are exact and the same in any order.
//
// One block scores all pages of a token and KV head (of 2 or 4 neighbouring tokens where their query heads leave room among the product's 16 rows), keeps
// the scores in LDS as numbers in their order, and picks the best by counting them in bins.  Where there are too few tokens to fill the chip, or too many pages for LDS,
// the scores go through memory, from one grid that is as wide as the pages to one that picks.
#include "kvh_bounds.hpp"

#include <algorithm>

namespace kvh {
namespace {

typedef int32_t i32x4 __attribute__((ext_vector_type(4)));

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
  uint32_t* keys;   // [token of this turn][head][pitch], where they go through memory
  int64_t pitch;    // keys of a token and head
  int token0;       // the turn's first token
  uint32_t tiles;   // blocks that score a token and head
  int in_lds;       // whether the picking kernel has room for a token's keys
  Divisor by_block, by_heads, by_tiles;
};

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

// What a token asks of its request's pages.
struct Asked {
  int end;  // pages that it may choose from
  __device__ __forceinline__ Asked() : end(0) {}
  __device__ __forceinline__ Asked(const SelectParams& a, const Request& rq, int row) {
    const int p = rq.len - rq.n + (row - rq.start);
    end = p < 0 ? 0 : (int)a.by_block.quotient((uint32_t)p) + 1;
  }
};

// The scores of pages [base, base + 64) for TPT tokens, by one wave: lane l looks up page base + l; a product takes 16 of them.  `put(token, page, key)` is called by
// the lanes that hold a key.  end[i] is 0 for what is no token of the request.
template <int DT, int D, int TPT, typename Put>
__device__ __forceinline__ bool score64(const SelectParams& a, const int32_t* table, int head, int base, int most, const int (&end)[TPT], const Queries<DT, D>& first,
                                        const uint16_t* rows, int lane, Put&& put) {
  constexpr int kSums = 2 * D / 64, kTiles = 4;
  const int l16 = lane % 16, grp = lane / 16;
  int page = -1;
  if (base + lane < most) page = table[base + lane];
  const bool there = page >= 0 && page < a.pages;
  const bool bad = base + lane < most && !there;
  if (!there) page = 0;
  i32x4 box[kTiles][kSums];
#pragma unroll
  for (int t = 0; t < kTiles; ++t) {
    const int8_t* from = a.codes + (int64_t)__shfl(page, 16 * t + l16) * a.b_ps + (int64_t)head * 2 * D + grp * 16;
    if (base + 16 * t < most) {
#pragma unroll
      for (int kk = 0; kk < kSums; ++kk) box[t][kk] = *reinterpret_cast<const i32x4*>(from + kk * 64);
    }
  }
  const float scale = a.scale[(int64_t)page * a.bs_ps + head];
  const uint64_t here = __ballot(there);
  float best[kTiles];
#pragma unroll
  for (int t = 0; t < kTiles; ++t) best[t] = -INFINITY;
  auto take = [&](const Queries<DT, D>& q, int u0) {
    float size[4];
    bool real[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int r = grp * 4 + i;
      size[i] = __shfl(q.size, r);
      real[i] = u0 + r % (16 / TPT) < a.group;
    }
#pragma unroll
    for (int t = 0; t < kTiles; ++t) {
      if (base + 16 * t >= most) break;
      i32x4 dot = {0, 0, 0, 0};
#pragma unroll
      for (int kk = 0; kk < kSums; ++kk) dot = __builtin_amdgcn_mfma_i32_16x16x64_i8(q.code[kk], box[t][kk], dot, 0, 0, 0);
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (real[i]) best[t] = fmaxf(best[t], (float)dot[i] * size[i]);
    }
  };
  take(first, 0);
  if constexpr (TPT == 1) {
    for (int u0 = 16; u0 < a.group; u0 += 16) {
      Queries<DT, D> q;
      const bool real = u0 + l16 < a.group;
      q.load(rows + (u0 + (real ? l16 : 0)) * D, real, grp);
      take(q, u0);
    }
  }
  const int token = grp * TPT / 4, own = end[token];
#pragma unroll
  for (int t = 0; t < kTiles; ++t) {
    if (base + 16 * t >= most) break;
    if constexpr (TPT <= 2) best[t] = fmaxf(best[t], __shfl_xor(best[t], 16));
    if constexpr (TPT == 1) best[t] = fmaxf(best[t], __shfl_xor(best[t], 32));
    const int j = base + 16 * t + l16;
    const float s = __shfl(scale, 16 * t + l16), score = best[t] * s;
    uint32_t key = !(score == score) || !(fabsf(s) < INFINITY) ? kInfinite : order_of(score);
    if (j < a.first || j >= own - a.last) key = kAlways;
    if (grp % (4 / TPT) == 0 && j < own) put(token, j, (here >> (16 * t + l16) & 1u) != 0 ? key : 0u);
  }
  return bad;
}

// ---- picking ------------------------------------------------------------------------------------------------------
// W waves choose `count` of n keys; a block has GROUPS such teams, whose barriers are common.  The keys' range is cut into bins and counted, then that of the bin
// in which the last chosen key lies, until that bin is a single key, or is chosen as a whole.
constexpr int kLogBins = 10, kBins = 1 << kLogBins;

template <int W, int GROUPS>
struct PickLds {
  uint32_t bins[GROUPS][kBins];
  uint32_t low[GROUPS][W], high[GROUPS][W], some[GROUPS][W], sure[GROUPS][W];
  uint32_t found[GROUPS][3];
};

template <int W, int GROUPS, typename Keys>
__device__ __forceinline__ void pick(const Keys& key, int n, int count, int32_t* out, PickLds<W, GROUPS>& lds, int team, int wave, int lane) {
  constexpr int kThreads = W * kWave;
  const int id = wave * kWave + lane;
  uint32_t low = ~0u, high = 0, some = 0, sure = 0;
  for (int j0 = wave * kWave; j0 < n; j0 += kThreads) {
    const uint32_t k = j0 + lane < n ? key(j0 + lane) : 0;
    const bool candidate = k != 0 && k != kAlways;
    if (candidate) low = min(low, k), high = max(high, k);
    some += __popcll(__ballot(candidate)), sure += __popcll(__ballot(k == kAlways));
  }
#pragma unroll
  for (int d = 1; d < kWave; d *= 2) {
    low = min(low, (uint32_t)__shfl_xor((int)low, d));
    high = max(high, (uint32_t)__shfl_xor((int)high, d));
  }
  if (lane == 0) lds.low[team][wave] = low, lds.high[team][wave] = high, lds.some[team][wave] = some, lds.sure[team][wave] = sure;
  __syncthreads();
  some = sure = 0;
#pragma unroll
  for (int w = 0; w < W; ++w) {
    low = min(low, lds.low[team][w]), high = max(high, lds.high[team][w]);
    some += lds.some[team][w], sure += lds.sure[team][w];
  }
  uint32_t want = (uint32_t)count - sure;         // first + last <= count
  uint32_t least = want == 0 ? kAlways - 1 : 0, equal = 0;  // keys above it are chosen, and the first `equal` ones of those that are it
  bool open = want != 0 && some > want;
  while (__syncthreads_or(open)) {
    const int bits = 32 - __builtin_clz((high - low) | 1u), shift = bits > kLogBins ? bits - kLogBins : 0;
    if (open)
      for (int i = id; i < kBins; i += kThreads) lds.bins[team][i] = 0;
    __syncthreads();
    if (open)
      for (int j = id; j < n; j += kThreads) {
        const uint32_t k = key(j);
        if (k >= low && k <= high) atomicAdd(&lds.bins[team][(k - low) >> shift], 1u);
      }
    __syncthreads();
    if (open && wave == 0) {  // the bin of the want-th from above: a lane has 16 of them
      constexpr int kMine = kBins / kWave;
      uint32_t mine[kMine], sum = 0;
#pragma unroll
      for (int i = 0; i < kMine; ++i) sum += mine[i] = lds.bins[team][lane * kMine + i];
      uint32_t above = sum;  // of this lane and those behind it
#pragma unroll
      for (int d = 1; d < kWave; d *= 2) {
        const uint32_t x = __shfl_down(above, d);
        if (lane + d < kWave) above += x;
      }
      above -= sum;
      if (above < want && above + sum >= want) {
#pragma unroll
        for (int i = kMine - 1; i >= 0; --i) {
          if (above < want && above + mine[i] >= want) lds.found[team][0] = lane * kMine + i, lds.found[team][1] = above, lds.found[team][2] = mine[i];
          above += mine[i];
        }
      }
    }
    __syncthreads();
    if (open) {
      want -= lds.found[team][1];
      low += lds.found[team][0] << shift;
      if (shift == 0)
        least = low, equal = want, open = false;
      else if (lds.found[team][2] == want)
        least = low - 1, open = false;
      else
        high = min(high, low + (1u << shift) - 1);
    }
  }
  // The chosen ones in order: a wave has a run of the keys.
  const int each = (n + kThreads - 1) / kThreads * kWave, begin = wave * each, stop = begin + each < n ? begin + each : n;
  uint32_t more = 0, same = 0;
  for (int j0 = begin; j0 < stop; j0 += kWave) {
    const uint32_t k = j0 + lane < stop ? key(j0 + lane) : 0;
    more += __popcll(__ballot(k > least)), same += __popcll(__ballot(k == least && k != 0));
  }
  if (lane == 0) lds.some[team][wave] = more, lds.sure[team][wave] = same;
  __syncthreads();
  uint32_t at = 0, before = 0, total = 0, alike = 0;
#pragma unroll
  for (int w = 0; w < W; ++w) {
    if (w == wave) at = total, before = alike;
    total += lds.some[team][w], alike += lds.sure[team][w];
  }
  at += min(before, equal), total += min(alike, equal);
  const uint64_t under = ((uint64_t)1 << lane) - 1;
  for (int j0 = begin; j0 < stop; j0 += kWave) {
    const uint32_t k = j0 + lane < stop ? key(j0 + lane) : 0;
    const uint64_t is = __ballot(k == least && k != 0);
    const bool take = k > least || (k == least && k != 0 && before + __popcll(is & under) < equal);
    const uint64_t taken = __ballot(take);
    if (take) out[at + __popcll(taken & under)] = j0 + lane;
    at += __popcll(taken), before += __popcll(is);
  }
  if (out != nullptr)
    for (int i = (int)total + id; i < count; i += kThreads) out[i] = -1;
}

// ---- kernels ------------------------------------------------------------------------------------------------------
constexpr int kSelectWaves = 8, kSelectThreads = kSelectWaves * kWave;

// Scores and choice of TPT neighbouring tokens and a head.
template <int DT, int D, int TPT>
__global__ __launch_bounds__(kSelectThreads, 4) void select_kernel(SelectParams a) {
  constexpr int kRows = 16 / TPT, W = kSelectWaves / TPT;  // query heads of a token; waves of a team
  __shared__ PickLds<W, TPT> lds;
  extern __shared__ uint32_t keys[];
  const int lane = threadIdx.x % kWave, wave = uniform((int32_t)(threadIdx.x / kWave)), l16 = lane % 16, grp = lane / 16;
  tell_refused(a.req, a.status);
  const uint32_t tile = a.by_heads.quotient(blockIdx.x);
  const int head = (int)(blockIdx.x - tile * a.heads), row0 = (int)tile * TPT;
  const int past = row0 + TPT < a.req.n_tokens ? row0 + TPT : a.req.n_tokens;
  const uint16_t* rows = a.q + ((int64_t)row0 + l16 / kRows) * a.q_ts + (int64_t)head * a.group * D;
  Queries<DT, D> q;
  {
    const int u = l16 % kRows;
    const bool real = u < a.group && row0 + l16 / kRows < past;
    q.load(real ? rows + u * D : a.q, real, grp);
  }
  for (int row = row0; row < past;) {
    int b;
    Request rq;
    if (!request_of(a.req, row, lane, b, rq)) {
      ++row;
      continue;
    }
    const int stop = rq.start + rq.n < past ? rq.start + rq.n : past;  // the request's rows of this tile
    int end[TPT];
#pragma unroll
    for (int i = 0; i < TPT; ++i) end[i] = row0 + i >= row && row0 + i < stop ? Asked(a, rq, row0 + i).end : 0;
    const int most = Asked(a, rq, stop - 1).end;
    const int32_t* table = a.req.table + (int64_t)b * a.req.table_stride;
    bool bad = false;
    for (int base = wave * kWave; base < most; base += kSelectThreads)
      bad |= score64<DT, D, TPT>(a, table, head, base, most, end, q, rows, lane, [&](int token, int j, uint32_t key) { keys[token * a.pitch + j] = key; });
    if (__any(bad) && lane == 0 && a.status != nullptr) a.status[b] = KVH_DEV_BAD_REQUEST;
    __syncthreads();
    const int team = wave / W, mine = row0 + team;
    int n = 0;
#pragma unroll
    for (int i = 0; i < TPT; ++i) n = i == team ? end[i] : n;
    int32_t* out = mine >= row && mine < stop ? a.out + ((int64_t)mine * a.heads + head) * a.count : nullptr;
    const uint32_t* from = keys + team * a.pitch;
    pick<W, TPT>([&](int j) { return from[j]; }, n, a.count, out, lds, team, wave % W, lane);
    __syncthreads();
    row = stop;
  }
}

// Scores of one token and head, 64 pages a wave, to memory.
template <int DT, int D>
__global__ __launch_bounds__(kBlockThreads) void score_kernel(SelectParams a) {
  const int lane = threadIdx.x % kWave, wave = uniform((int32_t)(threadIdx.x / kWave)), l16 = lane % 16, grp = lane / 16;
  if (a.token0 == 0) tell_refused(a.req, a.status);
  const uint32_t unit = a.by_tiles.quotient(blockIdx.x), tile = blockIdx.x - unit * a.tiles;
  const uint32_t token = a.by_heads.quotient(unit);
  const int head = (int)(unit - token * a.heads), row = a.token0 + (int)token;
  const uint16_t* rows = a.q + (int64_t)row * a.q_ts + (int64_t)head * a.group * D;
  Queries<DT, D> q;
  q.load(rows + (l16 < a.group ? l16 : 0) * D, l16 < a.group, grp);
  int b;
  Request rq;
  if (!request_of(a.req, row, lane, b, rq)) return;
  const int end[1] = {Asked(a, rq, row).end};
  const int base = (int)tile * kBlockThreads + wave * kWave;
  if (base >= end[0]) return;
  uint32_t* keys = a.keys + ((int64_t)token * a.heads + head) * a.pitch;
  const bool bad = score64<DT, D, 1>(a, a.req.table + (int64_t)b * a.req.table_stride, head, base, end[0], end, q, rows, lane,
                                     [&](int, int j, uint32_t key) { keys[j] = key; });
  if (__any(bad) && lane == 0 && a.status != nullptr) a.status[b] = KVH_DEV_BAD_REQUEST;
}

constexpr int kPickWaves = 16, kPickThreads = kPickWaves * kWave;

__global__ __launch_bounds__(kPickThreads) void pick_kernel(SelectParams a) {
  __shared__ PickLds<kPickWaves, 1> lds;
  extern __shared__ uint32_t mine[];
  const int lane = threadIdx.x % kWave, wave = uniform((int32_t)(threadIdx.x / kWave));
  const uint32_t token = a.by_heads.quotient(blockIdx.x);
  const int head = (int)(blockIdx.x - token * a.heads), row = a.token0 + (int)token;
  int b;
  Request rq;
  if (!request_of(a.req, row, lane, b, rq)) return;
  const int n = Asked(a, rq, row).end;
  const uint32_t* keys = a.keys + ((int64_t)token * a.heads + head) * a.pitch;
  int32_t* out = a.out + ((int64_t)row * a.heads + head) * a.count;
  if (a.in_lds) {
    for (int j = threadIdx.x; j < n; j += kPickThreads) mine[j] = keys[j];
    __syncthreads();
    pick<kPickWaves, 1>([&](int j) { return mine[j]; }, n, a.count, out, lds, 0, wave, lane);
  } else {
    pick<kPickWaves, 1>([&](int j) { return keys[j]; }, n, a.count, out, lds, 0, wave, lane);
  }
}

// ---- launch -------------------------------------------------------------------------------------------------------
constexpr int kMostListed = 4096;
constexpr int kLds = 64 << 10;  // of a block
constexpr int64_t kFewUnits = 256, kManyPages = 1024;

int64_t pitch_of(int table_pages) { return ((int64_t)table_pages + 3) & ~(int64_t)3; }

// Tokens that share a block's products; 0 where scores go through memory.
int together(int n_requests, int n_tokens, int heads, int group, int table_pages, bool room) {
  const int64_t keys = pitch_of(table_pages) * (int64_t)sizeof(uint32_t);
  if (keys + (int64_t)sizeof(PickLds<kSelectWaves, 1>) > kLds) return 0;
  if (room && (int64_t)n_tokens * heads < kFewUnits && table_pages > kManyPages) return 0;
  const int64_t each = (int64_t)n_tokens / n_requests;
  if (each >= 4 && group <= 4 && 4 * keys + (int64_t)sizeof(PickLds<kSelectWaves / 4, 4>) <= kLds) return 4;
  if (each >= 2 && group <= 8 && 2 * keys + (int64_t)sizeof(PickLds<kSelectWaves / 2, 2>) <= kLds) return 2;
  return 1;
}

template <int DT, int D>
void launch_select(const SelectParams& a, int tokens, hipStream_t stream) {
  const dim3 grid((unsigned)(((int64_t)a.req.n_tokens + tokens - 1) / tokens * a.heads)), block(kSelectThreads);
  const unsigned lds = (unsigned)(tokens * a.pitch * sizeof(uint32_t));
  if (tokens == 4)
    launch_kernel(select_kernel<DT, D, 4>, grid, block, lds, stream, a);
  else if (tokens == 2)
    launch_kernel(select_kernel<DT, D, 2>, grid, block, lds, stream, a);
  else
    launch_kernel(select_kernel<DT, D, 1>, grid, block, lds, stream, a);
}

template <int DT, int D>
void launch_score(const SelectParams& a, unsigned tokens, hipStream_t stream) {
  launch_kernel(score_kernel<DT, D>, dim3(tokens * a.heads * a.tiles), dim3(kBlockThreads), 0, stream, a);
  const unsigned lds = a.in_lds ? (unsigned)(a.pitch * sizeof(uint32_t)) : 0;
  hipLaunchKernelGGL(pick_kernel, dim3(tokens * a.heads), dim3(kPickThreads), lds, stream, a);
}

}  // namespace
}  // namespace kvh

using namespace kvh;

extern "C" {

size_t kvh_select_workspace(int n_requests, int n_tokens, int heads, int table_pages) {
  if (n_requests < 1 || n_requests > kMaxRequests || n_tokens < 1 || heads < 1 || heads > 4096 || table_pages < 1) return 0;
  if (together(n_requests, n_tokens, heads, 1, table_pages, true) != 0) return 0;
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
  a.pitch = pitch_of(requests->table_pages);
  a.by_block = Divisor((uint32_t)bounds->block_tokens), a.by_heads = Divisor((uint32_t)bounds->heads);
  if ((int64_t)requests->n_tokens * a.heads >= (int64_t)1 << 31) return KVH_E_SHAPE;
  hipStream_t s = static_cast<hipStream_t>(stream);
  const int64_t token = (int64_t)a.heads * a.pitch * sizeof(uint32_t);
  int64_t turn = workspace_dev == nullptr ? 0 : (int64_t)(workspace_bytes / (size_t)token);
  const int tokens = together(requests->n_requests, requests->n_tokens, a.heads, a.group, requests->table_pages, turn > 0);
  const bool f16 = dt == KVH_F16, wide = bounds->head_dim == 128;
  if (tokens != 0) {
    if (f16)
      wide ? launch_select<KVH_F16, 128>(a, tokens, s) : launch_select<KVH_F16, 64>(a, tokens, s);
    else
      wide ? launch_select<KVH_BF16, 128>(a, tokens, s) : launch_select<KVH_BF16, 64>(a, tokens, s);
    KVH_HIP_CHECK_LAUNCH();
    return KVH_OK;
  }
  if (turn < 1) return KVH_E_SIZE;
  a.keys = static_cast<uint32_t*>(workspace_dev);
  a.tiles = (uint32_t)((requests->table_pages + kBlockThreads - 1) / kBlockThreads);
  a.in_lds = a.pitch * (int64_t)sizeof(uint32_t) + (int64_t)sizeof(PickLds<kPickWaves, 1>) <= kLds;
  a.by_tiles = Divisor(a.tiles);
  if ((int64_t)a.heads * a.tiles >= (int64_t)1 << 31) return KVH_E_SHAPE;
  turn = std::min({turn, (int64_t)requests->n_tokens, (((int64_t)1 << 31) - 1) / ((int64_t)a.heads * a.tiles)});
  for (int64_t t0 = 0; t0 < requests->n_tokens; t0 += turn) {
    a.token0 = (int)t0;
    const unsigned here = (unsigned)std::min<int64_t>(turn, requests->n_tokens - t0);
    if (f16)
      wide ? launch_score<KVH_F16, 128>(a, here, s) : launch_score<KVH_F16, 64>(a, here, s);
    else
      wide ? launch_score<KVH_BF16, 128>(a, here, s) : launch_score<KVH_BF16, 64>(a, here, s);
    KVH_HIP_CHECK_LAUNCH();
  }
  return KVH_OK;
}

}  // extern "C"
