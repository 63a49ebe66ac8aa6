// kvh_select_pages: the pages that a token's queries may find large products on, by a score from the bounds of the pages' keys.
//
// A key k of the page lies in the box [lowest, highest], so q . k <= sum_d max(q_d lowest_d, q_d highest_d) = q- . lowest + q+ . highest with
// q- = min(q, 0) and q+ = max(q, 0): a matrix product with rows [q-, q+] and columns [lowest, highest] of 2 D bytes, which is how a page's bounds lie in memory.
// Both are int8, so the 16x16x64 products are exact and the same in any order.
//
// One block scores all pages of a token and KV head (of 2 or 4 neighbouring tokens where their query heads leave room among the product's 16 rows), keeps
// the scores in LDS as numbers in their order, and picks the best by counting them in bins.  Where there are too few tokens to fill the chip, or too many pages for LDS,
// the scores go through memory, from one grid that is as wide as the pages to one that picks.
//
// What bounds it: the bounds' bytes (256 of a page and head) come at 3.2 TB/s where many tokens have many pages (64 of 1000 pages: 41 us); below that, trips to memory that wait for
// each other - request, table, bounds - and for one token the picking.  A single block takes in 13 bytes a clock, so that one token of 1000 pages took 16 us in one launch and takes 10.5 in two.
// Measured, 8 KV heads of 128, 32 query heads, calls among others with other inputs in turn (in brackets scores and picking, each by itself in a trace): 64 requests of 4096 tokens (lognormal, pages of
// 16) 19.3 us (13.0 and 5.2), one of 131072 16 us (5.8 and 8.8), 16 of 64 pages for each of 64 9, of 256 pages 12.7, 512 new tokens of a request of 2080 pages 62 (44 and 22).
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
  int token0, tokens;  // of this turn
  uint32_t units;   // groups of tokens, and heads, that a block scores
  Divisor by_block, by_heads, by_units;
};

// The product's 16 rows: row r is query head u0 + r % (16 / TPT) of token row0 + r / (16 / TPT), as [q-, q+] in bytes, and a_u (0 where it counts as zeros).
template <int D>
struct QueryLds {
  static constexpr int kPitch = 2 * D + 16;  // bytes of a row
  alignas(16) uint8_t code[16][kPitch];
  float size[16];
};

// By the first 16 D / 8 threads of a block: 8 channels each, which are loaded ahead.
template <int D, int TPT>
__device__ __forceinline__ u32x4 load_queries(const SelectParams& a, int row0, int past, int head, int u0) {
  constexpr int kLanes = D / 8, kRows = 16 / TPT;
  const int r = threadIdx.x / kLanes, c = threadIdx.x % kLanes, u = u0 + r % kRows, row = row0 + r / kRows;
  u32x4 raw = {0, 0, 0, 0};
  if (r < 16 && u < a.group && row < past) raw = *reinterpret_cast<const u32x4*>(a.q + (int64_t)row * a.q_ts + ((int64_t)head * a.group + u) * D + c * 8);
  return raw;
}

template <int DT, int D>
__device__ __forceinline__ void quantise(const u32x4& raw, QueryLds<D>& lds) {
  constexpr int kLanes = D / 8;
  const int r = threadIdx.x / kLanes, c = threadIdx.x % kLanes;
  if (r >= 16) return;
  float x[8], most = 0.0f;
  widen8<DT>(raw, x);
#pragma unroll
  for (int e = 0; e < 8; ++e) most = fmaxf(most, fabsf(x[e]));
#pragma unroll
  for (int e = 0; e < 4; ++e)
    if (has_odd<DT, KVH_CACHE_16>(raw[e])) most = INFINITY;
#pragma unroll
  for (int d = 1; d < kLanes; d *= 2) most = fmaxf(most, __shfl_xor(most, d));
  const bool none = !(most < INFINITY) || most < 0x1p-100f;
  const Part127 part127(none ? 1.0f : most);
  u32x2 below, above;
#pragma unroll
  for (int w = 0; w < 2; ++w) {
    float v[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = none ? 0.0f : __builtin_rintf(part127.of(x[4 * w + e]));
    below[w] = four_codes(fminf(v[0], 0.0f), fminf(v[1], 0.0f), fminf(v[2], 0.0f), fminf(v[3], 0.0f));
    above[w] = four_codes(fmaxf(v[0], 0.0f), fmaxf(v[1], 0.0f), fmaxf(v[2], 0.0f), fmaxf(v[3], 0.0f));
  }
  *reinterpret_cast<u32x2*>(&lds.code[r][c * 8]) = below;
  *reinterpret_cast<u32x2*>(&lds.code[r][D + c * 8]) = above;
  if (c == 0) lds.size[r] = none ? 0.0f : most;
}

// A wave's rows of the product: lane l has row l % 16, bytes 64 kk + 16 (l / 16) and on, and the sizes of the four rows whose results it gets.
template <int D, int TPT>
struct Queries {
  static constexpr int kSums = 2 * D / 64;
  i32x4 code[kSums];
  float size[4];
  bool real[4];
  __device__ __forceinline__ Queries(const SelectParams& a, const QueryLds<D>& lds, int u0, int lane) {
#pragma unroll
    for (int kk = 0; kk < kSums; ++kk) code[kk] = *reinterpret_cast<const i32x4*>(&lds.code[lane % 16][kk * 64 + lane / 16 * 16]);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int r = lane / 16 * 4 + i;
      size[i] = lds.size[r];
      real[i] = u0 + r % (16 / TPT) < a.group;
    }
  }
};

// Pages that a token of the request may choose from.
__device__ __forceinline__ int pages_seen(const SelectParams& a, const Request& rq, int row) {
  const int p = rq.len - rq.n + (row - rq.start);
  return p < 0 ? 0 : (int)a.by_block.quotient((uint32_t)p) + 1;
}

// The scores of pages [base, base + kSpan) for TPT tokens, by one wave, 16 of them a product; entry[t] is the table's entry of page base + 16 t + l % 16 in lane l.  A lane
// gets those of token lane / 16 * TPT / 4, which chooses among `own` pages (0: it is no token of the request).  `best_of(page)` and `put(page, word)` are called by the lanes that
// hold a score: where the query heads come in several turns of 16, the largest so far is kept as it is, and the last turn makes the key of it.
constexpr int kTiles = 2, kSpan = 16 * kTiles;

template <int D>
struct Boxes {
  static constexpr int kSums = 2 * D / 64;
  i32x4 box[kTiles][kSums];
  float scale[kTiles];
  bool there[kTiles];
  __device__ __forceinline__ Boxes(const SelectParams& a, const int (&entry)[kTiles], int head, int lane) {
#pragma unroll
    for (int t = 0; t < kTiles; ++t) {
      there[t] = entry[t] >= 0 && entry[t] < a.pages;
      const int page = there[t] ? entry[t] : 0;  // (what lies past the last page is read as page 0 and not used: a condition would have each tile wait for the one before)
      const int8_t* from = a.codes + (int64_t)page * a.b_ps + (int64_t)head * 2 * D + lane / 16 * 16;
#pragma unroll
      for (int kk = 0; kk < kSums; ++kk) box[t][kk] = *reinterpret_cast<const i32x4*>(from + kk * 64);
      scale[t] = a.scale[(int64_t)page * a.bs_ps + head];
    }
  }
};

template <int D, int TPT, typename Best, typename Put>
__device__ __forceinline__ bool score_span(const SelectParams& a, const Boxes<D>& x, int base, int most, int own, const Queries<D, TPT>& q, bool first, bool last,
                                           int lane, Best&& best_of, Put&& put) {
  constexpr int kSums = 2 * D / 64;
  const int l16 = lane % 16, grp = lane / 16;
  bool bad = false;
#pragma unroll
  for (int t = 0; t < kTiles; ++t) {
    i32x4 dot = {0, 0, 0, 0};
#pragma unroll
    for (int kk = 0; kk < kSums; ++kk) dot = __builtin_amdgcn_mfma_i32_16x16x64_i8(q.code[kk], x.box[t][kk], dot, 0, 0, 0);
    float best = -INFINITY;
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (q.real[i]) best = fmaxf(best, (float)dot[i] * q.size[i]);
    if constexpr (TPT == 2) {
      const f32x2 x = apart16(best);
      best = fmaxf(x[0], x[1]);
    }
    if constexpr (TPT == 1) best = over_groups_max(best);
    const int j = base + 16 * t + l16;
    bad |= j < most && !x.there[t];
    if (grp % (4 / TPT) != 0 || j >= own) continue;
    if (!first) best = fmaxf(best, best_of(j));
    if (!last) {
      put(j, __builtin_bit_cast(uint32_t, best));
      continue;
    }
    const float score = best * x.scale[t];
    uint32_t key = !(score == score) || !(fabsf(x.scale[t]) < INFINITY) ? kInfinite : order_of(score);
    if (j < a.first || j >= own - a.last) key = kAlways;
    put(j, x.there[t] ? key : 0u);
  }
  return bad;
}

// The table's entries of pages [base, base + kSpan) as score_span takes them.
__device__ __forceinline__ void look_up(const int32_t* table, int base, int most, int lane, int (&entry)[kTiles]) {
#pragma unroll
  for (int t = 0; t < kTiles; ++t) {
    const int j = base + 16 * t + lane % 16;
    entry[t] = j < most ? table[j] : -1;
  }
}

// ---- picking ------------------------------------------------------------------------------------------------------
// W waves choose `count` of n keys; a block has GROUPS such teams, whose barriers are common.  The keys' range is cut into bins and counted, then that of the bin
// in which the last chosen key lies, until that bin is a single key, or is chosen as a whole.
constexpr int kLogBins = 10, kBins = 1 << kLogBins, kLaneBins = kBins / kWave;

template <int W, int GROUPS>
struct PickLds {
  alignas(16) uint32_t bins[GROUPS][kBins];
  uint32_t low[GROUPS][W], high[GROUPS][W], more[GROUPS][W], same[GROUPS][W];
  uint32_t found[GROUPS][2], open[GROUPS];
};

// four(g): keys 4 g .. 4 g + 3, 0 past the last one.  The code is short on purpose: it runs once, and its instructions have to be fetched.
template <int W, int GROUPS, typename Four>
__device__ __forceinline__ void pick(const Four& four, int n, int count, int first, int last, int32_t* out, PickLds<W, GROUPS>& lds, int team, int wave, int lane) {
  constexpr int kThreads = W * kWave;
  const int groups = (n + 3) / 4, each = (groups + kThreads - 1) / kThreads * kWave, begin = wave * each;  // a wave has a run of the keys
  const int stop = begin + each < groups ? begin + each : groups;
  // Those that are chosen in any case lie at the ends; they, and what is no candidate, take no part in the range.
  uint32_t sure = 0;
  for (int i = 0; i < first + last; i += kWave) {
    const int at = i + lane, j = at < first ? at : n - (first + last) + at;
    sure += __popcll(__ballot(at < first + last && j >= 0 && j < n && (at < first || j >= first) && four(j / 4)[j % 4] == kAlways));
  }
  uint32_t high = 0, not_low = 0;  // the largest key + 1, and the inverse of the least key - 1, in numbers that wrap
#pragma unroll 2
  for (int g = begin + lane; g < stop; g += kWave) {
    const u32x4 k = four(g);
#pragma unroll
    for (int e = 0; e < 4; ++e) high = max(high, k[e] + 1), not_low = max(not_low, ~(k[e] - 1));
  }
  high = wave_max(high), not_low = wave_max(not_low);
  uint32_t want = (uint32_t)count - sure;  // first + last <= count
  bool open = n > count && want != 0;
  if (lane == 0) lds.low[team][wave] = not_low, lds.high[team][wave] = high;
  if (wave == 0 && lane == 0) lds.open[team] = open;
#pragma unroll 1
  for (int i = wave * kWave + lane; i < kBins / 4; i += kThreads) reinterpret_cast<u32x4*>(lds.bins[team])[i] = u32x4{0, 0, 0, 0};
  __syncthreads();
  bool any_open = false;  // of the block's teams, whether one still looks for its least key
#pragma unroll
  for (int g = 0; g < GROUPS; ++g) any_open |= lds.open[g] == 1;
  high = wave_max(lane < W ? lds.high[team][lane] : 0) - 1;  // lane w has what wave w found
  uint32_t low = ~wave_max(lane < W ? lds.low[team][lane] : 0) + 1;
  // Without a key of another sort than those two there is no range, and nothing to look for: high is then 0, or kAlways, and what is chosen in any case is all.  (With one, a key
  // of 0 is further from low than high is, in numbers that wrap.)
  open = open && high - 1 < kInfinite;
  uint32_t least = want == 0 ? kAlways - 1 : 0, equal = 0;  // keys above it are chosen, and the first `equal` ones of those that are it
#pragma unroll 1
  while (any_open) {
    const uint32_t range = high - low;
    const int bits = 32 - __builtin_clz(range | 1u), shift = bits > kLogBins ? bits - kLogBins : 0;
    if (open) {
#pragma unroll 2
      for (int g = begin + lane; g < stop; g += kWave) {
        const u32x4 k = four(g);
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (k[e] - low <= range) atomicAdd(&lds.bins[team][(k[e] - low) >> shift], 1u);
      }
    }
    __syncthreads();
    if (wave == 0) {
      uint32_t on = 0;  // 1: the search goes on; 2: there are not so many
      if (open) {  // the bin of the want-th from above: a lane has 16 neighbouring ones
        uint32_t sum = 0;
#pragma unroll
        for (int i = 0; i < kLaneBins / 4; ++i) {
          const u32x4 x = reinterpret_cast<const u32x4*>(lds.bins[team])[lane * (kLaneBins / 4) + i];
          sum += x[0] + x[1] + x[2] + x[3];
        }
        uint32_t upto = row_sum_from(sum);
        const uint32_t r1 = __builtin_amdgcn_readlane(upto, 16), r2 = __builtin_amdgcn_readlane(upto, 32), r3 = __builtin_amdgcn_readlane(upto, 48);
        upto += (lane < 16 ? r1 : 0) + (lane < 32 ? r2 : 0) + (lane < 48 ? r3 : 0);
        const uint64_t enough = __ballot(upto >= want);
        if (enough == 0) {
          on = 2;
        } else {
          const int at = 63 - __builtin_clzll(enough);  // the last lane with so many from it on
          const uint32_t past = (uint32_t)__builtin_amdgcn_readlane(upto - sum, at);
          const uint32_t mine = lds.bins[team][at * kLaneBins + (lane & (kLaneBins - 1))];
          const uint32_t from = row_sum_from(mine) + past;
          const int bin = 63 - __builtin_clzll(__ballot(lane < kLaneBins && from >= want));
          const uint32_t inside = __builtin_amdgcn_readlane(mine, bin), before = (uint32_t)__builtin_amdgcn_readlane(from, bin) - inside;
          on = shift != 0 && inside != want - before;
          if (lane == 0) lds.found[team][0] = (uint32_t)(at * kLaneBins + bin), lds.found[team][1] = before;
        }
      }
      if (lane == 0) lds.open[team] = on;
    }
    __syncthreads();
    if (open && lds.open[team] == 2) {
      open = false;  // all candidates: they are above 0
    } else if (open) {
      want -= lds.found[team][1];
      low += lds.found[team][0] << shift;
      open = lds.open[team] == 1;
      if (open)
        high = min(high, low + (1u << shift) - 1);
      else if (shift == 0)
        least = low, equal = want;
      else
        least = low - 1;
    }
    any_open = false;
#pragma unroll
    for (int g = 0; g < GROUPS; ++g) any_open |= lds.open[g] == 1;
    if (any_open) {
#pragma unroll 1
      for (int i = wave * kWave + lane; i < kBins / 4; i += kThreads) reinterpret_cast<u32x4*>(lds.bins[team])[i] = u32x4{0, 0, 0, 0};
      __syncthreads();
    }
  }
  // Where a wave's chosen keys go, and how many of the equal ones lie before it.
  uint32_t more = 0, same = 0;
#pragma unroll 2
  for (int g = begin + lane; g < stop; g += kWave) {
    const u32x4 k = four(g);
#pragma unroll
    for (int e = 0; e < 4; ++e) more += k[e] > least, same += k[e] == least;
  }
  uint32_t all_more, all_same;
  wave_sum_to(more, all_more), wave_sum_to(same, all_same);
  if (lane == 0) lds.more[team][wave] = all_more, lds.same[team][wave] = all_same;
  __syncthreads();
  const uint32_t their_more = lane < W ? lds.more[team][lane] : 0, their_same = lane < W ? lds.same[team][lane] : 0;
  uint32_t before = row_sum(lane < wave ? their_same : 0), at = row_sum(lane < wave ? their_more : 0) + min(before, equal);
  const uint32_t total = row_sum(their_more) + min(row_sum(their_same), equal);
#pragma unroll 1
  for (int g0 = begin; g0 < stop; g0 += kWave) {
    u32x4 k = {0, 0, 0, 0};
    if (g0 + lane < stop) k = four(g0 + lane);
    uint32_t alike = 0;
    if (equal != 0) {  // the equal ones that are past the first `equal` become less
      uint32_t here = 0;
#pragma unroll
      for (int e = 0; e < 4; ++e) here += k[e] == least;
      uint32_t rank = before + wave_sum_to(here, alike) - here;
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (k[e] == least) k[e] = rank++ < equal ? kAlways : 0;
    }
    before += alike;
    uint32_t mine = 0, all;
#pragma unroll
    for (int e = 0; e < 4; ++e) mine += k[e] > least;
    uint32_t to = at + wave_sum_to(mine, all) - mine;
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (k[e] > least) out[to++] = 4 * (g0 + lane) + e;
    at += all;
  }
  if (out != nullptr) {
#pragma unroll 1
    for (int i = (int)total + wave * kWave + lane; i < count; i += kThreads) out[i] = -1;
  }
}

// ---- kernels ------------------------------------------------------------------------------------------------------
constexpr int kSelectWaves = 8, kSelectThreads = kSelectWaves * kWave;

// Scores and choice of TPT neighbouring tokens and a head.
template <int DT, int D, int TPT>
__global__ __launch_bounds__(kSelectThreads, 4) void select_kernel(SelectParams a) {
  constexpr int kRows = 16 / TPT, W = kSelectWaves / TPT;  // query heads that a product takes of a token; waves of a team
  __shared__ PickLds<W, TPT> lds;
  __shared__ QueryLds<D> queries;
  extern __shared__ __align__(16) uint32_t keys[];
  const int lane = threadIdx.x % kWave, wave = uniform((int32_t)(threadIdx.x / kWave));
  tell_refused<kSelectThreads>(a.req, a.status);
  const uint32_t tile = a.by_heads.quotient(blockIdx.x);
  const int head = (int)(blockIdx.x - tile * a.heads), row0 = (int)tile * TPT;
  const int past = row0 + TPT < a.req.n_tokens ? row0 + TPT : a.req.n_tokens;
  u32x4 raw = load_queries<D, TPT>(a, row0, past, head, 0);
  for (int row = row0; row < past;) {
    int b, next;
    Request rq;
    if (!request_of(a.req, row, lane, b, rq, next)) {
      row = next;
      continue;
    }
    const int stop = rq.start + rq.n < past ? rq.start + rq.n : past;  // the request's rows of this tile
    int end[TPT];
#pragma unroll
    for (int i = 0; i < TPT; ++i) end[i] = row0 + i >= row && row0 + i < stop ? pages_seen(a, rq, row0 + i) : 0;
    const int most = pages_seen(a, rq, stop - 1);
    const int32_t* table = a.req.table + (int64_t)b * a.req.table_stride;
    bool bad = false;
    const int token = lane / 16 * TPT / 4;
    int own = end[0];
#pragma unroll
    for (int i = 1; i < TPT; ++i) own = token == i ? end[i] : own;
    uint32_t* mine = keys + token * a.pitch;
    if (most <= a.count) {  // all there are: no score decides
      for (int j = threadIdx.x; j < most; j += kSelectThreads) {
        const int page = table[j];
        const bool there = page >= 0 && page < a.pages;
        bad |= !there;
#pragma unroll
        for (int i = 0; i < TPT; ++i)
          if (j < end[i]) keys[i * a.pitch + j] = there;
      }
    } else {
      for (int u0 = 0; u0 < a.group; u0 += kRows) {  // (one turn, but where a token has more than 16 query heads)
        int entry[kTiles];
        look_up(table, wave * kSpan, most, lane, entry);
        if (u0 > 0) __syncthreads();
        quantise<DT, D>(raw, queries);  // while the table's entries are on their way
        if (kRows < a.group) raw = load_queries<D, TPT>(a, row0, past, head, u0 + kRows < a.group ? u0 + kRows : 0);
        __syncthreads();
        const Queries<D, TPT> q(a, queries, u0, lane);
        for (int base = wave * kSpan; base < most; base += kSelectWaves * kSpan) {
          const Boxes<D> boxes(a, entry, head, lane);
          look_up(table, base + kSelectWaves * kSpan, most, lane, entry);
          bad |= score_span<D, TPT>(a, boxes, base, most, own, q, u0 == 0, u0 + kRows >= a.group, lane, [&](int j) { return __builtin_bit_cast(float, mine[j]); },
                                    [&](int j, uint32_t key) { mine[j] = key; });
        }
      }
    }
    if (__any(bad) && lane == 0 && a.status != nullptr) a.status[b] = KVH_DEV_BAD_REQUEST;
    __syncthreads();
    const int team = wave / W, its = row0 + team;
    int n = 0;
#pragma unroll
    for (int i = 0; i < TPT; ++i) n = i == team ? end[i] : n;
    int32_t* out = its >= row && its < stop ? a.out + ((int64_t)its * a.heads + head) * a.count : nullptr;
    uint32_t* from = keys + team * a.pitch;
    if (n + lane < ((n + 3) & ~3)) from[n + lane] = 0;  // (all waves of the team do)
    __syncthreads();
    pick<W, TPT>([&](int g) { return reinterpret_cast<const u32x4*>(from)[g]; }, n, a.count, a.first, a.last, out, lds, team, wave % W, lane);
    __syncthreads();
    row = stop;
  }
}

constexpr int kScoreTurns = 2, kScorePages = kScoreTurns * kWavesPerBlock * kSpan;

// Scores of one token and head, kScoreTurns times kSpan pages a wave, to memory.
template <int DT, int D>
__global__ __launch_bounds__(kBlockThreads) void score_kernel(SelectParams a) {
  __shared__ QueryLds<D> queries;
  const int lane = threadIdx.x % kWave, wave = uniform((int32_t)(threadIdx.x / kWave));
  if (a.token0 == 0) tell_refused(a.req, a.status);
  const uint32_t tile = a.by_units.quotient(blockIdx.x), unit = blockIdx.x - tile * a.units;  // the tiles that few requests reach come last
  const uint32_t token = a.by_heads.quotient(unit);
  const int head = (int)(unit - token * a.heads), row = a.token0 + (int)token;
  int b;
  Request rq;
  if (!request_of(a.req, row, lane, b, rq)) return;
  const int end = pages_seen(a, rq, row), first = (int)tile * kScorePages;
  if (first >= end) return;
  u32x4 raw = load_queries<D, 1>(a, row, row + 1, head, 0);
  const int32_t* table = a.req.table + (int64_t)b * a.req.table_stride;
  int entry[kScoreTurns][kTiles];
#pragma unroll
  for (int i = 0; i < kScoreTurns; ++i) look_up(table, first + (i * kWavesPerBlock + wave) * kSpan, end, lane, entry[i]);
  uint32_t* keys = a.keys + ((int64_t)token * a.heads + head) * a.pitch;
  bool bad = false;
  for (int u0 = 0; u0 < a.group; u0 += 16) {
    if (u0 > 0) {
      raw = load_queries<D, 1>(a, row, row + 1, head, u0);
      __syncthreads();
    }
    quantise<DT, D>(raw, queries);
    __syncthreads();
    const Queries<D, 1> q(a, queries, u0, lane);
#pragma unroll
    for (int i = 0; i < kScoreTurns; ++i) {
      const int base = first + (i * kWavesPerBlock + wave) * kSpan;
      if (base >= end) break;
      const Boxes<D> boxes(a, entry[i], head, lane);
      bad |= score_span<D, 1>(a, boxes, base, end, end, q, u0 == 0, u0 + 16 >= a.group, lane, [&](int j) { return __builtin_bit_cast(float, keys[j]); },
                              [&](int j, uint32_t key) { keys[j] = key; });
    }
  }
  if (__any(bad) && lane == 0 && a.status != nullptr) a.status[b] = KVH_DEV_BAD_REQUEST;
}

// Scores of M times TPT neighbouring tokens and a head in the same way.  What is loaded of a page serves all tokens.
template <int DT, int D, int TPT, int M>
__global__ __launch_bounds__(kBlockThreads) void score_many_kernel(SelectParams a) {
  constexpr int kTokens = TPT * M;
  __shared__ QueryLds<D> queries[M];
  const int lane = threadIdx.x % kWave, wave = uniform((int32_t)(threadIdx.x / kWave));
  if (a.token0 == 0) tell_refused(a.req, a.status);
  const uint32_t tile = a.by_units.quotient(blockIdx.x), unit = blockIdx.x - tile * a.units;
  const uint32_t group = a.by_heads.quotient(unit);
  const int head = (int)(unit - group * a.heads), row0 = a.token0 + (int)group * kTokens, first = (int)tile * kScorePages;
  const int past = row0 + kTokens < a.token0 + a.tokens ? row0 + kTokens : a.token0 + a.tokens;
  bool ready = false;  // the queries
  for (int row = row0; row < past;) {
    int b, next;
    Request rq;
    if (!request_of(a.req, row, lane, b, rq, next)) {
      row = next;
      continue;
    }
    const int begin = row, stop = rq.start + rq.n < past ? rq.start + rq.n : past;  // the request's rows of this tile
    row = stop;
    const int most = pages_seen(a, rq, stop - 1);
    if (first >= most) continue;
    if (!ready) {
      u32x4 raw[M];
#pragma unroll
      for (int m = 0; m < M; ++m) raw[m] = load_queries<D, TPT>(a, row0 + m * TPT, past, head, 0);
#pragma unroll
      for (int m = 0; m < M; ++m) quantise<DT, D>(raw[m], queries[m]);
      __syncthreads();
      ready = true;
    }
    const int32_t* table = a.req.table + (int64_t)b * a.req.table_stride;
    int entry[kScoreTurns][kTiles];
#pragma unroll
    for (int i = 0; i < kScoreTurns; ++i) look_up(table, first + (i * kWavesPerBlock + wave) * kSpan, most, lane, entry[i]);
    bool bad = false;
#pragma unroll
    for (int i = 0; i < kScoreTurns; ++i) {
      const int base = first + (i * kWavesPerBlock + wave) * kSpan;
      if (base >= most) break;
      const Boxes<D> boxes(a, entry[i], head, lane);
#pragma unroll 1
      for (int m = 0; m < M; ++m) {
        const int r = row0 + m * TPT + lane / 16 * TPT / 4, own = r >= begin && r < stop ? pages_seen(a, rq, r) : 0;
        if (!__any(own != 0)) continue;
        uint32_t* keys = a.keys + ((int64_t)((own != 0 ? r : begin) - a.token0) * a.heads + head) * a.pitch;
        const Queries<D, TPT> q(a, queries[m], 0, lane);
        bad |= score_span<D, TPT>(a, boxes, base, most, own, q, true, true, lane, [](int) { return 0.0f; }, [&](int j, uint32_t key) { keys[j] = key; });
      }
    }
    if (__any(bad) && lane == 0 && a.status != nullptr) a.status[b] = KVH_DEV_BAD_REQUEST;
  }
}

template <int W>
__global__ __launch_bounds__(W * kWave) void pick_kernel(SelectParams a) {
  constexpr int kThreads = W * kWave, kStaged = W == 4 ? 4096 : 8 * kThreads;
  __shared__ PickLds<W, 1> lds;
  __shared__ u32x4 staged[kStaged / 4];
  const int lane = threadIdx.x % kWave, wave = uniform((int32_t)(threadIdx.x / kWave));
  const uint32_t token = a.by_heads.quotient(blockIdx.x);
  const int head = (int)(blockIdx.x - token * a.heads), row = a.token0 + (int)token;
  int b;
  Request rq;
  if (!request_of(a.req, row, lane, b, rq)) return;
  const int n = pages_seen(a, rq, row);
  const uint32_t* keys = a.keys + ((int64_t)token * a.heads + head) * a.pitch;
  int32_t* out = a.out + ((int64_t)row * a.heads + head) * a.count;
  const u32x4* fours = reinterpret_cast<const u32x4*>(keys);
  auto from_memory = [&](int g) {  // (what a row holds past its last key is of no account)
    u32x4 k = fours[g];
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (4 * g + e >= n) k[e] = 0;
    return k;
  };
  if (n <= kStaged) {  // read again and again: from LDS
    constexpr int kEach = kStaged / 4 / kThreads;
    u32x4 k[kEach];
#pragma unroll
    for (int i = 0; i < kEach; ++i) k[i] = 4 * (i * kThreads + (int)threadIdx.x) < n ? from_memory(i * kThreads + threadIdx.x) : u32x4{0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < kEach; ++i) staged[i * kThreads + threadIdx.x] = k[i];
    __syncthreads();
    pick<W, 1>([&](int g) { return staged[g]; }, n, a.count, a.first, a.last, out, lds, 0, wave, lane);
  } else {
    pick<W, 1>(from_memory, n, a.count, a.first, a.last, out, lds, 0, wave, lane);
  }
}

// ---- launch -------------------------------------------------------------------------------------------------------
constexpr int kMostListed = 4096;
constexpr int kLds = 64 << 10;  // of a block
// Tokens and heads below which scores of more pages than kManyPages go through memory: 64 requests of 4096 (lognormal) 19.3 us so, 20.4 in one launch (the longest has 1364 pages); one of 1000
// pages 10.5 and 16; where 64 are of one length the other way is the faster one, of 512 pages 23.5 and 19.1, of 1000 41 and 36.  A table of 256 pages: 64 requests 15.7 and 12.7, one request 10.5 and 8.4.
// More tokens and heads, where neighbouring tokens share products: 512 of 2080 pages 62 us through memory and 79 in one launch, of 500 pages 28.6 and 30.4.
constexpr int64_t kFewUnits = 1024, kManyPages = 256, kShared = 1024;

int64_t pitch_of(int table_pages) { return ((int64_t)table_pages + 3) & ~(int64_t)3; }

// Tokens that share a product: their query heads are its rows.
int together(int n_requests, int n_tokens, int group) {
  const int64_t each = (int64_t)n_tokens / n_requests;
  return each >= 4 && group <= 4 ? 4 : each >= 2 && group <= 8 ? 2 : 1;
}
// Whether a block keeps its scores in LDS.
bool fits(int tokens, int table_pages) {
  const int64_t picks = tokens == 4 ? sizeof(PickLds<kSelectWaves / 4, 4>) : tokens == 2 ? sizeof(PickLds<kSelectWaves / 2, 2>) : sizeof(PickLds<kSelectWaves, 1>);
  return tokens * pitch_of(table_pages) * (int64_t)sizeof(uint32_t) + picks + (int64_t)sizeof(QueryLds<128>) <= kLds;
}
bool by_memory(int n_tokens, int heads, int tokens, int table_pages) {
  return table_pages > kManyPages && ((int64_t)n_tokens * heads < kFewUnits || (tokens > 1 && table_pages > kShared));
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

// Picks from which on a team has 4 waves and not 8, of which more wait at a time: 4096 of 2080 keys 22 us, 32 with 8; 512 of them 7.2 and 6.3.
constexpr unsigned kManyPicks = 1024;
// Products of a block that scores neighbouring tokens (the kernel alone, one after the other): 512 tokens of 2080 pages 48 us, with 2 65, with 8 56; 64 tokens 12.5, 11 and 19.
constexpr int kMany = 4;

template <int DT, int D>
void launch_score(const SelectParams& a, int together, int64_t tiles, hipStream_t stream) {
  const dim3 grid((unsigned)(a.units * tiles)), block(kBlockThreads);
  if (together == 4)
    launch_kernel(score_many_kernel<DT, D, 4, kMany>, grid, block, 0, stream, a);
  else if (together == 2)
    launch_kernel(score_many_kernel<DT, D, 2, kMany>, grid, block, 0, stream, a);
  else
    launch_kernel(score_kernel<DT, D>, grid, block, 0, stream, a);
  const dim3 picks((unsigned)(a.tokens * a.heads));
  if (a.pitch <= 4096 && picks.x >= kManyPicks)
    hipLaunchKernelGGL(pick_kernel<4>, picks, dim3(4 * kWave), 0, stream, a);
  else if (a.pitch <= 4096)
    hipLaunchKernelGGL(pick_kernel<8>, picks, dim3(8 * kWave), 0, stream, a);
  else
    hipLaunchKernelGGL(pick_kernel<16>, picks, dim3(16 * kWave), 0, stream, a);
}

}  // namespace
}  // namespace kvh

using namespace kvh;

extern "C" {

size_t kvh_select_workspace(int n_requests, int n_tokens, int heads, int table_pages) {
  if (n_requests < 1 || n_requests > kMaxRequests || n_tokens < 1 || heads < 1 || heads > 4096 || table_pages < 1) return 0;
  // (The query heads are not known here: with few a KV head, neighbouring tokens share products.)
  if (fits(1, table_pages) && !by_memory(n_tokens, heads, together(n_requests, n_tokens, 1), table_pages)) return 0;
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
  const bool f16 = dt == KVH_F16, wide = bounds->head_dim == 128;
  int tokens = together(requests->n_requests, requests->n_tokens, a.group);
  if (turn < 1 || !by_memory(requests->n_tokens, a.heads, tokens, requests->table_pages)) {
    int here = tokens;
    while (here > 1 && !fits(here, requests->table_pages)) here /= 2;
    if (fits(here, requests->table_pages)) {
      if (f16)
        wide ? launch_select<KVH_F16, 128>(a, here, s) : launch_select<KVH_F16, 64>(a, here, s);
      else
        wide ? launch_select<KVH_BF16, 128>(a, here, s) : launch_select<KVH_BF16, 64>(a, here, s);
      KVH_HIP_CHECK_LAUNCH();
      return KVH_OK;
    }
  }
  if (turn < 1) return KVH_E_SIZE;
  a.keys = static_cast<uint32_t*>(workspace_dev);
  const int64_t tiles = ((int64_t)requests->table_pages + kScorePages - 1) / kScorePages, most = ((int64_t)1 << 31) - 1;
  if (a.heads * tiles > most) return KVH_E_SHAPE;
  if (turn < tokens * kMany || requests->n_tokens / requests->n_requests < tokens * kMany) tokens = 1;
  const int each = tokens > 1 ? tokens * kMany : 1;  // tokens of a block
  turn = std::min<int64_t>({turn, (int64_t)requests->n_tokens, most / a.heads / tiles * each});
  if (turn < requests->n_tokens) turn -= turn % each;
  for (int64_t t0 = 0; t0 < requests->n_tokens; t0 += turn) {
    a.token0 = (int)t0, a.tokens = (int)std::min<int64_t>(turn, requests->n_tokens - t0);
    a.units = (uint32_t)((a.tokens + each - 1) / each * a.heads);
    a.by_units = Divisor(a.units);
    if (f16)
      wide ? launch_score<KVH_F16, 128>(a, tokens, tiles, s) : launch_score<KVH_F16, 64>(a, tokens, tiles, s);
    else
      wide ? launch_score<KVH_BF16, 128>(a, tokens, tiles, s) : launch_score<KVH_BF16, 64>(a, tokens, tiles, s);
    KVH_HIP_CHECK_LAUNCH();
  }
  return KVH_OK;
}

}  // extern "C"
