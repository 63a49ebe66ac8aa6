// What the two attention kernels share: parameters, the list of items, operands, the page table.
#pragma once

#include "kvh_cache.hpp"

namespace kvh {

constexpr int kStep = 32;  // tokens a wave takes at once: two tiles of 16
constexpr int kLogManyRows = 7, kManyRows = 1 << kLogManyRows;  // a tile of the kernel for many rows (kvh_attention_many.hip)
constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;
constexpr float kLeastScale = 0x1p-60f;  // V scales below it keep it in the exponent; the rest goes onto the weight

struct AttnParams {
  Requests req;
  const uint16_t* q;
  uint16_t* out;
  float* lse;
  int64_t q_ts, o_ts;  // elements
  const uint8_t *ck, *cv;  // of the layer
  const float *sk, *sv;
  int64_t c_ts, s_ps;
  int pages, block_tokens, heads, group;
  float scale;
  int causal, sink, window;
  int32_t* status;
  float* part;       // partial outputs [slot][rows][D], then (maximum, sum) [slot][rows][2]; nullptr: nothing is split
  float* part_ml;
  struct Joint* joints;  // of the tiles, for the joining kernel, and how many they are
  int32_t* joints_n;
  int target;        // chunks that the batch is cut into
  int least;         // steps of a chunk at least
  int64_t slots;     // partial results that there is room for, of each head
  int64_t tiles;     // tiles of the batch at most
  int log_hw;        // few rows: a block's waves take 2^log_hw heads
  Divisor by_block, by_group, by_heads;  // by_heads: heads, or groups of them that a block takes
};

// ---- items --------------------------------------------------------------------------------------------------------
// A request's rows come in tiles, its tokens in steps of 32; the tiles of a batch, each with its steps, make one long row of steps.  Where
// the batch is cut, that row is cut every `chunk` steps and block k of the grid takes chunk k, one tile after the other: no block has more to do
// than another.  All blocks work out the same cuts from the lengths, which the host need not know.  The partial result of tile r (counted
// over the batch) in chunk k has place k + r: a tile's last chunk is the next one's first, or lies before it.  Where nothing is cut, block r
// takes tile r.
__device__ __forceinline__ int steps_of(const AttnParams& a, const Request& rq, int log_rows) {
  const int all = (rq.len + kStep - 1) / kStep;
  int64_t some = all;
  if (a.window != 0) {
    const int64_t reach = (int64_t)a.window + (1 << log_rows) + 4 * kStep;  // of a tile's rows, with two steps begun on either side
    some = reach / kStep + (a.sink + kStep - 1) / kStep + 1;
  }
  const int steps = all < some ? all : (int)some;
  return steps < 2 ? 2 : steps + 1 & ~1;  // some, also where there is no token: its rows have to be written
}

struct Item {
  int b, tile, tiles;  // request; tile of its rows, and how many they are
  int from, count;     // steps of the tile
  bool last, split;    // its last ones; some of them are another item's
  int64_t slot;        // of its partial result
  Request rq;
};

// What the joining kernel has to know of a tile, written by the block that has its first part.
struct Joint {
  int32_t start, n, len, tile;  // of the request; the tile of its rows
  int32_t parts, spare;
  int64_t slot;                 // of the first one
};
static_assert(sizeof(Joint) == 32, "two 16-byte accesses");

// Quotients by a number of the launch that only the device knows; both below 2^50.
struct WideDivisor {
  int64_t d;
  double inv;
  __device__ __forceinline__ explicit WideDivisor(int64_t d_) : d(d_), inv(1.0 / (double)d_) {}
  __device__ __forceinline__ int64_t quotient(int64_t x) const {
    int64_t q = (int64_t)((double)x * inv);  // within one of it
    const int64_t r = x - q * d;
    if (r < 0) --q;
    if (r >= d) ++q;
    return q;
  }
};

// The value of lane l, which is the same for the whole wave.
__device__ __forceinline__ int32_t of_lane(int32_t v, int l) { return __builtin_amdgcn_readlane(v, l); }
__device__ __forceinline__ int64_t of_lane(int64_t v, int l) {
  return (int64_t)((uint64_t)(uint32_t)of_lane((int32_t)((uint64_t)v >> 32), l) << 32 | (uint32_t)of_lane((int32_t)(uint64_t)v, l));
}

struct Schedule {
  const AttnParams& a;
  const int log_rows, lane;
  // of request b0 + lane: its tiles and the steps of each, and the tiles and steps up to its end
  int b0, tiles, steps;
  Request rq;
  int64_t tile_end, step_end;

  __device__ __forceinline__ Schedule(const AttnParams& a_, int log_rows_, int lane_) : a(a_), log_rows(log_rows_), lane(lane_) { group(0, 0, 0); }

  __device__ __forceinline__ void group(int first, int64_t tile_base, int64_t step_base) {
    b0 = first;
    rq = Request{0, 0, 0, false};
    tiles = steps = 0;
    const int b = first + lane;
    if (b < a.req.n) {
      rq.start = a.req.starts[b];
      const int32_t end = a.req.starts[b + 1];
      rq.len = a.req.lens[b];
      rq.n = end - rq.start;
      rq.ok = request_ok(a.req, rq.start, end, rq.len);
      if (rq.ok && rq.n > 0) {
        tiles = (int)(((int64_t)rq.n * a.group + (1 << log_rows) - 1) >> log_rows);
        steps = steps_of(a, rq, log_rows);
      }
    }
    tile_end = tiles, step_end = (int64_t)tiles * steps;
    const int many = a.req.n - first;
    for (int d = 1; d < kWave && d < many; d *= 2) {
      const int64_t t = __shfl_up((long long)tile_end, d), s = __shfl_up((long long)step_end, d);
      if (lane >= d) tile_end += t, step_end += s;
    }
    // lanes past the last request stand at its end
    if (many < kWave) {
      const int64_t t = of_lane(tile_end, many - 1), s = of_lane(step_end, many - 1);
      if (lane >= many) tile_end = t, step_end = s;
    }
    tile_end += tile_base, step_end += step_base;
  }
  __device__ __forceinline__ bool next_group() {
    if (b0 + kWave >= a.req.n) return false;
    group(b0 + kWave, of_lane(tile_end, kWave - 1), of_lane(step_end, kWave - 1));
    return true;
  }

  // The lane of the request for which `here` holds, with its group in the lanes; -1 where there is none.
  template <typename F>
  __device__ __forceinline__ int find(F&& here) {
    do {
      const uint64_t who = __ballot(rq.ok && here());
      if (who != 0) return __builtin_ctzll(who);
    } while (next_group());
    return -1;
  }

  __device__ __forceinline__ void take(int l, Item& it) const {
    it.b = b0 + l;
    it.rq.start = of_lane(rq.start, l);
    it.rq.n = of_lane(rq.n, l);
    it.rq.len = of_lane(rq.len, l);
    it.rq.ok = true;
    it.tiles = of_lane(tiles, l);
  }

  // Item `k` of a batch that is not cut.  A request's last tile, which sees the most tokens, comes first.
  __device__ __forceinline__ bool whole(int64_t k, Item& it) {
    const int l = find([&] { return k < tile_end && k >= tile_end - tiles; });
    if (l < 0) return false;
    take(l, it);
    it.tile = (int32_t)(of_lane(tile_end, l) - k) - 1;
    it.from = 0, it.count = of_lane(steps, l);
    it.last = true, it.split = false;
    it.slot = 0;
    return true;
  }

  // Of a batch that is cut: what chunk k holds from step `at` on (its first, if `at` is negative) that is of one tile; `at` becomes the step
  // after.  `tells`: this block writes what the joining kernel has to know.
  __device__ __forceinline__ bool part(int64_t k, int64_t& at, int64_t& past, Item& it, bool tells) {
    while (next_group()) {}
    const int64_t total = of_lane(step_end, kWave - 1);
    if (tells && k == 0) {
      const int64_t n = of_lane(tile_end, kWave - 1);
      if (lane == 0) *a.joints_n = (int32_t)(n < a.tiles ? n : a.tiles);
    }
    int64_t size = (total + a.target - 1) / a.target;
    if (size < a.least) size = a.least;
    const WideDivisor chunk(uniform((size + 3) & ~(int64_t)3));  // four waves may share it
    if (at < 0) at = k * chunk.d;
    const int64_t mine = (k + 1) * chunk.d < total ? (k + 1) * chunk.d : total;
    past = mine;
    if (at >= mine) return false;
    if (a.req.n > kWave) group(0, 0, 0);
    const int l = find([&] { return at < step_end && at >= step_end - (int64_t)tiles * steps; });
    if (l < 0) return false;
    take(l, it);
    const int each = of_lane(steps, l);
    const int64_t step0 = of_lane((step_end - (int64_t)tiles * steps), l);
    const int64_t tile0 = of_lane((tile_end - tiles), l);
    it.tile = it.tiles > 1 ? uniform((int32_t)((at - step0) / each)) : 0;
    const int64_t begin = step0 + (int64_t)it.tile * each, end = begin + each, rank = tile0 + it.tile;
    it.from = (int)(at - begin);
    it.last = end <= mine;
    it.count = (int)((it.last ? end : mine) - at);
    it.split = at > begin || !it.last;
    it.slot = k + rank;
    if (tells && at == begin && lane == 0 && rank < a.tiles) {
      Joint j;
      j.start = it.rq.start, j.n = it.rq.n, j.len = it.rq.len, j.tile = it.tile;
      j.parts = (int32_t)(uniform(chunk.quotient(end - 1)) - k) + 1;
      j.spare = 0;
      j.slot = it.slot;
      const u32x4* w = reinterpret_cast<const u32x4*>(&j);
      u32x4* p = reinterpret_cast<u32x4*>(a.joints + rank);
      p[0] = w[0], p[1] = w[1];
    }
    at += it.count;
    return true;
  }
};

// The items of block k, one after the other.  (lane is made opaque: what follows from it is worked out anew for each item, and does not take
// registers from one to the next.)
struct Items {
  int64_t at = -1, past = 0;  // steps of a batch that is cut: the next one, and the end of the block's
  __device__ __forceinline__ bool next(const AttnParams& a, int log_rows, int64_t k, bool tells, int& lane, Item& it) {
    if (at >= past) return false;
    asm volatile("" : "+v"(lane));
    Schedule schedule(a, log_rows, lane);
    if (a.part != nullptr) return schedule.part(k, at, past, it, tells);
    at = past = 0;
    return schedule.whole(k, it);
  }
};

// Says which requests are refused; the kernels pass over them.  (Written out for these kernels: the general one moves their scalar registers about, which
// costs a call for one token of 300 0.35 of 8.5 us.)
__device__ __forceinline__ void tell_refused(const AttnParams& a) {
  if (blockIdx.x != 0 || a.status == nullptr) return;
  for (int b = threadIdx.x; b < a.req.n; b += kBlockThreads)
    if (!request_ok(a.req, a.req.starts[b], a.req.starts[b + 1], a.req.lens[b])) a.status[b] = KVH_DEV_BAD_REQUEST;
}

// ---- operands -----------------------------------------------------------------------------------------------------
template <int DT, int KIND>
constexpr bool kBf16 = KIND == KVH_CACHE_16 && DT == KVH_BF16;  // the products' type; fp16 otherwise

template <bool BF>
__device__ __forceinline__ f32x4 mfma(const u32x4& x, const u32x4& y, const f32x4& c) {
  if constexpr (BF)
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, x), __builtin_bit_cast(bf16x8, y), c, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, x), __builtin_bit_cast(f16x8, y), c, 0, 0, 0);
}

// bytes (lo, hi) of offset-binary codes q + 128 in the low byte of each half, 0x64 above: 1024 + 128 + q in fp16
__device__ __forceinline__ uint32_t less_1152(uint32_t w) {
  const f16x2 h = __builtin_bit_cast(f16x2, w), o = {(_Float16)-1152.0f, (_Float16)-1152.0f};
  return __builtin_bit_cast(uint32_t, h + o);
}

// 4 codes of one word -> 2 words of fp16 pairs, in order.
template <int KIND>
__device__ __forceinline__ void widen4(uint32_t w, uint32_t& lo, uint32_t& hi) {
  if constexpr (KIND == KVH_CACHE_I8) {
    w ^= 0x80808080u;
    lo = less_1152(__builtin_amdgcn_perm(0x64646464u, w, 0x04010400u));
    hi = less_1152(__builtin_amdgcn_perm(0x64646464u, w, 0x04030402u));
  } else {
    lo = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.0f, false));
    hi = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.0f, true));
  }
}

// The same 4 channels of two tokens x, y -> pairs (x, y) of each channel.
template <int KIND>
__device__ __forceinline__ void zip4(uint32_t x, uint32_t y, uint32_t (&p)[4]) {
  widen4<KIND>(__builtin_amdgcn_perm(y, x, 0x05010400u), p[0], p[1]);
  widen4<KIND>(__builtin_amdgcn_perm(y, x, 0x07030602u), p[2], p[3]);
}

template <int N>
struct Words {
  uint32_t w[N];
};
// N words from memory, in the widest accesses (N a power of two; the address is aligned to 4 N bytes, 16 at most).
template <int N>
__device__ __forceinline__ Words<N> fetch(const uint8_t* p) {
  Words<N> r;
  if constexpr (N == 1) {
    r.w[0] = *reinterpret_cast<const uint32_t*>(p);
  } else if constexpr (N == 2) {
    const u32x2 v = *reinterpret_cast<const u32x2*>(p);
    r.w[0] = v[0], r.w[1] = v[1];
  } else {
#pragma unroll
    for (int i = 0; i < N / 4; ++i) {
      const u32x4 v = *reinterpret_cast<const u32x4*>(p + 16 * i);
#pragma unroll
      for (int e = 0; e < 4; ++e) r.w[4 * i + e] = v[e];
    }
  }
  return r;
}

// ---- the page table, 64 entries at a time in the lanes ---------------------------------------------------------------
struct PageRun {
  int base, entry;  // entry of page base + lane; -1 where it is none of the cache's
  int ahead;        // the same of the 64 pages after those

  __device__ __forceinline__ PageRun() : base(-1000), entry(-1), ahead(-1) {}
  // Makes page `first` the run's first; pages past `last` are not looked at.
  __device__ __forceinline__ void load(const AttnParams& a, const int32_t* table, int first, int last, int lane) {
    entry = first == base + kWave ? ahead : read(a, table, first + lane, last);
    ahead = read(a, table, first + kWave + lane, last);
    base = first;
  }
  static __device__ __forceinline__ int read(const AttnParams& a, const int32_t* table, int at, int last) {
    int e = -1;
    if (at <= last) e = table[at];
    return e < a.pages ? e : -1;
  }
};

// What a row at logical position p sees: tokens up to `last`, and of them those past `low` or before the sink's end.
struct Sight {
  int last, low;
  __device__ __forceinline__ Sight() {}
  // `end` is past the last token that any row of the item sees.
  __device__ __forceinline__ Sight(const AttnParams& a, int end, int p) : last(a.causal && p < end ? p : end - 1), low(a.window != 0 ? (p > 0 ? p : 0) - a.window : -1) {}
  __device__ __forceinline__ bool sees(const AttnParams& a, int token) const { return token <= last && (token > low || token < a.sink); }
  // Of tokens [t0, t0 + 64), those it sees.
  __device__ __forceinline__ uint64_t seen(const AttnParams& a, int t0) const {
    int last = this->last, low = this->low;
    asm volatile("" : "+v"(last), "+v"(low));  // rarely asked: nothing of it is worked out ahead of a loop
    auto below = [&](int token) {  // those before it
      const int n = token - t0;
      return n <= 0 ? (uint64_t)0 : n >= 64 ? ~(uint64_t)0 : ((uint64_t)1 << n) - 1;
    };
    return below(last + 1) & (~below(low < 0 ? 0 : low + 1) | below(a.sink));
  }
};

// An item's steps: those of the first `sink` tokens, then those from its first row's window on.
struct Steps {
  int first, sunk, count;
  __device__ __forceinline__ Steps(const AttnParams& a, int p_least, int end) {
    first = sunk = 0;
    if (a.window != 0) {
      const int from = (p_least > 0 ? p_least : 0) - a.window + 1;  // positions below 0 see nothing
      first = from > 0 ? from / kStep & ~1 : 0;
      sunk = (a.sink + kStep - 1) / kStep + 1 & ~1;
      if (sunk >= first) first = sunk = 0;
    }
    count = end > 0 ? sunk + (end + kStep - 1) / kStep - first : 0;
  }
  __device__ __forceinline__ int token(int step) const { return (step < sunk ? step : step - sunk + first) * kStep; }
  // Of an item's, those there are.
  __device__ __forceinline__ void part_of(const Item& it, int& begin, int& end) const {
    begin = it.from < count ? it.from : count;
    end = it.last || it.from + it.count > count ? count : it.from + it.count;
  }
};

// Operands of the second product where it holds an infinity or NaN that some rows do not see.  A weight of zero does not keep these from a row,
// so they are taken out of the product, and what they do to the rows that see them comes from products of ones: where (ones of the tokens
// that a row sees) x (ones where a value is NaN, or +infinity, or -infinity) is not zero, that value is added to the row's output.
template <bool BF>
struct Odd {
  static constexpr uint32_t kExp = BF ? 0x7f80u : 0x7c00u, kOne = BF ? 0x3f80u : 0x3c00u;
  static __device__ __forceinline__ float value(int which) { return which == 0 ? NAN : which == 1 ? INFINITY : -INFINITY; }
  static __device__ __forceinline__ uint32_t without(uint32_t w) {
    return ((w & kExp) == kExp ? 0u : w & 0xffffu) | ((w >> 16 & kExp) == kExp ? 0u : w & 0xffff0000u);
  }
  static __device__ __forceinline__ bool is(uint32_t h, int which) {
    return which == 0 ? (h & 0x7fffu) > kExp : h == (which == 1 ? kExp : kExp | 0x8000u);
  }
  static __device__ __forceinline__ uint32_t ones(uint32_t w, int which) {
    return (is(w & 0xffffu, which) ? kOne : 0u) | (is(w >> 16, which) ? kOne << 16 : 0u);
  }
  static __device__ __forceinline__ u32x4 without(const u32x4& v) { return u32x4{without(v[0]), without(v[1]), without(v[2]), without(v[3])}; }
  static __device__ __forceinline__ u32x4 ones(const u32x4& v, int which) {
    return u32x4{ones(v[0], which), ones(v[1], which), ones(v[2], which), ones(v[3], which)};
  }
};

// A V scale as the softmax takes it: its logarithm goes into the exponent, its inverse into the sum.  Two sorts of scales are not taken as they are.  One of
// zero (or next to it) keeps its tokens in the sum and takes their values off the weight: kLeastScale, with the rest of it as a factor.  The
// page of one that is no finite number holds NaN: rows that see the page become that, and the scale is taken as 1, since neither a weight of zero nor a
// hidden score would keep NaN and infinities from the other rows.
__device__ __forceinline__ bool odd_scale(float z) { return !(__builtin_fabsf(z) < INFINITY); }
struct ValueScale {
  float used, rest;
  __device__ __forceinline__ explicit ValueScale(float z) {
    used = odd_scale(z) ? 1.0f : z < kLeastScale ? kLeastScale : z;
    rest = odd_scale(z) ? NAN : z < kLeastScale ? z * (1.0f / kLeastScale) : 1.0f;
  }
};
// Whether one of several scales is of either sort: the words of numbers that are not negative are in their order, infinity and NaN above them.
struct ScaleRange {
  uint32_t top = 0, low = ~0u;
  __device__ __forceinline__ void add(float k, float v) {
    const uint32_t kw = __builtin_bit_cast(uint32_t, k), vw = __builtin_bit_cast(uint32_t, v);
    top = top > kw ? top : kw;
    top = top > vw ? top : vw;
    low = low < vw ? low : vw;
  }
  __device__ __forceinline__ bool rare() const {
    return top >= __builtin_bit_cast(uint32_t, INFINITY) || low < __builtin_bit_cast(uint32_t, kLeastScale);
  }
};

// bf16 values of a row -> fp16 with the power of two that brings its largest to [1, 2): the factor, and what undoes it.
__device__ __forceinline__ f32x2 row_power(float most) {
  int ex = (int)(__builtin_bit_cast(uint32_t, most) >> 23) - 127;
  if (ex < -100 || ex > 127) ex = 0;  // nothing but zeros (or next to it); infinities stay what they are
  const float down = __builtin_bit_cast(float, (uint32_t)(127 - (ex > 126 ? 126 : ex)) << 23);
  return f32x2{down, 1.0f / down};
}

void launch_attention_many(const AttnParams& a, int dt, int kind, int head_dim, unsigned blocks, hipStream_t stream);

}  // namespace kvh
