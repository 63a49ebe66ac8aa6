// What the two attention kernels share: parameters, the list of items, operands, the page table.
#pragma once

#include "kvh_cache.hpp"

namespace kvh {

constexpr int kStep = 32;  // tokens a wave takes at once: two tiles of 16
constexpr int kManyRows = 128;  // a tile of the kernel for many rows (kvh_attention_many.hip)
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
  int target;        // items that the batch is cut into, about
  int least;         // steps of an item at least, where a request is cut
  int64_t items;     // partial results that there is room for, of each head
  Divisor by_block, by_group, by_heads;
};

// ---- items --------------------------------------------------------------------------------------------------------
// A request's rows come in tiles of `tile_rows`, its tokens in steps of 32, and an item is a tile and a run of `chunk` steps.  All
// blocks work out the same list from the lengths: no block is idle while another has two requests' worth of tokens, and the host
// need not know the lengths.
__device__ __forceinline__ int steps_of(const AttnParams& a, const Request& rq, int tile_rows) {
  if (!rq.ok || rq.n == 0) return 0;
  const int all = (rq.len + kStep - 1) / kStep;
  if (a.window == 0) return all;
  const int64_t reach = (int64_t)a.window + tile_rows + 4 * kStep;  // of a tile's rows, with two steps begun on either side
  const int64_t some = reach / kStep + (a.sink + kStep - 1) / kStep + 1;
  return all < some ? all : (int)some;
}

struct Item {
  int b, tile, part, parts;  // parts: of the request's tokens
  int tiles;                 // of the request's rows; the last one, which sees the most tokens, comes first
  int chunk;
  Request rq;
};

__device__ __forceinline__ Request read_request(const AttnParams& a, int b) {
  Request rq{0, 0, 0, false};
  if (b < a.req.n) {
    rq.start = a.req.starts[b];
    const int32_t end = a.req.starts[b + 1];
    rq.len = a.req.lens[b];
    rq.n = end - rq.start;
    rq.ok = request_ok(a.req, rq.start, end, rq.len);
  }
  return rq;
}

// Steps of an item, from the steps of the batch.
__device__ __forceinline__ int chunk_of(const AttnParams& a, int tile_rows, int lane) {
  if (a.part == nullptr) return 0x7fffffff;
  int64_t total = 0;
  for (int b0 = 0; b0 < a.req.n; b0 += kWave) {
    const Request rq = read_request(a, b0 + lane);
    const int tiles = (int)(((int64_t)(rq.ok ? rq.n : 0) * a.group + tile_rows - 1) / tile_rows);
    int64_t s = (int64_t)tiles * steps_of(a, rq, tile_rows);
#pragma unroll
    for (int d = 1; d < kWave; d *= 2) s += __shfl_xor((long long)s, d);
    total += s;
  }
  int64_t chunk = (total + a.target - 1) / a.target;
  if (chunk < a.least) chunk = a.least;
  chunk = (chunk + 3) & ~(int64_t)3;  // four waves share it
  return chunk < 0x7fffffff ? (int)chunk : 0x7fffffff;
}

// The request whose item (or, with by_row, whose packed row) `want` is.  Returns false where there is none.
__device__ __forceinline__ bool find_item(const AttnParams& a, int tile_rows, int64_t want, bool by_row, int lane, Item& it) {
  it.chunk = uniform(chunk_of(a, tile_rows, lane));
  int64_t base = 0;
  for (int b0 = 0; b0 < a.req.n; b0 += kWave) {
    const Request rq = read_request(a, b0 + lane);
    const int steps = steps_of(a, rq, tile_rows);
    const int tiles = (int)(((int64_t)(rq.ok ? rq.n : 0) * a.group + tile_rows - 1) / tile_rows);
    int parts = steps == 0 ? 1 : 1 + (steps - 1) / it.chunk;
    const int64_t mine = (int64_t)tiles * parts;
    int64_t upto = mine;
#pragma unroll
    for (int d = 1; d < kWave; d *= 2) {
      const int64_t o = __shfl_up((long long)upto, d);
      if (lane >= d) upto += o;
    }
    const bool here = by_row ? rq.ok && want >= rq.start && want < (int64_t)rq.start + rq.n
                             : want >= base + upto - mine && want < base + upto;
    const uint64_t who = __ballot(here);
    if (who != 0) {
      const int l = __builtin_ctzll(who);
      it.b = b0 + l;
      it.rq.start = uniform(__shfl(rq.start, l));
      it.rq.n = uniform(__shfl(rq.n, l));
      it.rq.len = uniform(__shfl(rq.len, l));
      it.rq.ok = true;
      it.parts = uniform(__shfl(parts, l));
      it.tiles = uniform(__shfl(tiles, l));
      const int64_t first = base + __shfl((long long)(upto - mine), l);
      if (by_row) {
        it.tile = 0;
        it.part = (int)first;  // the request's first item
      } else {
        const int in = uniform((int)(want - first));
        it.tile = it.tiles - 1 - in / it.parts;
        it.part = in % it.parts;
      }
      return true;
    }
    base += __shfl((long long)upto, kWave - 1);
  }
  return false;
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

__device__ __forceinline__ float over_groups_max(float v) {  // of the 4 lanes that hold a row
  v = fmaxf(v, __shfl_xor(v, 16));
  return fmaxf(v, __shfl_xor(v, 32));
}
__device__ __forceinline__ float over_groups_sum(float v) {
  v += __shfl_xor(v, 16);
  return v + __shfl_xor(v, 32);
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
  __device__ __forceinline__ Sight(const AttnParams& a, int end, int p) : last(a.causal && p < end ? p : end - 1), low(a.window != 0 ? p - a.window : -1) {}
  __device__ __forceinline__ bool sees(const AttnParams& a, int token) const { return token <= last && (token > low || token < a.sink); }
};

// An item's steps: those of the first `sink` tokens, then those from its first row's window on.
struct Steps {
  int first, sunk, count;
  __device__ __forceinline__ Steps(const AttnParams& a, int p_least, int end) {
    first = sunk = 0;
    if (a.window != 0) {
      const int from = p_least - a.window + 1;
      first = from > 0 ? from / kStep & ~1 : 0;
      sunk = (a.sink + kStep - 1) / kStep + 1 & ~1;
      if (sunk >= first) first = sunk = 0;
    }
    count = end > 0 ? sunk + (end + kStep - 1) / kStep - first : 0;
  }
  __device__ __forceinline__ int token(int step) const { return (step < sunk ? step : step - sunk + first) * kStep; }
  // The steps [begin, end) of part `part` of `parts`, `chunk` steps each.
  __device__ __forceinline__ void part_of(const Item& it, int& begin, int& end) const {
    const int64_t b = (int64_t)it.part * it.chunk, e = b + it.chunk;
    begin = uniform((int32_t)(b < count ? b : count));
    end = uniform((int32_t)(it.part + 1 == it.parts || e > count ? count : e));
  }
};

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

// A V scale as the softmax takes it: its logarithm goes into the exponent, its inverse into the sum; a scale of zero (or next to it) keeps
// its tokens in the sum and takes their values off the weight.
struct ValueScale {
  float log, inv, rest;
  __device__ __forceinline__ explicit ValueScale(float z) {
    const float used = z < kLeastScale ? kLeastScale : z;
    rest = z < kLeastScale ? z * (1.0f / kLeastScale) : 1.0f;
    log = __builtin_amdgcn_logf(used);
    inv = __builtin_amdgcn_rcpf(used);
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
