// kvh_attention: the queries of a request's new tokens over one layer of the paged cache.
//
// S^T = K Q^T and O^T = V^T P^T, tile by tile, with a running maximum and sum (one pass over the cache).  Both products put the
// query rows on the columns of the matrix instruction (16x16x32: lane l holds column l % 16), so everything that belongs to a
// query row - its maximum, its sum, the factor that rescales its output - is a value of the lane's own, and the weights leave
// the first product in the very lanes in which the second one wants them: the order of the tokens inside its sum is free, and
// is chosen so.  The rows of one KV head are the (new token, query head) pairs that read it, token-major: 16 of them a tile.
//
// A code enters the products as the number it is (an int8 or e4m3 is exact in fp16; the queries are brought to fp16 with a power of
// two of their row's own), the K scale of its page multiplies the finished dot product, and the V scale sv of its page enters the
// exponent: with s' = s + log2 sv and m' = max s', the weight exp2(s' - m') <= 1 multiplies the code and exp2(s' - m') / sv adds
// to the sum.  A weight is thus as exact as fp16 is, however the scales of a request's pages differ between 2^-60 (kLeastScale) and 2^60.
//
// This kernel is the one for few rows (single tokens, short questions): each byte of the cache is read once and used by 16 rows at most, so it is bound
// by memory, and where little is read by the chain table -> page -> scores -> values of a step.  Keys and values go from memory to the
// registers that the matrix instructions take them from, without LDS: no other wave wants them.
// Measured: 64 requests of 4096 tokens (lognormal), 8 KV heads of 128, 32 query heads: bf16 186 us = 5.2 TB/s (a plain read reaches 6.5), int8 and e4m3 110 us =
// 4.4 TB/s (a head's rows are 128 bytes there; waves wait for memory 57 % of their time, vector instructions take 39 % of the SIMDs': too little is under
// way at a time); one of 131072, e4m3: 67 us = 4.0 TB/s, 10 of them joining; one of 300: 8.6 us.
#include "kvh_attention.hpp"

#include <algorithm>

namespace kvh {
namespace {

// ---- the kernel ---------------------------------------------------------------------------------------------------
// NR tiles of 16 query rows share each K and V tile that is read.  PAGE16: pages hold a multiple of 16 tokens, so a tile lies on
// one page and its address and scales are the wave's; otherwise every lane looks its tokens' pages up.
template <int DT, int KIND, int D, int NR, bool PAGE16>
struct Worker {
  static constexpr bool kBf = kBf16<DT, KIND>;
  static constexpr bool kScaled = KIND != KVH_CACHE_16;
  static constexpr int kWidth = kScaled ? 1 : 2;
  static constexpr int kSums = D / 32;                 // matrix instructions of a dot product
  static constexpr int kChans = D / 16;                // channels of V that a lane reads of a token, and channel tiles of the output
  static constexpr int kKWords = D * kWidth / 16;      // words of K that a lane reads of a tile
  static constexpr int kVWords = kChans * kWidth / 4;  // words of V that a lane reads of a token
  static constexpr int kScales = kScaled ? (PAGE16 ? 2 : 8) : 1;
  // Loads of the next step under way while this one is worked on: where lanes look pages up before they load and registers allow it (40 requests
  // of 4000, pages of 24, D 64: int8 63 us, 74 without, e4m3 60 and 63; D 128, where it was not kept: 83 and 83, 80 and 80; pages of 16, 64 requests of 4096, int8,
  // D 128: 114 and 110).
  static constexpr bool kAhead = NR == 1 && kScaled && !PAGE16 && D == 64;

  // A step's tokens as they are in the cache.  Token slot 4 i + r of a lane is token 16 i + 4 grp + r of the step.
  struct Raw {
    Words<kKWords> k[2];
    Words<kVWords> v[8];
    float ks[kScales], vs[kScales];  // of the step's two tiles (PAGE16), or of the lane's token slots
    uint32_t absent;                 // token slots on no page of the cache
  };

  const AttnParams& a;
  Request rq;
  const int32_t* table;
  int head, row0, rows;  // of the tile: its first row, rows it has
  int lane, l16, grp;
  int end;               // tokens at and past it are seen by no row
  int p_least, p_most;   // logical positions of the tile's first and last row

  u32x4 q[NR][kSums];
  float coef[NR];  // what turns a dot product into an exponent of 2
  Sight sight[NR];
  f32x4 o[NR][kChans];
  float m[NR], l[NR];
  PageRun run;
  int in, row;           // PAGE16: where the next tile of 16 tokens lies: in the request's page `in`, `row` rows from its start
  uint32_t k_from, v_from;  // PAGE16: bytes from a tile's first row to what the lane reads of it
  bool bad;  // a token that a row should see lies on no page of the cache

  __device__ __forceinline__ Worker(const AttnParams& a_) : a(a_) {}

  // Channel of element i of sum kk in lane group g, the same for K and Q.  K is read in 16-byte pieces: 8 channels of 16 bits, or 16 of 8
  // bits for two sums.
  static __device__ __forceinline__ int channel(int kk, int g) {
    return KIND == KVH_CACHE_16 ? kk * 32 + g * 8 : (kk / 2) * 64 + g * 16 + (kk % 2) * 8;
  }

  __device__ __forceinline__ void begin() {
#pragma unroll
    for (int t = 0; t < NR; ++t) {
      const int r = t * 16 + l16;
      const bool real = r < rows;
      const int at = row0 + (real ? r : 0), token = (int)a.by_group.quotient((uint32_t)at), u = at - token * a.group;
      sight[t] = Sight(a, end, rq.len - rq.n + token);
      const uint16_t* src = a.q + ((int64_t)rq.start + token) * a.q_ts + ((int64_t)head * a.group + u) * D;
      float most = 0.0f;
      u32x4 raw[kSums];
#pragma unroll
      for (int kk = 0; kk < kSums; ++kk) {
        raw[kk] = u32x4{0, 0, 0, 0};
        if (real) raw[kk] = *reinterpret_cast<const u32x4*>(src + channel(kk, grp));
      }
      coef[t] = a.scale * kLog2e;
      if constexpr (KIND != KVH_CACHE_16 && DT == KVH_BF16) {
        // bf16 -> fp16 with a power of two that brings the row's largest value to [1, 2)
#pragma unroll
        for (int kk = 0; kk < kSums; ++kk) {
          float x[8];
          widen8<DT>(raw[kk], x);
#pragma unroll
          for (int e = 0; e < 8; ++e) most = fmaxf(most, fabsf(x[e]));
        }
        most = over_groups_max(most);
        const f32x2 power = row_power(most);
        coef[t] *= power[1];
#pragma unroll
        for (int kk = 0; kk < kSums; ++kk) {
          float x[8];
          widen8<DT>(raw[kk], x);
#pragma unroll
          for (int e = 0; e < 4; ++e) q[t][kk][e] = narrow2<KVH_F16>(x[2 * e] * power[0], x[2 * e + 1] * power[0]);
        }
      } else {
#pragma unroll
        for (int kk = 0; kk < kSums; ++kk) q[t][kk] = raw[kk];
      }
      m[t] = -INFINITY;
      l[t] = 0.0f;
#pragma unroll
      for (int ct = 0; ct < kChans; ++ct) o[t][ct] = f32x4{0, 0, 0, 0};
    }
    bad = false;
    const uint32_t row_bytes = (uint32_t)a.c_ts * kWidth;
    k_from = l16 * row_bytes + grp * 16;
    v_from = grp * 4 * row_bytes + l16 * (kChans * kWidth);
  }

  // The next step fetched is that of tokens t0 and on.
  __device__ __forceinline__ void seek(int t0) {
    in = (int)a.by_block.quotient((uint32_t)t0);
    row = t0 - in * a.block_tokens;
  }

  // Starts the loads of tokens [t0, t0 + 32), t0 < end, where seek or the step before left off.  Nothing here waits for them.
  __device__ __forceinline__ void fetch_step(Raw& x, int t0) {
    const int last = end - 1;
    const int64_t row_bytes = a.c_ts * kWidth, head_at = (int64_t)head * D * kWidth;
    x.absent = 0;
    if constexpr (PAGE16) {
      // A tile lies on one page: its rows past the end are the page's too, and only have to be kept from the sums.
      if ((unsigned)(in - run.base) > (unsigned)(kWave - 2)) run.load(a, table, in, (int)a.by_block.quotient((uint32_t)last), lane);
      int64_t at = 0;
      int page = 0;
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        if (i == 0 || t0 + 16 <= last) {  // a tile past the end stands for the one before
          page = uniform(__builtin_amdgcn_readlane(run.entry, in - run.base));
          if (page < 0) {
            page = 0;
            x.absent |= 15u << 4 * i;
          }
          at = ((int64_t)page * a.block_tokens + row) * row_bytes + head_at;
          row += 16;
          if (row == a.block_tokens) row = 0, ++in;
        }
#pragma unroll
        for (int j = 0; j < kKWords / 4; ++j) {
          const u32x4 w = *reinterpret_cast<const u32x4*>(a.ck + at + k_from + j * 64);
#pragma unroll
          for (int e = 0; e < 4; ++e) x.k[i].w[4 * j + e] = w[e];
        }
#pragma unroll
        for (int r = 0; r < 4; ++r) x.v[4 * i + r] = fetch<kVWords>(a.cv + at + r * row_bytes + v_from);
        if constexpr (kScaled) {
          x.ks[i] = a.sk[(int64_t)page * a.s_ps + head];
          x.vs[i] = a.sv[(int64_t)page * a.s_ps + head];
        }
      }
    } else {
      const int at0 = (int)a.by_block.quotient((uint32_t)t0), tz = t0 + kStep - 1 < last ? t0 + kStep - 1 : last;
      const int at1 = (int)a.by_block.quotient((uint32_t)tz);
      if (at0 < run.base || at1 - run.base >= kWave) run.load(a, table, at0, (int)a.by_block.quotient((uint32_t)last), lane);
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int t = t0 + 16 * i + l16 < last ? t0 + 16 * i + l16 : last;  // a token past the end stands for the last one
        const int at = (int)a.by_block.quotient((uint32_t)t);
        const int page = __shfl(run.entry, at - run.base);
        const int64_t r = (int64_t)(page < 0 ? 0 : page) * a.block_tokens + (t - at * a.block_tokens);
        const uint8_t* kp = a.ck + head_at + r * row_bytes + grp * 16;
#pragma unroll
        for (int j = 0; j < kKWords / 4; ++j) {
          const u32x4 w = *reinterpret_cast<const u32x4*>(kp + j * 64);
#pragma unroll
          for (int e = 0; e < 4; ++e) x.k[i].w[4 * j + e] = w[e];
        }
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int tok = t0 + 16 * (i / 4) + grp * 4 + i % 4, t = tok < last ? tok : last;
        const int at = (int)a.by_block.quotient((uint32_t)t);
        int page = __shfl(run.entry, at - run.base);
        if (page < 0) {
          page = 0;
          x.absent |= 1u << i;
        }
        const int64_t r = (int64_t)page * a.block_tokens + (t - at * a.block_tokens);
        x.v[i] = fetch<kVWords>(a.cv + head_at + r * row_bytes + l16 * (kChans * kWidth));
        if constexpr (kScaled) {
          x.ks[i] = a.sk[(int64_t)page * a.s_ps + head];
          x.vs[i] = a.sv[(int64_t)page * a.s_ps + head];
        }
      }
    }
  }

  // Takes the tokens [t0, t0 + 32) into the sums.
  __device__ __forceinline__ void take(Raw& x, int t0) {
    // Whether some row does not see all of these tokens.
    const bool hidden_any = t0 + kStep > end || (a.causal && t0 + kStep - 1 > p_least) || (a.window != 0 && t0 <= p_most - a.window) ||
                            (PAGE16 ? x.absent != 0 : __any(x.absent != 0));
    float lsv[kScales], inv[kScales], rest[kScales];
    bool rare = false;  // some scale leaves a rest
    if constexpr (kScaled) {
      ScaleRange range;
#pragma unroll
      for (int i = 0; i < kScales; ++i) range.add(x.ks[i], x.vs[i]);
      rare = __any(range.rare());
      if (__builtin_expect(rare, 0)) {
#pragma unroll
        for (int i = 0; i < kScales; ++i) {
          const ValueScale z(x.vs[i]);
          x.vs[i] = z.used, rest[i] = z.rest;
          if (odd_scale(x.ks[i])) x.ks[i] = NAN;  // and so are the scores, until those are hidden that a row does not see
        }
      }
#pragma unroll
      for (int i = 0; i < kScales; ++i) lsv[i] = __builtin_amdgcn_logf(x.vs[i]), inv[i] = __builtin_amdgcn_rcpf(x.vs[i]);
    }
    auto of = [](int i) { return PAGE16 ? i / 4 : i; };  // token slot -> its scale

    f32x4 s[NR][2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
#pragma unroll
      for (int t = 0; t < NR; ++t) s[t][i] = f32x4{0, 0, 0, 0};
#pragma unroll
      for (int kk = 0; kk < kSums; ++kk) {
        u32x4 kop;
        if constexpr (!kScaled) {
#pragma unroll
          for (int e = 0; e < 4; ++e) kop[e] = x.k[i].w[4 * kk + e];
        } else {
          uint32_t w[4];
          widen4<KIND>(x.k[i].w[2 * kk], w[0], w[1]);
          widen4<KIND>(x.k[i].w[2 * kk + 1], w[2], w[3]);
#pragma unroll
          for (int e = 0; e < 4; ++e) kop[e] = w[e];
        }
#pragma unroll
        for (int t = 0; t < NR; ++t) s[t][i] = mfma<kBf>(kop, q[t][kk], s[t][i]);
      }
    }

    u32x4 p[NR];
#pragma unroll
    for (int t = 0; t < NR; ++t) {
      float y[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        if constexpr (!kScaled)
          y[i] = s[t][i / 4][i % 4] * coef[t];
        else
          y[i] = __builtin_fmaf(s[t][i / 4][i % 4], x.ks[of(i)] * coef[t], lsv[of(i)]);
      }
      if (hidden_any) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const bool seen = sight[t].sees(a, t0 + 16 * (i / 4) + grp * 4 + i % 4), none = (x.absent >> i & 1u) != 0;
          bad |= seen && none;
          if (!seen || none) y[i] = -INFINITY;
        }
      }
      float most = y[0];
#pragma unroll
      for (int i = 1; i < 8; ++i) most = fmaxf(most, y[i]);
      most = over_groups_max(most);
      // The maximum is followed at once (the kernel for many rows lets it lag): the largest weight is then 1, which rounds to itself, and
      // often decides the row.  bf16, one token: 1.2 times the error of the output's own rounding against 1.35.
      if (__any(most > m[t])) {
        const float now = fmaxf(m[t], most);
        const float down = now == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(m[t] - now);
        m[t] = now;
        l[t] *= down;
#pragma unroll
        for (int ct = 0; ct < kChans; ++ct) o[t][ct] *= down;
      }
      const float top = m[t] == -INFINITY ? 0.0f : m[t];  // nothing seen yet: the weights below are zeros
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        y[i] = __builtin_amdgcn_exp2f(y[i] - top);
        if constexpr (!kScaled)
          l[t] += y[i];
        else
          l[t] = __builtin_fmaf(y[i], inv[of(i)], l[t]);
      }
      if constexpr (kScaled) {
        if (__builtin_expect(rare, 0)) {
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const bool none = hidden_any && (!sight[t].sees(a, t0 + 16 * (i / 4) + grp * 4 + i % 4) || (x.absent >> i & 1u) != 0);
            y[i] = none ? 0.0f : y[i] * rest[of(i)];  // the rest may be NaN
          }
        }
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) p[t][e] = narrow2<kBf ? KVH_BF16 : KVH_F16>(y[2 * e], y[2 * e + 1]);
    }

    if (hidden_any) {
      // What no row sees is not multiplied at all; what some rows see and others do not may only meet those that do.
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int tok = t0 + 16 * (i / 4) + grp * 4 + i % 4;
        const bool none = tok >= end || (x.absent >> i & 1u);
#pragma unroll
        for (int e = 0; e < kVWords; ++e) x.v[i].w[e] = none ? 0u : x.v[i].w[e];
      }
      if constexpr (KIND != KVH_CACHE_I8) {
        bool any = false;  // an infinity or NaN among them
#pragma unroll
        for (int i = 0; i < 8; ++i)
#pragma unroll
          for (int e = 0; e < kVWords; ++e) any |= has_odd<DT, KIND>(x.v[i].w[e]);
        if (__any(any)) {
          weigh<true>(x.v, p, t0);
          return;
        }
      }
    }
    weigh<false>(x.v, p, t0);
  }

  // The second product: ODD where some values are infinities or NaN that some rows do not see.
  template <bool ODD>
  __device__ __forceinline__ void weigh(const Words<kVWords> (&v)[8], const u32x4 (&p)[NR], int t0) {
    using Bad = Odd<kBf>;
    u32x4 one[ODD ? NR : 1];  // of the tokens that the lane's row sees
    if constexpr (ODD) {
#pragma unroll
      for (int t = 0; t < NR; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          one[t][e] = 0;
#pragma unroll
          for (int n = 0; n < 2; ++n)
            if (sight[t].sees(a, t0 + 16 * (e / 2) + grp * 4 + 2 * (e % 2) + n)) one[t][e] |= Bad::kOne << 16 * n;
        }
    }
#pragma unroll
    for (int c4 = 0; c4 < kVWords; ++c4) {
      constexpr int kPer = 4 / kWidth;  // channels of a word
      uint32_t z[4][kPer];              // pairs of tokens, of each channel
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        if constexpr (KIND == KVH_CACHE_16) {
          z[e][0] = __builtin_amdgcn_perm(v[2 * e + 1].w[c4], v[2 * e].w[c4], 0x05040100u);
          z[e][1] = __builtin_amdgcn_perm(v[2 * e + 1].w[c4], v[2 * e].w[c4], 0x07060302u);
        } else {
          zip4<KIND>(v[2 * e].w[c4], v[2 * e + 1].w[c4], z[e]);
        }
      }
#pragma unroll
      for (int j = 0; j < kPer; ++j) {
        const u32x4 vop = {z[0][j], z[1][j], z[2][j], z[3][j]};
#pragma unroll
        for (int t = 0; t < NR; ++t) {
          f32x4& to = o[t][c4 * kPer + j];
          to = mfma<kBf>(ODD ? Bad::without(vop) : vop, p[t], to);
          if constexpr (ODD) {
#pragma unroll 1
            for (int which = 0; which < 3; ++which) {
              const f32x4 hit = mfma<kBf>(Bad::ones(vop, which), one[t], f32x4{0, 0, 0, 0});
#pragma unroll
              for (int r = 0; r < 4; ++r) to[r] += hit[r] > 0.0f ? Bad::value(which) : 0.0f;
            }
          }
        }
      }
    }
  }

  // Steps [s0, s1).
  __device__ __forceinline__ void walk(const Steps& steps, int s0, int s1) {
    if (s0 >= s1) return;
    int t = steps.token(s0);
    seek(t);
    if constexpr (!kAhead) {
      for (int s = s0; s < s1; ++s) {
        const int t1 = steps.token(s);
        if (s > s0 && t1 != t + kStep) seek(t1);
        t = t1;
        Raw x;
        fetch_step(x, t);
        take(x, t);
      }
    } else {
      Raw x[2];
      fetch_step(x[0], t);
      auto next = [&](int s, Raw& to) {  // the step after s
        if (s + 1 >= s1) return t;
        const int t1 = steps.token(s + 1);
        if (t1 != t + kStep) seek(t1);
        fetch_step(to, t1);
        return t1;
      };
      for (int s = s0;;) {
        int t1 = next(s, x[1]);
        take(x[0], t);
        t = t1;
        if (++s >= s1) break;
        t1 = next(s, x[0]);
        take(x[1], t);
        t = t1;
        if (++s >= s1) break;
      }
    }
  }
};

constexpr int kLogFewWaves = 2, kFewWaves = 1 << kLogFewWaves, kFewThreads = kFewWaves * kWave;

constexpr int few_log_rows(int nr) { return nr == 1 ? 4 : 5; }

template <int DT, int KIND, int D, int NR, bool PAGE16>
__device__ __forceinline__ void attend(const AttnParams& a, const Item& it, int head0, int wave, int lane, float* lds, float (*lds_ml)[16 * NR][2]) {
  using W = Worker<DT, KIND, D, NR, PAGE16>;
  constexpr int kTile = 16 * NR;
  constexpr int kPitch = D + 4;  // floats of a row in LDS
  W w(a);
  w.lane = lane, w.l16 = lane % 16, w.grp = lane / 16;
  w.rq = it.rq;
  w.head = head0 + (wave & (1 << a.log_hw) - 1);
  w.row0 = it.tile * kTile;
  const int all = it.rq.n * a.group;
  w.rows = all - w.row0 < kTile ? all - w.row0 : kTile;
  w.p_least = it.rq.len - it.rq.n + (int)a.by_group.quotient((uint32_t)w.row0);
  w.p_most = it.rq.len - it.rq.n + (int)a.by_group.quotient((uint32_t)(w.row0 + w.rows - 1));
  w.end = a.causal && w.p_most + 1 < it.rq.len ? w.p_most + 1 : it.rq.len;
  w.table = a.req.table + (int64_t)it.b * a.req.table_stride;
  w.begin();
  const Steps steps(a, w.p_least, w.end);
  int s0, s1;
  steps.part_of(it, s0, s1);
  const int log_tw = kLogFewWaves - a.log_hw, tw = 1 << log_tw;  // the waves of a head share its steps
  const int mine = (s1 - s0 + tw - 1) >> log_tw;
  const int b0 = s0 + (wave >> a.log_hw) * mine, b1 = b0 + mine < s1 ? b0 + mine : s1;
  w.walk(steps, b0, b1);
  if (__any(w.bad) && lane == 0 && a.status != nullptr) a.status[it.b] = KVH_DEV_BAD_REQUEST;

  // The results of a head's waves become one.
#pragma unroll
  for (int t = 0; t < NR; ++t) {
    const float sum = over_groups_sum(w.l[t]);
    if (w.grp == 0) {
      lds_ml[wave][t * 16 + w.l16][0] = w.m[t];
      lds_ml[wave][t * 16 + w.l16][1] = sum;
    }
  }
  const int log_hw = a.log_hw, hw = 1 << log_hw;
#pragma unroll
  for (int t = 0; t < NR; ++t) {
    if (t * 16 >= w.rows) break;
    if (t > 0) __syncthreads();
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
      for (int ct = 0; ct < W::kChans; ct += 4) {
        const f32x4 x = {w.o[t][ct][r], w.o[t][ct + 1][r], w.o[t][ct + 2][r], w.o[t][ct + 3][r]};
        *reinterpret_cast<f32x4*>(&lds[(wave * 16 + w.l16) * kPitch + (4 * w.grp + r) * W::kChans + ct]) = x;
      }
    __syncthreads();
    // a thread: D / 16 channels of one row, head by head.  The start is 0 in a form that the compiler takes for the lane's own: with a plain 0
    // one request of 300 takes 9.4 us, so 8.8.
    const int r = threadIdx.x % 256 / 16, ch = (threadIdx.x % 16) * W::kChans, row = t * 16 + r;
    for (int h = threadIdx.x / 256; h < hw && row < w.rows; h += kFewWaves / 4) {
      const int head = head0 + h;
      float m = -INFINITY;
      for (int v = h; v < kFewWaves; v += hw) m = fmaxf(m, lds_ml[v][row][0]);
      float l = 0.0f, x[W::kChans];
#pragma unroll
      for (int e = 0; e < W::kChans; ++e) x[e] = 0.0f;
      for (int v = h; v < kFewWaves; v += hw) {
        const float mv = lds_ml[v][row][0], f = mv == m ? 1.0f : __builtin_amdgcn_exp2f(mv - m);
        l = __builtin_fmaf(f, lds_ml[v][row][1], l);
#pragma unroll
        for (int e = 0; e < W::kChans; ++e) x[e] = __builtin_fmaf(f, lds[(v * 16 + r) * kPitch + ch + e], x[e]);
      }
      if (it.split) {
        const int64_t at = (it.slot * a.heads + head) * kTile + row;
        float* to = a.part + at * D + ch;
#pragma unroll
        for (int e = 0; e < W::kChans; e += 4) *reinterpret_cast<f32x4*>(to + e) = f32x4{x[e], x[e + 1], x[e + 2], x[e + 3]};
        if (ch == 0) *reinterpret_cast<f32x2*>(a.part_ml + at * 2) = f32x2{m, l};
      } else {
        const int at = w.row0 + row, token = (int)a.by_group.quotient((uint32_t)at), u = at - token * a.group;
        const bool blind = it.rq.len == 0 || (a.causal && it.rq.len - it.rq.n + token < 0);
        const float by = 1.0f / l;
        const int64_t packed = (int64_t)it.rq.start + token;
        uint16_t* to = a.out + packed * a.o_ts + ((int64_t)head * a.group + u) * D + ch;
        uint32_t y[W::kChans / 2];
#pragma unroll
        for (int e = 0; e < W::kChans / 2; ++e) y[e] = blind ? 0u : narrow2<DT>(x[2 * e] * by, x[2 * e + 1] * by);
        if constexpr (W::kChans == 8)
          *reinterpret_cast<u32x4*>(to) = u32x4{y[0], y[1], y[2], y[3]};
        else
          *reinterpret_cast<u32x2*>(to) = u32x2{y[0], y[1]};
        if (a.lse != nullptr && ch == 0)
          a.lse[packed * ((int64_t)a.heads * a.group) + (int64_t)head * a.group + u] = blind ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * kLn2;
      }
    }
  }
}

template <int DT, int KIND, int D, int NR, bool PAGE16>
__global__ __launch_bounds__(kFewThreads, 8 / kFewWaves) void attention_kernel(AttnParams a) {
  __shared__ float lds[kFewWaves * 16 * (D + 4)];
  __shared__ float lds_ml[kFewWaves][16 * NR][2];
  int lane = threadIdx.x % kWave;
  const int wave = uniform((int32_t)(threadIdx.x / kWave));
  // The head groups of an item run on one XCD (consecutive blocks go to the 8 of them in turn), one after the other: they read neighbouring memory.
  const uint32_t g = blockIdx.x / 8, hi = a.by_heads.quotient(g), k = hi * 8 + blockIdx.x % 8;
  const int head = (int)(g - hi * a.by_heads.d) << a.log_hw;
  tell_refused(a);
  Item it;
  for (Items items; items.next(a, few_log_rows(NR), k, head == 0 && wave == 0, lane, it);) {
    if (it.split && it.slot >= a.slots) continue;  // requests that share rows of the batch
    attend<DT, KIND, D, NR, PAGE16>(a, it, head, wave, lane, lds, lds_ml);
    __syncthreads();
  }
}

// Joins the partial results of the tiles that were cut: WAVES waves take one row, all of a block's where there are few rows, whose parts are
// then many, and one where there are many.
// The parts' factors come first, 64 in the lanes, so that the sums are loads that wait for nothing but each other.
template <int DT, int D, int WAVES>
__global__ __launch_bounds__(kBlockThreads) void join_kernel(AttnParams a, int log_rows) {
  constexpr int kPer = D / 64, kAtOnce = WAVES == 1 ? 8 : 16, kLogRows = WAVES == 1 ? 2 : 0;  // of a block
  __shared__ float lds[WAVES > 1 ? WAVES : 1][D];
  const int lane = threadIdx.x % kWave, wave = uniform((int32_t)(threadIdx.x / kWave));
  const uint32_t unit = blockIdx.x >> (log_rows - kLogRows), tile = a.by_heads.quotient(unit);
  const int head = (int)(unit - tile * (uint32_t)a.heads);
  const int share = WAVES == 1 ? 0 : wave;  // the wave's parts of 64: those, and every WAVES-th after them
  const int row = ((int)(blockIdx.x & ((1u << (log_rows - kLogRows)) - 1)) << kLogRows) + (WAVES == 1 ? wave : 0);
  const u32x4* from_joint = reinterpret_cast<const u32x4*>(a.joints + tile);
  const u32x4 j0 = from_joint[0], j1 = from_joint[1];
  if (tile >= (uint32_t)uniform(*a.joints_n)) return;  // (the room is there; what it holds is of no account)
  const int start = uniform((int32_t)j0[0]), n = uniform((int32_t)j0[1]), len = uniform((int32_t)j0[2]), parts = uniform((int32_t)j1[0]);
  const int64_t slot = uniform((int64_t)((uint64_t)j1[3] << 32 | j1[2]));
  if (parts == 1 || slot + parts > a.slots) return;  // (past them: requests that share rows of the batch)
  const int64_t row0 = (int64_t)uniform((int32_t)j0[3]) << log_rows, all = (int64_t)n * a.group;
  const int64_t next = (int64_t)a.heads << log_rows;  // rows of partial results from one part to the next
  const int q_heads = a.heads * a.group;
  if (row0 + row >= all) return;
  const int64_t first = ((slot * a.heads + head) << log_rows) + row;
  float m = -INFINITY, l = 0.0f, x[kPer];
#pragma unroll
  for (int e = 0; e < kPer; ++e) x[e] = 0.0f;
  for (int p0 = 0; p0 < parts; p0 += kWave) {
    const int here = parts - p0 < kWave ? parts - p0 : kWave;
    const float* from = a.part + (first + p0 * next) * D + lane * kPer;
    float y[kAtOnce][kPer];
    auto fetch_parts = [&](int i) {
#pragma unroll
      for (int e = 0; e < kAtOnce; ++e)
#pragma unroll
        for (int c = 0; c < kPer; ++c) {
          const int p = (i + e) * WAVES + share;
          y[e][c] = p < here ? from[(int64_t)p * next * D + c] : 0.0f;
        }
    };
    fetch_parts(0);
    f32x2 ml = {-INFINITY, 0.0f};
    if (lane < here) ml = *reinterpret_cast<const f32x2*>(a.part_ml + 2 * (first + (p0 + lane) * next));
    float most = ml[0];
#pragma unroll
    for (int d = 1; d < kWave; d *= 2) most = fmaxf(most, __shfl_xor(most, d));
    const float now = fmaxf(m, most), down = m == now ? 1.0f : __builtin_amdgcn_exp2f(m - now);
    m = now;
    const float f = lane < here ? (ml[0] == now ? 1.0f : __builtin_amdgcn_exp2f(ml[0] - now)) : 0.0f;
    float sum = f * ml[1];
#pragma unroll
    for (int d = 1; d < kWave; d *= 2) sum += __shfl_xor(sum, d);
    l = __builtin_fmaf(l, down, sum);
#pragma unroll
    for (int c = 0; c < kPer; ++c) x[c] *= down;
    for (int i = 0; i * WAVES < here; i += kAtOnce) {
      if (i > 0) fetch_parts(i);
#pragma unroll
      for (int e = 0; e < kAtOnce; ++e) {
        const int p = (i + e) * WAVES + share;
        const float by = p < here ? __shfl(f, p & (kWave - 1)) : 0.0f;
#pragma unroll
        for (int c = 0; c < kPer; ++c) x[c] = __builtin_fmaf(by, y[e][c], x[c]);
      }
    }
  }
  if constexpr (WAVES > 1) {
#pragma unroll
    for (int c = 0; c < kPer; ++c) lds[wave][lane * kPer + c] = x[c];
    __syncthreads();
    if (wave != 0) return;
#pragma unroll
    for (int c = 0; c < kPer; ++c)
#pragma unroll
      for (int w = 1; w < WAVES; ++w) x[c] += lds[w][lane * kPer + c];
  }
  const int64_t at = row0 + row;
  const int token = (int)a.by_group.quotient((uint32_t)at), u = head * a.group + (int)(at - (int64_t)token * a.group);
  const int64_t packed = (int64_t)start + token;
  const bool blind = len == 0 || (a.causal && len - n + token < 0);
  const float by = 1.0f / l;
  uint16_t* to = a.out + packed * a.o_ts + (int64_t)u * D + lane * kPer;
  if constexpr (kPer == 2)
    *reinterpret_cast<uint32_t*>(to) = blind ? 0u : narrow2<DT>(x[0] * by, x[1] * by);
  else
    *to = blind ? 0 : (uint16_t)narrow2<DT>(x[0] * by, 0.0f);
  if (a.lse != nullptr && lane == 0) a.lse[packed * q_heads + u] = blind ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * kLn2;
}

// ---- launch -------------------------------------------------------------------------------------------------------
// Rules with both sides measured (us, 8 KV heads of 128, 32 query heads unless said; "after": new tokens after cached ones).
// Blocks of 4 waves that fill the chip: 2 on a compute unit, for which 16 bits of 128 channels have registers (190).  Others would have room for more (int8
// of 128 channels 3, at 130 registers; heads of 64 4, at 100 to 127), which is not tried.  Chunks for 512 / 256 / 1024 blocks: 512 after 32768,
// int8: 391 / 590 / 419; one of 131072, e4m3: 67 / 62 / 67; 64 of 4096, int8: 113 / - / 119.
constexpr int kFill = 512;
// Steps of a chunk at least: 4, one for each wave (one request of 2100: 12; 16 steps: 15), but 16 where a wave takes all of a chunk by itself
// (8 of 6000, bf16: 50; 4 steps: 53).
constexpr int kLeastSteps = 4, kLeastWide = 16;
// Steps that cutting has to take from the longest tile to be worth the partial results and the second launch.  Few rows: one of 700 cut 11, whole
// 13; 16 of 500 cut 18, whole 12.  Many: 128 after 1000 cut 25, whole 45; a prompt of 1024 cut 53, whole 42; 8 of 300 after 500 cut 98, whole 70.
constexpr int kGainFew = 16, kGainMany = 24;
// Steps of all heads from which on a block's waves take neighbouring heads, whose rows of a token lie together, and not parts of one head's tokens, which
// shorten what a step waits for: 64 of 4096, int8: 110, 126 by tokens; 4 of 10000, int8: 28 by tokens, 35 by heads; one of 8000: 16 and 32.
constexpr int kWideSteps = 40 * kFill;

// 17 to 32 rows: two tiles of 16 share what is read, but for 128 channels of 16 bits, where both tiles' outputs do not fit the registers beside it; the
// kernel for many rows takes those.  16 requests, 8 after 4000: int8 62, with the other kernel 68; e4m3, which spills 25 registers of 128 channels, 64 and
// 70 (pages of 24, 38 spilled: 77 and 73); bf16 95 and 82; bf16 with heads of 64: 46 and 52.
// More rows are the other kernel's (9 after 8000: 25; with pairs of tiles 44).
template <int KIND, int D>
constexpr bool kTwoTiles = KIND != KVH_CACHE_16 || D == 64;
bool two_tiles(int kind, int head_dim) { return kind != KVH_CACHE_16 || head_dim == 64; }

struct Plan {
  int nr;          // tiles of 16 rows of the kernel for few rows; 0: the kernel for many
  int log_rows;    // of a tile
  int log_hw;      // heads that a block takes where it takes several
  int64_t tiles;   // row tiles of the batch at most
  int64_t target;  // chunks, where the batch is cut
  size_t slot;     // bytes of a partial result, of all heads
  // Whether a batch of this size is cut at all: its tiles alone may give every block two of them to do.
  bool may_cut(int heads) const { return tiles * heads < 2 * kFill; }
  int64_t slots() const { return target + tiles; }
  size_t joints() const { return (size_t)(tiles + 1) * sizeof(Joint); }  // bytes: what the joining kernel reads
};

Plan plan_of(int n_requests, int max_new, int n_tokens, int heads, int q_heads, int head_dim, bool two_tiles) {
  Plan p;
  const int64_t group = q_heads / heads;
  const int64_t most = (int64_t)(max_new < n_tokens ? max_new : n_tokens) * group;
  p.nr = most <= 16 ? 1 : most <= 32 && two_tiles ? 2 : 0;
  p.log_rows = p.nr != 0 ? few_log_rows(p.nr) : kLogManyRows;
  p.log_hw = 0;
  if (p.nr != 0)
    while (p.log_hw < kLogFewWaves && (heads >> p.log_hw & 1) == 0) ++p.log_hw;
  p.tiles = ((int64_t)n_tokens * group >> p.log_rows) + n_requests;
  p.target = (int64_t)((kFill + heads - 1) / heads) << p.log_hw;
  p.slot = (size_t)heads * (head_dim + 2) * sizeof(float) << p.log_rows;
  return p;
}

template <int DT, int KIND, int D, int NR>
void launch_pages(const AttnParams& a, dim3 grid, hipStream_t stream) {
  if (a.block_tokens % 16 == 0)  // 64 requests of 4096, int8: 110 us, 124 by looking every token up; one of 300: 8.5 and 9.3
    launch_kernel(attention_kernel<DT, KIND, D, NR, true>, grid, dim3(kFewThreads), 0, stream, a);
  else
    launch_kernel(attention_kernel<DT, KIND, D, NR, false>, grid, dim3(kFewThreads), 0, stream, a);
}

template <int DT, int KIND, int D>
void launch_rows(const AttnParams& a, int nr, dim3 grid, hipStream_t stream) {
  if constexpr (kTwoTiles<KIND, D>) {
    if (nr == 2) return launch_pages<DT, KIND, D, 2>(a, grid, stream);
  }
  launch_pages<DT, KIND, D, 1>(a, grid, stream);
}

template <int DT, int KIND>
void launch_dim(const AttnParams& a, int head_dim, int nr, dim3 grid, hipStream_t stream) {
  if (head_dim == 128)
    launch_rows<DT, KIND, 128>(a, nr, grid, stream);
  else
    launch_rows<DT, KIND, 64>(a, nr, grid, stream);
}

template <int DT>
void launch_kind(const AttnParams& a, int kind, int head_dim, int nr, dim3 grid, hipStream_t stream) {
  switch (kind) {
    case KVH_CACHE_16: return launch_dim<DT, KVH_CACHE_16>(a, head_dim, nr, grid, stream);
    case KVH_CACHE_I8: return launch_dim<DT, KVH_CACHE_I8>(a, head_dim, nr, grid, stream);
    default: return launch_dim<DT, KVH_CACHE_E4M3>(a, head_dim, nr, grid, stream);
  }
}

template <int DT, int D>
void launch_join(const AttnParams& a, int64_t tiles, int log_rows, hipStream_t stream) {
  const int64_t rows = tiles * a.heads << log_rows;
  if (rows <= 4096)  // one of 128K tokens (128 rows, 256 parts): 10 us, 23 with a wave a row; 512 after 32K (17408 rows, 4 parts): 11 us, 33 with four
    hipLaunchKernelGGL((join_kernel<DT, D, kWavesPerBlock>), dim3((unsigned)rows), dim3(kBlockThreads), 0, stream, a, log_rows);
  else
    hipLaunchKernelGGL((join_kernel<DT, D, 1>), dim3((unsigned)(rows / kWavesPerBlock)), dim3(kBlockThreads), 0, stream, a, log_rows);
}

template <int DT>
void launch_join(const AttnParams& a, int64_t tiles, int head_dim, int log_rows, hipStream_t stream) {
  if (head_dim == 128)
    launch_join<DT, 128>(a, tiles, log_rows, stream);
  else
    launch_join<DT, 64>(a, tiles, log_rows, stream);
}

bool heads_fit(int heads, int q_heads) { return heads >= 1 && q_heads >= heads && q_heads % heads == 0 && q_heads <= 65536; }

}  // namespace
}  // namespace kvh

using namespace kvh;

extern "C" {

size_t kvh_attention_workspace(int n_requests, int max_new, int n_tokens, int heads, int q_heads, int head_dim) {
  if (n_requests < 1 || n_requests > kMaxRequests || max_new < 1 || n_tokens < 1 || !heads_fit(heads, q_heads)) return 0;
  if (head_dim != 64 && head_dim != 128) return 0;
  size_t most = 0;
  for (bool two : {false, true}) {
    const Plan p = plan_of(n_requests, max_new, n_tokens, heads, q_heads, head_dim, two);
    if (p.may_cut(heads)) most = std::max(most, p.joints() + (size_t)p.slots() * p.slot);
  }
  return most;
}

int kvh_attention(const kvh_cache* cache, int layer, const kvh_requests* requests, kvh_dtype dt, const kvh_rows* q,
                  const kvh_rows* out, int q_heads, float* lse_dev, float scale, int causal, int sink, int window,
                  void* workspace_dev, size_t workspace_bytes, int32_t* status_dev, void* stream) {
  if ((dt != KVH_F16 && dt != KVH_BF16) || q == nullptr || out == nullptr) return KVH_E_ARG;
  if (int rc = check_cache(cache)) return rc;
  if (int rc = check_requests(requests)) return rc;
  if (layer < 0 || layer >= cache->layers || !heads_fit(cache->heads, q_heads)) return KVH_E_SHAPE;
  for (const kvh_rows* r : {q, out})
    if (int rc = check_rows(r, (int64_t)q_heads * cache->head_dim, requests->n_tokens)) return rc;
  if (!std::isfinite(scale) || sink < 0 || window < 0 || (window > 0 && !causal) || (window == 0 && sink != 0)) return KVH_E_ARG;
  if (!is_aligned16(workspace_dev) || (reinterpret_cast<uintptr_t>(lse_dev) & 3u) != 0) return KVH_E_ALIGN;
  if (requests->n_tokens == 0) return KVH_OK;
  hipStream_t s = static_cast<hipStream_t>(stream);
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
  a.causal = causal != 0, a.window = window;
  a.sink = (int)std::min<int64_t>(sink, a.req.capacity);  // no request has a token past it, and steps are counted in 32 bits
  a.status = status_dev;
  a.by_block = Divisor((uint32_t)cache->block_tokens);
  a.by_group = Divisor((uint32_t)a.group);
  a.by_heads = Divisor((uint32_t)a.heads);
  if ((int64_t)a.req.max_new * a.group >= (int64_t)1 << 31) return KVH_E_SHAPE;
  Plan p = plan_of(a.req.n, a.req.max_new, a.req.n_tokens, a.heads, q_heads, cache->head_dim, two_tiles(cache->kind, cache->head_dim));
  // The steps of the longest tile, and what all tiles come to at most.  The lengths are the device's; the host knows what the table has room for.
  int64_t longest = std::min<int64_t>((a.req.capacity + kStep - 1) / kStep, 1 << 26);
  if (window != 0) longest = std::min(longest, ((int64_t)window + a.sink + (1 << p.log_rows)) / kStep + 5);
  const int64_t most = std::min<int64_t>(p.tiles * a.heads, 2 * kFill) * longest;
  if (most < kWideSteps) p.target >>= p.log_hw, p.log_hw = 0;
  // What the longest way through the batch is in whole tiles, and cut: with one request the tiles are alike, but for the new tokens that a causal
  // prompt's earlier ones do not see; where there are more tiles than blocks at a time, some wait for the shortest.  Steps in chunks cost a quarter more, with
  // all blocks busy.  One request, bf16, cut and whole: 2100 after 30000 1460 and 2110, 3000 after 30000 2170 and 2140, 3900 after 30000 2890 and
  // 2480, 2500 after 8000 560 and 610, 2500 after 2000 260 and 220, a prompt of 2050 127 and 82.  How the lengths of several requests differ is not known here.
  int64_t gain = longest - kLeastSteps;
  if (a.req.n == 1) {
    int64_t whole = longest;
    if (p.tiles * a.heads > kFill) whole += longest - (causal && window == 0 ? std::min<int64_t>(a.req.n_tokens / kStep, longest) : 0);
    gain = whole - std::max<int64_t>(most / kFill * 5 / 4, kLeastSteps);
  }
  const int64_t room = workspace_dev == nullptr || workspace_bytes < p.joints() ? 0 : (int64_t)((workspace_bytes - p.joints()) / p.slot);
  const bool cut = p.may_cut(a.heads) && gain >= (p.nr == 0 ? kGainMany : kGainFew) && room > p.tiles;
  if (cut && room < p.slots()) p.target = room - p.tiles;
  a.log_hw = p.log_hw;
  a.by_heads = Divisor((uint32_t)(a.heads >> a.log_hw));
  int64_t blocks = cut ? p.target : p.tiles;
  if (p.nr != 0) blocks = (blocks + 7) & ~(int64_t)7;  // see attention_kernel's order
  blocks *= a.by_heads.d;
  if (blocks > 0x7fffffff) return KVH_E_SHAPE;
  a.target = (int)p.target;
  a.least = p.log_hw != 0 ? kLeastWide : kLeastSteps;
  if (cut) {
    a.slots = p.slots();
    a.tiles = p.tiles;
    a.joints_n = static_cast<int32_t*>(workspace_dev);
    a.joints = static_cast<Joint*>(workspace_dev) + 1;
    a.part = reinterpret_cast<float*>(a.joints + p.tiles);
    a.part_ml = a.part + ((size_t)a.slots * a.heads * cache->head_dim << p.log_rows);
  }
  const dim3 grid((unsigned)blocks);
  if (p.nr == 0)
    launch_attention_many(a, dt, cache->kind, cache->head_dim, grid.x, s);
  else if (dt == KVH_F16)
    launch_kind<KVH_F16>(a, cache->kind, cache->head_dim, p.nr, grid, s);
  else
    launch_kind<KVH_BF16>(a, cache->kind, cache->head_dim, p.nr, grid, s);
  KVH_HIP_CHECK_LAUNCH();
  if (cut) {
    a.by_heads = Divisor((uint32_t)a.heads);
    if (dt == KVH_F16)
      launch_join<KVH_F16>(a, p.tiles, cache->head_dim, p.log_rows, s);
    else
      launch_join<KVH_BF16>(a, p.tiles, cache->head_dim, p.log_rows, s);
    KVH_HIP_CHECK_LAUNCH();
  }
  return KVH_OK;
}

}  // extern "C"
