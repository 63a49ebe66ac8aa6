// The worker of the attention kernels for few rows: a wave's 16 or 32 query rows over its steps of 32 tokens, and how a block's waves join.  What it
// computes and how the products are laid out: kvh_attention.hip.
#pragma once

#include "kvh_attention.hpp"

namespace kvh {

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

// `table_of()`: the table of the item's pages.
template <int DT, int KIND, int D, int NR, bool PAGE16, typename Table>
__device__ __forceinline__ void attend(const AttnParams& a, const Item& it, Table&& table_of, int head0, int wave, int lane, float* lds, float (*lds_ml)[16 * NR][2]) {
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
  w.table = table_of();
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

}  // namespace kvh
