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
// to the sum.  A weight is thus as exact as fp16 is, however the scales of a request's pages differ.
#include "kvh_attention.hpp"

namespace kvh {
namespace {

// ---- the kernel ---------------------------------------------------------------------------------------------------
// NR tiles of 16 query rows share each K and V tile that is read.  PAGE16: pages hold a multiple of 16 tokens, so a tile lies on
// one page and its address and scales are the wave's; otherwise every lane looks its tokens' pages up.
template <int DT, int KIND, int D, int NR, bool PAGE16>
struct Worker {
  static constexpr bool kBf = kBf16<DT, KIND>;
  static constexpr int kWidth = KIND == KVH_CACHE_16 ? 2 : 1;
  static constexpr int kSums = D / 32;           // matrix instructions of a dot product
  static constexpr int kChans = D / 16;          // channels of V that a lane reads of a token, and channel tiles of the output
  static constexpr int kKWords = D * kWidth / 16;       // words of K that a lane reads of a tile
  static constexpr int kVWords = kChans * kWidth / 4;   // words of V that a lane reads of a token

  const AttnParams& a;
  Request rq;
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
  }

  // One step: tokens [t0, t0 + 32), t0 < end, a multiple of 32.
  __device__ __forceinline__ void step(const int32_t* table, int t0) {
    const int last = end - 1;
    Words<kKWords> k[2];
    Words<kVWords> v[8];
    float ks[8], lsv[8], inv[8], rest[8];  // by token slot: 4 i + r is token 16 i + 4 grp + r
    bool hidden_any = false;
    uint32_t absent = 0;  // token slots on no page of the cache
    const int64_t row_bytes = a.c_ts * kWidth;
    const int64_t head_at = (int64_t)head * D * kWidth;
    if constexpr (PAGE16) {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        int t = t0 + 16 * i;
        if (t > last) t = last & ~15;  // a tile past the end reads the last one again, and is masked
        const int at = (int)a.by_block.quotient((uint32_t)t);
        if ((unsigned)(at - run.base) >= (unsigned)kWave) run.load(a, table, at, (int)a.by_block.quotient((uint32_t)last), lane);
        int page = uniform(__builtin_amdgcn_readlane(run.entry, at - run.base));
        if (page < 0) {
          page = 0;
          absent |= 15u << 4 * i;
        }
        const int64_t row = (int64_t)page * a.block_tokens + (t - at * a.block_tokens);
        const uint8_t *kt = a.ck + head_at + row * row_bytes, *vt = a.cv + head_at + row * row_bytes;
        const int most = last - t;  // rows past it are none of the request's: the last one is read again, and masked
        const int kr = l16 < most ? l16 : most;
        const uint8_t* kp = kt + (uint32_t)kr * (uint32_t)row_bytes + grp * 16;
#pragma unroll
        for (int j = 0; j < kKWords / 4; ++j) {
          const u32x4 w = *reinterpret_cast<const u32x4*>(kp + j * 64);
#pragma unroll
          for (int e = 0; e < 4; ++e) k[i].w[4 * j + e] = w[e];
        }
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int vr = grp * 4 + r < most ? grp * 4 + r : most;
          v[4 * i + r] = fetch<kVWords>(vt + (uint32_t)vr * (uint32_t)row_bytes + l16 * (kChans * kWidth));
        }
        if constexpr (KIND != KVH_CACHE_16) {
          const float s = a.sk[(int64_t)page * a.s_ps + head], z = a.sv[(int64_t)page * a.s_ps + head];
#pragma unroll
          for (int r = 0; r < 4; ++r) ks[4 * i + r] = s, lsv[4 * i + r] = z;
        }
      }
    } else {
      const int at0 = (int)a.by_block.quotient((uint32_t)t0), tz = t0 + kStep - 1 < last ? t0 + kStep - 1 : last;
      const int at1 = (int)a.by_block.quotient((uint32_t)tz);
      if (at0 < run.base || at1 - run.base >= kWave) run.load(a, table, at0, (int)a.by_block.quotient((uint32_t)last), lane);
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int t = t0 + 16 * i + l16 < last ? t0 + 16 * i + l16 : last;
        const int at = (int)a.by_block.quotient((uint32_t)t);
        const int page = __shfl(run.entry, at - run.base);
        const int64_t row = (int64_t)(page < 0 ? 0 : page) * a.block_tokens + (t - at * a.block_tokens);
        const uint8_t* kp = a.ck + head_at + row * row_bytes + grp * 16;
#pragma unroll
        for (int j = 0; j < kKWords / 4; ++j) {
          const u32x4 w = *reinterpret_cast<const u32x4*>(kp + j * 64);
#pragma unroll
          for (int e = 0; e < 4; ++e) k[i].w[4 * j + e] = w[e];
        }
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int tok = t0 + 16 * (i / 4) + grp * 4 + i % 4, t = tok < last ? tok : last;
        const int at = (int)a.by_block.quotient((uint32_t)t);
        int page = __shfl(run.entry, at - run.base);
        if (page < 0) {
          page = 0;
          absent |= 1u << i;
        }
        const int64_t row = (int64_t)page * a.block_tokens + (t - at * a.block_tokens);
        v[i] = fetch<kVWords>(a.cv + head_at + row * row_bytes + l16 * (kChans * kWidth));
        if constexpr (KIND != KVH_CACHE_16) {
          ks[i] = a.sk[(int64_t)page * a.s_ps + head];
          lsv[i] = a.sv[(int64_t)page * a.s_ps + head];
        }
      }
    }
    // Whether some row does not see all of these tokens.
    hidden_any = t0 + kStep > end || (a.causal && t0 + kStep - 1 > p_least) || (a.window != 0 && t0 <= p_most - a.window) ||
                 __any(absent != 0);
    if constexpr (KIND != KVH_CACHE_16) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const ValueScale z(lsv[i]);
        lsv[i] = z.log, inv[i] = z.inv, rest[i] = z.rest;
      }
    }

    u32x4 kop[2][kSums];
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int kk = 0; kk < kSums; ++kk) {
        if constexpr (KIND == KVH_CACHE_16) {
#pragma unroll
          for (int e = 0; e < 4; ++e) kop[i][kk][e] = k[i].w[4 * kk + e];
        } else {
          uint32_t w[4];
          widen4<KIND>(k[i].w[2 * kk], w[0], w[1]);
          widen4<KIND>(k[i].w[2 * kk + 1], w[2], w[3]);
#pragma unroll
          for (int e = 0; e < 4; ++e) kop[i][kk][e] = w[e];
        }
      }

    u32x4 p[NR];
    float w[NR][8];
#pragma unroll
    for (int t = 0; t < NR; ++t) {
      f32x4 s[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        s[i] = f32x4{0, 0, 0, 0};
#pragma unroll
        for (int kk = 0; kk < kSums; ++kk) s[i] = mfma<kBf>(kop[i][kk], q[t][kk], s[i]);
      }
      float x[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        if constexpr (KIND == KVH_CACHE_16)
          x[i] = s[i / 4][i % 4] * coef[t];
        else
          x[i] = __builtin_fmaf(s[i / 4][i % 4], ks[i] * coef[t], lsv[i]);
      }
      if (hidden_any) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const bool seen = sight[t].sees(a, t0 + 16 * (i / 4) + grp * 4 + i % 4), none = (absent >> i & 1u) != 0;
          bad |= seen && none;
          if (!seen || none) x[i] = -INFINITY;
        }
      }
      float most = x[0];
#pragma unroll
      for (int i = 1; i < 8; ++i) most = fmaxf(most, x[i]);
      most = over_groups_max(most);
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
        float e = __builtin_amdgcn_exp2f(x[i] - top);
        if constexpr (KIND == KVH_CACHE_16) {
          l[t] += e;
        } else {
          l[t] = __builtin_fmaf(e, inv[i], l[t]);
          e *= rest[i];
        }
        w[t][i] = e;
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) p[t][e] = narrow2<kBf ? KVH_BF16 : KVH_F16>(w[t][2 * e], w[t][2 * e + 1]);
    }

    if (hidden_any) {
      // What no row sees is not multiplied at all; what some rows see and others do not may only meet those that do.
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int tok = t0 + 16 * (i / 4) + grp * 4 + i % 4;
        const bool none = tok >= end || (absent >> i & 1u);
#pragma unroll
        for (int e = 0; e < kVWords; ++e) v[i].w[e] = none ? 0u : v[i].w[e];
      }
      if constexpr (KIND != KVH_CACHE_I8) {
        bool any = false;  // an infinity or NaN among them
#pragma unroll
        for (int i = 0; i < 8; ++i)
#pragma unroll
          for (int e = 0; e < kVWords; ++e) any |= has_odd<DT, KIND>(v[i].w[e]);
        if (__any(any)) {
          weigh<true>(v, p, t0);
          return;
        }
      }
    }
    weigh<false>(v, p, t0);
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
};

template <int DT, int KIND, int D, int NR, bool PAGE16>
__global__ __launch_bounds__(kBlockThreads, 2) void attention_kernel(AttnParams a) {
  using W = Worker<DT, KIND, D, NR, PAGE16>;
  constexpr int kTile = 16 * NR;
  constexpr int kPitch = D + 4;  // floats of a row in LDS
  __shared__ float lds[kWavesPerBlock * 16 * kPitch];
  __shared__ float lds_ml[kWavesPerBlock][kTile][2];
  const int lane = threadIdx.x % kWave, wave = uniform((int32_t)(threadIdx.x / kWave));
  const uint32_t item = a.by_heads.quotient(blockIdx.x);  // the heads of an item run together: they read neighbouring memory
  const int head = (int)(blockIdx.x - item * (uint32_t)a.heads);
  Item it;
  if (!find_item(a, kTile, item, false, lane, it)) return;
  W w(a);
  w.lane = lane, w.l16 = lane % 16, w.grp = lane / 16;
  w.rq = it.rq;
  w.head = head;
  w.row0 = it.tile * kTile;
  const int all = it.rq.n * a.group;
  w.rows = all - w.row0 < kTile ? all - w.row0 : kTile;
  w.p_least = it.rq.len - it.rq.n + (int)a.by_group.quotient((uint32_t)w.row0);
  w.p_most = it.rq.len - it.rq.n + (int)a.by_group.quotient((uint32_t)(w.row0 + w.rows - 1));
  w.end = a.causal && w.p_most + 1 < it.rq.len ? w.p_most + 1 : it.rq.len;
  w.begin();
  const Steps steps(a, w.p_least, w.end);
  int s0, s1;
  steps.part_of(it, s0, s1);
  const int mine = (s1 - s0 + kWavesPerBlock - 1) / kWavesPerBlock;
  const int b0 = s0 + wave * mine, b1 = b0 + mine < s1 ? b0 + mine : s1;
  const int32_t* table = a.req.table + (int64_t)it.b * a.req.table_stride;
  for (int s = b0; s < b1; ++s) w.step(table, steps.token(s));
  if (__any(w.bad) && lane == 0 && a.status != nullptr) a.status[it.b] = KVH_DEV_BAD_REQUEST;

  // The four waves' results become one.
#pragma unroll
  for (int t = 0; t < NR; ++t) {
    const float sum = over_groups_sum(w.l[t]);
    if (w.grp == 0) {
      lds_ml[wave][t * 16 + w.l16][0] = w.m[t];
      lds_ml[wave][t * 16 + w.l16][1] = sum;
    }
  }
  const bool split = it.parts > 1;
  const int64_t slot = blockIdx.x;
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
    // thread: row threadIdx / 16, D / 16 channels
    const int r = threadIdx.x / 16, ch = (threadIdx.x % 16) * W::kChans, row = t * 16 + r;
    if (row < w.rows) {
      float m = -INFINITY;
#pragma unroll
      for (int v = 0; v < kWavesPerBlock; ++v) m = fmaxf(m, lds_ml[v][row][0]);
      float l = 0.0f, x[W::kChans];
#pragma unroll
      for (int e = 0; e < W::kChans; ++e) x[e] = 0.0f;
#pragma unroll
      for (int v = 0; v < kWavesPerBlock; ++v) {
        const float mv = lds_ml[v][row][0], f = mv == m ? 1.0f : __builtin_amdgcn_exp2f(mv - m);
        l = __builtin_fmaf(f, lds_ml[v][row][1], l);
#pragma unroll
        for (int e = 0; e < W::kChans; ++e) x[e] = __builtin_fmaf(f, lds[(v * 16 + r) * kPitch + ch + e], x[e]);
      }
      if (split) {
        float* to = a.part + (slot * kTile + row) * D + ch;
#pragma unroll
        for (int e = 0; e < W::kChans; e += 4) *reinterpret_cast<f32x4*>(to + e) = f32x4{x[e], x[e + 1], x[e + 2], x[e + 3]};
        if (ch == 0) {
          a.part_ml[(slot * kTile + row) * 2] = m;
          a.part_ml[(slot * kTile + row) * 2 + 1] = l;
        }
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

// Joins the partial results of the requests that were cut: a wave takes one query row.
template <int DT, int D>
__global__ __launch_bounds__(kBlockThreads) void join_kernel(AttnParams a, int tile_rows) {
  const int lane = threadIdx.x % kWave;
  const int q_heads = a.heads * a.group;
  const int64_t unit = (int64_t)blockIdx.x * kWavesPerBlock + uniform((int32_t)(threadIdx.x / kWave));
  const int64_t packed = unit / q_heads;
  if (packed >= a.req.n_tokens) return;
  const int u = (int)(unit - packed * q_heads), head = u / a.group;
  Item it;
  if (!find_item(a, tile_rows, packed, true, lane, it) || it.parts == 1) return;
  const int token = (int)(packed - it.rq.start);
  const int64_t at = (int64_t)token * a.group + (u - head * a.group);
  const int tile = (int)(at / tile_rows), row = (int)(at - (int64_t)tile * tile_rows);
  const int64_t slot0 = it.part + (int64_t)(it.tiles - 1 - tile) * it.parts;
  if (slot0 + it.parts > a.items) return;  // requests that share rows of the batch: none of the kernel's
  constexpr int kPer = D / 64;
  float m = -INFINITY, l = 0.0f, x[kPer];
#pragma unroll
  for (int e = 0; e < kPer; ++e) x[e] = 0.0f;
  for (int p = 0; p < it.parts; ++p) {
    const int64_t s = ((slot0 + p) * a.heads + head) * tile_rows + row;
    const float mp = a.part_ml[2 * s], lp = a.part_ml[2 * s + 1];
    const float now = fmaxf(m, mp);
    const float fo = m == now ? 1.0f : __builtin_amdgcn_exp2f(m - now), fp = mp == now ? 1.0f : __builtin_amdgcn_exp2f(mp - now);
    m = now;
    l = __builtin_fmaf(l, fo, fp * lp);
#pragma unroll
    for (int e = 0; e < kPer; ++e) x[e] = __builtin_fmaf(x[e], fo, fp * a.part[s * D + lane * kPer + e]);
  }
  const bool blind = it.rq.len == 0 || (a.causal && it.rq.len - it.rq.n + token < 0);
  const float by = 1.0f / l;
  uint16_t* to = a.out + packed * a.o_ts + (int64_t)u * D + lane * kPer;
  if constexpr (kPer == 2)
    *reinterpret_cast<uint32_t*>(to) = blind ? 0u : narrow2<DT>(x[0] * by, x[1] * by);
  else
    *to = blind ? 0 : (uint16_t)narrow2<DT>(x[0] * by, 0.0f);
  if (a.lse != nullptr && lane == 0) a.lse[packed * q_heads + u] = blind ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * kLn2;
}

// Says which requests are refused; the kernels above pass over them.
__global__ __launch_bounds__(kBlockThreads) void refuse_kernel(AttnParams a) {
  const int b = blockIdx.x * kBlockThreads + threadIdx.x;
  if (b < a.req.n && !read_request(a, b).ok) a.status[b] = KVH_DEV_BAD_REQUEST;
}

// ---- launch -------------------------------------------------------------------------------------------------------
constexpr int kTarget = 512;  // blocks of 4 waves that fill the chip: 2 on each compute unit

struct Plan {
  int nr;          // tiles of 16 rows of the kernel for few rows; 0: the kernel for many
  int rows;        // of an item
  int64_t tiles;   // row tiles of the batch at most
  int64_t items;   // items at most, if requests are cut; the grid otherwise
  int target;      // what the kernel aims at
  size_t bytes;    // workspace of these items
};

size_t slot_bytes(int rows, int head_dim) { return (size_t)rows * (head_dim + 2) * sizeof(float); }

Plan plan_of(int n_requests, int max_new, int n_tokens, int heads, int q_heads, int head_dim) {
  Plan p;
  const int64_t group = q_heads / heads;
  const int64_t most = (int64_t)(max_new < n_tokens ? max_new : n_tokens) * group;
  p.nr = most <= 16 ? 1 : most <= 32 ? 2 : 0;
  p.rows = p.nr != 0 ? 16 * p.nr : kManyRows;
  p.tiles = (int64_t)n_tokens * group / p.rows + n_requests;
  const int64_t aim = (kTarget + heads - 1) / heads;
  p.target = (int)aim;
  p.items = p.target + p.tiles;  // each tile's last chunk may be short
  p.bytes = (size_t)p.items * heads * slot_bytes(p.rows, head_dim);
  return p;
}

template <int DT, int KIND, int D, int NR>
void launch_pages(const AttnParams& a, dim3 grid, hipStream_t stream) {
  if (a.block_tokens % 16 == 0)
    launch_kernel(attention_kernel<DT, KIND, D, NR, true>, grid, dim3(kBlockThreads), 0, stream, a);
  else
    launch_kernel(attention_kernel<DT, KIND, D, NR, false>, grid, dim3(kBlockThreads), 0, stream, a);
}

template <int DT, int KIND, int D>
void launch_rows(const AttnParams& a, int nr, dim3 grid, hipStream_t stream) {
  if (nr == 1)
    launch_pages<DT, KIND, D, 1>(a, grid, stream);
  else
    launch_pages<DT, KIND, D, 2>(a, grid, stream);
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

template <int DT>
void launch_join(const AttnParams& a, int head_dim, int tile_rows, hipStream_t stream) {
  const int64_t units = (int64_t)a.req.n_tokens * a.heads * a.group;
  const dim3 grid((unsigned)((units + kWavesPerBlock - 1) / kWavesPerBlock));
  if (head_dim == 128)
    hipLaunchKernelGGL((join_kernel<DT, 128>), grid, dim3(kBlockThreads), 0, stream, a, tile_rows);
  else
    hipLaunchKernelGGL((join_kernel<DT, 64>), grid, dim3(kBlockThreads), 0, stream, a, tile_rows);
}

bool heads_fit(int heads, int q_heads) { return heads >= 1 && q_heads >= heads && q_heads % heads == 0 && q_heads <= 65536; }

}  // namespace
}  // namespace kvh

using namespace kvh;

extern "C" {

size_t kvh_attention_workspace(int n_requests, int max_new, int n_tokens, int heads, int q_heads, int head_dim) {
  if (n_requests < 1 || n_requests > kMaxRequests || max_new < 1 || n_tokens < 1 || !heads_fit(heads, q_heads)) return 0;
  if (head_dim != 64 && head_dim != 128) return 0;
  return plan_of(n_requests, max_new, n_tokens, heads, q_heads, head_dim).bytes;
}

int kvh_attention(const kvh_cache* cache, int layer, const kvh_requests* requests, kvh_dtype dt, const kvh_rows* q,
                  const kvh_rows* out, int q_heads, float* lse_dev, float scale, int causal, int sink, int window,
                  void* workspace_dev, size_t workspace_bytes, int32_t* status_dev, void* stream) {
  if ((dt != KVH_F16 && dt != KVH_BF16) || q == nullptr || out == nullptr) return KVH_E_ARG;
  if (int rc = check_cache(cache)) return rc;
  if (int rc = check_requests(requests)) return rc;
  if (layer < 0 || layer >= cache->layers || !heads_fit(cache->heads, q_heads)) return KVH_E_SHAPE;
  for (const kvh_rows* r : {q, out})
    if (int rc = check_rows(r, (int64_t)q_heads * cache->head_dim)) return rc;
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
  a.causal = causal != 0, a.sink = sink, a.window = window;
  a.status = status_dev;
  a.by_block = Divisor((uint32_t)cache->block_tokens);
  a.by_group = Divisor((uint32_t)a.group);
  a.by_heads = Divisor((uint32_t)a.heads);
  if ((int64_t)a.req.max_new * a.group >= (int64_t)1 << 31) return KVH_E_SHAPE;
  Plan p = plan_of(a.req.n, a.req.max_new, a.req.n_tokens, a.heads, q_heads, cache->head_dim);
  // Requests are cut where the row tiles alone leave the chip idle and there is room for the parts.
  const size_t one = (size_t)a.heads * slot_bytes(p.rows, cache->head_dim);
  const size_t room = workspace_dev == nullptr ? 0 : workspace_bytes / one;
  bool cut = p.tiles * a.heads < 2 * kTarget;
  if (cut && room < (size_t)p.items) {
    if (room >= (size_t)p.tiles + 1)
      p.target = (int)(room - p.tiles), p.items = (int64_t)room;
    else
      cut = false;
  }
  if (!cut) p.items = p.tiles;
  if (p.items * a.heads > 0x7fffffff) return KVH_E_SHAPE;
  a.target = p.target;
  a.items = p.items;
  a.least = 16;
  if (cut) {
    a.part = static_cast<float*>(workspace_dev);
    a.part_ml = a.part + (size_t)p.items * a.heads * p.rows * cache->head_dim;
  }
  if (status_dev != nullptr) {
    hipLaunchKernelGGL(refuse_kernel, dim3((a.req.n + kBlockThreads - 1) / kBlockThreads), dim3(kBlockThreads), 0, s, a);
    KVH_HIP_CHECK_LAUNCH();
  }
  const dim3 grid((unsigned)(p.items * a.heads));
  if (p.nr == 0)
    launch_attention_many(a, dt, cache->kind, cache->head_dim, grid.x, s);
  else if (dt == KVH_F16)
    launch_kind<KVH_F16>(a, cache->kind, cache->head_dim, p.nr, grid, s);
  else
    launch_kind<KVH_BF16>(a, cache->kind, cache->head_dim, p.nr, grid, s);
  KVH_HIP_CHECK_LAUNCH();
  if (cut) {
    if (dt == KVH_F16)
      launch_join<KVH_F16>(a, cache->head_dim, p.rows, s);
    else
      launch_join<KVH_BF16>(a, cache->head_dim, p.rows, s);
    KVH_HIP_CHECK_LAUNCH();
  }
  return KVH_OK;
}

}  // extern "C"
