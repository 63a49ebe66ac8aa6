// The attention of many query rows (a prompt, or a question after a cached context): tiles of 128 rows of one KV head, which share
// every tile of 64 tokens that is read.
//
// A block has 4 waves of 32 rows and walks over its tokens.  The tile's keys [64][D] and its values, transposed to [D][64], lie in LDS as the 16-bit
// operands of 32x32x16 matrix instructions: codes are widened once for all rows when a tile is stored.  As with few rows, S^T = K Q^T
// and O^T = V^T P^T put a query row on a column, so a lane keeps the statistics of its own row, and the weights leave the first product in
// the lanes in which the second takes them; the values' tokens lie in LDS in the order in which the weights' lanes hold them.
// Two buffers: the next tile's loads are under way while this one is multiplied, and it is stored into the other buffer afterwards, so a
// tile costs one barrier.  16-byte units are placed by an exclusive or with bits of their row, which spreads both the stores and the matrix
// operands' loads over the banks.
//
// Measured, 8 KV heads of 128, 32 query heads: a prompt of 8192, bf16: 662 to 700 us from card to card = 790 to 830 TFLOP/s (a plain product reaches 1200), e4m3:
// 730; 512 new tokens after 32768, int8: 396 us = 700 TFLOP/s, e4m3: 407.
//
// What bounds it, by counters over the prompt: 64 tokens and 32 rows take 2890 cycles of a SIMD, where its matrix instructions are busy for 1024 of them (35 %), other
// vector instructions for some 1080 (37 %; 512 of them exponentials), and LDS for 1070 (37 %, a quarter of it bank conflicts) for the four
// SIMDs' pieces.  No unit is full: with two blocks a compute unit, which is what registers allow, the three take turns more than they overlap.  512 after
// 32768, int8: matrix 29 %, all vector instructions 47 % (codes are widened), LDS 33 %.  Registers: 224 to 256 with 128 channels; e4m3 over pages that are no
// multiple of 16 tokens spills 7 to 9 there.
#include "kvh_attention.hpp"

namespace kvh {
namespace {

typedef float f32x16 __attribute__((ext_vector_type(16)));

constexpr int kManyTokens = 64;  // of a tile
constexpr int kManyWaveRows = 32;
static_assert(kManyRows == kManyWaveRows * kWavesPerBlock, "rows of a block");

template <bool BF>
__device__ __forceinline__ f32x16 mfma32(const u32x4& x, const u32x4& y, const f32x16& c) {
  if constexpr (BF)
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, x), __builtin_bit_cast(bf16x8, y), c, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, x), __builtin_bit_cast(f16x8, y), c, 0, 0, 0);
}

template <int DT, int KIND, int D, bool PAGE16>
struct Tiles {
  static constexpr bool kBf = kBf16<DT, KIND>;
  static constexpr int kWidth = KIND == KVH_CACHE_16 ? 2 : 1;
  static constexpr int kSums = D / 16;                                  // matrix instructions of a dot product
  static constexpr int kOuts = D / 32;                                  // channel tiles of the output
  static constexpr int kKUnits = D * kWidth / 16;                       // 16-byte units of a token's K row in the cache
  static constexpr int kKEach = kManyTokens * kKUnits / kBlockThreads;  // of them, those a thread moves
  static constexpr int kVChans = D / 32;                                // channels of V that a thread moves, of 8 tokens
  static constexpr int kVBytes = kVChans * kWidth;                      // 8, 4 or 2
  static constexpr int kVWords = (kVBytes + 3) / 4;
  static constexpr int kKTile = kManyTokens * D * 2, kVTile = D * kManyTokens * 2;
  static constexpr int kBuffer = kKTile + kVTile;
  static constexpr int kScales = KIND != KVH_CACHE_16 && !PAGE16 ? kManyTokens : 1;

  const AttnParams& a;
  uint8_t* lds;                     // two buffers
  uint32_t (*odd)[kWavesPerBlock];  // of each buffer, by the wave that stored them: an infinity or NaN among its values
  float (*scales)[3][kScales];      // of each buffer, where a tile's tokens lie on pages of any size: K scales, and V scales' logarithms and inverses
  const int32_t* table;
  int head, end, lane, wave;
  PageRun run;
  // PAGE16: bytes from a group of 16 tokens' first row to what the thread moves of it, and where the next group lies: in the
  // request's page `in`, `past` bytes (and `row` rows) from its start.
  uint32_t k_from, v_from;
  uint32_t k_to, v_to;  // and where it goes in a buffer
  int in, row;
  int64_t past;

  // what the thread has under way for the next tile
  u32x4 k[kKEach];
  uint32_t v[8][kVWords];
  uint32_t none;         // of its 8 tokens of V, those past the end or on no page of the cache
  uint64_t absent;       // the tile's tokens on no page of the cache
  bool odd_page;         // a scale of the tile is no finite number; known when the tile has been stored, and the scales are ones to be used then
  bool edge;             // some row of the block does not see all of the tile
  float ks[4], vs[4];    // scales of the tile's groups of 16 tokens (PAGE16), or of its token `lane` in [0]

  __device__ __forceinline__ Tiles(const AttnParams& a_) : a(a_) {}

  static __device__ __forceinline__ int k_place(int token, int unit) { return token * (D * 2) + ((unit ^ token & 7) << 4); }
  // Rows (channels) are 8 units long.  The store puts rows kVChans apart side by side, the operands take neighbouring rows: both differ in
  // all three bits of this.
  static __device__ __forceinline__ int v_place(int ch, int unit) {
    const int x = kVChans == 4 ? (ch >> 2 & 1) | ((ch ^ ch >> 3) & 1) << 1 | ((ch >> 1 ^ ch >> 4) & 1) << 2
                               : (ch >> 1 & 1) | (ch >> 2 & 1) << 1 | ((ch ^ ch >> 3) & 1) << 2;
    return ch * (kManyTokens * 2) + ((unit ^ x) << 4);
  }
  // Token of element e of unit u = 2 g + h: of the 16 tokens of group g, those whose weights lane half h holds.
  static __device__ __forceinline__ int v_token(int u, int e) { return 16 * (u / 2) + 4 * (u % 2) + 8 * (e / 4) + e % 4; }
  // The thread's unit of V and its first channel; a wave's units are those of one group of 16 tokens.
  __device__ __forceinline__ int v_unit() const { return threadIdx.x / 32; }
  __device__ __forceinline__ int v_chan() const { return threadIdx.x % 32 * kVChans; }

  __device__ __forceinline__ void begin() {
    const uint32_t row_bytes = (uint32_t)a.c_ts * kWidth;
    k_from = threadIdx.x / kKUnits % 16 * row_bytes + threadIdx.x % kKUnits * 16;
    v_from = v_unit() % 2 * 4 * row_bytes + v_chan() * kWidth;
    k_to = (uint32_t)k_place(threadIdx.x / kKUnits, threadIdx.x % kKUnits * (KIND == KVH_CACHE_16 ? 1 : 2));
    v_to = kKTile + (uint32_t)v_place(v_chan(), v_unit());
  }

  static __device__ __forceinline__ void fetch_v(uint32_t (&to)[kVWords], const uint8_t* p) {
    if constexpr (kVBytes == 2) {
      to[0] = *reinterpret_cast<const uint16_t*>(p);
    } else {
      const Words<kVWords> w = fetch<kVWords>(p);
#pragma unroll
      for (int c = 0; c < kVWords; ++c) to[c] = w.w[c];
    }
  }

  // The next tile is that of tokens t0 and on.
  __device__ __forceinline__ void seek(int t0) {
    in = (int)a.by_block.quotient((uint32_t)t0);
    row = t0 - in * a.block_tokens;
    past = (int64_t)row * (a.c_ts * kWidth);
  }

  // Starts the loads of tokens [t0, t0 + 64), t0 < end, where seek or the tile before left off.  Nothing here waits for them.
  __device__ __forceinline__ void fetch_tile(int t0, int p_first) {
    const int last = end - 1, tid = threadIdx.x;
    const int64_t row_bytes = a.c_ts * kWidth, head_at = (int64_t)head * D * kWidth;
    const int u = v_unit();
    none = 0;
    if constexpr (PAGE16) {
      // Each group of 16 tokens lies on one page: its rows past the end are the page's too, and only have to be kept from the sums.
      absent = 0;
      if ((unsigned)(in - run.base) > (unsigned)(kWave - 4)) run.load(a, table, in, (int)a.by_block.quotient((uint32_t)last), lane);
      int64_t at[4];  // bytes to the group's first row
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        if (g > 0 && t0 + 16 * g > last) {  // a group past the end stands for the one before
          at[g] = at[g - 1];
          ks[g] = ks[g - 1], vs[g] = vs[g - 1];
          continue;
        }
        int page = uniform(__builtin_amdgcn_readlane(run.entry, in - run.base));
        if (page < 0) {
          page = 0;
          absent |= (uint64_t)0xffff << 16 * g;
        }
        at[g] = (int64_t)page * a.block_tokens * row_bytes + past + head_at;
        if constexpr (KIND != KVH_CACHE_16) {
          ks[g] = a.sk[(int64_t)page * a.s_ps + head];
          vs[g] = a.sv[(int64_t)page * a.s_ps + head];
        }
        row += 16, past += 16 * row_bytes;
        if (row == a.block_tokens) row = 0, past = 0, ++in;
      }
#pragma unroll
      for (int i = 0; i < kKEach; ++i) {
        constexpr int kWaveTokens = kWave / kKUnits, kStride = kBlockThreads / kKUnits;  // of an access
        const int g = (wave * kWaveTokens + i * kStride) / 16;
        const int64_t from = g == 0 ? at[0] : g == 1 ? at[1] : g == 2 ? at[2] : at[3];
        k[i] = *reinterpret_cast<const u32x4*>(a.ck + from + k_from);
      }
      const uint8_t* vg = a.cv + (wave == 0 ? at[0] : wave == 1 ? at[1] : wave == 2 ? at[2] : at[3]);
#pragma unroll
      for (int e = 0; e < 8; ++e) fetch_v(v[e], vg + (8 * (e / 4) + e % 4) * row_bytes + v_from);
    } else {
      const int tz = t0 + kManyTokens - 1 < last ? t0 + kManyTokens - 1 : last;
      const int at0 = (int)a.by_block.quotient((uint32_t)t0), at1 = (int)a.by_block.quotient((uint32_t)tz);
      if (at0 < run.base || at1 - run.base >= kWave) run.load(a, table, at0, (int)a.by_block.quotient((uint32_t)last), lane);
      // the bytes to the rows of tokens t0 + lane, in the lanes; a token past the end stands for the last one, one on no page for row 0
      const int mine = t0 + lane < last ? t0 + lane : last, in = (int)a.by_block.quotient((uint32_t)mine);
      const int page = __shfl(run.entry, in - run.base);
      absent = __ballot(page < 0);
      const int64_t at = page < 0 ? head_at : ((int64_t)page * a.block_tokens + (mine - in * a.block_tokens)) * row_bytes + head_at;
      // One lane number for all of a thread's rows: the others are it and a number that the exchange itself adds.
      auto row_of = [&](int lane4, int more) {
        const uint32_t lo = __builtin_amdgcn_ds_bpermute(lane4 + 4 * more, (int)at), hi = __builtin_amdgcn_ds_bpermute(lane4 + 4 * more, (int)(at >> 32));
        return (int64_t)((uint64_t)hi << 32 | lo);
      };
      const int k_lane = tid / kKUnits * 4, v_lane = v_token(u, 0) * 4;
#pragma unroll
      for (int i = 0; i < kKEach; ++i)
        k[i] = *reinterpret_cast<const u32x4*>(a.ck + row_of(k_lane, kBlockThreads / kKUnits * i) + tid % kKUnits * 16);
#pragma unroll
      for (int e = 0; e < 8; ++e) fetch_v(v[e], a.cv + row_of(v_lane, v_token(0, e)) + v_chan() * kWidth);
      if constexpr (KIND != KVH_CACHE_16) {
        const int64_t p = page < 0 ? 0 : page;
        ks[0] = a.sk[p * a.s_ps + head];
        vs[0] = a.sv[p * a.s_ps + head];
      }
    }
    edge = t0 + kManyTokens > end || absent != 0 || (a.causal && t0 + kManyTokens - 1 > p_first) || a.window != 0;
    if (edge) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int t = v_token(u, 0), more = v_token(0, e);  // what differs from thread to thread, and what does not
        if (t0 + t + more >= end || (absent >> t >> more & 1) != 0) none |= 1u << e;
      }
    }
  }

  static __device__ __forceinline__ uint32_t without_odd(uint32_t w) {
    if constexpr (KIND == KVH_CACHE_16) {
      return Odd<kBf>::without(w);
    } else {  // a code of NaN becomes one of zero
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if ((w >> 8 * e & 0x7fu) == 0x7fu) w &= ~(0xffu << 8 * e);
      return w;
    }
  }

  // The operand of the second product for channel 32 c + l of lane half h and group g of the tile at t0, again from the cache: ones where a
  // value is the `which`th odd one.
  __device__ __forceinline__ u32x4 odd_ones(int t0, int c, int g, int which) const {
    u32x4 w;
    int lane = this->lane;
    asm volatile("" : "+v"(lane));  // nothing of this is worked out ahead of the loop: there are no registers for it
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      w[e] = 0;
#pragma unroll
      for (int n = 0; n < 2; ++n) {
        const int tok = t0 + v_token(2 * g + lane / 32, 2 * e + n);
        if (tok >= end) continue;
        const int p = (int)a.by_block.quotient((uint32_t)tok), page = table[p];
        if (page < 0 || page >= a.pages) continue;
        const int64_t row = (int64_t)page * a.block_tokens + (tok - p * a.block_tokens);
        const uint8_t* src = a.cv + (row * a.c_ts + (int64_t)head * D + 32 * c + lane % 32) * kWidth;
        bool is;
        if constexpr (KIND == KVH_CACHE_16)
          is = Odd<kBf>::is(*reinterpret_cast<const uint16_t*>(src), which);
        else
          is = which == 0 && (*src & 0x7fu) == 0x7fu;
        if (is) w[e] |= Odd<kBf>::kOne << 16 * n;
      }
    }
    return w;
  }

  // The tokens of the tile at t0 whose scales are no finite numbers, again from the cache.
  __device__ __forceinline__ void odd_tokens(int t0, uint64_t& k, uint64_t& v) const {
    int lane = this->lane;
    asm volatile("" : "+v"(lane));  // as in odd_ones
    bool odd_k = false, odd_v = false;
    if (t0 + lane < end) {
      const int page = table[a.by_block.quotient((uint32_t)(t0 + lane))];
      if (page >= 0 && page < a.pages) {
        odd_k = odd_scale(a.sk[(int64_t)page * a.s_ps + head]);
        odd_v = odd_scale(a.sv[(int64_t)page * a.s_ps + head]);
      }
    }
    k = __ballot(odd_k), v = __ballot(odd_v);
  }

  // Stores what was fetched into a buffer, as operands.
  __device__ __forceinline__ void store_tile(int buffer) {
    const uint32_t kb = k_to + buffer * kBuffer, vb = v_to + buffer * kBuffer;
    const int tid = threadIdx.x;
#pragma unroll
    for (int i = 0; i < kKEach; ++i) {  // the thread's tokens are a multiple of 8 apart
      constexpr int kApart = kBlockThreads / kKUnits * (D * 2);
      static_assert(kBlockThreads / kKUnits % 8 == 0, "units keep their places");
      if constexpr (KIND == KVH_CACHE_16) {
        *reinterpret_cast<u32x4*>(lds + kb + i * kApart) = k[i];
      } else {
#pragma unroll
        for (int p = 0; p < 2; ++p) {
          uint32_t w[4];
          widen4<KIND>(k[i][2 * p], w[0], w[1]);
          widen4<KIND>(k[i][2 * p + 1], w[2], w[3]);
          *reinterpret_cast<u32x4*>(lds + (kb ^ p * 16) + i * kApart) = u32x4{w[0], w[1], w[2], w[3]};
        }
      }
    }
    if (__any(none != 0)) {  // what no row may meet
#pragma unroll
      for (int e = 0; e < 8; ++e)
#pragma unroll
        for (int c = 0; c < kVWords; ++c) v[e][c] = none >> e & 1 ? 0u : v[e][c];
    }
    const int u = v_unit();
    if constexpr (KIND != KVH_CACHE_I8) {
      // Where some row does not see all of the tile, its infinities and NaN stay out of the product: see Odd.
      bool any = false;
      if (edge) {
#pragma unroll
        for (int e = 0; e < 8; ++e)
#pragma unroll
          for (int c = 0; c < kVWords; ++c) any |= has_odd<DT, KIND>(v[e][c]);
        any = __any(any);
      }
      if (lane == 0) odd[buffer][wave] = any;
      if (any) {
#pragma unroll
        for (int e = 0; e < 8; ++e)
#pragma unroll
          for (int c = 0; c < kVWords; ++c) v[e][c] = without_odd(v[e][c]);
      }
    }
    uint32_t z[4][kVChans];  // pairs of tokens, of each channel
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const uint32_t(&x)[kVWords] = v[2 * e], (&y)[kVWords] = v[2 * e + 1];
      if constexpr (KIND == KVH_CACHE_16) {
#pragma unroll
        for (int c = 0; c < kVWords; ++c) {
          z[e][2 * c] = __builtin_amdgcn_perm(y[c], x[c], 0x05040100u);
          z[e][2 * c + 1] = __builtin_amdgcn_perm(y[c], x[c], 0x07060302u);
        }
      } else if constexpr (kVChans == 4) {
        zip4<KIND>(x[0], y[0], z[e]);
      } else {
        widen4<KIND>(__builtin_amdgcn_perm(y[0], x[0], 0x05010400u), z[e][0], z[e][1]);
      }
    }
    if constexpr (KIND != KVH_CACHE_16) {
      ScaleRange range;
#pragma unroll
      for (int g = 0; g < (PAGE16 ? 4 : 1); ++g) range.add(ks[g], vs[g]);
      odd_page = false;
      if (__builtin_expect(__any(range.rare()), 0)) {
        // Below the least that the exponent takes the rest goes onto the values.
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          float r[2];
#pragma unroll
          for (int n = 0; n < 2; ++n) {
            const float s = PAGE16 ? (wave == 0 ? vs[0] : wave == 1 ? vs[1] : wave == 2 ? vs[2] : vs[3])
                                   : __int_as_float(__builtin_amdgcn_ds_bpermute(v_token(u, 0) * 4 + 4 * v_token(0, 2 * e + n), __float_as_int(vs[0])));
            r[n] = odd_scale(s) ? 1.0f : ValueScale(s).rest;
          }
          const f16x2 by = __builtin_bit_cast(f16x2, narrow2<KVH_F16>(r[0], r[1]));
#pragma unroll
          for (int j = 0; j < kVChans; ++j) z[e][j] = __builtin_bit_cast(uint32_t, __builtin_bit_cast(f16x2, z[e][j]) * by);
        }
#pragma unroll
        for (int g = 0; g < (PAGE16 ? 4 : 1); ++g) {
          odd_page |= __any(odd_scale(ks[g]) || odd_scale(vs[g]));
          ks[g] = odd_scale(ks[g]) ? 1.0f : ks[g];
          vs[g] = ValueScale(vs[g]).used;
        }
      }
    }
#pragma unroll
    for (int j = 0; j < kVChans; ++j) {  // channel ch + j: j rows on, with j's bits in the unit's place (see v_place)
      constexpr int kOne = kVChans == 4 ? 32 : 64, kTwo = 64;
      *reinterpret_cast<u32x4*>(lds + (vb ^ (j % 2 * kOne | j / 2 * kTwo)) + j * (kManyTokens * 2)) = u32x4{z[0][j], z[1][j], z[2][j], z[3][j]};
    }
    if constexpr (KIND != KVH_CACHE_16 && !PAGE16) {
      if (tid < kManyTokens) {
        scales[buffer][0][tid] = ks[0];
        scales[buffer][1][tid] = __builtin_amdgcn_logf(vs[0]);
        scales[buffer][2][tid] = __builtin_amdgcn_rcpf(vs[0]);
      }
    }
  }
};

template <int DT, int KIND, int D, bool PAGE16>
struct Shared {
  using T = Tiles<DT, KIND, D, PAGE16>;
  __attribute__((aligned(16))) uint8_t buffers[2 * T::kBuffer];
  __attribute__((aligned(16))) float scales[2][3][T::kScales];
  uint32_t odd[2][kWavesPerBlock];
};

template <int DT, int KIND, int D, bool PAGE16>
__device__ __forceinline__ void attend(const AttnParams& a, const Item& it, int head, int wave, int lane, Shared<DT, KIND, D, PAGE16>& shared) {
  using T = Tiles<DT, KIND, D, PAGE16>;
  constexpr bool kScaled = KIND != KVH_CACHE_16;
  uint8_t* lds = shared.buffers;
  auto& odd = shared.odd;
  auto& scales = shared.scales;
  const int col = lane % 32, half = lane / 32;
  const Request rq = it.rq;
  const int all = rq.n * a.group;
  const int row0 = it.tile * kManyRows;
  const int block_rows = all - row0 < kManyRows ? all - row0 : kManyRows;
  const int before = rq.len - rq.n;
  const int p_first = before + (int)a.by_group.quotient((uint32_t)row0);
  const int p_last = before + (int)a.by_group.quotient((uint32_t)(row0 + block_rows - 1));
  const int end = a.causal && p_last + 1 < rq.len ? p_last + 1 : rq.len;
  const Steps steps(a, p_first, end);
  int s0, s1;
  steps.part_of(it, s0, s1);

  // The lane's row, and the positions of the wave's rows.
  const int wave_row = row0 + wave * kManyWaveRows;
  const int wave_rows = all - wave_row < kManyWaveRows ? all - wave_row : kManyWaveRows;  // < 1: the wave only moves tiles
  const bool works = wave_rows > 0, real = col < wave_rows;
  const int at = real ? wave_row + col : row0, token = (int)a.by_group.quotient((uint32_t)at), u = at - token * a.group;
  const int pos = before + token;
  const Sight sight(a, end, pos);
  const int p_least = works ? before + (int)a.by_group.quotient((uint32_t)wave_row) : 0;
  const int p_most = works ? before + (int)a.by_group.quotient((uint32_t)(wave_row + wave_rows - 1)) : 0;

  u32x4 q[T::kSums];
  float coef = fmaxf(fabsf(a.scale) * kLog2e, 0x1p-126f);  // positive, also where the scale is 0: see f below
  {
    const uint32_t sign = a.scale < 0.0f ? 0x80008000u : 0u;
    const uint16_t* src = a.q + ((int64_t)rq.start + token) * a.q_ts + ((int64_t)head * a.group + u) * D;
#pragma unroll
    for (int kk = 0; kk < T::kSums; ++kk) {
      q[kk] = u32x4{0, 0, 0, 0};
      if (real) q[kk] = *reinterpret_cast<const u32x4*>(src + kk * 16 + half * 8) ^ sign;
    }
    if constexpr (kScaled && DT == KVH_BF16) {
      float most = 0.0f;
#pragma unroll
      for (int kk = 0; kk < T::kSums; ++kk) {
        float x[8];
        widen8<DT>(q[kk], x);
#pragma unroll
        for (int e = 0; e < 8; ++e) most = fmaxf(most, fabsf(x[e]));
      }
      most = over_halves_max(most);
      const f32x2 power = row_power(most);
      coef *= power[1];
#pragma unroll
      for (int kk = 0; kk < T::kSums; ++kk) {
        float x[8];
        widen8<DT>(q[kk], x);
#pragma unroll
        for (int e = 0; e < 4; ++e) q[kk][e] = narrow2<KVH_F16>(x[2 * e] * power[0], x[2 * e + 1] * power[0]);
      }
    }
  }

  f32x16 o[T::kOuts];
#pragma unroll
  for (int c = 0; c < T::kOuts; ++c)
#pragma unroll
    for (int j = 0; j < 16; ++j) o[c][j] = 0.0f;
  float m = -INFINITY, l = 0.0f;
  // The lane's row sees: a token on no page of the cache; one whose V scale is no finite number; one whose K scale is none.
  bool bad = false, spoiled = false, lost = false;

  T t(a);
  t.lds = lds, t.odd = odd, t.scales = scales, t.lane = lane, t.head = head, t.end = end;
  t.table = a.req.table + (int64_t)it.b * a.req.table_stride;
  t.wave = wave;
  t.begin();
  if (s0 < s1) {
    t.seek(steps.token(s0));
    t.fetch_tile(steps.token(s0), p_first);
  }
  // Where the lane's operands lie in a buffer: unit 2 e + half of its row, whose place differs from unit half's by an exclusive or with 32 e.
  const uint32_t k_at = (uint32_t)T::k_place(col, half), v_at = T::kKTile + (uint32_t)T::v_place(col, half);
  int buffer = 0;
  for (int s = s0; s < s1; s += 2, buffer ^= 1) {
    const int t0 = steps.token(s);
    t.store_tile(buffer);
    const uint64_t absent = t.absent;
    const bool odd_page = kScaled && t.odd_page;
    // An element's exponent of 2 is f x + z, by groups of 16 tokens (one group where there are no scales).
    constexpr int kGroups = kScaled && PAGE16 ? 4 : 1;
    float f[kGroups], z[kGroups], inv[kGroups];
#pragma unroll
    for (int g = 0; g < kGroups; ++g) {
      f[g] = coef, z[g] = 0.0f, inv[g] = 1.0f;
      if constexpr (kScaled && PAGE16) {
        f[g] = fmaxf(t.ks[g] * coef, 0x1p-126f);  // never 0 or NaN: a hidden score is minus infinity, and has to stay it
        z[g] = __builtin_amdgcn_logf(t.vs[g]), inv[g] = __builtin_amdgcn_rcpf(t.vs[g]);
      } else if constexpr (kScaled) {
        f[g] = 1.0f;  // its tokens' own scales are applied to the scores at once
      }
    }
    __syncthreads();
    if (s + 2 < s1) {
      const int next = steps.token(s + 2);
      if (PAGE16 && next != t0 + kManyTokens) t.seek(next);
      t.fetch_tile(next, p_first);
    }
    const bool hidden = t0 + kManyTokens > end || (a.causal && t0 + kManyTokens - 1 > p_least) || (a.window != 0 && t0 <= p_most - a.window) || absent != 0;
    const bool blank = !works || (a.causal && t0 > p_most);  // no row of the wave sees any of it
    if (blank) continue;
    if constexpr (kScaled) {
      if (__builtin_expect(odd_page, 0)) {
        const uint64_t seen = sight.seen(a, t0);
        uint64_t k, v;
        t.odd_tokens(t0, k, v);
        spoiled |= (seen & v) != 0;
        lost |= (seen & k) != 0;
      }
    }
    const uint32_t kb = k_at + buffer * T::kBuffer, vb = v_at + buffer * T::kBuffer;
    f32x16 x[2];  // element j of x[i] is token 32 i + 8 (j / 4) + 4 half + j % 4 of the tile, of its group 2 i + j / 8
    {
      u32x4 kf[2 * T::kSums];
#pragma unroll
      for (int kk = 0; kk < 2 * T::kSums; ++kk)
        kf[kk] = *reinterpret_cast<const u32x4*>(lds + (kb ^ kk % 4 * 32) + kk / T::kSums * (32 * D * 2) + kk % T::kSums / 4 * 128);
#pragma unroll
      for (int i = 0; i < 2; ++i) {
#pragma unroll
        for (int j = 0; j < 16; ++j) x[i][j] = 0.0f;
#pragma unroll
        for (int kk = 0; kk < T::kSums; ++kk) x[i] = mfma32<T::kBf>(kf[i * T::kSums + kk], q[kk], x[i]);
      }
      // Operands are read ahead of the instructions that take them: four first, then one with each product.
      __builtin_amdgcn_sched_group_barrier(0x100, 4, 0);
#pragma unroll
      for (int kk = 4; kk < 2 * T::kSums; ++kk) {
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
        __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
      }
      __builtin_amdgcn_sched_group_barrier(0x008, 4, 0);
    }
    if constexpr (kScaled && !PAGE16) {
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j4 = 0; j4 < 4; ++j4) {
          const f32x4 kz = *reinterpret_cast<const f32x4*>(&scales[buffer][0][32 * i + 8 * j4 + 4 * half]);
          const f32x4 lz = *reinterpret_cast<const f32x4*>(&scales[buffer][1][32 * i + 8 * j4 + 4 * half]);
#pragma unroll
          for (int e = 0; e < 4; ++e) x[i][4 * j4 + e] = __builtin_fmaf(x[i][4 * j4 + e], kz[e] * coef, lz[e]);
        }
    }
    if (hidden) {
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 16; ++j) {
          const int in = 32 * i + 8 * (j / 4) + j % 4;  // and 4 half more
          const bool seen = sight.sees(a, t0 + 4 * half + in), none = (absent >> 4 * half >> in & 1) != 0;
          bad |= seen && none;
          x[i][j] = !seen || none ? -INFINITY : x[i][j];
        }
    }
    float most = -INFINITY;
#pragma unroll
    for (int g = 0; g < kGroups; ++g) {  // f is positive: the largest score of a group has its largest exponent
      constexpr int kPer = 32 / kGroups;
      float top = x[g * kPer / 16][g * kPer % 16];
#pragma unroll
      for (int j = 1; j < kPer; ++j) top = fmaxf(top, x[(g * kPer + j) / 16][(g * kPer + j) % 16]);
      most = fmaxf(most, __builtin_fmaf(top, f[g], z[g]));
    }
    most = over_halves_max(most);
    // The maximum may lag behind by 2^8: weights up to 256 are as good, and the outputs are hardly ever rescaled.
    if (__any(most > m + 8.0f)) {
      const float now = fmaxf(m, most);
      const float down = now == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(m - now);
      m = now;
      l *= down;
#pragma unroll
      for (int c = 0; c < T::kOuts; ++c)
#pragma unroll
        for (int j = 0; j < 16; ++j) o[c][j] *= down;
    }
    const float top = m == -INFINITY ? 0.0f : m;
#pragma unroll
    for (int g = 0; g < kGroups; ++g) z[g] -= top;
    u32x4 p[4];  // of each 16 tokens: the lane's 8 weights
    auto weights = [&](int i) {
#pragma unroll
      for (int j4 = 0; j4 < 4; ++j4) {
        f32x4 by = {1, 1, 1, 1};
        if constexpr (kScaled && !PAGE16) by = *reinterpret_cast<const f32x4*>(&scales[buffer][2][32 * i + 8 * j4 + 4 * half]);
        const int g = kGroups == 4 ? 2 * i + j4 / 2 : 0;
        float w[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          w[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(x[i][4 * j4 + e], f[g], z[g]));
          if constexpr (!kScaled)
            l += w[e];
          else
            l = __builtin_fmaf(w[e], PAGE16 ? inv[g] : by[e], l);
        }
        p[2 * i + j4 / 2][2 * (j4 % 2)] = narrow2<T::kBf ? KVH_BF16 : KVH_F16>(w[0], w[1]);
        p[2 * i + j4 / 2][2 * (j4 % 2) + 1] = narrow2<T::kBf ? KVH_BF16 : KVH_F16>(w[2], w[3]);
      }
    };
    auto operand = [&](int c, int g) { return *reinterpret_cast<const u32x4*>(lds + (vb ^ g * 32) + c * (32 * kManyTokens * 2)); };
    weights(0);
    __builtin_amdgcn_sched_barrier(0);
    {
      u32x4 vf[2 * T::kOuts];
#pragma unroll
      for (int e = 0; e < 2 * T::kOuts; ++e) vf[e] = operand(e / 2, e % 2);
      weights(1);
#pragma unroll
      for (int e = 0; e < 2 * T::kOuts; ++e) o[e / 2] = mfma32<T::kBf>(vf[e], p[e % 2], o[e / 2]);
      // the first half's products run under the second half's exponentials
      __builtin_amdgcn_sched_group_barrier(0x100, 4, 1);
#pragma unroll
      for (int e = 0; e < 2 * T::kOuts; ++e) {
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 1);
        if (e + 4 < 2 * T::kOuts) __builtin_amdgcn_sched_group_barrier(0x100, 1, 1);
        __builtin_amdgcn_sched_group_barrier(0x402, 56 / (2 * T::kOuts), 1);
      }
    }
    __builtin_amdgcn_sched_barrier(0);
    {
      u32x4 vf[2 * T::kOuts];
#pragma unroll
      for (int e = 0; e < 2 * T::kOuts; ++e) vf[e] = operand(e / 2, 2 + e % 2);
#pragma unroll
      for (int e = 0; e < 2 * T::kOuts; ++e) o[e / 2] = mfma32<T::kBf>(vf[e], p[2 + e % 2], o[e / 2]);
      __builtin_amdgcn_sched_group_barrier(0x100, 4, 2);
#pragma unroll
      for (int e = 0; e < 2 * T::kOuts; ++e) {
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 2);
        if (e + 4 < 2 * T::kOuts) __builtin_amdgcn_sched_group_barrier(0x100, 1, 2);
      }
    }
    if constexpr (KIND != KVH_CACHE_I8) {
      if ((odd[buffer][0] | odd[buffer][1] | odd[buffer][2] | odd[buffer][3]) != 0) {
        using Bad = Odd<T::kBf>;
        int half = lane / 32;
        asm volatile("" : "+v"(half));  // as in odd_ones
#pragma unroll 1
        for (int g = 0; g < 4; ++g) {
          u32x4 one;  // of the group's tokens that the lane's row sees
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            one[e] = 0;
#pragma unroll
            for (int n = 0; n < 2; ++n)
              if (sight.sees(a, t0 + T::v_token(2 * g + half, 2 * e + n))) one[e] |= Bad::kOne << 16 * n;
          }
#pragma unroll
          for (int c = 0; c < T::kOuts; ++c) {
#pragma unroll 1
            for (int which = 0; which < 3; ++which) {
              f32x16 hit;
#pragma unroll
              for (int j = 0; j < 16; ++j) hit[j] = 0.0f;
              hit = mfma32<T::kBf>(t.odd_ones(t0, c, g, which), one, hit);
#pragma unroll
              for (int j = 0; j < 16; ++j) o[c][j] += hit[j] > 0.0f ? Bad::value(which) : 0.0f;
            }
          }
        }
      }
    }
  }
  if (__any(bad) && lane == 0 && a.status != nullptr) a.status[it.b] = KVH_DEV_BAD_REQUEST;

  const float sum = kScaled && lost ? NAN : over_halves_sum(l);
  if (kScaled && __any(spoiled)) {
#pragma unroll
    for (int c = 0; c < T::kOuts; ++c)
#pragma unroll
      for (int j = 0; j < 16; ++j) o[c][j] = spoiled ? NAN : o[c][j];
  }
  if (it.split) {
    if (real) {
      const int64_t row = (it.slot * a.heads + head) * kManyRows + wave * kManyWaveRows + col;
      float* to = a.part + row * D + 4 * half;
#pragma unroll
      for (int c = 0; c < T::kOuts; ++c)
#pragma unroll
        for (int j4 = 0; j4 < 4; ++j4)
          *reinterpret_cast<f32x4*>(to + 32 * c + 8 * j4) = f32x4{o[c][4 * j4], o[c][4 * j4 + 1], o[c][4 * j4 + 2], o[c][4 * j4 + 3]};
      if (half == 0) {
        a.part_ml[2 * row] = m;
        a.part_ml[2 * row + 1] = sum;
      }
    }
    return;
  }
  __syncthreads();  // the buffers become the outputs' way to whole rows: 2 D bytes of a row, a wave's 32 rows apart from the others'
  const bool blind = rq.len == 0 || (a.causal && pos < 0);
  const float by = 1.0f / sum;
  uint8_t* mine = lds + wave * (kManyWaveRows * D * 2);
  auto place = [&](int row, int unit) { return row * (D * 2) + ((unit ^ row & 7) << 4); };
#pragma unroll
  for (int c = 0; c < T::kOuts; ++c)
#pragma unroll
    for (int j4 = 0; j4 < 4; ++j4) {
      u32x2 w = {narrow2<DT>(o[c][4 * j4] * by, o[c][4 * j4 + 1] * by), narrow2<DT>(o[c][4 * j4 + 2] * by, o[c][4 * j4 + 3] * by)};
      if (blind) w = u32x2{0, 0};
      *reinterpret_cast<u32x2*>(mine + place(col, 4 * c + j4) + 8 * half) = w;
    }
  __builtin_amdgcn_wave_barrier();
  constexpr int kUnits = D / 8;  // 16-byte units of a row
#pragma unroll
  for (int i = 0; i < kManyWaveRows * kUnits / kWave; ++i) {
    const int idx = i * kWave + lane, row = idx / kUnits, unit = idx % kUnits;
    if (row < wave_rows) {
      const int ar = wave_row + row, tr = (int)a.by_group.quotient((uint32_t)ar), ur = ar - tr * a.group;
      *reinterpret_cast<u32x4*>(a.out + ((int64_t)rq.start + tr) * a.o_ts + ((int64_t)head * a.group + ur) * D + unit * 8) =
          *reinterpret_cast<const u32x4*>(mine + place(row, unit));
    }
  }
  if (a.lse != nullptr && real && half == 0)
    a.lse[((int64_t)rq.start + token) * ((int64_t)a.heads * a.group) + (int64_t)head * a.group + u] = blind ? -INFINITY : (m + __builtin_amdgcn_logf(sum)) * kLn2;
}

template <int DT, int KIND, int D, bool PAGE16, bool CUT>
__global__ __launch_bounds__(kBlockThreads, 2) void attention_many_kernel(AttnParams a) {
  __shared__ Shared<DT, KIND, D, PAGE16> shared;
  int lane = threadIdx.x % kWave;
  const int wave = uniform((int32_t)(threadIdx.x / kWave));
  const uint32_t k = a.by_heads.quotient(blockIdx.x);
  const int head = (int)(blockIdx.x - k * (uint32_t)a.heads);
  tell_refused(a);
  Item it;
  if constexpr (!CUT) {
    if (Schedule(a, kLogManyRows, lane).whole(k, it)) attend<DT, KIND, D, PAGE16>(a, it, head, wave, lane, shared);
  } else {
    for (Items items; items.next(a, kLogManyRows, k, head == 0 && wave == 0, lane, it);) {
      if (it.split && it.slot >= a.slots) continue;  // requests that share rows of the batch
      attend<DT, KIND, D, PAGE16>(a, it, head, wave, lane, shared);
      __syncthreads();
    }
  }
}

template <int DT, int KIND, int D, bool PAGE16>
void launch_cut(const AttnParams& a, unsigned blocks, hipStream_t stream) {
  if (a.part != nullptr)
    launch_kernel(attention_many_kernel<DT, KIND, D, PAGE16, true>, dim3(blocks), dim3(kBlockThreads), 0, stream, a);
  else
    launch_kernel(attention_many_kernel<DT, KIND, D, PAGE16, false>, dim3(blocks), dim3(kBlockThreads), 0, stream, a);
}

template <int DT, int KIND, int D>
void launch_pages(const AttnParams& a, unsigned blocks, hipStream_t stream) {
  if (a.block_tokens % 16 == 0)
    launch_cut<DT, KIND, D, true>(a, blocks, stream);
  else
    launch_cut<DT, KIND, D, false>(a, blocks, stream);
}

template <int DT, int KIND>
void launch_dim(const AttnParams& a, int head_dim, unsigned blocks, hipStream_t stream) {
  if (head_dim == 128)
    launch_pages<DT, KIND, 128>(a, blocks, stream);
  else
    launch_pages<DT, KIND, 64>(a, blocks, stream);
}

template <int DT>
void launch_kind(const AttnParams& a, int kind, int head_dim, unsigned blocks, hipStream_t stream) {
  switch (kind) {
    case KVH_CACHE_16: return launch_dim<DT, KVH_CACHE_16>(a, head_dim, blocks, stream);
    case KVH_CACHE_I8: return launch_dim<DT, KVH_CACHE_I8>(a, head_dim, blocks, stream);
    default: return launch_dim<DT, KVH_CACHE_E4M3>(a, head_dim, blocks, stream);
  }
}

}  // namespace

void launch_attention_many(const AttnParams& a, int dt, int kind, int head_dim, unsigned blocks, hipStream_t stream) {
  if (dt == KVH_F16)
    launch_kind<KVH_F16>(a, kind, head_dim, blocks, stream);
  else
    launch_kind<KVH_BF16>(a, kind, head_dim, blocks, stream);
}

}  // namespace kvh
