// The attention of many query rows (a prompt, or a question after a cached context): tiles of 128 rows of one KV head, which share
// every tile of 64 tokens that is read.
//
// A block has 4 waves of 32 rows and walks over its tokens.  The tile's keys [64][D] and its values, transposed to [D][64], lie in LDS as the 16-bit
// operands of 32x32x16 matrix instructions: codes are widened once for all rows when a tile is stored.  As with few rows, S^T = K Q^T
// and O^T = V^T P^T put a query row on a column, so a lane keeps the statistics of its own row, and the weights leave the first product in
// the lanes in which the second takes them; the values' tokens lie in LDS in the order in which the weights' lanes hold them.
// Two buffers: the next tile's loads are under way while this one is multiplied, and it is stored into the other buffer afterwards, so a
// tile costs one barrier.  16-byte units are placed by an exclusive or with bits of their row, which keeps both the stores and the matrix
// operands' loads free of bank conflicts.
//
// Bounds: per 64 tokens and 32 rows the matrix instructions take 1024 cycles of a SIMD, the softmax about 900 (512 of them exponentials), the
// operands 32 KiB of LDS reads of a wave (4 waves: what LDS delivers in 1024 cycles).  Two blocks a compute unit let one's softmax run
// under the other's products.
#include "kvh_attention.hpp"

namespace kvh {
namespace {

typedef float f32x16 __attribute__((ext_vector_type(16)));

constexpr int kManyTokens = 64;             // of a tile
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
  float (*scales)[3][kScales];      // of each buffer, where a tile's tokens lie on pages of any size: K scales, ValueScale's log and inv
  const int32_t* table;
  int head, end, lane, wave;
  PageRun run;
  uint32_t k_from, v_from;  // bytes from a group of 16 tokens' first row to what the thread moves of it (PAGE16)

  // what the thread has under way for the next tile
  u32x4 k[kKEach];
  uint32_t v[8][kVWords];
  uint32_t none;         // of its 8 tokens of V, those past the end or on no page of the cache
  uint64_t absent;       // the tile's tokens on no page of the cache
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

  // Starts the loads of tokens [t0, t0 + 64), t0 < end.  Nothing here waits for them.
  __device__ __forceinline__ void fetch_tile(int t0) {
    const int last = end - 1, tid = threadIdx.x;
    const int tz = t0 + kManyTokens - 1 < last ? t0 + kManyTokens - 1 : last;
    const int at0 = (int)a.by_block.quotient((uint32_t)t0), at1 = (int)a.by_block.quotient((uint32_t)tz);
    if (at0 < run.base || at1 - run.base >= kWave) run.load(a, table, at0, (int)a.by_block.quotient((uint32_t)last), lane);
    const int64_t row_bytes = a.c_ts * kWidth, head_at = (int64_t)head * D * kWidth;
    const int u = v_unit();
    none = 0;
    if constexpr (PAGE16) {
      // Each group of 16 tokens lies on one page: its rows past the end are the page's too, and only have to be kept from the sums.
      absent = 0;
      int64_t at[4];  // bytes to the group's first row
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const int t = t0 + 16 * g <= last ? t0 + 16 * g : last & ~15;  // a group past the end stands for the last one
        const int in = (int)a.by_block.quotient((uint32_t)t);
        int page = uniform(__builtin_amdgcn_readlane(run.entry, in - run.base));
        if (page < 0) {
          page = 0;
          absent |= (uint64_t)0xffff << 16 * g;
        }
        at[g] = ((int64_t)page * a.block_tokens + (t - in * a.block_tokens)) * row_bytes + head_at;
        if constexpr (KIND != KVH_CACHE_16) {
          ks[g] = a.sk[(int64_t)page * a.s_ps + head];
          vs[g] = a.sv[(int64_t)page * a.s_ps + head];
        }
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
      // the bytes to the rows of tokens t0 + lane, in the lanes; a token past the end stands for the last one, one on no page for row 0
      const int mine = t0 + lane < last ? t0 + lane : last, in = (int)a.by_block.quotient((uint32_t)mine);
      const int page = __shfl(run.entry, in - run.base);
      absent = __ballot(page < 0);
      const int64_t at = page < 0 ? head_at : ((int64_t)page * a.block_tokens + (mine - in * a.block_tokens)) * row_bytes + head_at;
#pragma unroll
      for (int i = 0; i < kKEach; ++i) {
        const int idx = tid + kBlockThreads * i;
        k[i] = *reinterpret_cast<const u32x4*>(a.ck + __shfl((long long)at, idx / kKUnits) + idx % kKUnits * 16);
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) fetch_v(v[e], a.cv + __shfl((long long)at, v_token(u, e)) + v_chan() * kWidth);
      if constexpr (KIND != KVH_CACHE_16) {
        const int64_t p = page < 0 ? 0 : page;
        ks[0] = a.sk[p * a.s_ps + head];
        vs[0] = a.sv[p * a.s_ps + head];
      }
    }
    if (t0 + kManyTokens > end || absent != 0) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int t = v_token(u, 0), more = v_token(0, e);  // what differs from thread to thread, and what does not
        if (t0 + t + more >= end || (absent >> t >> more & 1) != 0) none |= 1u << e;
      }
    }
  }

  // Stores what was fetched into a buffer, as operands.
  __device__ __forceinline__ void store_tile(int buffer) {
    uint8_t* kb = lds + buffer * kBuffer;
    uint8_t* vb = kb + kKTile;
    const int tid = threadIdx.x;
#pragma unroll
    for (int i = 0; i < kKEach; ++i) {
      const int idx = tid + kBlockThreads * i, token = idx / kKUnits, unit = idx % kKUnits;
      if constexpr (KIND == KVH_CACHE_16) {
        *reinterpret_cast<u32x4*>(kb + k_place(token, unit)) = k[i];
      } else {
#pragma unroll
        for (int p = 0; p < 2; ++p) {
          uint32_t w[4];
          widen4<KIND>(k[i][2 * p], w[0], w[1]);
          widen4<KIND>(k[i][2 * p + 1], w[2], w[3]);
          *reinterpret_cast<u32x4*>(kb + k_place(token, 2 * unit + p)) = u32x4{w[0], w[1], w[2], w[3]};
        }
      }
    }
    if (__any(none != 0)) {  // what no row may meet
#pragma unroll
      for (int e = 0; e < 8; ++e)
#pragma unroll
        for (int c = 0; c < kVWords; ++c) v[e][c] = none >> e & 1 ? 0u : v[e][c];
    }
    const int u = v_unit(), ch = v_chan();
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
#pragma unroll
    for (int j = 0; j < kVChans; ++j) *reinterpret_cast<u32x4*>(vb + v_place(ch + j, u)) = u32x4{z[0][j], z[1][j], z[2][j], z[3][j]};
    if constexpr (KIND != KVH_CACHE_I8) {
      bool any = false;
#pragma unroll
      for (int e = 0; e < 8; ++e)
#pragma unroll
        for (int c = 0; c < kVWords; ++c) any |= has_odd<DT, KIND>(v[e][c]);
      any = __any(any);
      if (lane == 0) odd[buffer][wave] = any;
    }
    if constexpr (KIND != KVH_CACHE_16 && !PAGE16) {
      if (tid < kManyTokens) {
        const ValueScale z2(vs[0]);
        scales[buffer][0][tid] = ks[0];
        scales[buffer][1][tid] = z2.log;
        scales[buffer][2][tid] = z2.inv;
      }
    }
  }
};

template <int DT, int KIND, int D, bool PAGE16>
__global__ __launch_bounds__(kBlockThreads, 2) void attention_many_kernel(AttnParams a) {
  using T = Tiles<DT, KIND, D, PAGE16>;
  constexpr bool kScaled = KIND != KVH_CACHE_16;
  __shared__ __attribute__((aligned(16))) uint8_t lds[2 * T::kBuffer];
  __shared__ uint32_t odd[2][kWavesPerBlock];
  __shared__ __attribute__((aligned(16))) float scales[2][3][T::kScales];
  const int lane = threadIdx.x % kWave, wave = uniform((int32_t)(threadIdx.x / kWave));
  const int col = lane % 32, half = lane / 32;
  const uint32_t item = a.by_heads.quotient(blockIdx.x);
  const int head = (int)(blockIdx.x - item * (uint32_t)a.heads);
  Item it;
  if (!find_item(a, kManyRows, item, false, lane, it)) return;
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
  float coef = a.scale * kLog2e;
  {
    const uint16_t* src = a.q + ((int64_t)rq.start + token) * a.q_ts + ((int64_t)head * a.group + u) * D;
#pragma unroll
    for (int kk = 0; kk < T::kSums; ++kk) {
      q[kk] = u32x4{0, 0, 0, 0};
      if (real) q[kk] = *reinterpret_cast<const u32x4*>(src + kk * 16 + half * 8);
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
      most = fmaxf(most, __shfl_xor(most, 32));
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
  bool bad = false;

  T t(a);
  t.lds = lds, t.odd = odd, t.scales = scales, t.lane = lane, t.head = head, t.end = end;
  t.table = a.req.table + (int64_t)it.b * a.req.table_stride;
  t.wave = wave;
  t.begin();
  if (s0 < s1) t.fetch_tile(steps.token(s0));
  // Where the lane's operands lie in a buffer: those of a row differ in the unit's low bits, the rest is the same for all lanes.
  int k_at[4], v_at[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) k_at[e] = T::k_place(col, 2 * e + half), v_at[e] = T::v_place(col, 2 * e + half);
  int buffer = 0;
  for (int s = s0; s < s1; s += 2, buffer ^= 1) {
    const int t0 = steps.token(s);
    t.store_tile(buffer);
    const uint64_t absent = t.absent;
    float ks[4], lsv[4], inv[4], rest[4];
    bool faint = false;
    if constexpr (kScaled && PAGE16) {
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const ValueScale z(t.vs[g]);
        ks[g] = t.ks[g], lsv[g] = z.log, inv[g] = z.inv, rest[g] = z.rest;
        faint |= z.rest != 1.0f;
      }
    } else if constexpr (kScaled) {
      rest[0] = ValueScale(t.vs[0]).rest;  // of the tile's token `lane`
      faint = __any(rest[0] != 1.0f);
    }
    __syncthreads();
    if (s + 2 < s1) t.fetch_tile(steps.token(s + 2));
    const bool hidden = t0 + kManyTokens > end || (a.causal && t0 + kManyTokens - 1 > p_least) || (a.window != 0 && t0 <= p_most - a.window) || absent != 0;
    const bool blank = !works || (a.causal && t0 > p_most);  // no row of the wave sees any of it
    if (!blank) {
      const uint8_t* kb = lds + buffer * T::kBuffer;
      const uint8_t* vb = kb + T::kKTile;
      bool slow = false;
      if constexpr (KIND != KVH_CACHE_I8) slow = hidden && (odd[buffer][0] | odd[buffer][1] | odd[buffer][2] | odd[buffer][3]) != 0;
#pragma unroll
      for (int i = 0; i < 2; ++i) {  // 32 tokens at a time: element j of x is token 32 i + 8 (j / 4) + 4 half + j % 4 of the tile
        f32x16 x;
#pragma unroll
        for (int j = 0; j < 16; ++j) x[j] = 0.0f;
        u32x4 kf[T::kSums], vf[2 * T::kOuts];
#pragma unroll
        for (int kk = 0; kk < T::kSums; ++kk) kf[kk] = *reinterpret_cast<const u32x4*>(kb + k_at[kk % 4] + i * (32 * D * 2) + kk / 4 * 128);
#pragma unroll
        for (int kk = 0; kk < T::kSums; ++kk) x = mfma32<T::kBf>(kf[kk], q[kk], x);
        // Operands are read ahead of the instructions that take them: four of K first, then one with each product.
        __builtin_amdgcn_sched_group_barrier(0x100, 4, 0);
#pragma unroll
        for (int kk = 4; kk < T::kSums; ++kk) {
          __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
          __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
        }
        __builtin_amdgcn_sched_group_barrier(0x008, 4, 0);
        // and the first of V before the softmax
#pragma unroll
        for (int e = 0; e < 4; ++e) vf[e] = *reinterpret_cast<const u32x4*>(vb + v_at[2 * i + e % 2] + e / 2 * (32 * kManyTokens * 2));
        __builtin_amdgcn_sched_barrier(0);
        if constexpr (kScaled) {
#pragma unroll
          for (int j4 = 0; j4 < 4; ++j4) {
            if constexpr (PAGE16) {
              const int g = 2 * i + j4 / 2;
              const float f = ks[g] * coef;
#pragma unroll
              for (int e = 0; e < 4; ++e) x[4 * j4 + e] = __builtin_fmaf(x[4 * j4 + e], f, lsv[g]);
            } else {
              const f32x4 f = *reinterpret_cast<const f32x4*>(&scales[buffer][0][32 * i + 8 * j4 + 4 * half]);
              const f32x4 z = *reinterpret_cast<const f32x4*>(&scales[buffer][1][32 * i + 8 * j4 + 4 * half]);
#pragma unroll
              for (int e = 0; e < 4; ++e) x[4 * j4 + e] = __builtin_fmaf(x[4 * j4 + e], f[e] * coef, z[e]);
            }
          }
        }
        const float unit = kScaled ? 1.0f : coef;  // what is left to turn x into an exponent of 2
        if (hidden) {
#pragma unroll
          for (int j = 0; j < 16; ++j) {
            const int in = 32 * i + 8 * (j / 4) + j % 4;  // and 4 half more
            const bool seen = sight.sees(a, t0 + 4 * half + in), none = (absent >> 4 * half >> in & 1) != 0;
            bad |= seen && none;
            x[j] = !seen || none ? -INFINITY : x[j] * unit;
          }
        } else if constexpr (!kScaled) {
#pragma unroll
          for (int j = 0; j < 16; ++j) x[j] *= unit;
        }
        float most = x[0];
#pragma unroll
        for (int j = 1; j < 16; ++j) most = fmaxf(most, x[j]);
        most = fmaxf(most, __shfl_xor(most, 32));
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
        for (int j4 = 0; j4 < 4; ++j4) {
          f32x4 z = {1, 1, 1, 1};
          if constexpr (kScaled && !PAGE16) z = *reinterpret_cast<const f32x4*>(&scales[buffer][2][32 * i + 8 * j4 + 4 * half]);
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float w = __builtin_amdgcn_exp2f(x[4 * j4 + e] - top);
            if constexpr (!kScaled)
              l += w;
            else if constexpr (PAGE16)
              l = __builtin_fmaf(w, inv[2 * i + j4 / 2], l);
            else
              l = __builtin_fmaf(w, z[e], l);
            x[4 * j4 + e] = w;
          }
        }
        if constexpr (kScaled) {
          if (faint) {
#pragma unroll
            for (int j = 0; j < 16; ++j) {
              if constexpr (PAGE16)
                x[j] *= rest[2 * i + j / 8];
              else
                x[j] *= __shfl(rest[0], 32 * i + 8 * (j / 4) + 4 * half + j % 4);
            }
          }
        }
        u32x4 p[2];  // of each 16 tokens: the lane's 8 weights
#pragma unroll
        for (int g = 0; g < 2; ++g)
#pragma unroll
          for (int e = 0; e < 4; ++e) p[g][e] = narrow2<T::kBf ? KVH_BF16 : KVH_F16>(x[8 * g + 2 * e], x[8 * g + 2 * e + 1]);
        using Bad = Odd<T::kBf>;
#pragma unroll
        for (int e = 4; e < 2 * T::kOuts; ++e) vf[e] = *reinterpret_cast<const u32x4*>(vb + v_at[2 * i + e % 2] + e / 2 * (32 * kManyTokens * 2));
        if (slow) {
#pragma unroll
          for (int e = 0; e < 2 * T::kOuts; ++e) vf[e] = Bad::without(vf[e]);
        }
#pragma unroll
        for (int e = 0; e < 2 * T::kOuts; ++e) o[e / 2] = mfma32<T::kBf>(vf[e], p[e % 2], o[e / 2]);
        if (slow) {
          u32x4 one[2];  // of the tokens that the lane's row sees
#pragma unroll
          for (int g = 0; g < 2; ++g)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              one[g][e] = 0;
#pragma unroll
              for (int n = 0; n < 2; ++n) {
                const int j = 8 * g + 2 * e + n;
                if (sight.sees(a, t0 + 4 * half + 32 * i + 8 * (j / 4) + j % 4)) one[g][e] |= Bad::kOne << 16 * n;
              }
            }
#pragma unroll
          for (int c = 0; c < T::kOuts; ++c) {
#pragma unroll 1
            for (int which = 0; which < 3; ++which) {
              f32x16 hit;
#pragma unroll
              for (int j = 0; j < 16; ++j) hit[j] = 0.0f;
#pragma unroll
              for (int g = 0; g < 2; ++g)
                hit = mfma32<T::kBf>(Bad::ones(*reinterpret_cast<const u32x4*>(vb + v_at[2 * i + g] + c * (32 * kManyTokens * 2)), which), one[g], hit);
#pragma unroll
              for (int j = 0; j < 16; ++j) o[c][j] += hit[j] > 0.0f ? Bad::value(which) : 0.0f;
            }
          }
        }
      }
    }
  }
  if (__any(bad) && lane == 0 && a.status != nullptr) a.status[it.b] = KVH_DEV_BAD_REQUEST;

  const float sum = l + __shfl_xor(l, 32);
  if (it.parts > 1) {
    if (real) {
      const int64_t row = (int64_t)blockIdx.x * kManyRows + wave * kManyWaveRows + col;
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

template <int DT, int KIND, int D>
void launch_pages(const AttnParams& a, unsigned blocks, hipStream_t stream) {
  if (a.block_tokens % 16 == 0)
    launch_kernel(attention_many_kernel<DT, KIND, D, true>, dim3(blocks), dim3(kBlockThreads), 0, stream, a);
  else
    launch_kernel(attention_many_kernel<DT, KIND, D, false>, dim3(blocks), dim3(kBlockThreads), 0, stream, a);
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
