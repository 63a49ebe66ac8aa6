// kvh_append: keys and values of new tokens go into the pages of the serving cache, keys and queries rotated on the way.
//
// A lane holds 8 neighbouring channels (one 16-byte load, one 16- or 8-byte store), D / 8 lanes a head.  A wave takes a unit of one
// request.  Queries, and keys and values of a 16-bit cache: some rows of 512 / D neighbouring heads, so that an access is 1 KiB of one token and
// its lanes share the row's cosines and sines.  An 8-bit page is described by one scale a head, so there the unit is a page
// and a head: its new rows are read and rotated, their largest magnitude is found across the wave, and they are stored as codes.  The
// other half of a rotated pair is 0 lanes away or rot / 16 lanes, and comes by a lane exchange, which also makes q_out == q safe.
//
// Memory bounds it (some 6 operations an element), or for a step of single tokens the launch.  Measured, 8 KV heads of 128, 32 query heads: a
// prompt of 8192 into e4m3, rotated: 38.9 us = 4.9 TB/s, what a plain copy reaches; 16 prompts of 1500 in 16 bits (10 KV heads of 64): 49.8 us = 4.9
// TB/s; 32 layers of 256 tokens into int8: 11.5 us = 4.4 TB/s; 64 single tokens into int8: 5.5 us, one: 4.7 us, a kernel of 3.7.  The grid is as wide as the
// request with the most new tokens for every one: a prompt of 8192 beside 63 single tokens takes 234 us, apart 39 and 5.
#include "kvh_cache.hpp"

namespace kvh {
namespace {

constexpr int kPageRows = 16;  // rows of an 8-bit page that are taken at once
constexpr int kTileRows = 4;   // and of a unit of queries or of a 16-bit cache (8K prompt, e4m3, one head a unit: 41.4 us; 8 rows 44.0, 16 rows 51)

struct AppendParams {
  Requests req;
  const uint16_t *k, *v, *q;
  uint16_t* q_out;
  int64_t kv_ls, kv_ts, q_ls, q_ts, o_ls, o_ts;  // elements
  uint8_t *ck, *cv;
  float *sk, *sv;
  int64_t c_ls, c_ts;  // elements of the cache
  int64_t s_ls, s_ps;  // floats
  int pages, block_tokens, heads, q_heads;
  const float* table;
  const int32_t* positions;
  int64_t table_stride;
  int n_positions, rot, pairs;  // rot 0: nothing is rotated
  int32_t* status;
  uint32_t kv_units, units;  // of a request and layer
  Divisor by_block, by_kv;  // block_tokens; 2 heads
};

// Rows that are read once and written once pass by the caches (PAST), unless they are so few that what reads them next finds them there.
template <bool PAST, typename V>
__device__ __forceinline__ V get(const void* p) {
  if constexpr (PAST)
    return __builtin_nontemporal_load(reinterpret_cast<const V*>(p));
  else
    return *reinterpret_cast<const V*>(p);
}
template <bool PAST, typename V>
__device__ __forceinline__ void put(void* p, const V& v) {
  if constexpr (PAST)
    __builtin_nontemporal_store(v, reinterpret_cast<V*>(p));
  else
    *reinterpret_cast<V*>(p) = v;
}

// The 8 values of a lane, rotated by row `pos` of the table; cb is its first channel in the head.  All lanes of a head take part.
template <int DT>
__device__ __forceinline__ void turn8(const AppendParams& a, const u32x4& raw, int pos, int cb, int lane, float (&x)[8]) {
  widen8<DT>(raw, x);
  const float* row = a.table + (int64_t)pos * a.table_stride;
  if (a.pairs) {
    if (cb < a.rot) {
      const f32x4 c = *reinterpret_cast<const f32x4*>(row + cb / 2), n = *reinterpret_cast<const f32x4*>(row + (a.rot + cb) / 2);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float x1 = x[2 * e], x2 = x[2 * e + 1];
        x[2 * e] = x1 * c[e] - x2 * n[e];
        x[2 * e + 1] = x2 * c[e] + x1 * n[e];
      }
    }
    return;
  }
  const int half = a.rot / 2, far = half / 8;
  const bool low = cb < half;
  const int other = cb < a.rot ? (low ? lane + far : lane - far) : lane;
  u32x4 ow;
#pragma unroll
  for (int e = 0; e < 4; ++e) ow[e] = (uint32_t)__shfl((int)raw[e], other);
  if (cb < a.rot) {
    float y[8];
    widen8<DT>(ow, y);
    const float* t = row + (low ? cb : cb - half);
#pragma unroll
    for (int p = 0; p < 2; ++p) {
      const f32x4 c = *reinterpret_cast<const f32x4*>(t + 4 * p), n = *reinterpret_cast<const f32x4*>(t + half + 4 * p);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        float& v = x[4 * p + e];
        const float part = y[4 * p + e] * n[e];
        v = low ? v * c[e] - part : v * c[e] + part;
      }
    }
  }
}

template <int DT>
__device__ __forceinline__ u32x4 packed8(const float (&x)[8]) {
  return u32x4{narrow2<DT>(x[0], x[1]), narrow2<DT>(x[2], x[3]), narrow2<DT>(x[4], x[5]), narrow2<DT>(x[6], x[7])};
}

// The position of a request's new token i; -1 where the table has none for it.
__device__ __forceinline__ int position(const AppendParams& a, const Request& rq, int i) {
  const int pos = a.positions != nullptr ? a.positions[rq.start + i] : rq.len - rq.n + i;
  return pos < a.n_positions ? pos : -1;
}

// One head's rows [i0, i0 + 16) of a request (i < i_end) in registers: D / 8 lanes a row.
template <int DT, int D>
struct Tile {
  static constexpr int kLanes = D / 8;
  static constexpr int kRows = kWave / kLanes;  // of one access of the wave
  static constexpr int kSteps = kPageRows / kRows;
  float x[kSteps][8];
  bool valid[kSteps];

  // `turn`: rotate.  Returns whether a token had no position in the table, which then is not valid, rotated or not.
  __device__ __forceinline__ bool load(const AppendParams& a, const uint16_t* src, int64_t ts, const Request& rq, int i0, int i_end,
                                       bool turn, int lane) {
    const int col = lane % kLanes, sub = lane / kLanes;
    bool bad = false;
    u32x4 raw[kSteps];
    int pos[kSteps];
#pragma unroll
    for (int s = 0; s < kSteps; ++s) {
      const int i = i0 + s * kRows + sub;
      valid[s] = i < i_end;
      raw[s] = u32x4{0, 0, 0, 0};
      pos[s] = 0;
      if (valid[s]) {
        raw[s] = *reinterpret_cast<const u32x4*>(src + ((int64_t)rq.start + i) * ts + col * 8);
        if (a.rot != 0) {
          pos[s] = position(a, rq, i);
          if (pos[s] < 0) {
            bad = true;
            valid[s] = false;
            pos[s] = 0;
          }
        }
      }
    }
#pragma unroll
    for (int s = 0; s < kSteps; ++s) {
      if (turn)
        turn8<DT>(a, raw[s], pos[s], col * 8, lane, x[s]);
      else
        widen8<DT>(raw[s], x[s]);
    }
    return bad;
  }
};

template <int KIND>
__device__ __forceinline__ u32x2 codes8(const float (&y)[8]) {
  u32x2 w;
#pragma unroll
  for (int p = 0; p < 2; ++p) {
    if constexpr (KIND == KVH_CACHE_I8) {
      uint32_t b[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) b[e] = (uint32_t)(int)__builtin_rintf(y[4 * p + e]) & 0xffu;
      w[p] = b[0] | b[1] << 8 | b[2] << 16 | b[3] << 24;
    } else {
      int r = __builtin_amdgcn_cvt_pk_fp8_f32(y[4 * p], y[4 * p + 1], 0, false);
      w[p] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(y[4 * p + 2], y[4 * p + 3], r, true);
    }
  }
  return w;
}

template <int KIND>
__device__ __forceinline__ void values8(const u32x2& w, float (&y)[8]) {
#pragma unroll
  for (int p = 0; p < 2; ++p) {
    if constexpr (KIND == KVH_CACHE_I8) {
#pragma unroll
      for (int e = 0; e < 4; ++e) y[4 * p + e] = (float)(int8_t)(w[p] >> 8 * e);
    } else {
      y[4 * p] = __builtin_amdgcn_cvt_f32_fp8((int)w[p], 0);
      y[4 * p + 1] = __builtin_amdgcn_cvt_f32_fp8((int)w[p], 1);
      y[4 * p + 2] = __builtin_amdgcn_cvt_f32_fp8((int)w[p], 2);
      y[4 * p + 3] = __builtin_amdgcn_cvt_f32_fp8((int)w[p], 3);
    }
  }
}

__device__ __forceinline__ float wave_max(float v) {
#pragma unroll
  for (int d = 1; d < kWave; d *= 2) v = fmaxf(v, __shfl_xor(v, d));
  return v;
}

template <int DT, int KIND, int D, bool PAST>
__global__ __launch_bounds__(kBlockThreads) void append_kernel(AppendParams a) {
  using T = Tile<DT, D>;
  const int lane = threadIdx.x % kWave;
  const uint32_t u = uniform((int32_t)(blockIdx.x * kWavesPerBlock + threadIdx.x / kWave));
  if (u >= a.units) return;
  const int b = blockIdx.y, layer = blockIdx.z;
  Request rq;
  rq.start = a.req.starts[b];
  const int32_t end = a.req.starts[b + 1];
  rq.len = a.req.lens[b];
  rq.n = end - rq.start;
  rq.ok = request_ok(a.req, rq.start, end, rq.len) && rq.len >= rq.n;
  const bool tells = lane == 0 && a.status != nullptr;
  if (!rq.ok) {
    if (tells && u == 0) a.status[b] = KVH_DEV_BAD_REQUEST;
    return;
  }
  const int before = rq.len - rq.n, col = lane % T::kLanes, sub = lane / T::kLanes;
  const int32_t* table = a.req.table + (int64_t)b * a.req.table_stride;
  bool bad = false;
  // Rows [i0, i0 + 4) of heads [head0, head0 + 512 / D), from src; `page_of` looks up what `to` needs to say where a row goes
  // (nullptr: nowhere), in time.
  auto move_rows = [&](const uint16_t* src, int64_t ts, int heads, uint32_t unit, bool turn, auto&& page_of, auto&& to) {
    constexpr int kHeads = kWave / T::kLanes, kAtOnce = kTileRows;
    const uint32_t groups = (uint32_t)(heads + kHeads - 1) / kHeads, tile = unit / groups;
    const int head = (int)(unit - tile * groups) * kHeads + sub, i0 = (int)tile * kTileRows;
    const bool mine = head < heads;
    const int64_t at = (int64_t)(mine ? head : 0) * D + col * 8;
    if (i0 < rq.n) {
      u32x4 raw[kAtOnce];
      int pos[kAtOnce], page[kAtOnce];
#pragma unroll
      for (int s = 0; s < kAtOnce; ++s) {
        const int i = i0 + s < rq.n ? i0 + s : rq.n - 1;
        page[s] = page_of(i);
        raw[s] = get<PAST, u32x4>(src + ((int64_t)rq.start + i) * ts + at);
        pos[s] = a.rot != 0 ? position(a, rq, i) : 0;  // a token without one is not stored, its values no more than its keys
      }
#pragma unroll
      for (int s = 0; s < kAtOnce; ++s) {
        if (turn) {
          float x[8];
          turn8<DT>(a, raw[s], pos[s] < 0 ? 0 : pos[s], col * 8, lane, x);
          if (col * 8 < a.rot) raw[s] = packed8<DT>(x);  // other channels keep every bit, those of a NaN too
        }
        if (i0 + s >= rq.n) continue;
        uint16_t* row = pos[s] < 0 ? nullptr : to(i0 + s, page[s]);
        if (row == nullptr)
          bad = true;
        else if (mine)
          put<PAST>(row + at, raw[s]);
      }
    }
  };
  if (u >= a.kv_units) {  // queries
    uint16_t* out = a.q_out + layer * a.o_ls;
    move_rows(a.q + layer * a.q_ls, a.q_ts, a.q_heads, u - a.kv_units, a.rot != 0, [](int) { return 0; },
              [&](int i, int) { return out + ((int64_t)rq.start + i) * a.o_ts; });
  } else {
    if constexpr (KIND == KVH_CACHE_16) {
      const bool is_v = u >= a.kv_units / 2;
      uint16_t* cache = reinterpret_cast<uint16_t*>(is_v ? a.cv : a.ck) + layer * a.c_ls;
      move_rows((is_v ? a.v : a.k) + layer * a.kv_ls, a.kv_ts, a.heads, is_v ? u - a.kv_units / 2 : u, !is_v && a.rot != 0,
                [&](int i) { return table[a.by_block.quotient((uint32_t)(before + i))]; },
                [&](int i, int page) -> uint16_t* {
                  if (page < 0 || page >= a.pages) return nullptr;
                  const int slot = before + i, at = (int)a.by_block.quotient((uint32_t)slot);
                  return cache + ((int64_t)page * a.block_tokens + (slot - at * a.block_tokens)) * a.c_ts;
                });
    } else {
      const uint32_t part = a.by_kv.quotient(u);
      uint32_t head = u - part * 2u * (uint32_t)a.heads;
      const bool is_v = head >= (uint32_t)a.heads;
      if (is_v) head -= a.heads;
      const uint16_t* src = (is_v ? a.v : a.k) + layer * a.kv_ls + head * D;
      const bool turn = !is_v && a.rot != 0;
      uint8_t* cache = (is_v ? a.cv : a.ck) + layer * a.c_ls + head * D;
      T t;
      const int at = (int)a.by_block.quotient((uint32_t)before) + (int)part;  // the page's place in the request
      const int64_t page_slot = (int64_t)at * a.block_tokens;
      const int i0 = page_slot > before ? (int)(page_slot - before) : 0;
      if (i0 >= rq.n) return;
      const int64_t past = page_slot + a.block_tokens - before;
      const int i_end = past < rq.n ? (int)past : rq.n;
      const int page = table[at];
      bad = t.load(a, src, a.kv_ts, rq, i0, i_end, turn, lane);  // on the way while the page is looked up
      if (page < 0 || page >= a.pages) {
        if (tells) a.status[b] = KVH_DEV_BAD_REQUEST;
        return;
      }
      const int row0 = (int)(before + i0 - page_slot);  // the first new row of the page
      float* scale_at = (is_v ? a.sv : a.sk) + layer * a.s_ls + (int64_t)page * a.s_ps + head;
      const float old = row0 > 0 ? *scale_at : 0.0f;
      float most = 0.0f;
      for (int i = i0; i < i_end; i += kPageRows) {
        if (i > i0) bad |= t.load(a, src, a.kv_ts, rq, i, i_end, turn, lane);
#pragma unroll
        for (int s = 0; s < T::kSteps; ++s)
          if (t.valid[s]) {
#pragma unroll
            for (int e = 0; e < 8; ++e) most = fmaxf(most, fabsf(t.x[s][e]));
          }
      }
      most = wave_max(most);
      constexpr float kPart = 1.0f / (KIND == KVH_CACHE_I8 ? 127.0f : 448.0f);
      const float now = fmaxf(old, most < 0x1p-100f ? 0.0f : most * kPart);
      const float inv = now > 0.0f ? 1.0f / now : 0.0f;
      uint8_t* rows = cache + (int64_t)page * a.block_tokens * a.c_ts + col * 8;
      if (now > old && old > 0.0f) {  // earlier rows of the page under its new scale
        const float rate = old / now;
        for (int r = sub; r < row0; r += T::kRows) {
          u32x2* p = reinterpret_cast<u32x2*>(rows + (int64_t)r * a.c_ts);
          float y[8];
          values8<KIND>(*p, y);
#pragma unroll
          for (int e = 0; e < 8; ++e) y[e] *= rate;
          *p = codes8<KIND>(y);
        }
      }
      for (int i = i0; i < i_end; i += kPageRows) {
        if (i_end - i0 > kPageRows) t.load(a, src, a.kv_ts, rq, i, i_end, turn, lane);  // otherwise the rows are still here
#pragma unroll
        for (int s = 0; s < T::kSteps; ++s)
          if (t.valid[s]) {
            float y[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) y[e] = t.x[s][e] * inv;
            const int r = row0 + (i - i0) + s * T::kRows + sub;
            put<PAST>(rows + (int64_t)r * a.c_ts, codes8<KIND>(y));
          }
      }
      if (lane == 0) *scale_at = now;
    }
  }
  if (__any(bad) && tells) a.status[b] = KVH_DEV_BAD_REQUEST;
}

template <int DT, int KIND, int D>
void launch_past(const AppendParams& a, bool past, dim3 grid, hipStream_t stream) {
  if (past)
    launch_kernel(append_kernel<DT, KIND, D, true>, grid, dim3(kBlockThreads), 0, stream, a);
  else
    launch_kernel(append_kernel<DT, KIND, D, false>, grid, dim3(kBlockThreads), 0, stream, a);
}

template <int DT, int KIND>
void launch_dim(const AppendParams& a, int head_dim, bool past, dim3 grid, hipStream_t stream) {
  if (head_dim == 128)
    launch_past<DT, KIND, 128>(a, past, grid, stream);
  else
    launch_past<DT, KIND, 64>(a, past, grid, stream);
}

template <int DT>
void launch_kind(const AppendParams& a, int kind, int head_dim, bool past, dim3 grid, hipStream_t stream) {
  switch (kind) {
    case KVH_CACHE_16: return launch_dim<DT, KVH_CACHE_16>(a, head_dim, past, grid, stream);
    case KVH_CACHE_I8: return launch_dim<DT, KVH_CACHE_I8>(a, head_dim, past, grid, stream);
    default: return launch_dim<DT, KVH_CACHE_E4M3>(a, head_dim, past, grid, stream);
  }
}

}  // namespace
}  // namespace kvh

using namespace kvh;

extern "C" int kvh_append(const kvh_cache* cache, const kvh_requests* requests, kvh_dtype dt, const kvh_kv_view* kv, const kvh_rows* q,
                          const kvh_rows* q_out, int q_heads, const kvh_rotation* rotation, int32_t* status_dev, void* stream) {
  if (dt != KVH_F16 && dt != KVH_BF16) return KVH_E_ARG;
  if (int rc = check_cache(cache)) return rc;
  if (int rc = check_requests(requests)) return rc;
  if (kv == nullptr) return KVH_E_ARG;
  const int64_t c = (int64_t)cache->heads * cache->head_dim;
  for (void* p : {kv->k, kv->v}) {
    const kvh_rows rows{p, kv->layer_stride, kv->token_stride};
    if (int rc = check_rows(&rows, c, requests->n_tokens)) return rc;
  }
  AppendParams a{};
  if (q != nullptr) {
    if (q_out == nullptr) return KVH_E_ARG;
    if (q_heads < 1 || q_heads > 65536) return KVH_E_SHAPE;
    for (const kvh_rows* r : {q, q_out})
      if (int rc = check_rows(r, (int64_t)q_heads * cache->head_dim, requests->n_tokens)) return rc;
    a.q = static_cast<const uint16_t*>(q->p);
    a.q_out = static_cast<uint16_t*>(q_out->p);
    a.q_ls = q->layer_stride, a.q_ts = q->token_stride;
    a.o_ls = q_out->layer_stride, a.o_ts = q_out->token_stride;
    a.q_heads = q_heads;
  }
  if (rotation != nullptr) {
    if (rotation->table == nullptr || rotation->n_positions < 1 || rotation->table_stride < 0) return KVH_E_ARG;
    if (rotation->rot < 16 || rotation->rot % 16 != 0 || rotation->rot > cache->head_dim) return KVH_E_SHAPE;
    if (!is_aligned16(rotation->table) || rotation->table_stride % 4 != 0) return KVH_E_ALIGN;
    a.table = rotation->table;
    a.positions = rotation->positions;
    a.table_stride = rotation->table_stride;
    a.n_positions = rotation->n_positions;
    a.rot = rotation->rot;
    a.pairs = rotation->pairs;
  }
  if (requests->n_tokens == 0) return KVH_OK;
  a.req = Requests(*requests, cache->block_tokens);
  a.k = static_cast<const uint16_t*>(kv->k), a.v = static_cast<const uint16_t*>(kv->v);
  a.kv_ls = kv->layer_stride, a.kv_ts = kv->token_stride;
  a.ck = static_cast<uint8_t*>(cache->k), a.cv = static_cast<uint8_t*>(cache->v);
  a.sk = cache->k_scale, a.sv = cache->v_scale;
  a.c_ls = cache->layer_stride, a.c_ts = cache->token_stride;
  a.s_ls = cache->scale_layer_stride, a.s_ps = cache->scale_page_stride;
  a.pages = cache->pages, a.block_tokens = cache->block_tokens, a.heads = cache->heads;
  a.status = status_dev;
  a.by_block = Divisor((uint32_t)cache->block_tokens);
  a.by_kv = Divisor(2u * (uint32_t)cache->heads);
  const int most = requests->max_new < requests->n_tokens ? requests->max_new : requests->n_tokens;
  a.req.max_new = most;
  const int64_t tiles = (most + kTileRows - 1) / kTileRows, together = 512 / cache->head_dim;  // heads of a unit
  const int64_t spread = ((int64_t)most + cache->block_tokens - 2) / cache->block_tokens + 1;  // pages that `most` tokens touch at most
  const int64_t parts = spread < most ? spread : most;
  const int64_t kv_units = 2 * (cache->kind == KVH_CACHE_16 ? tiles * ((cache->heads + together - 1) / together) : parts * cache->heads);
  const int64_t units = kv_units + tiles * ((a.q_heads + together - 1) / together);
  // Measured at 8K tokens of 8 + 32 heads, e4m3: 39.6 us by the caches, 46.2 through them; at 64 single tokens the two are alike.
  const bool past = (int64_t)requests->n_tokens * cache->layers * (2 * cache->heads + a.q_heads) * cache->head_dim >= (int64_t)4 << 20;
  if (units >= (int64_t)1 << 31) return KVH_E_SHAPE;
  a.kv_units = (uint32_t)kv_units, a.units = (uint32_t)units;
  const dim3 grid((unsigned)((units + kWavesPerBlock - 1) / kWavesPerBlock), (unsigned)requests->n_requests, (unsigned)cache->layers);
  if (dt == KVH_F16)
    launch_kind<KVH_F16>(a, cache->kind, cache->head_dim, past, grid, static_cast<hipStream_t>(stream));
  else
    launch_kind<KVH_BF16>(a, cache->kind, cache->head_dim, past, grid, static_cast<hipStream_t>(stream));
  KVH_HIP_CHECK_LAUNCH();
  return KVH_OK;
}
