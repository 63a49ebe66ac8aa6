// kvh_copy_pages, kvh_fork, kvh_compact: pages of the serving cache change hands.
//
// Contents move by pairs of pages, 16 KiB a block; memory bounds that.  Who holds what is integer work on the table and the counts, which is bound by the trips to
// memory that wait for each other: a block plans, with the counts in LDS where they fit, and a second launch writes the rows and copies at the same
// time.  Counts change by atomic additions of whole numbers, whose order is of no account.
// Measured, calls among others: 512 pages of 8 layers (268 MB) copied 103 us = 5.2 TB/s (a plain copy of 4 GiB reaches 5.5); 3 pages of 32 layers, int8: 4.4 us; fork, 64 rows of 4096 tokens
// (lognormal) that grow by one: 14.9 us (plan 8 to 12), 16 requests of 4 beams: 13.2; compact, 450 pages of 8 layers: 84.5 us = 5.6 TB/s, 1024 pages of one layer: 6.8.  One block walks
// the counts, so large pools take their time: 64 rows that grow in a pool of 50000 pages 32 us, of 100000 49, of 200000 127; compact, one small layer, 15000 pages 30, 50000 72, 100000 132, 200000 230.
#include "kvh_cache.hpp"

#include <algorithm>

namespace kvh {
namespace {

// ---- copying ------------------------------------------------------------------------------------------------------
struct CopyParams {
  const int32_t *src, *dst;
  int32_t* status;
  uint8_t *ck, *cv;
  float *sk, *sv;
  int8_t* codes;   // of the bounds, or nullptr
  float* b_scale;
  int64_t c_ls, c_ts, s_ls, s_ps, b_ls, b_ps, bs_ls, bs_ps;  // cache and bounds' codes in bytes, scales in floats
  int pages, block_tokens, heads, box;  // box: 16-byte words of a page's bounds
  uint32_t row_words, words;  // 16-byte words of a row, and of a page
  uint32_t parts;             // blocks of a page and layer: those of K, those of V, one for the rest
  uint32_t layers;
  int past;                   // many pages pass by the caches
  Divisor by_parts, by_each, by_row;  // by_each: blocks of a pair
  int64_t each() const { return (int64_t)parts * layers; }  // blocks of a pair
};

constexpr int kCopyWords = 4;  // 16-byte words of a thread
constexpr int64_t kMostBlocks = ((int64_t)1 << 31) - 1;

// Part `in_pair` of a pair's parts * layers.
__device__ __forceinline__ void copy_part(const CopyParams& a, uint32_t i, uint32_t in_pair) {
  const uint32_t layer = a.by_parts.quotient(in_pair), part = in_pair - layer * a.parts;
  const int src = a.src[i], dst = a.dst[i];
  if (src < 0 || src == dst) return;
  if (src >= a.pages || dst < 0 || dst >= a.pages) {
    if (threadIdx.x == 0 && part == 0 && layer == 0 && a.status != nullptr) a.status[i] = KVH_DEV_BAD_REQUEST;
    return;
  }
  const uint32_t half = (a.parts - 1) / 2;
  if (part < 2 * half) {
    uint8_t* base = (part < half ? a.ck : a.cv) + layer * a.c_ls;
    const uint32_t w0 = (part < half ? part : part - half) * (kBlockThreads * kCopyWords) + threadIdx.x;
    const uint8_t* from = base + (int64_t)src * a.block_tokens * a.c_ts;
    uint8_t* to = base + (int64_t)dst * a.block_tokens * a.c_ts;
    u32x4 x[kCopyWords];
    int64_t at[kCopyWords];
#pragma unroll
    for (int e = 0; e < kCopyWords; ++e) {
      const uint32_t w = w0 + e * kBlockThreads, row = a.by_row.quotient(w);
      at[e] = row * a.c_ts + (int64_t)(w - row * a.row_words) * 16;
    }
    auto move = [&](auto&& get, auto&& put) {
#pragma unroll
      for (int e = 0; e < kCopyWords; ++e)
        if (w0 + e * kBlockThreads < a.words) x[e] = get(reinterpret_cast<const u32x4*>(from + at[e]));
#pragma unroll
      for (int e = 0; e < kCopyWords; ++e)
        if (w0 + e * kBlockThreads < a.words) put(x[e], reinterpret_cast<u32x4*>(to + at[e]));
    };
    if (a.past)
      move([](const u32x4* p) { return __builtin_nontemporal_load(p); }, [](const u32x4& v, u32x4* p) { __builtin_nontemporal_store(v, p); });
    else
      move([](const u32x4* p) { return *p; }, [](const u32x4& v, u32x4* p) { *p = v; });
    return;
  }
  for (int h = threadIdx.x; h < a.heads; h += kBlockThreads) {
    if (a.sk != nullptr) {
      float *k = a.sk + layer * a.s_ls + h, *v = a.sv + layer * a.s_ls + h;
      k[dst * a.s_ps] = k[src * a.s_ps];
      v[dst * a.s_ps] = v[src * a.s_ps];
    }
    if (a.b_scale != nullptr) {
      float* s = a.b_scale + layer * a.bs_ls + h;
      s[dst * a.bs_ps] = s[src * a.bs_ps];
    }
  }
  if (a.codes != nullptr) {
    int8_t* codes = a.codes + layer * a.b_ls;
    for (int w = threadIdx.x; w < a.box; w += kBlockThreads)
      *reinterpret_cast<u32x4*>(codes + dst * a.b_ps + (int64_t)w * 16) = *reinterpret_cast<const u32x4*>(codes + src * a.b_ps + (int64_t)w * 16);
  }
}

__global__ __launch_bounds__(kBlockThreads) void copy_kernel(CopyParams a) {
  const uint32_t i = a.by_each.quotient(blockIdx.x);
  copy_part(a, i, blockIdx.x - i * a.by_each.d);
}

// Pairs whose number the device knows, by the blocks of a launch from `first` on.
__device__ __forceinline__ void copy_many(const CopyParams& a, const int32_t* many, uint32_t first) {
  const uint32_t each = a.by_each.d, blocks = gridDim.x - first;
  const uint64_t units = (uint64_t)(uint32_t)uniform(*many) * each;
  for (uint64_t u = blockIdx.x - first; u < units; u += blocks) {
    const uint32_t i = u < (1u << 31) ? a.by_each.quotient((uint32_t)u) : (uint32_t)(u / each);
    copy_part(a, i, (uint32_t)(u - (uint64_t)i * each));
  }
}
// Blocks that such a launch has for them at most: enough to fill the chip, and not one for each copy that there might be.  Fork, where most rows copy nothing (32
// layers, 64 rows: 9.8 us, 10.2 with 16384; 256 rows: 17.8 and 20.4); compact, where many pages move (8 layers of 450 pages: 84.5 us, 90.5 with 4096, 96
// with 2048).
constexpr int64_t kForkBlocks = 4096, kCompactBlocks = 16384;

// Bytes of K and V from which on copies pass by the caches: 512 pages of 8 layers 4 us less than through them, of 113; compact, 450 pages of 8 layers, 11 of 100.  Fork copies
// a page that is appended to next.
constexpr int64_t kPastBytes = 16 << 20;

// What bounds and scales there are goes along.
int copy_params(const kvh_cache& c, const kvh_bounds* b, const int32_t* src, const int32_t* dst, int64_t pairs, int32_t* status, CopyParams& a) {
  const int width = c.kind == KVH_CACHE_16 ? 2 : 1;
  a.src = src, a.dst = dst, a.status = status;
  a.ck = static_cast<uint8_t*>(c.k), a.cv = static_cast<uint8_t*>(c.v);
  a.sk = c.k_scale, a.sv = c.v_scale;
  a.c_ls = c.layer_stride * width, a.c_ts = c.token_stride * width, a.s_ls = c.scale_layer_stride, a.s_ps = c.scale_page_stride;
  a.pages = c.pages, a.block_tokens = c.block_tokens, a.heads = c.heads;
  if (b != nullptr) {
    a.codes = b->codes, a.b_scale = b->scale;
    a.b_ls = b->layer_stride, a.b_ps = b->page_stride, a.bs_ls = b->scale_layer_stride, a.bs_ps = b->scale_page_stride;
    a.box = c.heads * 2 * c.head_dim / 16;
  }
  a.row_words = (uint32_t)(c.heads * c.head_dim * width / 16);
  const int64_t words = (int64_t)a.row_words * c.block_tokens, half = (words + kBlockThreads * kCopyWords - 1) / (kBlockThreads * kCopyWords);
  if (words >= (int64_t)1 << 30) return KVH_E_SHAPE;
  a.words = (uint32_t)words;
  a.parts = (uint32_t)(2 * half + 1);
  a.layers = (uint32_t)c.layers;
  a.past = pairs * words * 32 * c.layers >= kPastBytes;
  a.by_parts = Divisor(a.parts), a.by_row = Divisor(a.row_words);
  if (a.each() > kMostBlocks / 2) return KVH_E_SHAPE;
  a.by_each = Divisor((uint32_t)a.each());
  return KVH_OK;
}

// `pairs` of them at most.
int launch_copy(CopyParams& a, int64_t pairs, hipStream_t stream) {
  const int64_t most = kMostBlocks / a.each();  // of a launch
  for (int64_t i = 0; i < pairs; i += most) {
    const int64_t n = std::min(most, pairs - i);
    launch_kernel(copy_kernel, dim3((unsigned)(n * a.each())), dim3(kBlockThreads), 0, stream, a);
    KVH_HIP_CHECK_LAUNCH();
    a.src += n, a.dst += n;
    if (a.status != nullptr) a.status += n;
  }
  return KVH_OK;
}

// ---- forking ------------------------------------------------------------------------------------------------------
struct RowsParams {
  const int32_t* table;
  int32_t* table_out;
  int64_t ts, to_ts;
  const int32_t* lens;
  const int32_t* refs;
  int32_t* refs_out;
  int table_pages, n, pages, block_tokens;
  int64_t capacity;  // tokens that a row has pages for, and a request may have
  int32_t* status;
  Divisor by_block;
};

// What becomes of a row, in the workspace.
struct Child {
  int32_t parent;  // -1: none
  int32_t len;     // tokens after the call
  int32_t full, kept, after;  // pages that are shared, that are not fresh, and all
  int32_t ok, copies;  // whether an unfilled page is copied, which is entry `full` of the parent
  int32_t base;    // its place among the fresh pages; -1 where there are too few
};

struct ForkParams {
  RowsParams r;
  const int32_t *parents, *grow;
  int32_t* lens_out;
  // workspace
  Child* child;        // of each row
  int32_t *src, *dst;  // pairs to copy, and how many
  int32_t* pairs;
  int32_t* fresh;      // free pages in order
};

__device__ __forceinline__ int pages_of(const RowsParams& r, int tokens) { return tokens > 0 ? (int)r.by_block.quotient((uint32_t)tokens - 1) + 1 : 0; }

__global__ __launch_bounds__(kBlockThreads) void start_kernel(RowsParams r) {
  const int p = blockIdx.x * kBlockThreads + threadIdx.x;
  if (p < r.pages) r.refs_out[p] = r.refs[p];
}

// A row's child as its numbers say, without a look at the table and at the other rows; `tokens` are the parent's.
__device__ __forceinline__ Child child_of(const ForkParams& a, int b, int& tokens, bool& open) {
  const RowsParams& r = a.r;
  Child c{};
  c.parent = a.parents == nullptr ? b : a.parents[b];
  if (c.parent < 0) c.parent = -1;
  const int64_t grow = a.grow == nullptr ? 0 : a.grow[b];
  c.ok = c.parent < r.n && grow >= 0;
  tokens = c.ok && c.parent >= 0 ? r.lens[c.parent] : 0;
  c.ok = c.ok && tokens >= 0 && tokens + grow <= r.capacity;
  if (!c.ok) tokens = 0;
  c.len = c.ok ? (int)(tokens + grow) : 0;
  c.full = (int)r.by_block.quotient((uint32_t)tokens);
  open = tokens - c.full * r.block_tokens != 0;
  c.after = pages_of(r, c.len);
  return c;
}
// With what the table says - an entry of the parent's is none of the cache's - and whether a row before it has the parent's unfilled page.
__device__ __forceinline__ void settle(const ForkParams& a, int b, Child& c, bool open, bool odd, bool other) {
  if (odd) c.ok = 0;
  if (!c.ok) c.len = c.full = c.after = 0;
  c.copies = c.ok && open && other;
  c.kept = c.full + (c.ok && open && !other);
  a.child[b] = c;
  if (!c.ok && a.r.status != nullptr) a.r.status[b] = KVH_DEV_BAD_REQUEST;
}

// The row's references before the call and after it, but for fresh pages; those of a row that is its own child are the same as far as it keeps them.
template <int THREADS>
__device__ __forceinline__ void count_row(const RowsParams& r, int b, int len, int parent, int kept, int32_t* refs, int id) {
  const int32_t* old = r.table + (int64_t)b * r.ts;
  const int same = parent == b ? kept : 0;
  if (len > 0 && len <= r.capacity) {
#pragma unroll 4
    for (int j = same + id; j < pages_of(r, len); j += THREADS)
      if ((uint32_t)old[j] < (uint32_t)r.pages) atomicSub(&refs[old[j]], 1);
  }
  if (parent >= 0) {
    const int32_t* from = r.table + (int64_t)parent * r.ts;
#pragma unroll 4
    for (int j = same + id; j < kept; j += THREADS) atomicAdd(&refs[from[j]], 1);
  }
}

__global__ __launch_bounds__(kBlockThreads) void count_kernel(ForkParams a) {
  const RowsParams& r = a.r;
  const int b = blockIdx.x;
  int tokens;
  bool open, odd = false, other = false;
  Child c = child_of(a, b, tokens, open);
  if (c.ok && c.parent >= 0) {
    const int32_t* from = r.table + (int64_t)c.parent * r.ts;
    for (int j = threadIdx.x; j < c.full + open; j += kBlockThreads) odd |= (uint32_t)from[j] >= (uint32_t)r.pages;
    if (open && a.parents != nullptr)
      for (int i = threadIdx.x; i < b; i += kBlockThreads)  // (what a child that is refused would keep is not kept, and may be handed out)
        if (a.parents[i] == c.parent) other |= a.grow == nullptr || (a.grow[i] >= 0 && tokens + (int64_t)a.grow[i] <= r.capacity);
  }
  odd = __syncthreads_or(odd) != 0;
  other = __syncthreads_or(other) != 0;
  if (threadIdx.x == 0) settle(a, b, c, open, odd, other);
  const bool ok = c.ok && !odd;
  count_row<kBlockThreads>(r, b, r.lens[b], c.parent, ok ? c.full + (open && !other) : 0, r.refs_out, threadIdx.x);
}

constexpr int kScanThreads = 1024, kScanWaves = kScanThreads / kWave;

// The sum of all threads' values before this one's, and of all; one block of kScanThreads.
__device__ __forceinline__ int64_t before_me(int64_t v, int64_t* lds, int64_t& all) {
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  int64_t x = v;
#pragma unroll
  for (int d = 1; d < kWave; d *= 2) {
    const int64_t y = __shfl_up((long long)x, d);
    if (lane >= d) x += y;
  }
  __syncthreads();
  if (lane == kWave - 1) lds[wave] = x;
  __syncthreads();
  int64_t base = 0;
  all = 0;
  for (int w = 0; w < kScanWaves; ++w) {
    if (w == wave) base = all;
    all += lds[w];
  }
  return base + x - v;
}

// How many pages of a wave's run are free: refs counts all references but those to fresh pages.
struct Run {
  int begin, stop;
  __device__ __forceinline__ explicit Run(int pages) {
    const int each = (pages + kScanThreads - 1) / kScanThreads * kWave;
    begin = uniform((int32_t)(threadIdx.x / kWave)) * each;
    stop = begin + each < pages ? begin + each : pages;
  }
  __device__ __forceinline__ uint32_t count(const int32_t* refs, int lane) const {
    uint32_t n = 0;
    for (int p = begin; p < stop; p += kWave) n += __popcll(__ballot(p + lane < stop && refs[p + lane] == 0));
    return n;
  }
  // The first `given` free pages of all, from the at-th on, and the counts of what is handed out.
  __device__ __forceinline__ void give(int32_t* refs, int32_t* fresh, int64_t at, int64_t given, int lane) const {
    for (int p = begin; p < stop && at < given; p += kWave) {
      const bool free = p + lane < stop && refs[p + lane] == 0;
      const uint64_t who = __ballot(free);
      const int64_t rank = at + __popcll(who & (((uint64_t)1 << lane) - 1));
      if (free && rank < given) fresh[rank] = p + lane, refs[p + lane] = 1;
      at += __popcll(who);
    }
  }
};

// What a row gets, which needs `need` fresh pages after `from` of the rows before it, of `many`.  Rows that get some come first among those that need some.
__device__ __forceinline__ bool serve(const ForkParams& a, int b, const Child& c, int64_t from, int64_t many) {
  const int need = c.after - c.kept;
  const bool served = need == 0 || from + need <= many;
  a.child[b].base = need == 0 ? 0 : served ? (int32_t)from : -1;
  a.lens_out[b] = served ? c.len : 0;
  if (!served && a.r.status != nullptr) a.r.status[b] = KVH_DEV_NO_PAGES;
  return served;
}
__device__ __forceinline__ void note_copy(const ForkParams& a, const Child& c, int64_t pair, int64_t from) {
  a.src[pair] = a.r.table[(int64_t)c.parent * a.r.ts + c.full];
  a.dst[pair] = a.fresh[from];
}

__global__ __launch_bounds__(kScanThreads) void hand_out_kernel(ForkParams a) {
  __shared__ int64_t lds[kScanWaves];
  const RowsParams& r = a.r;
  const int lane = threadIdx.x % kWave;
  const Run run(r.pages);
  const uint32_t mine = run.count(r.refs_out, lane);
  int64_t many, wanted = 0, given = 0, all;
  const int64_t at = before_me(lane == 0 ? mine : 0, lds, many) - (lane == 0 ? 0 : mine);
  for (int b0 = 0; b0 < r.n; b0 += kScanThreads) {
    const int b = b0 + threadIdx.x;
    Child c{};
    if (b < r.n) c = a.child[b];
    const int need = c.after - c.kept;
    const int64_t from = wanted + before_me(need, lds, all);
    wanted += all;
    const bool served = b < r.n && serve(a, b, c, from, many);
    before_me(served ? need : 0, lds, all);
    given += all;
  }
  run.give(r.refs_out, a.fresh, at, given, lane);
  __syncthreads();
  int64_t pairs = 0;
  for (int b0 = 0; b0 < r.n; b0 += kScanThreads) {
    const int b = b0 + threadIdx.x;
    Child c{};
    if (b < r.n) c = a.child[b];
    const bool copies = c.copies && c.base >= 0;
    const int64_t pair = pairs + before_me(copies, lds, all);
    if (copies) note_copy(a, c, pair, c.base);
    pairs += all;
  }
  if (threadIdx.x == 0) *a.pairs = (int32_t)pairs;
}

// All of that by one block, with the counts in LDS, for kScanThreads rows at most: thread b has row b.
struct PlanRow {
  int32_t parent, limit;  // whose entries are looked at, and how many
  int32_t len, kept;
  int32_t first, odd;     // of its own children, the first one; whether an entry is none of the cache's
};

__global__ __launch_bounds__(kScanThreads) void plan_kernel(ForkParams a) {
  __shared__ uint32_t free_of[kScanWaves], need_of[kScanWaves], given_of[kScanWaves], copies_of[kScanWaves];
  extern __shared__ int32_t plan_lds[];
  const RowsParams& r = a.r;
  PlanRow* rows = reinterpret_cast<PlanRow*>(plan_lds);
  int32_t* refs = plan_lds + r.n * (int)(sizeof(PlanRow) / sizeof(int32_t));
  const int lane = threadIdx.x % kWave, wave = uniform((int32_t)(threadIdx.x / kWave)), b = threadIdx.x;
  const bool real = b < r.n;
  Child c{};
  int tokens = 0;
  bool open = false;
  if (real) {
    rows[b].first = INT32_MAX, rows[b].odd = 0;
    rows[b].len = r.lens[b];
    c = child_of(a, b, tokens, open);
    rows[b].parent = c.parent;
    rows[b].limit = c.ok && c.parent >= 0 ? c.full + open : 0;
  }
#pragma unroll 4
  for (int p = threadIdx.x; p < r.pages; p += kScanThreads) refs[p] = r.refs[p];
  __syncthreads();
  if (real && c.ok && c.parent >= 0) atomicMin(&rows[c.parent].first, b);  // (what a child that is refused here would keep is not kept, and may be handed out)
  for (int i = wave; i < r.n; i += kScanWaves) {
    const int limit = uniform(rows[i].limit);
    const int32_t* from = r.table + (int64_t)uniform(rows[i].parent) * r.ts;
    bool odd = false;
#pragma unroll 8
    for (int j = lane; j < limit; j += kWave) odd |= (uint32_t)from[j] >= (uint32_t)r.pages;
    if (odd) rows[i].odd = 1;
  }
  __syncthreads();
  if (real) {
    settle(a, b, c, open, rows[b].odd != 0, c.parent >= 0 && c.parent < r.n && rows[c.parent].first < b);
    rows[b].kept = c.kept;
  }
  __syncthreads();
  for (int i = wave; i < r.n; i += kScanWaves) {
    const int kept = uniform(rows[i].kept), len = uniform(rows[i].len), parent = uniform(rows[i].parent);
    count_row<kWave>(r, i, len, kept > 0 ? parent : -1, kept, refs, lane);
  }
  const int need = c.after - c.kept;
  uint32_t sum;
  const uint32_t before = wave_sum_to((uint32_t)need, sum) - (uint32_t)need;
  __syncthreads();
  const Run run(r.pages);
  const uint32_t mine = run.count(refs, lane);
  if (lane == 0) free_of[wave] = mine, need_of[wave] = sum;
  __syncthreads();
  const uint32_t frees = lane < kScanWaves ? free_of[lane] : 0, needs = lane < kScanWaves ? need_of[lane] : 0;
  const uint32_t many = row_sum(frees), at = row_sum(lane < wave ? frees : 0), from = row_sum(lane < wave ? needs : 0) + before;
  const bool served = real && serve(a, b, c, from, many);
  const uint32_t most = wave_max(served && need != 0 ? from + need : 0);
  const uint64_t copying = __ballot(served && c.copies);
  if (lane == 0) given_of[wave] = most, copies_of[wave] = __popcll(copying);
  __syncthreads();
  run.give(refs, a.fresh, at, wave_max(lane < kScanWaves ? given_of[lane] : 0), lane);
  const uint32_t copies = lane < kScanWaves ? copies_of[lane] : 0, earlier = row_sum(lane < wave ? copies : 0), pairs = row_sum(copies);
  __syncthreads();
  if (served && c.copies) note_copy(a, c, earlier + __popcll(copying & (((uint64_t)1 << lane) - 1)), from);
  if (threadIdx.x == 0) *a.pairs = (int32_t)pairs;
#pragma unroll 4
  for (int p = threadIdx.x; p < r.pages; p += kScanThreads) r.refs_out[p] = refs[p];
}

// The rows, by the first n blocks, and the copies.
__global__ __launch_bounds__(kBlockThreads) void rows_kernel(ForkParams a, CopyParams copy) {
  const RowsParams& r = a.r;
  if (blockIdx.x >= (uint32_t)r.n) return copy_many(copy, a.pairs, r.n);
  const int b = blockIdx.x;
  const Child c = a.child[b];
  const bool served = c.base >= 0;
  const int32_t* from = r.table + (int64_t)(c.parent < 0 || !c.ok ? 0 : c.parent) * r.ts;
  int32_t* to = r.table_out + (int64_t)b * r.to_ts;
#pragma unroll 4
  for (int j = threadIdx.x; j < r.table_pages; j += kBlockThreads) {
    int page = -1;
    if (j < c.kept) {
      page = from[j];
      if (!served) {
        atomicSub(&r.refs_out[page], 1);
        page = -1;
      }
    } else if (j < c.after && served) {
      page = a.fresh[c.base + j - c.kept];
    }
    to[j] = page;
  }
}

// ---- compacting ---------------------------------------------------------------------------------------------------
struct CompactParams {
  RowsParams r;
  int32_t* moved;
  int32_t *src, *dst;  // pairs to copy, pages / 2 of them at most, and how many
  int32_t* pairs;
};

// By one block: with U pages in use, the free ones below U and those in use from U on are as many, and go together in order.
__global__ __launch_bounds__(kScanThreads) void place_kernel(CompactParams a) {
  __shared__ uint32_t used_of[kScanWaves], below_of[kScanWaves];
  const RowsParams& r = a.r;
  const int lane = threadIdx.x % kWave, wave = uniform((int32_t)(threadIdx.x / kWave));
  const Run run(r.pages);
  auto in_use = [&](int p) { return p + lane < run.stop && r.refs[p + lane] > 0; };
  uint32_t mine = 0;
  for (int p = run.begin; p < run.stop; p += kWave) mine += __popcll(__ballot(in_use(p)));
  if (lane == 0) used_of[wave] = mine;
  __syncthreads();
  uint32_t of = lane < kScanWaves ? used_of[lane] : 0;
  const int used = (int)row_sum(of);
  uint32_t before = row_sum(lane < wave ? of : 0);  // pages in use before the run's next ones
  uint32_t below = 0;
  for (int p = run.begin; p < run.stop; p += kWave) below += __popcll(__ballot(in_use(p) && p + lane < used));
  if (lane == 0) below_of[wave] = below;
  __syncthreads();
  of = lane < kScanWaves ? below_of[lane] : 0;
  const int stay = (int)row_sum(of), strays = used - stay;
  const uint64_t under = ((uint64_t)1 << lane) - 1;
  for (int p0 = run.begin; p0 < run.stop; p0 += kWave) {
    const int p = p0 + lane;
    const bool is = in_use(p0);
    const uint64_t who = __ballot(is);
    const int rank = (int)(before + __popcll(who & under));  // pages in use before it
    before += __popcll(who);
    if (p >= run.stop) continue;
    if (is && p >= used) a.src[rank - stay] = p;
    if (!is && p < used) a.dst[p - rank] = p;
    a.moved[p] = is ? p : -1;
    r.refs_out[p] = is ? r.refs[p] : 0;
  }
  if (threadIdx.x == 0) *a.pairs = strays;
  __syncthreads();
  for (int i = threadIdx.x; i < strays; i += kScanThreads) {
    const int src = a.src[i], dst = a.dst[i];
    a.moved[src] = dst;
    r.refs_out[dst] = r.refs[src];
    r.refs_out[src] = 0;
  }
}

// The rows, by the first n blocks, and the copies.
__global__ __launch_bounds__(kBlockThreads) void renumber_kernel(CompactParams a, CopyParams copy) {
  const RowsParams& r = a.r;
  if (blockIdx.x >= (uint32_t)r.n) return copy_many(copy, a.pairs, r.n);
  const int b = blockIdx.x;
  const int32_t len = r.lens[b];
  bool bad = len < 0 || len > r.capacity;
  const int held = bad ? 0 : pages_of(r, len);
  const int32_t* from = r.table + (int64_t)b * r.ts;
  int32_t* to = r.table_out + (int64_t)b * r.to_ts;
#pragma unroll 4
  for (int j = threadIdx.x; j < r.table_pages; j += kBlockThreads) {
    int page = -1;
    if (j < held) {
      page = from[j];
      page = (uint32_t)page < (uint32_t)r.pages ? a.moved[page] : -1;
      bad |= page < 0;
    }
    to[j] = page;
  }
  if (bad && r.status != nullptr) r.status[b] = KVH_DEV_BAD_REQUEST;
}

// One block plans by itself where the counts and rows fit into its LDS and the table has no more entries than this, whatever they hold: 64 rows, 14895 pages 14.5 us, in three launches 39.
constexpr int64_t kPlanLds = 63 << 10, kPlanEntries = 512 << 10;

// ---- arguments ----------------------------------------------------------------------------------------------------
bool aligned4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }

int rows_params(const kvh_cache* cache, const kvh_bounds* bounds, const kvh_rows_of_pages* rows, int32_t* status, RowsParams& r) {
  if (int rc = check_cache(cache)) return rc;
  if (bounds != nullptr)
    if (int rc = check_bounds_of(bounds, cache)) return rc;
  if (rows == nullptr || rows->table == nullptr || rows->table_out == nullptr || rows->lens == nullptr || rows->refs == nullptr || rows->refs_out == nullptr) return KVH_E_ARG;
  if (rows->n_requests < 1 || rows->n_requests > kMaxRequests || rows->table_pages < 1) return KVH_E_ARG;
  const int64_t least = rows->n_requests > 1 ? rows->table_pages : 0;
  if (rows->table_stride < least || rows->table_out_stride < least) return KVH_E_ARG;
  if (rows->table == rows->table_out || rows->refs == rows->refs_out) return KVH_E_ARG;
  if (!aligned4(rows->table) || !aligned4(rows->table_out) || !aligned4(rows->lens) || !aligned4(rows->refs) || !aligned4(rows->refs_out)) return KVH_E_ALIGN;
  r.table = rows->table, r.table_out = rows->table_out;
  r.ts = rows->table_stride, r.to_ts = rows->table_out_stride;
  r.lens = rows->lens, r.refs = rows->refs, r.refs_out = rows->refs_out;
  r.table_pages = rows->table_pages, r.n = rows->n_requests, r.pages = cache->pages, r.block_tokens = cache->block_tokens;
  r.capacity = std::min<int64_t>((int64_t)rows->table_pages * cache->block_tokens, kMaxLength);
  r.status = status;
  r.by_block = Divisor((uint32_t)cache->block_tokens);
  return KVH_OK;
}

}  // namespace
}  // namespace kvh

using namespace kvh;

extern "C" {

int kvh_copy_pages(const kvh_cache* cache, const kvh_bounds* bounds, const int32_t* src_dev, const int32_t* dst_dev, int n, int32_t* status_dev, void* stream) {
  if (int rc = check_cache(cache)) return rc;
  if (bounds != nullptr)
    if (int rc = check_bounds_of(bounds, cache)) return rc;
  if (n < 0 || n > 1 << 24 || (n > 0 && (src_dev == nullptr || dst_dev == nullptr))) return KVH_E_ARG;
  if (!aligned4(src_dev) || !aligned4(dst_dev)) return KVH_E_ALIGN;
  CopyParams a{};
  if (int rc = copy_params(*cache, bounds, src_dev, dst_dev, n, status_dev, a)) return rc;
  return launch_copy(a, n, static_cast<hipStream_t>(stream));
}

size_t kvh_fork_workspace(int n_requests, int pages) {
  if (n_requests < 1 || n_requests > kMaxRequests || pages < 1) return 0;
  return (size_t)n_requests * (sizeof(Child) + 2 * sizeof(int32_t)) + ((size_t)pages + 1) * sizeof(int32_t);
}

int kvh_fork(const kvh_cache* cache, const kvh_bounds* bounds, const kvh_rows_of_pages* rows, const int32_t* parents_dev, const int32_t* grow_dev,
             int32_t* lens_out_dev, void* workspace_dev, size_t workspace_bytes, int32_t* status_dev, void* stream) {
  ForkParams a{};
  if (int rc = rows_params(cache, bounds, rows, status_dev, a.r)) return rc;
  if (lens_out_dev == nullptr || lens_out_dev == rows->lens || workspace_dev == nullptr) return KVH_E_ARG;
  if (!aligned4(lens_out_dev) || !aligned4(parents_dev) || !aligned4(grow_dev) || !aligned4(workspace_dev)) return KVH_E_ALIGN;
  if (workspace_bytes < kvh_fork_workspace(a.r.n, a.r.pages)) return KVH_E_SIZE;
  a.parents = parents_dev, a.grow = grow_dev, a.lens_out = lens_out_dev;
  a.child = static_cast<Child*>(workspace_dev);
  a.src = reinterpret_cast<int32_t*>(a.child + a.r.n), a.dst = a.src + a.r.n, a.pairs = a.dst + a.r.n, a.fresh = a.pairs + 1;
  CopyParams copy{};
  if (int rc = copy_params(*cache, bounds, a.src, a.dst, 0, nullptr, copy)) return rc;
  hipStream_t s = static_cast<hipStream_t>(stream);
  const int64_t lds = (int64_t)a.r.pages * sizeof(int32_t) + (int64_t)a.r.n * sizeof(PlanRow);
  if (a.r.n <= kScanThreads && lds <= kPlanLds && (int64_t)a.r.n * a.r.table_pages <= kPlanEntries) {
    launch_kernel(plan_kernel, dim3(1), dim3(kScanThreads), (unsigned)lds, s, a);
    KVH_HIP_CHECK_LAUNCH();
  } else {
    launch_kernel(start_kernel, dim3((unsigned)(((int64_t)a.r.pages + kBlockThreads - 1) / kBlockThreads)), dim3(kBlockThreads), 0, s, a.r);
    KVH_HIP_CHECK_LAUNCH();
    hipLaunchKernelGGL(count_kernel, dim3((unsigned)a.r.n), dim3(kBlockThreads), 0, s, a);
    KVH_HIP_CHECK_LAUNCH();
    hipLaunchKernelGGL(hand_out_kernel, dim3(1), dim3(kScanThreads), 0, s, a);
    KVH_HIP_CHECK_LAUNCH();
  }
  hipLaunchKernelGGL(rows_kernel, dim3((unsigned)(a.r.n + std::min(a.r.n * copy.each(), kForkBlocks))), dim3(kBlockThreads), 0, s, a, copy);
  KVH_HIP_CHECK_LAUNCH();
  return KVH_OK;
}

size_t kvh_compact_workspace(int pages) { return pages < 1 ? 0 : (size_t)(2 * ((int64_t)pages / 2) + 1) * sizeof(int32_t); }

int kvh_compact(const kvh_cache* cache, const kvh_bounds* bounds, const kvh_rows_of_pages* rows, int32_t* moved_out_dev, void* workspace_dev,
                size_t workspace_bytes, int32_t* status_dev, void* stream) {
  CompactParams a{};
  if (int rc = rows_params(cache, bounds, rows, status_dev, a.r)) return rc;
  if (moved_out_dev == nullptr || workspace_dev == nullptr) return KVH_E_ARG;
  if (!aligned4(moved_out_dev) || !aligned4(workspace_dev)) return KVH_E_ALIGN;
  if (workspace_bytes < kvh_compact_workspace(a.r.pages)) return KVH_E_SIZE;
  a.moved = moved_out_dev;
  a.pairs = static_cast<int32_t*>(workspace_dev), a.src = a.pairs + 1, a.dst = a.src + a.r.pages / 2;
  CopyParams copy{};
  if (int rc = copy_params(*cache, bounds, a.src, a.dst, a.r.pages / 2, nullptr, copy)) return rc;
  hipStream_t s = static_cast<hipStream_t>(stream);
  launch_kernel(place_kernel, dim3(1), dim3(kScanThreads), 0, s, a);
  KVH_HIP_CHECK_LAUNCH();
  const int64_t copies = std::min(a.r.pages / 2 * copy.each(), kCompactBlocks);
  hipLaunchKernelGGL(renumber_kernel, dim3((unsigned)(a.r.n + copies)), dim3(kBlockThreads), 0, s, a, copy);
  KVH_HIP_CHECK_LAUNCH();
  return KVH_OK;
}

}  // extern "C"
