// Pages of the cache: room for new tokens, rows taken over from others, pages moved to the front.  Decided by one workgroup on the
// device, so that no call waits for the host; what is copied is copied by a second launch over the whole chip.  Bound by latency where little is copied
// (32 rows of 33 blocks: reorder 3.0 us, reserve 7.6, 28 copies of 131 KB 4.8) and by memory where much is (1600 pages of 262 KB moved: 159 us, 5.3 TB/s).
#include "cache.hpp"
#include "cafeq_internal.hpp"

namespace cafeq {
namespace {

constexpr int kScan = 1024, kCopy = 256;
constexpr int64_t kSmallTable = 16384;      // words of LDS (64 KB) with which one workgroup reorders a table in one launch

// Scratch of all three calls, int32 throughout
struct PageWs {
  int32_t *head, *list, *list2, *map, *table, *lengths, *from, *to, *base;
};
size_t page_ws_ints(const cafeq_cache& c) { return 64 + 3 * size_t(c.pages) + size_t(c.sequences) * c.width + 4 * size_t(c.sequences); }
PageWs page_ws(const cafeq_cache& c, void* ws) {
  PageWs w;
  int32_t* p = static_cast<int32_t*>(ws);
  auto take = [&p](size_t n) { int32_t* q = p; p += n; return q; };
  w.head = take(64);
  w.list = take(c.pages);
  w.list2 = take(c.pages);
  w.map = take(c.pages);
  w.lengths = take(c.sequences);
  w.from = take(c.sequences);
  w.to = take(c.sequences);
  w.base = take(c.sequences);
  w.table = take(size_t(c.sequences) * c.width);
  return w;
}

// Sum of v over the threads before this one; total: over all of the workgroup
__device__ int scan_before(int v, int* total) {
  __shared__ int sums[kScan / 64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int s = v;
  for (int k = 1; k < 64; k <<= 1) {
    const int o = __shfl_up(s, k);
    if (lane >= k) s += o;
  }
  __syncthreads();          // the last call's sums have been read
  if (lane == 63) sums[wave] = s;
  __syncthreads();
  int before = 0, all = 0;
  for (int k = 0; k < kScan / 64; ++k) {
    if (k < wave) before += sums[k];
    all += sums[k];
  }
  *total = all;
  return before + s - v;
}

struct ReserveArgs {
  cafeq_cache c;
  PageWs w;
  const int32_t* starts;
  int n;
  int32_t *positions, *missing;
};

__device__ __forceinline__ int blocks_of(int64_t tokens, int B) { return int((tokens + B - 1) / B); }

__global__ __launch_bounds__(kScan) void reserve_kernel(const ReserveArgs a) {
  const cafeq_cache& c = a.c;
  const int tid = threadIdx.x, B = c.block;
  int want = 0, over = 0;
  for (int i0 = 0; i0 < c.sequences; i0 += kScan) {
    const int i = i0 + tid;
    int count = 0, beyond = 0;
    if (i < c.sequences) {
      const RowRange r = rows_of(a.starts, i, a.n);
      const int len = tokens_of(c, i), more = r.hi - r.lo, have = blocks_of(len, B), need = blocks_of(int64_t(len) + more, B);
      const int last = have > 0 ? page_of(c, i, have - 1) : -1;
      const bool copy = more > 0 && len % B && last >= 0 && c.refs[last] > 1;
      beyond = max(0, need - c.width);
      count = min(need, c.width) - have + (copy ? 1 : 0);
      a.w.from[i] = copy ? last : -1;
    }
    int total;
    const int before = scan_before(count, &total);
    if (i < c.sequences) a.w.base[i] = want + before;
    want += total;
    scan_before(beyond, &total);
    over += total;
  }
  // the lowest free pages, as many as are wanted
  int found = 0;
  for (int64_t p0 = 0; p0 < c.pages && found < want && over == 0; p0 += 4 * kScan) {
    int free = 0;
    bool is[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int64_t p = p0 + 4 * tid + e;
      is[e] = p < c.pages && c.refs[p] == 0;
      free += is[e];
    }
    int total, at = found + scan_before(free, &total);
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (is[e] && at < want) a.w.list[at++] = int(p0 + 4 * tid + e);
    found += total;
  }
  const int lack = over > 0 ? over : max(0, want - found);
  if (tid == 0) {
    *a.missing = lack;
    if (c.missing) *c.missing = lack;
    a.w.head[0] = lack;
  }
  if (lack) return;
  __syncthreads();
  // a wave a sequence
  for (int i = tid >> 6; i < c.sequences; i += kScan / 64) {
    const int lane = tid & 63;
    const RowRange r = rows_of(a.starts, i, a.n);
    const int len = tokens_of(c, i), more = r.hi - r.lo, have = blocks_of(len, B), need = blocks_of(int64_t(len) + more, B);
    int32_t* row = c.table + int64_t(i) * c.width;
    const int32_t* list = a.w.list + a.w.base[i];
    const int from = a.w.from[i], extra = from >= 0 ? 1 : 0;
    if (extra && lane == 0) {
      a.w.to[i] = list[0];
      row[have - 1] = list[0];
      c.refs[list[0]] = 1;
      atomicSub(c.refs + from, 1);
    }
    for (int e = lane; e < need - have; e += 64) {
      row[have + e] = list[extra + e];
      c.refs[list[extra + e]] = 1;
    }
    // the wave has read the length before it is written: its lanes run in step
    if (lane == 0 && more > 0) c.lengths[i] = len + more;
  }
}

// One page and head, keys or values (item = 2 head + side), of `bytes` bytes
__device__ __forceinline__ void copy_item(const cafeq_cache& c, int from, int to, int item) {
  const int head = item >> 1, bytes = c.block * c.d;
  int8_t* base = item & 1 ? c.v : c.k;
  float* scale = item & 1 ? c.vscale : c.kscale;
  const int64_t src = int64_t(from) * c.heads + head, dst = int64_t(to) * c.heads + head;
  const uint4* s = reinterpret_cast<const uint4*>(base + src * bytes);
  uint4* t = reinterpret_cast<uint4*>(base + dst * bytes);
  for (int e = threadIdx.x; e < bytes / 16; e += kCopy) t[e] = s[e];
  if (threadIdx.x == 0) scale[dst] = scale[src];
}

// The second part of reserve: positions of the new tokens, and copies
__global__ __launch_bounds__(kCopy) void copy_shared_kernel(const ReserveArgs a) {
  const cafeq_cache& c = a.c;
  const PageWs& w = a.w;
  const int i = blockIdx.x;
  const bool lack = w.head[0] != 0;
  if (a.positions) {
    const RowRange r = rows_of(a.starts, i, a.n);
    const int before = c.lengths[i] - (r.hi - r.lo);
    for (int e = r.lo + blockIdx.y * kCopy + threadIdx.x; e < r.hi; e += gridDim.y * kCopy) a.positions[e] = lack ? 0 : before + (e - r.lo);
  }
  if (lack || w.from[i] < 0) return;
  for (int item = blockIdx.y; item < 2 * c.heads; item += gridDim.y) copy_item(c, w.from[i], w.to[i], item);
}

__global__ __launch_bounds__(kCopy) void keep_table_kernel(const cafeq_cache c, const PageWs w) {
  const int64_t total = int64_t(c.sequences) * c.width, step = int64_t(gridDim.x) * kCopy, id = int64_t(blockIdx.x) * kCopy + threadIdx.x;
  for (int64_t e = id; e < total; e += step) w.table[e] = c.table[e];
  for (int64_t e = id; e < c.sequences; e += step) w.lengths[e] = tokens_of(c, int(e));
}

__global__ __launch_bounds__(kCopy) void reorder_kernel(const cafeq_cache c, const PageWs w, const int32_t* sources) {
  const int i = blockIdx.x, from = sources[i], B = c.block;
  if (from == i) return;
  const bool some = from >= 0 && from < c.sequences;
  const int len = some ? w.lengths[from] : 0, blocks = blocks_of(len, B), old = blocks_of(w.lengths[i], B);
  const int32_t* src = w.table + int64_t(some ? from : 0) * c.width;
  const int32_t* mine = w.table + int64_t(i) * c.width;
  int32_t* row = c.table + int64_t(i) * c.width;
  for (int b = threadIdx.x; b < c.width; b += kCopy) {
    const int p = b < blocks ? src[b] : -1, q = b < old ? mine[b] : -1;
    row[b] = p;
    if (p >= 0 && p < c.pages) atomicAdd(c.refs + p, 1);
    if (q >= 0 && q < c.pages) atomicSub(c.refs + q, 1);
  }
  if (threadIdx.x == 0) c.lengths[i] = len;
}

// The same for a table that LDS holds: one workgroup, one launch.
__global__ __launch_bounds__(kScan) void reorder_small_kernel(const cafeq_cache c, const int32_t* sources) {
  extern __shared__ int32_t held[];      // the table, then blocks of the rows, lengths and sources
  const int tid = threadIdx.x, total = c.sequences * c.width, B = c.block;
  int32_t *blocks = held + total, *lengths = blocks + c.sequences, *from = lengths + c.sequences;
  for (int e = tid; e < total; e += kScan) held[e] = c.table[e];
  for (int e = tid; e < c.sequences; e += kScan) {
    lengths[e] = tokens_of(c, e);
    blocks[e] = blocks_of(lengths[e], B);
    const int s = sources[e];
    from[e] = s >= 0 && s < c.sequences ? s : -1;
  }
  __syncthreads();
  // a wave a row
  for (int i = tid >> 6; i < c.sequences; i += kScan / 64) {
    const int s = from[i];
    if (s == i) continue;
    const int mine = blocks[i], theirs = s < 0 ? 0 : blocks[s];
    for (int b = tid & 63; b < c.width; b += 64) {
      const int p = b < theirs ? held[s * c.width + b] : -1, q = b < mine ? held[i * c.width + b] : -1;
      c.table[i * c.width + b] = p;
      if (p >= 0 && p < c.pages) atomicAdd(c.refs + p, 1);
      if (q >= 0 && q < c.pages) atomicSub(c.refs + q, 1);
    }
    if ((tid & 63) == 0) c.lengths[i] = s < 0 ? 0 : lengths[s];
  }
}

__global__ __launch_bounds__(kScan) void plan_compact_kernel(const cafeq_cache c, const PageWs w, int32_t* used) {
  const int tid = threadIdx.x;
  int count = 0, total;
  for (int64_t p = tid; p < c.pages; p += kScan) {
    count += c.refs[p] > 0;
    w.map[p] = int(p);
  }
  scan_before(count, &total);
  const int in_use = total;
  int moves = 0, holes = 0;
  for (int64_t p0 = 0; p0 < c.pages; p0 += 4 * kScan) {
    int move = 0, hole = 0;      // of the thread's four pages, by bits
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int64_t p = p0 + 4 * tid + e;
      const bool live = p < c.pages && c.refs[p] > 0;
      move |= int(live && p >= in_use) << e;
      hole |= int(p < in_use && !live) << e;
    }
    // both counts in one sum: a step has at most 4096 of either
    const int before = scan_before(__popc(move) | __popc(hole) << 16, &total);
    int at = moves + (before & 0xFFFF), to = holes + (before >> 16);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if (move >> e & 1) w.list[at++] = int(p0 + 4 * tid + e);
      if (hole >> e & 1) w.list2[to++] = int(p0 + 4 * tid + e);
    }
    moves += total & 0xFFFF;
    holes += total >> 16;
  }
  if (tid == 0) {
    *used = in_use;
    w.head[0] = moves;
  }
  __syncthreads();
  for (int e = tid; e < moves; e += kScan) {
    const int from = w.list[e], to = w.list2[e];
    w.map[from] = to;
    c.refs[to] = c.refs[from];
    c.refs[from] = 0;
  }
}

__global__ __launch_bounds__(kCopy) void compact_kernel(const cafeq_cache c, const PageWs w) {
  const int64_t total = int64_t(c.sequences) * c.width, step = int64_t(gridDim.x) * kCopy;
  const int moves = w.head[0];
  if (moves)
    for (int64_t e = int64_t(blockIdx.x) * kCopy + threadIdx.x; e < total; e += step) {
      const int p = c.table[e];
      if (p >= 0 && p < c.pages && w.map[p] != p) c.table[e] = w.map[p];
    }
  const int64_t items = int64_t(moves) * 2 * c.heads;
  for (int64_t x = blockIdx.x; x < items; x += gridDim.x) {
    const int e = int(x / (2 * c.heads));
    copy_item(c, w.list[e], w.list2[e], int(x % (2 * c.heads)));
  }
}

int check_pages(const cafeq_cache* c, const void* ws) {
  const int rc = check_cache(c);
  if (rc) return rc;
  if (!c->refs) return CAFEQ_ERR_INVALID_ARG;
  if (!ws) return CAFEQ_ERR_WORKSPACE;
  return aligned_to(ws, 16) ? CAFEQ_OK : CAFEQ_ERR_BAD_ALIGN;
}

}  // namespace
}  // namespace cafeq

using namespace cafeq;

extern "C" {

size_t cafeq_cache_pages_workspace_bytes(const cafeq_cache* cache) {
  return check_cache(cache) ? 0 : align_up(page_ws_ints(*cache) * sizeof(int32_t), 256);
}

int cafeq_cache_reserve(const cafeq_cache* cache, const int32_t* starts, int64_t n, int32_t* positions, int32_t* missing, void* ws,
                        void* stream) {
  const int rc = check_pages(cache, ws);
  if (rc) return rc;
  if (!starts || !missing) return CAFEQ_ERR_INVALID_ARG;
  if (n < 0) return CAFEQ_ERR_BAD_SHAPE;
  if (n > (int64_t(1) << 24)) return CAFEQ_ERR_UNSUPPORTED;
  if (!aligned_to(starts, 4) || !aligned_to(positions, 4) || !aligned_to(missing, 4)) return CAFEQ_ERR_BAD_ALIGN;
  hipStream_t st = static_cast<hipStream_t>(stream);
  const ReserveArgs a{*cache, page_ws(*cache, ws), starts, int(n), positions, missing};
  hipLaunchKernelGGL(reserve_kernel, dim3(1), dim3(kScan), 0, st, a);
  CAFEQ_CHECK_LAUNCH();
  if (cache->sequences == 0 || n == 0) return CAFEQ_OK;
  const int y = std::max(1, std::min(2 * cache->heads, 65536 / std::max(1, cache->sequences)));
  hipLaunchKernelGGL(copy_shared_kernel, dim3(unsigned(cache->sequences), unsigned(y)), dim3(kCopy), 0, st, a);
  CAFEQ_CHECK_LAUNCH();
  return CAFEQ_OK;
}

int cafeq_cache_reorder(const cafeq_cache* cache, const int32_t* sources, void* ws, void* stream) {
  const int rc = check_pages(cache, ws);
  if (rc) return rc;
  if (cache->sequences == 0) return CAFEQ_OK;
  if (!sources) return CAFEQ_ERR_INVALID_ARG;
  if (!aligned_to(sources, 4)) return CAFEQ_ERR_BAD_ALIGN;
  hipStream_t st = static_cast<hipStream_t>(stream);
  const PageWs w = page_ws(*cache, ws);
  const int64_t entries = int64_t(cache->sequences) * cache->width;
  const int64_t words = entries + 3 * int64_t(cache->sequences);
  if (words <= kSmallTable) {
    hipLaunchKernelGGL(reorder_small_kernel, dim3(1), dim3(kScan), size_t(words) * sizeof(int32_t), st, *cache, sources);
    CAFEQ_CHECK_LAUNCH();
    return CAFEQ_OK;
  }
  hipLaunchKernelGGL(keep_table_kernel, dim3(unsigned(std::min<int64_t>(1024, (entries + kCopy - 1) / kCopy))), dim3(kCopy), 0, st, *cache, w);
  CAFEQ_CHECK_LAUNCH();
  hipLaunchKernelGGL(reorder_kernel, dim3(unsigned(cache->sequences)), dim3(kCopy), 0, st, *cache, w, sources);
  CAFEQ_CHECK_LAUNCH();
  return CAFEQ_OK;
}

int cafeq_cache_compact(const cafeq_cache* cache, int32_t* used, void* ws, void* stream) {
  const int rc = check_pages(cache, ws);
  if (rc) return rc;
  if (!used) return CAFEQ_ERR_INVALID_ARG;
  if (!aligned_to(used, 4)) return CAFEQ_ERR_BAD_ALIGN;
  hipStream_t st = static_cast<hipStream_t>(stream);
  const PageWs w = page_ws(*cache, ws);
  hipLaunchKernelGGL(plan_compact_kernel, dim3(1), dim3(kScan), 0, st, *cache, w, used);
  CAFEQ_CHECK_LAUNCH();
  const int64_t items = std::max<int64_t>(cache->pages * 2 * cache->heads, (int64_t(cache->sequences) * cache->width + kCopy - 1) / kCopy);
  hipLaunchKernelGGL(compact_kernel, dim3(unsigned(std::min<int64_t>(8 * device_cu_count(), items))), dim3(kCopy), 0, st, *cache, w);
  CAFEQ_CHECK_LAUNCH();
  return CAFEQ_OK;
}

}  // extern "C"
