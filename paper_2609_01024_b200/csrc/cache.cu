// Page operations of a paged key/value cache: reserve (grow, copy on write), write, fork, keep, trim, compact.
//
// All bookkeeping lives on the device (lengths, reference counts, page tables), so a serving loop that reserves, forks,
// drops and compacts never waits for the host and can be recorded into a graph.  A page is free iff its reference count
// is zero and allocation takes the lowest free ids in call order: there is no free list whose order would depend on
// history, and every result is a function of the arguments alone.
//
// What bounds them: the bookkeeping is a chain of a few dependent loads (latency); the data movement is a copy, each
// moved row read and written once (HBM).  So the bookkeeping of a call is one block where an order over the call's
// sequences is needed (reserve, compact) and a block per sequence elsewhere, and the copies that follow are spread over
// the whole GPU by a second launch that finds its list in the workspace.  Measured (cold caches): reserving for 8
// sequences 8 us; writing 10 MB of new rows 10 us; compaction that moves 97 MB of pages 30 us, 6.4 TB/s read and
// written; accepting up to 9 drafts in each of 8 sequences 13 us.  In a steady loop, call by call: reserve 5.7, write 4.4, keep
// 8.3 (two launches), trim 1.6, fork 2.3, compaction of a compact pool 4.1 us.
#include <algorithm>

#include "cache.cuh"

namespace pcomoe {
namespace {

constexpr int kPlanThreads = 1024;

struct CacheWs {
  CacheHeader *head;
  int32_t *src, *dst;             // [max(pages, max_seqs)] page moves
  int32_t *list;                  // [pages] free pages in order / new id of every page
  size_t total;
};

CacheWs cache_ws(const pcomoe_cache *c, void *ws) {
  const size_t cap = (size_t)std::max(c->pages, c->max_seqs);
  const size_t moves = align256(4 * cap), list = align256(4 * (size_t)c->pages);
  char *b = (char *)ws;
  CacheWs w;
  w.head = (CacheHeader *)b;
  w.src = (int32_t *)(b + 256);
  w.dst = (int32_t *)(b + 256 + moves);
  w.list = (int32_t *)(b + 256 + 2 * moves);
  w.total = 256 + 2 * moves + list;
  return w;
}

// Exclusive prefix over the block's threads; *total gets the sum.  s: 33 ints of shared memory.
__device__ int block_scan(int x, int *s, int *total) {
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
  int y = x;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int z = __shfl_up_sync(~0u, y, o);
    if (lane >= o) y += z;
  }
  if (lane == 31) s[w] = y;
  __syncthreads();
  if (w == 0) {
    const int v = lane < (int)(blockDim.x >> 5) ? s[lane] : 0;
    int t = v;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int z = __shfl_up_sync(~0u, t, o);
      if (lane >= o) t += z;
    }
    s[lane] = t - v;
    if (lane == 31) s[32] = t;
  }
  __syncthreads();
  const int r = s[w] + y - x;
  *total = s[32];
  __syncthreads();
  return r;
}

// One block: how many pages each sequence needs, where the free ones are, and who gets which.
__global__ void __launch_bounds__(kPlanThreads) reserve_plan_kernel(CacheDev c, int n, const int32_t *seqs, const int32_t *add,
                                                                    CacheWs w) {
  pdl_grid_wait();
  __shared__ int s_last[kMaxSeqs];              // the shared, partly filled last page of entry i, or -1
  __shared__ int s_first[kMaxSeqs];             // pages given to the entries before i
  __shared__ uint32_t s_seen[kMaxSeqs / 32], s_copy[kMaxSeqs / 32];
  __shared__ int s_scan[33], s_bad, s_copies;
  const int tid = threadIdx.x, lane = tid & 31, wp = tid >> 5;
  // the free pages of each warp's contiguous run of the reference counts: their loads are under way while the chain list
  // -> length -> table -> count below is followed
  const int run = ((c.pages + 1023) / 1024) * 32;      // pages of a warp, a multiple of 32
  const int lo = min(wp * run, c.pages), hi = min(lo + run, c.pages);
  int mine = 0;
#pragma unroll 4
  for (int p = lo + lane; p < hi; p += 32) mine += c.ref[p] == 0;
  for (int i = tid; i < kMaxSeqs / 32; i += kPlanThreads) s_seen[i] = s_copy[i] = 0;
  if (tid == 0) { s_bad = 0; s_copies = 0; w.head->n_moves = 0; }
  __syncthreads();
  for (int i = tid; i < n; i += kPlanThreads) {
    const int id = seqs[i], a = add[i];
    int last = -1;
    bool bad = id < 0 || id >= c.max_seqs || a < 0;
    if (!bad) {
      bad = (atomicOr(&s_seen[id >> 5], 1u << (id & 31)) >> (id & 31)) & 1u;
      const int have = c.len[id];
      bad |= have < 0 || (int64_t)have + a > (int64_t)c.max_pages * c.page;
      if (!bad && a > 0 && (have & (c.page - 1))) {
        last = c.table[(int64_t)id * c.max_pages + (have >> c.shift)];
        if (last < 0 || last >= c.pages) bad = true;
        else if (c.ref[last] <= 1) last = -1;
      }
    }
    if (bad) s_bad = 1;
    s_last[i] = last;
  }
  __syncthreads();
  if (s_bad) {
    if (tid == 0) flag(w.head, PCOMOE_ERR_INDEX);
    return;
  }
  int total = 0;
  for (int i0 = 0; i0 < n; i0 += kPlanThreads) {
    const int i = i0 + tid;
    int need = 0;
    if (i < n) {
      const int id = seqs[i], have = c.len[id];
      need = min(pages_of(c, have + add[i]) - pages_of(c, have), c.pages + 1);
      const int last = s_last[i];
      if (last >= 0) {
        // sharers earlier in the call have left the page by then; the last holder keeps it
        int before = 0;
        for (int j = 0; j < i; ++j) before += s_last[j] == last;
        if (c.ref[last] - before > 1) {
          ++need;
          atomicOr(&s_copy[i >> 5], 1u << (i & 31));
        }
      }
    }
    int sum;
    const int first = block_scan(need, s_scan, &sum);
    if (i < n) s_first[i] = total + first;
    total += sum;
  }
  // the free pages in order
#pragma unroll
  for (int o = 16; o; o >>= 1) mine += __shfl_xor_sync(~0u, mine, o);
  int free_pages;
  int at = block_scan(lane == 0 ? mine : 0, s_scan, &free_pages);
  at = __shfl_sync(~0u, at, 0);
  if (total > free_pages) {
    if (tid == 0) flag(w.head, PCOMOE_ERR_CACHE_FULL);
    return;
  }
  for (int p0 = lo; p0 < hi && at < total; p0 += 32) {
    const bool is_free = p0 + lane < hi && c.ref[p0 + lane] == 0;
    const uint32_t b = __ballot_sync(~0u, is_free);
    const int r = at + __popc(b & ((1u << lane) - 1));
    if (is_free && r < total) w.list[r] = p0 + lane;
    at += __popc(b);
  }
  __syncthreads();
  for (int r = tid; r < total; r += kPlanThreads) {
    int a = 0, b = n;                                   // the last entry whose pages begin at or before r
    while (b - a > 1) {
      const int m = (a + b) >> 1;
      if (s_first[m] <= r) a = m; else b = m;
    }
    const int id = seqs[a], j = r - s_first[a], page = w.list[r];
    const int copy = (s_copy[a >> 5] >> (a & 31)) & 1;
    c.table[(int64_t)id * c.max_pages + pages_of(c, c.len[id]) - copy + j] = page;
    c.ref[page] = 1;
    if (copy && j == 0) {
      atomicSub(&c.ref[s_last[a]], 1);
      const int k = atomicAdd(&s_copies, 1);
      w.src[k] = s_last[a];
      w.dst[k] = page;
    }
  }
  __syncthreads();
  for (int i = tid; i < n; i += kPlanThreads) c.len[seqs[i]] += add[i];
  if (tid == 0) w.head->n_moves = s_copies;
}

// Whole pages from src to dst in every layer, K and V.  A block moves 16 KB pieces: four 16-byte loads per thread in
// flight before the first store.
constexpr int kPiece = 16384;
template <bool kRemap>
__global__ void __launch_bounds__(256) move_pages_kernel(CacheDev c, CacheWs w) {
  pdl_grid_wait();
  const int n = w.head->n_moves;
  if (kRemap && n) {                                      // the page tables follow the pages
    const int64_t entries = (int64_t)c.max_seqs * c.max_pages;
    for (int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; i < entries; i += (int64_t)gridDim.x * blockDim.x) {
      const int p = c.table[i];
      if (p >= 0 && p < c.pages) c.table[i] = w.list[p];
    }
  }
  const int pieces = (int)((c.page_bytes + kPiece - 1) / kPiece);
  const int64_t units = (int64_t)n * 2 * c.layers * pieces;
  for (int64_t u = blockIdx.x; u < units; u += gridDim.x) {
    const int piece = (int)(u % pieces);
    const int64_t q = u / pieces;
    const int kv = (int)(q & 1), layer = (int)((q >> 1) % c.layers), m = (int)((q >> 1) / c.layers);
    char *pool = (kv ? c.v : c.k) + (int64_t)layer * c.pages * c.page_bytes;
    const char *from = pool + (int64_t)w.src[m] * c.page_bytes;
    char *to = pool + (int64_t)w.dst[m] * c.page_bytes;
    const int64_t base = (int64_t)piece * kPiece + threadIdx.x * 16;
    uint4 x[4];
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (base + k * 4096 < c.page_bytes) x[k] = __ldcs((const uint4 *)(from + base + k * 4096));
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (base + k * 4096 < c.page_bytes) *(uint4 *)(to + base + k * 4096) = x[k];
  }
}

// Rows of K and V into their places: a block takes four rows of one layer and looks the four places up side by side.
constexpr int kWriteRows = 4;
__global__ void __launch_bounds__(256) cache_write_kernel(CacheDev c, int first_layer, int T, int n, const int32_t *seqs,
                                                          const int32_t *cu, const char *k, const char *v, int64_t row_bytes,
                                                          int64_t layer_bytes, CacheHeader *head) {
  pdl_grid_wait();
  __shared__ int s_page[kWriteRows], s_slot[kWriteRows];
  const int t0 = blockIdx.x * kWriteRows, layer = blockIdx.y;
  // positions without a row: they keep what their page held
  if (blockIdx.x == 0 && layer == 0 && threadIdx.x == kWriteRows && (cu[n] > T || cu[0] < 0)) flag(head, PCOMOE_ERR_INDEX);
  if (threadIdx.x < kWriteRows) {
    const int t = t0 + threadIdx.x;
    int page = -1, slot = 0;
    if (t < T && t < cu[n] && t >= cu[0]) {
      int a = 0, b = n;                                 // cu[a] <= t < cu[a + 1]
      while (b - a > 1) {
        const int m = (a + b) >> 1;
        if (cu[m] <= t) a = m; else b = m;
      }
      const int id = seqs[a];
      bool ok = id >= 0 && id < c.max_seqs && cu[a] <= t && t < cu[a + 1];
      if (ok) {
        const int p = c.len[id] - (cu[a + 1] - t);
        ok = p >= 0 && (p >> c.shift) < c.max_pages;
        if (ok) {
          page = c.table[(int64_t)id * c.max_pages + (p >> c.shift)];
          slot = p & (c.page - 1);
          ok = page >= 0 && page < c.pages && c.ref[page] == 1;
        }
      }
      if (!ok) { page = -1; flag(head, PCOMOE_ERR_INDEX); }
    }
    s_page[threadIdx.x] = page;
    s_slot[threadIdx.x] = slot;
  }
  __syncthreads();
  const int per = c.kv_heads * c.chunks;                 // 16-byte pieces of a row
  const int64_t in0 = (int64_t)layer * layer_bytes, out0 = (int64_t)(first_layer + layer) * c.pages * c.page_bytes;
  for (int u = threadIdx.x; u < 2 * per; u += blockDim.x) {
    const int kv = u >= per, e = kv ? u - per : u;
    const int head_i = e / c.chunks, chunk = e - head_i * c.chunks;
    const char *in = (kv ? v : k) + in0 + (int64_t)e * 16;
    char *out = (kv ? c.v : c.k) + out0;
    uint4 x[kWriteRows];
#pragma unroll
    for (int r = 0; r < kWriteRows; ++r)
      if (s_page[r] >= 0) x[r] = __ldcs((const uint4 *)(in + (int64_t)(t0 + r) * row_bytes));
#pragma unroll
    for (int r = 0; r < kWriteRows; ++r)
      if (s_page[r] >= 0)
        *(uint4 *)(out + (int64_t)s_page[r] * c.page_bytes + ((int64_t)(head_i * c.page + s_slot[r]) * c.chunks + chunk) * 16) = x[r];
  }
}

// A block per pair.
__global__ void __launch_bounds__(256) fork_kernel(CacheDev c, int n, const int32_t *parent, const int32_t *child, CacheHeader *head) {
  pdl_grid_wait();
  const int i = blockIdx.x, p = parent[i], k = child[i];
  int bad = p < 0 || p >= c.max_seqs || k < 0 || k >= c.max_seqs || p == k;
  for (int j = threadIdx.x; j < n; j += blockDim.x) bad |= (j != i && child[j] == k) || parent[j] == k;
  if (!bad) bad = c.len[k] != 0;
  if (__syncthreads_or(bad)) {
    if (threadIdx.x == 0) flag(head, PCOMOE_ERR_INDEX);
    return;
  }
  const int len = c.len[p], m = min(pages_of(c, len), c.max_pages);
  for (int s = threadIdx.x; s < m; s += blockDim.x) {
    const int page = c.table[(int64_t)p * c.max_pages + s];
    if (page >= 0 && page < c.pages) atomicAdd(&c.ref[page], 1);
    c.table[(int64_t)k * c.max_pages + s] = page;
  }
  __syncthreads();                                        // every thread has read len[k] before it changes
  if (threadIdx.x == 0) c.len[k] = len;
}

// A block per sequence.
__global__ void __launch_bounds__(256) trim_kernel(CacheDev c, int n, const int32_t *seqs, const int32_t *lens, CacheHeader *head) {
  pdl_grid_wait();
  const int i = blockIdx.x;
  bool ok = alone(seqs, n, i, c.max_seqs);
  const int id = seqs[i], want = lens[i], have = ok ? c.len[id] : 0;
  ok = ok && want >= 0 && want <= have;
  if (!ok) {
    if (threadIdx.x == 0) flag(head, PCOMOE_ERR_INDEX);
    return;
  }
  drop_pages(c, id, have, want);
  __syncthreads();
  if (threadIdx.x == 0) c.len[id] = want;
}

// Whether entry i of keep's list can be done.  Whole block; *base gets the position of the first drafted token.  Only the
// kernel that moves the rows asks: while the bookkeeping runs, reference counts fall and the answer could change.
__device__ bool keep_ok(const CacheDev &c, int n, const int32_t *seqs, const int32_t *cu, const int32_t *keep, int stride,
                        const int32_t *n_keep, int i, int *base) {
  bool ok = alone(seqs, n, i, c.max_seqs);
  const int id = seqs[i], drafts = cu[i + 1] - cu[i], m = n_keep[i];
  const int first = ok ? c.len[id] - drafts : -1;
  ok = ok && drafts >= 0 && first >= 0 && m >= 0 && m <= drafts && m <= stride && pages_of(c, first + drafts) <= c.max_pages;
  int bad = 0;
  if (ok)
    for (int j = threadIdx.x; j < m; j += blockDim.x) {
      const int x = keep[(int64_t)i * stride + j];
      if (x < 0 || x >= drafts || (j && keep[(int64_t)i * stride + j - 1] >= x)) {
        bad = 1;
        break;
      }
      const int from = c.table[(int64_t)id * c.max_pages + ((first + x) >> c.shift)];
      const int to = c.table[(int64_t)id * c.max_pages + ((first + j) >> c.shift)];
      bad |= from < 0 || from >= c.pages || to < 0 || to >= c.pages;
      if (!bad && x != j) bad |= c.ref[to] != 1;
    }
  *base = first;
  return !__syncthreads_or(bad) && ok;
}

// The accepted rows move up.  A thread owns one 16-byte piece of a row in one layer and head, K or V, and walks the rows
// in ascending order, eight loads before their stores: the numbers ascend, so a row is never overwritten before it was read.
__global__ void __launch_bounds__(256) keep_rows_kernel(CacheDev c, int n, const int32_t *seqs, const int32_t *cu,
                                                        const int32_t *keep, int stride, const int32_t *n_keep, CacheWs w) {
  pdl_grid_wait();
  const int i = blockIdx.y;
  int base;
  const bool ok = keep_ok(c, n, seqs, cu, keep, stride, n_keep, i, &base);
  if (blockIdx.x == 0 && threadIdx.x == 0) w.src[i] = ok;      // for the bookkeeping
  if (!ok) return;
  const int u = blockIdx.x * blockDim.x + threadIdx.x;
  const int per = c.kv_heads * c.chunks;
  if (u >= 2 * c.layers * per) return;
  const int e = u % per, kv = (u / per) & 1, layer = u / (2 * per);
  char *pool = (kv ? c.v : c.k) + (int64_t)layer * c.pages * c.page_bytes + (int64_t)(e / c.chunks) * c.page * c.chunks * 16 +
               (e % c.chunks) * 16;
  const int32_t *row = c.table + (int64_t)seqs[i] * c.max_pages;
  const int m = n_keep[i];
  auto place = [&](int p) { return pool + (int64_t)row[p >> c.shift] * c.page_bytes + (int64_t)(p & (c.page - 1)) * c.chunks * 16; };
  for (int j0 = 0; j0 < m; j0 += 8) {
    uint4 x[8];
    int from[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      from[k] = j0 + k < m ? keep[(int64_t)i * stride + j0 + k] : j0 + k;
      if (from[k] != j0 + k) x[k] = *(const uint4 *)place(base + from[k]);
    }
#pragma unroll
    for (int k = 0; k < 8; ++k)
      if (from[k] != j0 + k) *(uint4 *)place(base + j0 + k) = x[k];
  }
}

__global__ void __launch_bounds__(256) keep_book_kernel(CacheDev c, const int32_t *seqs, const int32_t *cu, const int32_t *n_keep,
                                                        CacheWs w) {
  pdl_grid_wait();
  const int i = blockIdx.x;
  if (!w.src[i]) {
    if (threadIdx.x == 0) flag(w.head, PCOMOE_ERR_INDEX);
    return;
  }
  const int id = seqs[i], have = c.len[id], want = have - (cu[i + 1] - cu[i]) + n_keep[i];
  drop_pages(c, id, have, want);
  __syncthreads();
  if (threadIdx.x == 0) c.len[id] = want;
}

// One block: the pages in use from `used` on and the free ones below it, paired in order, and the new id of every page.
__global__ void __launch_bounds__(kPlanThreads) compact_plan_kernel(CacheDev c, CacheWs w) {
  pdl_grid_wait();
  __shared__ int s_scan[33];
  const int tid = threadIdx.x, lane = tid & 31, wp = tid >> 5;
  const int run = ((c.pages + 1023) / 1024) * 32;
  const int lo = min(wp * run, c.pages), hi = min(lo + run, c.pages);
  int mine = 0, used;
  for (int p = lo + lane; p < hi; p += 32) mine += c.ref[p] > 0;
#pragma unroll
  for (int o = 16; o; o >>= 1) mine += __shfl_xor_sync(~0u, mine, o);
  int live_before = block_scan(lane == 0 ? mine : 0, s_scan, &used);
  live_before = __shfl_sync(~0u, live_before, 0);
  // live pages below `used`: those at or above it move, as many as there are holes below
  int low = 0, low_live;
  for (int p = lo + lane; p < hi; p += 32) low += p < used && c.ref[p] > 0;
#pragma unroll
  for (int o = 16; o; o >>= 1) low += __shfl_xor_sync(~0u, low, o);
  block_scan(lane == 0 ? low : 0, s_scan, &low_live);
  int live = live_before;                                 // live pages before p0
  for (int p0 = lo; p0 < hi; p0 += 32) {
    const int p = p0 + lane;
    const bool in = p < hi, is_live = in && c.ref[p] > 0;
    const uint32_t b = __ballot_sync(~0u, is_live);
    const int before = live + __popc(b & ((1u << lane) - 1));
    if (in) {
      if (is_live && p >= used) w.src[before - low_live] = p;
      if (!is_live && p < used) w.dst[p - before] = p;
      w.list[p] = p;
    }
    live += __popc(b);
  }
  __syncthreads();
  const int moves = used - low_live;
  for (int m = tid; m < moves; m += kPlanThreads) {
    w.list[w.src[m]] = w.dst[m];
    c.ref[w.dst[m]] = c.ref[w.src[m]];
    c.ref[w.src[m]] = 0;
  }
  if (tid == 0) w.head->n_moves = moves;
}

template <bool kRemap>
pcomoe_status launch_moves(const CacheDev &c, const CacheWs &w, int64_t most, int sms, cudaStream_t st) {
  const int64_t units = most * 2 * c.layers * ((c.page_bytes + kPiece - 1) / kPiece);
  const int grid = (int)std::max<int64_t>(1, std::min<int64_t>(units, (int64_t)sms * 8));
  PCOMOE_CUDA_TRY(launch_pdl(move_pages_kernel<kRemap>, dim3(grid), dim3(256), 0, st, c, w));
  count_launch();
  return PCOMOE_OK;
}

}  // namespace

pcomoe_status check_cache(const pcomoe_cache *c) {
  if (!c || c->struct_size != (int32_t)sizeof(pcomoe_cache)) return PCOMOE_ERR_INVALID_ARG;
  if (c->layers <= 0 || c->pages <= 0 || c->kv_heads <= 0 || c->head_dim <= 0 || c->max_seqs <= 0 || c->max_pages <= 0)
    return PCOMOE_ERR_INVALID_ARG;
  if (c->dtype != PCOMOE_BF16 && c->dtype != PCOMOE_FP32) return PCOMOE_ERR_INVALID_ARG;
  if (!c->d_k || !c->d_v || !c->d_seq_len || !c->d_page_ref || !c->d_page_table) return PCOMOE_ERR_INVALID_ARG;
  if (c->page_size != 16 && c->page_size != 32 && c->page_size != 64 && c->page_size != 128) return PCOMOE_ERR_UNSUPPORTED;
  if (((size_t)c->head_dim * dtype_size(c->dtype)) % 16 || (((uintptr_t)c->d_k | (uintptr_t)c->d_v) & 15)) return PCOMOE_ERR_UNSUPPORTED;
  if (c->max_seqs > kMaxSeqs || (int64_t)c->max_pages * c->page_size > INT32_MAX || c->pages > kMaxPages) return PCOMOE_ERR_SHAPE;
  return PCOMOE_OK;
}

}  // namespace pcomoe

using namespace pcomoe;

namespace {

// The checks that every cache call makes of its list and workspace.
pcomoe_status check_call(const pcomoe_cache *c, int32_t n, void *ws, size_t ws_bytes) {
  pcomoe_status st = check_cache(c);
  if (st != PCOMOE_OK) return st;
  if (n < 0) return PCOMOE_ERR_INVALID_ARG;
  if (n > c->max_seqs) return PCOMOE_ERR_SHAPE;
  if (!ws || ((uintptr_t)ws & 255) || ws_bytes < cache_ws(c, nullptr).total) return PCOMOE_ERR_WORKSPACE;
  return PCOMOE_OK;
}

}  // namespace

extern "C" {

pcomoe_status pcomoe_cache_workspace_bytes(const pcomoe_cache *cache, size_t *bytes) {
  if (!bytes) return PCOMOE_ERR_INVALID_ARG;
  pcomoe_status st = check_cache(cache);
  if (st != PCOMOE_OK) return st;
  *bytes = cache_ws(cache, nullptr).total;
  return PCOMOE_OK;
}

pcomoe_status pcomoe_cache_reserve(const pcomoe_cache *cache, int32_t n, const int32_t *d_seqs, const int32_t *d_add,
                                   void *d_workspace, size_t ws_bytes, void *stream) {
  pcomoe_status st = check_call(cache, n, d_workspace, ws_bytes);
  if (st != PCOMOE_OK) return st;
  if (n == 0) return PCOMOE_OK;
  if (!d_seqs || !d_add) return PCOMOE_ERR_INVALID_ARG;
  int sms;
  if ((st = current_sms(&sms)) != PCOMOE_OK) return st;
  const CacheDev c = cache_dev(cache);
  const CacheWs w = cache_ws(cache, d_workspace);
  PCOMOE_CUDA_TRY(launch_pdl(reserve_plan_kernel, dim3(1), dim3(kPlanThreads), 0, (cudaStream_t)stream, c, n, d_seqs, d_add, w));
  count_launch();
  return launch_moves<false>(c, w, n, sms, (cudaStream_t)stream);
}

pcomoe_status pcomoe_cache_write(const pcomoe_cache *cache, int32_t first_layer, int32_t n_layers, int32_t T, int32_t n,
                                 const int32_t *d_seqs, const int32_t *d_cu_len, const void *d_k, const void *d_v,
                                 int64_t row_stride, int64_t layer_stride, void *d_workspace, size_t ws_bytes, void *stream) {
  pcomoe_status st = check_call(cache, n, d_workspace, ws_bytes);
  if (st != PCOMOE_OK) return st;
  if (first_layer < 0 || n_layers < 0 || n_layers > cache->layers - first_layer) return PCOMOE_ERR_INVALID_ARG;
  if (T < 0) return PCOMOE_ERR_SHAPE;
  if (T == 0 || n == 0 || n_layers == 0) return PCOMOE_OK;
  const int64_t e = (int64_t)dtype_size(cache->dtype);
  if (!d_seqs || !d_cu_len || !d_k || !d_v || row_stride < (int64_t)cache->kv_heads * cache->head_dim || layer_stride < 0)
    return PCOMOE_ERR_INVALID_ARG;
  if ((((uintptr_t)d_k | (uintptr_t)d_v) & 15) || (row_stride * e) % 16 || (layer_stride * e) % 16) return PCOMOE_ERR_UNSUPPORTED;
  if (n_layers > 65535) return PCOMOE_ERR_SHAPE;
  PCOMOE_CUDA_TRY(launch_pdl(cache_write_kernel, dim3((T + kWriteRows - 1) / kWriteRows, n_layers), dim3(256), 0, (cudaStream_t)stream,
                             cache_dev(cache), first_layer, T, n, d_seqs, d_cu_len, (const char *)d_k, (const char *)d_v,
                             row_stride * e, layer_stride * e, cache_ws(cache, d_workspace).head));
  count_launch();
  return PCOMOE_OK;
}

pcomoe_status pcomoe_cache_fork(const pcomoe_cache *cache, int32_t n, const int32_t *d_parent, const int32_t *d_child,
                                void *d_workspace, size_t ws_bytes, void *stream) {
  pcomoe_status st = check_call(cache, n, d_workspace, ws_bytes);
  if (st != PCOMOE_OK || n == 0) return st;
  if (!d_parent || !d_child) return PCOMOE_ERR_INVALID_ARG;
  PCOMOE_CUDA_TRY(launch_pdl(fork_kernel, dim3(n), dim3(256), 0, (cudaStream_t)stream, cache_dev(cache), n, d_parent, d_child,
                             cache_ws(cache, d_workspace).head));
  count_launch();
  return PCOMOE_OK;
}

pcomoe_status pcomoe_cache_keep(const pcomoe_cache *cache, int32_t n, const int32_t *d_seqs, const int32_t *d_cu_len,
                                const int32_t *d_keep, int32_t keep_stride, const int32_t *d_n_keep, void *d_workspace,
                                size_t ws_bytes, void *stream) {
  pcomoe_status st = check_call(cache, n, d_workspace, ws_bytes);
  if (st != PCOMOE_OK || n == 0) return st;
  if (!d_seqs || !d_cu_len || !d_n_keep || keep_stride < 0 || (keep_stride > 0 && !d_keep)) return PCOMOE_ERR_INVALID_ARG;
  const CacheDev c = cache_dev(cache);
  const CacheWs w = cache_ws(cache, d_workspace);
  const int64_t threads = (int64_t)2 * c.layers * c.kv_heads * c.chunks;
  if (threads > INT32_MAX) return PCOMOE_ERR_SHAPE;
  PCOMOE_CUDA_TRY(launch_pdl(keep_rows_kernel, dim3((unsigned)((threads + 255) / 256), n), dim3(256), 0, (cudaStream_t)stream, c, n, d_seqs,
                             d_cu_len, d_keep, keep_stride, d_n_keep, w));
  PCOMOE_CUDA_TRY(launch_pdl(keep_book_kernel, dim3(n), dim3(256), 0, (cudaStream_t)stream, c, d_seqs, d_cu_len, d_n_keep, w));
  count_launch(2);
  return PCOMOE_OK;
}

pcomoe_status pcomoe_cache_trim(const pcomoe_cache *cache, int32_t n, const int32_t *d_seqs, const int32_t *d_len,
                                void *d_workspace, size_t ws_bytes, void *stream) {
  pcomoe_status st = check_call(cache, n, d_workspace, ws_bytes);
  if (st != PCOMOE_OK || n == 0) return st;
  if (!d_seqs || !d_len) return PCOMOE_ERR_INVALID_ARG;
  PCOMOE_CUDA_TRY(launch_pdl(trim_kernel, dim3(n), dim3(256), 0, (cudaStream_t)stream, cache_dev(cache), n, d_seqs, d_len,
                             cache_ws(cache, d_workspace).head));
  count_launch();
  return PCOMOE_OK;
}

pcomoe_status pcomoe_cache_compact(const pcomoe_cache *cache, void *d_workspace, size_t ws_bytes, void *stream) {
  pcomoe_status st = check_call(cache, 0, d_workspace, ws_bytes);
  if (st != PCOMOE_OK) return st;
  int sms;
  if ((st = current_sms(&sms)) != PCOMOE_OK) return st;
  const CacheDev c = cache_dev(cache);
  const CacheWs w = cache_ws(cache, d_workspace);
  PCOMOE_CUDA_TRY(launch_pdl(compact_plan_kernel, dim3(1), dim3(kPlanThreads), 0, (cudaStream_t)stream, c, w));
  count_launch();
  return launch_moves<true>(c, w, (c.pages + 1) / 2, sms, (cudaStream_t)stream);
}

}  // extern "C"
