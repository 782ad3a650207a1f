// Eviction from the paged cache by accumulated weight: which positions stay, their rows moved up in order, pages freed.
//
// Three launches.  The first, a block per sequence, finds the weight of the last position that stays by four rounds over its
// bits (a histogram of 256 bins each, from the top), lists the places that stay in order and moves the weights.  The second moves the
// rows: a block owns a column of 64 bytes of one head's rows in one layer, K or V, and walks over them in ascending windows; the
// places ascend and a row never moves up past itself, so a window only has to be read whole before it is written, and
// nothing that a later window reads is overwritten.  The third gives back the pages.
// What bounds it: the moved rows, read and written once (HBM); few sequences in few layers leave few columns to walk over.
#include <algorithm>

#include "cache.cuh"

namespace pcomoe {
namespace {

constexpr int kSelectThreads = 1024, kMoveThreads = 256;

struct EvictSeq {                          // what the first launch leaves for the others
  int32_t left;                            // new length; -1: the sequence stays as it is
  int32_t first;                           // first place whose row changes
};

struct EvictWs {
  CacheHeader *head;
  EvictSeq *seq;                           // [n]
  int32_t *list;                           // [n][room] places that stay
  int64_t room;
  size_t total;
};

EvictWs evict_ws(const pcomoe_cache *c, int32_t n, void *ws) {
  EvictWs w;
  w.room = (int64_t)c->max_pages * c->page_size;
  const size_t seqs = align256(sizeof(EvictSeq) * (size_t)n);
  w.head = (CacheHeader *)ws;
  w.seq = (EvictSeq *)((char *)ws + 256);
  w.list = (int32_t *)((char *)ws + 256 + seqs);
  w.total = 256 + seqs + align256(4 * (size_t)n * (size_t)w.room);
  return w;
}

// Order of weights as integers: larger is heavier, -0 is 0, a NaN the smallest.
__device__ __forceinline__ uint32_t heaviness(float w) {
  if (w != w) return 0u;
  const uint32_t b = __float_as_uint(w + 0.f);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}

// Exclusive prefix over the warps of one value per warp.  s: 33 ints.
__device__ __forceinline__ int warps_before(int x, int *s) {
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
  if (lane == 0) s[w] = x;
  __syncthreads();
  const int y = __reduce_add_sync(~0u, lane < w ? s[lane] : 0);
  __syncthreads();
  return y;
}

__global__ void __launch_bounds__(kSelectThreads) evict_select_kernel(CacheDev c, int n, const int32_t *seqs, const int32_t *budget, int sinks, int recent,
                                                                      float *weight, int64_t weight_stride, EvictWs ws) {
  pdl_grid_wait();
  static_assert(kSelectThreads == 1024, "a warp's lanes stand for the warps");
  __shared__ int s_bin[256], s_scan[33], s_pick, s_rest, s_first;
  const int i = blockIdx.x, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  EvictSeq *out = ws.seq + i;
  bool ok = alone(seqs, n, i, c.max_seqs);
  const int id = seqs[i], L = ok ? c.len[id] : 0, B = budget[i];
  ok = ok && B >= 0 && L >= 0 && pages_of(c, L) <= c.max_pages;
  const bool cuts = ok && L > B;
  if (cuts && (int64_t)sinks + recent > B) ok = false;
  if (!ok || !cuts) {
    if (tid == 0) {
      out->left = -1;
      if (!ok) flag(ws.head, PCOMOE_ERR_INDEX);
    }
    return;
  }
  float *w = weight + id * weight_stride;
  const int lo = sinks, hi = L - recent, need = B - sinks - recent;      // `need` of the positions [lo, hi) stay, fewer than there are
  // the key of the last one that stays, from its upper bits down, and how many with this key stay
  uint32_t key = 0xffffffffu;
  int equal = 0;
  if (need > 0) {
    key = 0;
    equal = need;
    for (int round = 0; round < 4; ++round) {
      const int sh = 24 - 8 * round;
      for (int b = tid; b < 256; b += kSelectThreads) s_bin[b] = 0;
      __syncthreads();
      for (int p = lo + tid; p < hi; p += kSelectThreads) {
        const uint32_t k = heaviness(w[p]);
        if (round == 0 || (k >> (sh + 8)) == (key >> (sh + 8))) atomicAdd(&s_bin[(k >> sh) & 255], 1);
      }
      __syncthreads();
      if (warp == 0) {
        // lane l: bins 255 - 8 l down; the bin in which the count passes `equal`
        int mine = 0;
        for (int b = 0; b < 8; ++b) mine += s_bin[255 - 8 * lane - b];
        int upto = mine;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
          const int y = __shfl_up_sync(~0u, upto, o);
          if (lane >= o) upto += y;
        }
        const uint32_t past = __ballot_sync(~0u, upto >= equal);
        if (lane == __ffs(past) - 1) {
          int before = upto - mine, b = 0;
          while (before + s_bin[255 - 8 * lane - b] < equal) before += s_bin[255 - 8 * lane - b++];
          s_pick = 255 - 8 * lane - b;
          s_rest = equal - before;
        }
      }
      __syncthreads();
      key |= (uint32_t)s_pick << sh;
      equal = s_rest;
      __syncthreads();
    }
  }
  // the places that stay: every warp has a run of positions, counts its own, then lists them
  const int run = ((L + 1023) / 1024) * 32, p0 = min(warp * run, L), p1 = min(p0 + run, L);
  int sure = 0, ties = 0;
  auto look = [&](int p, bool &stays, bool &tie) {
    stays = tie = false;
    if (p < p1) {
      if (p < lo || p >= hi) {
        stays = true;
      } else if (need > 0) {
        const uint32_t k = heaviness(w[p]);
        stays = k > key;
        tie = k == key;
      }
    }
  };
  for (int p = p0; p < p1; p += 32) {
    bool stays, tie;
    look(p + lane, stays, tie);
    sure += __popc(__ballot_sync(~0u, stays));
    ties += __popc(__ballot_sync(~0u, tie));
  }
  int tie_at = warps_before(ties, s_scan);
  const int own_ties = min(max(equal - tie_at, 0), ties);
  int at = warps_before(sure + own_ties, s_scan);
  int32_t *list = ws.list + i * ws.room;
  if (tid == 0) s_first = B;
  __syncthreads();
  int first = B;
  for (int p = p0; p < p1; p += 32) {
    bool stays, tie;
    look(p + lane, stays, tie);
    const uint32_t below = (1u << lane) - 1u, t = __ballot_sync(~0u, tie);
    if (tie) stays = tie_at + __popc(t & below) < equal;
    tie_at += __popc(t);
    const uint32_t b = __ballot_sync(~0u, stays);
    const int j = at + __popc(b & below);
    if (stays) {
      list[j] = p + lane;
      if (j != p + lane) first = min(first, j);
    }
    at += __popc(b);
  }
  first = __reduce_min_sync(~0u, first);
  if (lane == 0) atomicMin(&s_first, first);
  __syncthreads();
  first = s_first;
  // the pages written to are this sequence's alone, and all are pages
  const int32_t *row = c.table + (int64_t)id * c.max_pages;
  int bad = 0;
  for (int s = (first >> c.shift) + tid; s < pages_of(c, L); s += kSelectThreads) {
    const int page = row[s];
    bad |= page < 0 || page >= c.pages || (s < pages_of(c, B) && first < B && c.ref[page] != 1);
  }
  if (__syncthreads_or(bad)) {
    if (tid == 0) {
      out->left = -1;
      flag(ws.head, PCOMOE_ERR_INDEX);
    }
    return;
  }
  // the weights move as the rows do: a window is read before it is written
  for (int j0 = first; j0 < B; j0 += 4 * kSelectThreads) {
    float x[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int j = j0 + k * kSelectThreads + tid;
      if (j < B) x[k] = w[list[j]];
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int j = j0 + k * kSelectThreads + tid;
      if (j < B) w[j] = x[k];
    }
    __syncthreads();
  }
  if (tid == 0) { out->left = B; out->first = first; }
}

// blockIdx: (head and column, layer and K or V, sequence)
constexpr int kColumn = 4;                                 // 16-byte pieces of a row that a block moves
__global__ void __launch_bounds__(kMoveThreads) evict_move_kernel(CacheDev c, const int32_t *seqs, EvictWs ws) {
  pdl_grid_wait();
  constexpr int kRows = kMoveThreads / kColumn, U = 8;
  const int i = blockIdx.z;
  const EvictSeq s = ws.seq[i];
  if (s.left < 0 || s.first >= s.left) return;
  const int parts = (c.chunks + kColumn - 1) / kColumn, head = blockIdx.x / parts, chunk = (blockIdx.x % parts) * kColumn + threadIdx.x % kColumn;
  const bool has = chunk < c.chunks;
  const int layer = blockIdx.y >> 1;
  char *pool = (blockIdx.y & 1 ? c.v : c.k) + (int64_t)layer * c.pages * c.page_bytes + ((int64_t)head * c.page * c.chunks + chunk) * 16;
  const int32_t *row = c.table + (int64_t)seqs[i] * c.max_pages, *list = ws.list + i * ws.room;
  auto place = [&](int p) { return (uint4 *)(pool + (int64_t)row[p >> c.shift] * c.page_bytes + (int64_t)(p & (c.page - 1)) * c.chunks * 16); };
  const int r = threadIdx.x / kColumn;
  for (int j0 = s.first; j0 < s.left; j0 += kRows * U) {
    uint4 x[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int j = j0 + u * kRows + r;
      if (has && j < s.left) x[u] = *place(list[j]);
    }
    __syncthreads();                                       // the window is read
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int j = j0 + u * kRows + r;
      if (has && j < s.left) *place(j) = x[u];
    }
  }
}

__global__ void __launch_bounds__(256) evict_book_kernel(CacheDev c, const int32_t *seqs, EvictWs ws) {
  pdl_grid_wait();
  const int i = blockIdx.x, left = ws.seq[i].left;
  if (left < 0) return;
  const int id = seqs[i];
  drop_pages(c, id, c.len[id], left);
  __syncthreads();
  if (threadIdx.x == 0) c.len[id] = left;
}

}  // namespace
}  // namespace pcomoe

using namespace pcomoe;

extern "C" {

pcomoe_status pcomoe_evict_workspace_bytes(const pcomoe_cache *cache, int32_t n, size_t *bytes) {
  if (!bytes) return PCOMOE_ERR_INVALID_ARG;
  const pcomoe_status st = check_cache(cache);
  if (st != PCOMOE_OK) return st;
  if (n < 0) return PCOMOE_ERR_INVALID_ARG;
  if (n > cache->max_seqs) return PCOMOE_ERR_SHAPE;
  *bytes = evict_ws(cache, n, nullptr).total;
  return PCOMOE_OK;
}

pcomoe_status pcomoe_cache_evict(const pcomoe_cache *cache, int32_t n, const int32_t *d_seqs, const int32_t *d_budget, int32_t sinks, int32_t recent,
                                 float *d_weight, int64_t weight_stride, void *d_workspace, size_t ws_bytes, void *stream) {
  const pcomoe_status st = check_cache(cache);
  if (st != PCOMOE_OK) return st;
  if (n < 0 || sinks < 0 || recent < 0) return PCOMOE_ERR_INVALID_ARG;
  if (n > cache->max_seqs || cache->layers > 32767) return PCOMOE_ERR_SHAPE;
  if (!d_workspace || ((uintptr_t)d_workspace & 255) || ws_bytes < evict_ws(cache, n, nullptr).total) return PCOMOE_ERR_WORKSPACE;
  if (n == 0) return PCOMOE_OK;
  if (!d_seqs || !d_budget || !d_weight || weight_stride < (int64_t)cache->max_pages * cache->page_size) return PCOMOE_ERR_INVALID_ARG;
  const CacheDev c = cache_dev(cache);
  const EvictWs w = evict_ws(cache, n, d_workspace);
  const int64_t columns = (int64_t)c.kv_heads * ((c.chunks + kColumn - 1) / kColumn);
  if (columns > INT32_MAX) return PCOMOE_ERR_SHAPE;
  PCOMOE_CUDA_TRY(launch_pdl(evict_select_kernel, dim3(n), dim3(kSelectThreads), 0, (cudaStream_t)stream, c, n, d_seqs, d_budget, sinks, recent, d_weight,
                             weight_stride, w));
  PCOMOE_CUDA_TRY(launch_pdl(evict_move_kernel, dim3((unsigned)columns, 2 * c.layers, n), dim3(kMoveThreads), 0, (cudaStream_t)stream, c, d_seqs, w));
  PCOMOE_CUDA_TRY(launch_pdl(evict_book_kernel, dim3(n), dim3(256), 0, (cudaStream_t)stream, c, d_seqs, w));
  count_launch(3);
  return PCOMOE_OK;
}

}  // extern "C"
