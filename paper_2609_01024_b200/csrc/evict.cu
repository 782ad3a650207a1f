// Eviction from the paged cache by accumulated weight: which positions stay, their rows moved up in order, pages freed.
//
// Three launches.  The first, a cluster of blocks per sequence, finds the weight of the last position that stays by four rounds
// over its bits (a histogram of 256 bins each, from the top, added over the blocks), lists the places that stay in order, as rows of
// the pool, with their weights.  The second moves rows and weights: a block owns a column of 64 bytes of one head's rows in one layer, K
// or V, and walks over them in ascending windows; the places ascend and a row never moves up past itself, so a window only has
// to be read whole before it is written, and nothing that a later window reads is overwritten: the next window's rows come in
// while this one's are stored.  The third gives back the pages.
// What bounds it: the moved rows, read and written once (HBM); few sequences in few layers leave few columns to walk over.  Measured: one
// sequence of 131071 tokens cut to a quarter in 2 layers of 8 heads of 128, the move 107 us for 492 MB (4.6 TB/s; 128 blocks have a
// column), the choice 35 us; 8 sequences of 905 to 4050 tokens in 4 layers, the move 51 us, the choice 12.  Columns of 32 bytes took the
// whole pass over the long sequence from 478 to 508 us, of 128 bytes (half as many blocks) to 524; loads that bring 128 or 256 bytes into
// L2 583 and 527.
#include <algorithm>

#include "cache.cuh"

namespace pcomoe {
namespace {

constexpr int kSelectThreads = 1024;

struct EvictSeq {                          // what the first launch leaves for the others
  int32_t was, left;                       // old and new length; left -1: the sequence stays as it is
  int32_t first;                           // first place whose row changes
};

struct EvictWs {
  CacheHeader *head;
  EvictSeq *seq;                           // [n]
  int32_t *list;                           // [n][room] rows that stay: page * page_size + place in it
  float *kept;                             // [n][room] their weights
  int64_t room;
  size_t total;
};

EvictWs evict_ws(const pcomoe_cache *c, int32_t n, void *ws) {
  EvictWs w;
  w.room = (int64_t)c->max_pages * c->page_size;
  const size_t seqs = align256(sizeof(EvictSeq) * (size_t)n);
  w.head = (CacheHeader *)ws;
  w.seq = (EvictSeq *)((char *)ws + 256);
  const size_t lists = align256(4 * (size_t)n * (size_t)w.room);
  w.list = (int32_t *)((char *)ws + 256 + seqs);
  w.kept = (float *)((char *)ws + 256 + seqs + lists);
  w.total = 256 + seqs + 2 * lists;
  return w;
}

// Order of weights as integers: larger is heavier, -0 is 0, a NaN the smallest.
__device__ __forceinline__ uint32_t heaviness(float w) {
  if (w != w) return 0u;
  const uint32_t b = __float_as_uint(w + 0.f);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}

// A word of another block of the cluster, and the cluster's barrier; one block: its own.
template <int CL>
__device__ __forceinline__ int of_block(const int *p, int rank) {
  if (CL == 1) return *p;
  uint32_t q;
  int v;
  asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(q) : "r"((uint32_t)__cvta_generic_to_shared(p)), "r"(rank));
  asm volatile("ld.shared::cluster.s32 %0, [%1];" : "=r"(v) : "r"(q) : "memory");
  return v;
}
template <int CL>
__device__ __forceinline__ void all_blocks() {
  if (CL > 1) asm volatile("barrier.cluster.arrive.aligned;\n\tbarrier.cluster.wait.aligned;" ::: "memory");
  else __syncthreads();
}

template <int CL>
__global__ void __launch_bounds__(kSelectThreads) evict_select_kernel(CacheDev c, int n, const int32_t *seqs, const int32_t *budget, int sinks, int recent,
                                                                      float *weight, int64_t weight_stride, EvictWs ws) {
  pdl_grid_wait();
  constexpr int kWarps = kSelectThreads / 32;
  static_assert(kWarps == 32, "a warp's lanes stand for the warps");
  __shared__ int s_bin[2][256], s_all[256], s_warp[2][kWarps], s_pick, s_rest, s_first;
  const int i = blockIdx.x / CL, rank = CL > 1 ? (int)(blockIdx.x % CL) : 0, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  EvictSeq *out = ws.seq + i;
  // (every block of the cluster comes to the same answers)
  bool ok = alone(seqs, n, i, c.max_seqs);
  const int id = seqs[i], L = ok ? c.len[id] : 0, B = budget[i];
  ok = ok && B >= 0 && L >= 0 && pages_of(c, L) <= c.max_pages;
  const bool cuts = ok && L > B;
  if (cuts && (int64_t)sinks + recent > B) ok = false;
  if (!ok || !cuts) {
    if (tid == 0 && rank == 0) {
      out->left = -1;
      if (!ok) flag(ws.head, PCOMOE_ERR_INDEX);
    }
    return;
  }
  float *w = weight + id * weight_stride;
  const int lo = sinks, hi = L - recent, need = B - sinks - recent;      // `need` of the positions [lo, hi) stay, fewer than there are
  // a run of positions for every warp of the cluster, in order
  const int run = ((L + 1024 * CL - 1) / (1024 * CL)) * 32, p0 = min((rank * kWarps + warp) * run, L), p1 = min(p0 + run, L);
  // the key of the last one that stays, from its upper bits down, and how many with this key stay
  uint32_t key = 0xffffffffu;
  int equal = 0;
  if (need > 0) {
    key = 0;
    equal = need;
    for (int round = 0; round < 4; ++round) {
      const int sh = 24 - 8 * round;
      int *bin = s_bin[round & 1];
      for (int b = tid; b < 256; b += kSelectThreads) bin[b] = 0;
      __syncthreads();
#pragma unroll 4
      for (int p = max(p0, lo) + lane; p < min(p1, hi); p += 32) {
        const uint32_t k = heaviness(w[p]);
        if (round == 0 || (k >> (sh + 8)) == (key >> (sh + 8))) atomicAdd(&bin[(k >> sh) & 255], 1);
      }
      all_blocks<CL>();                                    // (two rounds on the bins are cleared again: all have read them by then)
      if (tid < 256) {
        int sum = 0;
#pragma unroll
        for (int r = 0; r < CL; ++r) sum += of_block<CL>(&bin[tid], r);
        s_all[tid] = sum;
      }
      __syncthreads();
      if (warp == 0) {
        // lane l: bins 255 - 8 l down; the bin in which the count passes `equal`
        int mine = 0;
        for (int b = 0; b < 8; ++b) mine += s_all[255 - 8 * lane - b];
        int upto = mine;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
          const int y = __shfl_up_sync(~0u, upto, o);
          if (lane >= o) upto += y;
        }
        const uint32_t past = __ballot_sync(~0u, upto >= equal);
        if (lane == __ffs(past) - 1) {
          int before = upto - mine, b = 0;
          while (before + s_all[255 - 8 * lane - b] < equal) before += s_all[255 - 8 * lane - b++];
          s_pick = 255 - 8 * lane - b;
          s_rest = equal - before;
        }
      }
      __syncthreads();
      key |= (uint32_t)s_pick << sh;
      equal = s_rest;
    }
  }
  // the places that stay: every warp counts those of its run, then lists them
  int sure = 0, ties = 0;
  auto look = [&](int p, float x, bool &stays, bool &tie) {
    stays = tie = false;
    if (p < p1) {
      if (p < lo || p >= hi) {
        stays = true;
      } else if (need > 0) {
        const uint32_t k = heaviness(x);
        stays = k > key;
        tie = k == key;
      }
    }
  };
#pragma unroll 4
  for (int p = p0; p < p1; p += 32) {
    bool stays, tie;
    look(p + lane, p + lane < p1 ? w[p + lane] : 0.f, stays, tie);
    sure += __popc(__ballot_sync(~0u, stays));
    ties += __popc(__ballot_sync(~0u, tie));
  }
  // what the warps before this one of the whole cluster have
  auto before = [&](int (&box)[kWarps], int x) {
    if (lane == 0) box[warp] = x;
    all_blocks<CL>();
    int y = 0;
#pragma unroll
    for (int r = 0; r < CL; ++r)
      if (r < rank || (r == rank && lane < warp)) y += of_block<CL>(&box[lane], r);
    return (int)__reduce_add_sync(~0u, y);
  };
  int tie_at = before(s_warp[0], ties);
  const int own_ties = min(max(equal - tie_at, 0), ties);
  if (tid == 0) s_first = B;
  int at = before(s_warp[1], sure + own_ties);
  const int32_t *row = c.table + (int64_t)id * c.max_pages;
  int32_t *list = ws.list + i * ws.room;
  float *kept = ws.kept + i * ws.room;
  int first = B, bad = 0;
  // (four steps together, so that the chains weight -> place -> page -> its count run side by side)
  constexpr int U = 4;
  for (int p = p0; p < p1; p += 32 * U) {
    bool stays[U], tie[U];
    float x[U];
    int page[U], to[U], j[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int o = p + 32 * u + lane;
      x[u] = o < p1 ? w[o] : 0.f;
      page[u] = o < p1 ? row[o >> c.shift] : 0;
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      look(p + 32 * u + lane, x[u], stays[u], tie[u]);
      const uint32_t below = (1u << lane) - 1u, t = __ballot_sync(~0u, tie[u]);
      if (tie[u]) stays[u] = tie_at + __popc(t & below) < equal;
      tie_at += __popc(t);
      const uint32_t b = __ballot_sync(~0u, stays[u]);
      j[u] = at + __popc(b & below);
      at += __popc(b);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) to[u] = stays[u] && j[u] != p + 32 * u + lane ? row[j[u] >> c.shift] : 0;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int o = p + 32 * u + lane;
      if (!stays[u]) continue;
      bad |= page[u] < 0 || page[u] >= c.pages;
      list[j[u]] = page[u] * c.page + (o & (c.page - 1));
      kept[j[u]] = x[u];
      if (j[u] != o) {
        first = min(first, j[u]);
        // a page that is written to is this sequence's alone
        bad |= to[u] < 0 || to[u] >= c.pages || c.ref[min(max(to[u], 0), c.pages - 1)] != 1;
      }
    }
  }
  // and all pages that are given back are pages
  for (int s = pages_of(c, B) + rank * kSelectThreads + tid; s < pages_of(c, L); s += CL * kSelectThreads) bad |= row[s] < 0 || row[s] >= c.pages;
  first = __reduce_min_sync(~0u, first);
  bad = __any_sync(~0u, bad);
  if (lane == 0) {
    atomicMin(&s_first, first);
    if (bad) atomicMin(&s_first, -1);
  }
  all_blocks<CL>();
  first = B;
#pragma unroll
  for (int r = 0; r < CL; ++r) first = min(first, of_block<CL>(&s_first, r));
  if (rank == 0 && tid == 0) {
    out->was = L;
    out->left = first < 0 ? -1 : B;
    out->first = first;
    if (first < 0) flag(ws.head, PCOMOE_ERR_INDEX);
  }
  all_blocks<CL>();                                        // nobody leaves while others read its first
}

// blockIdx: (head and column, layer and K or V, sequence); one column more, for the first layer's K, moves the weights.
constexpr int kColumn = 4;                                 // 16-byte pieces of a row that a block moves
template <int kMoveThreads>
__global__ void __launch_bounds__(kMoveThreads) evict_move_kernel(CacheDev c, const int32_t *seqs, float *weight, int64_t weight_stride, EvictWs ws) {
  pdl_grid_wait();
  constexpr int kRows = kMoveThreads / kColumn, U = 8, kWindow = kRows * U;
  const int i = blockIdx.z;
  const EvictSeq s = ws.seq[i];
  if (s.left < 0 || s.first >= s.left) return;
  const int id = seqs[i];
  const int parts = (c.chunks + kColumn - 1) / kColumn, head = blockIdx.x / parts, chunk = (blockIdx.x % parts) * kColumn + threadIdx.x % kColumn;
  if (head >= c.kv_heads) {
    if (blockIdx.y) return;
    for (int j = s.first + threadIdx.x; j < s.left; j += kMoveThreads) weight[id * weight_stride + j] = ws.kept[i * ws.room + j];
    return;
  }
  const bool has = chunk < c.chunks;
  const int layer = blockIdx.y >> 1;
  char *pool = (blockIdx.y & 1 ? c.v : c.k) + (int64_t)layer * c.pages * c.page_bytes + ((int64_t)head * c.page * c.chunks + chunk) * 16;
  const int32_t *row = c.table + (int64_t)id * c.max_pages, *list = ws.list + i * ws.room;
  const int64_t row_bytes = (int64_t)c.chunks * 16;
  auto place = [&](int page, int slot) { return pool + (int64_t)page * c.page_bytes + slot * row_bytes; };
  const int r = threadIdx.x / kColumn;
  // Windows at work: the places of one are asked for, those of the one before are at hand, the rows of the one before that come in, and
  // the first one's are stored.
  int from[U], to[U], from_next[U], to_next[U];
  uint4 x[U];
  auto ask = [&](int j0) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int j = j0 + u * kRows + r;
      from_next[u] = has && j < s.left ? list[j] : -1;
      to_next[u] = has && j < s.left ? row[j >> c.shift] : 0;
    }
  };
  auto take = [&]() {
#pragma unroll
    for (int u = 0; u < U; ++u) { from[u] = from_next[u]; to[u] = to_next[u]; }
  };
  auto fetch = [&]() {
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (from[u] >= 0) x[u] = *(const uint4 *)place(from[u] >> c.shift, from[u] & (c.page - 1));
  };
  ask(s.first);
  take();
  ask(s.first + kWindow);
  fetch();
  for (int j0 = s.first; j0 < s.left; j0 += kWindow) {
    __syncthreads();                                       // the window is read
    uint4 y[U];
    int at[U];
#pragma unroll
    for (int u = 0; u < U; ++u) { y[u] = x[u]; at[u] = to[u]; }
    take();
    ask(j0 + 2 * kWindow);
    fetch();                                               // of the next one: its rows lie behind all that is written now
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int j = j0 + u * kRows + r;
      if (has && j < s.left) *(uint4 *)place(at[u], j & (c.page - 1)) = y[u];
    }
  }
}

// blockIdx: (sequence, share of its pages)
__global__ void __launch_bounds__(256) evict_book_kernel(CacheDev c, const int32_t *seqs, EvictWs ws) {
  pdl_grid_wait();
  const int i = blockIdx.x;
  const EvictSeq s = ws.seq[i];
  if (s.left < 0) return;
  const int id = seqs[i];
  drop_pages(c, id, s.was, s.left, blockIdx.y * 256, gridDim.y * 256);
  if (blockIdx.y == 0 && threadIdx.x == 0) c.len[id] = s.left;
}

template <int CL>
pcomoe_status launch_select(const CacheDev &c, int n, const int32_t *seqs, const int32_t *budget, int sinks, int recent, float *weight, int64_t weight_stride,
                            const EvictWs &ws, cudaStream_t st) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)n * CL);
  cfg.blockDim = dim3(kSelectThreads);
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = CL;
  attr[1].val.clusterDim.y = 1;
  attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = CL > 1 ? 2 : 1;
  PCOMOE_CUDA_TRY(cudaLaunchKernelEx(&cfg, evict_select_kernel<CL>, c, n, seqs, budget, sinks, recent, weight, weight_stride, ws));
  return PCOMOE_OK;
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
  pcomoe_status st = check_cache(cache);
  if (st != PCOMOE_OK) return st;
  if (n < 0 || sinks < 0 || recent < 0) return PCOMOE_ERR_INVALID_ARG;
  if (n > cache->max_seqs || cache->layers > 32767) return PCOMOE_ERR_SHAPE;
  if (!d_workspace || ((uintptr_t)d_workspace & 255) || ws_bytes < evict_ws(cache, n, nullptr).total) return PCOMOE_ERR_WORKSPACE;
  if (n == 0) return PCOMOE_OK;
  if (!d_seqs || !d_budget || !d_weight || weight_stride < (int64_t)cache->max_pages * cache->page_size) return PCOMOE_ERR_INVALID_ARG;
  const CacheDev c = cache_dev(cache);
  const EvictWs w = evict_ws(cache, n, d_workspace);
  const int64_t columns = (int64_t)c.kv_heads * ((c.chunks + kColumn - 1) / kColumn) + 1;
  if (columns > INT32_MAX) return PCOMOE_ERR_SHAPE;
  int sms;
  if ((st = current_sms(&sms)) != PCOMOE_OK) return st;
  // Blocks of a cluster: a sequence may have more than 4096 positions for each, and the GPU two blocks for every SM.  The whole pass with 1, 2, 4
  // and 8: one sequence of 131071 tokens 608, 536, 497, 478 us; 8 of up to 4050 171, 174, 174, 175.
  int cl = 1;
  while (cl < 8 && w.room > 4096 * cl && (int64_t)n * 2 * cl <= 2 * sms) cl *= 2;
  const cudaStream_t s = (cudaStream_t)stream;
  switch (cl) {
    case 1: st = launch_select<1>(c, n, d_seqs, d_budget, sinks, recent, d_weight, weight_stride, w, s); break;
    case 2: st = launch_select<2>(c, n, d_seqs, d_budget, sinks, recent, d_weight, weight_stride, w, s); break;
    case 4: st = launch_select<4>(c, n, d_seqs, d_budget, sinks, recent, d_weight, weight_stride, w, s); break;
    default: st = launch_select<8>(c, n, d_seqs, d_budget, sinks, recent, d_weight, weight_stride, w, s); break;
  }
  if (st != PCOMOE_OK) return st;
  // A column each for few blocks is walked over with 512 threads, more of its rows under way; many blocks have 256 (one sequence of 131071
  // tokens cut to a quarter in 2 layers: the whole pass 478 us, with 256 threads 513; 8 sequences of 905 to 4050 in 4 layers 171, with
  // 512 threads 186).
  const dim3 grid((unsigned)columns, 2 * c.layers, n);
  if (columns * 2 * c.layers * n <= 2 * sms) PCOMOE_CUDA_TRY(launch_pdl(evict_move_kernel<512>, grid, dim3(512), 0, s, c, d_seqs, d_weight, weight_stride, w));
  else PCOMOE_CUDA_TRY(launch_pdl(evict_move_kernel<256>, grid, dim3(256), 0, s, c, d_seqs, d_weight, weight_stride, w));
  PCOMOE_CUDA_TRY(launch_pdl(evict_book_kernel, dim3(n, (unsigned)std::min((c.max_pages + 255) / 256, 64)), dim3(256), 0, s, c, d_seqs, w));
  count_launch(3);
  return PCOMOE_OK;
}

}  // extern "C"
