// What the kernels that work on a paged cache share: its limits, its description on the device, the status word, the
// checks of a call's list, pages that a shortened sequence gives back.
#pragma once
#include "common.cuh"

namespace pcomoe {
namespace {

constexpr int kMaxSeqs = 4096;
constexpr int kMaxPages = 1 << 18;       // a call's page count over kMaxSeqs sequences stays inside 31 bits

struct CacheHeader {              // start of the workspace
  int32_t reserved[8];
  int32_t status;                 // first device error, cleared by pcomoe_device_status (the place of the router's word)
  int32_t n_moves;                // pages that the copy kernel moves
};
static_assert(offsetof(CacheHeader, status) == offsetof(DevPlan, status_router), "status word");

inline size_t align256(size_t x) { return (x + 255) & ~size_t(255); }

// What the kernels need of a pcomoe_cache.
struct CacheDev {
  int32_t layers, pages, page, shift, kv_heads, max_seqs, max_pages;
  int32_t chunks;                 // 16-byte pieces of a row of one head
  char *k, *v;
  int32_t *len, *ref, *table;
  int64_t page_bytes;             // of one layer, K or V
};

inline CacheDev cache_dev(const pcomoe_cache *c) {
  CacheDev d;
  d.layers = c->layers; d.pages = c->pages; d.page = c->page_size; d.kv_heads = c->kv_heads;
  d.max_seqs = c->max_seqs; d.max_pages = c->max_pages;
  d.shift = 0;
  while ((1 << d.shift) < c->page_size) ++d.shift;
  const int64_t row = (int64_t)c->head_dim * (int64_t)dtype_size(c->dtype);
  d.chunks = (int32_t)(row / 16);
  d.k = (char *)c->d_k; d.v = (char *)c->d_v;
  d.len = c->d_seq_len; d.ref = c->d_page_ref; d.table = c->d_page_table;
  d.page_bytes = row * c->kv_heads * c->page_size;
  return d;
}

__device__ __forceinline__ void flag(CacheHeader *h, int32_t st) { atomicCAS(&h->status, 0, st); }
__device__ __forceinline__ int pages_of(const CacheDev &c, int n) { return (n + c.page - 1) >> c.shift; }

// Whether entry i of a list names a sequence in range that no other entry names.  Whole block.
__device__ inline bool alone(const int32_t *seqs, int n, int i, int max_seqs) {
  const int id = seqs[i];
  int bad = id < 0 || id >= max_seqs;
  for (int j = threadIdx.x; j < n; j += blockDim.x) bad |= j != i && seqs[j] == id;
  return !__syncthreads_or(bad);
}

// (by one block, or by several that start and step as far apart)
__device__ inline void drop_pages(const CacheDev &c, int id, int old_len, int new_len, int start = 0, int step = 0) {
  const int m = min(pages_of(c, old_len), c.max_pages);
  for (int s = pages_of(c, new_len) + start + threadIdx.x; s < m; s += step ? step : blockDim.x) {
    int32_t *e = &c.table[(int64_t)id * c.max_pages + s];
    if (*e >= 0 && *e < c.pages) atomicSub(&c.ref[*e], 1);
    *e = -1;
  }
}

}  // namespace
}  // namespace pcomoe
