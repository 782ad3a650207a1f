// What the kernels that weigh cached positions share: arguments and the sequences of a call.
#pragma once
#include <climits>

#include "cache.cuh"

namespace pcomoe {

struct WeighArgs {
  int32_t T, n, hq, hkv, g;
  float scale_log2;                     // scale * log2(e)
  const int32_t *seqs, *cu, *keep, *n_keep;
  int32_t keep_stride, fresh;
  const void *q, *k;                    // k: the layer's pool
  int64_t q_stride;                     // elements
  const float *lse;
  const int32_t *len, *table;
  int32_t pages, page, page_shift, max_seqs, max_pages;
  float *weight;
  int64_t weight_stride;
  int32_t *status;
  uint64_t limit_ns;
};

pcomoe_status launch_weigh_simt(const WeighArgs &a, int head_dim, float *partial, int64_t room, int sms, cudaStream_t st);
pcomoe_status launch_weigh_tc(const WeighArgs &a, int head_dim, float *partial, int64_t room, int sms, cudaStream_t st);
size_t weigh_part_bytes(int hkv, int64_t room, int n);       // of partial sums of n listed sequences of up to `room` positions

#ifdef __CUDACC__
namespace {

constexpr float kLog2ef = 1.4426950408889634f;

struct WeighSeq {
  int q0, n, m;         // first packed row, their number, counted ones
  int len, base, id;    // keys, position of the first counted row
};

// Which sequences a list names more than once, one bit each.  Whole block; s_bits: 2 * kMaxSeqs / 32 words.
__device__ __forceinline__ const uint32_t *find_repeats(const int32_t *seqs, int n, int max_seqs, uint32_t *s_bits) {
  uint32_t *seen = s_bits, *twice = s_bits + kMaxSeqs / 32;
  for (int i = threadIdx.x; i < 2 * (kMaxSeqs / 32); i += blockDim.x) s_bits[i] = 0u;
  __syncthreads();
  for (int i = threadIdx.x; i < n; i += blockDim.x) {
    const int id = seqs[i];
    if (id >= 0 && id < max_seqs && ((atomicOr(&seen[id >> 5], 1u << (id & 31)) >> (id & 31)) & 1u)) atomicOr(&twice[id >> 5], 1u << (id & 31));
  }
  __syncthreads();
  return twice;
}

__device__ __forceinline__ WeighSeq weigh_seq(const WeighArgs &a, int s, const uint32_t *twice) {
  WeighSeq r;
  r.q0 = a.cu[s];
  const int e = a.cu[s + 1];
  r.n = e - r.q0;
  r.id = a.seqs[s];
  r.m = a.n_keep ? a.n_keep[s] : r.n;
  bool ok = r.q0 >= 0 && r.n >= 0 && e <= a.T && r.m >= 0 && r.m <= r.n && (!a.n_keep || r.m <= a.keep_stride) && r.id >= 0 && r.id < a.max_seqs &&
            !((twice[(unsigned)r.id >> 5 & (kMaxSeqs / 32 - 1)] >> (r.id & 31)) & 1u);
  r.len = ok ? a.len[r.id] : 0;
  ok = ok && r.len >= r.m && ((r.len - 1) >> a.page_shift) < a.max_pages;
  if (!ok) atomicCAS(a.status, 0, (int)PCOMOE_ERR_INDEX);
  if (!ok || r.m == 0) r.m = r.len = r.id = 0;           // nothing is added
  r.base = r.len - r.m;
  return r;
}

// Packed row of the k-th counted row of a sequence, -1: none
__device__ __forceinline__ int counted_row(const WeighArgs &a, const WeighSeq &s, int list, int k) {
  if (!a.n_keep) return s.q0 + k;
  const int x = a.keep[(int64_t)list * a.keep_stride + k];
  if (x >= 0 && x < s.n) return s.q0 + x;
  atomicCAS(a.status, 0, (int)PCOMOE_ERR_INDEX);
  return -1;
}

// Row of head 0 of position p's page in the pool, rows of a head counted
__device__ __forceinline__ int64_t weigh_page_row(const WeighArgs &a, const int32_t *table, int p) {
  int page = table[p >> a.page_shift];
  if ((unsigned)page >= (unsigned)a.pages) {
    atomicCAS(a.status, 0, (int)PCOMOE_ERR_INDEX);
    page = 0;
  }
  return (int64_t)page * a.hkv * a.page + (p & (a.page - 1));
}

__device__ __forceinline__ float exp2_fast(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

}  // namespace
#endif

}  // namespace pcomoe
