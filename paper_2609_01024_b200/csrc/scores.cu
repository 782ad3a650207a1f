// Scores of tokens from logits: log probability of a given token, entropy, the best words, in one read of the logits.
//
// Mathematics.  With a reference m and e_i = exp(x_i - m): s = sum e_i and w = sum e_i (x_i - m) give
//   logZ = m + ln s,   H = logZ - sum p x = ln s - w / s.
// Moving the reference from m to m' multiplies s by r = exp(m - m') and turns w into r (w + s (m - m')), so both are
// kept while the maximum grows and partial results of different references join exactly.  The difference x - m is formed
// before it is scaled for the base-2 exponential, and held above -700 (exp gives 0 from -104 on): rows of the type's
// lowest value, masked words and NaN need no case of their own.
//
// Best words.  A warp reads 512 contiguous bytes of a row at a time (256 bf16 or 128 fp32 words, one 16-byte load per lane): a
// group.  The n best words under (value descending, id ascending) lie in the n best groups under (largest value
// descending, position ascending): n better groups each hold a better word.  So the pass over the row only records the
// largest value of every group, and afterwards at most n groups are read again (from L2) and ranked.
//
// What bounds it: HBM, with the exponentials close behind for bf16 (11.5 words per clock and SM at the copy rate, the
// special function unit does 16).
#include <algorithm>
#include <climits>
#include <type_traits>

#include "common.cuh"

namespace pcomoe {
namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kMaxTop = 32;
constexpr int kMaxVocab = 1 << 20;
constexpr int kMaxCand = 1024;
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLeast = -700.f;
constexpr float kNone = -INFINITY;

// Order of floats as integers (-inf lowest of what occurs here); kNoKey: nothing eligible.
__device__ __forceinline__ int key_of(float x) {
  const int b = __float_as_int(x);
  return b ^ ((b >> 31) & 0x7fffffff);
}
__device__ __forceinline__ float of_key(int k) { return __int_as_float(k ^ ((k >> 31) & 0x7fffffff)); }
constexpr int kNoKey = (int)0x807fffff;                  // key_of(-inf)

__device__ __forceinline__ float eligible(float x) { return fabsf(x) < INFINITY ? x : kNone; }

template <typename T> struct Vec;                        // words of one 16-byte load
template <> struct Vec<__nv_bfloat16> {
  static constexpr int N = 8;
  static __device__ __forceinline__ void unpack(const uint4 &v, float *x) {
    const uint32_t u[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[2 * i] = __uint_as_float(u[i] << 16);
      x[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u);
    }
  }
  static __device__ __forceinline__ float one(const __nv_bfloat16 *p) { return __bfloat162float(*p); }
};
template <> struct Vec<float> {
  static constexpr int N = 4;
  static __device__ __forceinline__ void unpack(const uint4 &v, float *x) {
    x[0] = __uint_as_float(v.x); x[1] = __uint_as_float(v.y); x[2] = __uint_as_float(v.z); x[3] = __uint_as_float(v.w);
  }
  static __device__ __forceinline__ float one(const float *p) { return *p; }
};

__device__ __forceinline__ float exp_fast(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x * kLog2e));
  return y;
}

struct Sums { float m, s, w; };                          // reference, sum, weighted sum

__device__ __forceinline__ Sums join(const Sums &a, const Sums &b) {
  if (a.s == 0.f) return b;
  if (b.s == 0.f) return a;
  const float m = fmaxf(a.m, b.m);
  const float da = fmaxf(a.m - m, kLeast), db = fmaxf(b.m - m, kLeast);
  const float ra = exp_fast(da), rb = exp_fast(db);
  return {m, a.s * ra + b.s * rb, ra * (a.w + a.s * da) + rb * (b.w + b.s * db)};
}

struct Args {
  const char *x;
  int64_t row_bytes;
  int T, V, top;
  const int32_t *tokens;
  float *logprob, *entropy, *top_lp;
  int32_t *top_ids;
};

// The words of group g that this lane holds.  Word ids begin at -shift: the row starts `shift` words after a 16-byte
// boundary, and the words before its start or past its end do not exist.
template <typename T>
__device__ __forceinline__ void load_words(const T *row, int shift, int V, int g, int lane, float *x) {
  constexpr int N = Vec<T>::N;
  const int i = (g * 32 + lane) * N - shift;
  if (i >= 0 && i + N <= V) {
    Vec<T>::unpack(__ldcs((const uint4 *)(row + i)), x);
  } else {
#pragma unroll
    for (int k = 0; k < N; ++k) x[k] = i + k >= 0 && i + k < V ? Vec<T>::one(row + i + k) : kNone;
  }
}

template <typename T, int CL>
__global__ void __launch_bounds__(kThreads) scores_kernel(Args a) {
  pdl_grid_wait();
  constexpr int N = Vec<T>::N, kUnroll = 32 / N;
  extern __shared__ int s_group[];                       // largest value of every group of this block, as keys
  __shared__ Sums s_sums[kWarps];
  __shared__ int s_pick[kMaxTop], s_ckey[kMaxCand], s_cid[kMaxCand], s_nc;
  __shared__ struct { Sums sums; int key[kMaxTop], id[kMaxTop]; } s_out;      // what the cluster's first block collects
  __shared__ float s_m, s_lns;                           // log p = (x - m) - ln s: exact where x is near the largest
  __shared__ int s_count[kWarps];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int rank = CL > 1 ? (int)(blockIdx.x % CL) : 0;
  const int t = blockIdx.x / CL;
  const T *row = (const T *)(a.x + (int64_t)t * a.row_bytes);
  const int shift = (int)(((uintptr_t)row & 15) / sizeof(T));
  const int groups = (a.V + shift + 32 * N - 1) / (32 * N);
  const int per = (groups + CL - 1) / CL;
  const int g0 = min(rank * per, groups), g1 = min(g0 + per, groups);

  Sums acc = {0.f, 0.f, 0.f};                            // of this lane; the reference is the warp's
  bool first = true;
  for (int g = g0 + warp * kUnroll; g < g1; g += kWarps * kUnroll) {
    float x[kUnroll][N];
    int most = kNoKey;
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      if (g + u < g1) {
        load_words<T>(row, shift, a.V, g + u, lane, x[u]);
      } else {
#pragma unroll
        for (int k = 0; k < N; ++k) x[u][k] = kNone;
      }
    }
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      float mx = x[u][0];
#pragma unroll
      for (int k = 1; k < N; ++k) mx = fmaxf(mx, x[u][k]);
      int key = __reduce_max_sync(~0u, mx == mx ? key_of(mx) : kNoKey);
      if (key >= key_of(INFINITY)) {                     // an infinite logit: it does not count
        mx = kNone;
#pragma unroll
        for (int k = 0; k < N; ++k) {
          x[u][k] = eligible(x[u][k]);
          mx = fmaxf(mx, x[u][k]);
        }
        key = __reduce_max_sync(~0u, key_of(mx));
      }
      if (lane == 0 && g + u < g1) s_group[g + u - g0] = key;
      most = max(most, key);
    }
    if (most == kNoKey) continue;
    const float m = of_key(most);
    if (first || m > acc.m) {
      if (!first) {
        const float d = fmaxf(acc.m - m, kLeast), r = exp_fast(d);
        acc.w = r * (acc.w + acc.s * d);
        acc.s *= r;
      }
      acc.m = m;
      first = false;
    }
#pragma unroll
    for (int u = 0; u < kUnroll; ++u)
#pragma unroll
      for (int k = 0; k < N; ++k) {
        const float d = fmaxf(x[u][k] - acc.m, kLeast);
        const float e = exp_fast(d);
        acc.s += e;
        acc.w = fmaf(e, d, acc.w);
      }
  }
#pragma unroll
  for (int o = 16; o; o >>= 1) {
    acc.s += __shfl_xor_sync(~0u, acc.s, o);
    acc.w += __shfl_xor_sync(~0u, acc.w, o);
  }
  if (lane == 0) s_sums[warp] = acc;
  if (tid == 0) s_nc = 0;
  __syncthreads();

  const int G = g1 - g0, want = a.top;
  if (warp == 0) {
    if (lane == 0) {
      Sums all = s_sums[0];
      for (int i = 1; i < kWarps; ++i) all = join(all, s_sums[i]);
      s_out.sums = all;
    }
    // the `want` best groups, one after another: every lane knows its best one (lane, lane + 32, ...)
    if (want) {
      int best = kNoKey, at = INT_MAX;
      for (int g = lane; g < G; g += 32)
        if (s_group[g] > best) { best = s_group[g]; at = g; }
      for (int i = 0; i < want; ++i) {
        const int top = __reduce_max_sync(~0u, best);
        const int pick = (int)__reduce_min_sync(~0u, best == top && top != kNoKey ? (unsigned)at : (unsigned)INT_MAX);
        if (lane == 0) s_pick[i] = pick == INT_MAX ? -1 : pick;
        if (pick == INT_MAX) continue;
        if (at == pick) {                                // the next best of this lane: lower, or equal and further on
          int b2 = kNoKey, a2 = INT_MAX;
          for (int g = lane; g < G; g += 32) {
            const int k = s_group[g];
            if ((k < best || (k == best && g > at)) && k > b2) { b2 = k; a2 = g; }
          }
          best = b2;
          at = a2;
        }
      }
    }
  }
  if (want) {
    __syncthreads();
    // every word of the picked groups that reaches the last picked group's largest value may be among the best
    int n_pick = 0;
    while (n_pick < want && s_pick[n_pick] >= 0) ++n_pick;
    int floor_key = n_pick ? s_group[s_pick[n_pick - 1]] : INT_MAX;
    if (n_pick && n_pick < want) {
      // fewer groups than ranks: the same bound from single lanes' words, by bisection of the key (the largest key that
      // at least `want` lanes reach)
      constexpr int kMine = kMaxTop / kWarps;
      int most[kMine];
#pragma unroll
      for (int q = 0; q < kMine; ++q) {
        most[q] = kNoKey;
        if (warp + q * kWarps < n_pick) {
          float x[N];
          load_words<T>(row, shift, a.V, g0 + s_pick[warp + q * kWarps], lane, x);
#pragma unroll
          for (int k = 0; k < N; ++k) most[q] = max(most[q], key_of(eligible(x[k])));
        }
      }
      int64_t lo = kNoKey + 1, hi = (int64_t)key_of(INFINITY);          // reached by enough lanes (or the least); not reached
      while (hi - lo > 1) {
        const int64_t mid = (lo + hi) >> 1;
        int mine = 0;
#pragma unroll
        for (int q = 0; q < kMine; ++q) mine += most[q] >= mid;
        int all = __reduce_add_sync(~0u, mine);
        if (lane == 0) s_count[warp] = all;
        __syncthreads();
        all = 0;
        for (int q = 0; q < kWarps; ++q) all += s_count[q];
        __syncthreads();
        if (all >= want) lo = mid; else hi = mid;
      }
      floor_key = (int)lo;
    }
    for (int i = warp; i < n_pick; i += kWarps) {
      float x[N];
      const int g = g0 + s_pick[i];
      load_words<T>(row, shift, a.V, g, lane, x);
#pragma unroll
      for (int k = 0; k < N; ++k) {
        const int key = key_of(eligible(x[k]));
        if (key >= floor_key) {
          const int c = atomicAdd(&s_nc, 1);
          if (c < kMaxCand) {
            s_ckey[c] = key;
            s_cid[c] = (g * 32 + lane) * N - shift + k;
          }
        }
      }
    }
    if (tid < want) { s_out.key[tid] = kNoKey; s_out.id[tid] = -1; }
    __syncthreads();
    const int nc = s_nc;
    if (nc <= kMaxCand) {
      for (int c = tid; c < nc; c += kThreads) {
        const int key = s_ckey[c], id = s_cid[c];
        int r = 0;
        for (int j = 0; j < nc && r < want; ++j) r += s_ckey[j] > key || (s_ckey[j] == key && s_cid[j] < id);
        if (r < want) { s_out.key[r] = key; s_out.id[r] = id; }
      }
    } else if (warp == 0) {
      // more equals than there is room for: rank after rank, the best word behind the last one in the order
      int pk = INT_MAX, pid = -1;
      for (int i = 0; i < want; ++i) {
        int bk = kNoKey, bid = INT_MAX;
        for (int p = 0; p < n_pick; ++p) {
          float x[N];
          const int g = g0 + s_pick[p];
          load_words<T>(row, shift, a.V, g, lane, x);
#pragma unroll
          for (int k = 0; k < N; ++k) {
            const int key = key_of(eligible(x[k])), id = (g * 32 + lane) * N - shift + k;
            if (key != kNoKey && (key < pk || (key == pk && id > pid)) && (key > bk || (key == bk && id < bid))) { bk = key; bid = id; }
          }
        }
        const int top = __reduce_max_sync(~0u, bk);
        const int id = (int)__reduce_min_sync(~0u, bk == top ? (unsigned)bid : (unsigned)INT_MAX);
        if (top == kNoKey) break;
        if (lane == 0) { s_out.key[i] = top; s_out.id[i] = id; }
        pk = top;
        pid = id;
      }
    }
  }

  if (CL > 1) {
    asm volatile("barrier.cluster.arrive.aligned;\n\tbarrier.cluster.wait.aligned;" ::: "memory");
    if (rank == 0) {
      // the blocks' sums in rank order; their best words ranked against one another
      if (tid == 0) s_nc = 0;
      __syncthreads();
      auto remote = [](const void *p, int r) {
        uint32_t l = (uint32_t)__cvta_generic_to_shared(p), q;
        asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(q) : "r"(l), "r"(r));
        return q;
      };
      auto ld = [](uint32_t p) {
        int v;
        asm volatile("ld.shared::cluster.b32 %0, [%1];" : "=r"(v) : "r"(p));
        return v;
      };
      if (tid == 0) {
        Sums all = s_out.sums;
        for (int r = 1; r < CL; ++r) {
          const uint32_t q = remote(&s_out.sums, r);
          all = join(all, Sums{__int_as_float(ld(q)), __int_as_float(ld(q + 4)), __int_as_float(ld(q + 8))});
        }
        s_sums[0] = all;
      }
      for (int i = tid; i < CL * want; i += kThreads) {
        s_ckey[i] = ld(remote(&s_out.key[i % want], i / want));
        s_cid[i] = ld(remote(&s_out.id[i % want], i / want));
      }
      __syncthreads();
      if (tid == 0) s_out.sums = s_sums[0];
      int key = kNoKey, id = -1, r = want;
      const int c = tid;
      static_assert(8 * kMaxTop <= kThreads, "a thread per candidate");
      if (c < CL * want && (key = s_ckey[c]) != kNoKey) {
        id = s_cid[c];
        r = 0;
        for (int j = 0; j < CL * want; ++j) r += s_ckey[j] > key || (s_ckey[j] == key && s_cid[j] < id && s_cid[j] >= 0);
      }
      // this block's own list is read by nobody else, and by its own threads before the barrier above
      if (tid < want) { s_out.key[tid] = kNoKey; s_out.id[tid] = -1; }
      __syncthreads();
      if (r < want) { s_out.key[r] = key; s_out.id[r] = id; }
    }
    asm volatile("barrier.cluster.arrive.aligned;\n\tbarrier.cluster.wait.aligned;" ::: "memory");
    if (rank != 0) return;
  }
  __syncthreads();
  if (tid == 0) {
    const Sums all = s_out.sums;
    const bool any = all.s > 0.f;
    const float ln_s = logf(all.s);
    s_m = any ? all.m : 0.f;
    s_lns = any ? ln_s : 0.f;
    if (a.entropy) a.entropy[t] = any ? ln_s - all.w / all.s : 0.f;
    if (a.logprob) {
      const int tok = a.tokens[t];
      float lp = 0.f;
      if (tok >= a.V) lp = NAN;
      else if (tok >= 0) lp = eligible(Vec<T>::one(row + tok)) - s_m - s_lns;
      a.logprob[t] = lp;
    }
  }
  __syncthreads();
  if (tid < want) {
    const int key = s_out.key[tid];
    a.top_ids[(int64_t)t * want + tid] = s_out.id[tid];
    a.top_lp[(int64_t)t * want + tid] = key == kNoKey ? kNone : of_key(key) - s_m - s_lns;
  }
}

template <typename T, int CL>
cudaError_t launch(const Args &a, size_t smem, cudaStream_t st) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)a.T * CL);
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim = {CL, 1, 1};
  cfg.attrs = attr;
  cfg.numAttrs = CL > 1 ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, scores_kernel<T, CL>, a);
}

template <typename T>
pcomoe_status run(const Args &a, int sms, cudaStream_t st) {
  const int groups = (a.V + 15) / (32 * Vec<T>::N) + 1;
  // blocks per row: enough rows fill the GPU by themselves; few rows are cut while a block keeps 16 groups
  int cl = 1;
  while (cl < 8 && (int64_t)a.T * cl < 2 * sms && groups / (2 * cl) >= 16) cl *= 2;
  const size_t smem = sizeof(int) * (size_t)((groups + cl - 1) / cl + 1);
  switch (cl) {
    case 1: PCOMOE_CUDA_TRY((launch<T, 1>(a, smem, st))); break;
    case 2: PCOMOE_CUDA_TRY((launch<T, 2>(a, smem, st))); break;
    case 4: PCOMOE_CUDA_TRY((launch<T, 4>(a, smem, st))); break;
    default: PCOMOE_CUDA_TRY((launch<T, 8>(a, smem, st)));
  }
  count_launch();
  return PCOMOE_OK;
}

}  // namespace
}  // namespace pcomoe

using namespace pcomoe;

extern "C" pcomoe_status pcomoe_token_logprobs(int32_t dtype, int32_t T, int32_t V, const void *d_logits, int64_t row_stride,
                                               const int32_t *d_tokens, int32_t top_n, float *d_logprob, float *d_entropy,
                                               int32_t *d_top_ids, float *d_top_logprob, void *stream) {
  if (dtype != PCOMOE_BF16 && dtype != PCOMOE_FP32) return PCOMOE_ERR_INVALID_ARG;
  if (T < 0 || V <= 0 || top_n < 0 || top_n > kMaxTop) return PCOMOE_ERR_SHAPE;
  if (V > kMaxVocab) return PCOMOE_ERR_UNSUPPORTED;
  if (T == 0) return PCOMOE_OK;
  const int64_t e = (int64_t)dtype_size(dtype);
  if (!d_logits || row_stride < V || (top_n > 0 && (!d_top_ids || !d_top_logprob)) || (d_tokens && !d_logprob) ||
      (!d_tokens && d_logprob) || ((uintptr_t)d_logits % e))
    return PCOMOE_ERR_INVALID_ARG;
  if ((int64_t)T * 8 > INT32_MAX) return PCOMOE_ERR_SHAPE;
  int sms;
  pcomoe_status st = current_sms(&sms);
  if (st != PCOMOE_OK) return st;
  const Args a = {(const char *)d_logits, row_stride * e, T, V, top_n, d_tokens, d_logprob, d_entropy, d_top_logprob, d_top_ids};
  return dtype == PCOMOE_BF16 ? run<__nv_bfloat16>(a, sms, (cudaStream_t)stream) : run<float>(a, sms, (cudaStream_t)stream);
}
