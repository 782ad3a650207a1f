// Scores of tokens from logits: log probability of a given token, entropy, the best words, in one read of the logits.
//
// Mathematics, base 2 (c = log2 e).  With a reference word m, M = c m rounded, r = c m - M, and d_i = c x_i - M, formed by one
// FMA: s = sum 2^d_i and w = sum 2^d_i d_i give
//   log p_i = (x_i - m) + ln 2 (r - log2 s),   H = ln 2 (log2 s - w / s).
// Moving the reference by D (from m to m': D = c (m - m') - r + r') multiplies s by 2^D and turns w into 2^D (w + s D), so
// both are kept while the maximum grows and partial results of different references join.  A d_i far below the reference
// must not be -inf (0 times it is NaN): words are held above -1e30 first, NaN and -inf with them (two bf16 in one operation).
// Rows whose maximum is 1e6 or more away from zero (a mask's lowest value, say) take d_i = c (x_i - m) instead, with r = 0.
//
// Best words.  A warp reads 512 contiguous bytes of a row at a time (256 bf16 or 128 fp32 words, one 16-byte load per lane): a
// group.  The n best words under (value descending, id ascending) lie in the n best groups under (largest value
// descending, position ascending): n better groups each hold a better word.  So the pass over the row only records the
// largest value of every group, and afterwards at most n groups are read again (from L2) and ranked.
//
// What bounds it: HBM, with the exponentials close behind for bf16 (11.5 words per clock and SM at the copy rate, the
// special function unit does 16).  What comes after the pass over a row is a chain of short steps that few threads take
// part in, so with many rows a row belongs to two or four warps and other rows' passes fill the gaps; with fewer rows to a
// block or to a cluster of up to 16 blocks.  Measured, bf16: 4096 rows of 32000 words 57 us, 4.6 TB/s (the issue slots 70 %
// busy, the special function unit 56 %, and teams that wait for the last rows); 4 rows of 128000 words 6.4 us; fp32: 1000
// rows of 128000 words 84 us, 6.1 TB/s.
#include <algorithm>
#include <climits>
#include <type_traits>

#include "words.cuh"

namespace pcomoe {
namespace {

constexpr int kMaxTop = 32;
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
  uint64_t d;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(*(uint64_t *)&a), "l"(*(uint64_t *)&b), "l"(*(uint64_t *)&c));
  return *(float2 *)&d;
}
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
  uint64_t d;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(*(uint64_t *)&a), "l"(*(uint64_t *)&b));
  return *(float2 *)&d;
}
struct Sums { float m, s, w; };                          // reference, sum, weighted sum

__device__ __forceinline__ bool plain_range(float m) { return fabsf(m) < 1e6f; }
__device__ __forceinline__ float rest(float m) { return plain_range(m) ? fmaf(m, kLog2e, -(m * kLog2e)) : 0.f; }
// by how much sums over reference `from` are lower over reference `to` (0 or less, and never -inf)
__device__ __forceinline__ float shift_of(float from, float to) { return fmaxf(fmaf(from - to, kLog2e, rest(to) - rest(from)), -1000.f); }

__device__ __forceinline__ Sums join(const Sums &a, const Sums &b) {
  if (a.s == 0.f) return b;
  if (b.s == 0.f) return a;
  const float m = fmaxf(a.m, b.m);
  const float da = shift_of(a.m, m), db = shift_of(b.m, m);
  const float ra = ex2(da), rb = ex2(db);
  return {m, a.s * ra + b.s * rb, ra * (a.w + a.s * da) + rb * (b.w + b.s * db)};
}

struct Args {
  const char *x;
  int64_t row_bytes;
  int T, V, top;
  int group_room;                                        // places of a team's group list
  const int32_t *tokens;
  float *logprob, *entropy, *top_lp;
  int32_t *top_ids;
};

// W warps (a team) per row and block-wide share of it, CL blocks (a cluster) per row; W < kWarps only with CL = 1, where
// a block holds several teams.
template <typename T, int kWarps, int W, int CL>
__global__ void __launch_bounds__(32 * kWarps) scores_kernel(Args a) {
  pdl_grid_wait();
  constexpr int N = Vec<T>::N, kLoads = 4, kTeams = kWarps / W, kThreads = 32 * W;      // threads of a team
  constexpr int kMaxCand = 1024 / kTeams > 512 ? 512 : 1024 / kTeams;
  static_assert(W == kWarps || CL == 1, "teams or clusters");
  extern __shared__ int s_all_groups[];                  // largest value of every group of this block's share, as keys
  struct Team {
    Sums sums[W];
    unsigned long long cand[kMaxCand];
    int pick[kMaxTop], nc, floor_key;
    struct { Sums sums; int key[kMaxTop], id[kMaxTop]; } out;      // what the cluster's first block collects
    float m, tail;                                       // reference, ln 2 (r - log2 s)
  };
  __shared__ Team s_team[kTeams];
  const int lane = threadIdx.x & 31, team = (threadIdx.x >> 5) / W, warp = (threadIdx.x >> 5) % W, tid = warp * 32 + lane;
  Team &s = s_team[team];
  auto sync = [&]() {
    if (W == kWarps) __syncthreads();
    else asm volatile("bar.sync %0, %1;" ::"r"(1 + team), "n"(kThreads) : "memory");
  };
  const int rank = CL > 1 ? (int)(blockIdx.x % CL) : 0;
  const int t = blockIdx.x / CL * kTeams + team;
  if (t >= a.T) return;                                  // a whole team (never with CL > 1)
  const T *row = (const T *)(a.x + (int64_t)t * a.row_bytes);
  const int shift = (int)(((uintptr_t)row & 15) / sizeof(T));
  const int groups = (a.V + shift + 32 * N - 1) / (32 * N);
  const int per = (groups + CL - 1) / CL;
  const int g0 = min(rank * per, groups), g1 = min(g0 + per, groups), G = g1 - g0;
  int *s_group = s_all_groups + team * a.group_room;

  Sums acc = {0.f, 0.f, 0.f};                            // of this lane; the reference is the warp's
  float most_so_far = kNone;
  uint4 raw[kLoads];
  auto fetch = [&](int g) {
    // all inside the row: no lane looks at its place
    if (g * 32 * N >= shift && (g + kLoads) * 32 * N - shift <= a.V && g + kLoads <= g1) {
      const uint4 *p = (const uint4 *)(row - shift) + g * 32 + lane;
#pragma unroll
      for (int u = 0; u < kLoads; ++u) raw[u] = __ldcs(p + 32 * u);
    } else {
      float none[N];
#pragma unroll
      for (int k = 0; k < N; ++k) none[k] = kNone;
#pragma unroll
      for (int u = 0; u < kLoads; ++u) raw[u] = g + u < g1 ? load_raw<T>(row, shift, a.V, g + u, lane) : Vec<T>::pack(none);
    }
  };
  int g = g0 + warp * kLoads;
  if (g < g1) fetch(g);
  for (; g < g1; g += W * kLoads) {
    uint4 v[kLoads];
#pragma unroll
    for (int u = 0; u < kLoads; ++u) v[u] = raw[u];
    if (g + W * kLoads < g1) fetch(g + W * kLoads);      // on its way while this one is summed
    int key[kLoads];
#pragma unroll
    for (int u = 0; u < kLoads; ++u) key[u] = __reduce_max_sync(~0u, key_of(Vec<T>::largest(v[u])));
    int most = max(max(key[0], key[1]), max(key[2], key[3]));
    if (most >= key_of(INFINITY)) {                      // infinite logits (or nothing but NaN in a lane): they do not count
#pragma unroll
      for (int u = 0; u < kLoads; ++u) {
        float x[N];
        Vec<T>::unpack(v[u], x);
#pragma unroll
        for (int k = 0; k < N; ++k) x[k] = eligible(x[k]);
        v[u] = Vec<T>::pack(x);
        key[u] = __reduce_max_sync(~0u, key_of(Vec<T>::largest(v[u])));
      }
      most = max(max(key[0], key[1]), max(key[2], key[3]));
    }
    static_assert(kLoads == 4, "a lane per group of the iteration");
    if (lane < kLoads && g + lane < g1)                  // (a NaN's key may lie below -inf's)
      s_group[g + lane - g0] = max(lane < 2 ? (lane ? key[1] : key[0]) : (lane == 2 ? key[2] : key[3]), kNoKey);
    if (most <= kNoKey) continue;
    const float m = of_key(most);
    if (m > most_so_far) {
      if (acc.s > 0.f) {
        const float d = shift_of(acc.m, m), r = ex2(d);
        acc.w = r * (acc.w + acc.s * d);
        acc.s *= r;
      }
      acc.m = most_so_far = m;
    }
    if (plain_range(acc.m)) {
      const float2 c = make_float2(kLog2e, kLog2e), minus = make_float2(-(acc.m * kLog2e), -(acc.m * kLog2e));
      float2 s2[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)}, w2[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
#pragma unroll
      for (int u = 0; u < kLoads; ++u) {
        float2 x[N / 2];
        Vec<T>::pairs(v[u], x);
#pragma unroll
        for (int k = 0; k < N / 2; ++k) {
          const float2 d = fma2(x[k], c, minus);
          const float2 e = make_float2(ex2(d.x), ex2(d.y));
          s2[k & 1] = add2(s2[k & 1], e);
          w2[k & 1] = fma2(e, d, w2[k & 1]);
        }
      }
      const float2 st = add2(s2[0], s2[1]), wt = add2(w2[0], w2[1]);
      acc.s += st.x + st.y;
      acc.w += wt.x + wt.y;
    } else {
#pragma unroll
      for (int u = 0; u < kLoads; ++u) {
        float x[N];
        Vec<T>::unpack(v[u], x);
#pragma unroll
        for (int k = 0; k < N; ++k) {
          const float d = fmaxf((eligible(x[k]) - acc.m) * kLog2e, -1000.f);
          const float e = ex2(d);
          acc.s += e;
          acc.w = fmaf(e, d, acc.w);
        }
      }
    }
  }
#pragma unroll
  for (int o = 16; o; o >>= 1) {
    acc.s += __shfl_xor_sync(~0u, acc.s, o);
    acc.w += __shfl_xor_sync(~0u, acc.w, o);
  }
  if (lane == 0) s.sums[warp] = acc;
  if (tid == 0) s.nc = 0;
  const int want = a.top;
  if (tid < want) { s.pick[tid] = -1; s.out.key[tid] = kNoKey; s.out.id[tid] = -1; }
  sync();

  if (warp == W - 1) {
    // the warps' sums, pairwise in a fixed order
    Sums all = lane < W ? s.sums[lane] : Sums{0.f, 0.f, 0.f};
#pragma unroll
    for (int o = 1; o < W; o <<= 1) all = join(all, Sums{__shfl_down_sync(~0u, all.m, o), __shfl_down_sync(~0u, all.s, o), __shfl_down_sync(~0u, all.w, o)});
    if (lane == 0) s.out.sums = all;
  }
  if (want) {
    // the `want` best groups
    if (W >= 8 && G <= 4 * kThreads) {
      // by counting the better ones
      for (int g = tid; g < G; g += kThreads) {
        const int key = s_group[g];
        if (key == kNoKey) continue;
        int r = 0;
#pragma unroll 8
        for (int j = 0; j < G; ++j) {
          const int k = s_group[j];
          r += k > key || (k == key && j < g);
        }
        if (r < want) s.pick[r] = g;
      }
    } else if (warp == 0) {
      // one after another: every lane knows its best one of lane, lane + 32, ...
      int best = kNoKey, at = INT_MAX;
      for (int g = lane; g < G; g += 32)
        if (s_group[g] > best) { best = s_group[g]; at = g; }
      for (int i = 0; i < want; ++i) {
        const int top = __reduce_max_sync(~0u, best);
        const int pick = (int)__reduce_min_sync(~0u, best == top && top != kNoKey ? (unsigned)at : (unsigned)INT_MAX);
        if (pick == INT_MAX) break;
        if (lane == 0) s.pick[i] = pick;
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
    sync();
    // every word of the picked groups that reaches the last picked group's largest value may be among the best
    int n_pick = 0;
    while (n_pick < want && s.pick[n_pick] >= 0) ++n_pick;
    int floor_key = n_pick ? s_group[s.pick[n_pick - 1]] : INT_MAX;
    if (n_pick && n_pick < want) {
      // fewer groups than ranks: the same bound from parts of the groups, 65 to 128 of them (or single lanes'), by counting
      int per_group = 32;
      while (n_pick * per_group > 128) per_group >>= 1;
      int *part = (int *)s.cand;                         // not in use yet
      static_assert(sizeof(s.cand) >= 128 * sizeof(int), "room for the parts");
      for (int i = warp; i < n_pick; i += W) {
        float x[N];
        load_words<T>(row, shift, a.V, g0 + s.pick[i], lane, x);
        int most = kNoKey;
#pragma unroll
        for (int k = 0; k < N; ++k) most = max(most, key_of(eligible(x[k])));
        for (int o = 32 / per_group / 2; o; o >>= 1) most = max(most, __shfl_xor_sync(~0u, most, o));
        const int lanes = 32 / per_group;
        if (lane % lanes == 0) part[i * per_group + lane / lanes] = most;
      }
      if (tid == 0) s.floor_key = kNoKey + 1;            // where fewer parts than ranks have an eligible word: all words
      sync();
      for (int e = tid; e < n_pick * per_group; e += kThreads) {
        const int key = part[e];
        int r = 0;
#pragma unroll 8
        for (int j = 0; j < n_pick * per_group; ++j) r += part[j] > key || (part[j] == key && j < e);
        if (r == want - 1 && key != kNoKey) s.floor_key = key;
      }
      sync();
      floor_key = s.floor_key;
    }
#pragma unroll 4
    for (int i = warp; i < n_pick; i += W) {
      float x[N];
      const int g = g0 + s.pick[i];
      load_words<T>(row, shift, a.V, g, lane, x);
#pragma unroll
      for (int k = 0; k < N; ++k) {
        const int key = key_of(eligible(x[k]));
        if (key >= floor_key) {
          const int c = atomicAdd(&s.nc, 1);
          if (c < kMaxCand) s.cand[c] = place_of(key, (g * 32 + lane) * N - shift + k);
        }
      }
    }
    sync();
    const int nc = s.nc;
    if (nc <= kMaxCand) {
      for (int c = tid; c < nc; c += kThreads) {
        const unsigned long long p = s.cand[c];
        int r = 0;
#pragma unroll 8
        for (int j = 0; j < nc; ++j) r += s.cand[j] > p;
        if (r < want) { s.out.key[r] = place_key(p); s.out.id[r] = place_id(p); }
      }
    } else if (warp == 0) {
      // more equals than there is room for: rank after rank, the best word behind the last one in the order
      int pk = INT_MAX, pid = -1;
      for (int i = 0; i < want; ++i) {
        int bk = kNoKey, bid = INT_MAX;
        for (int p = 0; p < n_pick; ++p) {
          float x[N];
          const int g = g0 + s.pick[p];
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
        if (lane == 0) { s.out.key[i] = top; s.out.id[i] = id; }
        pk = top;
        pid = id;
      }
    }
  }

  if (CL > 1) {
    asm volatile("barrier.cluster.arrive.aligned;\n\tbarrier.cluster.wait.aligned;" ::: "memory");
    if (rank == 0) {
      // the blocks' sums in rank order; their best words ranked against one another
      static_assert(CL == 1 || (CL * kMaxTop <= kThreads && CL * kMaxTop <= kMaxCand), "a thread per candidate");
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
      if (warp == W - 1) {
        Sums mine = {0.f, 0.f, 0.f};
        if (lane < CL) {
          const uint32_t q = remote(&s.out.sums, lane);
          mine = Sums{__int_as_float(ld(q)), __int_as_float(ld(q + 4)), __int_as_float(ld(q + 8))};
        }
#pragma unroll
        for (int o = 1; o < CL; o <<= 1) mine = join(mine, Sums{__shfl_down_sync(~0u, mine.m, o), __shfl_down_sync(~0u, mine.s, o), __shfl_down_sync(~0u, mine.w, o)});
        if (lane == 0) s.sums[0] = mine;
      }
      // a thread per candidate; blocks without enough words have (kNoKey, -1) in the rest of their lists
      unsigned long long place = 0;
      if (tid < CL * want) {
        const int r = tid / want, i = tid - r * want;
        const uint32_t q = remote(&s.out.key[i], r);
        const int key = ld(q), id = ld(q + (uint32_t)sizeof(s.out.key));
        place = key == kNoKey ? 0 : place_of(key, id);
        s.cand[tid] = place;
      }
      __syncthreads();
      if (tid == 0) s.out.sums = s.sums[0];
      int r = want;
      if (place) {
        r = 0;
#pragma unroll 8
        for (int j = 0; j < CL * want; ++j) r += s.cand[j] > place;
      }
      // this block's own list is read by nobody else, and by its own threads before the barrier above
      if (tid < want) { s.out.key[tid] = kNoKey; s.out.id[tid] = -1; }
      __syncthreads();
      if (r < want) { s.out.key[r] = place_key(place); s.out.id[r] = place_id(place); }
    }
    asm volatile("barrier.cluster.arrive.aligned;\n\tbarrier.cluster.wait.aligned;" ::: "memory");
    if (rank != 0) return;
  }
  sync();
  if (tid == 0) {
    const Sums all = s.out.sums;
    const bool any = all.s > 0.f;
    const float log2s = any ? log2f(all.s) : 0.f;
    s.m = any ? all.m : 0.f;
    s.tail = any ? kLn2 * (rest(all.m) - log2s) : 0.f;
    if (a.entropy) a.entropy[t] = any ? kLn2 * (log2s - all.w / all.s) : 0.f;
    if (a.logprob) {
      const int tok = a.tokens[t];
      float lp = 0.f;
      if (tok >= a.V) lp = NAN;
      else if (tok >= 0) lp = (eligible(Vec<T>::one(row + tok)) - s.m) + s.tail;
      a.logprob[t] = lp;
    }
  }
  sync();
  if (tid < want) {
    const int key = s.out.key[tid];
    a.top_ids[(int64_t)t * want + tid] = s.out.id[tid];
    a.top_lp[(int64_t)t * want + tid] = key == kNoKey ? kNone : (of_key(key) - s.m) + s.tail;
  }
}

template <typename T, int kWarps, int W, int CL>
struct Launch {
  cudaLaunchConfig_t cfg = {};
  cudaLaunchAttribute attr[2];
  Launch(int rows, int group_room, cudaStream_t st) {
    constexpr int kTeams = kWarps / W;
    cfg.gridDim = dim3((unsigned)((rows + kTeams - 1) / kTeams * CL));
    cfg.blockDim = dim3(32 * kWarps);
    cfg.dynamicSmemBytes = sizeof(int) * (size_t)group_room * kTeams;
    cfg.stream = st;
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim = {CL, 1, 1};
    cfg.attrs = attr;
    cfg.numAttrs = CL > 1 ? 2 : 1;
  }
};

template <typename T, int kWarps, int W, int CL>
pcomoe_status launch(Args a, int groups, cudaStream_t st) {
  a.group_room = (groups + CL - 1) / CL;
  const Launch<T, kWarps, W, CL> l(a.T, a.group_room, st);
  PCOMOE_CUDA_TRY((cudaLaunchKernelEx(&l.cfg, scores_kernel<T, kWarps, W, CL>, a)));
  count_launch();
  return PCOMOE_OK;
}

// Whether clusters of 16 blocks find room on the current device, which 8 always do: asked once for each device.
template <typename T>
bool room_for_16() {
  static std::atomic<uint64_t> asked{0}, room{0};
  int dev = -1;
  if (cudaGetDevice(&dev) != cudaSuccess) return false;
  const uint64_t bit = dev >= 0 && dev < 64 ? uint64_t(1) << dev : 0;
  if (asked.load(std::memory_order_acquire) & bit) return (room.load(std::memory_order_relaxed) & bit) != 0;
  const Launch<T, 16, 16, 16> l(1, kMaxVocab / (32 * Vec<T>::N) / 16 + 1, nullptr);
  int clusters = 0;
  const bool ok = cudaFuncSetAttribute(scores_kernel<T, 16, 16, 16>, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) == cudaSuccess &&
                  cudaOccupancyMaxActiveClusters(&clusters, scores_kernel<T, 16, 16, 16>, &l.cfg) == cudaSuccess && clusters > 0;
  if (!ok) cudaGetLastError();                             // the answer is no, not an error of a later call
  if (ok) room.fetch_or(bit, std::memory_order_relaxed);
  asked.fetch_or(bit, std::memory_order_release);
  return ok;
}

template <typename T>
pcomoe_status run(const Args &a, int sms, cudaStream_t st) {
  const int groups = (a.V + 15) / (32 * Vec<T>::N) + 1;
  // Teams of 1, 2 or 4 warps where there are rows enough to fill the GPU with them (a team's group list stays inside 24 KB
  // per block).  bf16, 5 best words:
  //   rows of at most 16 groups, where what follows the pass over a row counts most: one warp (2400 rows of 2000 words:
  //   11.9 us, two warps 15.2; of 8000 words 22.5 us, two warps 19.8);
  //   48 warps per SM with teams of two: these (4000 rows of 32000 words: 55 us, one warp 63; 3000 rows, teams of four 47, of
  //   two 49);
  //   18 warps per SM with teams of four: these (1000 rows of 128000 words: 58 us, blocks of 8 warps 97; 600 rows of 32000
  //   words: 19 us, blocks 17).
  // Blocks of 8 warps, four teams to a block: blocks of 4 or 2 warps take 72 and 61 us instead of 57 for 4096 rows of 32000.
  const auto fills = [&](int64_t warps, int64_t per_sm) { return (int64_t)a.T * warps >= per_sm * sms; };
  if (groups <= 16 && a.top <= 8 && fills(1, 16)) return launch<T, 8, 1, 1>(a, groups, st);
  if (groups <= 1536 && fills(2, 48)) return launch<T, 8, 2, 1>(a, groups, st);
  if (groups <= 2 * 1536 && fills(4, 18)) return launch<T, 8, 4, 1>(a, groups, st);
  // Fewer rows: a block of 8 warps each, or clusters of blocks of 16 while these find room and keep 16 groups each (a row of
  // 32000 words: 5.6 us, one block 6.7; of 128000: 6.2, one block 22; but 8000 words, 32 groups, 5.3 and one block 4.3).
  // Rows of 256 groups and more never go to one block (400 rows of 128000 words: 42 us, one block 57).
  int cl = 1;
  while (cl < 16 && (int64_t)a.T * 2 * cl <= 2 * sms && groups >= 64 && groups / (2 * cl) >= 16) cl *= 2;
  if (cl == 1 && groups >= 256) cl = 2;
  if (cl == 16 && !room_for_16<T>()) cl = 8;
  switch (cl) {
    case 1: return launch<T, 8, 8, 1>(a, groups, st);
    case 2: return launch<T, 16, 16, 2>(a, groups, st);
    case 4: return launch<T, 16, 16, 4>(a, groups, st);
    case 8: return launch<T, 16, 16, 8>(a, groups, st);
    default: return launch<T, 16, 16, 16>(a, groups, st);
  }
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
  if ((int64_t)T * 16 > INT32_MAX) return PCOMOE_ERR_SHAPE;
  int sms;
  pcomoe_status st = current_sms(&sms);
  if (st != PCOMOE_OK) return st;
  const Args a = {(const char *)d_logits, row_stride * e, T, V, top_n, 0, d_tokens, d_logprob, d_entropy, d_top_logprob, d_top_ids};
  return dtype == PCOMOE_BF16 ? run<__nv_bfloat16>(a, sms, (cudaStream_t)stream) : run<float>(a, sms, (cudaStream_t)stream);
}
