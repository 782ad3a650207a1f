// Verification of drafted tokens against the target's probabilities, from given random numbers, and the token that follows.
//
// Mathematics.  p = softmax(x / temperature) of a row's logits x, q the distribution that the drafts behind the row were drawn
// from (the drafter's row; all of it on the draft where none is given).  At a row whose drafts are c1, c2, ... with tokens t1,
// t2, ...: ci is taken iff u q(ti) R < r(ti), where r = p and R = 1 before the first, and a refusal leaves r <- max(r - R q, 0),
// R <- sum r.  With A the sum of the R so far that is r = max(p - A q, 0) at once, since q >= 0; where q is all on the draft it
// is p without the refused tokens.  The next token is the first one whose sum of r, in the order of ids, exceeds u_next times
// all of it.  Whatever decides an integer (exponentials, sums, products with random numbers) is formed in 64 bits: in 32 a
// sum over a vocabulary is off by 1e-7 of itself, and with 10^4 to 10^5 borders between words that changes a token in every few
// thousand.
//
// Two launches.  The first forms the largest logit, its lowest id and, in 32 bits, the sum of the exponentials of every row, rows
// side by side.  In the second a cluster of blocks per sequence has gathered meanwhile what each draft's test needs, walks over the
// drafts (they are numbered behind their parents, so one ascending pass meets every test in order) and reads the row that the walk
// ended at once more, for the sums of its groups of 512 bytes in 64 bits, from which the group of the next token and in it the token
// follow.  A test is made in 32 bits first, and in 64, with the row's sum formed again, where it lies within 2^-13 of its border.
// After a refusal of a drawn draft the row's sum is formed in 64 bits before the sums of max(p - A q, 0) are: where the drafter's probabilities are nearly
// the target's, the rest is made of words so near p = A q that the sum in 32 bits says nothing about them.
// What bounds them: the rows' one read (HBM) in the first; in the second a chain of dependent steps, since an operation in 64
// bits takes some 45 clocks until the next one can use it.  Measured, both together: 32 sequences of 9 rows of 32000 words in bf16 20.5 us (18
// MB; the first launch about 8), 8 trees of 17 to 48 rows 18.4, 5 sequences of 1 to 5 rows of 151936 words in fp32 20.5.
#include <algorithm>
#include <cfloat>

#include "words.cuh"

namespace pcomoe {
namespace {

struct VerifyHeader {
  int32_t reserved[8];
  int32_t status;                         // the place of the router's word
};
static_assert(offsetof(VerifyHeader, status) == offsetof(DevPlan, status_router), "status word");

struct RowSums {                          // of a row
  double s;                               // sum of 2^(c (x - m)), c = log2 e / temperature (not of greedy rows)
  float m;                                // largest logit; -inf: nothing eligible
  int32_t best;                           // its lowest id, -1
};

struct VerifyArgs {
  int32_t T, V, n;
  const int32_t *cu, *tokens, *parent;    // parent NULL: chains
  const char *x;
  int64_t row_bytes;
  const float *near;                      // the drafter's probabilities or NULL
  int64_t near_stride;
  const float *temperature, *u, *u_next;
  int32_t *keep, *n_keep, *next;
  int32_t keep_stride;
  int32_t most_rows;                      // of a sequence
  VerifyHeader *head;
  RowSums *sums;
};

constexpr int kTable = 16;
constexpr int kMaxGroups = 1040;          // of a block: 2^20 fp32 words over 8 blocks, and one

// 2^((x - m) c) in 64 bits for x <= m.  c16 = 16 c.  The nearest 16th apart, Taylor's series of the rest y / 16, |y| <= 1/2, up to the 5th
// power (the first term left out is below 2e-13 of the result) and a table of 2^(k/16): 16 entries of 8 bytes lie in as many pairs
// of banks, so that lanes that ask for different ones do not wait for one another.  0 below 2^-990 and where x is -inf.
__device__ __forceinline__ double pow2(float x, float m, double c16, float least, const double *table) {
  const double magic = 6755399441055744.0;                 // 1.5 * 2^52: its last place is 1
  const double d = (double)fmaxf(x, least) - (double)m, t = fma(d, c16, magic);
  const int k = __double2loint(t);
  const double y = fma(d, c16, magic - t);
  constexpr double u = 0.69314718055994530942 / 16;
  double p = fma(y, u * u * u * u * u / 120, u * u * u * u / 24);
  p = fma(p, y, u * u * u / 6);
  p = fma(p, y, u * u / 2);
  p = fma(p, y, u) * y;
  const double w = table[k & (kTable - 1)], r = fma(w, p, w);
  return x < least ? 0.0 : __hiloint2double(__double2hiint(r) + ((k >> 4) << 20), __double2loint(r));
}
// the smallest x that pow2 takes; span = 990 / c.  Rounded up: where the steps of fp32 at m are not small beside the span, a value below m - span
// may have a power that the exponent of 64 bits has no room for.
__device__ __forceinline__ float least_of(float m, double span) { return __double2float_ru(fmax((double)m - span, -(double)FLT_MAX)); }
__device__ __forceinline__ void fill_table(double *table) {
  for (int i = threadIdx.x; i < kTable; i += blockDim.x) table[i] = exp2(i * (1.0 / kTable));
}
__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
  uint64_t d;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(*(uint64_t *)&a), "l"(*(uint64_t *)&b));
  return *(float2 *)&d;
}
__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
  uint64_t d;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(*(uint64_t *)&a), "l"(*(uint64_t *)&b));
  return *(float2 *)&d;
}

// 2^((x - m) c) in 32 bits for x <= m, any of them finite (their difference need not be) or x = -inf
__device__ __forceinline__ float weight_of(float x, float m, float c) { return ex2(fmaxf((0.5f * x - 0.5f * m) * c * 2.f, -1000.f)); }

// max(e - cut q, 0), the same bits wherever it is formed (the compiler may not join the product with the difference): a sum of these is
// above 0 where one of them is
__device__ __forceinline__ double rest_of(double e, double cut, double q) { return fmax(__dsub_rn(e, __dmul_rn(cut, q)), 0.0); }

__device__ __forceinline__ float real(float q) { return q > 0.f && q < INFINITY ? q : 0.f; }      // what is no probability counts as 0

template <typename T> __device__ __forceinline__ const T *row_of(const VerifyArgs &a, int t) { return (const T *)(a.x + (int64_t)t * a.row_bytes); }
template <typename T> __device__ __forceinline__ int shift_of(const T *row) { return (int)(((uintptr_t)row & 15) / sizeof(T)); }

// log2 e / temperature, where the row is not greedy
__device__ __forceinline__ double rate_of(const VerifyArgs &a, int s) {
  const float t = a.temperature ? a.temperature[s] : 1.f;
  return 1.4426950408889634074 / (double)t;
}
__device__ __forceinline__ bool greedy_of(const VerifyArgs &a, int s) { return a.temperature && !(a.temperature[s] > 0.f && a.temperature[s] < INFINITY); }

// Rows of sequence s; empty and reported where the list is no list.
__device__ __forceinline__ int2 rows_of(const VerifyArgs &a, int s) {
  const int from = a.cu[s], to = a.cu[s + 1];
  if (from < 0 || to < from || to > a.T || to - from > a.most_rows) {
    atomicCAS(&a.head->status, 0, (int)PCOMOE_ERR_INDEX);
    return make_int2(0, 0);
  }
  return make_int2(from, to - from);
}

// A block's sum and largest place, joined over the cluster in the order of the blocks.  Places hold a key of a logit in the upper
// half.  `slot` alternates so that one barrier is enough.
struct Joined {
  double s;
  unsigned long long place;
};
template <int CL>
struct Cluster {
  Joined (*box)[2];                       // [CL] of this block
  int slot;
  __device__ int rank() const { return CL > 1 ? (int)(blockIdx.x % CL) : 0; }
  __device__ static void barrier() {
    if (CL > 1) asm volatile("barrier.cluster.arrive.aligned;\n\tbarrier.cluster.wait.aligned;" ::: "memory");
    else __syncthreads();
  }
  // every block's pair, in `all`; thread 0 gives this block's
  __device__ void gather(Joined mine, Joined (&all)[CL]) {
    slot ^= 1;
    if (threadIdx.x == 0) box[0][slot] = mine;
    barrier();
#pragma unroll
    for (int r = 0; r < CL; ++r) {
      if (CL == 1) {
        all[r] = box[0][slot];
      } else {
        const uint32_t at = (uint32_t)__cvta_generic_to_shared(&box[0][slot]);
        uint32_t q;
        asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(q) : "r"(at), "r"(r));
        asm volatile("ld.shared::cluster.f64 %0, [%1];" : "=d"(all[r].s) : "r"(q) : "memory");
        asm volatile("ld.shared::cluster.u64 %0, [%1];" : "=l"(all[r].place) : "r"(q + 8) : "memory");
      }
    }
    if (CL == 1) __syncthreads();         // the box may be written again
  }
};

__device__ __forceinline__ unsigned long long warp_max(unsigned long long x) {
#pragma unroll
  for (int o = 16; o; o >>= 1) x = max(x, __shfl_xor_sync(~0u, x, o));
  return x;
}

// The lowest id of a group whose word has the key; a warp.
template <typename T>
__device__ __forceinline__ int id_in_group(const T *row, int shift, int V, int g, int key) {
  constexpr int N = Vec<T>::N;
  const int lane = threadIdx.x & 31;
  float x[N];
  load_words<T>(row, shift, V, g, lane, x);
  unsigned id = INT_MAX;
#pragma unroll
  for (int k = N - 1; k >= 0; --k)
    if (key_of(eligible(x[k])) == key) id = (g * 32 + lane) * N - shift + k;
  return (int)__reduce_min_sync(~0u, id);
}

// Largest logit, its lowest id and sums of all rows, in 32 bits.  kSumWarps warps, CL blocks per row.
constexpr int kSumWarps = 16;
template <typename T, int CL>
__global__ void __launch_bounds__(32 * kSumWarps) row_sums_kernel(const __grid_constant__ VerifyArgs a) {
  pdl_grid_wait();
  constexpr int N = Vec<T>::N, kLoads = 4;
  __shared__ float s_sum[kSumWarps];
  __shared__ unsigned long long s_place[kSumWarps];
  __shared__ Joined s_box[2];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int t = blockIdx.x / CL;
  Cluster<CL> cl = {&s_box, 0};
  if (t >= a.T) return;                                    // (there is a block for no rows)
  const T *row = row_of<T>(a, t);
  const int shift = shift_of(row), groups = (a.V + shift + 32 * N - 1) / (32 * N), per = (groups + CL - 1) / CL;
  const int g0 = min(cl.rank() * per, groups), g1 = min(g0 + per, groups);
  // sums over the warp's largest logit so far
  float sum = 0.f;
  int key = kNoKey, best_g = 0;
  uint4 raw[kLoads];
  auto fetch = [&](int g) {
    if (g * 32 * N >= shift && (g + kLoads) * 32 * N - shift <= a.V && g + kLoads <= g1) {      // all inside the row
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
  if (g < g1) fetch(g);                                    // on its way while the sequence is looked up
  // the row's sequence
  int s = 0;
  {
    int hi = a.n;
    while (hi - s > 1) {
      const int step = (hi - s + 31) / 32, i = s + (lane + 1) * step;
      const int k = __popc(__ballot_sync(~0u, i < hi && a.cu[min(i, hi)] <= t));
      hi = min(s + (k + 1) * step, hi);
      s += k * step;
    }
  }
  if (t < a.cu[s] || t >= a.cu[s + 1]) {                   // (every block of the cluster)
    // nothing to draw from, should a list that does not ascend bring a walk here
    if (cl.rank() == 0 && threadIdx.x == 0) a.sums[t] = {0.0, -INFINITY, -1};
    return;
  }
  const bool greedy = greedy_of(a, s);
  const float c = (float)fmin(rate_of(a, s), 3e38);
  for (; g < g1; g += kSumWarps * kLoads) {
    uint4 v[kLoads];
#pragma unroll
    for (int u = 0; u < kLoads; ++u) v[u] = raw[u];
    if (g + kSumWarps * kLoads < g1) fetch(g + kSumWarps * kLoads);      // on its way while this one is summed
    int k4[kLoads];
#pragma unroll
    for (int u = 0; u < kLoads; ++u) k4[u] = __reduce_max_sync(~0u, key_of(Vec<T>::largest(v[u])));
    int most = max(max(k4[0], k4[1]), max(k4[2], k4[3]));
    if (most >= key_of(INFINITY)) {                        // infinite logits (or nothing but NaN in a lane): they do not count
#pragma unroll
      for (int u = 0; u < kLoads; ++u) {
        float x[N];
        Vec<T>::unpack(v[u], x);
#pragma unroll
        for (int k = 0; k < N; ++k) x[k] = eligible(x[k]);
        v[u] = Vec<T>::pack(x);
        k4[u] = __reduce_max_sync(~0u, key_of(Vec<T>::largest(v[u])));
      }
      most = max(max(k4[0], k4[1]), max(k4[2], k4[3]));
    }
    if (most > key) {
      if (sum > 0.f) sum *= weight_of(of_key(key), of_key(most), c);
#pragma unroll
      for (int u = kLoads - 1; u >= 0; --u)
        if (k4[u] == most) best_g = g + u;
      key = most;
    }
    if (greedy || key <= kNoKey) continue;
    const float m = of_key(key);
    if (fabsf(m) < 1e6f && c > 1e-20f) {                   // (words held above -1e30, NaN and -inf with them: their weight is 0)
      const float2 c2 = make_float2(c, c), minus = make_float2(-m, -m);
      float2 s2[4] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f), make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
#pragma unroll
      for (int u = 0; u < kLoads; ++u) {
        float2 x[N / 2];
        Vec<T>::pairs(v[u], x);
#pragma unroll
        for (int k = 0; k < N / 2; ++k) {
          const float2 d = mul2(add2(x[k], minus), c2);
          s2[u] = add2(s2[u], make_float2(ex2(d.x), ex2(d.y)));
        }
      }
      const float2 st = add2(add2(s2[0], s2[1]), add2(s2[2], s2[3]));
      sum += st.x + st.y;
    } else {
#pragma unroll
      for (int u = 0; u < kLoads; ++u) {
        float x[N];
        Vec<T>::unpack(v[u], x);
#pragma unroll
        for (int k = 0; k < N; ++k) sum += weight_of(eligible(x[k]), m, c);
      }
    }
  }
#pragma unroll
  for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(~0u, sum, o);
  if (lane == 0) { s_sum[warp] = sum; s_place[warp] = place_of(max(key, kNoKey), best_g); }
  __syncthreads();
  // the warps', then the blocks', over the largest of all; ties go to the lowest group
  const auto join = [&](float part, unsigned long long from, unsigned long long to) {
    return part > 0.f ? part * weight_of(of_key(place_key(from)), of_key(place_key(to)), c) : 0.f;
  };
  unsigned long long place = 0;
  float total = 0.f;
  if (warp == 0) {
    static_assert(kSumWarps == 16, "half a warp's lanes");
    const unsigned long long mine = s_place[lane & 15];
    place = warp_max(mine);
    total = join(s_sum[lane & 15], mine, place);
#pragma unroll
    for (int o = 8; o; o >>= 1) total += __shfl_xor_sync(~0u, total, o);
  }
  if (CL > 1) {
    Joined all[CL];
    cl.gather({(double)total, place}, all);
    if (cl.rank() == 0 && warp == 0) {
#pragma unroll
      for (int r = 0; r < CL; ++r) place = max(place, all[r].place);
      total = 0.f;
#pragma unroll
      for (int r = 0; r < CL; ++r) total += join((float)all[r].s, all[r].place, place);
    }
  }
  if (cl.rank() == 0 && warp == 0) {
    const int k = place_key(place), best = k == kNoKey ? -1 : id_in_group<T>(row, shift, a.V, place_id(place), k);
    if (lane == 0) a.sums[t] = {(double)total, of_key(k), best};
  }
  if (CL > 1) Cluster<CL>::barrier();                      // nobody leaves while others read its box
}

// The walk and the next token.  CL blocks per sequence.  kDrawn: there are probabilities that the drafts were drawn from.  (A kernel of its own without
// them: with the code for what refusals leave in it, walks that never run it took 0.8 us longer.)
constexpr int kWalkWarps = 16, kWalkThreads = 32 * kWalkWarps, kChunk = kWalkThreads;
// Whether 32 bits may not decide want < r.  A row's sum is off by at most 2^-14 of itself (20 times 2^-23 from the products' rounding
// where the words' own logarithms average 20 bits, and a step of 2^-24 for each addition of a lane); `size`: what want and r were formed from.
__device__ __forceinline__ bool near_border(float want, float r, float size) {
  return !(fabsf(want - r) > (1.f / 8192) * size) || fmaxf(want, r) < 1e-30f;
}
template <typename T, int CL, bool kDrawn>
__global__ void __launch_bounds__(kWalkThreads, 1) walk_kernel(const __grid_constant__ VerifyArgs a, int room) {
  // The launch before this one in the stream is row_sums_kernel's, which let this one begin only after all earlier work was
  // done: the arguments can be read before waiting for it, its sums and the caller's outputs not.
  constexpr int N = Vec<T>::N, kLoads = 16 / N;            // groups of a warp at a time: 16 words of a lane
  extern __shared__ __align__(16) uint8_t smem[];
  double *s_group = (double *)smem;                        // sums of this block's groups: of 2^(c (x - m)), or of what is left of it
  uint8_t *s_out = (uint8_t *)(s_group + room);            // refused words of given drafts, a bit each: a byte per lane and group
  __shared__ double s_table[kTable];
  __shared__ double s_warp[2][kWalkWarps];                 // what the warps hand to the cluster, in turn
  __shared__ float s_p[kChunk], s_q[kChunk], s_u[kChunk];
  __shared__ int s_parent[kChunk];
  __shared__ uint8_t s_first[kChunk];                      // the test where a draft is the first at its parent: 1 taken, 2 near its border
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int seq = blockIdx.x / CL, rank = CL > 1 ? (int)(blockIdx.x % CL) : 0;
  const bool first_block = rank == 0;
  const int2 rows = rows_of(a, seq);
  if (rows.y == 0) {
    pdl_grid_wait();
    if (first_block) {
      for (int i = tid; i < a.keep_stride; i += kWalkThreads) a.keep[(int64_t)seq * a.keep_stride + i] = -1;
      if (tid == 0) { a.n_keep[seq] = 0; a.next[seq] = -1; }
    }
    return;
  }
  fill_table(s_table);
  const bool greedy = greedy_of(a, seq);
  const double c = rate_of(a, seq), c16 = 16 * c, span = 990.0 / c;
  const float c32 = (float)fmin(c, 3e38);
  __syncthreads();
  auto parent_of = [&](int k) { return a.parent ? a.parent[rows.x + k] : k - 1; };

  int cur = 0, length = 1;
  int refused = 0;                                         // drafts refused at cur
  float gone = 0.f;                                        // p of the refused tokens, where drafts are given
  double A = 0.0, R = 1.0;                                 // where they were drawn: r = max(p - A q, 0), R = sum r (unless it is due)
  bool due = false, exact = false;                         // exact: sums.s is formed in 64 bits
  RowSums sums = {0.0, 0.f, -1};                           // of row cur, once asked for
  const T *row;
  int shift, groups, per, g0, g1, slot = 0;

  // Sums of row cur's groups, of this block in s_group, of every block in every thread: of e = 2^(c (x - m)), or (rest) of max(e - A s q, 0) with s
  // the sum of e over the row in 64 bits.
  double part[CL];
  // (always inlined: a call would put these arrays into local memory)
  using Words = uint4[kLoads];
  using Near = float[kLoads][N];
  using Weights = double[kLoads][N];
  auto look = [&]() __attribute__((always_inline)) {
    if (!exact) sums = a.sums[rows.x + cur];
    row = row_of<T>(a, rows.x + cur);
    shift = shift_of(row);
    groups = (a.V + shift + 32 * N - 1) / (32 * N);
    per = (groups + CL - 1) / CL;
    g0 = min(rank * per, groups);
    g1 = min(g0 + per, groups);
  };
  // the words of groups g, g + kWalkWarps, ..., and q there
  auto bring = [&](int g, bool rest, Words &raw, Near &y) __attribute__((always_inline)) {
    const float *near = rest ? a.near + (int64_t)(rows.x + cur) * a.near_stride : nullptr;
    if (g * 32 * N >= shift && (g + kWalkWarps * (kLoads - 1) + 1) * 32 * N - shift <= a.V && g + kWalkWarps * (kLoads - 1) < g1) {
      const uint4 *p = (const uint4 *)(row - shift) + g * 32 + lane;                    // all inside the row
#pragma unroll
      for (int i = 0; i < kLoads; ++i) raw[i] = p[32 * kWalkWarps * i];
      if (rest) {
        const float *q = near + (g * 32 + lane) * N - shift;
        if (((uintptr_t)q & 15) == 0) {
#pragma unroll
          for (int i = 0; i < kLoads; ++i)
#pragma unroll
            for (int k = 0; k < N; k += 4) *(float4 *)&y[i][k] = *(const float4 *)(q + 32 * kWalkWarps * N * i + k);
        } else {
#pragma unroll
          for (int i = 0; i < kLoads; ++i)
#pragma unroll
            for (int k = 0; k < N; ++k) y[i][k] = q[32 * kWalkWarps * N * i + k];
        }
      }
    } else {
      float none[N];
#pragma unroll
      for (int k = 0; k < N; ++k) none[k] = kNone;
#pragma unroll
      for (int i = 0; i < kLoads; ++i) {
        const bool there = g + kWalkWarps * i < g1;
        const int id = ((g + kWalkWarps * i) * 32 + lane) * N - shift;
        raw[i] = there ? load_raw<T>(row, shift, a.V, g + kWalkWarps * i, lane) : Vec<T>::pack(none);
        if (rest)
#pragma unroll
          for (int k = 0; k < N; ++k) y[i][k] = there && id + k >= 0 && id + k < a.V ? near[id + k] : 0.f;
      }
    }
  };
  auto form = [&](int g, bool marked, const Words &raw, Weights &e) __attribute__((always_inline)) {
    const float least = least_of(sums.m, span);
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      float x[N];
      Vec<T>::unpack(raw[i], x);
      const uint32_t out = marked && g + kWalkWarps * i < g1 ? s_out[(g + kWalkWarps * i - g0) * 32 + lane] : 0u;
#pragma unroll
      for (int k = 0; k < N; ++k) e[i][k] = pow2((out >> k) & 1 ? kNone : eligible(x[k]), sums.m, c16, least, s_table);
    }
  };
  auto leave = [&](const Near &y, Weights &e) __attribute__((always_inline)) {
    const double cut = A * sums.s;
#pragma unroll
    for (int i = 0; i < kLoads; ++i)
#pragma unroll
      for (int k = 0; k < N; ++k) e[i][k] = rest_of(e[i][k], cut, (double)real(y[i][k]));
  };
  // the groups' sums, to s_group and added to we
  auto add = [&](int g, const Weights &w, double &we) __attribute__((always_inline)) {
    Weights e;
#pragma unroll
    for (int i = 0; i < kLoads; ++i)
#pragma unroll
      for (int k = 0; k < N; ++k) e[i][k] = w[i][k];
#pragma unroll
    for (int i = 0; i < kLoads; ++i)
#pragma unroll
      for (int o = 1; o < N; o <<= 1)
#pragma unroll
        for (int k = 0; k < N; k += 2 * o) e[i][k] += e[i][k + o];
#pragma unroll
    for (int o = 16; o; o >>= 1)
#pragma unroll
      for (int i = 0; i < kLoads; ++i) e[i][0] += __shfl_xor_sync(~0u, e[i][0], o);
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      if (g + kWalkWarps * i >= g1) break;
      if (lane == 0) s_group[g + kWalkWarps * i - g0] = e[i][0];
      we += e[i][0];
    }
  };
  // the warps' sums to all of the cluster; returns the row's
  auto join = [&](double we) __attribute__((always_inline)) {
    slot ^= 1;
    if (lane == 0) s_warp[slot][warp] = we;
    Cluster<CL>::barrier();                                // (the next sums go to the other slot, the ones after that behind its barrier)
    constexpr int kRounds = (CL + 1) / 2;
    double v[kRounds];
#pragma unroll
    for (int i = 0; i < kRounds; ++i) {
      const double *from = &s_warp[slot][lane & 15];
      if (CL == 1) {
        v[i] = *from;
      } else {
        uint32_t q;
        asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(q) : "r"((uint32_t)__cvta_generic_to_shared(from)), "r"(2 * i + (lane >> 4)));
        asm volatile("ld.shared::cluster.f64 %0, [%1];" : "=d"(v[i]) : "r"(q) : "memory");
      }
    }
#pragma unroll
    for (int o = 8; o; o >>= 1)
#pragma unroll
      for (int i = 0; i < kRounds; ++i) v[i] += __shfl_xor_sync(~0u, v[i], o);
    double s = 0.0;
#pragma unroll
    for (int r = 0; r < CL; ++r) {
      part[r] = __shfl_sync(~0u, v[r / 2], (r & 1) * 16);
      s += part[r];
    }
    return s;
  };
  // the sums of e; marked: without the words that s_out marks
  auto pass = [&](bool marked) __attribute__((always_inline)) {
    look();
    double we = 0.0;
    for (int g = g0 + warp; g < g1; g += kWalkWarps * kLoads) {
      Words raw;
      Near y;
      Weights e;
      bring(g, false, raw, y);
      form(g, marked, raw, e);
      add(g, e, we);
    }
    return join(we);
  };
  // sums.s of row cur in 64 bits
  auto refine = [&]() __attribute__((always_inline)) {
    if (exact) return;
    sums.s = pass(false);
    exact = true;
  };
  // What is left of row cur after its refusals, in units of 2^(c m), and with it the row's sum in 64 bits.
  auto left_over = [&]() __attribute__((always_inline)) {
    look();
    Words raw;
    Near y;
    Weights e;
    double we = 0.0;
    if (per <= kWalkWarps * kLoads) {                      // a warp's words stay in registers between the two sums
      const int g = g0 + warp;
      if (g < g1) {
        bring(g, true, raw, y);
        form(g, false, raw, e);
      }
      if (!exact) {
        if (g < g1) add(g, e, we);
        sums.s = join(we);
        exact = true;
        we = 0.0;
      }
      if (g < g1) {
        leave(y, e);
        add(g, e, we);
      }
      return join(we);
    }
    for (;;) {
      const bool of_rest = exact;
      we = 0.0;
      for (int g = g0 + warp; g < g1; g += kWalkWarps * kLoads) {
        bring(g, true, raw, y);
        form(g, false, raw, e);
        if (of_rest) leave(y, e);
        add(g, e, we);
      }
      const double s = join(we);
      if (of_rest) return s;
      sums.s = s;
      exact = true;
    }
  };
  // p of a token at row cur, in 64 bits
  auto p_of = [&](int token) {
    if (greedy) return token == sums.best ? 1.0 : 0.0;
    const float x = eligible(Vec<T>::one(row_of<T>(a, rows.x + cur) + token));
    return x != kNone && sums.s > 0.0 ? pow2(x, sums.m, c16, least_of(sums.m, span), s_table) / sums.s : 0.0;
  };
  // whether one of the drafts [from, to) hangs on cur and has this token
  auto named = [&](int from, int to, int token) {
    bool yes = false;
    for (int b = from; b < to && !yes; b += 32) yes = __any_sync(~0u, b + lane < to && parent_of(b + lane) == cur && a.tokens[rows.x + b + lane] == token);
    return yes;
  };

  if (rows.y == 1 || a.keep_stride == 1) pdl_grid_wait();
  // what the tests of the drafts from `from` on need: p and q of each one's token at its parent's row, in 32 bits
  auto gather = [&](int from) {
    __syncthreads();
    const int j = from + tid, t = rows.x + j;
    int up = -1, token = -1;
    float x = kNone, q = 1.f, p = 0.f;
    if (j < rows.y && j > 0) {
      up = a.parent ? a.parent[t] : j - 1;
      token = a.tokens[t];
      s_u[tid] = a.u[t];
      if (up < 0 || up >= j || token < 0 || token >= a.V) {
        atomicCAS(&a.head->status, 0, (int)PCOMOE_ERR_INDEX);
        up = -1;
      } else {
        x = eligible(Vec<T>::one(row_of<T>(a, rows.x + up) + token));
        if (kDrawn) q = real(a.near[(int64_t)(rows.x + up) * a.near_stride + token]);
      }
    }
    s_parent[tid] = up;
    s_q[tid] = q;
    if (from == 0) pdl_grid_wait();
    if (up >= 0) {
      const RowSums at = a.sums[rows.x + up];
      if (greedy) p = token == at.best ? 1.f : 0.f;
      else if (x != kNone && at.s > 0.0) p = weight_of(x, at.m, c32) / (float)at.s;
    }
    s_p[tid] = p;
    {
      const float want = (j < rows.y && j > 0 ? s_u[tid] : 0.f) * q;
      s_first[tid] = near_border(want, p, want + p) ? 2 : want < p;
    }
    __syncthreads();
  };
  // Every warp of every block takes the same way.
  int c0 = -kChunk, next = 0;                              // drafts c0 .. c0 + kChunk are at hand, those from c0 + next on still to be tested
  double left = 0.0;                                       // of the row after the refusals so far, once asked for
  for (;;) {
    int hit = kChunk;                                      // the next draft on row cur; kChunk: there is none
    while (rows.y > 1 && length < a.keep_stride) {
      for (int b = next & ~31; c0 >= 0 && b < min(kChunk, rows.y - c0); b += 32) {
        const uint32_t m = __ballot_sync(~0u, b + lane >= next && s_parent[b + lane] == cur);
        if (m) {
          hit = b + __ffs(m) - 1;
          break;
        }
      }
      if (hit < kChunk || c0 + kChunk >= rows.y) break;
      c0 += kChunk;
      next = 0;
      gather(c0);
    }
    // what is left of the row is asked for by the next test, or by the next token
    if (due) {
      if (greedy) {
        // all of p lies on one word
        sums = a.sums[rows.x + cur];
        exact = true;
        left = R = sums.best >= 0 ? fmax(1.0 - A * (double)real(a.near[(int64_t)(rows.x + cur) * a.near_stride + sums.best]), 0.0) : 0.0;
      } else {
        left = left_over();
        R = sums.s > 0.0 ? left / sums.s : 0.0;
      }
      due = false;
      if (!(R > 0.0)) { A = 0.0; R = 1.0; }                // nothing is left: the target's own distribution again
    }
    if (hit == kChunk) break;
    const bool again = !kDrawn && refused && named(cur + 1, c0 + hit, a.tokens[rows.x + c0 + hit]);      // a given token that is gone
    bool taken, close;
    const float q = s_q[hit], u = s_u[hit];
    if (!refused) {
      taken = s_first[hit] & 1;
      close = s_first[hit] & 2;
    } else {
      const float p = s_p[hit], aq = (float)A * q, rr = kDrawn ? (float)R : 1.f - gone;
      const float r = again ? 0.f : p - aq, want = u * q * rr;
      taken = want < r;
      close = near_border(want, r, u * q * (kDrawn ? rr : 1.f) + p + aq);
    }
    if (close) {                                         // 64 bits give the answer
      const int token = a.tokens[rows.x + c0 + hit];
      if (greedy) {
        sums = a.sums[rows.x + cur];
        exact = true;
      }
      refine();
      const double p64 = p_of(token), r64 = again ? 0.0 : fmax(p64 - A * (double)q, 0.0);
      double R64 = R;
      if (!kDrawn) {
        for (int k = cur + 1; k < c0 + hit; ++k) {       // without the refused tokens, each once
          const int other = a.tokens[rows.x + k];
          if (parent_of(k) == cur && other >= 0 && other < a.V && !named(cur + 1, k, other)) R64 -= p_of(other);
        }
        if (!(R64 > 0.0)) R64 = 1.0;
      }
      taken = (double)u * R64 * (double)q < r64;
    }
    if (taken) {
      cur = c0 + hit;
      if (first_block && tid == 0) a.keep[(int64_t)seq * a.keep_stride + length] = cur;
      ++length;
      A = 0.0;
      R = 1.0;
      gone = 0.f;
      refused = 0;
      due = exact = false;
    } else {
      ++refused;
      if (kDrawn) {
        A += R;
        due = true;
      } else if (!again) {
        gone += s_p[hit];
      }
    }
    next = hit + 1;
  }
  if (first_block) {
    if (tid == 0) { a.keep[(int64_t)seq * a.keep_stride] = 0; a.n_keep[seq] = length; }
    for (int i = length + tid; i < a.keep_stride; i += kWalkThreads) a.keep[(int64_t)seq * a.keep_stride + i] = -1;
  }

  // the next token from row cur
  if (greedy) {
    if (first_block && tid == 0) a.next[seq] = a.sums[rows.x + cur].best;
  } else {
    const bool rest = A > 0.0;                             // of drawn drafts; what is left is formed already
    bool marked = !kDrawn && refused > 0;
    if (marked) {
      row = row_of<T>(a, rows.x + cur);
      shift = shift_of(row);
      per = ((a.V + shift + 32 * N - 1) / (32 * N) + CL - 1) / CL;
      for (int i = tid; i < per * 8; i += kWalkThreads) ((uint32_t *)s_out)[i] = 0u;
      __syncthreads();
      for (int k = cur + 1 + tid; k < rows.y; k += kWalkThreads) {
        const int token = a.tokens[rows.x + k];
        if (parent_of(k) == cur && token >= 0 && token < a.V) {
          const int w = token + shift - rank * per * 32 * N;         // place in this block's words
          if (w >= 0 && w < per * 32 * N) atomicOr((uint32_t *)s_out + (w / N) / 4, 1u << (((w / N) & 3) * 8 + w % N));
        }
      }
      __syncthreads();
    }
    double total = left;                                   // what the token is drawn from, block by block in `part`
    while (!rest) {
      total = pass(marked);
      if (total > 0.0 || !marked) break;
      marked = false;                                      // nothing is left: the target's own distribution
      __syncthreads();                                     // the sums are read before they are formed again
    }
    if (!(total > 0.0)) {
      if (first_block && tid == 0) a.next[seq] = -1;
    } else {
      // the block, the group and the word in which the sum passes the target
      const double target = (double)a.u_next[seq] * total;
      double before = 0.0;
      int owner = -1;
#pragma unroll
      for (int r = 0; r < CL; ++r) {
        if (owner < 0 && part[r] > 0.0 && before + part[r] > target) owner = r;
        if (owner < 0) before += part[r];
      }
      if (owner < 0) {                                     // rounding, or u_next at 1: the last word with any weight
        before = -INFINITY;
#pragma unroll
        for (int r = 0; r < CL; ++r)
          if (part[r] > 0.0) owner = r;
      }
      if (owner == rank && warp == 0) {
        const double goal = target - before, cut = A * sums.s;      // +inf: all of it
        const int mine = g1 - g0, each = (mine + 31) / 32;
        double sum = 0.0;
        int last = -1;                                     // the last group with any weight
        for (int i = lane * each; i < min((lane + 1) * each, mine); ++i) {
          const double x = s_group[i];
          sum += x;
          if (x > 0.0) last = i;
        }
        double upto = sum;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
          const double y = __shfl_up_sync(~0u, upto, o);
          if (lane >= o) upto += y;
        }
        const uint32_t past = __ballot_sync(~0u, last >= 0 && upto > goal);
        int g = __reduce_max_sync(~0u, last);
        double left = INFINITY;                            // what is to be passed inside of the group
        if (past) {
          // the first lane whose sum passes the goal.  Added one by one its groups may just not pass it, since the scan adds in another order: the
          // last word of the lane then.
          const int l = __ffs(past) - 1;
          double base = __shfl_sync(~0u, upto - sum, l);
          g = __shfl_sync(~0u, last, l);
          for (int i = l * each; i < min((l + 1) * each, mine); ++i) {
            const double x = s_group[i];
            if (x > 0.0 && base + x > goal) {
              g = i;
              left = goal - base;
              break;
            }
            base += x;
          }
        }
        float x[N];
        load_words<T>(row, shift, a.V, g0 + g, lane, x);
        const uint32_t out = marked ? s_out[g * 32 + lane] : 0u;
        const float *near = rest ? a.near + (int64_t)(rows.x + cur) * a.near_stride : nullptr;
        const int id = ((g0 + g) * 32 + lane) * N - shift;
        const float least = least_of(sums.m, span);
        double e[N], lane_sum = 0.0;
        int last_word = -1;
#pragma unroll
        for (int k = 0; k < N; ++k) {
          e[k] = pow2((out >> k) & 1 ? kNone : eligible(x[k]), sums.m, c16, least, s_table);
          if (rest) e[k] = rest_of(e[k], cut, id + k >= 0 && id + k < a.V ? (double)real(near[id + k]) : 0.0);
          lane_sum += e[k];
          if (e[k] > 0.0) last_word = id + k;
        }
        double incl = lane_sum;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
          const double y = __shfl_up_sync(~0u, incl, o);
          if (lane >= o) incl += y;
        }
        int pick = INT_MAX;
        double run = incl - lane_sum;
#pragma unroll
        for (int k = 0; k < N; ++k) {
          run += e[k];
          if (e[k] > 0.0 && run > left && pick == INT_MAX) pick = id + k;
        }
        const int lowest = (int)__reduce_min_sync(~0u, (unsigned)pick);
        const int highest = __reduce_max_sync(~0u, last_word);
        if (lane == 0) a.next[seq] = lowest == INT_MAX ? highest : lowest;
      }
    }
  }
  Cluster<CL>::barrier();                                  // nobody leaves while others read its sums
}

constexpr int kGroupBytes = 8 + 32;       // of shared memory for each group of a block: a sum, a byte per lane

template <typename... K, typename... A>
cudaError_t launch_clusters(void (*kernel)(K...), int items, int cl, int threads, size_t smem, cudaStream_t st, A... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(items * cl));
  cfg.blockDim = dim3((unsigned)threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = (unsigned)cl;
  attr[1].val.clusterDim.y = 1;
  attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = cl > 1 ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, kernel, K(args)...);
}

template <typename T, int CL>
pcomoe_status launch_sums(const VerifyArgs &a, cudaStream_t st) {
  PCOMOE_CUDA_TRY(launch_clusters(row_sums_kernel<T, CL>, std::max(a.T, 1), CL, 32 * kSumWarps, 0, st, a));
  count_launch();
  return PCOMOE_OK;
}
// Whether clusters of 16 blocks find room on the current device, which 8 always do: asked once for each device.
template <typename T, bool kDrawn>
bool room_for_16() {
  static std::atomic<uint64_t> asked{0}, there{0};
  int dev = -1;
  if (cudaGetDevice(&dev) != cudaSuccess) return false;
  const uint64_t bit = dev >= 0 && dev < 64 ? uint64_t(1) << dev : 0;
  if (asked.load(std::memory_order_acquire) & bit) return (there.load(std::memory_order_relaxed) & bit) != 0;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(16);
  cfg.blockDim = dim3(kWalkThreads);
  cfg.dynamicSmemBytes = kMaxGroups * kGroupBytes;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = 16;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  int clusters = 0;
  const bool ok = cudaFuncSetAttribute(walk_kernel<T, 16, kDrawn>, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) == cudaSuccess &&
                  cudaFuncSetAttribute(walk_kernel<T, 16, kDrawn>, cudaFuncAttributeMaxDynamicSharedMemorySize, kMaxGroups * kGroupBytes) == cudaSuccess &&
                  cudaOccupancyMaxActiveClusters(&clusters, walk_kernel<T, 16, kDrawn>, &cfg) == cudaSuccess && clusters > 0;
  if (!ok) cudaGetLastError();                             // the answer is no, not an error of a later call
  if (ok) there.fetch_or(bit, std::memory_order_relaxed);
  asked.fetch_or(bit, std::memory_order_release);
  return ok;
}

template <typename T, int CL, bool kDrawn>
pcomoe_status launch_walk(const VerifyArgs &a, int groups, cudaStream_t st) {
  const int room = ((groups + CL - 1) / CL + 1) & ~1;
  static PerDeviceOnce once;
  int dev = -1;
  PCOMOE_CUDA_TRY(cudaGetDevice(&dev));
  if (once.first_use(dev)) {
    PCOMOE_CUDA_TRY(cudaFuncSetAttribute(walk_kernel<T, CL, kDrawn>, cudaFuncAttributeMaxDynamicSharedMemorySize, kMaxGroups * kGroupBytes));
    once.done(dev);
  }
  PCOMOE_CUDA_TRY(launch_clusters(walk_kernel<T, CL, kDrawn>, a.n, CL, kWalkThreads, (size_t)room * kGroupBytes, st, a, room));
  count_launch();
  return PCOMOE_OK;
}

template <typename T, bool kDrawn>
pcomoe_status launch_walk(const VerifyArgs &a, int groups, int cl, cudaStream_t st) {
  if (cl == 16 && !room_for_16<T, kDrawn>()) cl = 8;
  switch (cl) {
    case 16: return launch_walk<T, 16, kDrawn>(a, groups, st);
    case 1: return launch_walk<T, 1, kDrawn>(a, groups, st);
    case 2: return launch_walk<T, 2, kDrawn>(a, groups, st);
    case 4: return launch_walk<T, 4, kDrawn>(a, groups, st);
    default: return launch_walk<T, 8, kDrawn>(a, groups, st);
  }
}

template <typename T>
pcomoe_status run(const VerifyArgs &a, int sms, cudaStream_t st) {
  const int groups = (a.V + 15) / (32 * Vec<T>::N) + 1;    // at any alignment
  // blocks per row and per sequence: while there is an SM for each and enough groups for its warps
  const auto blocks = [&](int items, int warps, int most) {
    int cl = 1;
    while (cl < most && ((int64_t)items * 2 * cl <= sms || groups > cl * (kMaxGroups - 2)) && groups >= 2 * cl * warps) cl *= 2;
    return cl;
  };
  pcomoe_status s = PCOMOE_OK;
  switch (blocks(std::max(a.T, 1), kSumWarps, 8)) {           // (launched for no rows too: the second launch leans on the first)
    case 1: s = launch_sums<T, 1>(a, st); break;
    case 2: s = launch_sums<T, 2>(a, st); break;
    case 4: s = launch_sums<T, 4>(a, st); break;
    default: s = launch_sums<T, 8>(a, st); break;
  }
  if (s != PCOMOE_OK) return s;
  const int cl = blocks(a.n, kWalkWarps, 16);
  return a.near ? launch_walk<T, true>(a, groups, cl, st) : launch_walk<T, false>(a, groups, cl, st);
}

struct Range {                            // of memory; NULL: none
  const void *at;
  int64_t bytes;
  bool meets(const Range &o) const {
    const uintptr_t a = (uintptr_t)at, b = (uintptr_t)o.at;
    return at && o.at && bytes > 0 && o.bytes > 0 && a < b + (uintptr_t)o.bytes && b < a + (uintptr_t)bytes;
  }
};

}  // namespace
}  // namespace pcomoe

using namespace pcomoe;

extern "C" {

pcomoe_status pcomoe_verify_workspace_bytes(int32_t max_tokens, size_t *bytes) {
  if (!bytes) return PCOMOE_ERR_INVALID_ARG;
  if (max_tokens < 0) return PCOMOE_ERR_SHAPE;
  *bytes = 256 + sizeof(RowSums) * (size_t)max_tokens;
  return PCOMOE_OK;
}

pcomoe_status pcomoe_verify_drafts(int32_t dtype, int32_t T, int32_t V, int32_t n, const int32_t *d_cu_len, const int32_t *d_tokens, const int32_t *d_parent,
                                   const void *d_logits, int64_t row_stride, const float *d_draft_probs, int64_t draft_stride, const float *d_temperature,
                                   const float *d_u, const float *d_u_next, int32_t *d_keep, int32_t keep_stride, int32_t *d_n_keep, int32_t *d_next,
                                   void *d_workspace, size_t ws_bytes, void *stream) {
  if (dtype != PCOMOE_BF16 && dtype != PCOMOE_FP32) return PCOMOE_ERR_INVALID_ARG;
  if (T < 0 || V <= 0 || n < 0 || n > 65535 || keep_stride < 0) return PCOMOE_ERR_SHAPE;
  if (V > kMaxVocab) return PCOMOE_ERR_UNSUPPORTED;
  if (n == 0) return PCOMOE_OK;
  const int64_t e = (int64_t)dtype_size(dtype);
  if (!d_cu_len || !d_keep || keep_stride == 0 || !d_n_keep || !d_next || !d_u_next || (T > 0 && (!d_tokens || !d_u || !d_logits))) return PCOMOE_ERR_INVALID_ARG;
  if (T > 0 && (row_stride < V || (uintptr_t)d_logits % e || (d_draft_probs && (draft_stride < V || (uintptr_t)d_draft_probs % 4)))) return PCOMOE_ERR_INVALID_ARG;
  if ((int64_t)T * 8 > INT32_MAX) return PCOMOE_ERR_SHAPE;
  if (!d_workspace || ((uintptr_t)d_workspace & 255) || ws_bytes < 256 + sizeof(RowSums) * (size_t)T) return PCOMOE_ERR_WORKSPACE;
  // An output among the inputs: the blocks of a cluster would read different things.  What only drafts need (tokens, parents, u) may be
  // an output's where there are none.
  const Range out[3] = {{d_keep, 4 * (int64_t)n * keep_stride}, {d_n_keep, 4 * (int64_t)n}, {d_next, 4 * (int64_t)n}};
  const Range in[5] = {{d_cu_len, 4 * ((int64_t)n + 1)}, {d_temperature, 4 * (int64_t)n}, {d_u_next, 4 * (int64_t)n},
                       {d_logits, T ? (((int64_t)T - 1) * row_stride + V) * e : 0}, {d_draft_probs, T ? (((int64_t)T - 1) * draft_stride + V) * 4 : 0}};
  const Range of_drafts[3] = {{d_tokens, 4 * (int64_t)T}, {d_parent, 4 * (int64_t)T}, {d_u, 4 * (int64_t)T}};
  bool shared = false;
  for (const Range &o : out) {
    for (const Range &i : in)
      if (o.meets(i)) return PCOMOE_ERR_INVALID_ARG;
    for (const Range &i : of_drafts) shared |= o.meets(i);
  }
  int sms;
  const pcomoe_status st = current_sms(&sms);
  if (st != PCOMOE_OK) return st;
  VerifyArgs a = {};
  a.most_rows = shared ? 1 : INT_MAX;
  a.T = T; a.V = V; a.n = n;
  a.cu = d_cu_len; a.tokens = d_tokens; a.parent = d_parent;
  a.x = (const char *)d_logits; a.row_bytes = row_stride * e;
  a.near = d_draft_probs; a.near_stride = draft_stride;
  a.temperature = d_temperature; a.u = d_u; a.u_next = d_u_next;
  a.keep = d_keep; a.n_keep = d_n_keep; a.next = d_next; a.keep_stride = keep_stride;
  a.head = (VerifyHeader *)d_workspace;
  a.sums = (RowSums *)((char *)d_workspace + 256);
  return dtype == PCOMOE_BF16 ? run<__nv_bfloat16>(a, sms, (cudaStream_t)stream) : run<float>(a, sms, (cudaStream_t)stream);
}

}  // extern "C"
