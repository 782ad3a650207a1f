// Accumulated attention weight of cached positions: host side, and the kernel of few counted rows.
//
// Mathematics.  w_p += sum over counted rows and heads of 2^(c q.k_p - c' lse), c = scale log2 e, c' = log2 e: the products of
// attention's first matrix product again, with the log sums that attention has left instead of a running maximum, so one
// pass over the keys and no pass over the values.  A position is a row of the product here and the counted rows are its
// columns, so that a position's sum stays inside a few lanes.
//
// What bounds it with few rows: one read of the keys (HBM).  A warp takes 16 keys of one head at a time (no piece crosses a
// page) through a ring of its own, filled with 16-byte asynchronous copies.  Its lanes read 16 bytes at a time as the fragments of the
// warp MMAs (m16n8k16): the order of the inner dimension is free as long as both operands have the same one, and the queries
// are laid out once per sequence in that order.  All heads of a block of keys are taken by one block of
// threads and added in order, so nothing is added across blocks and no atomics are needed.  Measured, 32 heads on 8 of 128, bf16: one
// row of each of 32 sequences of 1 to 4095 tokens (121 MB of keys) 30.8 us, 3.9 TB/s; 4 and 1 rows of two of 131 k and 100 k tokens
// (473 MB) 86 us, 5.5 TB/s, 0.85 of a plain copy's rate.
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "weigh.cuh"

namespace pcomoe {
namespace {

constexpr int kWarps = 12, kThreads = 32 * kWarps, kKeys = 16;
constexpr int kItems = 48;              // pieces of 16 keys of a head in a block of keys, about
constexpr int kMaxSubs = 16;            // pieces of 16 keys of one head in it
// From this many columns (counted rows x heads of a group) of a sequence on, on average, the tensor-core kernel is taken.  Of a list the
// host knows only how many rows it has room for: those are its counted rows here, or all packed rows if they are fewer.  Both, us, with 32
// heads on 8 of 128 and so many counted rows a sequence (4 columns each), this one and the other:
//   rows                       1          8           16          24          32          128
//   64 sequences of 512    21.0, 56.7  30.1, 57.0  51.0, 57.6  74.2, 60.5  96.3, 58.1  392, 103
//   32 sequences of 4096   53.3, 177   70.6, 178    128, 179    186, 179    242, 163   954, 274
//   4 sequences of 16384   32.9, 99.1  42.9, 100   73.6, 101    104, 101    133, 93.4  511, 148
//   8 sequences of 300     10.5, 17.8  13.3, 18.0  18.8, 18.7  24.9, 17.4  31.0, 17.0  105, 22.8
constexpr int kManyColumns = 96;
// And in fp32 from this many on:
//   rows                                         1            4            8            16          32          128
//   16 sequences of 512                    19.6, 47.3  41.1, 47.3  73.8, 47.6  140, 49.4   272, 78.8  1193, 298
//   8 sequences of 4096                    41.0, 148   90.4, 148    170, 149   328, 149    643, 255   2534, 935
//   8 sequences of 300, 8 heads on 2 of 64  8.5, 14.6  10.5, 14.5  12.5, 14.6  18.0, 14.6  28.8, 15.3  92.9, 27.2
constexpr int kManyColumnsF32 = 32;
constexpr int kStart = 8;               // cost of a sequence's beginning, in pieces of 16 keys
constexpr int kExtra = 6;               // cost of a piece of 16 keys besides its columns, in tiles of 8 columns

__device__ __forceinline__ void mma(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
               : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// 16 keys of a head in registers, and their weights over the columns [0, cols) at q, lse, lim (laid out in tiles of 8; lim: the last
// position that a column sees).  key0: position of the first.  Lane 0..15 of the result: key0 + lane.
template <typename T, int D> struct Piece;

template <int D> struct Piece<__nv_bfloat16, D> {
  // Keys come through a ring of the warp's own in shared memory, two pieces under way while one is worked on.  Odd rows have the two
  // halves of their 128 bytes exchanged, so that lanes of two rows read from different banks.
  static constexpr int kStages = 3, kBytes = kKeys * D * 2, kQBytes = 64 * 1024;      // stages, bytes of one; queries held at a time
  uint4 x[2][D / 32];
  static __device__ __forceinline__ void fetch(const __nv_bfloat16 *k, uint32_t to) {
    constexpr int C = D / 8;
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int j = 0; j < kKeys * C / 32; ++j) {
      const int u = j * 32 + lane, r = u / C, c = u % C;
      asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to + r * (D * 2) + ((c ^ ((r & 1) << 2)) << 4)), "l"((const char *)k + u * 16) : "memory");
    }
  }
  __device__ __forceinline__ void load(const char *from) {
    const int lane = threadIdx.x & 31, r = lane >> 2;
#pragma unroll
    for (int i = 0; i < D / 32; ++i) {
      const int at = r * (D * 2) + (((4 * i + (lane & 3)) ^ ((r & 1) << 2)) << 4);
      x[0][i] = *(const uint4 *)(from + at);
      x[1][i] = *(const uint4 *)(from + at + 8 * D * 2);
    }
  }
  // place of the 16 bytes c of column col in the layout that sums() reads: a tile of 8 columns, step by step, lane by lane
  static __device__ __forceinline__ int place(int col, int c) { return (((col >> 3) * (D / 32) + (c >> 2)) * 32 + (col & 7) * 4 + (c & 3)) * 16; }
  __device__ __forceinline__ float sums(const char *q, const float *lse, const int *lim, int cols, int key0, float scale) const {
    const int lane = threadIdx.x & 31;
    const int p0 = key0 + (lane >> 2), p1 = p0 + 8;
    float w0 = 0.f, w1 = 0.f;
    const auto form = [&](int t, auto many) {              // that many tiles of columns from t on, whose chains of products run side by side
      constexpr int M = many.value;
      float c[M][4];
#pragma unroll
      for (int k = 0; k < M; ++k) c[k][0] = c[k][1] = c[k][2] = c[k][3] = 0.f;
      const uint4 *b = (const uint4 *)q + t * (D / 32) * 32 + lane;
#pragma unroll
      for (int i = 0; i < D / 32; ++i) {
        uint4 y[M];
#pragma unroll
        for (int k = 0; k < M; ++k) y[k] = b[(k * (D / 32) + i) * 32];
#pragma unroll
        for (int k = 0; k < M; ++k) mma(c[k], x[0][i].x, x[1][i].x, x[0][i].y, x[1][i].y, y[k].x, y[k].y);
#pragma unroll
        for (int k = 0; k < M; ++k) mma(c[k], x[0][i].z, x[1][i].z, x[0][i].w, x[1][i].w, y[k].z, y[k].w);
      }
#pragma unroll
      for (int k = 0; k < M; ++k) {
        const float2 l = *(const float2 *)(lse + (t + k) * 8 + (lane & 3) * 2);
        const int2 m = *(const int2 *)(lim + (t + k) * 8 + (lane & 3) * 2);
        // chosen, not multiplied: what is not seen adds nothing whatever it is
        w0 += (p0 <= m.x ? exp2_fast(fmaf(c[k][0], scale, -l.x)) : 0.f) + (p0 <= m.y ? exp2_fast(fmaf(c[k][1], scale, -l.y)) : 0.f);
        w1 += (p1 <= m.x ? exp2_fast(fmaf(c[k][2], scale, -l.x)) : 0.f) + (p1 <= m.y ? exp2_fast(fmaf(c[k][3], scale, -l.y)) : 0.f);
      }
    };
    const int tiles = (cols + 7) / 8;
    int t = 0;
    for (; t + 4 <= tiles; t += 4) form(t, std::integral_constant<int, 4>());
    for (; t < tiles; ++t) form(t, std::integral_constant<int, 1>());
    w0 += __shfl_xor_sync(~0u, w0, 1);
    w1 += __shfl_xor_sync(~0u, w1, 1);
    w0 += __shfl_xor_sync(~0u, w0, 2);
    w1 += __shfl_xor_sync(~0u, w1, 2);
    // lane r holds key r
    const float lo = __shfl_sync(~0u, w0, (lane & 7) * 4), hi = __shfl_sync(~0u, w1, (lane & 7) * 4);
    return lane & 8 ? hi : lo;
  }
};

// fp32: a lane holds half of a key's row; rows are copied with 16 bytes between them
template <int D> struct Piece<float, D> {
  static constexpr int kStages = 2, kBytes = kKeys * (D * 4 + 16), kQBytes = 16 * 1024;
  float4 x[D / 8];
  static __device__ __forceinline__ void fetch(const float *k, uint32_t to) {
    constexpr int C = D / 4;
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int j = 0; j < kKeys * C / 32; ++j) {
      const int u = j * 32 + lane, r = u / C, c = u % C;
      asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to + r * (D * 4 + 16) + c * 16), "l"((const char *)k + u * 16) : "memory");
    }
  }
  __device__ __forceinline__ void load(const char *from) {
    const int lane = threadIdx.x & 31;
    const float4 *p = (const float4 *)(from + (lane & 15) * (D * 4 + 16)) + (lane >> 4) * (D / 8);
#pragma unroll
    for (int i = 0; i < D / 8; ++i) x[i] = p[i];
  }
  static __device__ __forceinline__ int place(int col, int c) { return (col * (D / 4) + c) * 16; }
  __device__ __forceinline__ float sums(const char *q, const float *lse, const int *lim, int cols, int key0, float scale) const {
    const int lane = threadIdx.x & 31, p = key0 + (lane & 15);
    const float4 *b = (const float4 *)q + (lane >> 4) * (D / 8);
    float w = 0.f;
    for (int c = 0; c < cols; ++c) {
      float s[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int i = 0; i < D / 8; ++i) {
        const float4 y = b[c * (D / 4) + i];
        s[0] = fmaf(x[i].x, y.x, s[0]);
        s[1] = fmaf(x[i].y, y.y, s[1]);
        s[2] = fmaf(x[i].z, y.z, s[2]);
        s[3] = fmaf(x[i].w, y.w, s[3]);
      }
      float t = (s[0] + s[1]) + (s[2] + s[3]);
      t += __shfl_xor_sync(~0u, t, 16);
      w += p <= lim[c] ? exp2_fast(fmaf(t, scale, -lse[c])) : 0.f;
    }
    return w;
  }
};

// Heads and columns of a head that are held at a time, and pieces of 16 keys of one head in a block of keys.
struct Cut {
  int heads, cols, subs;
};
template <typename T, int D>
__host__ __device__ inline Cut cut_of(int hkv, int hq, int64_t most_cols) {
  constexpr int kCols = Piece<T, D>::kQBytes / (D * (int)sizeof(T));
  Cut c;
  c.heads = hkv * 8 <= kCols ? hkv : kCols / 8;
  c.heads = c.heads < kItems ? c.heads : kItems;
  const int64_t fit = (int64_t)(kCols / c.heads) & ~int64_t(7), need = (most_cols + 7) & ~int64_t(7);
  c.cols = (int)(fit < need ? fit : need);
  c.subs = kItems / c.heads < kMaxSubs ? kItems / c.heads : kMaxSubs;
  return c;
}

template <typename T, int D>
__global__ void __launch_bounds__(kThreads, 1) weigh_kernel(const __grid_constant__ WeighArgs a) {
  constexpr int kCols = Piece<T, D>::kQBytes / (D * (int)sizeof(T)), kPieces = D * (int)sizeof(T) / 16;
  using P = Piece<T, D>;
  extern __shared__ __align__(16) char s_q[];            // queries, then a ring for every warp
  __shared__ float s_lse[kCols];
  __shared__ int s_lim[kCols], s_row[kCols];
  __shared__ float s_part[2][kItems][kKeys];
  __shared__ uint32_t s_bits[2 * (kMaxSeqs / 32)];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const char *ring = s_q + P::kQBytes + warp * P::kStages * P::kBytes;
  const uint32_t q_at = (uint32_t)__cvta_generic_to_shared(s_q), ring_at = (uint32_t)__cvta_generic_to_shared(ring);
  pdl_grid_wait();
  const uint32_t *twice = find_repeats(a.seqs, a.n, a.max_seqs, s_bits);

  // This block's share of the line of all sequences' pieces of 16 keys, which count for their columns; every warp finds it.  (Up to 32
  // sequences a lane keeps what it has read.)
  auto pieces_of = [&](const WeighSeq &s) { return (s.len + kKeys - 1) / kKeys; };
  auto units_of = [&](const WeighSeq &s) { return (uint64_t)(s.len ? kStart + pieces_of(s) : 0); };
  auto cost_of = [&](const WeighSeq &s) { return (uint64_t)(kExtra + ((int64_t)s.m * a.g + 7) / 8); };
  WeighSeq mine = {};
  uint64_t total = 0;
  for (int s0 = 0; s0 < a.n; s0 += 32) {
    mine = {};
    if (s0 + lane < a.n) mine = weigh_seq(a, s0 + lane, twice);
    uint64_t w = units_of(mine) * cost_of(mine);
#pragma unroll
    for (int o = 16; o; o >>= 1) w += __shfl_xor_sync(~0u, w, o);
    total += w;
  }
  const uint64_t share = (total + gridDim.x - 1) / gridDim.x, x0 = share * blockIdx.x, x1 = min(x0 + share, total);
  if (x0 >= x1) return;
  uint64_t at = 0;                                         // of the line: where sequence list begins
  int parity = 0;
  for (int s0 = 0; s0 < a.n && at < x1; s0 += 32) {
    if (a.n > 32) {
      mine = {};
      if (s0 + lane < a.n) mine = weigh_seq(a, s0 + lane, twice);
    }
    const uint64_t w = units_of(mine) * cost_of(mine);
    uint64_t upto = w;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const uint64_t y = __shfl_up_sync(~0u, upto, o);
      if (lane >= o) upto += y;
    }
    const uint32_t ours = __ballot_sync(~0u, w > 0 && at + upto > x0 && at + upto - w < x1);
    for (uint32_t left = ours; left; left &= left - 1) {
      const int l = __ffs(left) - 1, list = s0 + l;
      WeighSeq s;
      s.q0 = __shfl_sync(~0u, mine.q0, l);
      s.n = __shfl_sync(~0u, mine.n, l);
      s.m = __shfl_sync(~0u, mine.m, l);
      s.len = __shfl_sync(~0u, mine.len, l);
      s.base = s.len - s.m;
      s.id = __shfl_sync(~0u, mine.id, l);
      const uint64_t begin = at + __shfl_sync(~0u, upto - w, l), cost = cost_of(s);
      // the pieces that begin inside of the share
      const int b0 = begin >= x0 ? 0 : (int)max((int64_t)((x0 - begin + cost - 1) / cost) - kStart, (int64_t)0);
      const int b1 = (int)min((int64_t)pieces_of(s), (int64_t)((x1 - begin + cost - 1) / cost) - kStart);
      if (b0 >= b1) continue;
      const int32_t *table = a.table + (int64_t)s.id * a.max_pages;
      float *weight = a.weight + s.id * a.weight_stride;
      const int all_cols = s.m * a.g;
      const Cut cut = cut_of<T, D>(a.hkv, a.hq, all_cols);
      bool first = true;
      for (int h0 = 0; h0 < a.hkv; h0 += cut.heads)
        for (int c0 = 0; c0 < all_cols; c0 += cut.cols) {
          const int heads = min(cut.heads, a.hkv - h0);
          const int cols = min(cut.cols, all_cols - c0), tiles = (cols + 7) >> 3;
          // A block of keys, cut.subs pieces, after another, the warps in turn its (piece, head) pairs; the page of a pair is looked
          // up one pair ahead of its copies.
          const int up = kWarps / heads, over = kWarps % heads, sub0 = warp / heads, head0 = warp % heads;
          auto on = [&](int &sub, int &h) {                // to a warp's next pair: piece of the block, head
            sub += up;
            h += over;
            if (h >= heads) { h -= heads; ++sub; }
          };
          int nb = b0, ni = warp, nsub = sub0, nh = head0; // the pair that is looked up
          auto pairs_of = [&](int b) { return min(cut.subs, b1 - b) * heads; };
          auto look = [&]() -> const T * {
            if (ni >= pairs_of(nb)) { ni = warp; nsub = sub0; nh = head0; nb += cut.subs; }       // (a later block has no more pairs than this one)
            if (ni >= pairs_of(nb)) nb = b1;
            if (nb >= b1) return nullptr;
            return (const T *)a.k + (weigh_page_row(a, table, (nb + nsub) * kKeys) + (int64_t)(h0 + nh) * a.page) * D;
          };
          uint32_t in = 0, out = 0;                        // pairs sent for, pairs done
          const T *from = look();
          auto fetch = [&]() {
            if (from) {
              P::fetch(from, ring_at + (in % P::kStages) * P::kBytes);
              ni += kWarps;
              on(nsub, nh);
              from = look();
            }
            asm volatile("cp.async.commit_group;" ::: "memory");
            ++in;
          };
#pragma unroll
          for (int i = 0; i < P::kStages - 1; ++i) fetch();
          __syncthreads();                                 // the last ones are done with what is replaced
          // the columns, then their queries
          for (int u = tid; u < heads * tiles * 8; u += kThreads) {
            const int col = u % (tiles * 8), h = u / (tiles * 8);
            int lim = -1, row = -1;
            float lse = 0.f;
            if (col < cols) {
              const int k = (c0 + col) / a.g, head = (h0 + h) * a.g + c0 + col - k * a.g;
              row = counted_row(a, s, list, k);
              if (row >= 0) {
                lse = a.lse[(int64_t)row * a.hq + head];
                if (lse != -INFINITY) lim = s.base + k;    // a row that saw nothing adds nothing
              }
            }
            s_lse[u] = lse * kLog2ef;
            s_lim[u] = lim;
            s_row[u] = row;
          }
          __syncthreads();
          for (int u = tid; u < heads * tiles * 8 * kPieces; u += kThreads) {
            const int c = u % kPieces, hc = u / kPieces, col = hc % (tiles * 8), h = hc / (tiles * 8), row = s_row[hc];
            const int head = (h0 + h) * a.g + (c0 + col) % a.g;
            const char *from = (const char *)((const T *)a.q + (row < 0 ? 0 : row * a.q_stride + (int64_t)head * D)) + c * 16;
            asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(q_at + h * tiles * 8 * kPieces * 16 + P::place(col, c)), "l"(from), "r"(row < 0 ? 0 : 16) : "memory");
          }
          asm volatile("cp.async.wait_all;" ::: "memory");
          __syncthreads();
          for (int b = b0; b < b1; b += cut.subs) {
            const int pairs = pairs_of(b);
            int sub = sub0, h = head0;
            for (int i = warp; i < pairs; i += kWarps, on(sub, h)) {
              fetch();
              asm volatile("cp.async.wait_group %0;" ::"n"(P::kStages - 1) : "memory");
              __syncwarp();
              P now;
              now.load(ring + (out % P::kStages) * P::kBytes);
              ++out;
              const float w16 = now.sums(s_q + (size_t)h * tiles * 8 * kPieces * 16, s_lse + h * tiles * 8, s_lim + h * tiles * 8, cols, (b + sub) * kKeys, a.scale_log2);
              if (lane < kKeys) s_part[parity][i][lane] = w16;
              __syncwarp();                                // the stage is read before it is filled again
            }
            __syncthreads();
            const int p = b * kKeys + tid;
            if (tid < min(cut.subs, b1 - b) * kKeys && p < s.len) {
              float sum = 0.f;
              for (int h = 0; h < heads; ++h) sum += s_part[parity][(tid / kKeys) * heads + h][tid % kKeys];
              weight[p] = first && a.fresh && p >= s.base ? sum : weight[p] + sum;
            }
            parity ^= 1;
          }
          first = false;
          asm volatile("cp.async.wait_all;" ::: "memory");
        }
    }
    at += __shfl_sync(~0u, upto, 31);
  }
}

template <typename T, int D>
pcomoe_status run(const WeighArgs &a, int sms, cudaStream_t st) {
  constexpr int kSmem = Piece<T, D>::kQBytes + kWarps * Piece<T, D>::kStages * Piece<T, D>::kBytes;
  static PerDeviceOnce once;
  int dev = -1;
  PCOMOE_CUDA_TRY(cudaGetDevice(&dev));
  if (once.first_use(dev)) {
    PCOMOE_CUDA_TRY(cudaFuncSetAttribute(weigh_kernel<T, D>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmem));
    once.done(dev);
  }
  PCOMOE_CUDA_TRY(launch_pdl(weigh_kernel<T, D>, dim3(sms), dim3(kThreads), kSmem, st, a));
  count_launch();
  return PCOMOE_OK;
}

pcomoe_status check_config(const pcomoe_attn_config *c, const pcomoe_cache *cache) {
  if (!c || c->struct_size != (int32_t)sizeof(pcomoe_attn_config)) return PCOMOE_ERR_INVALID_ARG;
  if (c->q_heads <= 0 || c->kv_heads <= 0 || c->q_heads % c->kv_heads || c->head_dim <= 0 || !(c->scale > 0.f) || !std::isfinite(c->scale))
    return PCOMOE_ERR_INVALID_ARG;
  if (c->dtype != PCOMOE_BF16 && c->dtype != PCOMOE_FP32) return PCOMOE_ERR_INVALID_ARG;
  if (c->head_dim != 64 && c->head_dim != 128) return PCOMOE_ERR_UNSUPPORTED;
  if (c->q_heads > 4096) return PCOMOE_ERR_SHAPE;
  const pcomoe_status st = check_cache(cache);
  if (st != PCOMOE_OK) return st;
  if (cache->kv_heads != c->kv_heads || cache->head_dim != c->head_dim || cache->dtype != c->dtype) return PCOMOE_ERR_INVALID_ARG;
  return PCOMOE_OK;
}

// Workspace: a status word, partial sums of the kernel of many rows.
size_t workspace_of(const pcomoe_attn_config *c, const pcomoe_cache *cache, int n) {
  return 256 + weigh_part_bytes(c->kv_heads, (int64_t)cache->max_pages * cache->page_size, n);
}

}  // namespace
}  // namespace pcomoe

using namespace pcomoe;

extern "C" {

pcomoe_status pcomoe_weigh_workspace_bytes(const pcomoe_attn_config *cfg, const pcomoe_cache *cache, int32_t n, size_t *bytes) {
  if (!bytes) return PCOMOE_ERR_INVALID_ARG;
  const pcomoe_status st = check_config(cfg, cache);
  if (st != PCOMOE_OK) return st;
  if (n < 0) return PCOMOE_ERR_INVALID_ARG;
  if (n > cache->max_seqs) return PCOMOE_ERR_SHAPE;
  *bytes = workspace_of(cfg, cache, n);
  return PCOMOE_OK;
}

pcomoe_status pcomoe_cache_weigh(const pcomoe_attn_config *cfg, const pcomoe_cache *cache, int32_t layer, int32_t T, int32_t n, const int32_t *d_seqs,
                                 const int32_t *d_cu_len, const void *d_q, int64_t q_stride, const float *d_lse, const int32_t *d_keep,
                                 int32_t keep_stride, const int32_t *d_n_keep, int32_t fresh, float *d_weight, int64_t weight_stride,
                                 void *d_workspace, size_t ws_bytes, void *stream) {
  pcomoe_status st = check_config(cfg, cache);
  if (st != PCOMOE_OK) return st;
  if (layer < 0 || layer >= cache->layers || n < 0) return PCOMOE_ERR_INVALID_ARG;
  if (T < 0 || n > cache->max_seqs) return PCOMOE_ERR_SHAPE;
  if (T == 0 || n == 0) return PCOMOE_OK;
  if (!d_seqs || !d_cu_len || !d_q || !d_lse || !d_weight || !d_keep != !d_n_keep || (d_keep && keep_stride <= 0)) return PCOMOE_ERR_INVALID_ARG;
  if (q_stride < (int64_t)cfg->q_heads * cfg->head_dim || weight_stride < (int64_t)cache->max_pages * cache->page_size) return PCOMOE_ERR_INVALID_ARG;
  const int64_t e = (int64_t)dtype_size(cfg->dtype);
  if (((uintptr_t)d_q & 15) || (q_stride * e) % 16) return PCOMOE_ERR_UNSUPPORTED;
  if ((int64_t)T * (cfg->q_heads / cfg->kv_heads) > INT32_MAX - 1024) return PCOMOE_ERR_SHAPE;
  if (!d_workspace || ((uintptr_t)d_workspace & 255) || ws_bytes < workspace_of(cfg, cache, n)) return PCOMOE_ERR_WORKSPACE;
  int sms;
  if ((st = current_sms(&sms)) != PCOMOE_OK) return st;
  WeighArgs a = {};
  a.T = T; a.n = n; a.hq = cfg->q_heads; a.hkv = cfg->kv_heads; a.g = cfg->q_heads / cfg->kv_heads;
  a.scale_log2 = cfg->scale * 1.4426950408889634f;
  a.seqs = d_seqs; a.cu = d_cu_len; a.keep = d_keep; a.n_keep = d_n_keep; a.keep_stride = keep_stride; a.fresh = fresh != 0;
  a.q = d_q; a.q_stride = q_stride; a.lse = d_lse;
  a.k = (const char *)cache->d_k + (int64_t)layer * cache->pages * cache->kv_heads * cache->page_size * cache->head_dim * e;
  a.len = cache->d_seq_len; a.table = cache->d_page_table;
  a.pages = cache->pages; a.page = cache->page_size; a.max_seqs = cache->max_seqs; a.max_pages = cache->max_pages;
  for (a.page_shift = 0; (1 << a.page_shift) < cache->page_size;) ++a.page_shift;
  a.weight = d_weight; a.weight_stride = weight_stride;
  a.status = (int32_t *)((char *)d_workspace + offsetof(DevPlan, status_router));
  a.limit_ns = wait_limit_ns();
  // Many counted rows (columns, with the heads of a group) per sequence: the kernels that divide them into tiles.
  float *partial = (float *)((char *)d_workspace + 256);
  const int64_t room = (int64_t)cache->max_pages * cache->page_size;
  const int64_t counted = d_keep ? std::min<int64_t>(T, (int64_t)n * keep_stride) : T;
  if (counted * a.g >= (int64_t)(cfg->dtype == PCOMOE_BF16 ? kManyColumns : kManyColumnsF32) * n)
    return cfg->dtype == PCOMOE_BF16 ? launch_weigh_tc(a, cfg->head_dim, partial, room, sms, (cudaStream_t)stream)
                                     : launch_weigh_simt(a, cfg->head_dim, partial, room, sms, (cudaStream_t)stream);
  if (cfg->dtype == PCOMOE_BF16) return cfg->head_dim == 64 ? run<__nv_bfloat16, 64>(a, sms, (cudaStream_t)stream) : run<__nv_bfloat16, 128>(a, sms, (cudaStream_t)stream);
  return cfg->head_dim == 64 ? run<float, 64>(a, sms, (cudaStream_t)stream) : run<float, 128>(a, sms, (cudaStream_t)stream);
}

}  // extern "C"
