// Attention of a few rows over the paged cache, bf16: decode steps and small drafts (tiles of 16 rows per kv head and sequence).
//
// Mathematics as in the other attention kernels: one pass over the keys with a running maximum and sum per row, base 2.
// What bounds it: reading the cache once (HBM).  With g heads on a kv head a byte of K or V takes part in g
// multiply-adds, so 16-row warp MMAs (m16n8k16) do the products with most of their time to spare (the second one takes the
// weights in bf16, the type of its other operand, an error of at most 2^-8 of each; their sum takes them unrounded), and the
// kernel is built around loads in flight: every warp has its own ring of three pieces of 16 keys (K and V, 8 KB at D =
// 128), filled with 16-byte asynchronous copies, and takes every fourth piece of the CTA's share; nothing in the loop waits
// for another warp.  16 keys never cross a page (pages hold a multiple of 16), so a piece is one page lookup and one
// contiguous run per K and V.  Two CTAs per SM: while one joins its warps' results the other one's loads go on.
// Measured with the joining launch, 32 heads on 8 of 128: 32 sequences of 1 to 4095 tokens 46 us for 243 MB, 5.2 TB/s (ends and
// beginnings of pieces and the second launch); two of 131071 and 100003 tokens 155 us for 946 MB, 6.1 TB/s, 0.93 of a
// plain copy's rate; two sequences of 4 tokens 5.7 us.
#include <algorithm>

#include "attn.cuh"

namespace pcomoe {
namespace {

constexpr int BM = 16, BN = 64, kWarps = 4, kThreads = 32 * kWarps, kStages = 3, kKeys = 16;
constexpr int kExtra = 3;              // blocks of 64 keys that a piece of work costs besides its own

template <int D> constexpr int stage_bytes() { return 2 * kKeys * D * 2; }
template <int D> constexpr int smem_bytes() { return kWarps * kStages * stage_bytes<D>(); }

__device__ __forceinline__ void ldsm4(uint32_t at, uint32_t (&r)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at) : "memory");
}
__device__ __forceinline__ void ldsm4t(uint32_t at, uint32_t (&r)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at) : "memory");
}
__device__ __forceinline__ void mma(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
  const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
  return *(const uint32_t *)&v;
}

// Rows of a tile that may have to be formed again, every fourth to a warp.
template <int D>
__device__ __noinline__ void form_again(const AttnArgs &a, Seq seq, int kvh, int tile, int b0, int b1, int rows, bool whole, int slot, const uint8_t *bad) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, mine = lane % BM;      // row of this lane
  const bool met = met_unseen<D, true>(a, seq, kvh, (tile * BM + min(mine, rows - 1)) / a.g, b0 * BN, b1 * BN, seq.base, bad[mine]);
  const uint32_t todo = __ballot_sync(~0u, met && lane < BM && lane % kWarps == warp);
  plain_rows<D, BM, true>(a, seq, kvh, tile * BM, 0, todo, b0 * BN, b1 * BN, whole, slot);
}

template <int D>
__global__ void __launch_bounds__(kThreads, 2) few_kernel(const __grid_constant__ AttnArgs a) {
  constexpr int kChunks = D / 8;                          // 16-byte pieces of a row
  extern __shared__ __align__(1024) uint8_t smem[];
  __shared__ float2 s_ml[kWarps][BM];
  __shared__ uint8_t s_bad[BM];
  __shared__ int s_again;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const uint32_t ring = smem_u32(smem) + warp * kStages * stage_bytes<D>();
  pdl_grid_wait();
  CacheWalk<BM, BN, kExtra, 8> w;
  CacheWalk<BM, BN, kExtra, 8>::Piece p;
  w.start(a, blockIdx.x, gridDim.x);
  while (w.next(a, p)) {
    const Seq seq = w.seq;
    const int rows = min(BM, seq.n * a.g - p.tile * BM);
    const int r0 = lane >> 2, r1 = r0 + 8;                // the rows of this lane's fragments
    int tok[2];
    tok[0] = (p.tile * BM + min(r0, rows - 1)) / a.g;
    tok[1] = (p.tile * BM + min(r1, rows - 1)) / a.g;
    float o[D / 8][4];
#pragma unroll
    for (int n = 0; n < D / 8; ++n) o[n][0] = o[n][1] = o[n][2] = o[n][3] = 0.f;
    float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};
    const int32_t *table = a.table + (int64_t)seq.id * a.max_pages;
    const int p0 = p.b0 * BN, p1 = min(p.b1 * BN, max(seq.len, 1));
    const int steps = (p1 - p0 + kKeys * (kWarps - warp) - 1) / (kKeys * kWarps);       // pieces of this warp
    auto first_key = [&](int i) { return p0 + (i * kWarps + warp) * kKeys; };
    // pages are looked up one piece ahead of the copies that use them
    auto look = [&](int i) { return i < steps && first_key(i) < seq.len ? page_row(a, table, p.kvh, first_key(i)) : (int64_t)0; };
    int64_t next_row = look(0);
    auto load = [&](int i) {
      if (i < steps) {
        const int left = seq.len - first_key(i);          // keys that exist; the rest becomes zero
        const uint32_t to = ring + (i % kStages) * stage_bytes<D>();
        const char *k = (const char *)a.k + next_row * (D * 2), *v = (const char *)a.v + next_row * (D * 2);
#pragma unroll
        for (int j = 0; j < kKeys * kChunks / 32; ++j) {
          const int u = j * 32 + lane, r = u / kChunks, c = u % kChunks;
          const uint32_t at = to + r * (D * 2) + ((c ^ (r & 7)) << 4);
          copy16(at, k + u * 16, r < left);
          copy16(at + kKeys * D * 2, v + u * 16, r < left);
        }
        next_row = look(i + 1);
      }
      asm volatile("cp.async.commit_group;" ::: "memory");
    };
#pragma unroll
    for (int i = 0; i < kStages - 1; ++i) load(i);
    uint32_t q[D / 16][4];                                // A fragments of the queries
    {
      const __nv_bfloat16 *row[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int rr = p.tile * BM + min(i ? r1 : r0, rows - 1);
        row[i] = (const __nv_bfloat16 *)a.q + (int64_t)(seq.q0 + tok[i]) * a.q_stride + (p.kvh * a.g + rr - tok[i] * a.g) * D + (lane & 3) * 2;
      }
#pragma unroll
      for (int k = 0; k < D / 16; ++k) {
        q[k][0] = *(const uint32_t *)(row[0] + k * 16);
        q[k][1] = *(const uint32_t *)(row[1] + k * 16);
        q[k][2] = *(const uint32_t *)(row[0] + k * 16 + 8);
        q[k][3] = *(const uint32_t *)(row[1] + k * 16 + 8);
      }
    }
    for (int i = 0; i < steps; ++i) {
      load(i + kStages - 1);
      asm volatile("cp.async.wait_group %0;" ::"n"(kStages - 1) : "memory");
      __syncwarp();
      const uint32_t kt = ring + (i % kStages) * stage_bytes<D>(), vt = kt + kKeys * D * 2;
      float s[2][4] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
      {
        // one x4 load: keys 0-7 and 8-15, two 8-column pieces each
        const int r = (lane & 7) + ((lane >> 4) << 3), half = (lane >> 3) & 1;
#pragma unroll
        for (int k = 0; k < D / 16; ++k) {
          uint32_t b[4];
          ldsm4(kt + r * (D * 2) + (((2 * k + half) ^ (r & 7)) << 4), b);
          mma(s[0], q[k], b[0], b[1]);
          mma(s[1], q[k], b[2], b[3]);
        }
      }
      const int key0 = first_key(i);
      if (key0 + kKeys > seq.base) {
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          const uint32_t bits = seen_bits<true>(a, seq, tok[x], key0) >> ((lane & 3) * 2);
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            if (!((bits >> (8 * j)) & 1)) s[j][2 * x] = -INFINITY;
            if (!((bits >> (8 * j + 1)) & 1)) s[j][2 * x + 1] = -INFINITY;
          }
        }
      }
      float mb[2];
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        mb[x] = fmaxf(fmaxf(s[0][2 * x], s[0][2 * x + 1]), fmaxf(s[1][2 * x], s[1][2 * x + 1]));
        mb[x] = fmaxf(mb[x], __shfl_xor_sync(~0u, mb[x], 1));
        mb[x] = fmaxf(mb[x], __shfl_xor_sync(~0u, mb[x], 2)) * a.scale_log2;
      }
      if (__any_sync(~0u, mb[0] > m[0] || mb[1] > m[1])) {
        float c[2];
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          const float mn = fmaxf(m[x], mb[x]);
          c[x] = mn == -INFINITY ? 1.f : ex2f(m[x] - mn);
          m[x] = mn;
          l[x] *= c[x];
        }
#pragma unroll
        for (int n = 0; n < D / 8; ++n) { o[n][0] *= c[0]; o[n][1] *= c[0]; o[n][2] *= c[1]; o[n][3] *= c[1]; }
      }
      uint32_t w4[4];                                      // the weights as the A fragment of the second product
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        const float ms = m[x] == -INFINITY ? 0.f : m[x];
        float e[2][2];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          e[j][0] = ex2f(fmaf(s[j][2 * x], a.scale_log2, -ms));
          e[j][1] = ex2f(fmaf(s[j][2 * x + 1], a.scale_log2, -ms));
        }
        l[x] += (e[0][0] + e[0][1]) + (e[1][0] + e[1][1]);
        w4[x] = pack2(e[0][0], e[0][1]);
        w4[2 + x] = pack2(e[1][0], e[1][1]);
      }
      {
        const int r = (lane & 7) + (((lane >> 3) & 1) << 3), half = lane >> 4;
#pragma unroll
        for (int n = 0; n < D / 16; ++n) {
          uint32_t b[4];
          ldsm4t(vt + r * (D * 2) + (((2 * n + half) ^ (r & 7)) << 4), b);
          mma(o[2 * n], w4, b[0], b[1]);
          mma(o[2 * n + 1], w4, b[2], b[3]);
        }
      }
      __syncwarp();                                        // the stage is read before it is filled again
    }
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      l[x] += __shfl_xor_sync(~0u, l[x], 1);
      l[x] += __shfl_xor_sync(~0u, l[x], 2);
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
    __syncthreads();                                       // every warp is done with its ring: the rings hold the sums now
    constexpr int kPad = D + 4;
    float *so = (float *)smem;
    if ((lane & 3) == 0) {
      s_ml[warp][r0] = make_float2(m[0], l[0]);
      s_ml[warp][r1] = make_float2(m[1], l[1]);
    }
#pragma unroll
    for (int n = 0; n < D / 8; ++n) {
      const int c = n * 8 + (lane & 3) * 2;
      *(float2 *)(so + (warp * BM + r0) * kPad + c) = make_float2(o[n][0], o[n][1]);
      if (rows > 8) *(float2 *)(so + (warp * BM + r1) * kPad + c) = make_float2(o[n][2], o[n][3]);
    }
    if (tid < BM) s_bad[tid] = 0;
    if (tid == 0) s_again = 0;
    __syncthreads();
    const int slot = part_slot(blockIdx.x, p.b0 == 0);
    for (int u = tid; u < rows * (D / 4); u += kThreads) {
      const int r = u / (D / 4), c = u - r * (D / 4);
      float mm = s_ml[0][r].x;
#pragma unroll
      for (int i = 1; i < kWarps; ++i) mm = fmaxf(mm, s_ml[i][r].x);
      const float ms = mm == -INFINITY ? 0.f : mm;
      float ll = 0.f;
      float4 x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int i = 0; i < kWarps; ++i) {
        const float2 ml = s_ml[i][r];
        if (ml.y == 0.f) continue;                         // a warp in which the row saw nothing (kNoPart)
        const float wt = part_weight(ml.x, ml.y, ms);
        const float4 y = *(const float4 *)(so + (i * BM + r) * kPad + 4 * c);
        ll += wt * ml.y;
        x.x += wt * y.x; x.y += wt * y.y; x.z += wt * y.z; x.w += wt * y.w;
      }
      if (!(fabsf(x.x) < INFINITY && fabsf(x.y) < INFINITY && fabsf(x.z) < INFINITY && fabsf(x.w) < INFINITY) && ll == ll) {
        s_bad[r] = 1;                                      // (with a NaN score the row is NaN whatever the values are)
        s_again = 1;
      }
      if (p.whole) {
        const int row = p.tile * BM + r, tk = row / a.g, head = p.kvh * a.g + row - tk * a.g;
        const float inv = ll == 0.f ? 0.f : 1.f / ll;
        store4<__nv_bfloat16>((__nv_bfloat16 *)a.out + (int64_t)(seq.q0 + tk) * a.out_stride + head * D + 4 * c,
                              make_float4(x.x * inv, x.y * inv, x.z * inv, x.w * inv));
        if (c == 0 && a.lse) a.lse[(int64_t)(seq.q0 + tk) * a.hq + head] = ll == 0.f ? -INFINITY : ms * kLn2f + logf(ll);
      } else {
        const int64_t at = (int64_t)slot * BM + r;
        *(float4 *)(a.part + at * D + 4 * c) = x;
        if (c == 0) *((float2 *)a.part_ml + at) = make_float2(mm, ll);
      }
    }
    __syncthreads();
    if (s_again) {
      form_again<D>(a, seq, p.kvh, p.tile, p.b0, p.b1, rows, p.whole, slot, s_bad);
      __syncthreads();
    }
    __syncthreads();                                       // the rings are free again
  }
  if (tid == 0) w.record(a, blockIdx.x);
}

template <int D>
pcomoe_status run(const AttnArgs &a, int sms, cudaStream_t st) {
  static PerDeviceOnce once;
  int dev = -1;
  PCOMOE_CUDA_TRY(cudaGetDevice(&dev));
  if (once.first_use(dev)) {
    PCOMOE_CUDA_TRY(cudaFuncSetAttribute(few_kernel<D>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem_bytes<D>()));
    once.done(dev);
  }
  PCOMOE_CUDA_TRY(launch_pdl(few_kernel<D>, dim3(2 * sms), dim3(kThreads), smem_bytes<D>(), st, a));
  count_launch();
  return launch_attn_join(a, D, PCOMOE_BF16, BM, 2 * sms, st);
}

}  // namespace

size_t attn_few_part_rows(int sms) { return (size_t)4 * sms * BM; }

pcomoe_status launch_attn_few(const AttnArgs &a, int D, int sms, cudaStream_t st) {
  return D == 64 ? run<64>(a, sms, st) : run<128>(a, sms, st);
}

}  // namespace pcomoe
