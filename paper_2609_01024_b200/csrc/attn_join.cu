// Joins the partial results of tiles that the cached attention kernels cut: a second launch, so that all SMs take part.
//
// o = sum_i 2^(m_i - m) o_i / sum_i 2^(m_i - m) l_i over a row's parts, in their order.  A block looks at the record of one
// CTA and takes up to 32 rows of the tile that it left unfinished, four rows per warp.  All it waits for is L2: eight lanes
// per row hold the parts' maxima and sums, and the sums of four parts are on their way before the weights are known.
// Measured (cold caches): 7 us for the parts of 32 decoding sequences, 10 us for 148 parts of up to 256 rows of 128.
#include <algorithm>

#include "attn.cuh"

namespace pcomoe {
namespace {

constexpr int kWarps = 8;

template <typename T, int V> __device__ __forceinline__ void store_row(T *p, const float (&x)[V], float by) {
#pragma unroll
  for (int k = 0; k < V; k += 2) {
    if (sizeof(T) == 4) {
      *(float2 *)(p + k) = make_float2(x[k] * by, x[k + 1] * by);
    } else {
      const __nv_bfloat162 v = __floats2bfloat162_rn(x[k] * by, x[k + 1] * by);
      *(uint32_t *)(p + k) = *(const uint32_t *)&v;
    }
  }
}

template <typename T, int D, int BM>
__global__ void __launch_bounds__(32 * kWarps) join_kernel(AttnArgs a) {
  pdl_grid_wait();
  constexpr int R = 4, U = 4, V = D / 32;                  // rows and parts at a time, columns of a lane
  const JoinRec s = a.recs[blockIdx.x];
  if (s.n_parts == 0) return;
  const int kvh = s.kvh, tile = s.tile, first_cta = blockIdx.x, n_parts = s.n_parts;
  const int rows = min(BM, s.n * a.g - tile * BM), lane = threadIdx.x & 31, mine = lane & 7;
  const int r0 = (blockIdx.y * kWarps + (threadIdx.x >> 5)) * R;
  if (r0 < rows) {
    float x[U][R][V], o[R][V];
    auto fetch = [&](int i0) {
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int i = min(i0 + u, n_parts - 1);
#pragma unroll
        for (int j = 0; j < R; ++j) {
          const float *src = a.part + ((int64_t)part_slot(first_cta + i, i == 0) * BM + min(r0 + j, rows - 1)) * D + lane * V;
          if (V == 4) {
            const float4 y = __ldcg((const float4 *)src);
            x[u][j][0] = y.x; x[u][j][1] = y.y; x[u][j][V - 2] = y.z; x[u][j][V - 1] = y.w;
          } else {
            const float2 y = __ldcg((const float2 *)src);
            x[u][j][0] = y.x; x[u][j][1] = y.y;
          }
        }
      }
    };
    fetch(0);
    const int row8 = min(r0 + (lane >> 3), rows - 1);      // the row of this lane's parts (mine, mine + 8, ...)
    auto stat = [&](int i) { return __ldcg((const float2 *)a.part_ml + (int64_t)part_slot(first_cta + i, i == 0) * BM + row8); };
    const float2 ml0 = mine < n_parts ? stat(mine) : make_float2(-INFINITY, 0.f);
    float m = ml0.x;
    for (int i = mine + 8; i < n_parts; i += 8) m = fmaxf(m, stat(i).x);
#pragma unroll
    for (int h = 4; h; h >>= 1) m = fmaxf(m, __shfl_xor_sync(~0u, m, h));
    const float ms = m == -INFINITY ? 0.f : m;
    float l = 0.f, w = 0.f;
#pragma unroll
    for (int j = 0; j < R; ++j)
#pragma unroll
      for (int k = 0; k < V; ++k) o[j][k] = 0.f;
    for (int i0 = 0; i0 < n_parts; i0 += U) {
      if ((i0 & 7) == 0) {                                 // the weights of eight parts, one per lane
        const float2 ml = i0 == 0 ? ml0 : i0 + mine < n_parts ? stat(i0 + mine) : make_float2(-INFINITY, 0.f);
        w = part_weight(ml.x, ml.y, ms);
        if (w != kNoPart) l += w * ml.y;
      }
      if (i0) fetch(i0);
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int j = 0; j < R; ++j) {
          const float wi = __shfl_sync(~0u, w, 8 * j + ((i0 + u) & 7));
          if (wi != kNoPart && i0 + u < n_parts)
#pragma unroll
            for (int k = 0; k < V; ++k) o[j][k] = fmaf(wi, x[u][j][k], o[j][k]);
        }
    }
#pragma unroll
    for (int h = 4; h; h >>= 1) l += __shfl_xor_sync(~0u, l, h);
#pragma unroll
    for (int j = 0; j < R; ++j) {
      const float lj = __shfl_sync(~0u, l, 8 * j), mj = __shfl_sync(~0u, ms, 8 * j);
      if (r0 + j >= rows) continue;
      const int row = tile * BM + r0 + j, tok = row / a.g, head = kvh * a.g + row - tok * a.g;
      const int64_t t = s.q0 + tok;
      const float inv = lj == 0.f ? 0.f : 1.f / lj;
      store_row<T, V>((T *)a.out + t * a.out_stride + head * D + lane * V, o[j], inv);
      if (lane == 0 && a.lse) a.lse[t * a.hq + head] = lj == 0.f ? -INFINITY : mj * kLn2f + logf(lj);
    }
  }
}

template <typename T, int D, int BM>
pcomoe_status run(const AttnArgs &a, int ctas, cudaStream_t st) {
  PCOMOE_CUDA_TRY(launch_pdl(join_kernel<T, D, BM>, dim3(ctas, (BM + 4 * kWarps - 1) / (4 * kWarps)), dim3(32 * kWarps), 0, st, a));
  count_launch();
  return PCOMOE_OK;
}

}  // namespace

// rows: of a partial result's place: 64 for fp32, 16 or 256 for bf16
pcomoe_status launch_attn_join(const AttnArgs &a, int D, int dtype, int rows, int ctas, cudaStream_t st) {
  using bf16 = __nv_bfloat16;
  if (dtype == PCOMOE_FP32) return D == 64 ? run<float, 64, 64>(a, ctas, st) : run<float, 128, 64>(a, ctas, st);
  if (rows == 16) return D == 64 ? run<bf16, 64, 16>(a, ctas, st) : run<bf16, 128, 16>(a, ctas, st);
  return D == 64 ? run<bf16, 64, 256>(a, ctas, st) : run<bf16, 128, 256>(a, ctas, st);
}

}  // namespace pcomoe
