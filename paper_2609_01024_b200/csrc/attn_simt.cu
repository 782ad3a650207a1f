// Attention with plain FMA, fp32: prompts and cached.  The fp32 layers' counterpart of the tensor-core kernels.
//
// One pass over the keys with the running maximum m and sum l of each row's softmax (in the base-2 domain):
//   m' = max(m, max s),  o <- 2^(m-m') o + sum 2^(s-m') v,  l <- 2^(m-m') l + sum 2^(s-m').
// A block of 256 threads owns a tile of 64 rows (prompts too small to fill the GPU with them: 16) and walks blocks of 64 keys
// through shared memory; a thread holds up to 4 rows x 4 columns of the scores and 4 rows x D/16 columns of the output in
// registers.  The weights lie over the keys, so that two blocks of threads fit on an SM at D = 128 and one computes
// while the other's copies are on their way (31 sequences of about 300 tokens with 5 to 63 drafts, 8 heads on 4: 117 us; one
// per SM 157).
// What bounds it: the shared-memory reads that feed the FMA pipe (with four rows to a thread 8 reads of 16 bytes to 64 FMA in the
// first product, and in the second, where a weight is a read of its own, 5 to 16 at D = 64 and 6 to 32 at 128; with one
// row 5 to 16 in the first), each block's wait for its own copies, and few tiles.  Two causal prompts of 1024 with 8 heads
// on 2: of 64 141 us, 15.3 TFLOP/s, the FMA pipe 45 % busy, of 128 248 us, 17.3 TFLOP/s, the last tiles' chains of 16
// blocks; 32 sequences of 2048 tokens with a token each, 16 heads on 4 of 128: 176 us, 1.5 TB/s.
#include <algorithm>

#include "attn.cuh"

namespace pcomoe {
namespace {

constexpr int BN = 64, kThreads = 256;

template <int D, int BM> constexpr int smem_floats() { return (BM + 2 * BN) * (D + 4); }

// RM: rows of a thread; a tile with few rows left takes fewer of them.

template <int D, int BM, int RM, bool kCached>
__device__ __forceinline__ void run_rows(const AttnArgs &a, const Seq &s, int kvh, int tile, int b0, int b1, bool whole, int slot, float *sm) {
  constexpr int DP = D + 4, PP = BN + 4, NC = D / 64;
  static_assert(BM * PP <= BN * DP, "the weights fit over the keys");
  float *Q = sm, *K = Q + BM * DP, *V = K + BN * DP, *P = K;      // weights over the keys, once every thread has its scores
  const int tid = threadIdx.x, ty = tid >> 4, tx = tid & 15;
  const int rows = min(16 * RM, s.n * a.g - tile * BM);
  // Everything comes in by asynchronous copies: the page lookups of all of a thread's rows are under way at once, and the
  // values arrive while the scores are formed.
  constexpr int kRowChunks = D / 4;
  __syncthreads();                                        // the last piece's readers are done
#pragma unroll
  for (int i = 0; i < 16 * RM * kRowChunks / kThreads; ++i) {
    const int u = tid + i * kThreads, r = u / kRowChunks, c = u - r * kRowChunks;
    const int row = tile * BM + min(r, rows - 1), t = row / a.g, head = kvh * a.g + row - t * a.g;
    copy16(smem_u32(Q + r * DP + 4 * c), (const float *)a.q + (int64_t)(s.q0 + t) * a.q_stride + head * D + 4 * c, r < rows);
  }
  float m[RM], l[RM];
  float4 o[RM][NC];
  int tok[RM];
#pragma unroll
  for (int i = 0; i < RM; ++i) {
    m[i] = -INFINITY;
    l[i] = 0.f;
    tok[i] = (tile * BM + min(ty * RM + i, rows - 1)) / a.g;
#pragma unroll
    for (int c = 0; c < NC; ++c) o[i][c] = make_float4(0.f, 0.f, 0.f, 0.f);
  }
  const int32_t *table = kCached ? a.table + (int64_t)s.id * a.max_pages : nullptr;
  for (int b = b0; b < b1; ++b) {
    const int p0 = b * BN;
    __syncthreads();
    constexpr int kCopies = BN * kRowChunks / kThreads;
    const int c4 = 4 * (tid % kRowChunks);
    int64_t from[kCopies];
#pragma unroll
    for (int i = 0; i < kCopies; ++i) {
      const int p = p0 + (tid + i * kThreads) / kRowChunks;
      from[i] = p >= s.len ? -1 : kCached ? page_row(a, table, kvh, p) : s.q0 + p;
    }
    // past the end: zero, so that no stale value can matter
#pragma unroll
    for (int i = 0; i < kCopies; ++i) {
      const int64_t at = max(from[i], (int64_t)0) * (kCached ? D : a.k_stride) + (kCached ? 0 : kvh * D) + c4;
      copy16(smem_u32(K + (tid + i * kThreads) / kRowChunks * DP + c4), (const float *)a.k + at, from[i] >= 0);
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
#pragma unroll
    for (int i = 0; i < kCopies; ++i) {
      const int64_t at = max(from[i], (int64_t)0) * (kCached ? D : a.v_stride) + (kCached ? 0 : kvh * D) + c4;
      copy16(smem_u32(V + (tid + i * kThreads) / kRowChunks * DP + c4), (const float *)a.v + at, from[i] >= 0);
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
    asm volatile("cp.async.wait_group 1;" ::: "memory");
    __syncthreads();
    float acc[RM][4];
#pragma unroll
    for (int i = 0; i < RM; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) acc[i][j] = 0.f;
#pragma unroll 4
    for (int d = 0; d < D; d += 4) {
      float4 kk[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) kk[j] = *(const float4 *)(K + (tx + 16 * j) * DP + d);
#pragma unroll
      for (int i = 0; i < RM; ++i) {
        const float4 qq = *(const float4 *)(Q + (ty * RM + i) * DP + d);
#pragma unroll
        for (int j = 0; j < 4; ++j)
          acc[i][j] = fmaf(qq.x, kk[j].x, fmaf(qq.y, kk[j].y, fmaf(qq.z, kk[j].z, fmaf(qq.w, kk[j].w, acc[i][j]))));
      }
    }
    // some row of the tile may not see all of the block
    const bool masked = p0 + BN > s.base || p0 + BN > s.len;
    asm volatile("cp.async.wait_group 0;" ::: "memory");
    float odd = 0.f;                                         // NaN once a value that this thread copied is NaN or infinite
    if (masked)
#pragma unroll
      for (int i = 0; i < kCopies; ++i) {
        const float4 y = *(const float4 *)(V + (tid + i * kThreads) / kRowChunks * DP + c4);
        odd = fmaf(0.f, y.x, fmaf(0.f, y.y, fmaf(0.f, y.z, fmaf(0.f, y.w, odd))));
      }
    const bool careful = __syncthreads_or(odd != 0.f);       // the values are there, and every thread is done with the keys
#pragma unroll
    for (int i = 0; i < RM; ++i) {
      float x[4], mx = -INFINITY;
      uint32_t lo = ~0u, hi = ~0u;
      if (masked) {
        lo = seen_bits<kCached>(a, s, tok[i], p0);
        hi = seen_bits<kCached>(a, s, tok[i], p0 + 32);
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const uint32_t w = j < 2 ? lo : hi;
        x[j] = (w >> (tx + 16 * (j & 1))) & 1u ? acc[i][j] * a.scale_log2 : -INFINITY;
        mx = fmaxf(mx, x[j]);
      }
#pragma unroll
      for (int q = 8; q; q >>= 1) mx = fmaxf(mx, __shfl_xor_sync(~0u, mx, q));
      const float mn = fmaxf(m[i], mx), ms = mn == -INFINITY ? 0.f : mn;
      const float r = ex2f(m[i] - ms);
      float sum = 0.f;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float p = ex2f(x[j] - ms);
        sum += p;
        P[(ty * RM + i) * PP + tx + 16 * j] = p;
      }
#pragma unroll
      for (int q = 8; q; q >>= 1) sum += __shfl_xor_sync(~0u, sum, q);
      l[i] = l[i] * r + sum;
      m[i] = mn;
#pragma unroll
      for (int c = 0; c < NC; ++c) { o[i][c].x *= r; o[i][c].y *= r; o[i][c].z *= r; o[i][c].w *= r; }
    }
    __syncwarp();                                            // a row's weights are written and read by one warp
    if (!careful) {
#pragma unroll 4
      for (int n = 0; n < BN; ++n)
#pragma unroll
        for (int c = 0; c < NC; ++c) {
          const float4 vv = *(const float4 *)(V + n * DP + 4 * tx + 64 * c);
#pragma unroll
          for (int i = 0; i < RM; ++i) {
            const float p = P[(ty * RM + i) * PP + n];
            o[i][c].x = fmaf(p, vv.x, o[i][c].x); o[i][c].y = fmaf(p, vv.y, o[i][c].y);
            o[i][c].z = fmaf(p, vv.z, o[i][c].z); o[i][c].w = fmaf(p, vv.w, o[i][c].w);
          }
        }
    } else {
      // a value that a row does not see does not touch it, NaN and infinities included; one that it sees does, with a weight
      // that is 0 in fp32 too
#pragma unroll 1
      for (int n = 0; n < BN; ++n) {
        uint32_t sees = 0;
#pragma unroll
        for (int i = 0; i < RM; ++i) sees |= ((seen_bits<kCached>(a, s, tok[i], p0 + (n & 32)) >> (n & 31)) & 1u) << i;
#pragma unroll
        for (int c = 0; c < NC; ++c) {
          const float4 vv = *(const float4 *)(V + n * DP + 4 * tx + 64 * c);
#pragma unroll
          for (int i = 0; i < RM; ++i) {
            const float p = P[(ty * RM + i) * PP + n];
            if ((sees >> i) & 1) {
              o[i][c].x = fmaf(p, vv.x, o[i][c].x); o[i][c].y = fmaf(p, vv.y, o[i][c].y);
              o[i][c].z = fmaf(p, vv.z, o[i][c].z); o[i][c].w = fmaf(p, vv.w, o[i][c].w);
            }
          }
        }
      }
    }
  }
#pragma unroll
  for (int i = 0; i < RM; ++i) {
    const int r = ty * RM + i;
    if (r >= rows) continue;
    if (whole) {
      const int row = tile * BM + r, head = kvh * a.g + row - tok[i] * a.g;
      const int64_t t = s.q0 + tok[i];
      const float inv = l[i] == 0.f ? 0.f : 1.f / l[i];
#pragma unroll
      for (int c = 0; c < NC; ++c)
        store4<float>((float *)a.out + t * a.out_stride + head * D + 4 * tx + 64 * c,
                  make_float4(o[i][c].x * inv, o[i][c].y * inv, o[i][c].z * inv, o[i][c].w * inv));
      if (tx == 0 && a.lse) a.lse[t * a.hq + head] = l[i] == 0.f ? -INFINITY : m[i] * kLn2f + logf(l[i]);
    } else {
      const int64_t at = (int64_t)slot * BM + r;
#pragma unroll
      for (int c = 0; c < NC; ++c) *(float4 *)(a.part + at * D + 4 * tx + 64 * c) = o[i][c];
      if (tx == 0) *((float2 *)a.part_ml + at) = make_float2(m[i], l[i]);
    }
  }
}

template <int D, int BM, bool kCached>
__device__ __forceinline__ void run_piece(const AttnArgs &a, const Seq &s, int kvh, int tile, int b0, int b1, bool whole, int slot, float *sm) {
  const int rows = s.n * a.g - tile * BM;
  if (BM == 16 || rows <= 16)
    run_rows<D, BM, 1, kCached>(a, s, kvh, tile, b0, b1, whole, slot, sm);
  else if (rows <= 32)
    run_rows<D, BM, 2, kCached>(a, s, kvh, tile, b0, b1, whole, slot, sm);
  else
    run_rows<D, BM, 4, kCached>(a, s, kvh, tile, b0, b1, whole, slot, sm);
}

template <int D>
__global__ void __launch_bounds__(kThreads, 2) simt_cached_kernel(AttnArgs a) {
  pdl_grid_wait();
  extern __shared__ float4 sm4[];
  CacheWalk<64, BN, 2, 1> w;
  CacheWalk<64, BN, 2, 1>::Piece p;
  w.start(a, blockIdx.x, gridDim.x);
  while (w.next(a, p))
    run_piece<D, 64, true>(a, w.seq, p.kvh, p.tile, p.b0, p.b1, p.whole, part_slot(blockIdx.x, p.b0 == 0), (float *)sm4);
  if (threadIdx.x == 0) w.record(a, blockIdx.x);
}

// One tile per block; the tiles are counted from the last one back, so that those with the most keys start first.
template <int D, int BM>
__global__ void __launch_bounds__(kThreads, 2) simt_prompt_kernel(AttnArgs a) {
  pdl_grid_wait();
  extern __shared__ float4 sm4[];
  const int lane = threadIdx.x & 31;
  int want = gridDim.x - 1 - blockIdx.x, tile = -1, s = 0;
  for (int s0 = 0; s0 < a.n_seqs && tile < 0; s0 += 32) {
    const int n = s0 + lane < a.n_seqs ? (load_seq<false>(a, s0 + lane).n * a.g + BM - 1) / BM : 0;
    int upto = n;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int y = __shfl_up_sync(~0u, upto, o);
      if (lane >= o) upto += y;
    }
    const uint32_t hit = __ballot_sync(~0u, upto > want);
    if (hit) {
      const int l = __ffs(hit) - 1;
      s = s0 + l;
      tile = want - __shfl_sync(~0u, upto - n, l);
    } else {
      want -= __shfl_sync(~0u, upto, 31);
    }
  }
  if (tile < 0) return;
  const Seq seq = load_seq<false>(a, s);
  run_piece<D, BM, false>(a, seq, blockIdx.y, tile, 0, key_blocks<false, BN>(a, seq, (tile + 1) * BM), true, 0, (float *)sm4);
}

template <typename F>
pcomoe_status launch(F *kernel, PerDeviceOnce &once, dim3 grid, size_t smem, const AttnArgs &a, cudaStream_t st) {
  int dev = -1;
  PCOMOE_CUDA_TRY(cudaGetDevice(&dev));
  if (once.first_use(dev)) {
    PCOMOE_CUDA_TRY(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem));
    once.done(dev);
  }
  PCOMOE_CUDA_TRY(launch_pdl(kernel, grid, dim3(kThreads), smem, st, a));
  count_launch();
  return PCOMOE_OK;
}

template <int D>
pcomoe_status run_cached(const AttnArgs &a, int sms, cudaStream_t st) {
  static PerDeviceOnce once;
  const pcomoe_status r = launch(simt_cached_kernel<D>, once, dim3(2 * sms), smem_floats<D, 64>() * sizeof(float), a, st);
  return r == PCOMOE_OK ? launch_attn_join(a, D, PCOMOE_FP32, 64, 2 * sms, st) : r;
}

template <int D, int BM>
pcomoe_status run_prompt(const AttnArgs &a, cudaStream_t st) {
  static PerDeviceOnce once;
  const int64_t tiles = (int64_t)a.T * a.g / BM + std::min(a.n_seqs, a.T);
  if (tiles > INT32_MAX) return PCOMOE_ERR_SHAPE;
  return launch(simt_prompt_kernel<D, BM>, once, dim3((unsigned)tiles, a.hkv), smem_floats<D, BM>() * sizeof(float), a, st);
}

}  // namespace

size_t attn_simt_part_rows(int sms) { return (size_t)4 * sms * 64; }

pcomoe_status launch_attn_simt(const AttnArgs &a, int D, int sms, cudaStream_t st) {
  if (a.table) return D == 64 ? run_cached<64>(a, sms, st) : run_cached<128>(a, sms, st);
  // Prompts: tiles of 16 rows where each of them gets an SM of its own (head size 128, 8 heads on 2: 4 prompts of 64 tokens
  // 10.5 us, with 64 rows 12.3 us), else of 64 (4 prompts of 256: 52 us, with 16 rows 68 us).
  if (((int64_t)a.T * a.g / 16 + std::min(a.n_seqs, a.T)) * a.hkv <= sms) return D == 64 ? run_prompt<64, 16>(a, st) : run_prompt<128, 16>(a, st);
  return D == 64 ? run_prompt<64, 64>(a, st) : run_prompt<128, 64>(a, st);
}

}  // namespace pcomoe
