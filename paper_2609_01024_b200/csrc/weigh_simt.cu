// Weights of cached positions from many counted rows, fp32.
//
// Mathematics as in the kernel of few rows.  A unit of work is 64 keys of one kv head, whose rows lie in shared memory while tiles of 64
// columns (a counted row and a query head each) pass by, the next one on its way while one is worked on.  16 x 16 threads have 4 keys and 4
// columns each, 16 sums of products in registers; a key's sum over all columns stays in the 16 threads that have it.  Rows are held 16
// bytes further apart than they are long, so that the threads that read different rows read from different banks.
// What bounds it: reads of shared memory and the FMA pipe, 2 D operations for each key, column and head.  Measured, 32 heads on 8 of 128, 400
// counted rows of each of 8 sequences of 4496: 2.99 ms, 38 TFLOP/s (elements one by one instead of in pairs 3.06; 8 x 8 pairs for four lanes
// that have a quarter of the elements each, with half as many reads, 3.34).
#include <algorithm>

#include "weigh_parts.cuh"

namespace pcomoe {
namespace {

constexpr int kTile = 64, kThreads = 256;
template <int D> struct Tiles {
  static constexpr int kRow = D + 4;                      // floats
  static constexpr int kSmem = 3 * kTile * kRow * 4;      // keys, two tiles of queries
};

__device__ __forceinline__ void copy16(uint32_t dst, const float *src, bool there) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(there ? 16 : 0) : "memory");
}

__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
  uint64_t d;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(*(uint64_t *)&a), "l"(*(uint64_t *)&b), "l"(*(uint64_t *)&c));
  return *(float2 *)&d;
}

template <int D>
__global__ void __launch_bounds__(kThreads, 2) weigh_simt_kernel(const __grid_constant__ PartArgs a) {
  constexpr int kRow = Tiles<D>::kRow, kPer = D / 16;     // 16-byte pieces of a row that a thread copies: 4 threads a row
  extern __shared__ __align__(16) float s_tiles[];
  __shared__ __align__(16) float s_lse[2][kTile];
  __shared__ __align__(16) int s_lim[2][kTile];
  __shared__ uint32_t s_bits[2 * (kMaxSeqs / 32)];
  pdl_grid_wait();
  const uint32_t *twice = find_repeats(a.w.seqs, a.w.n, a.w.max_seqs, s_bits);
  const int tid = threadIdx.x, tx = tid & 15, ty = tid >> 4, r = tid >> 2, part = tid & 3;
  const uint32_t to = (uint32_t)__cvta_generic_to_shared(s_tiles) + (r * kRow + part * 4) * 4;       // this thread's first piece of a tile
  const float *keys = s_tiles + ty * kRow;
  Line<kTile, kTile> line = {0, 0, {}, 0, false};
  for (uint32_t round = 0;; ++round) {
    Unit it;
    line.get(a, twice, (int64_t)round * gridDim.x + (round & 1 ? gridDim.x - 1 - blockIdx.x : blockIdx.x), it);
    if (it.p0 < 0) break;
    const int64_t cols = (int64_t)it.seq.m * a.w.g;
    // A tile's queries are sent for; the log sum of the thread's column comes into a register, to be put down when the tile before is done with.
    float lse = 0.f;
    int lim = -1;
    auto send = [&](int i) {
      const int64_t col = (int64_t)(it.first + i * a.parts) * kTile + r;
      const float *from = (const float *)a.w.q;
      lse = 0.f;
      lim = -1;
      bool there = false;
      if (col < cols) {
        const int k = (int)col / a.w.g, head = it.head * a.w.g + (int)col - k * a.w.g, row = counted_row(a.w, it.seq, it.list, k);
        if (row >= 0) {
          there = true;
          from += row * a.w.q_stride + (int64_t)head * D;
          lse = a.w.lse[(int64_t)row * a.w.hq + head];
          lim = it.seq.base + k;
        }
      }
#pragma unroll
      for (int c = 0; c < kPer; ++c) copy16(to + (1 + (i & 1)) * kTile * kRow * 4 + c * 64, from + (there ? c * 16 + part * 4 : 0), there);
      asm volatile("cp.async.commit_group;" ::: "memory");
    };
    auto put = [&](int i) {
      if (part == 0) {
        s_lse[i & 1][r] = lse * kLog2ef;
        s_lim[i & 1][r] = lse != -INFINITY ? lim : -1;     // a row that saw nothing adds nothing
      }
    };
    float sum[4] = {0.f, 0.f, 0.f, 0.f};
    if (it.steps) {
      const int p = it.p0 + r;
      const bool there = p < it.seq.len;
      const float *from = (const float *)a.w.k;
      if (there) from += (weigh_page_row(a.w, a.w.table + (int64_t)it.seq.id * a.w.max_pages, p) + (int64_t)it.head * a.w.page) * D + part * 4;
#pragma unroll
      for (int c = 0; c < kPer; ++c) copy16(to + c * 64, from + (there ? c * 16 : 0), there);
      send(0);
      put(0);
    }
    for (int i = 0; i < it.steps; ++i) {
      if (i + 1 < it.steps) {
        send(i + 1);
        asm volatile("cp.async.wait_group 1;" ::: "memory");
      } else {
        asm volatile("cp.async.wait_group 0;" ::: "memory");
      }
      __syncthreads();
      const float *q = s_tiles + (1 + (i & 1)) * kTile * kRow + tx * kRow;
      float2 c[4][4];                                      // of even and of odd elements
#pragma unroll
      for (int y = 0; y < 4; ++y)
#pragma unroll
        for (int x = 0; x < 4; ++x) c[y][x] = make_float2(0.f, 0.f);
#pragma unroll 8
      for (int d = 0; d < D; d += 4) {
        float4 kk[4], qq[4];
#pragma unroll
        for (int y = 0; y < 4; ++y) kk[y] = *(const float4 *)(keys + 16 * y * kRow + d);
#pragma unroll
        for (int x = 0; x < 4; ++x) qq[x] = *(const float4 *)(q + 16 * x * kRow + d);
#pragma unroll
        for (int y = 0; y < 4; ++y)
#pragma unroll
          for (int x = 0; x < 4; ++x) {
            c[y][x] = fma2(make_float2(kk[y].x, kk[y].y), make_float2(qq[x].x, qq[x].y), c[y][x]);
            c[y][x] = fma2(make_float2(kk[y].z, kk[y].w), make_float2(qq[x].z, qq[x].w), c[y][x]);
          }
      }
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        const float l = s_lse[i & 1][tx + 16 * x];
        const int m = s_lim[i & 1][tx + 16 * x];
        // chosen, not multiplied: what is not seen adds nothing whatever it is
#pragma unroll
        for (int y = 0; y < 4; ++y) sum[y] += it.p0 + ty + 16 * y <= m ? exp2_fast(fmaf(c[y][x].x + c[y][x].y, a.w.scale_log2, -l)) : 0.f;
      }
      if (i + 1 < it.steps) put(i + 1);
      __syncthreads();                                     // the tile is read before the one after the next takes its place
    }
#pragma unroll
    for (int y = 0; y < 4; ++y) {
#pragma unroll
      for (int o = 8; o; o >>= 1) sum[y] += __shfl_xor_sync(~0u, sum[y], o);
      const int p = it.p0 + ty + 16 * y;
      if (tx == 0 && p < it.seq.len) a.partial[((int64_t)it.list * (a.w.hkv * a.parts) + it.part * a.w.hkv + it.head) * a.room + p] = sum[y];
    }
  }
}

template <int D>
pcomoe_status run(const PartArgs &a, int sms, cudaStream_t st) {
  static PerDeviceOnce once;
  int dev = -1;
  PCOMOE_CUDA_TRY(cudaGetDevice(&dev));
  if (once.first_use(dev)) {
    PCOMOE_CUDA_TRY(cudaFuncSetAttribute(weigh_simt_kernel<D>, cudaFuncAttributeMaxDynamicSharedMemorySize, Tiles<D>::kSmem));
    once.done(dev);
  }
  PCOMOE_CUDA_TRY(launch_pdl(weigh_simt_kernel<D>, dim3(2 * sms), dim3(kThreads), Tiles<D>::kSmem, st, a));
  count_launch();
  return launch_join(a, sms, st);
}

}  // namespace

pcomoe_status launch_weigh_simt(const WeighArgs &w, int D, float *partial, int64_t room, int sms, cudaStream_t st) {
  PartArgs a = {};
  a.w = w;
  a.partial = partial;
  a.room = room;
  a.parts = parts_of(w.hkv);
  return D == 64 ? run<64>(a, sms, st) : run<128>(a, sms, st);
}

}  // namespace pcomoe
