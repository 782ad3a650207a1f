// What the kernels of many counted rows share: units of keys and columns in one line, and their partial sums.
#pragma once
#include <algorithm>

#include "weigh.cuh"

namespace pcomoe {
namespace {

struct Unit {
  WeighSeq seq;
  int list, head, part;
  int p0;               // first key; -1: no more work
  int first, steps;     // column tile of the first step, and their number; tiles are `parts` apart
};

struct PartArgs {
  WeighArgs w;
  float *partial;       // [n][hkv * parts][room]
  int64_t room;
  int32_t parts;
};

// The units of a call, KEYS keys of one head and tiles of COLS columns, in one line: sequence, keys, part and head, the last fastest.  A warp.
template <int KEYS, int COLS>
struct Line {
  int s0;               // sequences s0 + lane are in hand
  int64_t before;       // units before them
  WeighSeq mine;
  int64_t upto;
  bool held;

  __device__ __forceinline__ void hold(const PartArgs &a, const uint32_t *twice) {
    const int lane = threadIdx.x & 31;
    mine = {};
    if (s0 + lane < a.w.n) mine = weigh_seq(a.w, s0 + lane, twice);
    upto = (int64_t)((mine.len + KEYS - 1) / KEYS) * (a.w.hkv * a.parts);
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int64_t y = __shfl_up_sync(~0u, upto, o);
      if (lane >= o) upto += y;
    }
    held = true;
  }
  // unit u, no smaller than any asked for before
  __device__ __forceinline__ void get(const PartArgs &a, const uint32_t *twice, int64_t u, Unit &it) {
    it.p0 = -1;
    while (s0 < a.w.n) {
      if (!held) hold(a, twice);
      const uint32_t hit = __ballot_sync(~0u, before + upto > u);
      if (hit) {
        const int l = __ffs(hit) - 1;
        const int64_t upto_l = __shfl_sync(~0u, upto, l);
        const int lanes_len = __shfl_sync(~0u, mine.len, l), P = a.w.hkv * a.parts;
        const int64_t count = (int64_t)((lanes_len + KEYS - 1) / KEYS) * P, at = u - (before + upto_l - count);
        it.seq.q0 = __shfl_sync(~0u, mine.q0, l);
        it.seq.n = __shfl_sync(~0u, mine.n, l);
        it.seq.m = __shfl_sync(~0u, mine.m, l);
        it.seq.len = lanes_len;
        it.seq.base = it.seq.len - it.seq.m;
        it.seq.id = __shfl_sync(~0u, mine.id, l);
        it.list = s0 + l;
        const int r = (int)(at % P);
        it.head = r % a.w.hkv;
        it.part = r / a.w.hkv;
        it.p0 = (int)(at / P) * KEYS;
        const int64_t cols = (int64_t)it.seq.m * a.w.g, from = (int64_t)max(0, it.p0 - it.seq.base) * a.w.g;
        const int tiles = (int)((cols + COLS - 1) / COLS);
        it.first = (int)(from / COLS) + it.part;
        it.steps = max(0, (tiles - it.first + a.parts - 1) / a.parts);
        return;
      }
      before += __shfl_sync(~0u, upto, 31);
      s0 += 32;
      held = false;
    }
  }
};

// Partial sums added in order.  blockIdx.y: sequences, a grid's height apart.
__global__ void __launch_bounds__(256) weigh_join_kernel(const __grid_constant__ PartArgs a) {
  __shared__ uint32_t s_bits[2 * (kMaxSeqs / 32)];
  pdl_grid_wait();
  const uint32_t *twice = find_repeats(a.w.seqs, a.w.n, a.w.max_seqs, s_bits);
  const int P = a.w.hkv * a.parts;
  for (int i = blockIdx.y; i < a.w.n; i += gridDim.y) {
    const WeighSeq s = weigh_seq(a.w, i, twice);
    float *w = a.w.weight + s.id * a.w.weight_stride;
    const float *part = a.partial + (int64_t)i * P * a.room;
    for (int p = blockIdx.x * 256 + threadIdx.x; p < s.len; p += gridDim.x * 256) {
      float sum = 0.f;
#pragma unroll 8
      for (int r = 0; r < P; ++r) sum += part[r * a.room + p];
      w[p] = a.w.fresh && p >= s.base ? sum : w[p] + sum;
    }
  }
}

inline pcomoe_status launch_join(const PartArgs &a, int sms, cudaStream_t st) {
  // a position per thread, while that makes no more than 16 blocks for every SM
  const unsigned wide = (unsigned)std::min<int64_t>((a.room + 255) / 256, std::max(1, 16 * sms / a.w.n));
  PCOMOE_CUDA_TRY(launch_pdl(weigh_join_kernel, dim3(wide, (unsigned)std::min(a.w.n, 65535)), dim3(256), 0, st, a));
  count_launch();
  return PCOMOE_OK;
}

// Shares of a head's columns: enough units where there are few heads.
inline int parts_of(int hkv) { return hkv >= 8 ? 1 : 8 / hkv; }

}  // namespace
}  // namespace pcomoe
