// Weights of cached positions from many counted rows, bf16, on the tensor cores (tcgen05).
//
// Mathematics as in the kernel of few rows: w_p += sum over columns 2^(c q.k_p - c' lse); a column is a counted row and a query head.
// A unit of work is 128 keys of one kv head: S^T = K Q^T with the keys as the accumulator's rows, so a position is a TMEM lane and one
// thread's, its sum over the columns never leaves that thread, and the log sums are the same for all lanes (shared memory, one
// broadcast load for four columns).  There is no second product and nothing is written back.
//   warp 0: MMAs (128 keys x 128 columns a step), owner of TMEM     warps 1, 2: queries and log sums of the steps
//   warp 3: finds the CTA's units                                   warps 4-15: exponentials and sums, three groups in turn
// The keys are the MMA's first operand and lie in TMEM (two elements a column, written there by the threads that own their rows), so
// that shared memory feeds only the queries to the tensor cores.  With both operands in shared memory a step moved 64 KB out of it
// and 32 KB into it, at its limit.  Two units' keys and three accumulators of 128 columns fill TMEM; the queries come through six
// stages of 32 KB, as one box per 64 columns of the head where all packed rows are counted and a tile holds whole rows, else by
// 16-byte copies (counted rows may be any of the packed ones, and a group of heads need not divide a tile).
// Units leave partial sums, one for each head (or each share of a head's columns, where there are fewer than 8 heads), which a
// second launch adds in order: no atomics, and the bits do not depend on which CTA took which unit.  CTAs take units from both
// ends of rounds of the grid's size in turn, so that in a prompt, whose later keys are seen by fewer rows, all get about the same
// work.  (Drawn from a counter as they were finished the units took as long.)
//
// What bounds it: for the most part the special function unit, 16 exponentials per clock and SM (1024 clocks a step, in which the tensor cores work
// 512), and in long runs the power limit.  Measured: a prompt of 8192 tokens, 32 heads on 8 of 128, 0.36 ms in runs of a few
// milliseconds and 0.39 ms in long ones (1.72 GHz at 980 W), 275 GFLOP and 1.07e9 exponentials.  The fullest CTA has 476 steps there (450 on
// average), so a step takes 1400 to 1500 clocks: some 400 are not the exponentials' and were not taken apart.  Two groups instead of three took 6 %
// longer; a polynomial on the FMA pipe for a quarter of the exponentials 0.35 ms in short runs and no less in long ones.
#include <algorithm>
#include <type_traits>

#include "tc_ptx.cuh"
#include "weigh_parts.cuh"

namespace pcomoe {
namespace {

constexpr int BK_ROWS = 128, BC = 128;          // keys of a unit, columns of a step
constexpr int kGroups = 3, kFirst = 128, kThreads = kFirst + 128 * kGroups;      // warp groups that sum, from thread kFirst on
constexpr int kStages = 6, kBuffers = 3, kSlots = 8;       // of queries, of accumulators, of log sums
constexpr int kUnits = 4;                       // units in hand
constexpr uint32_t kKeyCols = 64, kAccAt = 2 * kKeyCols;    // TMEM columns: keys of two units, then the accumulators
template <int D> struct Shape {
  static constexpr int kHalves = D / 64;
  static constexpr int kHalfBytes = 128 * 128;
  static constexpr int kTileBytes = kHalves * kHalfBytes;
  static constexpr int kSmem = kStages * kTileBytes;
};

__device__ __forceinline__ bool elect_lane() {
  uint32_t e;
  asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(e));
  return e;
}
// D (+)= A B, A from TMEM
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, uint32_t acc) {
  asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d), "r"(a),
               "l"(b), "r"(idesc), "r"(acc)
               : "memory");
}
// 16 columns of this thread's TMEM lane
__device__ __forceinline__ void tmem_st16(uint32_t taddr, const uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15};" ::"r"(r[0]),
      "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]),
      "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(taddr)
      : "memory");
}
__device__ __forceinline__ void copy16(uint32_t dst, const void *src, bool there) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(there ? 16 : 0) : "memory");
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

__device__ __forceinline__ void tma_load_3d(uint32_t dst, const CUtensorMap *map, int32_t x, int32_t y, int32_t z, uint32_t bar) {
  asm volatile("cp.async.bulk.tensor.3d.shared::cta.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(dst), "l"(map),
               "r"(x), "r"(y), "r"(z), "r"(bar)
               : "memory");
}

// kBoxes: all packed rows are counted and a tile holds whole rows, so a tile of queries is one box per 64 columns of the head.
template <int D, bool kBoxes>
__global__ void __launch_bounds__(kThreads, 1) weigh_tc_kernel(const __grid_constant__ CUtensorMap q_map, const __grid_constant__ PartArgs a) {
  using S = Shape<D>;
  constexpr uint32_t kIdesc = (1u << 4) | (1u << 7) | (1u << 10) | ((128u >> 3) << 17) | ((128u >> 4) << 24);
  constexpr int C = D / 8, kSide = 32 / C;                // 16-byte pieces of a row; rows that a warp copies side by side
  extern __shared__ __align__(1024) uint8_t smem[];
  __shared__ __align__(8) uint64_t s_qfull[kStages], s_qempty[kStages], s_kfull[2], s_kempty[2], s_sfull[kBuffers], s_sempty[kBuffers], s_lfull[kSlots], s_lempty[kSlots], s_ifull[kUnits],
      s_iempty[kUnits], s_join[kUnits];
  __shared__ Unit s_item[kUnits];
  __shared__ __align__(16) float s_lse[kSlots][BC];
  __shared__ __align__(16) int s_lim[kSlots][BC];
  __shared__ int s_least[kSlots][2];                      // the smallest limit of either half of a step's columns
  __shared__ int64_t s_at[2][64];                         // of the copying warps: where rows are, -1: nowhere
  __shared__ float s_sum[kUnits][kGroups - 1][BK_ROWS];
  __shared__ uint32_t s_bits[2 * (kMaxSeqs / 32)];
  __shared__ uint32_t s_tmem;
  __shared__ int s_flags[2];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const uint32_t q_at = smem_u32(smem);
  volatile int *flags = s_flags;

  if (tid == 0) {
    s_flags[0] = q_at & 1023 ? 1 : 0;                     // the swizzle needs it
    s_flags[1] = 0;
    for (int i = 0; i < kStages; ++i) { mbar_init(smem_u32(&s_qfull[i]), kBoxes ? 1 : 2); mbar_init(smem_u32(&s_qempty[i]), 1); }
    for (int i = 0; i < kBuffers; ++i) { mbar_init(smem_u32(&s_sfull[i]), 1); mbar_init(smem_u32(&s_sempty[i]), 4); }
    for (int i = 0; i < kSlots; ++i) { mbar_init(smem_u32(&s_lfull[i]), kBoxes ? 1 : 2); mbar_init(smem_u32(&s_lempty[i]), 4); }
    for (int i = 0; i < 2; ++i) { mbar_init(smem_u32(&s_kfull[i]), 4); mbar_init(smem_u32(&s_kempty[i]), 1); }
    for (int i = 0; i < kUnits; ++i) {
      mbar_init(smem_u32(&s_ifull[i]), 1);
      mbar_init(smem_u32(&s_iempty[i]), 3 + 4 * kGroups);  // every warp but the one that fills them
      mbar_init(smem_u32(&s_join[i]), 4 * (kGroups - 1));
    }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 0) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&s_tmem)), "r"(512) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = s_tmem;
  pdl_grid_wait();
  const uint32_t *twice = find_repeats(a.w.seqs, a.w.n, a.w.max_seqs, s_bits);

  uint32_t n_item = 0, step = 0;                          // units and steps so far
  auto item_ready = [&](bool ok) { return __all_sync(~0u, ok && wait_bar(&s_ifull[n_item % kUnits], (n_item / kUnits) & 1, flags, a.w.limit_ns)); };
  auto item_done = [&]() {
    __syncwarp();
    if (lane == 0) mbar_arrive(smem_u32(&s_iempty[n_item % kUnits]));
    ++n_item;
  };
  if (warp >= kFirst / 32) {
    const int group = (warp - kFirst / 32) >> 2, key = (warp & 3) * 32 + lane;
    const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
    const float scale = a.w.scale_log2;
    bool ok = true;
    uint32_t n_unit = 0, n_k = 0;
    // The groups in turn bring a unit's keys into TMEM: a thread its own row, straight from its page, two elements to a column.  Unit
    // number n's are brought while the one before it is worked on; n_k units with steps came before it.
    auto load_keys = [&](uint32_t n) {
      if (ok) ok = wait_bar(&s_ifull[n % kUnits], (n / kUnits) & 1, flags, a.w.limit_ns);
      __syncwarp();
      const Unit &it = s_item[n % kUnits];
      if (!__all_sync(~0u, ok) || it.p0 < 0 || it.steps == 0) return;
      if ((int)(n_k % kGroups) != group) {
        ++n_k;
        return;
      }
      const int p = it.p0 + key;
      const uint4 *row = nullptr;
      if (p < it.seq.len)
        row = (const uint4 *)((const __nv_bfloat16 *)a.w.k + (weigh_page_row(a.w, a.w.table + (int64_t)it.seq.id * a.w.max_pages, p) + (int64_t)it.head * a.w.page) * D);
      // (all of the row is asked for before any of it is used)
      uint32_t x[D / 32][16];
#pragma unroll
      for (int c = 0; c < D / 32; ++c)
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const uint4 y = row ? row[4 * c + k] : make_uint4(0, 0, 0, 0);
          x[c][4 * k] = y.x; x[c][4 * k + 1] = y.y; x[c][4 * k + 2] = y.z; x[c][4 * k + 3] = y.w;
        }
      ok = wait_bar(&s_kempty[n_k & 1], ((n_k >> 1) & 1) ^ 1, flags, a.w.limit_ns);
      __syncwarp();
      tc_fence_after();
#pragma unroll
      for (int c = 0; c < D / 32; ++c) {
        __syncwarp();
        tmem_st16(tmem + (n_k & 1) * kKeyCols + 16 * c + lanes, x[c]);
      }
      asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(smem_u32(&s_kfull[n_k & 1]));
      ++n_k;
    };
    load_keys(0);
    while (item_ready(ok)) {
      const Unit &it = s_item[n_item % kUnits];
      if (it.p0 < 0) break;
      // (before the group's own steps: those wait for this unit's products, and the next unit's keys would wait behind them)
      load_keys(n_item + 1);
      const int p = it.p0 + key, last = it.p0 + BK_ROWS - 1, steps = it.steps, len = it.seq.len;
      float total = 0.f;
      for (int i = 0; i < steps; ++i) {
        const uint32_t at = step + i, b = at % kBuffers, slot = at % kSlots;
        if ((int)(at % kGroups) != group) continue;
        if (ok) ok = wait_bar(&s_sfull[b], (at / kBuffers) & 1, flags, a.w.limit_ns) && wait_bar(&s_lfull[slot], (at / kSlots) & 1, flags, a.w.limit_ns);
        __syncwarp();
        tc_fence_after();
        float2 sum[4] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f), make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
        const float2 scale2 = make_float2(scale, scale);
        // 32 columns in hand, the next 32 on their way.  (Two loops, so that the one without a mask is one stretch of code: with the
        // question inside of it a step took twice as long.)
        const auto sums = [&](auto masked) {
          uint32_t x[2][32];
          tmem_ld32_issue(tmem + kAccAt + b * BC + lanes, x[0]);
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            tmem_wait_ld();
            reg_fence32(x[c & 1]);
            if (c < 3) {
              tmem_ld32_issue(tmem + kAccAt + b * BC + 32 * (c + 1) + lanes, x[(c + 1) & 1]);
            } else {
              tc_fence_before();
              __syncwarp();
              if (lane == 0) mbar_arrive(smem_u32(&s_sempty[b]));
            }
#pragma unroll
            for (int k = 0; k < 32; k += 4) {
              const float4 l = *(const float4 *)&s_lse[slot][32 * c + k];        // minus the log sum
              float2 e = fma2(make_float2(__uint_as_float(x[c & 1][k]), __uint_as_float(x[c & 1][k + 1])), scale2, make_float2(l.x, l.y));
              float2 f = fma2(make_float2(__uint_as_float(x[c & 1][k + 2]), __uint_as_float(x[c & 1][k + 3])), scale2, make_float2(l.z, l.w));
              e = make_float2(exp2_fast(e.x), exp2_fast(e.y));
              f = make_float2(exp2_fast(f.x), exp2_fast(f.y));
              if (masked.value) {                          // chosen, not multiplied
                const int4 m = *(const int4 *)&s_lim[slot][32 * c + k];
                e = make_float2(p <= m.x ? e.x : 0.f, p <= m.y ? e.y : 0.f);
                f = make_float2(p <= m.z ? f.x : 0.f, p <= m.w ? f.y : 0.f);
              }
              sum[(k >> 2) & 1] = add2(sum[(k >> 2) & 1], e);
              sum[2 + ((k >> 2) & 1)] = add2(sum[2 + ((k >> 2) & 1)], f);
            }
          }
        };
        if (last > min(s_least[slot][0], s_least[slot][1])) sums(std::true_type());
        else sums(std::false_type());
        const float2 s = add2(add2(sum[0], sum[1]), add2(sum[2], sum[3]));
        total += s.x + s.y;
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&s_lempty[slot]));
      }
      step += steps;
      // the other groups hand their sums to the first.  (They get to the unit that takes the same place and barrier only when all are
      // done with this one.)
      if (group) {
        s_sum[n_unit % kUnits][group - 1][key] = total;
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&s_join[n_unit % kUnits]));
      } else {
        if (ok) ok = wait_bar(&s_join[n_unit % kUnits], (n_unit / kUnits) & 1, flags, a.w.limit_ns);
        __syncwarp();
#pragma unroll
        for (int g = 1; g < kGroups; ++g) total += s_sum[n_unit % kUnits][g - 1][key];
        if (p < len) a.partial[((int64_t)it.list * (a.w.hkv * a.parts) + it.part * a.w.hkv + it.head) * a.room + p] = total;
      }
      ++n_unit;
      item_done();
    }
  } else if (warp == 1 || warp == 2) {
    // ---- the columns of the steps and their log sums.  Where rows are copied one by one each of the two warps takes 64 columns, and up to
    // two copies are under way before the oldest is waited for and handed on.
    const int half = warp - 1;
    uint64_t *wait0[2] = {nullptr, nullptr}, *wait1[2] = {nullptr, nullptr};       // barriers of the copies under way, oldest last
    bool ok = true;
    auto hand_on = [&](int i) {
      if (!wait0[i]) return;
      if (lane == 0) {
        mbar_arrive(smem_u32(wait0[i]));
        if (wait1[i]) mbar_arrive(smem_u32(wait1[i]));
      }
      wait0[i] = nullptr;
    };
    auto flush = [&]() {
      if (!wait0[0] && !wait0[1]) return;
      asm volatile("cp.async.wait_all;" ::: "memory");
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
      __syncwarp();
      hand_on(1);
      hand_on(0);
    };
    auto begun = [&](uint64_t *b0, uint64_t *b1) {
      asm volatile("cp.async.commit_group;" ::: "memory");
      if (wait0[1]) {
        asm volatile("cp.async.wait_group 2;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncwarp();
        hand_on(1);
      }
      wait0[1] = wait0[0]; wait1[1] = wait1[0];
      wait0[0] = b0; wait1[0] = b1;
    };
    auto wait = [&](uint64_t *bar, uint32_t parity) {
      if (!__all_sync(~0u, probe_bar(smem_u32(bar), parity))) {
        flush();                                           // nobody waits for a copy that waits for this
        ok = __all_sync(~0u, ok && wait_bar(bar, parity, flags, a.w.limit_ns));
      }
      return ok;
    };
    // 64 rows whose places are in s_at, to rows half * 64 .. of the tile at `to`
    auto copy_rows = [&](const void *base, uint32_t to) {
      const int c = lane % C;
      const uint32_t dst = to + (c >> 3) * S::kHalfBytes;
#pragma unroll 8
      for (int r0 = 0; r0 < 64; r0 += kSide) {
        const int r = r0 + lane / C, row = half * 64 + r;
        const int64_t at = s_at[half][r];
        copy16(dst + row * 128 + (((c & 7) ^ (row & 7)) << 4), (const __nv_bfloat16 *)base + (at < 0 ? 0 : at) + c * 8, at >= 0);
      }
    };
    // The next unit comes when the groups are done with one before it, which may wait for a copy that is not handed on yet (units
    // without steps lie between).
    auto next_item = [&]() {
      if (!__all_sync(~0u, probe_bar(smem_u32(&s_ifull[n_item % kUnits]), (n_item / kUnits) & 1))) flush();
      return item_ready(ok);
    };
    for (; next_item(); item_done()) {
      const Unit it = s_item[n_item % kUnits];
      if (it.p0 < 0) break;
      if (it.steps == 0) continue;
      if (kBoxes) {
        // the first warp sends for the queries; the second has the log sums on their way kAhead steps before they are used
        constexpr int kAhead = 3;
        const int cols = it.seq.m * a.w.g, gs = __ffs(a.w.g) - 1;          // a tile holds whole rows: g is a power of 2
        float ahead[kAhead][4];
        auto fetch = [&](int i, float (&to)[4]) {
          const int c0 = (it.first + i * a.parts) * BC + 4 * lane;
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const int col = c0 + j, k = col >> gs;
            to[j] = i < it.steps && col < cols ? a.w.lse[(int64_t)(it.seq.q0 + k) * a.w.hq + (it.head << gs) + col - (k << gs)] : -INFINITY;
          }
        };
        if (half)
#pragma unroll
          for (int k = 0; k < kAhead; ++k) fetch(k, ahead[k]);
        for (int i = 0; i < it.steps; ++i, ++step) {
          const uint32_t st = step % kStages, slot = step % kSlots;
          const int c0 = (it.first + i * a.parts) * BC;
          if (!half) {
            if (!wait(&s_qempty[st], ((step / kStages) & 1) ^ 1)) break;
            if (lane == 0) {
              mbar_arrive_expect_tx(smem_u32(&s_qfull[st]), S::kTileBytes);
#pragma unroll
              for (int h = 0; h < S::kHalves; ++h)
                tma_load_3d(q_at + st * S::kTileBytes + h * S::kHalfBytes, &q_map, h * 64, it.head << gs, it.seq.q0 + (c0 >> gs), smem_u32(&s_qfull[st]));
            }
            __syncwarp();
          } else {
            if (!wait(&s_lempty[slot], ((step / kSlots) & 1) ^ 1)) break;
            float lse[4];
            int lim[4], least = INT32_MAX;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              lse[j] = ahead[0][j];
#pragma unroll
              for (int k = 0; k + 1 < kAhead; ++k) ahead[k][j] = ahead[k + 1][j];
            }
            fetch(i + kAhead, ahead[kAhead - 1]);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              lim[j] = lse[j] != -INFINITY ? it.seq.base + ((c0 + 4 * lane + j) >> gs) : -1;
              least = min(least, lim[j]);
              lse[j] = lim[j] >= 0 ? -lse[j] * kLog2ef : 0.f;
            }
            *(float4 *)&s_lse[slot][4 * lane] = make_float4(lse[0], lse[1], lse[2], lse[3]);
            *(int4 *)&s_lim[slot][4 * lane] = make_int4(lim[0], lim[1], lim[2], lim[3]);
            least = __reduce_min_sync(~0u, least);
            if (lane < 2) s_least[slot][lane] = least;
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&s_lfull[slot]));
          }
        }
      } else
      for (int i = 0; i < it.steps; ++i, ++step) {
        const uint32_t st = step % kStages, slot = step % kSlots;
        if (!wait(&s_qempty[st], ((step / kStages) & 1) ^ 1) || !wait(&s_lempty[slot], ((step / kSlots) & 1) ^ 1)) break;
        const int64_t c0 = (int64_t)(it.first + i * a.parts) * BC + half * 64, cols = (int64_t)it.seq.m * a.w.g;
        int least = INT32_MAX;
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const int r = 32 * j + lane;
          const int64_t col = c0 + r;
          int64_t at = -1;
          float lse = 0.f;
          int lim = -1;
          if (col < cols) {
            const int k = (int)col / a.w.g, head = it.head * a.w.g + (int)col - k * a.w.g, row = counted_row(a.w, it.seq, it.list, k);
            if (row >= 0) {
              at = row * a.w.q_stride + (int64_t)head * D;
              lse = a.w.lse[(int64_t)row * a.w.hq + head];
              if (lse != -INFINITY) lim = it.seq.base + k;
            }
          }
          s_at[half][r] = at;
          s_lse[slot][half * 64 + r] = lim >= 0 ? -lse * kLog2ef : 0.f;
          s_lim[slot][half * 64 + r] = lim;
          least = min(least, lim);
        }
        least = __reduce_min_sync(~0u, least);
        if (lane == 0) s_least[slot][half] = least;
        __syncwarp();
        copy_rows(a.w.q, q_at + st * S::kTileBytes);
        __syncwarp();
        begun(&s_qfull[st], &s_lfull[slot]);
      }
      if (!ok) break;
    }
    flush();
    asm volatile("cp.async.wait_all;" ::: "memory");
  } else if (warp == 0) {
    // ---- MMAs; the whole warp walks along, one lane issues
    bool ok = true;
    uint32_t n_k = 0;
    auto wait = [&](uint64_t *bar, uint32_t p) { return ok = __all_sync(~0u, wait_bar(bar, p, flags, a.w.limit_ns)); };
    const uint64_t q_desc = umma_desc(q_at);
    for (; item_ready(ok); item_done()) {
      const int p0 = s_item[n_item % kUnits].p0, steps = s_item[n_item % kUnits].steps;
      if (p0 < 0) break;
      if (steps == 0) continue;
      if (!wait(&s_kfull[n_k & 1], (n_k >> 1) & 1)) break;
      const uint32_t keys = tmem + (n_k & 1) * kKeyCols;
      for (int i = 0; i < steps; ++i, ++step) {
        const uint32_t st = step % kStages, b = step % kBuffers;
        if (!wait(&s_sempty[b], ((step / kBuffers) & 1) ^ 1)) break;
        if (!wait(&s_qfull[st], (step / kStages) & 1)) break;
        tc_fence_after();
        const uint64_t db = q_desc + (uint64_t)(st * (S::kTileBytes >> 4));
        if (elect_lane()) {
#pragma unroll
          for (int k = 0; k < D / 16; ++k) {
            const uint64_t off = (uint64_t)((k >> 2) * (S::kHalfBytes >> 4) + (k & 3) * 2);
            mma_ts(tmem + kAccAt + b * BC, keys + k * 8, db + off, kIdesc, k != 0);
          }
          umma_commit(smem_u32(&s_sfull[b]));
          umma_commit(smem_u32(&s_qempty[st]));
          if (i == steps - 1) umma_commit(smem_u32(&s_kempty[n_k & 1]));
        }
        __syncwarp();
      }
      if (!ok) break;
      ++n_k;
    }
  } else {
    // ---- the units: from both ends of rounds of the grid's size in turn
    Line<BK_ROWS, BC> line = {0, 0, {}, 0, false};
    for (uint32_t r = 0;; ++r, ++n_item) {
      Unit it = {};
      line.get(a, twice, (int64_t)r * gridDim.x + (r & 1 ? gridDim.x - 1 - blockIdx.x : blockIdx.x), it);
      if (!__all_sync(~0u, wait_bar(&s_iempty[n_item % kUnits], ((n_item / kUnits) & 1) ^ 1, flags, a.w.limit_ns))) break;
      if (lane == 0) {
        s_item[n_item % kUnits] = it;
        mbar_arrive(smem_u32(&s_ifull[n_item % kUnits]));
      }
      __syncwarp();
      if (it.p0 < 0) break;
    }
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (s_flags[0]) timeout_record_and_drain(a.w.status);
  __syncthreads();
  if (warp == 0) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512) : "memory");
}

template <int D, bool kBoxes>
pcomoe_status run(const CUtensorMap &q_map, const PartArgs &a, int sms, cudaStream_t st) {
  static PerDeviceOnce once;
  int dev = -1;
  PCOMOE_CUDA_TRY(cudaGetDevice(&dev));
  if (once.first_use(dev)) {
    PCOMOE_CUDA_TRY(cudaFuncSetAttribute(weigh_tc_kernel<D, kBoxes>, cudaFuncAttributeMaxDynamicSharedMemorySize, Shape<D>::kSmem));
    once.done(dev);
  }
  PCOMOE_CUDA_TRY(launch_pdl(weigh_tc_kernel<D, kBoxes>, dim3(sms), dim3(kThreads), Shape<D>::kSmem, st, q_map, a));
  const pcomoe_status s = launch_join(a, sms, st);
  if (s != PCOMOE_OK) return s;
  count_launch();
  return PCOMOE_OK;
}

}  // namespace

size_t weigh_part_bytes(int hkv, int64_t room, int n) { return sizeof(float) * (size_t)n * (size_t)(hkv * parts_of(hkv)) * (size_t)room; }

pcomoe_status launch_weigh_tc(const WeighArgs &w, int D, float *partial, int64_t room, int sms, cudaStream_t st) {
  PartArgs a = {};
  a.w = w;
  a.partial = partial;
  a.room = room;
  a.parts = parts_of(w.hkv);
  CUtensorMap q = {};
  if (w.n_keep || BC % w.g) return D == 64 ? run<64, false>(q, a, sms, st) : run<128, false>(q, a, sms, st);
  EncodeTiledFn fn = encode_fn();
  if (!fn) return PCOMOE_ERR_CUDA;
  cuuint64_t dims[3] = {(cuuint64_t)D, (cuuint64_t)w.hq, (cuuint64_t)w.T}, strides[2] = {(cuuint64_t)D * 2, (cuuint64_t)w.q_stride * 2};
  cuuint32_t box[3] = {BK, (cuuint32_t)w.g, (cuuint32_t)(BC / w.g)}, estr[3] = {1, 1, 1};
  if (fn(&q, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void *>(w.q), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
         CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS)
    return PCOMOE_ERR_CUDA;
  return D == 64 ? run<64, true>(q, a, sms, st) : run<128, true>(q, a, sms, st);
}

}  // namespace pcomoe
