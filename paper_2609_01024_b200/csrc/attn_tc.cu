// Attention on the tensor cores (tcgen05), bf16: packed prompts, and new or drafted tokens over the paged cache.
//
// One pass over the keys with the running maximum m and sum l of each row's softmax, base 2:
//   m' = max(m, max s),  o <- 2^(m-m') o + sum 2^(s-m') v,  l <- 2^(m-m') l + sum 2^(s-m').
// The maximum only has to keep the weights in range, so it is raised only when a row's new one is more than 8 above it
// (weights then stay below 2^8): the rescaling of o, a round trip through tensor memory, is rare after the first blocks.
//
// A CTA owns 256 rows (tokens x heads of one kv head's group) as two tiles of 128, one TMEM lane and one thread per row.
// Scores S = Q K^T (128 x 128 fp32) of a tile sit in TMEM; its 128 threads read them, and write the weights back as bf16
// over them, where the second product O += P V takes them as its A operand.  The two tiles take turns: while one's
// weights are formed, the tensor cores work for the other.  With at most 128 rows both tiles hold the same rows and
// take alternate blocks of keys, so a few drafted tokens over a long cache still keep both busy; the halves are joined
// at the end.
//   warps 0-3, 4-7: softmax of tile 0 and 1, and its epilogue     warp 8: issues the MMAs and owns TMEM
//   warp 9: TMA loads of K and V into a ring (128-byte swizzle)   warp 10: nothing (register shares go by four warps)
//   warp 11: finds the CTA's pieces of work and hands them to the others through shared memory
// K is the K-major B operand of the first product; V ([key][d] as it lies in memory) the MN-major B operand of the second.
// The softmax threads clear the V rows past the end of a sequence before they hand over the weights of that block, which
// keeps stale memory out of the sums; a NaN or infinity in a row of V that only some rows of a tile see meets
// the others with weight 0 and would turn them into NaN: a row whose output is not finite is formed again without the
// tensor cores, from what it sees alone.
#include <algorithm>

#include "attn.cuh"

namespace pcomoe {
namespace {

constexpr int BM = 256, BN = 128;              // rows of a CTA, keys of a block
constexpr int kSoftmaxThreads = 256, kThreads = 384;
constexpr int kSoftmaxRegs = 208, kOtherRegs = 88, kLaunchRegs = 168;
static_assert(256 * kSoftmaxRegs + 128 * kOtherRegs <= kThreads * kLaunchRegs, "register split");
constexpr float kSlack = 8.f;                  // how far a maximum may run ahead of the one in use, in powers of two

template <int D> struct Shape {
  static constexpr int kHalves = D / 64;                    // 64-column halves, one 128-byte swizzle row each
  static constexpr int kHalfBytes = 128 * 128;
  static constexpr int kTileBytes = kHalves * kHalfBytes;   // 128 rows of Q, K or V
  static constexpr int kStages = D == 128 ? 5 : 8;
  static constexpr int kSmem = 1024 + (2 + kStages) * kTileBytes;
  static constexpr uint32_t kS = 0, kO = 256;               // TMEM columns: scores of the tiles (128 each), outputs (D each)
};

struct TcMaps {
  CUtensorMap k, v;
};

// mbar_wait without its call: the register split of the kernel leaves no room for the calling convention.
__device__ __forceinline__ bool wait_bar(uint64_t *bar_ptr, uint32_t parity, volatile int *abort_flag, uint64_t limit_ns) {
  const uint32_t bar = smem_u32(bar_ptr);
  if (mbar_try_wait(bar, parity)) return true;
  const uint64_t t0 = global_ns();
  for (uint32_t it = 1; it < (1u << 24); ++it) {
    if (mbar_try_wait(bar, parity)) return true;
    if (*abort_flag) return false;
    if (global_ns() - t0 > limit_ns) break;
  }
  *abort_flag = 1;
  return false;
}

// D (+)= A B, fp32 accumulators, bf16 operands; A from shared memory or from TMEM
__device__ __forceinline__ void mma_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t acc) {
  asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d), "l"(a),
               "l"(b), "r"(idesc), "r"(acc)
               : "memory");
}
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, uint32_t acc) {
  asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d), "r"(a),
               "l"(b), "r"(idesc), "r"(acc)
               : "memory");
}
// [key][d] tile as the MN-major B operand: 64 columns in a swizzle row, 8 keys to 1024 bytes, halves kHalfBytes apart
__device__ __forceinline__ uint64_t mn_desc(uint32_t saddr, uint32_t half_bytes) {
  return (uint64_t)((saddr & 0x3FFFFu) >> 4) | ((uint64_t)(half_bytes >> 4) << 16) | ((uint64_t)(1024 >> 4) << 32) | ((uint64_t)1 << 46) |
         ((uint64_t)2 << 61);
}
// 16 columns of this thread's TMEM lane; wider vectors would not leave the scores their registers
__device__ __forceinline__ void tmem_st16(uint32_t taddr, const uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15};" ::"r"(r[0]),
      "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]),
      "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(taddr)
      : "memory");
}
__device__ __forceinline__ void tmem_ld16(uint32_t taddr, uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];\n\ttcgen05.wait::ld.sync.aligned;"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]),
        "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
      : "r"(taddr)
      : "memory");
}
__device__ __forceinline__ void tmem_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void fence_async_smem() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
  return *(const uint32_t *)&v;
}

// A piece of work: blocks [b0, b1) of keys for the rows of one tile of 256.
struct Item {
  Seq seq;
  int kvh, tile, b0, b1;
  int rows;             // of 256; 0: no more work
  bool both;            // two tiles of rows; else two sets of blocks for one tile
  bool whole;
  int slot, first_cta, n_parts;

  __device__ int blocks() const { return b1 - b0; }
};

// The walk over a CTA's items (one warp, all lanes).
template <bool kCached> struct Walk;

template <> struct Walk<true> {
  CacheWalk<BM, BN> w;
  bool some;
  __device__ void start(const AttnArgs &a) { some = w.start(a, blockIdx.x, gridDim.x, 4); }
  __device__ bool next(const AttnArgs &a, Item &it) {
    if (!some || w.at >= w.end) return false;
    const auto p = w.next(a);
    it.seq = w.seq; it.kvh = p.kvh; it.tile = p.tile; it.b0 = p.b0; it.b1 = p.b1;
    it.whole = p.whole; it.slot = part_slot(blockIdx.x, p.b0 == 0); it.first_cta = p.first_cta; it.n_parts = p.n_parts;
    it.rows = min(BM, it.seq.n * a.g - it.tile * BM);
    it.both = it.rows > 128;
    return true;
  }
};

// Prompts: one tile per CTA, counted from the last one back, so that those with the most keys start first.
template <> struct Walk<false> {
  int s, tile;
  bool some;
  __device__ void start(const AttnArgs &a) {
    const int lane = threadIdx.x & 31;
    int want = (int)(gridDim.x - 1 - blockIdx.x) / a.hkv;
    some = false;
    for (int s0 = 0; s0 < a.n_seqs; s0 += 32) {
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
        some = true;
        return;
      }
      want -= __shfl_sync(~0u, upto, 31);
    }
  }
  __device__ bool next(const AttnArgs &a, Item &it) {
    if (!some) return false;
    some = false;
    it.seq = load_seq<false>(a, s);
    it.kvh = (int)(gridDim.x - 1 - blockIdx.x) % a.hkv;
    it.tile = tile; it.b0 = 0; it.b1 = tile_blocks<false, BM, BN>(a, it.seq, tile);
    it.whole = true; it.slot = it.first_cta = 0; it.n_parts = 1;
    it.rows = min(BM, it.seq.n * a.g - tile * BM);
    it.both = it.rows > 128;
    return true;
  }
};

// Blocks that tile t of an item works on.
template <bool kCached>
__device__ __forceinline__ int tile_steps(const AttnArgs &a, const Item &it, int t) {
  const int n = it.blocks();
  if (!it.both) return (n + 1 - t) >> 1;
  if (kCached || t) return n;
  return min(n, tile_blocks<false, 128, BN>(a, it.seq, 2 * it.tile) - it.b0);
}

template <int D, bool kCached>
__global__ void __launch_bounds__(kThreads, 1) attn_tc_kernel(const __grid_constant__ TcMaps maps, const __grid_constant__ AttnArgs a) {
  using S = Shape<D>;
  constexpr uint32_t kIdescS = (1u << 4) | (1u << 7) | (1u << 10) | ((128u >> 3) << 17) | ((128u >> 4) << 24);
  constexpr uint32_t kIdescO = (1u << 4) | (1u << 7) | (1u << 10) | (1u << 16) | (((uint32_t)D >> 3) << 17) | ((128u >> 4) << 24);
  extern __shared__ uint8_t smem_raw[];
  __shared__ __align__(8) uint64_t s_full[S::kStages], s_empty[S::kStages], s_sfull[2], s_pfull[2], s_ofull[2], s_qfull;
  __shared__ uint32_t s_tmem;
  __shared__ int s_abort, s_flag, s_again;
  __shared__ __align__(8) uint64_t s_ifull[2], s_iempty[2];
  __shared__ Item s_item[2];
  __shared__ uint8_t s_bad[BM];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  const uint32_t q_at = base, ring = base + 2 * S::kTileBytes;
  // maxima and sums of the two tiles, for items with one tile of rows: in the place of the second tile's queries
  float2 *s_ml = (float2 *)(smem_raw + (q_at + S::kTileBytes - smem_u32(smem_raw)));
  volatile int *abort_flag = &s_abort;

  if (tid == 0) {
    s_abort = 0;
    s_again = 0;
    for (int i = 0; i < S::kStages; ++i) { mbar_init(smem_u32(&s_full[i]), 1); mbar_init(smem_u32(&s_empty[i]), 1); }
    for (int t = 0; t < 2; ++t) { mbar_init(smem_u32(&s_sfull[t]), 1); mbar_init(smem_u32(&s_pfull[t]), 4); mbar_init(smem_u32(&s_ofull[t]), 1); }
    mbar_init(smem_u32(&s_qfull), 8);
    for (int i = 0; i < 2; ++i) { mbar_init(smem_u32(&s_ifull[i]), 1); mbar_init(smem_u32(&s_iempty[i]), 10); }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 8) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&s_tmem)), "r"(512) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = s_tmem;
  pdl_grid_wait();

  uint32_t pos = 0;                                       // ring stages used so far
  auto stage = [&](uint32_t p) { return p % S::kStages; };
  auto phase = [&](uint32_t p) { return (p / S::kStages) & 1; };
  uint32_t n_item = 0;                                    // pieces so far
  auto item_ready = [&](bool ok) { return ok && wait_bar(&s_ifull[n_item & 1], (n_item >> 1) & 1, abort_flag, a.limit_ns); };
  auto item_done = [&]() {
    __syncwarp();
    if (lane == 0) mbar_arrive(smem_u32(&s_iempty[n_item & 1]));
    ++n_item;
  };
  if (warp < 8) {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kSoftmaxRegs));
    const int t = warp >> 2;                              // tile
    const int r = (warp & 3) * 32 + lane;                 // row of the tile = TMEM lane
    const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
    const uint32_t s_col = tmem + S::kS + t * 128 + lanes, o_col = tmem + S::kO + t * D + lanes;
    uint32_t n_s = 0, n_o0 = 0, n_o1 = 0;                 // steps so far of this tile, finished outputs of both
    bool ok = true;
    // a warp that gives up a wait goes on without waiting to the end of its piece (the barriers below need every warp);
    // the next piece is begun by all eight or by none
    while (all_first<kSoftmaxThreads>(item_ready(ok))) {
      const Item &it = s_item[n_item & 1];
      if (it.rows == 0) break;
      // queries into shared memory, rows past the end as zero
      const int q_rows = it.both ? 256 : 128;
      for (int u0 = tid; u0 < q_rows * (D / 8); u0 += kSoftmaxThreads * 4) {
        uint4 x[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int u = u0 + i * kSoftmaxThreads, qr = u / (D / 8), c = u % (D / 8);
          x[i] = make_uint4(0, 0, 0, 0);
          if (u < q_rows * (D / 8) && qr < it.rows) {
            const int row = it.tile * BM + qr, tok = row / a.g, head = it.kvh * a.g + row - tok * a.g;
            x[i] = *(const uint4 *)((const __nv_bfloat16 *)a.q + (int64_t)(it.seq.q0 + tok) * a.q_stride + head * D + c * 8);
          }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int u = u0 + i * kSoftmaxThreads, qr = u / (D / 8), c = u % (D / 8);
          if (u >= q_rows * (D / 8)) continue;
          const uint32_t at = q_at + (qr >> 7) * S::kTileBytes + (c >> 3) * S::kHalfBytes + (qr & 127) * 128 + (((c & 7) ^ (qr & 7)) << 4);
          asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(x[i].x), "r"(x[i].y), "r"(x[i].z), "r"(x[i].w) : "memory");
        }
      }
      fence_async_smem();
      __syncwarp();
      if (lane == 0) mbar_arrive(smem_u32(&s_qfull));

      const int my_row = it.both ? t * 128 + r : r;       // of the item's rows
      const int tok = (it.tile * BM + min(my_row, it.rows - 1)) / a.g;
      const int first_tok = __shfl_sync(~0u, tok, 0);
      const int steps = tile_steps<kCached>(a, it, t);
      float m = -INFINITY, l = 0.f;
      for (int i = 0; i < steps; ++i, ++n_s) {
        const int b = it.b0 + (it.both ? i : 2 * i + t), p0 = b * BN;
        if (ok) ok = wait_bar(&s_sfull[t], n_s & 1, abort_flag, a.limit_ns);
        __syncwarp();
        tc_fence_after();
        uint32_t s[4][32];
#pragma unroll
        for (int c = 0; c < 4; ++c) tmem_ld32_issue(s_col + 32 * c, s[c]);
        tmem_wait_ld();
#pragma unroll
        for (int c = 0; c < 4; ++c) reg_fence32(s[c]);
        if (p0 + BN > (kCached ? it.seq.base : first_tok + 1) || p0 + BN > it.seq.len) {
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            const uint32_t bits = seen_bits<kCached>(a, it.seq, tok, p0 + 32 * c);
#pragma unroll
            for (int k = 0; k < 32; ++k)
              if (!((bits >> k) & 1)) s[c][k] = 0xff800000u;
          }
          __syncwarp();
        }
        float mx[4];
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          mx[c] = __uint_as_float(s[c][0]);
#pragma unroll
          for (int k = 1; k < 32; ++k) mx[c] = fmaxf(mx[c], __uint_as_float(s[c][k]));
        }
        const float mb = fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3])) * a.scale_log2;
        const bool raise = mb > m + kSlack || (m == -INFINITY && mb > m);
        if (__any_sync(~0u, raise)) {
          const float mn = raise ? mb : m, c = raise ? ex2f(m - mn) : 1.f;
          m = mn;
          l *= c;
          if (i > 0) {
#pragma unroll 1
            for (int h = 0; h < D / 16; ++h) {
              uint32_t o[16];
              tmem_ld16(o_col + 16 * h, o);
#pragma unroll
              for (int k = 0; k < 16; ++k) o[k] = __float_as_uint(__uint_as_float(o[k]) * c);
              tmem_st16(o_col + 16 * h, o);
            }
          }
        }
        const float ms = m == -INFINITY ? 0.f : m;
        float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          uint32_t p[16];
#pragma unroll
          for (int k = 0; k < 16; ++k) {
            const float x = ex2f(fmaf(__uint_as_float(s[c][2 * k]), a.scale_log2, -ms));
            const float y = ex2f(fmaf(__uint_as_float(s[c][2 * k + 1]), a.scale_log2, -ms));
            sum[k & 1] += x;
            sum[2 + (k & 1)] += y;
            p[k] = pack_bf16(x, y);
          }
          tmem_st16(s_col + 16 * c, p);
        }
        l += (sum[0] + sum[1]) + (sum[2] + sum[3]);
        if (b == it.b1 - 1 && p0 + BN > it.seq.len) {
          // the last V of the piece lies in its last ring stage; the scores of this block say that every earlier stage of
          // the ring's last round was filled, so the phase waited for is the one that is pending
          const uint32_t last = pos + 2 * it.blocks() - 1, st = stage(last);
          if (ok) ok = wait_bar(&s_full[st], phase(last), abort_flag, a.limit_ns);
          const int first = max(it.seq.len - p0, 0), rest = (BN - first) * 8;      // 16-byte pieces of a half
          for (int u = r; u < rest * S::kHalves; u += 128) {
            const int h = u / rest, x = u - h * rest;
            asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(ring + st * S::kTileBytes + h * S::kHalfBytes + first * 128 + x * 16),
                         "r"(0)
                         : "memory");
          }
          fence_async_smem();
          __syncwarp();
        }
        tmem_wait_st();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&s_pfull[t]));
      }

      pos += 2 * it.blocks();

      // epilogue: a thread writes its row, or, where both tiles hold the same rows, half of the columns of both
      if (!it.both) s_ml[t * 128 + r] = make_float2(m, l);
      s_bad[t * 128 + r] = 0;
      sync_first<kSoftmaxThreads>();
      const bool row_here = my_row < it.rows;
      const int row = it.tile * BM + my_row, head = it.kvh * a.g + row - tok * a.g;
      const int64_t tg = it.seq.q0 + tok;
      float w0 = t ? 0.f : 1.f, w1 = t ? 1.f : 0.f, inv = 1.f;      // weights of the tiles' sums
      int c0 = 0, c1 = D;
      if (it.both) {
        if (ok) ok = t ? wait_bar(&s_ofull[1], n_o1 & 1, abort_flag, a.limit_ns) : wait_bar(&s_ofull[0], n_o0 & 1, abort_flag, a.limit_ns);
        ++n_o0;
        ++n_o1;
      } else {
        const float2 x = s_ml[r], y = s_ml[128 + r];
        m = fmaxf(x.x, y.x);
        const float ms = m == -INFINITY ? 0.f : m;
        w0 = ex2f(x.x - ms);
        w1 = ex2f(y.x - ms);
        l = w0 * x.y + w1 * y.y;
        c0 = t * (D / 2);
        c1 = c0 + D / 2;
        if (ok) ok = wait_bar(&s_ofull[0], n_o0 & 1, abort_flag, a.limit_ns);
        ++n_o0;
        if (it.blocks() > 1) {
          if (ok) ok = wait_bar(&s_ofull[1], n_o1 & 1, abort_flag, a.limit_ns);
          ++n_o1;
        }
      }
      if (it.whole) inv = l == 0.f ? 0.f : 1.f / l;
      __syncwarp();
      tc_fence_after();
      bool finite = true;
      const int64_t part_row = (int64_t)it.slot * BM + my_row;
#pragma unroll 1
      for (int c = c0; c < c1; c += 32) {
        __syncwarp();
        float o[32];
#pragma unroll
        for (int k = 0; k < 32; ++k) o[k] = 0.f;
#pragma unroll
        for (int q = 0; q < 2; ++q) {
          if (it.both ? q != t : q >= it.blocks()) continue;
          uint32_t x[32];
          tmem_ld32_issue(tmem + S::kO + q * D + lanes + c, x);
          tmem_wait_ld();
          reg_fence32(x);
          // a tile in which the row saw nothing has no say, whatever its sums hold
          const float w = q ? w1 : w0;
          if (w != 0.f)
#pragma unroll
            for (int k = 0; k < 32; ++k) o[k] = fmaf(w, __uint_as_float(x[k]), o[k]);
        }
#pragma unroll
        for (int k = 0; k < 32; ++k) finite &= fabsf(o[k]) < INFINITY;
        if (!row_here) continue;
        if (it.whole) {
          __nv_bfloat16 *to = (__nv_bfloat16 *)a.out + tg * a.out_stride + head * D + c;
#pragma unroll
          for (int k = 0; k < 32; k += 8)
            *(uint4 *)(to + k) = make_uint4(pack_bf16(o[k] * inv, o[k + 1] * inv), pack_bf16(o[k + 2] * inv, o[k + 3] * inv),
                                            pack_bf16(o[k + 4] * inv, o[k + 5] * inv), pack_bf16(o[k + 6] * inv, o[k + 7] * inv));
        } else {
#pragma unroll
          for (int k = 0; k < 32; k += 4) *(float4 *)(a.part + part_row * D + c + k) = make_float4(o[k], o[k + 1], o[k + 2], o[k + 3]);
        }
      }
      if (row_here && c0 == 0) {
        if (!it.whole) *((float2 *)a.part_ml + part_row) = make_float2(m, l);
        else if (a.lse) a.lse[tg * a.hq + head] = l == 0.f ? -INFINITY : m * kLn2f + logf(l);
      }
      tc_fence_before();
      if (row_here && !finite) {
        s_bad[my_row] = 1;
        s_again = 1;
      }
      sync_first<kSoftmaxThreads>();
      if (s_again) {
        for (int x = warp; x < it.rows; x += 8)
          if (s_bad[x]) plain_row<D, BM, kCached>(a, it.seq, it.kvh, it.tile, x, it.b0 * BN, it.b1 * BN, it.whole, it.slot);
        sync_first<kSoftmaxThreads>();
        if (tid == 0) s_again = 0;
        sync_first<kSoftmaxThreads>();
      }
      if (!it.whole && last_part<kSoftmaxThreads>(a, it.first_cta, it.n_parts, &s_flag))
        join_parts<__nv_bfloat16, D, BM, kSoftmaxThreads>(a, it.seq, it.kvh, it.tile, it.first_cta, it.n_parts,
                                                           (float *)(smem_raw + (q_at - smem_u32(smem_raw))), 2 * S::kTileBytes / 4);
      item_done();
    }
  } else {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kOtherRegs));
    if (warp == 9) {
      // ---- loads: K and V blocks in the order in which the MMAs take them
      bool ok = true;
      for (; __all_sync(~0u, item_ready(ok)); item_done()) {
        const Item it = s_item[n_item & 1];
        if (it.rows == 0) break;
        const int n = it.blocks(), lag = it.both ? 1 : 2;
        const int32_t *table = kCached ? a.table + (int64_t)it.seq.id * a.max_pages : nullptr;
        for (int i = 0; ok && i < n + lag; ++i)
          for (int kv = 1; kv >= 0; --kv) {               // V of an earlier block before the K of this one
            const int j = kv ? i - lag : i;
            if (j < 0 || j >= n) continue;
            const uint32_t st = stage(pos);
            ok = wait_bar(&s_empty[st], phase(pos) ^ 1, abort_flag, a.limit_ns);
            ok = __all_sync(~0u, ok);
            if (!ok) break;
            const uint32_t bar = smem_u32(&s_full[st]), to = ring + st * S::kTileBytes;
            const CUtensorMap *map = kv ? &maps.v : &maps.k;
            const int p0 = (it.b0 + j) * BN;
            if (lane == 0) mbar_arrive_expect_tx(bar, S::kTileBytes);
            __syncwarp();
            if (kCached) {
              const int boxes = max(1, BN >> a.page_shift), box_rows = min(BN, a.page);
              for (int u = lane; u < boxes * S::kHalves; u += 32) {
                const int h = u % S::kHalves, x = u / S::kHalves, p = p0 + x * box_rows;
                int64_t at = 0;                           // past the end: any page, its weights are 0 and its V rows are cleared
                if (p < it.seq.len) at = page_row(a, table, it.kvh, p);
                tma_load_2d(to + h * S::kHalfBytes + x * box_rows * 128, map, h * 64, (int32_t)at, bar);
              }
            } else if (lane < S::kHalves) {
              tma_load_2d(to + lane * S::kHalfBytes, map, it.kvh * D + lane * 64, it.seq.q0 + p0, bar);
            }
            ++pos;
          }
      }
    } else if (warp == 8) {
      // ---- MMAs, all from one thread
      uint32_t n_p[2] = {0, 0}, n_q = 0;
      bool ok = true;
      auto wait = [&](uint64_t *bar, uint32_t ph) { return wait_bar(bar, ph, abort_flag, a.limit_ns); };
      auto scores = [&](int t, int q, uint32_t st) {      // S_t = Q_q K^T
        const uint64_t da = umma_desc(q_at + q * S::kTileBytes), db = umma_desc(ring + st * S::kTileBytes);
#pragma unroll
        for (int k = 0; k < D / 16; ++k) {
          const uint64_t off = (uint64_t)((k >> 2) * (S::kHalfBytes >> 4) + (k & 3) * 2);
          mma_ss(tmem + S::kS + t * 128, da + off, db + off, kIdescS, k != 0);
        }
        umma_commit(smem_u32(&s_sfull[t]));
      };
      auto output = [&](int t, uint32_t st, bool first) {  // O_t += P_t V
        const uint64_t dv = mn_desc(ring + st * S::kTileBytes, S::kHalfBytes);
#pragma unroll
        for (int k = 0; k < BN / 16; ++k)
          mma_ts(tmem + S::kO + t * D, tmem + S::kS + t * 128 + k * 8, dv + (uint64_t)(k * (2048 >> 4)), kIdescO, !first || k != 0);
      };
      for (; __all_sync(~0u, item_ready(ok)); item_done()) {
        const Item &it = s_item[n_item & 1];
        if (it.rows == 0) break;
        if (lane == 0) {
          const int n = it.blocks();
          const int steps0 = tile_steps<kCached>(a, it, 0);
          ok = wait(&s_qfull, n_q++ & 1);
          tc_fence_after();
          if (it.both) {
            for (int j = 0; ok && j <= n; ++j) {
              const uint32_t pv = pos, pk = j ? pos + 1 : pos;
              pos = pk + (j < n ? 1 : 0);
              if (j > 0) {
                ok = wait(&s_full[stage(pv)], phase(pv));
              }
              if (ok && j < n) ok = wait(&s_full[stage(pk)], phase(pk));
#pragma unroll
              for (int t = 0; t < 2; ++t) {
                const int steps = t ? n : steps0;
                if (ok && j > 0 && j - 1 < steps) {
                  ok = wait(&s_pfull[t], n_p[t]++ & 1);
                  if (!ok) break;
                  tc_fence_after();
                  output(t, stage(pv), j == 1);
                  if (j == steps) umma_commit(smem_u32(&s_ofull[t]));
                }
                if (t == 1 && ok && j > 0) umma_commit(smem_u32(&s_empty[stage(pv)]));
                if (ok && j < steps) scores(t, t, stage(pk));
                if (t == 1 && ok && j < n) umma_commit(smem_u32(&s_empty[stage(pk)]));
              }
            }
          } else {
            for (int i = 0; ok && i < n + 2; ++i) {
              const int t = i & 1;
              if (i >= 2) {
                const uint32_t pv = pos++;
                ok = wait(&s_full[stage(pv)], phase(pv));
                if (ok) ok = wait(&s_pfull[t], n_p[t]++ & 1);
                if (!ok) break;
                tc_fence_after();
                output(t, stage(pv), i < 4);
                umma_commit(smem_u32(&s_empty[stage(pv)]));
                if (i >= n) umma_commit(smem_u32(&s_ofull[t]));
              }
              if (i < n) {
                const uint32_t pk = pos++;
                ok = wait(&s_full[stage(pk)], phase(pk));
                if (!ok) break;
                scores(t, 0, stage(pk));
                umma_commit(smem_u32(&s_empty[stage(pk)]));
              }
            }
          }
        }
        ok = __shfl_sync(~0u, (int)ok, 0);
      }
    } else if (warp == 11) {
      // ---- the pieces of work
      Walk<kCached> walk;
      walk.start(a);
      for (bool more = true; more; ++n_item) {
        Item it;
        more = walk.next(a, it);
        if (!more) it.rows = 0;
        if (!__all_sync(~0u, wait_bar(&s_iempty[n_item & 1], ((n_item >> 1) & 1) ^ 1, abort_flag, a.limit_ns))) break;
        if (lane == 0) {
          s_item[n_item & 1] = it;
          mbar_arrive(smem_u32(&s_ifull[n_item & 1]));
        }
        __syncwarp();
      }
    }
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (s_abort) timeout_record_and_drain(a.status);
  __syncthreads();
  if (warp == 8) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512) : "memory");
}

bool make_rows_map(CUtensorMap *m, const void *base, uint64_t rows, uint64_t cols, uint64_t stride, uint32_t box_rows) {
  EncodeTiledFn fn = encode_fn();
  if (!fn) return false;
  cuuint64_t dims[2] = {cols, rows}, strides[1] = {stride * 2};
  cuuint32_t box[2] = {BK, box_rows}, estr[2] = {1, 1};
  return fn(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void *>(base), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
            CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int D, bool kCached>
pcomoe_status run(const TcMaps &m, const AttnArgs &a, unsigned grid, cudaStream_t st) {
  static PerDeviceOnce once;
  int dev = -1;
  PCOMOE_CUDA_TRY(cudaGetDevice(&dev));
  if (once.first_use(dev)) {
    // the register split draws on what the block was launched with: fewer and the larger share would never come
    cudaFuncAttributes at;
    PCOMOE_CUDA_TRY(cudaFuncGetAttributes(&at, attn_tc_kernel<D, kCached>));
    if (at.numRegs < kLaunchRegs) return PCOMOE_ERR_CUDA;
    PCOMOE_CUDA_TRY(cudaFuncSetAttribute(attn_tc_kernel<D, kCached>, cudaFuncAttributeMaxDynamicSharedMemorySize, Shape<D>::kSmem));
    once.done(dev);
  }
  PCOMOE_CUDA_TRY(launch_pdl(attn_tc_kernel<D, kCached>, dim3(grid), dim3(kThreads), Shape<D>::kSmem, st, m, a));
  count_launch();
  return PCOMOE_OK;
}

}  // namespace

size_t attn_tc_part_rows(int sms) { return (size_t)2 * sms * BM; }

pcomoe_status launch_attn_tc(const AttnArgs &a, int D, int sms, cudaStream_t st) {
  TcMaps m;
  if (a.table) {
    const uint64_t rows = (uint64_t)a.pages * a.hkv * a.page;
    if (rows > INT32_MAX) return PCOMOE_ERR_UNSUPPORTED;                 // row numbers of a TMA copy are 32 bits
    const uint32_t box = std::min(BN, a.page);
    if (!make_rows_map(&m.k, a.k, rows, D, D, box) || !make_rows_map(&m.v, a.v, rows, D, D, box)) return PCOMOE_ERR_CUDA;
    return D == 64 ? run<64, true>(m, a, sms, st) : run<128, true>(m, a, sms, st);
  }
  if (!make_rows_map(&m.k, a.k, a.T, (uint64_t)a.hkv * D, a.k_stride, BN) || !make_rows_map(&m.v, a.v, a.T, (uint64_t)a.hkv * D, a.v_stride, BN))
    return PCOMOE_ERR_CUDA;
  const int64_t tiles = (int64_t)a.T * a.g / BM + std::min(a.n_seqs, a.T);
  if (tiles * a.hkv > INT32_MAX) return PCOMOE_ERR_SHAPE;
  return D == 64 ? run<64, false>(m, a, (unsigned)(tiles * a.hkv), st) : run<128, false>(m, a, (unsigned)(tiles * a.hkv), st);
}

}  // namespace pcomoe
