// Attention on the tensor cores (tcgen05), bf16: packed prompts, and new or drafted tokens over the paged cache.
//
// One pass over the keys with the running maximum m and sum l of each row's softmax, base 2:
//   m' = max(m, max s),  o <- 2^(m-m') o + sum 2^(s-m') v,  l <- 2^(m-m') l + sum 2^(s-m').
// The maximum only has to keep the weights in range, so it is raised only when a row's new one is more than 8 above it
// (weights then stay below 2^8): the rescaling of o, a round trip through tensor memory, is rare after the first blocks.
//
// A CTA owns 256 rows (tokens x heads of one kv head's group) as two tiles of 128, one TMEM lane and one thread per row.
// Scores S = Q K^T (128 x 128 fp32) of a tile sit in TMEM; its 128 threads read them, and write the weights back as bf16
// over them, where the second product O += P V takes them as its A operand (its operands have one type: an error of at most
// 2^-8 of each weight, as of the output's own rounding; the sums l take the weights unrounded).  The two tiles take turns: while one's
// weights are formed, the tensor cores work for the other.  With at most 128 rows both tiles hold the same rows and
// take alternate blocks of keys, so a few drafted tokens over a long cache still keep both busy; the halves are joined
// at the end.
//   warp 0: issues the MMAs and owns TMEM                         warp 1: TMA loads of K and V into a ring (128-byte swizzle)
//   warp 2: copies the queries                                    warp 3: finds the CTA's pieces of work and hands them out
//   warps 4-7, 8-11: softmax of tile 0 and 1, and its epilogue
// The CTAs are persistent and every role runs ahead of the next as far as its buffers allow: the next piece's queries,
// keys and first scores come in while the last one's output is written.  Prompts: pieces are whole tiles, drawn from a
// counter in order of falling length, so that the last ones to finish are short.  Cache: every CTA has an equal share.
// Measured: one prompt of 16384 tokens, 16 heads of 128: 0.93 ms in runs of a few milliseconds, 1.18 PFLOP/s, and 1.07 ms in runs
// of seconds, where the power limit lowers the clock, 1.03 PFLOP/s: 0.73 and 0.75 of a library matrix product's rate in
// the same regime; prompts of 1531, 1523, 977, 64 and 1 tokens, 32 heads on 8: 67 us (a third of it the pieces'
// beginnings and ends); 17 to 48 drafts over 8 sequences of 905 to 4050 tokens, 32 heads on 8: 42 us with the joining
// launch, 85 MB.  (168 registers at launch; 36 bytes a thread spilled in the prompt forms, 72 in the cached ones.)
//
// What bounds it once the products are fed is the chain of a tile: scores done -> read, maximum, 128 exponentials per thread
// -> weights written -> two products; the special function unit's rate (16 per clock and SM) makes the middle 1024 clocks
// long at least, and the products 1024.  Tried and not kept, for one prompt of 16384 tokens with 16 heads (this form
// 0.93 ms): a polynomial on the FMA pipe for 1, 2 or 3 of 8 exponentials 0.92, 0.94, 0.97 ms (issue slots are
// as scarce as exponentials); two threads per row 0.99; scores read twice so that loops stay short 0.97; weights formed with
// a stale maximum while a vote is out 1.35.
// The softmax threads clear the V rows past the end of a sequence before they hand over the weights of that block, which
// keeps stale memory out of the sums; a NaN or infinity in a row of V that only some rows of a tile see meets
// the others with weight 0 and turns them into NaN: a row that met such a value is formed again without the tensor cores,
// from what it sees alone.
#include <algorithm>

#include "attn.cuh"

namespace pcomoe {
namespace {

constexpr int BM = 256, BN = 128;              // rows of a CTA, keys of a block
constexpr int kFirst = 128, kTileThreads = 128, kSoftmaxThreads = 256, kThreads = 384;      // softmax threads from thread kFirst on
constexpr int kSoftmaxRegs = 208, kOtherRegs = 88, kLaunchRegs = 168;
static_assert(256 * kSoftmaxRegs + 128 * kOtherRegs <= kThreads * kLaunchRegs, "register split");
constexpr float kSlack = 8.f;                  // how far a maximum may run ahead of the one in use, in powers of two

template <int D> struct Shape {
  static constexpr int kHalves = D / 64;                    // 64-column halves, one 128-byte swizzle row each
  static constexpr int kHalfBytes = 128 * 128;
  static constexpr int kTileBytes = kHalves * kHalfBytes;   // 128 rows of Q, K or V
  static constexpr int kStages = D == 128 ? 5 : 8;
  static constexpr int kSmem = (2 + kStages) * kTileBytes;
  static constexpr uint32_t kS = 0, kO = 256;               // TMEM columns: scores of the tiles (128 each), outputs (D each)
};

struct TcMaps {
  CUtensorMap q, k, v;
};

__device__ __forceinline__ bool elect_lane() {
  uint32_t e;
  asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(e));
  return e;
}

__device__ __forceinline__ void tma_load_3d(uint32_t dst, const CUtensorMap *map, int32_t x, int32_t y, int32_t z, uint32_t bar) {
  asm volatile("cp.async.bulk.tensor.3d.shared::cta.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(dst), "l"(map),
               "r"(x), "r"(y), "r"(z), "r"(bar)
               : "memory");
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
// 32 bytes at once, a whole sector: rows are a thread each, so a warp's stores lie far apart
__device__ __forceinline__ void store32(void *p, const uint32_t (&x)[8]) {
  asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(x[0]), "r"(x[1]), "r"(x[2]), "r"(x[3]), "r"(x[4]), "r"(x[5]),
               "r"(x[6]), "r"(x[7])
               : "memory");
}

// A piece of work: blocks [b0, b1) of keys for the rows of one tile.
struct Item {
  Seq seq;
  int kvh, row0, b0, b1;
  int rows;             // up to 256 from row0 on; 0: no more work
  bool both;            // two tiles of rows; else two sets of blocks for one tile
  bool whole;
  int slot;             // place of a partial result

  __device__ int blocks() const { return b1 - b0; }
};

// The walk over a CTA's items (one warp, all lanes).
template <bool kCached> struct Walk;

template <> struct Walk<true> {
  CacheWalk<BM, BN, 2, 4> w;
  __device__ void start(const AttnArgs &a) { w.start(a, blockIdx.x, gridDim.x); }
  __device__ bool next(const AttnArgs &a, Item &it) {
    CacheWalk<BM, BN, 2, 4>::Piece p;
    if (!w.next(a, p)) return false;
    it.seq = w.seq; it.kvh = p.kvh; it.row0 = p.tile * BM; it.b0 = p.b0; it.b1 = p.b1;
    it.whole = p.whole; it.slot = part_slot(blockIdx.x, p.b0 == 0);
    it.rows = min(BM, it.seq.n * a.g - it.row0);
    it.both = it.rows > 128;
    return true;
  }
  __device__ void finish(const AttnArgs &a) {
    if ((threadIdx.x & 31) == 0) w.record(a, blockIdx.x);
  }
};

// Prompts: whole tiles from a counter, longest first.  The order needs every sequence's number of tiles at hand: four per
// lane.  Beyond 128 sequences they are taken from the last packed row back instead (a tile is then a small part of the
// whole, and its place matters little).
template <> struct Walk<false> {
  int mine[4];
  int total;
  bool first;
  int rows;             // of a tile: 256, or 128 where that leaves SMs idle (its keys then go to both halves of the CTA)
  __device__ int tiles_of(const AttnArgs &a, int s) const { return s < a.n_seqs ? (load_seq<false>(a, s).n * a.g + rows - 1) / rows : 0; }
  __device__ static int sum(int x) { return (int)__reduce_add_sync(~0u, (unsigned)x); }
  __device__ void start(const AttnArgs &a) {
    const int lane = threadIdx.x & 31;
    // (An upper bound of the number of tiles: every sequence may end in a part of one.  Prompts of 200 and 3404 tokens,
    // 4 heads of 64 on 2: 31 us with 128 rows, 51 us with 256.)
    rows = ((int64_t)a.T * a.g / BM + a.n_seqs) * a.hkv < a.sms ? 128 : BM;
    total = 0;
#pragma unroll
    for (int k = 0; k < 4; ++k) total += mine[k] = tiles_of(a, 32 * k + lane);
    for (int s = 128 + lane; s < a.n_seqs; s += 32) total += tiles_of(a, s);
    total = sum(total);
    first = true;
  }
  // tiles whose number inside their sequence is at least x
  __device__ int from(int x) const { return sum(max(0, mine[0] - x) + max(0, mine[1] - x) + max(0, mine[2] - x) + max(0, mine[3] - x)); }
  __device__ bool next(const AttnArgs &a, Item &it) {
    const int lane = threadIdx.x & 31;
    int w = blockIdx.x;                                    // the first piece needs no counter
    if (!first) {
      if (lane == 0) w = gridDim.x + atomicAdd(&a.counters[0], 1);
      w = __shfl_sync(~0u, w, 0);
    }
    first = false;
    if (w >= total * a.hkv) return false;
    it.kvh = w % a.hkv;
    int want = w / a.hkv, s = 0, tile = 0;
    if (a.n_seqs <= 128) {
      int lo = 0, hi = (int)__reduce_max_sync(~0u, (unsigned)max(max(mine[0], mine[1]), max(mine[2], mine[3])));
      while (hi - lo > 1) {                                // the largest number with more than `want` tiles from it on
        const int mid = (lo + hi) >> 1;
        if (from(mid) > want) lo = mid; else hi = mid;
      }
      want -= from(lo + 1);                                // the want-th of the sequences that have tile lo
      tile = lo;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const uint32_t b = __ballot_sync(~0u, mine[k] > lo);
        const uint32_t hit = __ballot_sync(~0u, mine[k] > lo && __popc(b & ((1u << lane) - 1)) == want);
        if (hit) s = 32 * k + __ffs(hit) - 1;
        want -= __popc(b);
      }
    } else {
      want = total - 1 - want;
      for (int s0 = 0; s0 < a.n_seqs; s0 += 32) {
        const int n = tiles_of(a, s0 + lane);
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
          break;
        }
        want -= __shfl_sync(~0u, upto, 31);
      }
    }
    it.seq = load_seq<false>(a, s);
    it.row0 = tile * rows;
    it.b0 = 0; it.b1 = key_blocks<false, BN>(a, it.seq, it.row0 + rows);
    it.whole = true; it.slot = 0;
    it.rows = min(rows, it.seq.n * a.g - it.row0);
    it.both = it.rows > 128;
    return true;
  }
  // the last CTA to leave sets the counter back
  __device__ void finish(const AttnArgs &a) {
    if ((threadIdx.x & 31) == 0 && atomicAdd(&a.counters[1], 1) == (int)gridDim.x - 1)
      a.counters[0] = a.counters[1] = 0;
  }
};

// Blocks that tile t of an item works on.
template <bool kCached>
__device__ __forceinline__ int tile_steps(const AttnArgs &a, const Item &it, int t) {
  const int n = it.blocks();
  if (!it.both) return (n + 1 - t) >> 1;
  if (kCached || t) return n;
  return min(n, key_blocks<false, BN>(a, it.seq, it.row0 + 128) - it.b0);
}

// Rows of a warp (my_row: this lane's) that may have to be formed again.  Not in line: the registers that it takes are those of
// the softmax (in line, and with the counter outside, prompts took 2 % longer and trees over the cache 4 %).
template <int D, bool kCached>
__device__ __noinline__ void form_again(const AttnArgs &a, const Item &it, int my_row, uint8_t *bad_rows, int *flags) {
  const int lane = threadIdx.x & 31;
  if (lane == 0) atomicAdd(&flags[1], 1);
  const bool bad = bad_rows[my_row];
  if (bad) bad_rows[my_row] = 0;
  const int tok = (it.row0 + min(my_row, it.rows - 1)) / a.g, first_tok = __shfl_sync(~0u, tok, 0);
  const uint32_t todo = __ballot_sync(~0u, met_unseen<D, kCached>(a, it.seq, it.kvh, tok, it.b0 * BN, it.b1 * BN, kCached ? it.seq.base : first_tok + 1, bad));
  plain_rows<D, BM, kCached>(a, it.seq, it.kvh, it.row0, my_row - lane, todo, it.b0 * BN, it.b1 * BN, it.whole, it.slot);
  __syncwarp();
  if (lane == 0) atomicSub(&flags[1], 1);
}

template <int D, bool kCached>
__global__ void __launch_bounds__(kThreads, 1) attn_tc_kernel(const __grid_constant__ TcMaps maps, const __grid_constant__ AttnArgs a) {
  using S = Shape<D>;
  constexpr uint32_t kIdescS = (1u << 4) | (1u << 7) | (1u << 10) | ((128u >> 3) << 17) | ((128u >> 4) << 24);
  constexpr uint32_t kIdescO = (1u << 4) | (1u << 7) | (1u << 10) | (1u << 16) | (((uint32_t)D >> 3) << 17) | ((128u >> 4) << 24);
  extern __shared__ __align__(1024) uint8_t smem[];
  __shared__ __align__(8) uint64_t s_full[S::kStages], s_empty[S::kStages], s_sfull[2], s_pfull[2][2], s_ofull[2], s_qfull[2], s_qempty[2], s_join;
  __shared__ __align__(8) uint64_t s_ifull[2], s_iempty[2];
  __shared__ Item s_item[2];
  __shared__ float2 s_ml[2][128];                         // maxima and sums of the two tiles, where they hold the same rows
  __shared__ uint8_t s_bad[BM];
  __shared__ uint32_t s_tmem;
  __shared__ int s_flags[2];                              // see wait_bar
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const bool wide = (((uintptr_t)a.out | (uintptr_t)(a.out_stride * 2)) & 31) == 0;      // rows begin on whole sectors
  const uint32_t q_at = smem_u32(smem), ring = q_at + 2 * S::kTileBytes;
  volatile int *flags = s_flags;

  if (tid == 0) {
    s_flags[0] = q_at & 1023 ? 1 : 0;                     // the swizzle needs it; nothing would be right otherwise
    s_flags[1] = 0;
    for (int i = 0; i < S::kStages; ++i) { mbar_init(smem_u32(&s_full[i]), 1); mbar_init(smem_u32(&s_empty[i]), 1); }
    for (int t = 0; t < 2; ++t) {
      mbar_init(smem_u32(&s_sfull[t]), 1);
      mbar_init(smem_u32(&s_pfull[t][0]), 4);
      mbar_init(smem_u32(&s_pfull[t][1]), 4);
      mbar_init(smem_u32(&s_ofull[t]), 1);
      mbar_init(smem_u32(&s_qfull[t]), 1);
      mbar_init(smem_u32(&s_qempty[t]), 1);
      mbar_init(smem_u32(&s_ifull[t]), 1);
      mbar_init(smem_u32(&s_iempty[t]), 11);              // every warp but the one that fills them
    }
    mbar_init(smem_u32(&s_join), kSoftmaxThreads / 32);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (tid < BM) s_bad[tid] = 0;
  if (warp == 0) {
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
  auto item_ready = [&](bool ok) { return ok && wait_bar(&s_ifull[n_item & 1], (n_item >> 1) & 1, flags, a.limit_ns); };
  auto item_done = [&]() {
    __syncwarp();
    if (lane == 0) mbar_arrive(smem_u32(&s_iempty[n_item & 1]));
    ++n_item;
  };
  if (warp >= kFirst / 32) {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kSoftmaxRegs));
    const int t = (warp - kFirst / 32) >> 2;              // tile
    const int r = (warp & 3) * 32 + lane;                 // row of the tile = TMEM lane
    const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
    const uint32_t s_col = tmem + S::kS + t * 128 + lanes, o_col = tmem + S::kO + t * D + lanes;
    auto all_tile = [&](bool yes) {
      int out;
      __syncwarp();
      asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.b32 p, %1, 0;\n\tbarrier.cta.red.and.aligned.pred q, %2, %3, p;\n\tselp.b32 %0, 1, 0, q;\n\t}"
                   : "=r"(out) : "r"((int)yes), "r"(2 + t), "n"(kTileThreads) : "memory");
      return out != 0;
    };
    uint32_t n_s = 0, n_o0 = 0, n_o1 = 0;                 // steps so far of this tile, finished outputs of both
    const float scale_log2 = a.scale_log2;
    bool ok = true;
    uint32_t n_join = 0;
    // all softmax warps: bounded like every wait, so that a tile's warps that have given up hold nobody
    auto sync_both = [&]() {
      __syncwarp();
      if (lane == 0) mbar_arrive(smem_u32(&s_join));
      if (ok) ok = wait_bar(&s_join, n_join & 1, flags, a.limit_ns);
      ++n_join;
      __syncwarp();
    };
    // a warp that gives up a wait goes on without waiting to the end of its piece (the tile's barriers need every warp);
    // the next piece is begun by all eight warps of a tile or by none
    while (all_tile(item_ready(ok))) {
      const Item &it = s_item[n_item & 1];
      if (it.rows == 0) break;
      const int my_row = it.both ? t * 128 + r : r;       // of the item's rows
      const int tok = (it.row0 + min(my_row, it.rows - 1)) / a.g;
      const int first_tok = __shfl_sync(~0u, tok, 0);
      const int steps = tile_steps<kCached>(a, it, t), len = it.seq.len, base = it.seq.base, b0 = it.b0, b_last = it.b1 - 1;
      const bool both = it.both;                           // (in registers: shared memory is busy feeding the MMAs)
      float m = -INFINITY, l = 0.f;
      for (int i = 0; i < steps; ++i, ++n_s) {
        const int b = b0 + (both ? i : 2 * i + t), p0 = b * BN;
        if (ok) ok = wait_bar(&s_sfull[t], n_s & 1, flags, a.limit_ns);
        __syncwarp();
        tc_fence_after();
        const bool masked = p0 + BN > (kCached ? base : first_tok + 1) || p0 + BN > len;
        uint32_t x[4][32];
        tmem_ld32_issue(s_col, x[0]);
        tmem_ld32_issue(s_col + 32, x[1]);
        tmem_ld32_issue(s_col + 64, x[2]);
        tmem_ld32_issue(s_col + 96, x[3]);
        tmem_wait_ld();
#pragma unroll
        for (int c = 0; c < 4; ++c) reg_fence32(x[c]);
        if (masked) {
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            const uint32_t bits = seen_bits<kCached>(a, it.seq, tok, p0 + 32 * c);
#pragma unroll
            for (int k = 0; k < 32; ++k)
              if (!((bits >> k) & 1)) x[c][k] = 0xff800000u;
          }
          __syncwarp();
        }
        float mx[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) mx[k] = fmaxf(__uint_as_float(x[0][2 * k]), __uint_as_float(x[0][2 * k + 1]));
#pragma unroll
        for (int k = 8; k < 64; ++k) mx[k & 7] = fmaxf(mx[k & 7], fmaxf(__uint_as_float(x[k >> 4][(2 * k) & 31]), __uint_as_float(x[k >> 4][((2 * k) & 31) + 1])));
#pragma unroll
        for (int k = 0; k < 4; ++k) mx[k] = fmaxf(mx[k], mx[k + 4]);
        const float mb = fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3])) * scale_log2;
        const bool raise = mb > m + kSlack;                // also from -inf
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
        if (b == b_last && p0 + BN > len) {
          // the last V of the piece lies in its last ring stage; the scores of this block say that every earlier stage of
          // the ring's last round was filled, so the phase waited for is the one that is pending
          const uint32_t last = pos + 2 * it.blocks() - 1, st = stage(last);
          if (ok) ok = wait_bar(&s_full[st], phase(last), flags, a.limit_ns);
          const int first = max(len - p0, 0), rest = (BN - first) * 8;      // 16-byte pieces of a half
          for (int u = r; u < rest * S::kHalves; u += kTileThreads) {
            const int h = u / rest, x = u - h * rest;
            asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(ring + st * S::kTileBytes + h * S::kHalfBytes + first * 128 + x * 16),
                         "r"(0)
                         : "memory");
          }
          fence_async_smem();
          __syncwarp();
        }
        const float ms = m == -INFINITY ? 0.f : m;
        const float2 scale = make_float2(scale_log2, scale_log2), minus = make_float2(-ms, -ms);
        float2 sum[4] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f), make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          uint32_t p[16];
#pragma unroll
          for (int k = 0; k < 16; ++k) {
            float2 e = fma2(make_float2(__uint_as_float(x[c][2 * k]), __uint_as_float(x[c][2 * k + 1])), scale, minus);
            e = make_float2(ex2f(e.x), ex2f(e.y));
            sum[k & 3] = add2(sum[k & 3], e);
            p[k] = pack_bf16(e.x, e.y);
          }
          tmem_st16(s_col + 16 * c, p);
          if (c & 1) {                                     // a half goes
            tmem_wait_st();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&s_pfull[t][c >> 1]));
          }
        }
        l += ((sum[0].x + sum[0].y) + (sum[1].x + sum[1].y)) + ((sum[2].x + sum[2].y) + (sum[3].x + sum[3].y));
      }
      pos += 2 * it.blocks();

      // epilogue: a thread writes its row, or, where both tiles hold the same rows, half of the columns from both of them
      float w0 = 0.f, w1 = 0.f, inv = 1.f;                 // weights of the tiles' sums, where they hold the same rows
      int c0 = 0, c1 = D;
      if (it.both) {
        if (ok) ok = t ? wait_bar(&s_ofull[1], n_o1 & 1, flags, a.limit_ns) : wait_bar(&s_ofull[0], n_o0 & 1, flags, a.limit_ns);
        ++n_o0;
        ++n_o1;
      } else {
        s_ml[t][r] = make_float2(m, l);
        sync_both();
        const float2 x = s_ml[0][r], y = s_ml[1][r];
        m = fmaxf(x.x, y.x);
        const float ms = m == -INFINITY ? 0.f : m;
        w0 = part_weight(x.x, x.y, ms);
        w1 = part_weight(y.x, y.y, ms);
        l = w0 * x.y + w1 * y.y;                           // kNoPart times 0 adds nothing
        c0 = t * (D / 2);
        c1 = c0 + D / 2;
        if (ok) ok = wait_bar(&s_ofull[0], n_o0 & 1, flags, a.limit_ns);
        ++n_o0;
        if (it.blocks() > 1) {
          if (ok) ok = wait_bar(&s_ofull[1], n_o1 & 1, flags, a.limit_ns);
          ++n_o1;
        }
      }
      const bool row_here = my_row < it.rows;
      const int row = it.row0 + my_row, head = it.kvh * a.g + row - tok * a.g;
      const int64_t tg = it.seq.q0 + tok, part_row = (int64_t)it.slot * BM + my_row;
      if (it.whole) inv = l == 0.f ? 0.f : 1.f / l;
      bool finite = true;
      __nv_bfloat16 *out = (__nv_bfloat16 *)a.out + tg * a.out_stride + head * D;
      float *part = a.part + part_row * D;
      auto write = [&](uint32_t (&o)[32], int c) {         // columns [c, c + 32) of this thread's row
        float2 z = make_float2(0.f, 0.f);                  // not 0 where some value is not finite
#pragma unroll
        for (int k = 0; k < 32; k += 2) z = fma2(make_float2(__uint_as_float(o[k]), __uint_as_float(o[k + 1])), make_float2(0.f, 0.f), z);
        finite &= z.x + z.y == 0.f;
        if (!row_here) return;
        if (it.whole) {
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            uint32_t x[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) x[k] = pack_bf16(__uint_as_float(o[16 * h + 2 * k]) * inv, __uint_as_float(o[16 * h + 2 * k + 1]) * inv);
            if (wide) {
              store32(out + c + 16 * h, x);
            } else {
              *(uint4 *)(out + c + 16 * h) = make_uint4(x[0], x[1], x[2], x[3]);
              *(uint4 *)(out + c + 16 * h + 8) = make_uint4(x[4], x[5], x[6], x[7]);
            }
          }
        } else {
#pragma unroll
          for (int h = 0; h < 4; ++h) {
            uint32_t x[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) x[k] = o[8 * h + k];
            store32(part + c + 8 * h, x);
          }
        }
      };
      tc_fence_after();
      if (it.both) {
#pragma unroll 1
        for (int c = 0; c < D; c += 32) {
          uint32_t o[32];
          __syncwarp();
          tmem_ld32_issue(o_col + c, o);
          tmem_wait_ld();
          reg_fence32(o);
          if (l == 0.f)                                    // a row that saw nothing: whatever the sums hold
#pragma unroll
            for (int k = 0; k < 32; ++k) o[k] = 0;
          write(o, c);
        }
      } else {
#pragma unroll 1
        for (int c = c0; c < c1; c += 32) {
          uint32_t o[32], y[32];
          __syncwarp();
          tmem_ld32_issue(tmem + S::kO + lanes + c, o);
          if (it.blocks() > 1) tmem_ld32_issue(tmem + S::kO + D + lanes + c, y);
          tmem_wait_ld();
          reg_fence32(o);
          reg_fence32(y);
          // a tile in which the row saw nothing has no say, whatever its sums hold
#pragma unroll
          for (int k = 0; k < 32; ++k) {
            const float v = w0 != kNoPart ? w0 * __uint_as_float(o[k]) : 0.f;
            o[k] = __float_as_uint(w1 != kNoPart ? fmaf(w1, __uint_as_float(y[k]), v) : v);
          }
          write(o, c);
        }
      }
      tc_fence_before();
      if (row_here && c0 == 0) {
        if (!it.whole) *((float2 *)a.part_ml + part_row) = make_float2(m, l);
        else if (a.lse) a.lse[tg * a.hq + head] = l == 0.f ? -INFINITY : m * kLn2f + logf(l);
      }
      // rows that may have to be formed again (with a NaN score a row is NaN whatever the values are); also: every thread is
      // done with the outputs and with s_ml
      if (row_here && !finite && l == l) s_bad[my_row] = 1;
      if (!it.both) sync_both();
      if (it.both || t == 0) {
        if (__any_sync(~0u, s_bad[my_row])) form_again<D, kCached>(a, it, my_row, s_bad, s_flags);
      }
      item_done();
    }
  } else {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kOtherRegs));
    if (warp == 1) {
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
            ok = wait_bar(&s_empty[st], phase(pos) ^ 1, flags, a.limit_ns);
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
    } else if (warp == 2) {
      // ---- queries: rows of a tile into the K-major operand layout, rows past the end as zero
      uint32_t n_q[2] = {0, 0};
      bool ok = true;
      for (; __all_sync(~0u, item_ready(ok)); item_done()) {
        const Item &it = s_item[n_item & 1];
        if (it.rows == 0) break;
#pragma unroll
        for (int q = 0; q < 2; ++q) {
          if (q && !it.both) continue;
          ok = ok && wait_bar(&s_qempty[q], (n_q[q] & 1) ^ 1, flags, a.limit_ns);
          ok = __all_sync(~0u, ok);
          if (!ok) break;
          ++n_q[q];
          if (128 % a.g == 0) {
            // whole tokens: one box of 128 / g tokens x g heads per half.  Rows past the end are other rows or zero; their
            // scores are nobody's.
            if (lane == 0) mbar_arrive_expect_tx(smem_u32(&s_qfull[q]), S::kTileBytes);
            __syncwarp();
            if (lane < S::kHalves)
              tma_load_3d(q_at + q * S::kTileBytes + lane * S::kHalfBytes, &maps.q, lane * 64, it.kvh * a.g, it.seq.q0 + (it.row0 + q * 128) / a.g,
                          smem_u32(&s_qfull[q]));
            continue;
          }
          const int rows = it.rows - q * 128;
          constexpr int C = D / 8, P = 32 / C;             // pieces of a row; rows that a warp copies side by side
          const int c = lane % C;
          const uint32_t to = q_at + q * S::kTileBytes + (c >> 3) * S::kHalfBytes;
          int tok = (it.row0 + q * 128 + lane / C) / a.g, hd = it.row0 + q * 128 + lane / C - tok * a.g;
          for (int qr = lane / C; qr < 128; qr += P) {
            const bool there = qr < rows;
            const __nv_bfloat16 *src = (const __nv_bfloat16 *)a.q + (there ? (int64_t)(it.seq.q0 + tok) * a.q_stride + (it.kvh * a.g + hd) * D + c * 8 : 0);
            copy16(to + qr * 128 + (((c & 7) ^ (qr & 7)) << 4), src, there);
            for (hd += P; hd >= a.g; hd -= a.g) ++tok;
          }
          asm volatile("cp.async.wait_all;" ::: "memory");
          fence_async_smem();
          __syncwarp();
          if (lane == 0) mbar_arrive(smem_u32(&s_qfull[q]));
        }
      }
    } else if (warp == 0) {
      // ---- MMAs.  The whole warp walks along, so that addresses and descriptors stay warp-uniform; one lane issues.
      uint32_t n_q0 = 0, n_q1 = 0, n_p0 = 0, n_p1 = 0;
      bool ok = true;
      uint32_t st = 0, ph = 0;                            // next ring stage and its phase
      auto advance = [&]() {
        if (++st == S::kStages) { st = 0; ph ^= 1; }
      };
      auto wait = [&](uint64_t *bar, uint32_t p) { return ok = __all_sync(~0u, wait_bar(bar, p, flags, a.limit_ns)); };
      const uint64_t q_desc = umma_desc(q_at), k_desc = umma_desc(ring), v_desc = mn_desc(ring, S::kHalfBytes);
      auto scores = [&](int t, int q, uint32_t at, bool last_q, bool last_k) {      // S_t = Q_q K^T
        const uint64_t da = q_desc + (uint64_t)(q * (S::kTileBytes >> 4)), db = k_desc + (uint64_t)(at * (S::kTileBytes >> 4));
        if (elect_lane()) {
#pragma unroll
          for (int k = 0; k < D / 16; ++k) {
            const uint64_t off = (uint64_t)((k >> 2) * (S::kHalfBytes >> 4) + (k & 3) * 2);
            mma_ss(tmem + S::kS + t * 128, da + off, db + off, kIdescS, k != 0);
          }
          umma_commit(smem_u32(&s_sfull[t]));
          if (last_q) umma_commit(smem_u32(&s_qempty[q]));
          if (last_k) umma_commit(smem_u32(&s_empty[at]));
        }
        __syncwarp();
      };
      // O_t += P_t V, as its two halves come
      auto output = [&](int t, uint32_t at, bool first, bool last_v, bool last_o) {
        const uint64_t dv = v_desc + (uint64_t)(at * (S::kTileBytes >> 4));
        const uint32_t p = t ? n_p1++ & 1 : n_p0++ & 1;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          if (!wait(&s_pfull[t][h], p)) return;
          tc_fence_after();
          if (elect_lane()) {
#pragma unroll
            for (int k = 4 * h; k < 4 * h + 4; ++k)
              mma_ts(tmem + S::kO + t * D, tmem + S::kS + t * 128 + k * 8, dv + (uint64_t)(k * (2048 >> 4)), kIdescO, !first || k != 0);
            if (h && last_v) umma_commit(smem_u32(&s_empty[at]));
            if (h && last_o) umma_commit(smem_u32(&s_ofull[t]));
          }
          __syncwarp();
        }
      };
      for (; __all_sync(~0u, item_ready(ok)); item_done()) {
        const Item &it = s_item[n_item & 1];
        if (it.rows == 0) break;
        const int n = it.blocks();
        if (it.both) {
          const int steps0 = tile_steps<kCached>(a, it, 0);
          for (int j = 0; ok && j <= n; ++j) {
            uint32_t v = st, k = st;
            if (j > 0) {
              if (!wait(&s_full[st], ph)) break;
              advance();
            }
            if (j < n) {
              k = st;
              if (!wait(&s_full[st], ph)) break;
              advance();
            }
            if (j > 0 && j - 1 < steps0) output(0, v, j == 1, false, j == steps0);
            if (ok && j < steps0) {
              if (j == 0) wait(&s_qfull[0], n_q0++ & 1);
              if (!ok) break;
              scores(0, 0, k, j == steps0 - 1, false);
            }
            if (ok && j > 0) output(1, v, j == 1, true, j == n);
            if (ok && j < n) {
              if (j == 0) wait(&s_qfull[1], n_q1++ & 1);
              if (!ok) break;
              scores(1, 1, k, j == n - 1, true);
            }
          }
        } else {
          wait(&s_qfull[0], n_q0++ & 1);
          tc_fence_after();
          for (int i = 0; ok && i < n + 2; ++i) {
            if (i >= 2) {
              const uint32_t v = st;
              if (!wait(&s_full[st], ph)) break;
              advance();
              if (i & 1) output(1, v, i < 4, true, i >= n); else output(0, v, i < 4, true, i >= n);
              if (!ok) break;
            }
            if (i < n) {
              const uint32_t k = st;
              if (!wait(&s_full[st], ph)) break;
              advance();
              scores(i & 1, 0, k, i == n - 1, true);
            }
          }
        }
      }
    } else if (warp == 3) {
      // ---- the pieces of work
      Walk<kCached> walk;
      walk.start(a);
      for (bool more = true; more; ++n_item) {
        Item it;
        more = walk.next(a, it);
        if (!more) it.rows = 0;
        if (!__all_sync(~0u, wait_bar(&s_iempty[n_item & 1], ((n_item >> 1) & 1) ^ 1, flags, a.limit_ns))) break;
        if (lane == 0) {
          s_item[n_item & 1] = it;
          mbar_arrive(smem_u32(&s_ifull[n_item & 1]));
        }
        __syncwarp();
      }
      walk.finish(a);
    }
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (s_flags[0]) timeout_record_and_drain(a.status);
  __syncthreads();
  if (warp == 0) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512) : "memory");
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
    // the register split draws on what the block was launched with: with fewer the larger share would never come
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
  const int tokens = 128 % a.g ? 1 : 128 / a.g, heads = 128 % a.g ? 1 : a.g;      // of a tile; else the map is not used
  EncodeTiledFn fn = encode_fn();
  if (!fn) return PCOMOE_ERR_CUDA;
  cuuint64_t dims[3] = {(cuuint64_t)D, (cuuint64_t)a.hq, (cuuint64_t)a.T}, strides[2] = {(cuuint64_t)D * 2, (cuuint64_t)a.q_stride * 2};
  cuuint32_t box[3] = {BK, (cuuint32_t)heads, (cuuint32_t)tokens}, estr[3] = {1, 1, 1};
  if (fn(&m.q, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void *>(a.q), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
         CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS)
    return PCOMOE_ERR_CUDA;
  if (a.table) {
    const uint64_t rows = (uint64_t)a.pages * a.hkv * a.page;
    if (rows > INT32_MAX) return PCOMOE_ERR_UNSUPPORTED;                 // row numbers of a TMA copy are 32 bits
    const uint32_t box = std::min(BN, a.page);
    if (!make_rows_map(&m.k, a.k, rows, D, D, box) || !make_rows_map(&m.v, a.v, rows, D, D, box)) return PCOMOE_ERR_CUDA;
    const pcomoe_status r = D == 64 ? run<64, true>(m, a, sms, st) : run<128, true>(m, a, sms, st);
    return r == PCOMOE_OK ? launch_attn_join(a, D, PCOMOE_BF16, BM, sms, st) : r;
  }
  if (!make_rows_map(&m.k, a.k, a.T, (uint64_t)a.hkv * D, a.k_stride, BN) || !make_rows_map(&m.v, a.v, a.T, (uint64_t)a.hkv * D, a.v_stride, BN))
    return PCOMOE_ERR_CUDA;
  const int64_t tiles = ((int64_t)a.T * a.g / 128 + std::min(a.n_seqs, a.T)) * a.hkv;      // no more than that
  if (tiles > INT32_MAX) return PCOMOE_ERR_SHAPE;
  const unsigned grid = (unsigned)std::min<int64_t>(tiles, sms);
  return D == 64 ? run<64, false>(m, a, grid, st) : run<128, false>(m, a, grid, st);
}

}  // namespace pcomoe
