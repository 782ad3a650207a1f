// What the attention kernels share: the arguments, the way work is cut, masks, the joining of partial results.
//
// Rows.  The query heads that share a kv head are packed into the rows of a tile: row r of (sequence, kv head) is token
// r / g, head r % g of the group, so a tile reads every key and value once for all of them, whatever g is.
//
// Work over a cache.  A tile's blocks of keys are numbered through: (sequence, kv head, tile, block), blocks fastest.  Every
// block (CTA) of the grid takes an equal, contiguous share of that line, found on the device from the lengths alone (no
// host copy of them, no plan step), so ragged batches are balanced to one block of keys.  A tile cut by a share's
// border leaves partial sums, which a second kernel joins in order of the shares.  (Joined by the CTA that finished last
// instead, the sums of a 192-row tile took 13 us of one SM's time, and fences and counters another 3.)
#pragma once
#include "tc_ptx.cuh"

namespace pcomoe {

struct AttnArgs {
  int32_t T, n_seqs, hq, hkv, g, sms;
  float scale_log2;                     // scale * log2(e)
  const int32_t *cu, *seqs;
  const void *q, *k, *v;                // k, v: packed rows, or the layer's page pools
  int64_t q_stride, k_stride, v_stride, out_stride;      // elements
  void *out;
  float *lse;
  const uint32_t *mask;
  int32_t words;
  const int32_t *len, *table;           // the cache's lengths and page tables; NULL: packed prompts
  int32_t pages, page, page_shift, max_seqs, max_pages;
  int32_t *status, *counters;           // counters: next piece of the prompts, CTAs done; zero between calls
  struct JoinRec *recs;                 // one per CTA of the grid
  float *part, *part_ml;                // [2 * grid][rows][D] and [2 * grid][rows][2]
  uint64_t limit_ns;
};

// The tile that a CTA of the grid began and did not finish; n_parts = 0: none.
struct JoinRec {
  int32_t q0, n, kvh, tile, n_parts;
};
constexpr int kAttnMaxCtas = 4096;
constexpr int kAttnMaxSeqs = 65535;
constexpr int kAttnMaxWords = 8;
constexpr float kLn2f = 0.6931471805599453f;

pcomoe_status launch_attn_join(const AttnArgs &a, int head_dim, int dtype, int rows, int ctas, cudaStream_t st);
pcomoe_status launch_attn_tc(const AttnArgs &a, int head_dim, int sms, cudaStream_t st);
size_t attn_tc_part_rows(int sms);
pcomoe_status launch_attn_few(const AttnArgs &a, int head_dim, int sms, cudaStream_t st);
size_t attn_few_part_rows(int sms);
pcomoe_status launch_attn_simt(const AttnArgs &a, int head_dim, int sms, cudaStream_t st);
size_t attn_simt_part_rows(int sms);

#ifdef __CUDACC__
namespace {

__device__ __forceinline__ float ex2f(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// 16 bytes to shared memory; zeros where there is nothing to copy
__device__ __forceinline__ void copy16(uint32_t dst, const void *src, bool there) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(there ? 16 : 0) : "memory");
}

// Weight of a partial sum l over the maximum m when the whole's is `to` (finite): NaN where l is (scores that are NaN raise no
// maximum), and kNoPart for a part in which the row saw nothing, whose sums may hold anything.  A part's largest weight is
// 2^-8 or more, so l is 0 for no other; a part that the row saw counts even with a weight that is 0 in fp32, as a single
// key does: 0 times a NaN is NaN, wherever the cut falls.
constexpr float kNoPart = -1.f;
__device__ __forceinline__ float part_weight(float m, float l, float to) { return l == 0.f ? kNoPart : l == l ? ex2f(m - to) : l; }

struct Seq {
  int q0, n;            // first packed row and their number
  int len, base;        // keys; those before `base` are seen by every row, the others by mask or order
  int id;               // sequence in the cache
};

template <bool kCached>
__device__ __forceinline__ Seq load_seq(const AttnArgs &a, int s) {
  Seq r;
  r.q0 = a.cu[s];
  const int e = a.cu[s + 1];
  r.n = e - r.q0;
  r.id = 0;
  if (r.q0 < 0 || r.n < 0 || e > a.T) {
    atomicCAS(a.status, 0, (int)PCOMOE_ERR_INDEX);
    r.q0 = r.n = r.len = r.base = 0;
    return r;
  }
  if (!kCached) {
    r.len = r.n;
    r.base = 0;
    return r;
  }
  r.id = a.seqs[s];
  const bool known = r.id >= 0 && r.id < a.max_seqs;
  const int len = known ? a.len[r.id] : 0;
  if (r.n > 0 && (!known || len < r.n || ((len - 1) >> a.page_shift) >= a.max_pages || (a.mask && r.n > 32 * a.words))) {
    atomicCAS(a.status, 0, (int)PCOMOE_ERR_INDEX);
    r.len = r.base = r.id = 0;           // its rows see nothing
    return r;
  }
  r.len = len;
  r.base = len - r.n;
  return r;
}

// Blocks of BN keys that the rows before `row_end` of a sequence look at; at least one, so that rows that see nothing are
// still written.
template <bool kCached, int BN>
__device__ __forceinline__ int key_blocks(const AttnArgs &a, const Seq &s, int row_end) {
  int keys = s.len;
  if (!kCached) keys = min(keys, (min(row_end, s.n * a.g) - 1) / a.g + 1);
  return max(1, (keys + BN - 1) / BN);
}

// Which of the 32 positions from p0 on row `tok` of a sequence sees, as bits.
template <bool kCached>
__device__ __forceinline__ uint32_t seen_bits(const AttnArgs &a, const Seq &s, int tok, int p0) {
  const int m0 = p0 - s.base;
  if (m0 + 32 <= 0) return ~0u;                          // all before the queries' own
  uint32_t bits;
  if (kCached && a.mask) {
    const uint32_t *row = a.mask + (int64_t)(s.q0 + tok) * a.words;
    const int w = m0 >> 5, sh = m0 & 31;                 // floor
    const uint32_t lo = w >= 0 && w < a.words ? row[w] : 0u, hi = w + 1 < a.words ? row[w + 1] : 0u;
    bits = sh ? (lo >> sh) | (hi << (32 - sh)) : lo;
    const int rest = s.n - m0;                           // drafts from here on
    if (rest < 32) bits &= rest > 0 ? (1u << rest) - 1u : 0u;
  } else {
    const int rest = tok + 1 - m0;
    bits = rest >= 32 ? ~0u : rest > 0 ? (1u << rest) - 1u : 0u;
  }
  if (m0 < 0) bits |= (1u << -m0) - 1u;                  // -m0 < 32
  const int left = s.len - p0;
  if (left < 32) bits &= left > 0 ? (1u << left) - 1u : 0u;
  return bits;
}

// A CTA's share of the line of blocks, and its walk along it.  All of it is the same in every thread of a warp.  A tile
// counts for its blocks and kExtra more, which stand for what a piece of work costs besides (a sequence of one block of keys
// is no cheaper to begin than one of a thousand): without them the CTA that met the shortest sequences finished last.
// (A share is never less than one block, so that short sequences still spread over the GPU: with shares of four blocks and
// more a draft tree over 100 to 400 keys took 20 us instead of 14.)  Where every tile can have a CTA of its own and none
// is longer than kFlat blocks, tiles are not cut: parts would cost more to write and join than they save.
template <int BM, int BN, int kExtra, int kFlat>
struct CacheWalk {
  uint32_t at, end;     // units of this share still to do
  uint32_t share;
  uint32_t seq_at;      // number of the current sequence's first unit
  int s;                // sequence
  Seq seq;
  int tiles, blocks;    // of the current sequence: row tiles, blocks of a tile
  bool flat;            // a CTA per tile: a tile is one unit

  __device__ void measure(const AttnArgs &a) {
    seq = load_seq<true>(a, s);
    tiles = (seq.n * a.g + BM - 1) / BM;
    blocks = max(1, (seq.len + BN - 1) / BN);
  }
  __device__ uint32_t units() const { return flat ? 1u : (uint32_t)(blocks + kExtra); }
  __device__ uint64_t weight(const AttnArgs &a) const { return (uint64_t)((int64_t)tiles * a.hkv) * units(); }

  // One warp, all lanes.  An empty share gives no piece.
  __device__ void start(const AttnArgs &a, int cta, int ctas) {
    const int lane = threadIdx.x & 31;
    uint64_t total = 0;
    int own = 0, longest = 0;                              // tiles, up to one more than CTAs; blocks of the longest
    begun.n_parts = 0;
    flat = false;
    for (int s0 = 0; s0 < a.n_seqs; s0 += 32) {
      s = s0 + lane;
      uint64_t w = 0;
      if (s < a.n_seqs) {
        measure(a);
        w = weight(a);
        own = (int)min((int64_t)ctas + 1, own + (int64_t)tiles * a.hkv);
        longest = max(longest, tiles ? blocks : 0);
      }
#pragma unroll
      for (int o = 16; o; o >>= 1) w += __shfl_xor_sync(~0u, w, o);
      total += w;
    }
    const uint32_t all = __reduce_add_sync(~0u, (unsigned)own);
    flat = all <= (uint32_t)ctas && __reduce_max_sync(~0u, (unsigned)longest) <= kFlat;
    if (flat) total = all;
    at = end = 0;
    if (total > (uint64_t)INT32_MAX) {                     // more than any memory holds, unless a sequence is named very often
      atomicCAS(a.status, 0, (int)PCOMOE_ERR_SHAPE);
      return;
    }
    share = flat ? 1 : max(((uint32_t)total + ctas - 1) / ctas, (uint32_t)(1 + kExtra));
    if ((uint64_t)cta * share >= total) return;
    at = cta * share;
    end = min(at + share, (uint32_t)total);
    uint32_t before = 0;
    for (int s0 = 0; s0 < a.n_seqs; s0 += 32) {
      s = s0 + lane;
      uint32_t w = 0;
      if (s < a.n_seqs) {
        if (a.n_seqs > 32) measure(a);                     // else it is what the lane has
        w = (uint32_t)weight(a);
      }
      uint32_t upto = w;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const uint32_t y = __shfl_up_sync(~0u, upto, o);
        if (lane >= o) upto += y;
      }
      const uint32_t hit = __ballot_sync(~0u, before + upto > at);
      if (hit) {
        const int l = __ffs(hit) - 1;
        s = s0 + l;
        seq_at = before + __shfl_sync(~0u, upto - w, l);
        if (a.n_seqs <= 32) {                              // what lane l has read already
          seq.q0 = __shfl_sync(~0u, seq.q0, l);
          seq.n = __shfl_sync(~0u, seq.n, l);
          seq.len = __shfl_sync(~0u, seq.len, l);
          seq.base = __shfl_sync(~0u, seq.base, l);
          seq.id = __shfl_sync(~0u, seq.id, l);
          tiles = __shfl_sync(~0u, tiles, l);
          blocks = __shfl_sync(~0u, blocks, l);
          return;
        }
        break;
      }
      before += __shfl_sync(~0u, upto, 31);
    }
    measure(a);
  }

  struct Piece {
    int kvh, tile, b0, b1;     // blocks [b0, b1) of a tile of `blocks`
    bool whole;
  };

  __device__ bool next(const AttnArgs &a, Piece &p) {
    while (at < end) {
      while (at >= seq_at + (uint32_t)(tiles * a.hkv) * units()) {
        seq_at += (uint32_t)(tiles * a.hkv) * units();
        ++s;
        measure(a);
      }
      const uint32_t t = (at - seq_at) / units(), tile_at = seq_at + t * units();
      if (flat) {
        at = tile_at + 1;
        p = {(int)t / tiles, (int)t % tiles, 0, blocks, true};
        return true;
      }
      const uint32_t upto = min(end, tile_at + units());
      p.b0 = max((int)(at - tile_at) - kExtra, 0);
      p.b1 = (int)(upto - tile_at) - kExtra;
      at = upto;
      if (p.b1 <= p.b0) continue;                          // of this tile only what stands for its cost
      p.kvh = (int)t / tiles;
      p.tile = (int)t - p.kvh * tiles;
      p.whole = p.b0 == 0 && p.b1 == blocks;
      if (p.b0 == 0 && !p.whole) {                         // then it is the share's last piece
        const uint32_t first = tile_at + kExtra;
        begun = {seq.q0, seq.n, p.kvh, p.tile, (int)((first + blocks - 1) / share - first / share) + 1};
      }
      return true;
    }
    return false;
  }

  JoinRec begun;
  __device__ void record(const AttnArgs &a, int cta) const { a.recs[cta] = begun; }      // one thread, at the end
};

// Place of a partial result: a CTA leaves at most two, of the tile that its share begins inside and of the one that it
// begins itself and does not finish.
__device__ __forceinline__ int part_slot(int cta, bool begins_tile) { return 2 * cta + (begins_tile ? 1 : 0); }

template <typename T> __device__ __forceinline__ void store4(T *p, float4 v);
template <> __device__ __forceinline__ void store4<float>(float *p, float4 v) { *(float4 *)p = v; }
template <> __device__ __forceinline__ void store4<__nv_bfloat16>(__nv_bfloat16 *p, float4 v) {
  uint2 u;
  *(__nv_bfloat162 *)&u.x = __floats2bfloat162_rn(v.x, v.y);
  *(__nv_bfloat162 *)&u.y = __floats2bfloat162_rn(v.z, v.w);
  *(uint2 *)p = u;
}

// Row of a page pool ([page][head][place in the page]) that holds position p.
__device__ __forceinline__ int64_t page_row(const AttnArgs &a, const int32_t *table, int kvh, int p) {
  int page = table[p >> a.page_shift];
  if ((unsigned)page >= (unsigned)a.pages) {
    atomicCAS(a.status, 0, (int)PCOMOE_ERR_INDEX);
    page = 0;
  }
  return ((int64_t)page * a.hkv + kvh) * a.page + (p & (a.page - 1));
}

// Place of position p's row of K or V, in elements; bf16 kernels.
template <int D, bool kCached>
__device__ __forceinline__ int64_t row_at(const AttnArgs &a, const Seq &s, int kvh, int p, int64_t stride) {
  return kCached ? page_row(a, a.table + (int64_t)s.id * a.max_pages, kvh, p) * D : (int64_t)(s.q0 + p) * stride + kvh * D;
}

// Rows whose sums are not finite.  The products of a tile take every row through every value, with weight 0 where the row does not
// see it, and 0 times a NaN or an infinity is NaN.  So such a row is right as it stands, unless one of the values that it does
// not see is NaN or infinite: only then it is formed again (plain_rows).  Each lane asks for its own row, of token tok; p0 to
// p1 are the positions that went into the sums, and every row of the warp sees those before `from`.  A warp.
template <int D, bool kCached>
__device__ __forceinline__ bool met_unseen(const AttnArgs &a, const Seq &s, int kvh, int tok, int p0, int p1, int from, bool asks) {
  constexpr int C = D / 8, P = 32 / C;                   // lanes of a row, rows side by side
  const int lane = threadIdx.x & 31;
  bool met = false;
  p1 = min(p1, s.len);
  for (int g = max(p0, from) & ~31; g < p1; g += 32) {
    uint32_t odd = 0;                                    // which of the 32 positions hold such a value
#pragma unroll 4
    for (int k = 0; k < 32; k += P) {
      const int p = g + k + lane / C;
      uint4 x = make_uint4(0, 0, 0, 0);
      if (p < p1) x = *(const uint4 *)((const __nv_bfloat16 *)a.v + row_at<D, kCached>(a, s, kvh, p, a.v_stride) + (lane % C) * 8);
      auto not_finite = [](uint32_t u) { return (u & 0x7f80u) == 0x7f80u || (u & 0x7f800000u) == 0x7f800000u; };
      const uint32_t b = __ballot_sync(~0u, not_finite(x.x) || not_finite(x.y) || not_finite(x.z) || not_finite(x.w));
#pragma unroll
      for (int j = 0; j < P; ++j)
        if ((b >> (j * C)) & ((1u << C) - 1u)) odd |= 1u << (k + j);
    }
    if (odd && asks) met |= (odd & ~seen_bits<kCached>(a, s, tok, g)) != 0;
    if (__all_sync(~0u, met || !asks)) break;
  }
  return met;
}

// bf16 rows without the tensor cores, by a warp: the rows r0 + i of bits i of `todo`, four at a time, over the positions [p0, p1)
// that each of them sees, 32 at a time: a lane per key for the scores, and every lane its columns of the head for the sums.
// Once all columns of a row are NaN nothing can change them, and the maximum and sum of the first pass, which come from the
// scores alone, stay.  Rare, so plain: in a prompt of 16384 tokens (16 heads of 128, 0.94 ms) an infinity at row 12543, the last
// of its tile, sends 255 rows of every head here and makes it 30 ms; one at row 0, which every row sees, sends none (1.13 ms).
template <int D, int BM, bool kCached>
__device__ __forceinline__ void plain_rows(const AttnArgs &a, const Seq &s, int kvh, int row0, int r0, uint32_t todo, int p0, int p1, bool whole, int slot) {
  constexpr int N = D / 32, U = 8, R = 4;                 // columns of a lane; values under way; rows at a time
  const int lane = threadIdx.x & 31;
  p1 = min(p1, s.len);
  while (todo) {
    int r[R];                                             // the last one again where there are fewer
    int n = 0;
#pragma unroll
    for (int i = 0; i < R; ++i) {
      r[i] = todo ? r0 + __ffs(todo) - 1 : r[max(i - 1, 0)];
      n += todo != 0;
      todo &= todo - 1;
    }
    float o[R][N], m[R], l[R];
#pragma unroll
    for (int i = 0; i < R; ++i) {
      m[i] = -INFINITY;
      l[i] = 0.f;
#pragma unroll
      for (int k = 0; k < N; ++k) o[i][k] = 0.f;
    }
    auto q_row = [&](int i) {
      const int row = row0 + r[i], tok = row / a.g;
      return (const uint4 *)((const __nv_bfloat16 *)a.q + (int64_t)(s.q0 + tok) * a.q_stride + (kvh * a.g + row - tok * a.g) * D);
    };
    uint32_t lost = 0;                                    // rows whose columns are all NaN
    for (int g = p0; g < p1 && lost != (1u << R) - 1u; g += 32) {
      uint32_t bits[R], any = 0;
#pragma unroll
      for (int i = 0; i < R; ++i) any |= bits[i] = seen_bits<kCached>(a, s, (row0 + r[i]) / a.g, g);       // none past the end of the sequence
      const int p = g + lane;
      float x[R];
#pragma unroll
      for (int i = 0; i < R; ++i) x[i] = 0.f;
      int64_t v_at = 0;
      if ((any >> lane) & 1) {
        const uint4 *k = (const uint4 *)((const __nv_bfloat16 *)a.k + row_at<D, kCached>(a, s, kvh, p, a.k_stride));
        v_at = row_at<D, kCached>(a, s, kvh, p, a.v_stride);
#pragma unroll 1
        for (int c0 = 0; c0 < D / 8; c0 += 4) {
          uint4 y[4];
#pragma unroll
          for (int c = 0; c < 4; ++c) y[c] = k[c0 + c];
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            const uint32_t u[4] = {y[c].x, y[c].y, y[c].z, y[c].w};
#pragma unroll
            for (int i = 0; i < R; ++i) {
              const uint4 z = q_row(i)[c0 + c];
              const uint32_t w[4] = {z.x, z.y, z.z, z.w};
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                x[i] = fmaf(__uint_as_float(u[e] << 16), __uint_as_float(w[e] << 16), x[i]);
                x[i] = fmaf(__uint_as_float(u[e] & 0xffff0000u), __uint_as_float(w[e] & 0xffff0000u), x[i]);
              }
            }
          }
        }
      }
      __syncwarp();
#pragma unroll
      for (int i = 0; i < R; ++i) {
        x[i] = (bits[i] >> lane) & 1 ? x[i] * a.scale_log2 : -INFINITY;
        float mn = x[i];
#pragma unroll
        for (int h = 16; h; h >>= 1) mn = fmaxf(mn, __shfl_xor_sync(~0u, mn, h));
        mn = fmaxf(mn, m[i]);
        const float ms = mn == -INFINITY ? 0.f : mn, c = ex2f(m[i] - ms);
        x[i] = ex2f(x[i] - ms);                           // the weight
        float sum = x[i];
#pragma unroll
        for (int h = 16; h; h >>= 1) sum += __shfl_xor_sync(~0u, sum, h);
        l[i] = l[i] * c + sum;
        m[i] = mn;
#pragma unroll
        for (int k = 0; k < N; ++k) o[i][k] *= c;
      }
#pragma unroll 1
      for (int j0 = 0; j0 < 32; j0 += U) {
        uint32_t v[U][N / 2];
#pragma unroll
        for (int j = 0; j < U; ++j) {
          const int64_t at = __shfl_sync(~0u, v_at, j0 + j);
#pragma unroll
          for (int k = 0; k < N / 2; ++k)
            v[j][k] = (any >> (j0 + j)) & 1 ? ((const uint32_t *)((const __nv_bfloat16 *)a.v + at + lane * N))[k] : 0u;
        }
#pragma unroll
        for (int j = 0; j < U; ++j)
#pragma unroll
          for (int i = 0; i < R; ++i) {
            const float w = __shfl_sync(~0u, x[i], j0 + j);
            if ((bits[i] >> (j0 + j)) & 1)
#pragma unroll
              for (int k = 0; k < N / 2; ++k) {
                o[i][2 * k] = fmaf(w, __uint_as_float(v[j][k] << 16), o[i][2 * k]);
                o[i][2 * k + 1] = fmaf(w, __uint_as_float(v[j][k] & 0xffff0000u), o[i][2 * k + 1]);
              }
          }
      }
#pragma unroll
      for (int i = 0; i < R; ++i) {
        bool all = true;
#pragma unroll
        for (int k = 0; k < N; ++k) all &= o[i][k] != o[i][k];
        lost |= (uint32_t)__all_sync(~0u, all) << i;
      }
    }
#pragma unroll
    for (int i = 0; i < R; ++i) {
      if (i >= n) continue;
      const bool keep = (lost >> i) & 1;                  // what the first pass left of the maximum and sum
      if (whole) {
        const int row = row0 + r[i], tok = row / a.g, head = kvh * a.g + row - tok * a.g;
        const int64_t t = s.q0 + tok;
        const float inv = l[i] == 0.f ? 0.f : 1.f / l[i];
#pragma unroll
        for (int k = 0; k < N; ++k) ((__nv_bfloat16 *)a.out)[t * a.out_stride + head * D + lane * N + k] = __float2bfloat16_rn(o[i][k] * inv);
        if (lane == 0 && a.lse && !keep) a.lse[t * a.hq + head] = l[i] == 0.f ? -INFINITY : m[i] * kLn2f + logf(l[i]);
      } else {
        const int64_t at = (int64_t)slot * BM + r[i];
#pragma unroll
        for (int k = 0; k < N; ++k) a.part[at * D + lane * N + k] = o[i][k];
        if (lane == 0 && !keep) *((float2 *)a.part_ml + at) = make_float2(m[i], l[i]);
      }
    }
  }
}

}  // namespace
#endif

}  // namespace pcomoe
