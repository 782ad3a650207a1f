// Norm and rotation of the heads of queries and keys, and keys and values on their way into the paged cache, in one pass.
//
// Mathematics.  A head x of D elements: y = x w / sqrt(mean x^2 + eps), where it has a weight w; then each of the first rot / 2
// pairs (a, b) of y becomes (a cos t - b sin t, a sin t + b cos t), t = position * inv_freq.  The angle is formed in turns in
// 64 bits (position * inv_freq / 2 pi less its nearest integer), since in 32 a position of 10^5 leaves an error of 0.01
// radians; sine and cosine of the rest are taken in 32.  Sums and products are fp32, and the result is rounded once.
//
// What bounds it: HBM, every row read and written once (with few rows the latency of one chain position -> angle and list ->
// length -> page).  D / 16 lanes hold a head, two 16-byte pieces each, chosen so that both elements of a pair lie in one lane
// and a lane's angles are the same for all heads of its token: a warp forms a token's angles once and walks over its
// heads, the next heads' loads under way.  Measured, 16384 tokens of 16 + 16 + 16 heads of 128 into packed rows and pages: 86 us, 5.5
// TB/s read and written, 0.85 of a plain copy's rate.  (Four heads' loads ahead and half the warps per SM took 111 us, no load
// ahead and 32 warps 94, packed two-element arithmetic 93.)  32 decode rows of 32 + 8 + 8 heads: 4 us.
#include <algorithm>
#include <cmath>

#include "cache.cuh"

namespace pcomoe {
namespace {

constexpr int kWarps = 2;

struct RotateArgs {
  int32_t T, hq, hkv, rot, neighbours;
  int32_t slots, per, parts;              // heads of a token; steps of a warp; warps of a token
  float eps;
  const int32_t *position;
  const double *inv_freq;
  const void *qw, *kw;
  const char *q, *k, *v;
  char *qo, *ko;                          // ko may be NULL
  int64_t qs, ks, vs, qos, kos;           // bytes from row to row
  const int32_t *seqs, *cu;               // cu NULL: no cache
  int32_t n;
  CacheDev c;
  int64_t layer_at;                       // bytes before the layer's pool
  CacheHeader *head;
};

template <typename T> struct Eight;       // 8 elements, as they lie in memory
template <> struct Eight<__nv_bfloat16> {
  uint4 x;
  __device__ __forceinline__ void load(const char *p) { x = *(const uint4 *)p; }
  __device__ __forceinline__ void store(char *p) const { *(uint4 *)p = x; }
  __device__ __forceinline__ void get(float *f) const {
    const uint32_t u[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) { f[2 * i] = __uint_as_float(u[i] << 16); f[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u); }
  }
  __device__ __forceinline__ void set(const float *f) {
    uint32_t u[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const __nv_bfloat162 v = __floats2bfloat162_rn(f[2 * i], f[2 * i + 1]);
      u[i] = *(const uint32_t *)&v;
    }
    x = make_uint4(u[0], u[1], u[2], u[3]);
  }
};
template <> struct Eight<float> {
  float4 x, y;
  __device__ __forceinline__ void load(const char *p) { x = ((const float4 *)p)[0]; y = ((const float4 *)p)[1]; }
  __device__ __forceinline__ void store(char *p) const { ((float4 *)p)[0] = x; ((float4 *)p)[1] = y; }
  __device__ __forceinline__ void get(float *f) const {
    f[0] = x.x; f[1] = x.y; f[2] = x.z; f[3] = x.w; f[4] = y.x; f[5] = y.y; f[6] = y.z; f[7] = y.w;
  }
  __device__ __forceinline__ void set(const float *f) { x = make_float4(f[0], f[1], f[2], f[3]); y = make_float4(f[4], f[5], f[6], f[7]); }
};

// The last entry of cu[0 .. n) at or before t, by a warp: 32 places looked at side by side.
__device__ __forceinline__ int sequence_of(const int32_t *cu, int n, int t) {
  const int lane = threadIdx.x & 31;
  int lo = 0, hi = n;
  while (hi - lo > 1) {
    const int step = (hi - lo + 31) / 32, i = lo + (lane + 1) * step;
    const int k = __popc(__ballot_sync(~0u, i < hi && cu[min(i, hi)] <= t));
    hi = min(lo + (k + 1) * step, hi);
    lo += k * step;
  }
  return lo;
}

// Bytes from the start of a layer's pool to the row of head 0 that packed row t belongs in; -1: there is none.  A warp.
__device__ __forceinline__ int64_t place_of(const RotateArgs &a, int t) {
  const int s = sequence_of(a.cu, a.n, t), from = a.cu[s], to = a.cu[s + 1], id = a.seqs[s];
  bool ok = from <= t && t < to && id >= 0 && id < a.c.max_seqs;
  int page = -1, slot = 0;
  if (ok) {
    const int p = a.c.len[id] - (to - t);
    ok = p >= 0 && (p >> a.c.shift) < a.c.max_pages;
    if (ok) {
      page = a.c.table[(int64_t)id * a.c.max_pages + (p >> a.c.shift)];
      slot = p & (a.c.page - 1);
      ok = page >= 0 && page < a.c.pages && a.c.ref[page] == 1;
    }
  }
  if (!ok) {
    flag(a.head, PCOMOE_ERR_INDEX);
    return -1;
  }
  return (int64_t)page * a.c.page_bytes + (int64_t)slot * a.c.chunks * 16;
}

template <typename T, int D>
__global__ void __launch_bounds__(32 * kWarps, 12) rotate_kernel(const __grid_constant__ RotateArgs a) {
  constexpr int G = D / 16, kHeads = 32 / G, E = (int)sizeof(T);
  pdl_grid_wait();
  const int lane = threadIdx.x & 31, l = lane % G, sub = lane / G;
  const int unit = blockIdx.x * kWarps + (threadIdx.x >> 5);
  const int t = unit / a.parts, part = unit - t * a.parts;
  if (a.cu && unit == 0 && lane == 0 && (a.cu[a.n] > a.T || a.cu[0] < 0)) flag(a.head, PCOMOE_ERR_INDEX);
  if (t >= a.T || (a.cu && (t < a.cu[0] || t >= a.cu[a.n]))) return;
  const int s0 = part * a.per * kHeads, s1 = min(s0 + a.per * kHeads, a.slots);       // this warp's heads
  const int heads = a.hq + a.hkv;

  // the two pieces of a head: elements e0.. and e1..
  const bool turns = l < a.rot / 16;
  const bool halves = turns && !a.neighbours;
  const int e0 = halves ? 8 * l : 16 * l, e1 = halves ? 8 * l + a.rot / 2 : 16 * l + 8;
  auto source = [&](int s) {
    return s < a.hq ? a.q + t * a.qs + (int64_t)s * D * E : s < heads ? a.k + t * a.ks + (int64_t)(s - a.hq) * D * E : a.v + t * a.vs + (int64_t)(s - heads) * D * E;
  };
  Eight<T> x0, x1, n0, n1;                                 // a head's pieces, and the next one's on their way
  auto fetch = [&](int h) {
    if (h < s1) {
      const char *p = source(h);
      n0.load(p + e0 * E);
      n1.load(p + e1 * E);
    }
  };
  auto send = [&](char *to) {
    x0.store(to + e0 * E);
    x1.store(to + e1 * E);
  };
  fetch(s0 + sub);
  const int64_t place = a.cu && s1 > a.hq ? place_of(a, t) : -1;
  float cs[8], sn[8];
  if (turns && s0 < heads) {
    const double p = (double)a.position[t] * 0.15915494309189533577;                 // 1 / 2 pi
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const double y = p * a.inv_freq[8 * l + i];
      sincospif(2.f * (float)(y - rint(y)), &sn[i], &cs[i]);
    }
  }
  for (int s = s0; s < s1; s += kHeads) {
    const int h = s + sub;
    x0 = n0;
    x1 = n1;
    fetch(h + kHeads);
    if (s < heads) {                                       // not values alone
      const char *wp = (const char *)(h < a.hq ? a.qw : a.kw);
      float f[16];
      x0.get(f);
      x1.get(f + 8);
      float ss = 0.f;
#pragma unroll
      for (int k = 0; k < 16; ++k) ss = fmaf(f[k], f[k], ss);
#pragma unroll
      for (int o = G / 2; o; o >>= 1) ss += __shfl_xor_sync(~0u, ss, o);
      if (h < s1 && h < heads) {
        if (wp) {
          const float inv = rsqrtf(ss * (1.f / D) + a.eps);
          Eight<T> w0, w1;
          float w[16];
          w0.load(wp + e0 * E);
          w1.load(wp + e1 * E);
          w0.get(w);
          w1.get(w + 8);
#pragma unroll
          for (int k = 0; k < 16; ++k) f[k] *= inv * w[k];
        }
        if (turns) {
          if (a.neighbours) {
#pragma unroll
            for (int k = 0; k < 8; ++k) {
              const float u = f[2 * k], v = f[2 * k + 1];
              f[2 * k] = u * cs[k] - v * sn[k];
              f[2 * k + 1] = u * sn[k] + v * cs[k];
            }
          } else {
#pragma unroll
            for (int k = 0; k < 8; ++k) {
              const float u = f[k], v = f[k + 8];
              f[k] = u * cs[k] - v * sn[k];
              f[k + 8] = u * sn[k] + v * cs[k];
            }
          }
        }
        if (wp || turns) {
          x0.set(f);
          x1.set(f + 8);
        }
      }
    }
    if (h < s1) {
      const int kv = h - a.hq, head = kv < a.hkv ? kv : kv - a.hkv;
      if (kv < 0) send(a.qo + t * a.qos + (int64_t)h * D * E);
      else if (a.ko && kv < a.hkv) send(a.ko + t * a.kos + (int64_t)kv * D * E);
      if (kv >= 0 && place >= 0) send((kv < a.hkv ? a.c.k : a.c.v) + a.layer_at + place + (int64_t)head * a.c.page * D * E);
    }
  }
}

pcomoe_status check_config(const pcomoe_rotate_config *c) {
  if (!c || c->struct_size != (int32_t)sizeof(pcomoe_rotate_config)) return PCOMOE_ERR_INVALID_ARG;
  if (c->q_heads <= 0 || c->kv_heads <= 0 || c->head_dim <= 0 || c->rot_dim < 0 || c->rot_dim > c->head_dim || !(c->eps >= 0.f) || !std::isfinite(c->eps) ||
      (c->pairs != PCOMOE_ROTATE_HALVES && c->pairs != PCOMOE_ROTATE_NEIGHBOURS))
    return PCOMOE_ERR_INVALID_ARG;
  if (c->dtype != PCOMOE_BF16 && c->dtype != PCOMOE_FP32) return PCOMOE_ERR_INVALID_ARG;
  if ((c->head_dim != 64 && c->head_dim != 128) || c->rot_dim % 16) return PCOMOE_ERR_UNSUPPORTED;
  if (c->q_heads > 4096 || c->kv_heads > 4096) return PCOMOE_ERR_SHAPE;
  return PCOMOE_OK;
}

// What both calls check and set: rows of q and k, their outputs (ko may be NULL where there is a cache), weights, angles.
pcomoe_status fill(RotateArgs &a, const pcomoe_rotate_config *c, int32_t T, const int32_t *position, const double *inv_freq, const void *qw, const void *kw,
                   const void *q, int64_t qs, const void *k, int64_t ks, void *qo, int64_t qos, void *ko, int64_t kos) {
  const int64_t e = (int64_t)dtype_size(c->dtype), qrow = (int64_t)c->q_heads * c->head_dim, krow = (int64_t)c->kv_heads * c->head_dim;
  if (!q || !k || !qo || (c->rot_dim > 0 && (!position || !inv_freq))) return PCOMOE_ERR_INVALID_ARG;
  if (qs < qrow || qos < qrow || ks < krow || (ko && kos < krow)) return PCOMOE_ERR_INVALID_ARG;
  if (((uintptr_t)q | (uintptr_t)k | (uintptr_t)qo | (uintptr_t)ko | (uintptr_t)qw | (uintptr_t)kw) & 15) return PCOMOE_ERR_UNSUPPORTED;
  if ((qs * e) % 16 || (ks * e) % 16 || (qos * e) % 16 || (ko && (kos * e) % 16) || (uintptr_t)inv_freq % 8) return PCOMOE_ERR_UNSUPPORTED;
  a = RotateArgs{};
  a.T = T; a.hq = c->q_heads; a.hkv = c->kv_heads; a.rot = c->rot_dim; a.neighbours = c->pairs == PCOMOE_ROTATE_NEIGHBOURS;
  a.eps = c->eps;
  a.position = position; a.inv_freq = inv_freq; a.qw = qw; a.kw = kw;
  a.q = (const char *)q; a.k = (const char *)k; a.qo = (char *)qo; a.ko = (char *)ko;
  a.qs = qs * e; a.ks = ks * e; a.qos = qos * e; a.kos = kos * e;
  return PCOMOE_OK;
}

template <typename T, int D>
pcomoe_status run(RotateArgs &a, cudaStream_t st) {
  int sms;
  const pcomoe_status s = current_sms(&sms);
  if (s != PCOMOE_OK) return s;
  constexpr int kHeads = 512 / D;                        // of a warp's step
  a.slots = a.hq + a.hkv * (a.cu ? 2 : 1);
  const int steps = (a.slots + kHeads - 1) / kHeads;
  // One step per warp until there are 32 warps for every SM, then more: a warp's angles serve all its steps.
  a.per = (int)std::min<int64_t>(steps, std::max<int64_t>(1, (int64_t)a.T * steps / ((int64_t)sms * 32)));
  a.parts = (steps + a.per - 1) / a.per;
  const int64_t units = (int64_t)a.T * a.parts;
  if (units > INT32_MAX - kWarps) return PCOMOE_ERR_SHAPE;
  PCOMOE_CUDA_TRY(launch_pdl(rotate_kernel<T, D>, dim3((unsigned)((units + kWarps - 1) / kWarps)), dim3(32 * kWarps), 0, st, a));
  count_launch();
  return PCOMOE_OK;
}

pcomoe_status run(RotateArgs &a, const pcomoe_rotate_config *c, cudaStream_t st) {
  if (c->dtype == PCOMOE_BF16) return c->head_dim == 64 ? run<__nv_bfloat16, 64>(a, st) : run<__nv_bfloat16, 128>(a, st);
  return c->head_dim == 64 ? run<float, 64>(a, st) : run<float, 128>(a, st);
}

}  // namespace
}  // namespace pcomoe

using namespace pcomoe;

extern "C" {

pcomoe_status pcomoe_heads_rotate(const pcomoe_rotate_config *cfg, int32_t T, const int32_t *d_position, const double *d_inv_freq, const void *d_q_weight,
                                  const void *d_k_weight, const void *d_q, int64_t q_stride, const void *d_k, int64_t k_stride, void *d_q_out,
                                  int64_t q_out_stride, void *d_k_out, int64_t k_out_stride, void *stream) {
  pcomoe_status st = check_config(cfg);
  if (st != PCOMOE_OK) return st;
  if (T < 0) return PCOMOE_ERR_SHAPE;
  if (T == 0) return PCOMOE_OK;
  if (!d_k_out) return PCOMOE_ERR_INVALID_ARG;
  RotateArgs a;
  st = fill(a, cfg, T, d_position, d_inv_freq, d_q_weight, d_k_weight, d_q, q_stride, d_k, k_stride, d_q_out, q_out_stride, d_k_out, k_out_stride);
  return st != PCOMOE_OK ? st : run(a, cfg, (cudaStream_t)stream);
}

pcomoe_status pcomoe_heads_rotate_cached(const pcomoe_rotate_config *cfg, const pcomoe_cache *cache, int32_t layer, int32_t T, int32_t n, const int32_t *d_seqs,
                                         const int32_t *d_cu_len, const int32_t *d_position, const double *d_inv_freq, const void *d_q_weight,
                                         const void *d_k_weight, const void *d_q, int64_t q_stride, const void *d_k, int64_t k_stride, const void *d_v,
                                         int64_t v_stride, void *d_q_out, int64_t q_out_stride, void *d_k_out, int64_t k_out_stride, void *d_workspace,
                                         size_t ws_bytes, void *stream) {
  pcomoe_status st = check_config(cfg);
  if (st != PCOMOE_OK) return st;
  if ((st = check_cache(cache)) != PCOMOE_OK) return st;
  if (cache->kv_heads != cfg->kv_heads || cache->head_dim != cfg->head_dim || cache->dtype != cfg->dtype || layer < 0 || layer >= cache->layers || n < 0)
    return PCOMOE_ERR_INVALID_ARG;
  if (T < 0 || n > cache->max_seqs) return PCOMOE_ERR_SHAPE;
  if (!d_workspace || ((uintptr_t)d_workspace & 255) || ws_bytes < 256) return PCOMOE_ERR_WORKSPACE;
  if (T == 0 || n == 0) return PCOMOE_OK;
  const int64_t e = (int64_t)dtype_size(cfg->dtype);
  if (!d_seqs || !d_cu_len || !d_v || v_stride < (int64_t)cfg->kv_heads * cfg->head_dim) return PCOMOE_ERR_INVALID_ARG;
  if (((uintptr_t)d_v & 15) || (v_stride * e) % 16) return PCOMOE_ERR_UNSUPPORTED;
  RotateArgs a;
  st = fill(a, cfg, T, d_position, d_inv_freq, d_q_weight, d_k_weight, d_q, q_stride, d_k, k_stride, d_q_out, q_out_stride, d_k_out, k_out_stride);
  if (st != PCOMOE_OK) return st;
  a.v = (const char *)d_v; a.vs = v_stride * e;
  a.seqs = d_seqs; a.cu = d_cu_len; a.n = n;
  a.c = cache_dev(cache);
  a.layer_at = (int64_t)layer * a.c.pages * a.c.page_bytes;
  a.head = (CacheHeader *)d_workspace;
  return run(a, cfg, (cudaStream_t)stream);
}

}  // extern "C"
