// What the kernels that read rows of logits share: the order of words, and rows taken in groups of 512 bytes, 16 bytes a lane.
#pragma once
#include <climits>

#include "common.cuh"

namespace pcomoe {
namespace {

constexpr int kMaxVocab = 1 << 20;
constexpr float kNone = -INFINITY;

// Order of floats as integers (-inf lowest of what occurs here, -0 as 0); kNoKey: nothing eligible.
__device__ __forceinline__ int key_of(float x) {
  const int b = __float_as_int(x + 0.f);
  return b ^ ((b >> 31) & 0x7fffffff);
}
__device__ __forceinline__ float of_key(int k) { return __int_as_float(k ^ ((k >> 31) & 0x7fffffff)); }
constexpr int kNoKey = (int)0x807fffff;                  // key_of(-inf)

// A word's place in the order: larger is better (value descending, then id ascending).
__device__ __forceinline__ unsigned long long place_of(int key, int id) { return ((unsigned long long)((uint32_t)key ^ 0x80000000u) << 32) | (uint32_t)~id; }
__device__ __forceinline__ int place_key(unsigned long long p) { return (int)((uint32_t)(p >> 32) ^ 0x80000000u); }
__device__ __forceinline__ int place_id(unsigned long long p) { return (int)~(uint32_t)p; }

__device__ __forceinline__ float eligible(float x) { return fabsf(x) < INFINITY ? x : kNone; }

__device__ __forceinline__ uint32_t max_bf16x2(uint32_t a, uint32_t b) {      // NaN loses
  uint32_t d;
  asm("max.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
  return d;
}

// The words of one 16-byte load.
template <typename T> struct Vec;
template <> struct Vec<__nv_bfloat16> {
  static constexpr int N = 8;
  static __device__ __forceinline__ float lo(uint32_t u) { return __uint_as_float(u << 16); }
  static __device__ __forceinline__ float hi(uint32_t u) { return __uint_as_float(u & 0xffff0000u); }
  static __device__ __forceinline__ void unpack(const uint4 &v, float *x) {
    const uint32_t u[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) { x[2 * i] = lo(u[i]); x[2 * i + 1] = hi(u[i]); }
  }
  static __device__ __forceinline__ uint4 pack(const float *x) {       // exact: words and -inf
    uint4 v;
    uint32_t *u = &v.x;
#pragma unroll
    for (int i = 0; i < 4; ++i) u[i] = (__float_as_uint(x[2 * i]) >> 16) | (__float_as_uint(x[2 * i + 1]) & 0xffff0000u);
    return v;
  }
  static __device__ __forceinline__ float largest(const uint4 &v) {    // of those that are no NaN (NaN if none is)
    const uint32_t m = max_bf16x2(max_bf16x2(v.x, v.y), max_bf16x2(v.z, v.w));
    return fmaxf(lo(m), hi(m));
  }
  // pairs of words held above -1e30
  static __device__ __forceinline__ void pairs(const uint4 &v, float2 *x) {
    const uint32_t u[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t w = max_bf16x2(u[i], 0xf149f149u);                // -1e30 in bf16
      x[i] = make_float2(lo(w), hi(w));
    }
  }
  static __device__ __forceinline__ float one(const __nv_bfloat16 *p) { return __bfloat162float(*p); }
};
template <> struct Vec<float> {
  static constexpr int N = 4;
  static __device__ __forceinline__ void unpack(const uint4 &v, float *x) {
    x[0] = __uint_as_float(v.x); x[1] = __uint_as_float(v.y); x[2] = __uint_as_float(v.z); x[3] = __uint_as_float(v.w);
  }
  static __device__ __forceinline__ uint4 pack(const float *x) {
    return make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3]));
  }
  static __device__ __forceinline__ float largest(const uint4 &v) {
    return fmaxf(fmaxf(__uint_as_float(v.x), __uint_as_float(v.y)), fmaxf(__uint_as_float(v.z), __uint_as_float(v.w)));
  }
  static __device__ __forceinline__ void pairs(const uint4 &v, float2 *x) {
    x[0] = make_float2(fmaxf(__uint_as_float(v.x), -1e30f), fmaxf(__uint_as_float(v.y), -1e30f));
    x[1] = make_float2(fmaxf(__uint_as_float(v.z), -1e30f), fmaxf(__uint_as_float(v.w), -1e30f));
  }
  static __device__ __forceinline__ float one(const float *p) { return *p; }
};

// The words of group g that this lane holds, as they lie in memory.  Word ids begin at -shift: the row starts `shift` words
// after a 16-byte boundary, and words before its start or past its end are -inf.
template <typename T>
__device__ __forceinline__ uint4 load_raw(const T *row, int shift, int V, int g, int lane) {
  constexpr int N = Vec<T>::N;
  const int i = (g * 32 + lane) * N - shift;
  if (i >= 0 && i + N <= V) return __ldcs((const uint4 *)(row + i));
  float x[N];
#pragma unroll
  for (int k = 0; k < N; ++k) x[k] = i + k >= 0 && i + k < V ? Vec<T>::one(row + i + k) : kNone;
  return Vec<T>::pack(x);
}
template <typename T>
__device__ __forceinline__ void load_words(const T *row, int shift, int V, int g, int lane, float *x) {
  Vec<T>::unpack(load_raw<T>(row, shift, V, g, lane), x);
}

}  // namespace
}  // namespace pcomoe
