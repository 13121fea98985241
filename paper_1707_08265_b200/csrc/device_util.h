// Device helpers of the language-model kernels: 8 elements at a time in any float type, e4m3 rounding, reductions.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp8.h>
#include <cuda_runtime.h>

#include "../../include/dragon.h"

namespace dragon {

__device__ __forceinline__ float bf16_low(unsigned w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_high(unsigned w) { return __uint_as_float(w & 0xffff0000u); }
// nearest bf16, ties to even, by the conversion instruction
__device__ __forceinline__ unsigned bf16_pair(float lo, float hi) {
  const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const unsigned*>(&v);
}
__device__ __forceinline__ unsigned short bf16_one(float v) { return __bfloat16_as_ushort(__float2bfloat16_rn(v)); }
__device__ __forceinline__ float bf16_rounded(float v) { return bf16_low(bf16_one(v)); }

// V consecutive elements (V = 8: 16-byte aligned, 2 or 1) as they are in memory, so that loads can be issued
// together and converted later.  DT -1: a type known at run time, -2: an absent operand.
template <int DT, int V> struct Raw;
template <> struct Raw<DRAGON_BF16, 8> {
  uint4 u;
  __device__ __forceinline__ void load(const void* p, int, size_t i) { u = __ldg(reinterpret_cast<const uint4*>(reinterpret_cast<const unsigned short*>(p) + i)); }
  __device__ __forceinline__ void get(float* v) const {
    v[0] = bf16_low(u.x); v[1] = bf16_high(u.x); v[2] = bf16_low(u.y); v[3] = bf16_high(u.y);
    v[4] = bf16_low(u.z); v[5] = bf16_high(u.z); v[6] = bf16_low(u.w); v[7] = bf16_high(u.w);
  }
  __device__ __forceinline__ void set(const float* v) { u = make_uint4(bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3]), bf16_pair(v[4], v[5]), bf16_pair(v[6], v[7])); }
  __device__ __forceinline__ void store(void* p, int, size_t i) const { *reinterpret_cast<uint4*>(reinterpret_cast<unsigned short*>(p) + i) = u; }
};
template <> struct Raw<DRAGON_F32, 8> {
  float4 a, b;
  __device__ __forceinline__ void load(const void* p, int, size_t i) {
    const float4* q = reinterpret_cast<const float4*>(reinterpret_cast<const float*>(p) + i);
    a = __ldg(q); b = __ldg(q + 1);
  }
  __device__ __forceinline__ void get(float* v) const { v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w; }
  __device__ __forceinline__ void set(const float* v) { a = make_float4(v[0], v[1], v[2], v[3]); b = make_float4(v[4], v[5], v[6], v[7]); }
  __device__ __forceinline__ void store(void* p, int, size_t i) const {
    float4* q = reinterpret_cast<float4*>(reinterpret_cast<float*>(p) + i);
    q[0] = a; q[1] = b;
  }
};
template <> struct Raw<DRAGON_BF16, 2> {      // (4-byte aligned)
  unsigned u;
  __device__ __forceinline__ void load(const void* p, int, size_t i) { u = __ldg(reinterpret_cast<const unsigned*>(reinterpret_cast<const unsigned short*>(p) + i)); }
  __device__ __forceinline__ void get(float* v) const { v[0] = bf16_low(u); v[1] = bf16_high(u); }
  __device__ __forceinline__ void set(const float* v) { u = bf16_pair(v[0], v[1]); }
  __device__ __forceinline__ void store(void* p, int, size_t i) const { *reinterpret_cast<unsigned*>(reinterpret_cast<unsigned short*>(p) + i) = u; }
};
template <> struct Raw<DRAGON_F32, 2> {       // (8-byte aligned)
  float2 a;
  __device__ __forceinline__ void load(const void* p, int, size_t i) { a = __ldg(reinterpret_cast<const float2*>(reinterpret_cast<const float*>(p) + i)); }
  __device__ __forceinline__ void get(float* v) const { v[0] = a.x; v[1] = a.y; }
  __device__ __forceinline__ void set(const float* v) { a = make_float2(v[0], v[1]); }
  __device__ __forceinline__ void store(void* p, int, size_t i) const { *reinterpret_cast<float2*>(reinterpret_cast<float*>(p) + i) = a; }
};
template <> struct Raw<DRAGON_BF16, 1> {
  unsigned short u;
  __device__ __forceinline__ void load(const void* p, int, size_t i) { u = __ldg(reinterpret_cast<const unsigned short*>(p) + i); }
  __device__ __forceinline__ void get(float* v) const { v[0] = bf16_low(u); }
  __device__ __forceinline__ void set(const float* v) { u = bf16_one(v[0]); }
  __device__ __forceinline__ void store(void* p, int, size_t i) const { reinterpret_cast<unsigned short*>(p)[i] = u; }
};
template <> struct Raw<DRAGON_F32, 1> {
  float a;
  __device__ __forceinline__ void load(const void* p, int, size_t i) { a = __ldg(reinterpret_cast<const float*>(p) + i); }
  __device__ __forceinline__ void get(float* v) const { v[0] = a; }
  __device__ __forceinline__ void set(const float* v) { a = v[0]; }
  __device__ __forceinline__ void store(void* p, int, size_t i) const { reinterpret_cast<float*>(p)[i] = a; }
};
template <int V> struct Raw<-1, V> {
  float f[V];
  __device__ __forceinline__ void load(const void* p, int dtype, size_t i) {
    if (dtype == DRAGON_F32) { Raw<DRAGON_F32, V> r; r.load(p, 0, i); r.get(f); }
    else { Raw<DRAGON_BF16, V> r; r.load(p, 0, i); r.get(f); }
  }
  __device__ __forceinline__ void get(float* v) const {
#pragma unroll
    for (int e = 0; e < V; ++e) v[e] = f[e];
  }
  __device__ __forceinline__ void set(const float* v) {
#pragma unroll
    for (int e = 0; e < V; ++e) f[e] = v[e];
  }
  __device__ __forceinline__ void store(void* p, int dtype, size_t i) const {
    if (dtype == DRAGON_F32) { Raw<DRAGON_F32, V> r; r.set(f); r.store(p, 0, i); }
    else { Raw<DRAGON_BF16, V> r; r.set(f); r.store(p, 0, i); }
  }
};
template <int V> struct Raw<-2, V> {
  __device__ __forceinline__ void load(const void*, int, size_t) {}
  __device__ __forceinline__ void get(float* v) const {
#pragma unroll
    for (int e = 0; e < V; ++e) v[e] = 0.f;
  }
};

template <int V> __device__ __forceinline__ void load_any(const void* p, int dtype, size_t i, float* v) {
  Raw<-1, V> r;
  r.load(p, dtype, i);
  r.get(v);
}
template <int V> __device__ __forceinline__ void store_any(void* p, int dtype, size_t i, const float* v) {
  Raw<-1, V> r;
  r.set(v);
  r.store(p, dtype, i);
}

// e4m3 of v, nearest (ties to even), magnitudes beyond 448 become 448, NaN stays NaN
__device__ __forceinline__ unsigned e4m3_pair(float lo, float hi) { return __nv_cvt_float2_to_fp8x2(make_float2(lo, hi), __NV_SATFINITE, __NV_E4M3); }
__device__ __forceinline__ unsigned char e4m3_of(float v) { return __nv_cvt_float_to_fp8(v, __NV_SATFINITE, __NV_E4M3); }

// V e4m3 values of v * inv (V = 8: at an address that is a multiple of 8)
template <int V> __device__ __forceinline__ void store_e4m3(unsigned char* p, const float* v, float inv) {
  if (V == 1) { *p = e4m3_of(v[0] * inv); return; }
  uint2 w;
  w.x = e4m3_pair(v[0] * inv, v[1 % V] * inv) | (e4m3_pair(v[2 % V] * inv, v[3 % V] * inv) << 16);
  w.y = e4m3_pair(v[4 % V] * inv, v[5 % V] * inv) | (e4m3_pair(v[6 % V] * inv, v[7 % V] * inv) << 16);
  *reinterpret_cast<uint2*>(p) = w;
}

// Largest magnitude of a block as the integer that orders floats of one sign: a NaN is larger than everything and stays
__device__ __forceinline__ unsigned magnitude(float v) { return __float_as_uint(v) & 0x7fffffffu; }
template <int DT> __device__ __forceinline__ unsigned largest_magnitude(const Raw<DT, 8>& r) {
  float v[8];
  r.get(v);
  unsigned m = 0;
#pragma unroll
  for (int e = 0; e < 8; ++e) m = max(m, magnitude(v[e]));
  return m;
}
template <> __device__ __forceinline__ unsigned largest_magnitude<DRAGON_BF16>(const Raw<DRAGON_BF16, 8>& r) {      // two at a time
  constexpr unsigned k = 0x7fff7fffu;
  const unsigned m = __vmaxu2(__vmaxu2(r.u.x & k, r.u.y & k), __vmaxu2(r.u.z & k, r.u.w & k));
  return max(m & 0xffff0000u, m << 16);
}
__device__ __forceinline__ float scale_of(unsigned magnitude_bits) {
  const float s = __fdiv_rn(__uint_as_float(magnitude_bits), 448.f);
  return s < 1.17549435e-38f ? 1.17549435e-38f : s;      // 2^-126; a comparison with NaN is false, so NaN stays
}

}  // namespace dragon
