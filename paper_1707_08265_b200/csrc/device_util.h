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

// V consecutive elements (V = 8: 16-byte aligned, or V = 1) as they are in memory, so that loads can be issued
// together and converted later
template <int DT, int V> struct Raw;
template <> struct Raw<DRAGON_BF16, 8> {
  uint4 u;
  __device__ __forceinline__ void load(const void* p, size_t i) { u = __ldg(reinterpret_cast<const uint4*>(reinterpret_cast<const unsigned short*>(p) + i)); }
  __device__ __forceinline__ void get(float* v) const {
    v[0] = bf16_low(u.x); v[1] = bf16_high(u.x); v[2] = bf16_low(u.y); v[3] = bf16_high(u.y);
    v[4] = bf16_low(u.z); v[5] = bf16_high(u.z); v[6] = bf16_low(u.w); v[7] = bf16_high(u.w);
  }
};
template <> struct Raw<DRAGON_F32, 8> {
  float4 a, b;
  __device__ __forceinline__ void load(const void* p, size_t i) {
    const float4* q = reinterpret_cast<const float4*>(reinterpret_cast<const float*>(p) + i);
    a = __ldg(q); b = __ldg(q + 1);
  }
  __device__ __forceinline__ void get(float* v) const { v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w; }
};
template <> struct Raw<DRAGON_BF16, 1> {
  unsigned short u;
  __device__ __forceinline__ void load(const void* p, size_t i) { u = __ldg(reinterpret_cast<const unsigned short*>(p) + i); }
  __device__ __forceinline__ void get(float* v) const { v[0] = bf16_low(u); }
};
template <> struct Raw<DRAGON_F32, 1> {
  float a;
  __device__ __forceinline__ void load(const void* p, size_t i) { a = __ldg(reinterpret_cast<const float*>(p) + i); }
  __device__ __forceinline__ void get(float* v) const { v[0] = a; }
};
template <int V> struct Raw<-1, V> {      // an absent operand
  __device__ __forceinline__ void load(const void*, size_t) {}
  __device__ __forceinline__ void get(float* v) const {
#pragma unroll
    for (int e = 0; e < V; ++e) v[e] = 0.f;
  }
};

template <int V> __device__ __forceinline__ void load_any(const void* p, int dtype, size_t i, float* v) {
  if (dtype == DRAGON_F32) { Raw<DRAGON_F32, V> r; r.load(p, i); r.get(v); }
  else { Raw<DRAGON_BF16, V> r; r.load(p, i); r.get(v); }
}
template <int V> __device__ __forceinline__ void store_any(void* p, int dtype, size_t i, const float* v) {
  if (V == 8) {
    if (dtype == DRAGON_F32) {
      float4* q = reinterpret_cast<float4*>(reinterpret_cast<float*>(p) + i);
      q[0] = make_float4(v[0], v[1], v[2], v[3]);
      q[1] = make_float4(v[4], v[5], v[6], v[7]);
    } else {
      *reinterpret_cast<uint4*>(reinterpret_cast<unsigned short*>(p) + i) =
          make_uint4(bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3]), bf16_pair(v[4], v[5]), bf16_pair(v[6], v[7]));
    }
  } else {
    if (dtype == DRAGON_F32) reinterpret_cast<float*>(p)[i] = v[0];
    else reinterpret_cast<unsigned short*>(p)[i] = bf16_one(v[0]);
  }
}

// e4m3 of v, nearest (ties to even), magnitudes beyond 448 become 448, NaN stays NaN
__device__ __forceinline__ unsigned e4m3_pair(float lo, float hi) { return __nv_cvt_float2_to_fp8x2(make_float2(lo, hi), __NV_SATFINITE, __NV_E4M3); }
__device__ __forceinline__ unsigned char e4m3_of(float v) { return __nv_cvt_float_to_fp8(v, __NV_SATFINITE, __NV_E4M3); }

// Largest magnitude of a block as the integer that orders floats of one sign: a NaN is larger than everything and stays
__device__ __forceinline__ unsigned magnitude(float v) { return __float_as_uint(v) & 0x7fffffffu; }
__device__ __forceinline__ float scale_of(unsigned magnitude_bits) {
  const float s = __fdiv_rn(__uint_as_float(magnitude_bits), 448.f);
  return s < 1.17549435e-38f ? 1.17549435e-38f : s;      // 2^-126; a comparison with NaN is false, so NaN stays
}

}  // namespace dragon
