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

// two fp32 values in one 64-bit register, and arithmetic on both at once
typedef unsigned long long Pair;
__device__ __forceinline__ Pair pair_of(float lo, float hi) { Pair p; asm("mov.b64 %0, {%1, %2};" : "=l"(p) : "f"(lo), "f"(hi)); return p; }
__device__ __forceinline__ Pair pair_of(uint32_t lo, uint32_t hi) { Pair p; asm("mov.b64 %0, {%1, %2};" : "=l"(p) : "r"(lo), "r"(hi)); return p; }
__device__ __forceinline__ float2 both(Pair p) { float2 v; asm("mov.b64 {%0, %1}, %2;" : "=f"(v.x), "=f"(v.y) : "l"(p)); return v; }
__device__ __forceinline__ Pair fma_pair(Pair a, Pair b, Pair c) { Pair d; asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c)); return d; }
__device__ __forceinline__ Pair add_pair(Pair a, Pair b) { Pair d; asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b)); return d; }
__device__ __forceinline__ Pair mul_pair(Pair a, Pair b) { Pair d; asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b)); return d; }

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

// Four consecutive elements for each lane of a warp, lane after lane, from an element on that is no multiple of 4: every lane
// reads the aligned vector that its first element lies in, and takes the rest from the next lane's.
template <int DT> struct Quad;
template <> struct Quad<DRAGON_BF16> {
  typedef uint2 Vec;
  uint2 u;
  __device__ __forceinline__ void get(float* v) const { v[0] = bf16_low(u.x); v[1] = bf16_high(u.x); v[2] = bf16_low(u.y); v[3] = bf16_high(u.y); }
  static __device__ __forceinline__ uint2 part(const char* p, int n) {      // the first n of an aligned vector's elements (n < 4)
    const unsigned short* q = reinterpret_cast<const unsigned short*>(p);
    uint2 v = make_uint2(0, 0);
    if (n > 0) v.x = __ldg(q);
    if (n > 1) v.x |= (unsigned)__ldg(q + 1) << 16;
    if (n > 2) v.y = __ldg(q + 2);
    return v;
  }
  static __device__ __forceinline__ uint2 next_lane(uint2 v) { return make_uint2(__shfl_down_sync(0xffffffffu, v.x, 1), __shfl_down_sync(0xffffffffu, v.y, 1)); }
  static __device__ __forceinline__ uint2 of_lane(uint2 v, int l) { return make_uint2(__shfl_sync(0xffffffffu, v.x, l), __shfl_sync(0xffffffffu, v.y, l)); }
  static __device__ __forceinline__ uint2 join(uint2 v, uint2 n, int lead) {      // elements lead .. lead + 3 of the two
    if (lead & 2) { v.x = v.y; v.y = n.x; n.x = n.y; }
    if (lead & 1) { v.x = __funnelshift_r(v.x, v.y, 16); v.y = __funnelshift_r(v.y, n.x, 16); }
    return v;
  }
};
template <> struct Quad<DRAGON_F32> {
  typedef uint4 Vec;
  uint4 u;
  __device__ __forceinline__ void get(float* v) const { v[0] = __uint_as_float(u.x); v[1] = __uint_as_float(u.y); v[2] = __uint_as_float(u.z); v[3] = __uint_as_float(u.w); }
  static __device__ __forceinline__ uint4 part(const char* p, int n) {
    const unsigned* q = reinterpret_cast<const unsigned*>(p);
    uint4 v = make_uint4(0, 0, 0, 0);
    if (n > 0) v.x = __ldg(q);
    if (n > 1) v.y = __ldg(q + 1);
    if (n > 2) v.z = __ldg(q + 2);
    return v;
  }
  static __device__ __forceinline__ uint4 next_lane(uint4 v) {
    return make_uint4(__shfl_down_sync(0xffffffffu, v.x, 1), __shfl_down_sync(0xffffffffu, v.y, 1), __shfl_down_sync(0xffffffffu, v.z, 1), 0);
  }
  static __device__ __forceinline__ uint4 of_lane(uint4 v, int l) {
    return make_uint4(__shfl_sync(0xffffffffu, v.x, l), __shfl_sync(0xffffffffu, v.y, l), __shfl_sync(0xffffffffu, v.z, l), 0);
  }
  static __device__ __forceinline__ uint4 join(uint4 v, uint4 n, int lead) {
    if (lead & 2) { v = make_uint4(v.z, v.w, n.x, n.y); n.x = n.z; }
    if (lead & 1) v = make_uint4(v.y, v.z, v.w, n.x);
    return v;
  }
};
// In two steps, so that the loads of several such pieces are in flight together.  i0: the first lane's first element; left: how
// many elements the tensor has from it on (what is behind them reads as 0, what is behind the piece as it is: the caller masks).
// First every lane's vector, and by some lane the one behind the last lane's; then, by the whole warp, the elements.
template <int DT> __device__ __forceinline__ typename Quad<DT>::Vec vector_from(const void* p, size_t i0, long long left, int at) {
  const int lead = (int)(i0 & 3);
  const char* q = static_cast<const char*>(p) + (i0 - lead + 4 * at) * (DT == DRAGON_F32 ? 4 : 2);
  if (left >= 132) return __ldg(reinterpret_cast<const typename Quad<DT>::Vec*>(q));
  const int room = (int)left + lead - 4 * at;        // elements from this vector on
  return room >= 4 ? __ldg(reinterpret_cast<const typename Quad<DT>::Vec*>(q)) : Quad<DT>::part(q, room);
}
template <int DT> __device__ __forceinline__ Quad<DT> quads_of(typename Quad<DT>::Vec own, typename Quad<DT>::Vec behind, int holder, size_t i0, int lane) {
  Quad<DT> q;
  typename Quad<DT>::Vec next = Quad<DT>::next_lane(own), last = Quad<DT>::of_lane(behind, holder);
  q.u = Quad<DT>::join(own, lane == 31 ? last : next, (int)(i0 & 3));
  return q;
}
// Four bytes for each lane, likewise; the first n of the warp's 128 are written.
__device__ __forceinline__ void store_byte_quads(unsigned char* p, size_t i0, int n, unsigned w, int lane) {
  const int lead = (int)(i0 & 3), first = 4 * lane - lead;         // of the aligned word of this lane, counted from i0
  unsigned char* at = p + i0;
  if (lead == 0 && n == 128) { *reinterpret_cast<unsigned*>(at + first) = w; return; }
  const unsigned before = __shfl_up_sync(0xffffffffu, w, 1), head = __shfl_sync(0xffffffffu, w, 0), tail = __shfl_sync(0xffffffffu, w, 31);
  const unsigned word = __funnelshift_l(before, w, 8 * lead);
  // the first 4 - lead bytes and the last lead ones are no whole word: one byte each for four lanes
  const int edge = lane < 4 - lead ? lane : 124 + lane;
  if (lane < 4 && edge < n) at[edge] = (unsigned char)((edge < 4 ? head : tail) >> (8 * lane));
  if (lane == 0) return;
  if (first + 4 <= n) *reinterpret_cast<unsigned*>(at + first) = word;
  else
    for (int e = 0; first + e < n; ++e) at[first + e] = (unsigned char)(word >> (8 * e));
}
template <int DT> __device__ __forceinline__ unsigned largest_magnitude(const Quad<DT>& q, int n) {      // of its first n elements
  float v[4];
  q.get(v);
  if (n >= 4) return max(max(magnitude(v[0]), magnitude(v[1])), max(magnitude(v[2]), magnitude(v[3])));
  unsigned m = 0;
#pragma unroll
  for (int e = 0; e < 3; ++e)
    if (e < n) m = max(m, magnitude(v[e]));
  return m;
}
template <int DT> __device__ __forceinline__ unsigned e4m3_of(const Quad<DT>& q, float inv) {
  float v[4];
  q.get(v);
  return e4m3_pair(v[0] * inv, v[1] * inv) | (e4m3_pair(v[2] * inv, v[3] * inv) << 16);
}

}  // namespace dragon
