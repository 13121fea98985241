// HeadNorm and Rotate: every head of a row over its root mean square, and turned by the row's position.
//
//   u = x / sqrt(mean(x^2) + eps) * g;  y = amplitude (a cos t - b sin t, b cos t + a sin t) over pairs (a, b) of u's first dims
//   elements, t = position * f_i.  Backwards, with d = the rotation by -t of dy:
//   dg = sum over rows and heads of d x r,  dx = r (d g - x r mean(d g x r)),  r = 1 / sqrt(mean(x^2) + eps).
//
// Angles: f_i / 2 pi is kept as a 64-bit fraction of a turn, so position * f_i modulo one turn is one wrapping integer product
// (no rounding grows with the position); its top 32 bits go through sincospi in fp32.  They are the same for every head of a
// row: a CTA computes those of its rows once, into shared memory.
//
// Bound: HBM (every element is read and written once), and next to it instructions (8192 rows, 32 + 8 heads of 128 in bf16: forward 36 us,
// 4.7 TB/s, gradient 59, 4.2, with 0.55 and 0.60 of the issue slots; three CTAs an SM spill: 99 us for both become 145).  A warp works on one row at a time: 8 elements a
// lane, a head in the next power of two of lanes, so that the head's sums are a few shuffles.  Where pairs are halves apart a lane
// has 4 elements and their 4 partners.  Gain and angle are multiplied once a row: y = r (a (g c) - b (g' s)), and stay in registers
// while the warp walks the row's heads.  Tensors of the same rows (queries and keys) are one launch.
#include <cuda_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>

#include "device_util.h"
#include "plan.h"

namespace dragon {
namespace {

constexpr int kHeadCtas = 2;            // of an SM: persistent, each with its next accesses on the way while it computes
constexpr int kHeadThreads = 256, kHeadWarps = kHeadThreads / 32;
constexpr int kHeadRowsMost = kHeadWarps;       // rows of a tile: their angles are computed together
constexpr int kPairsMost = kMaxRotatedWidth / 2;

enum Pairing { P_NONE, P_NEIGHBOURS, P_HALVES, P_ANY };   // where a lane finds the partners of its 8 elements: nowhere, next to them, in its own other half, anywhere

struct HeadJob {
  const void *x, *gain, *dy;
  void *u, *y;             // backwards: y receives dx
  float* dgain;            // partial rows [grid][width]
  int xt, gt, dyt, ut, yt;
  int round_u;             // u is rounded to bf16 before it is rotated
  int heads;
  float eps;
};
struct HeadArgs {
  HeadJob job[kHeadsPerLaunch];
  const int* pos;
  int *status_clear;
  int rows, width, dims, lanes;   // lanes: of a head, a power of two
  int tile;                // rows of a tile, a power of two
  float amplitude;
  unsigned long long freq[kPairsMost];   // turns per position, times 2^64
};

// (amplitude cos, amplitude sin) of pair i, where every lane finds those of its elements without a bank in common
__device__ __forceinline__ int place_of(int i) { return (i & 7) * (kPairsMost / 8 + 1) + (i >> 3); }
constexpr int kPlaces = 8 * (kPairsMost / 8 + 1);

// the angles of a tile: a warp a row (its rows are at most as many as the warps), or several warps a row; position: of the warp's row
__device__ __forceinline__ void fill_angles(const HeadArgs& a, const unsigned long long* freq, float2 (*cs)[kPlaces], int position, int r, int part, int side) {
  const int pairs = a.dims >> 1;
  const unsigned long long pos = (unsigned long long)(long long)position;
  for (int k = (threadIdx.x & 31) + 32 * part; k < pairs; k += 32 * side) {
    float s, c;
    sincospif((float)(int)((pos * freq[k]) >> 32) * 0x1p-31f, &s, &c);
    cs[r][place_of(k)] = make_float2(a.amplitude * c, a.amplitude * s);
  }
}

// 4 consecutive elements (of a multiple of 4), as they are in memory
template <int DT> struct Four;
template <> struct Four<DRAGON_BF16> {
  uint2 u;
  __device__ __forceinline__ void load(const void* p, int, size_t i) { u = __ldg(reinterpret_cast<const uint2*>(reinterpret_cast<const unsigned short*>(p) + i)); }
  __device__ __forceinline__ void get(float* v) const { v[0] = bf16_low(u.x); v[1] = bf16_high(u.x); v[2] = bf16_low(u.y); v[3] = bf16_high(u.y); }
  static __device__ __forceinline__ void store(void* p, int, size_t i, const float* v) {
    *reinterpret_cast<uint2*>(reinterpret_cast<unsigned short*>(p) + i) = make_uint2(bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3]));
  }
};
template <> struct Four<DRAGON_F32> {
  float4 u;
  __device__ __forceinline__ void load(const void* p, int, size_t i) { u = __ldg(reinterpret_cast<const float4*>(reinterpret_cast<const float*>(p) + i)); }
  __device__ __forceinline__ void get(float* v) const { v[0] = u.x; v[1] = u.y; v[2] = u.z; v[3] = u.w; }
  static __device__ __forceinline__ void store(void* p, int, size_t i, const float* v) { *reinterpret_cast<float4*>(reinterpret_cast<float*>(p) + i) = make_float4(v[0], v[1], v[2], v[3]); }
};
template <> struct Four<-1> {
  float4 u;
  __device__ __forceinline__ void load(const void* p, int dtype, size_t i) {
    float v[4];
    if (dtype == DRAGON_F32) { Four<DRAGON_F32> f; f.load(p, 0, i); f.get(v); }
    else { Four<DRAGON_BF16> f; f.load(p, 0, i); f.get(v); }
    u = make_float4(v[0], v[1], v[2], v[3]);
  }
  __device__ __forceinline__ void get(float* v) const { v[0] = u.x; v[1] = u.y; v[2] = u.z; v[3] = u.w; }
  static __device__ __forceinline__ void store(void* p, int dtype, size_t i, const float* v) {
    if (dtype == DRAGON_F32) Four<DRAGON_F32>::store(p, 0, i, v);
    else Four<DRAGON_BF16>::store(p, 0, i, v);
  }
};
// a lane's 8 elements: one access where they are neighbours, two of 4 where they are halves apart
template <int DT, bool kApart> struct Eight {
  Raw<DT, 8> r;
  __device__ __forceinline__ void load(const void* p, int dtype, size_t i, int) { r.load(p, dtype, i); }
  __device__ __forceinline__ void get(float* v) const { r.get(v); }
  static __device__ __forceinline__ void store(void* p, int dtype, size_t i, int, const float* v) { Raw<DT, 8> o; o.set(v); o.store(p, dtype, i); }
};
template <int DT> struct Eight<DT, true> {
  Four<DT> a, b;
  __device__ __forceinline__ void load(const void* p, int dtype, size_t i, int apart) { a.load(p, dtype, i); b.load(p, dtype, i + apart); }
  __device__ __forceinline__ void get(float* v) const { a.get(v); b.get(v + 4); }
  static __device__ __forceinline__ void store(void* p, int dtype, size_t i, int apart, const float* v) { Four<DT>::store(p, dtype, i, v); Four<DT>::store(p, dtype, i + apart, v + 4); }
};

// The factors of this lane's elements, in pairs: x'[e] = x[e] own[e] + x[partner] other[e].  Elements behind dims: 1 and 0.  at[e]: their
// places in the head; back: by the negative angle
template <int kPairing, bool kBack> __device__ __forceinline__ void load_angles(const float2* cs, const int* at, int dims, Pair* own, Pair* other) {
  const int half = dims >> 1;
  float x[8], y[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const bool in = at[e] < dims;
    const int i = kPairing == P_NEIGHBOURS ? at[e] >> 1 : at[e] < half ? at[e] : at[e] - half;
    const bool first = kPairing == P_NEIGHBOURS ? (e & 1) == 0 : at[e] < half;
    const float2 t = in ? cs[place_of(i)] : make_float2(1.f, 0.f);
    x[e] = t.x;
    y[e] = first != kBack ? -t.y : t.y;
  }
#pragma unroll
  for (int p = 0; p < 4; ++p) { own[p] = pair_of(x[2 * p], x[2 * p + 1]); other[p] = pair_of(y[2 * p], y[2 * p + 1]); }
}
// the partners of pair p of a lane's values (P_NEIGHBOURS, P_HALVES)
template <int kPairing> __device__ __forceinline__ Pair partners(const Pair* v, int p) {
  if (kPairing == P_HALVES) return v[p ^ 2];
  const float2 f = both(v[p]);
  return pair_of(f.y, f.x);
}
__device__ __forceinline__ Pair twice(float v) { return pair_of(v, v); }
__device__ __forceinline__ float sum_of(Pair a, Pair b) { const float2 s = both(add_pair(a, b)); return s.x + s.y; }

template <int kLanes> __device__ __forceinline__ float sum_over_lanes(float v, int lanes) {
#pragma unroll
  for (int s = 16; s; s >>= 1)
    if (kLanes ? kLanes > s : lanes > s) v += __shfl_xor_sync(0xffffffffu, v, s);
  return v;
}

// DT: the type of x, u and y (backwards: x, dy and dx), -1 for a mixture.  kU: u is written, or rounded before it is rotated.  kLanes: of a
// head, where every lane of every access has elements (the head's width 8 times a power of two, heads a multiple of those of an
// access), otherwise 0
template <int DT, int kPairing, bool kBack, bool kU, int kLanes> __global__ void __launch_bounds__(kHeadThreads, kHeadCtas) head_kernel(const __grid_constant__ HeadArgs a) {
  constexpr int kUnroll = (kBack ? 2 : 4) / (DT == DRAGON_BF16 ? 1 : 2);
  constexpr bool kApart = kPairing == P_HALVES;
  constexpr bool scaled_there = !kBack && !kU && (kPairing == P_NEIGHBOURS || kPairing == P_HALVES);      // gains go with the angles
  __shared__ float2 cs[kPairing == P_NONE ? 1 : kHeadRowsMost][kPlaces];
  __shared__ unsigned long long freq[kPairing == P_NONE ? 1 : kPairsMost];      // (lanes that index parameters apart wait for one another)
  __shared__ float buf[kPairing == P_ANY ? kHeadWarps : 1][256];
  __shared__ float sums[kBack ? kHeadWarps : 1][kMaxRotatedWidth];
  const HeadJob& jb = a.job[blockIdx.y];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (a.status_clear && blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0) *a.status_clear = 0;
  if (kPairing != P_NONE && threadIdx.x < a.dims >> 1) freq[threadIdx.x] = a.freq[threadIdx.x];      // (seen behind the tile's first barrier)
  const int lanes = kLanes ? kLanes : a.lanes, width = kLanes ? 8 * kLanes : a.width, l = lane & (lanes - 1);
  const bool active = kLanes || 8 * l < width;
  // this lane's elements: from e0 on, and (P_HALVES) 4 of them `apart` further
  int e0 = 8 * l, apart = 4;
  if (kApart && e0 < a.dims) { e0 = 4 * l; apart = a.dims >> 1; }
  int at_head[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) at_head[e] = e0 + (e & 3) + (e >= 4 ? apart : 0);
  const int per_warp = 32 / lanes, sub = lane / lanes;      // heads of one warp access
  const int groups = (jb.heads + per_warp - 1) / per_warp;
  const int side = kHeadWarps / a.tile, my_row = warp / side, my_side = warp - my_row * side;      // warps of a row
  const float inv_width = 1.f / (float)width;
  const bool norm = jb.gain != nullptr;
  Pair g[4], dg[4];
#pragma unroll
  for (int p = 0; p < 4; ++p) { g[p] = twice(1.f); dg[p] = 0; }
  if (norm && active) {
    Eight<-1, true> r;
    float f[8];
    r.load(jb.gain, jb.gt, e0, apart);
    r.get(f);
#pragma unroll
    for (int p = 0; p < 4; ++p) g[p] = pair_of(f[2 * p], f[2 * p + 1]);
  }
  const long long stride = (long long)gridDim.x * a.tile;
  struct Batch { Eight<DT, kApart> x[kUnroll], d[kUnroll]; };
  // this lane's first elements of the warp's row of the tile: 32-bit offsets from there to the other heads (a row is at most 2^26 long)
  auto row_of = [&](long long r0) { return (size_t)(r0 + my_row) * jb.heads * width + sub * width + e0; };
  auto fetch = [&](size_t row, bool there, int i0, Batch& b) {
    if (!there) return;
#pragma unroll
    for (int k = 0; k < kUnroll; ++k) {
      const int grp = i0 + k * side;
      if (kLanes ? grp < groups : active && grp * per_warp + sub < jb.heads) {
        const size_t at = row + (unsigned)(grp * (per_warp * width));
        if (!kBack || norm) b.x[k].load(jb.x, jb.xt, at, apart);
        if (kBack) b.d[k].load(jb.dy, jb.dyt, at, apart);
      }
    }
  };
  Batch now;
  // the row whose angles this warp computes, and its position, known a tile ahead
  const int angle_row = warp & (a.tile - 1), angle_part = warp / a.tile;
  auto position_of = [&](long long r0) { return kPairing != P_NONE && r0 + angle_row < a.rows ? __ldg(a.pos + r0 + angle_row) : 0; };
  int position = position_of((long long)blockIdx.x * a.tile);
  const size_t row_stride = (size_t)stride * jb.heads * width;
  size_t row = row_of((long long)blockIdx.x * a.tile);
  fetch(row, (long long)blockIdx.x * a.tile + my_row < a.rows, my_side, now);
  for (long long r0 = (long long)blockIdx.x * a.tile; r0 < a.rows; r0 += stride, row += row_stride) {
    const int rows = (int)min((long long)a.tile, a.rows - r0);
    Pair own[4], other[4];
    if (kPairing != P_NONE) {
      __syncthreads();
      if (angle_row < rows) fill_angles(a, freq, cs, position, angle_row, angle_part, side);
      position = position_of(r0 + stride);
      __syncthreads();
    }
    if (my_row >= rows) continue;
    if (kPairing != P_NONE) {
      load_angles<kPairing, kBack>(cs[my_row], at_head, a.dims, own, other);
      if (scaled_there) {      // with the gains: the norm's own multiplication by them is done there
#pragma unroll
        for (int p = 0; p < 4; ++p) { own[p] = mul_pair(own[p], g[p]); other[p] = mul_pair(other[p], partners<kPairing>(g, p)); }
      }
    }
    for (int i0 = my_side; i0 < groups; i0 += side * kUnroll) {
      Batch next;
      const bool last = i0 + side * kUnroll >= groups;
      fetch(last ? row + row_stride : row, !last || r0 + stride + my_row < a.rows, last ? my_side : i0 + side * kUnroll, next);
#pragma unroll
      for (int k = 0; k < kUnroll; ++k) {
        if (i0 + k * side >= groups) break;       // the whole warp
        const bool ok = kLanes || (active && (i0 + k * side) * per_warp + sub < jb.heads);
        const size_t at = row + (unsigned)((i0 + k * side) * (per_warp * width));
        Pair x[4] = {0, 0, 0, 0}, v[4] = {0, 0, 0, 0};
        float f[8];
        if (ok && (!kBack || norm)) {
          now.x[k].get(f);
#pragma unroll
          for (int p = 0; p < 4; ++p) x[p] = pair_of(f[2 * p], f[2 * p + 1]);
        }
        if (kBack && ok) {
          now.d[k].get(f);
#pragma unroll
          for (int p = 0; p < 4; ++p) v[p] = pair_of(f[2 * p], f[2 * p + 1]);
        }
        float inv = 1.f;
        if (norm) {
          const float q = sum_of(fma_pair(x[0], x[0], mul_pair(x[1], x[1])), fma_pair(x[2], x[2], mul_pair(x[3], x[3])));
          inv = rsqrtf(sum_over_lanes<kLanes>(q, lanes) * inv_width + jb.eps);
          if (kBack && !ok) inv = 0.f;      // (lanes without a head: an infinite root times their zeros would go into dg)
        }
        const Pair r = twice(inv);
        if (!kBack) {
          if (scaled_there) {
#pragma unroll
            for (int p = 0; p < 4; ++p) v[p] = mul_pair(r, fma_pair(x[p], own[p], mul_pair(partners<kPairing>(x, p), other[p])));
          } else {
#pragma unroll
            for (int p = 0; p < 4; ++p) {
              x[p] = mul_pair(mul_pair(x[p], r), g[p]);
              const float2 t = both(x[p]);
              f[2 * p] = t.x; f[2 * p + 1] = t.y;
            }
            if (kU && jb.u && ok) Eight<-1, kApart>::store(jb.u, jb.ut, at, apart, f);
            if (kU && jb.round_u) {
#pragma unroll
              for (int p = 0; p < 4; ++p) x[p] = pair_of(bf16_rounded(f[2 * p]), bf16_rounded(f[2 * p + 1]));
            }
          }
        }
        const Pair* from = kBack ? v : x;      // what is rotated
        const Pair kept[4] = {v[0], v[1], v[2], v[3]};
        if (kPairing == P_ANY) {
          float* b = buf[kPairing == P_ANY ? warp : 0];
          const int half = a.dims >> 1;
          __syncwarp();
#pragma unroll
          for (int p = 0; p < 4; ++p) *reinterpret_cast<Pair*>(b + lane * 8 + 2 * p) = from[p];
          __syncwarp();
          const float* head = b + lane * 8 - e0;
#pragma unroll
          for (int p = 0; p < 4; ++p) {
            float o[2];
#pragma unroll
            for (int e = 0; e < 2; ++e) { const int i = e0 + 2 * p + e; o[e] = head[i < half ? i + half : i - half]; }
            v[p] = e0 + 2 * p < a.dims ? fma_pair(from[p], own[p], mul_pair(pair_of(o[0], o[1]), other[p])) : from[p];
          }
        } else if ((kBack || kU) && kPairing != P_NONE) {
          Pair w[4];
#pragma unroll
          for (int p = 0; p < 4; ++p) w[p] = fma_pair(from[p], own[p], mul_pair(partners<kPairing>(from, p), other[p]));
#pragma unroll
          for (int p = 0; p < 4; ++p) v[p] = w[p];
        } else if (!kBack && kPairing == P_NONE) {
#pragma unroll
          for (int p = 0; p < 4; ++p) v[p] = x[p];
        }
        // elements behind dims (whole pairs) are copied: not even 0 times another one goes into them
        if ((kPairing == P_NEIGHBOURS || kPairing == P_HALVES) && a.dims < width) {
#pragma unroll
          for (int p = 0; p < 4; ++p)
            if (at_head[2 * p] >= a.dims) v[p] = kBack ? kept[p] : scaled_there ? mul_pair(r, mul_pair(x[p], own[p])) : x[p];
        }
        if (kBack && norm) {
          // on the normalised values u = x r: no power of r above the first, which alone may leave fp32's range (heads of 1e13 and more)
          Pair t[4], u[4];
#pragma unroll
          for (int p = 0; p < 4; ++p) { t[p] = mul_pair(v[p], g[p]); u[p] = mul_pair(x[p], r); }
          const float m = sum_of(fma_pair(t[0], u[0], mul_pair(t[1], u[1])), fma_pair(t[2], u[2], mul_pair(t[3], u[3])));
          const Pair c = twice(-sum_over_lanes<kLanes>(m, lanes) * inv_width);
#pragma unroll
          for (int p = 0; p < 4; ++p) {
            dg[p] = fma_pair(v[p], u[p], dg[p]);
            v[p] = mul_pair(r, fma_pair(u[p], c, t[p]));
          }
        }
        if (jb.y && ok) {
#pragma unroll
          for (int p = 0; p < 4; ++p) { const float2 t = both(v[p]); f[2 * p] = t.x; f[2 * p + 1] = t.y; }
          Eight<DT, kApart>::store(jb.y, jb.yt, at, apart, f);
        }
      }
      now = next;
    }
  }
  if (kBack && jb.dgain) {      // the CTA's part of dg: lanes of the same elements, then the warps, in a fixed order
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      float d = e & 1 ? both(dg[e >> 1]).y : both(dg[e >> 1]).x;
      for (int s = lanes; s < 32; s <<= 1) d += __shfl_xor_sync(0xffffffffu, d, s);
      if (lane < lanes && active) sums[warp][at_head[e]] = d;
    }
    __syncthreads();
    for (int c = threadIdx.x; c < a.width; c += kHeadThreads) {
      float t = 0.f;
      for (int w = 0; w < kHeadWarps; ++w) t += sums[w][c];
      jb.dgain[(size_t)blockIdx.x * a.width + c] = t;
    }
  }
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
}

// dg: the partial rows in a fixed order (in fp64), 32 columns a CTA
struct FinishArgs {
  const float* part[kHeadsPerLaunch];
  void* out[kHeadsPerLaunch];
  int type[kHeadsPerLaunch];
  int n, width;
};
__global__ void __launch_bounds__(1024) head_finish(const __grid_constant__ FinishArgs a) {
  __shared__ double sh[32][33];
  const int lane = threadIdx.x & 31, slice = threadIdx.x >> 5, c = blockIdx.x * 32 + lane;
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const float* part = a.part[blockIdx.y];
  double s = 0.0;
  if (c < a.width) {
    int i = slice;
    for (; i + 96 < a.n; i += 128) {
      const float v0 = part[(size_t)i * a.width + c], v1 = part[(size_t)(i + 32) * a.width + c], v2 = part[(size_t)(i + 64) * a.width + c], v3 = part[(size_t)(i + 96) * a.width + c];
      s += ((double)v0 + (double)v1) + ((double)v2 + (double)v3);
    }
    for (; i < a.n; i += 32) s += (double)part[(size_t)i * a.width + c];
  }
  sh[slice][lane] = s;
  __syncthreads();
  if (slice == 0 && c < a.width) {
    for (int k = 1; k < 32; ++k) s += sh[k][lane];
    const float v = (float)s;
    store_any<1>(a.out[blockIdx.y], a.type[blockIdx.y], (size_t)c, &v);
  }
}

// Rows of a tile: as many as leave tiles enough for four CTAs on every SM, and so many that each warp of a row has an access to make
// (964 rows of one head with gradients: 34 us with tiles of one row, of whose eight warps seven had nothing to do, 14.5 with eight rows)
int tile_rows(int64_t rows, int accesses, int sm_count) {
  int t = kHeadRowsMost;
  while (t > 1 && rows < t * (4 * (int64_t)sm_count) && accesses >= 2 * kHeadWarps / t) t /= 2;
  return t;
}
struct HeadTiles { int tile, grid; };
// x: where a job's operand of [rows, heads * width] stands among its `reads`
HeadTiles head_tiles(const Step& s, const std::vector<MemRef>& mems, int x, int reads, int sm_count) {
  const int width = (int)s.num[hn::WIDTH];
  int lanes = 1;
  while (lanes * 8 < width) lanes *= 2;
  int64_t accesses = 1;
  for (size_t at = x; at < s.rd.size(); at += reads) accesses = std::max(accesses, (mems[s.rd[at]].shape.d[1] / width * lanes + 31) / 32);
  const int64_t rows = mems[s.rd[x]].shape.d[0];
  HeadTiles t;
  t.tile = tile_rows(rows, (int)std::min<int64_t>(accesses, kHeadWarps), sm_count);
  t.grid = (int)std::min<int64_t>((rows + t.tile - 1) / t.tile, kHeadCtas * (int64_t)sm_count);
  return t;
}

template <int DT, int kPairing, bool kBack, bool kU> void launch_lanes(const HeadArgs& a, bool full, dim3 grid, cudaStream_t st) {
  if constexpr (DT != -1 && kPairing != P_NONE && kPairing != P_ANY) {
    if (full && a.lanes >= 4) {      // heads of 32, 64, 128 and 256
      if (a.lanes == 4) head_kernel<DT, kPairing, kBack, kU, 4><<<grid, kHeadThreads, 0, st>>>(a);
      else if (a.lanes == 8) head_kernel<DT, kPairing, kBack, kU, 8><<<grid, kHeadThreads, 0, st>>>(a);
      else if (a.lanes == 16) head_kernel<DT, kPairing, kBack, kU, 16><<<grid, kHeadThreads, 0, st>>>(a);
      else head_kernel<DT, kPairing, kBack, kU, 32><<<grid, kHeadThreads, 0, st>>>(a);
      return;
    }
  }
  head_kernel<DT, kPairing, kBack, kU, 0><<<grid, kHeadThreads, 0, st>>>(a);
}
template <int DT, bool kBack, bool kU> void launch_pairing(const HeadArgs& a, int pairing, bool full, dim3 grid, cudaStream_t st) {
  switch (pairing) {
    case P_NONE: launch_lanes<DT, P_NONE, kBack, kU>(a, full, grid, st); break;
    case P_NEIGHBOURS: launch_lanes<DT, P_NEIGHBOURS, kBack, kU>(a, full, grid, st); break;
    case P_HALVES: launch_lanes<DT, P_HALVES, kBack, kU>(a, full, grid, st); break;
    default: launch_lanes<DT, P_ANY, kBack, kU>(a, full, grid, st);
  }
}

template <bool kBack> cudaError_t launch(HeadArgs& a, const Step& s, int jobs, dim3 grid, cudaStream_t st) {
  const std::vector<double>& n = s.num;
  a.lanes = 1;
  while (a.lanes * 8 < a.width) a.lanes *= 2;
  int pairing = P_NONE;
  if (a.pos) {
    a.dims = (int)n[hn::DIMS];
    a.amplitude = (float)n[hn::AMPLITUDE];
    std::copy(s.freq.begin(), s.freq.end(), a.freq);
    pairing = n[hn::INTERLEAVED] != 0.0 ? P_NEIGHBOURS : a.dims % 8 == 0 ? P_HALVES : P_ANY;
  }
  bool all[2] = {true, true}, with_u = false, full = a.lanes * 8 == a.width;      // every tensor is f32, is bf16
  for (int j = 0; j < jobs; ++j) {
    const HeadJob& b = a.job[j];
    with_u |= b.u || b.round_u;
    full &= b.heads % (32 / a.lanes) == 0;
    for (int t = 0; t < 2; ++t) {
      const int type = t ? DRAGON_BF16 : DRAGON_F32;
      all[t] &= (!b.x || b.xt == type) && (!b.y || b.yt == type) && (!kBack || b.dyt == type);
    }
  }
  if (!kBack && with_u) launch_pairing<-1, false, true>(a, pairing, full, grid, st);
  else if (all[1]) launch_pairing<DRAGON_BF16, kBack, false>(a, pairing, full, grid, st);
  else if (all[0]) launch_pairing<DRAGON_F32, kBack, false>(a, pairing, full, grid, st);
  else launch_pairing<-1, kBack, false>(a, pairing, full, grid, st);
  return cudaGetLastError();
}

}  // namespace

int head_bwd_partials(const Step& s, const std::vector<MemRef>& mems, int sm_count) { return head_tiles(s, mems, hb::DY, hb::READS, sm_count).grid; }

cudaError_t launch_head(const StepRun& r) {
  const Step& s = r.s;
  const Shape& sh = r.mems[s.rd[hd::X]].shape;
  HeadArgs a = {};
  a.width = (int)s.num[hn::WIDTH];
  a.rows = (int)sh.d[0];
  const int jobs = (int)s.rd.size() / hd::READS;
  bool rotated = false;
  for (int j = 0; j < jobs; ++j) {
    HeadJob& b = a.job[j];
    const int rd = hd::READS * j, wr = hd::WRITES * j;
    b.x = r.rd(rd + hd::X); b.xt = r.rd_type(rd + hd::X);
    b.gain = r.rd(rd + hd::GAIN); b.gt = r.rd_type(rd + hd::GAIN);
    b.u = r.wr(wr + hd::U); b.ut = r.wr_type(wr + hd::U);
    b.y = r.wr(wr + hd::Y); b.yt = r.wr_type(wr + hd::Y);
    rotated = b.y != nullptr;      // (steps are joined only where all of them rotate, or none does)
    if (!b.y) { b.y = b.u; b.yt = b.ut; b.u = nullptr; }      // the norm alone writes its result as the last step
    b.round_u = rotated && s.head_round[j] == DRAGON_BF16;
    b.eps = s.head_eps[j];
    b.heads = (int)(r.mems[s.rd[rd + hd::X]].shape.d[1] / a.width);
  }
  a.pos = rotated ? reinterpret_cast<const int*>(r.rd(hd::POS)) : nullptr;
  a.status_clear = r.status_clear;
  const HeadTiles t = head_tiles(s, r.mems, hd::X, hd::READS, r.sm_count);
  a.tile = t.tile;
  return launch<false>(a, s, jobs, dim3(t.grid, jobs), reinterpret_cast<cudaStream_t>(r.stream));
}

cudaError_t launch_head_bwd(const StepRun& r) {
  const Step& s = r.s;
  const Shape& sh = r.mems[s.rd[hb::DY]].shape;
  HeadArgs a = {};
  FinishArgs f = {};
  a.width = f.width = (int)s.num[hn::WIDTH];
  a.rows = (int)sh.d[0];
  const int jobs = (int)s.rd.size() / hb::READS;
  const HeadTiles t = head_tiles(s, r.mems, hb::DY, hb::READS, r.sm_count);
  const int grid = t.grid;
  int sums = 0;
  for (int j = 0; j < jobs; ++j) {
    HeadJob& b = a.job[j];
    const int rd = hb::READS * j, wr = hb::WRITES * j;
    b.x = r.rd(rd + hb::X); b.xt = r.rd_type(rd + hb::X);
    b.gain = r.rd(rd + hb::GAIN); b.gt = r.rd_type(rd + hb::GAIN);
    b.dy = r.rd(rd + hb::DY); b.dyt = r.rd_type(rd + hb::DY);
    b.y = r.wr(wr + hb::DX); b.yt = r.wr_type(wr + hb::DX);
    b.eps = s.head_eps[j];
    b.heads = (int)(r.mems[s.rd[rd + hb::DY]].shape.d[1] / a.width);
    if (s.wr[wr + hb::DGAIN] >= 0) {
      b.dgain = reinterpret_cast<float*>(r.ws + s.colpart_off) + (size_t)j * grid * a.width;
      f.part[sums] = b.dgain;
      f.out[sums] = r.wr(wr + hb::DGAIN);
      f.type[sums++] = r.wr_type(wr + hb::DGAIN);
    }
  }
  a.pos = reinterpret_cast<const int*>(r.rd(hb::POS));
  a.status_clear = r.status_clear;
  a.tile = t.tile;
  cudaStream_t st = reinterpret_cast<cudaStream_t>(r.stream);
  const cudaError_t e = launch<true>(a, s, jobs, dim3(grid, jobs), st);
  if (e != cudaSuccess || !sums) return e;
  f.n = grid;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((a.width + 31) / 32, sums);
  cfg.blockDim = dim3(1024);
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, head_finish, f);
}

}  // namespace dragon
