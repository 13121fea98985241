// The 2-norm over many tensors, and every tensor times min(1, limit / norm).
//   norm = sqrt(sum_i sum_e t_i[e]^2),  c_i = t_i * (norm > limit ? limit / norm : 1)
// Bound: bytes (every tensor read for the norm, then read and written; read once where all of them fit the registers of the
// GPU, 19 MB).  All tensors are one list of chunks that persistent CTAs walk, so that a launch takes any mix of sizes; the
// addresses travel in the launch's parameters.  Measured, 393M bf16 in 49 tensors: norm 144 us (5.5 TB/s read), clipping 259 us
// (6.1 TB/s, what L2 holds of the norm's last reads included); 0.65M fp32 in 5 tensors, both in one launch: 8 us, of which the
// launch and the barrier are nearly all.
// Squares are added in fp32 over the 16 or 32 elements a thread holds at a time and in fp64 beyond; elements whose squares
// could leave fp32's range are squared in fp64.  The order of the sums is fixed, so the norm is the same in every run.
#include <cooperative_groups.h>

#include <algorithm>

#include "device_util.h"
#include "plan.h"

namespace dragon {
namespace {

constexpr int kThreads = 256;
constexpr int kChunkBytes = 4 * 16 * kThreads;     // four accesses of 16 bytes a thread
constexpr int kCtasPerSm = 4;
__host__ __device__ constexpr int chunk_elements(bool f32) { return kChunkBytes / (f32 ? 4 : 2); }

// the tensors of a launch, in its parameters; a short form for few tensors (parameters are copied at every launch)
template <int kMost> struct TensorListOf {
  const void* src[kMost];
  void* dst[kMost];
  long long n[kMost];
  int first[kMost + 1];                            // first chunk of each tensor
  unsigned char dtype[kMost];
  int count;
};
constexpr int kFewTensors = 24;

struct NormOut {
  double* part;                                    // one partial sum per CTA of every launch
  int part_first, part_total;                      // this launch's place, and how many there are when it is done
  bool last_launch;
  float* norm;
  float* factor;
  float limit;
  int* status_clear;
};

// A CTA takes every gridDim.x-th chunk of the list, so that the CTAs together read one place after another.  Walked upwards
// by the norm and downwards by the clipping: what the norm read last is what L2 still holds.  What the chunk's tensor is like
// is looked up when the walk comes to another tensor.
struct Walk {
  int c, left, step;           // chunk, chunks that come after it plus one, distance of the next
  int k, lo, hi;               // its tensor, that tensor's chunks
  const void* src;
  void* dst;
  long long n, first;          // the tensor's elements, the chunk's first one
  int sdt, ddt;
  template <typename TensorList> __device__ __forceinline__ Walk(const TensorList& t, int dir) {
    const int chunks = t.first[t.count], mine = (int)blockIdx.x < chunks ? (chunks - 1 - (int)blockIdx.x) / (int)gridDim.x + 1 : 0;
    left = mine;
    step = dir * (int)gridDim.x;
    c = (int)blockIdx.x + (dir > 0 ? 0 : max(mine - 1, 0) * (int)gridDim.x);
    int a = 0, b = t.count - 1;                    // the last tensor whose first chunk is not behind c
    while (a < b) {
      const int mid = (a + b + 1) >> 1;
      if (t.first[mid] <= c) a = mid; else b = mid - 1;
    }
    k = a;
    look_up(t);
  }
  template <typename TensorList> __device__ __forceinline__ void look_up(const TensorList& t) {
    lo = t.first[k];
    hi = t.first[k + 1];
    src = t.src[k];
    dst = t.dst[k];
    n = t.n[k];
    sdt = t.dtype[k] & 15;
    ddt = t.dtype[k] >> 4;
    first = (long long)(c - lo) * chunk_elements(f32());
  }
  __device__ __forceinline__ bool f32() const { return sdt == DRAGON_F32; }
  __device__ __forceinline__ bool more() const { return left > 0; }
  template <typename TensorList> __device__ __forceinline__ void next(const TensorList& t) {
    c += step;
    if (--left <= 0) return;
    if (c >= lo && c < hi) { first += (long long)step * chunk_elements(f32()); return; }
    while (c >= t.first[k + 1]) ++k;
    while (c < t.first[k]) --k;
    look_up(t);
  }
};

// A chunk of a tensor as it is in memory: four accesses of 16 bytes a thread, 4 or 8 elements each.  What is behind the
// tensor's last whole access reads as zeros and is handled by itself.
struct Chunk {
  uint4 u[4];
  template <bool kKeep> __device__ __forceinline__ void load(const void* src, bool f32, long long first, long long n) {
    const int per = f32 ? 4 : 8;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const long long i = first + (k * kThreads + (int)threadIdx.x) * per;
      u[k] = make_uint4(0, 0, 0, 0);
      if (i + per <= n) {
        const uint4* p = reinterpret_cast<const uint4*>(reinterpret_cast<const char*>(src) + i * (f32 ? 4 : 2));
        u[k] = kKeep ? __ldg(p) : __ldcs(p);
      }
    }
  }
};
__device__ __forceinline__ void values_of(uint4 a, float (&v)[4]) { v[0] = __uint_as_float(a.x); v[1] = __uint_as_float(a.y); v[2] = __uint_as_float(a.z); v[3] = __uint_as_float(a.w); }
__device__ __forceinline__ void values_of(uint4 a, float (&v)[8]) {
  v[0] = bf16_low(a.x); v[1] = bf16_high(a.x); v[2] = bf16_low(a.y); v[3] = bf16_high(a.y);
  v[4] = bf16_low(a.z); v[5] = bf16_high(a.z); v[6] = bf16_low(a.w); v[7] = bf16_high(a.w);
}
// the elements behind the last whole access of a tensor, if the chunk that starts at `first` holds them: this thread's, or none
__device__ __forceinline__ bool tail_element(bool f32, long long first, long long n, long long* i) {
  const int per = f32 ? 4 : 8;
  *i = n / per * per + threadIdx.x;
  return *i < n && *i >= first && *i < first + chunk_elements(f32);
}

__device__ __forceinline__ float factor_of(float norm, float limit) { return norm > limit ? limit / norm : (norm == norm ? 1.f : norm); }

// sum of the squares of N values
template <int N> __device__ __forceinline__ double squares(const float* v) {
  unsigned m = 0;
  float s = 0.f;
#pragma unroll
  for (int e = 0; e < N; ++e) { m = max(m, magnitude(v[e])); s += v[e] * v[e]; }
  // the largest magnitude in [2^-40, 2^60]: no square overflows, and one that underflows is below 2^-46 of the sum
  if (m == 0 || (m >= 0x2b800000u && m <= 0x5d800000u)) return (double)s;
  double d = 0.0;
#pragma unroll
  for (int e = 0; e < N; ++e) d += (double)v[e] * (double)v[e];
  return d;
}
// ... of 32 bf16 in 16 words, two at a time
__device__ __forceinline__ double squares_of_bf16(const uint4 (&u)[4]) {
  const unsigned* w = reinterpret_cast<const unsigned*>(u);
  unsigned m = 0;
  unsigned long long s = 0;
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    m = __vmaxu2(m, w[i] & 0x7fff7fffu);
    unsigned long long v;
    asm("mov.b64 %0, {%1, %2};" : "=l"(v) : "f"(bf16_low(w[i])), "f"(bf16_high(w[i])));
    asm("fma.rn.f32x2 %0, %1, %1, %0;" : "+l"(s) : "l"(v));
  }
  m = max(m & 0xffffu, m >> 16);
  float a, b;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(s));
  if (m == 0 || (m >= 0x2b80u && m <= 0x5d80u)) return (double)(a + b);
  double d = 0.0;
#pragma unroll
  for (int i = 0; i < 16; ++i) d += (double)bf16_low(w[i]) * (double)bf16_low(w[i]) + (double)bf16_high(w[i]) * (double)bf16_high(w[i]);
  return d;
}
__device__ __forceinline__ double chunk_squares(const Chunk& ch, const void* src, bool f32, long long first, long long n) {
  double d;
  if (f32) {
    float v[4][4];
#pragma unroll
    for (int j = 0; j < 4; ++j) values_of(ch.u[j], v[j]);
    d = squares<16>(v[0]);
  } else {
    d = squares_of_bf16(ch.u);
  }
  long long i;
  if (tail_element(f32, first, n, &i)) {
    float x;
    load_any<1>(src, f32 ? DRAGON_F32 : DRAGON_BF16, i, &x);
    d += squares<1>(&x);
  }
  return d;
}

__device__ __forceinline__ double block_sum(double v, double* sh) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  if ((threadIdx.x & 31) == 0) sh[threadIdx.x >> 5] = v;
  __syncthreads();
  double r = sh[0];
#pragma unroll
  for (int i = 1; i < kThreads / 32; ++i) r += sh[i];
  __syncthreads();
  return r;
}

// The grid-wide barriers here and in norm_and_clip_kernel are those of a cooperative launch: all CTAs run at once, so every wait
// ends, and nothing in the caller's workspace has to be zero before a run (it may have served another function in between).
template <typename TensorList> __global__ void __launch_bounds__(kThreads, kCtasPerSm) global_norm_kernel(const __grid_constant__ TensorList t, const NormOut o) {
  __shared__ double sh[kThreads / 32];
  if (o.status_clear && blockIdx.x == 0 && threadIdx.x == 0) *o.status_clear = 0;
  double sum = 0.0;
  Walk w(t, 1);
  Chunk next;
  if (w.more()) next.load<true>(w.src, w.f32(), w.first, w.n);
  while (w.more()) {
    const Chunk now = next;
    const Walk here = w;
    w.next(t);
    if (w.more()) next.load<true>(w.src, w.f32(), w.first, w.n);
    sum += chunk_squares(now, here.src, here.f32(), here.first, here.n);
  }
  sum = block_sum(sum, sh);
  if (threadIdx.x == 0) __stcg(o.part + o.part_first + blockIdx.x, sum);
  if (!o.last_launch) return;
  cooperative_groups::this_grid().sync();
  if (blockIdx.x != 0) return;
  // one CTA adds all partial sums, in their order
  double total = 0.0;
  for (int i = threadIdx.x; i < o.part_total; i += kThreads) total += __ldcg(o.part + i);
  total = block_sum(total, sh);
  if (threadIdx.x == 0) {
    const float norm = (float)sqrt(total);
    if (o.norm) *o.norm = norm;
    if (o.factor) *o.factor = factor_of(norm, o.limit);
  }
}

// a chunk times f, in the type of its destination
__device__ __forceinline__ void store_clipped(const Chunk& now, const void* src, int sdt, void* dst, int ddt, long long first, long long n, float f) {
  const bool f32 = sdt == DRAGON_F32;
  if (f32) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const long long i = first + (j * kThreads + (int)threadIdx.x) * 4;
      float v[4];
      values_of(now.u[j], v);
      if (i + 4 > n) continue;
      if (ddt == DRAGON_F32) *reinterpret_cast<float4*>(reinterpret_cast<float*>(dst) + i) = make_float4(v[0] * f, v[1] * f, v[2] * f, v[3] * f);
      else *reinterpret_cast<uint2*>(reinterpret_cast<unsigned short*>(dst) + i) = make_uint2(bf16_pair(v[0] * f, v[1] * f), bf16_pair(v[2] * f, v[3] * f));
    }
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const long long i = first + (j * kThreads + (int)threadIdx.x) * 8;
      float v[8];
      values_of(now.u[j], v);
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] *= f;
      if (i + 8 <= n) store_any<8>(dst, ddt, i, v);
    }
  }
  long long i;
  if (tail_element(f32, first, n, &i)) {
    float v;
    load_any<1>(src, sdt, i, &v);
    v *= f;
    store_any<1>(dst, ddt, i, &v);
  }
}

// Norm and clipping in one cooperative launch, for tensors of which every CTA holds its whole share (kHeld chunks) in
// registers: read once, summed, and after a grid-wide barrier scaled and written.
constexpr int kHeld = 2;
template <typename TensorList> __global__ void __launch_bounds__(kThreads, kCtasPerSm) norm_and_clip_kernel(const __grid_constant__ TensorList t, const NormOut o) {
  __shared__ double sh[kThreads / 32];
  if (o.status_clear && blockIdx.x == 0 && threadIdx.x == 0) *o.status_clear = 0;
  Chunk held[kHeld];
  Walk w(t, 1);
  int tensor[kHeld];
  long long first[kHeld];
#pragma unroll
  for (int h = 0; h < kHeld; ++h) {
    tensor[h] = -1;
    if (!w.more()) continue;
    tensor[h] = w.k;
    first[h] = w.first;
    held[h].load<false>(w.src, w.f32(), w.first, w.n);
    w.next(t);
  }
  double sum = 0.0;
#pragma unroll
  for (int h = 0; h < kHeld; ++h)
    if (tensor[h] >= 0) sum += chunk_squares(held[h], t.src[tensor[h]], (t.dtype[tensor[h]] & 15) == DRAGON_F32, first[h], t.n[tensor[h]]);
  // the elements behind the last whole access are read again when they are written: before the barrier nobody writes
  sum = block_sum(sum, sh);
  if (threadIdx.x == 0) __stcg(o.part + blockIdx.x, sum);
  cooperative_groups::this_grid().sync();
  double total = 0.0;
  for (int i = threadIdx.x; i < (int)gridDim.x; i += kThreads) total += __ldcg(o.part + i);
  total = block_sum(total, sh);
  const float norm = (float)sqrt(total), f = factor_of(norm, o.limit);
  if (threadIdx.x == 0 && blockIdx.x == 0) {
    *o.norm = norm;
    if (o.factor) *o.factor = f;
  }
#pragma unroll
  for (int h = 0; h < kHeld; ++h) {
    const int k = tensor[h];
    if (k < 0 || (f == 1.f && t.src[k] == t.dst[k])) continue;
    store_clipped(held[h], t.src[k], t.dtype[k] & 15, t.dst[k], t.dtype[k] >> 4, first[h], t.n[k], f);
  }
}

template <typename TensorList> __global__ void __launch_bounds__(kThreads, kCtasPerSm) clip_kernel(const __grid_constant__ TensorList t, const float* norm, float limit, int* status_clear) {
  if (status_clear && blockIdx.x == 0 && threadIdx.x == 0) *status_clear = 0;
  const float f = factor_of(__ldg(norm), limit);
  Walk w(t, -1);
  Chunk next;
  auto load = [&] {
    if (w.more() && !(f == 1.f && w.src == w.dst)) next.load<false>(w.src, w.f32(), w.first, w.n);
  };
  load();
  while (w.more()) {
    const Chunk now = next;
    const Walk here = w;
    w.next(t);
    load();
    if (f == 1.f && here.src == here.dst) continue;      // in place and nothing to change
    store_clipped(now, here.src, here.sdt, here.dst, here.ddt, here.first, here.n, f);
  }
}

__global__ void clip_factor_kernel(const float* norm, float limit, float* factor, int* status_clear) {
  if (status_clear) *status_clear = 0;
  *factor = factor_of(*norm, limit);
}

// chunk table of tensors [k0, k1); false if a launch cannot hold it
template <typename TensorList> bool add_tensor(TensorList* t, const void* src, void* dst, int sdt, int ddt, int64_t n) {
  const int i = t->count;
  const int per = chunk_elements(sdt == DRAGON_F32);
  const int64_t chunks = (n + per - 1) / per;
  if ((int64_t)t->first[i] + chunks > 0x3fffffffLL) return false;
  t->src[i] = src;
  t->dst[i] = dst;
  t->n[i] = n;
  t->dtype[i] = (unsigned char)(sdt | (ddt << 4));
  t->first[i + 1] = t->first[i] + (int)chunks;
  ++t->count;
  return true;
}

}  // namespace

size_t global_norm_scratch_bytes(int n_tensors, int sm_count) { return (size_t)launches_of_tensors(n_tensors) * sm_count * kCtasPerSm * sizeof(double); }

bool norm_and_clip_fit_one_launch(const std::vector<int64_t>& numel, const std::vector<int>& dtype, int sm_count) {
  if ((int)numel.size() > kTensorsPerLaunch) return false;
  int64_t chunks = 0;
  for (size_t i = 0; i < numel.size(); ++i) {
    const int per = chunk_elements(dtype[i] == DRAGON_F32);
    chunks += (numel[i] + per - 1) / per;
  }
  return chunks <= (int64_t)sm_count * kCtasPerSm * kHeld;
}

namespace {

template <typename TensorList> cudaError_t launch(void (*kernel)(TensorList, NormOut), int grid, bool cooperative, cudaStream_t st, const TensorList& t, const NormOut& o) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(grid);
  cfg.blockDim = dim3(kThreads);
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeCooperative;
  attr[0].val.cooperative = 1;
  cfg.attrs = attr;
  cfg.numAttrs = cooperative ? 1 : 0;
  return cudaLaunchKernelEx(&cfg, kernel, t, o);
}

template <int kMost> cudaError_t global_norm_of(const StepRun& r, cudaStream_t st) {
  const int n = (int)r.s.rd.size(), launches = launches_of_tensors(n);
  NormOut o{reinterpret_cast<double*>(r.ws + r.s.scratch_off), 0, 0, false, reinterpret_cast<float*>(r.wr(gn::NORM)), reinterpret_cast<float*>(r.wr(gn::FACTOR)),
            (float)r.s.attr, r.status_clear};
  for (int l = 0; l < launches; ++l) {
    TensorListOf<kMost> t;
    t.count = 0;
    t.first[0] = 0;
    for (int k = l * kTensorsPerLaunch; k < std::min(n, (l + 1) * kTensorsPerLaunch); ++k)
      if (!add_tensor(&t, r.rd(k), nullptr, r.rd_type(k), 0, r.mems[r.s.rd[k]].shape.numel())) return cudaErrorInvalidValue;
    const int grid = std::min(t.first[t.count], r.sm_count * kCtasPerSm);
    o.part_first = o.part_total;
    o.part_total += grid;
    o.last_launch = l + 1 == launches;
    const cudaError_t e = launch(global_norm_kernel<TensorListOf<kMost>>, grid, o.last_launch, st, t, o);
    if (e != cudaSuccess) return e;
    o.status_clear = nullptr;
  }
  return cudaSuccess;
}

template <int kMost> cudaError_t clip_of(const StepRun& r, cudaStream_t st) {
  const int n = (int)r.s.wr.size();
  int* clear = r.status_clear;
  for (int k0 = 0; k0 < n; k0 += kTensorsPerLaunch) {
    TensorListOf<kMost> t;
    t.count = 0;
    t.first[0] = 0;
    for (int k = k0; k < std::min(n, k0 + kTensorsPerLaunch); ++k) {
      if (r.s.wr[k] < 0) continue;
      if (!add_tensor(&t, r.rd(cl::FIRST + k), r.wr(k), r.rd_type(cl::FIRST + k), r.wr_type(k), r.mems[r.s.rd[cl::FIRST + k]].shape.numel())) return cudaErrorInvalidValue;
    }
    if (!t.count) continue;
    clip_kernel<<<std::min(t.first[t.count], r.sm_count * kCtasPerSm), kThreads, 0, st>>>(t, reinterpret_cast<const float*>(r.rd(cl::NORM)), (float)r.s.attr, clear);
    clear = nullptr;
  }
  return cudaGetLastError();
}

template <int kMost> cudaError_t norm_and_clip_of(const StepRun& r, cudaStream_t st) {
  TensorListOf<kMost> t;
  t.count = 0;
  t.first[0] = 0;
  for (int k = 0; k < (int)r.s.rd.size(); ++k)
    if (!add_tensor(&t, r.rd(k), r.wr(gn::CLIPPED + k), r.rd_type(k), r.wr_type(gn::CLIPPED + k), r.mems[r.s.rd[k]].shape.numel())) return cudaErrorInvalidValue;
  const NormOut o{reinterpret_cast<double*>(r.ws + r.s.scratch_off), 0, 0, true, reinterpret_cast<float*>(r.wr(gn::NORM)), reinterpret_cast<float*>(r.wr(gn::FACTOR)),
                  (float)r.s.attr, r.status_clear};
  // no more CTAs than hold their share: at most kHeld chunks each, and all of them on the GPU at once
  return launch(norm_and_clip_kernel<TensorListOf<kMost>>, std::min(t.first[t.count], r.sm_count * kCtasPerSm), true, st, t, o);
}

}  // namespace

cudaError_t launch_global_norm(const StepRun& r) {
  cudaStream_t st = reinterpret_cast<cudaStream_t>(r.stream);
  return r.s.rd.size() <= kFewTensors ? global_norm_of<kFewTensors>(r, st) : global_norm_of<kTensorsPerLaunch>(r, st);
}

cudaError_t launch_clip_factor(const StepRun& r) {
  clip_factor_kernel<<<1, 1, 0, reinterpret_cast<cudaStream_t>(r.stream)>>>(reinterpret_cast<const float*>(r.rd(0)), (float)r.s.attr, reinterpret_cast<float*>(r.wr(0)), r.status_clear);
  return cudaGetLastError();
}

cudaError_t launch_clip(const StepRun& r) {
  cudaStream_t st = reinterpret_cast<cudaStream_t>(r.stream);
  return r.s.wr.size() <= kFewTensors ? clip_of<kFewTensors>(r, st) : clip_of<kTensorsPerLaunch>(r, st);
}

cudaError_t launch_norm_and_clip(const StepRun& r) {
  cudaStream_t st = reinterpret_cast<cudaStream_t>(r.stream);
  return r.s.rd.size() <= kFewTensors ? norm_and_clip_of<kFewTensors>(r, st) : norm_and_clip_of<kTensorsPerLaunch>(r, st);
}

}  // namespace dragon
