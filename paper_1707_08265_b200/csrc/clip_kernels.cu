// The 2-norm over many tensors, and every tensor times min(1, limit / norm).
//   norm = sqrt(sum_i sum_e t_i[e]^2),  c_i = t_i * (norm > limit ? limit / norm : 1)
// Bound: bytes (every tensor read for the norm, then read and written).  All tensors are one list of chunks that
// persistent CTAs walk, so that a launch takes any mix of sizes; the addresses travel in the launch's parameters.
// Squares are added in fp32 over the 32 elements a thread holds at a time and in fp64 beyond; elements whose squares
// could leave fp32's range are squared in fp64.  The order of the sums is fixed, so the norm is the same in every run.
#include <algorithm>

#include "device_util.h"
#include "plan.h"

namespace dragon {
namespace {

constexpr int kThreads = 256;
constexpr int kChunk = 8192;                       // elements: 32 per thread
constexpr int kCtasPerSm = 4;

struct TensorList {
  const void* src[kTensorsPerLaunch];
  void* dst[kTensorsPerLaunch];
  long long n[kTensorsPerLaunch];
  int first[kTensorsPerLaunch + 1];                // first chunk of each tensor
  unsigned char dtype[kTensorsPerLaunch];
  int count;
};

struct NormOut {
  double* part;                                    // one partial sum per CTA of every launch
  int part_first, part_total;                      // this launch's place, and how many there are when it is done
  bool last_launch;
  float* norm;
  float* factor;
  float limit;
  unsigned* counter;
  int* status_clear;
};

__device__ __forceinline__ int tensor_of_chunk(const TensorList& t, int c) {
  int lo = 0, hi = t.count - 1;                    // the last tensor whose first chunk is not behind c
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (t.first[mid] <= c) lo = mid; else hi = mid - 1;
  }
  return lo;
}

__device__ __forceinline__ float factor_of(float norm, float limit) { return norm > limit ? limit / norm : (norm == norm ? 1.f : norm); }

template <int DT>
__device__ __forceinline__ double chunk_squares(const void* src, long long first, long long n) {
  float v[32];
  Raw<DT, 8> raw[4];
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const long long i = first + (k * kThreads + (int)threadIdx.x) * 8;
    if (i + 8 <= n) raw[k].load(src, i);
  }
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const long long i = first + (k * kThreads + (int)threadIdx.x) * 8;
    if (i + 8 <= n) raw[k].get(v + 8 * k);
    else
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        v[8 * k + e] = 0.f;
        if (i + e < n) { Raw<DT, 1> one; one.load(src, i + e); one.get(v + 8 * k + e); }
      }
  }
  unsigned m = 0;
  float s = 0.f;
#pragma unroll
  for (int e = 0; e < 32; ++e) { m = max(m, magnitude(v[e])); s += v[e] * v[e]; }
  // the largest magnitude in [2^-40, 2^60]: no square overflows, and one that underflows is below 2^-46 of the sum
  if (m == 0 || (m >= 0x2b800000u && m <= 0x5d800000u)) return (double)s;
  double d = 0.0;
#pragma unroll
  for (int e = 0; e < 32; ++e) d += (double)v[e] * (double)v[e];
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

__global__ void __launch_bounds__(kThreads) global_norm_kernel(const __grid_constant__ TensorList t, const NormOut o) {
  __shared__ double sh[kThreads / 32];
  __shared__ bool last;
  if (o.status_clear && blockIdx.x == 0 && threadIdx.x == 0) *o.status_clear = 0;
  double sum = 0.0;
  const int n_chunks = t.first[t.count];
  for (int c = blockIdx.x; c < n_chunks; c += gridDim.x) {
    const int k = tensor_of_chunk(t, c);
    const long long first = (long long)(c - t.first[k]) * kChunk;
    sum += t.dtype[k] == DRAGON_F32 ? chunk_squares<DRAGON_F32>(t.src[k], first, t.n[k]) : chunk_squares<DRAGON_BF16>(t.src[k], first, t.n[k]);
  }
  sum = block_sum(sum, sh);
  if (threadIdx.x == 0) {
    o.part[o.part_first + blockIdx.x] = sum;
    __threadfence();
    last = o.last_launch && atomicAdd(o.counter, 1u) == gridDim.x - 1;
  }
  __syncthreads();
  if (!last) return;
  // the last CTA to arrive adds all partial sums, in their order
  __threadfence();
  double total = 0.0;
  for (int i = threadIdx.x; i < o.part_total; i += kThreads) total += __ldcg(o.part + i);
  total = block_sum(total, sh);
  if (threadIdx.x == 0) {
    const float norm = (float)sqrt(total);
    if (o.norm) *o.norm = norm;
    if (o.factor) *o.factor = factor_of(norm, o.limit);
    *o.counter = 0;
  }
}

template <int DT>
__device__ __forceinline__ void clip_chunk(const void* src, void* dst, long long first, long long n, float f) {
  Raw<DT, 8> raw[4];
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const long long i = first + (k * kThreads + (int)threadIdx.x) * 8;
    if (i + 8 <= n) raw[k].load(src, i);
  }
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const long long i = first + (k * kThreads + (int)threadIdx.x) * 8;
    if (i + 8 <= n) {
      float v[8];
      raw[k].get(v);
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] *= f;
      store_any<8>(dst, DT, i, v);
    } else {
      for (int e = 0; e < 8; ++e)
        if (i + e < n) {
          float v;
          Raw<DT, 1> one;
          one.load(src, i + e);
          one.get(&v);
          v *= f;
          store_any<1>(dst, DT, i + e, &v);
        }
    }
  }
}
// the clipped tensor's type may differ from the tensor's
__device__ __forceinline__ void clip_chunk_converting(const void* src, int sdt, void* dst, int ddt, long long first, long long n, float f) {
  for (long long i = first + threadIdx.x; i < n && i < first + kChunk; i += kThreads) {
    float v;
    load_any<1>(src, sdt, i, &v);
    v *= f;
    store_any<1>(dst, ddt, i, &v);
  }
}

__global__ void __launch_bounds__(kThreads) clip_kernel(const __grid_constant__ TensorList t, const float* norm, float limit, int* status_clear) {
  if (status_clear && blockIdx.x == 0 && threadIdx.x == 0) *status_clear = 0;
  const float f = factor_of(__ldg(norm), limit);
  const int n_chunks = t.first[t.count];
  // from the last chunk to the first: what the norm's launch read last is still in L2
  for (int c = n_chunks - 1 - (int)blockIdx.x; c >= 0; c -= gridDim.x) {
    const int k = tensor_of_chunk(t, c);
    const long long first = (long long)(c - t.first[k]) * kChunk;
    const int sdt = t.dtype[k] & 15, ddt = t.dtype[k] >> 4;
    if (f == 1.f && t.src[k] == t.dst[k]) continue;      // in place and nothing to change
    if (sdt != ddt) clip_chunk_converting(t.src[k], sdt, t.dst[k], ddt, first, t.n[k], f);
    else if (sdt == DRAGON_F32) clip_chunk<DRAGON_F32>(t.src[k], t.dst[k], first, t.n[k], f);
    else clip_chunk<DRAGON_BF16>(t.src[k], t.dst[k], first, t.n[k], f);
  }
}

__global__ void clip_factor_kernel(const float* norm, float limit, float* factor, int* status_clear) {
  if (status_clear) *status_clear = 0;
  *factor = factor_of(*norm, limit);
}

// chunk table of tensors [k0, k1); false if a launch cannot hold it
bool add_tensor(TensorList* t, const void* src, void* dst, int sdt, int ddt, int64_t n) {
  const int i = t->count;
  const int64_t chunks = (n + kChunk - 1) / kChunk;
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

cudaError_t launch_global_norm(const StepRun& r) {
  cudaStream_t st = reinterpret_cast<cudaStream_t>(r.stream);
  const int n = (int)r.s.rd.size(), launches = launches_of_tensors(n);
  NormOut o{reinterpret_cast<double*>(r.ws + r.s.scratch_off), 0, 0, false, reinterpret_cast<float*>(r.wr(gn::NORM)), reinterpret_cast<float*>(r.wr(gn::FACTOR)),
            (float)r.s.attr, r.counter, r.status_clear};
  for (int l = 0; l < launches; ++l) {
    TensorList t;
    t.count = 0;
    t.first[0] = 0;
    for (int k = l * kTensorsPerLaunch; k < std::min(n, (l + 1) * kTensorsPerLaunch); ++k)
      if (!add_tensor(&t, r.rd(k), nullptr, r.rd_type(k), 0, r.mems[r.s.rd[k]].shape.numel())) return cudaErrorInvalidValue;
    const int grid = std::min(t.first[t.count], r.sm_count * kCtasPerSm);
    o.part_first = o.part_total;
    o.part_total += grid;
    o.last_launch = l + 1 == launches;
    global_norm_kernel<<<grid, kThreads, 0, st>>>(t, o);
    o.status_clear = nullptr;
  }
  return cudaGetLastError();
}

cudaError_t launch_clip_factor(const StepRun& r) {
  clip_factor_kernel<<<1, 1, 0, reinterpret_cast<cudaStream_t>(r.stream)>>>(reinterpret_cast<const float*>(r.rd(0)), (float)r.s.attr, reinterpret_cast<float*>(r.wr(0)), r.status_clear);
  return cudaGetLastError();
}

cudaError_t launch_clip(const StepRun& r) {
  cudaStream_t st = reinterpret_cast<cudaStream_t>(r.stream);
  const int n = (int)r.s.wr.size();
  int* clear = r.status_clear;
  for (int k0 = 0; k0 < n; k0 += kTensorsPerLaunch) {
    TensorList t;
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

}  // namespace dragon
