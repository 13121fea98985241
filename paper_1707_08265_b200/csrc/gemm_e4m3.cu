// ScaledInnerProduct  Y[m,n] = sum_b sx[m,b] sw[n/128,b] sum_{k in block b} Xq[m,k] Wq[n,k]: e4m3 operands with a scale for
// each block of 128 along K, fp32 accumulation, fp32 or bf16 output.
#include <algorithm>

#include "device_util.h"
#include "plan.h"

namespace dragon {
namespace {

struct Gemm8Args {
  const unsigned char *x, *w;
  const float *sx, *sw;
  void* y;
  int ydt, M, N, K, kb;
  int* status_clear;
};

__device__ __forceinline__ float e4m3_value(unsigned char b) {
  return __half2float(__half(__nv_cvt_fp8_to_halfraw(b, __NV_E4M3)));
}

// 32 x 32 outputs per CTA, one per thread
__global__ void __launch_bounds__(1024) gemm_e4m3_simple_kernel(const Gemm8Args g) {
  __shared__ float xs[32][33], ws[32][33];
  if (g.status_clear && blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0) *g.status_clear = 0;
  const int tx = threadIdx.x & 31, ty = threadIdx.x >> 5;
  const long long m = (long long)blockIdx.y * 32 + ty;
  const int n = blockIdx.x * 32 + tx;
  float acc = 0.f;
  for (int b = 0; b < g.kb; ++b) {
    float part = 0.f;
    for (int k0 = b * 128; k0 < std::min(g.K, (b + 1) * 128); k0 += 32) {
      const int k = k0 + tx;
      const int wn = blockIdx.x * 32 + ty;
      xs[ty][tx] = m < g.M && k < g.K ? e4m3_value(g.x[(size_t)m * g.K + k]) : 0.f;
      ws[ty][tx] = wn < g.N && k < g.K ? e4m3_value(g.w[(size_t)wn * g.K + k]) : 0.f;
      __syncthreads();
      for (int i = 0; i < 32; ++i) part += xs[ty][i] * ws[tx][i];
      __syncthreads();
    }
    if (m < g.M && n < g.N) acc += part * (g.sx[(size_t)m * g.kb + b] * g.sw[(size_t)(n >> 7) * g.kb + b]);
  }
  if (m < g.M && n < g.N) store_any<1>(g.y, g.ydt, (size_t)m * g.N + n, &acc);
}

}  // namespace

int launch_gemm_e4m3(const StepRun& r) {
  const Shape &sx = r.mems[r.s.rd[g8::XQ]].shape, &sw = r.mems[r.s.rd[g8::WQ]].shape;
  Gemm8Args g{reinterpret_cast<const unsigned char*>(r.rd(g8::XQ)), reinterpret_cast<const unsigned char*>(r.rd(g8::WQ)),
              reinterpret_cast<const float*>(r.rd(g8::SX)), reinterpret_cast<const float*>(r.rd(g8::SW)), r.wr(g8::Y), r.wr_type(g8::Y),
              (int)sx.d[0], (int)sw.d[0], (int)sx.d[1], (int)((sx.d[1] + 127) / 128), r.status_clear};
  dim3 grid((g.N + 31) / 32, (g.M + 31) / 32);
  if (grid.y > 65535) { set_error("ScaledInnerProduct: too many rows"); return DRAGON_ERR_UNSUPPORTED; }
  gemm_e4m3_simple_kernel<<<grid, 1024, 0, reinterpret_cast<cudaStream_t>(r.stream)>>>(g);
  const cudaError_t e = cudaGetLastError();
  if (e != cudaSuccess) { set_error("ScaledInnerProduct: launch failed: %s", cudaGetErrorString(e)); return DRAGON_ERR_CUDA; }
  return DRAGON_OK;
}

}  // namespace dragon
