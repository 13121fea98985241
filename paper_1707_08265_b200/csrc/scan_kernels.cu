// Gated linear recurrence over packed sequences, and its gradient.
//   h[t] = f[t] h[t-1] + (1 - f[t]) x[t],  f = sigmoid(gate);   h[-1] = the sequence's row of h0 (or 0); a row with reset
//   starts from 0.
//   D[t] = dh[t] + f[t+1] D[t+1] (nothing from a row that starts afresh);  dx = (1 - f) D,  dgate = D (h[t-1] - x) f (1 - f),
//   dh0 = f[0] D[0].
// The state is fp32.
#include <algorithm>

#include "device_util.h"
#include "plan.h"

namespace dragon {
namespace {

struct ScanArgs {
  const void *gate, *x, *h0, *dh;
  const int* reset;
  void *h, *dgate, *dx, *dh0;
  float* carry;            // state in front of each tile of kScanTileRows rows
  int gdt, xdt, h0dt, dhdt, hdt, dgdt, dxdt, dh0dt;
  int rows, cols, length;  // length: rows per sequence
  int* status_clear;
};

// f and 1 - f = exp(-z) f, each to full relative precision; exp(-z) is kept finite (a comparison with NaN is false)
__device__ __forceinline__ void gate_of(float z, float* f, float* keep) {
  float u = -z * 1.4426950408889634f;
  u = u > 126.f ? 126.f : u;
  const float t = exp2f(u);
  *f = __fdividef(1.f, 1.f + t);
  *keep = t * *f;
}

__global__ void __launch_bounds__(128) scan_simple_kernel(const ScanArgs a, int seqs) {
  if (a.status_clear && blockIdx.x == 0 && threadIdx.x == 0) *a.status_clear = 0;
  const long long i = (long long)blockIdx.x * 128 + threadIdx.x;
  if (i >= (long long)seqs * a.cols) return;
  const long long q = i / a.cols;
  const int c = (int)(i - q * a.cols);
  float h = 0.f;
  if (a.h0) load_any<1>(a.h0, a.h0dt, (size_t)q * a.cols + c, &h);
  for (int l = 0; l < a.length; ++l) {
    const size_t row = (size_t)q * a.length + l, at = row * a.cols + c;
    if (a.carry && row % kScanTileRows == 0) a.carry[row / kScanTileRows * a.cols + c] = h;
    if (a.reset && a.reset[row]) h = 0.f;
    float z, x, f, keep;
    load_any<1>(a.gate, a.gdt, at, &z);
    load_any<1>(a.x, a.xdt, at, &x);
    gate_of(z, &f, &keep);
    h = f * h + keep * x;
    if (a.h) store_any<1>(a.h, a.hdt, at, &h);
  }
}

__global__ void __launch_bounds__(128) scan_bwd_simple_kernel(const ScanArgs a, int seqs) {
  if (a.status_clear && blockIdx.x == 0 && threadIdx.x == 0) *a.status_clear = 0;
  const long long i = (long long)blockIdx.x * 128 + threadIdx.x;
  if (i >= (long long)seqs * a.cols) return;
  const long long q = i / a.cols;
  const int c = (int)(i - q * a.cols);
  float d = 0.f;     // f[t+1] D[t+1], or 0
  float hp[kScanTileRows];
  const long long first = q * a.length;
  long long last = first + a.length - 1;
  while (last >= first) {
    const long long tile = std::max<long long>(last / kScanTileRows * kScanTileRows, first);
    float h = 0.f;
    if (tile == first) { if (a.h0) load_any<1>(a.h0, a.h0dt, (size_t)q * a.cols + c, &h); }
    else h = a.carry[tile / kScanTileRows * a.cols + c];
    for (long long row = tile; row <= last; ++row) {
      const size_t at = (size_t)row * a.cols + c;
      float z, x, f, keep;
      load_any<1>(a.gate, a.gdt, at, &z);
      load_any<1>(a.x, a.xdt, at, &x);
      gate_of(z, &f, &keep);
      if (a.reset && a.reset[row]) h = 0.f;
      hp[row - tile] = h;
      h = f * h + keep * x;
    }
    for (long long row = last; row >= tile; --row) {
      const size_t at = (size_t)row * a.cols + c;
      float z, x, g, f, keep;
      load_any<1>(a.gate, a.gdt, at, &z);
      load_any<1>(a.x, a.xdt, at, &x);
      load_any<1>(a.dh, a.dhdt, at, &g);
      gate_of(z, &f, &keep);
      d += g;
      const float dx = d * keep, dz = d * (hp[row - tile] - x) * (f * keep);
      if (a.dx) store_any<1>(a.dx, a.dxdt, at, &dx);
      if (a.dgate) store_any<1>(a.dgate, a.dgdt, at, &dz);
      d = (a.reset && a.reset[row]) ? 0.f : f * d;
    }
    last = tile - 1;
  }
  if (a.dh0) store_any<1>(a.dh0, a.dh0dt, (size_t)q * a.cols + c, &d);
}

ScanArgs scan_args(const StepRun& r, bool backward) {
  const Shape& sh = r.mems[r.s.rd[sc::GATE]].shape;
  ScanArgs a{};
  a.gate = r.rd(sc::GATE); a.x = r.rd(sc::X); a.h0 = r.rd(sc::H0); a.reset = reinterpret_cast<const int*>(r.rd(sc::RESET));
  a.gdt = r.rd_type(sc::GATE); a.xdt = r.rd_type(sc::X); a.h0dt = r.rd_type(sc::H0);
  a.rows = (int)sh.d[0];
  a.cols = (int)sh.d[1];
  a.length = (int)(sh.d[0] / (int64_t)r.s.attr);
  a.status_clear = r.status_clear;
  if (backward) {
    a.dh = r.rd(sc::DH); a.dhdt = r.rd_type(sc::DH);
    a.carry = reinterpret_cast<float*>(r.rd(sc::CARRY_IN));
    a.dgate = r.wr(sc::DGATE); a.dx = r.wr(sc::DX); a.dh0 = r.wr(sc::DH0);
    a.dgdt = r.wr_type(sc::DGATE); a.dxdt = r.wr_type(sc::DX); a.dh0dt = r.wr_type(sc::DH0);
  } else {
    a.h = r.wr(sc::H); a.hdt = r.wr_type(sc::H);
    a.carry = reinterpret_cast<float*>(r.wr(sc::CARRY));
  }
  return a;
}

}  // namespace

size_t scan_scratch_bytes(int64_t rows, int64_t cols) { return 0 * rows * cols; }

cudaError_t launch_scan(const StepRun& r) {
  const ScanArgs a = scan_args(r, false);
  const long long n = (long long)r.s.attr * a.cols;
  scan_simple_kernel<<<(unsigned)((n + 127) / 128), 128, 0, reinterpret_cast<cudaStream_t>(r.stream)>>>(a, (int)r.s.attr);
  return cudaGetLastError();
}

cudaError_t launch_scan_bwd(const StepRun& r) {
  const ScanArgs a = scan_args(r, true);
  const long long n = (long long)r.s.attr * a.cols;
  scan_bwd_simple_kernel<<<(unsigned)((n + 127) / 128), 128, 0, reinterpret_cast<cudaStream_t>(r.stream)>>>(a, (int)r.s.attr);
  return cudaGetLastError();
}

}  // namespace dragon
