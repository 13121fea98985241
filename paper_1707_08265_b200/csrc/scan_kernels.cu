// Gated linear recurrence over packed sequences, and its gradient.
//   h[t] = f[t] h[t-1] + (1 - f[t]) x[t],  f = sigmoid(gate);   h[-1] = the sequence's row of h0 (or 0); a row with reset
//   starts from 0.
//   D[t] = dh[t] + e[t],  e[t-1] = f[t] D[t] (0 from a row that starts afresh);  dx = (1 - f) D,
//   dgate = D (h[t-1] - x) f (1 - f),  dh0 = f[0] D[0].
// Bound: bytes.  A recurrence h -> f h + b composes: rows r..s act on the state in front of them as h -> A h + B with A the
// product of the f and B the state they reach from 0.  A CTA takes a tile of 128 rows x 64 columns; each of its 16 warps
// folds 8 rows into (A, B) from registers, the warps' pairs are folded through shared memory, and the state in front of the
// tile comes from the tiles before it: a tile publishes its (A, B) as soon as it has it and its end state once it knows its
// start; a tile looks back over published pairs until it meets an end state.  Everything is read once and written once,
// whatever the number of sequences: a long one is spread over the whole GPU.  Tiles are handed out by a counter in time
// order, so a tile waits only for tiles that are running or done; the wait is bounded (DRAGON_ERR_TIMEOUT).
// A row that starts afresh cuts the chain by selection, not by a factor of 0: what is in front of it cannot reach it, NaN
// or not.  The state is fp32; the gradient recomputes it from the state in front of each tile, which the forward keeps.
#include <algorithm>

#include "device_util.h"
#include "plan.h"

namespace dragon {
namespace {

constexpr int kWarps = 16;
constexpr int kRows = kScanTileRows / kWarps;      // rows per warp
constexpr int kThreads = kWarps * 32;
constexpr long long kWaitBudgetCycles = 4000000000LL;   // about two seconds

struct ScanArgs {
  const void *gate, *x, *h0, *dh;
  const int* reset;
  void *h, *dgate, *dx, *dh0;
  float* carry;            // state in front of each tile
  int gdt, xdt, h0dt, dhdt, hdt, dgdt, dxdt, dh0dt;
  int rows, cols, length;  // length: rows per sequence
  int tiles, groups;       // tiles of 128 rows, groups of 32 * CH columns
  // look-back (null: no tile needs another one): counter, a flag per tile and group (1: pair, 2: end state), pairs, end states
  unsigned* counter;
  int* flag;
  float4* pair;
  float2* end;
  int *status, *status_clear;
};

// CH neighbouring columns as they are in memory
template <int DT, int CH> struct Cell;
template <> struct Cell<DRAGON_BF16, 2> {
  unsigned u;
  __device__ __forceinline__ void load(const void* p, size_t i) { u = __ldg(reinterpret_cast<const unsigned*>(reinterpret_cast<const unsigned short*>(p) + i)); }
  __device__ __forceinline__ float get(int e) const { return e ? bf16_high(u) : bf16_low(u); }
};
template <> struct Cell<DRAGON_F32, 2> {
  float2 u;
  __device__ __forceinline__ void load(const void* p, size_t i) { u = __ldg(reinterpret_cast<const float2*>(reinterpret_cast<const float*>(p) + i)); }
  __device__ __forceinline__ float get(int e) const { return e ? u.y : u.x; }
};
template <> struct Cell<DRAGON_BF16, 1> {
  unsigned short u;
  __device__ __forceinline__ void load(const void* p, size_t i) { u = __ldg(reinterpret_cast<const unsigned short*>(p) + i); }
  __device__ __forceinline__ float get(int) const { return bf16_low(u); }
};
template <> struct Cell<DRAGON_F32, 1> {
  float u;
  __device__ __forceinline__ void load(const void* p, size_t i) { u = __ldg(reinterpret_cast<const float*>(p) + i); }
  __device__ __forceinline__ float get(int) const { return u; }
};
template <int CH> __device__ __forceinline__ void store_cell(void* p, int dtype, size_t i, const float* v) {
  if (CH == 1) { store_any<1>(p, dtype, i, v); return; }
  if (dtype == DRAGON_F32) *reinterpret_cast<float2*>(reinterpret_cast<float*>(p) + i) = make_float2(v[0], v[CH - 1]);
  else *reinterpret_cast<unsigned*>(reinterpret_cast<unsigned short*>(p) + i) = bf16_pair(v[0], v[CH - 1]);
}

// f and 1 - f = exp(-z) f, each to full relative precision; exp(-z) is kept finite (a comparison with NaN is false)
__device__ __forceinline__ void gate_of(float z, float* f, float* keep) {
  float u = -z * 1.4426950408889634f;
  u = u > 126.f ? 126.f : u;
  const float t = exp2f(u);
  *f = __fdividef(1.f, 1.f + t);
  *keep = t * *f;
}

// which of a warp's rows exist, start afresh, and start from h0: lane r looks at row r
struct RowMarks {
  int n;                     // rows of the warp inside the tensor
  unsigned fresh, from_h0;   // bit r
  int seq;                   // this lane's row: its sequence
};
__device__ __forceinline__ RowMarks row_marks(const ScanArgs& a, int row0, int lane) {
  RowMarks m;
  m.n = max(0, min(kRows, a.rows - row0));
  const int row = row0 + lane;
  bool start = false, reset = false;
  m.seq = 0;
  if (lane < m.n) {
    m.seq = row / a.length;
    start = row - m.seq * a.length == 0;
    reset = a.reset != nullptr && __ldg(a.reset + row) != 0;
  }
  m.fresh = __ballot_sync(0xffffffffu, start || reset);
  m.from_h0 = __ballot_sync(0xffffffffu, start && !reset);
  return m;
}

__device__ __forceinline__ int load_flag(const int* p) {
  int v;
  asm volatile("ld.acquire.gpu.global.s32 %0, [%1];" : "=r"(v) : "l"(p) : "memory");
  return v;
}
__device__ __forceinline__ void store_flag(int* p, int v) { asm volatile("st.release.gpu.global.s32 [%0], %1;" ::"l"(p), "r"(v) : "memory"); }

// One warp, 2 columns a lane: publishes the tile's pair, finds the state in front of it (dir -1: from the tiles before it;
// +1, the gradient: from the tiles behind it), publishes its end state.  `closed`: a row of the tile starts afresh, so the
// end state is B whatever comes in; `open`: the incoming state is needed.  Returns it.
__device__ __forceinline__ float2 look_back(const ScanArgs& a, int tile, int group, int lane, float4 ab, bool closed, bool open, int dir) {
  const int last = dir < 0 ? 0 : a.tiles - 1;      // the tile with nothing in front of it
  auto slot = [&](int t) { return (size_t)t * a.groups + group; };
  float2 in = make_float2(0.f, 0.f);
  if (closed) {
    __stcg(a.end + slot(tile) * 32 + lane, make_float2(ab.z, ab.w));
    __threadfence();
    __syncwarp();
    if (lane == 0) store_flag(a.flag + slot(tile), 2);
  } else if (tile != last) {
    __stcg(a.pair + slot(tile) * 32 + lane, ab);
    __threadfence();
    __syncwarp();
    if (lane == 0) store_flag(a.flag + slot(tile), 1);
  }
  if (open && tile != last) {
    float4 acc = make_float4(1.f, 1.f, 0.f, 0.f);  // the tiles between the one looked at and this one
    int at = tile + dir;
    const long long t0 = clock64();
    for (bool done = false; !done;) {
      // 32 tiles at once, lane i the i-th nearest
      const int mine = at + dir * lane;
      const bool exists = dir < 0 ? mine >= last : mine <= last;
      const int v = exists ? load_flag(a.flag + slot(mine)) : 0;
      const unsigned some = __ballot_sync(0xffffffffu, v >= 1), full = __ballot_sync(0xffffffffu, v == 2);
      const int ready = some == 0xffffffffu ? 32 : __ffs(~some) - 1;       // nearest tiles that have something
      int use = min(ready, full ? __ffs(full) - 1 : 32);                   // pairs in front of the nearest end state
      const bool found = full != 0 && __ffs(full) - 1 < ready;
      __threadfence();
      for (int i = 0; i < use; ++i) {
        const float4 p = __ldcg(a.pair + slot(at + dir * i) * 32 + lane);
        acc.z = fmaf(acc.x, p.z, acc.z);
        acc.w = fmaf(acc.y, p.w, acc.w);
        acc.x *= p.x;
        acc.y *= p.y;
      }
      at += dir * use;
      if (found) {
        const float2 e = __ldcg(a.end + slot(at) * 32 + lane);
        in = make_float2(fmaf(acc.x, e.x, acc.z), fmaf(acc.y, e.y, acc.w));
        done = true;
      } else if (use == 0 && clock64() - t0 > kWaitBudgetCycles) {
        if (lane == 0) atomicExch(a.status, DRAGON_ERR_TIMEOUT);
        done = true;
      }
      done = __all_sync(0xffffffffu, done);      // the clocks of the lanes may differ by one look
    }
  }
  if (!closed) {
    __stcg(a.end + slot(tile) * 32 + lane, make_float2(fmaf(ab.x, in.x, ab.z), fmaf(ab.y, in.y, ab.w)));
    __threadfence();
    __syncwarp();
    if (lane == 0) store_flag(a.flag + slot(tile), 2);
  }
  return in;
}

struct TileShared {
  float4 ab[kWarps][32];     // each warp's pair (A, A', B, B')
  unsigned fresh[kWarps];    // whether one of its rows starts afresh
  float2 in[32];             // the state in front of the tile
  unsigned ticket;
};

// fold of warps [w0, w1) in time order (dir -1) or against it, applied to `in`
__device__ __forceinline__ float2 through(const TileShared& sh, int lane, int w0, int w1, int dir, float2 in) {
  for (int w = w0; w != w1; w += dir) {
    const float4 p = sh.ab[w][lane];
    in = sh.fresh[w] ? make_float2(p.z, p.w) : make_float2(fmaf(p.x, in.x, p.z), fmaf(p.y, in.y, p.w));
  }
  return in;
}
// the tile's own pair and whether it is closed
__device__ __forceinline__ float4 fold_tile(const TileShared& sh, int lane, int dir, bool* closed) {
  float4 ab = make_float4(1.f, 1.f, 0.f, 0.f);
  *closed = false;
  for (int i = 0; i < kWarps; ++i) {
    const int w = dir > 0 ? i : kWarps - 1 - i;
    const float4 p = sh.ab[w][lane];
    if (sh.fresh[w]) { ab = make_float4(0.f, 0.f, p.z, p.w); *closed = true; }
    else ab = make_float4(ab.x * p.x, ab.y * p.y, fmaf(p.x, ab.z, p.z), fmaf(p.y, ab.w, p.w));
  }
  return ab;
}

// the tile of this CTA: handed out in the order of time where tiles wait for one another
__device__ __forceinline__ unsigned take_ticket(const ScanArgs& a, TileShared& sh) {
  if (!a.counter) return blockIdx.x;
  if (threadIdx.x == 0) sh.ticket = atomicAdd(a.counter, 1u);
  __syncthreads();
  return sh.ticket;
}

template <int GDT, int XDT, int CH>
__global__ void __launch_bounds__(kThreads, 2) scan_kernel(const ScanArgs a) {
  __shared__ TileShared sh;
  if (a.status_clear && blockIdx.x == 0 && threadIdx.x == 0) *a.status_clear = 0;
  const unsigned ticket = take_ticket(a, sh);
  const int tile = ticket / a.groups, group = ticket - tile * a.groups;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int c = (group * 32 + lane) * CH, row0 = tile * kScanTileRows + warp * kRows;
  const bool mine = c < a.cols;
  const size_t base = (size_t)row0 * a.cols + c;
  Cell<GDT, CH> gate[kRows];
  Cell<XDT, CH> x[kRows];
  const RowMarks m = row_marks(a, row0, lane);
#pragma unroll
  for (int r = 0; r < kRows; ++r)
    if (mine && r < m.n) { gate[r].load(a.gate, base + (size_t)r * a.cols); x[r].load(a.x, base + (size_t)r * a.cols); }
  float f[kRows][CH], b[kRows][CH];
#pragma unroll
  for (int r = 0; r < kRows; ++r)
#pragma unroll
    for (int e = 0; e < CH; ++e) {
      f[r][e] = 1.f;         // rows and columns outside the tensor pass the state on
      b[r][e] = 0.f;
      if (mine && r < m.n) {
        float keep;
        gate_of(gate[r].get(e), &f[r][e], &keep);
        b[r][e] = keep * x[r].get(e);
      }
    }
  if (a.h0 && m.from_h0) {
#pragma unroll
    for (int r = 0; r < kRows; ++r) {
      const int seq = __shfl_sync(0xffffffffu, m.seq, r);
      if (mine && (m.from_h0 >> r & 1)) {
#pragma unroll
        for (int e = 0; e < CH; ++e) {
          float v;
          load_any<1>(a.h0, a.h0dt, (size_t)seq * a.cols + c + e, &v);
          b[r][e] = fmaf(f[r][e], v, b[r][e]);
        }
      }
    }
  }
  float A[2] = {1.f, 1.f}, B[2] = {0.f, 0.f};
#pragma unroll
  for (int r = 0; r < kRows; ++r) {
    const bool fresh = m.fresh >> r & 1;
#pragma unroll
    for (int e = 0; e < CH; ++e) {
      A[e] *= f[r][e];
      B[e] = fresh ? b[r][e] : fmaf(f[r][e], B[e], b[r][e]);
    }
  }
  sh.ab[warp][lane] = make_float4(A[0], A[1], B[0], B[1]);
  if (lane == 0) sh.fresh[warp] = m.fresh;
  __syncthreads();
  if (warp == 0) {
    float2 in = make_float2(0.f, 0.f);
    if (a.counter) {
      bool closed;
      const float4 ab = fold_tile(sh, lane, 1, &closed);
      in = look_back(a, tile, group, lane, ab, closed, !(m.fresh & 1), -1);
    }
    sh.in[lane] = in;
    if (a.carry && mine) {
      a.carry[(size_t)tile * a.cols + c] = in.x;
      if (CH == 2) a.carry[(size_t)tile * a.cols + c + 1] = in.y;
    }
  }
  __syncthreads();
  if (!a.h) return;
  const float2 in = through(sh, lane, 0, warp, 1, sh.in[lane]);
  float h[2] = {in.x, in.y};
#pragma unroll
  for (int r = 0; r < kRows; ++r) {
    const bool fresh = m.fresh >> r & 1;
#pragma unroll
    for (int e = 0; e < CH; ++e) h[e] = fresh ? b[r][e] : fmaf(f[r][e], h[e], b[r][e]);
    if (mine && r < m.n) store_cell<CH>(a.h, a.hdt, base + (size_t)r * a.cols, h);
  }
}

template <int GDT, int XDT, int DDT, int CH>
__global__ void __launch_bounds__(kThreads, GDT == DRAGON_F32 && XDT == DRAGON_F32 && DDT == DRAGON_F32 ? 1 : 2) scan_bwd_kernel(const ScanArgs a) {
  __shared__ TileShared sh;
  if (a.status_clear && blockIdx.x == 0 && threadIdx.x == 0) *a.status_clear = 0;
  const unsigned ticket = take_ticket(a, sh);
  const int tile = a.tiles - 1 - (int)(ticket / a.groups), group = ticket % a.groups;     // against time
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int c = (group * 32 + lane) * CH, row0 = tile * kScanTileRows + warp * kRows;
  const bool mine = c < a.cols;
  const size_t base = (size_t)row0 * a.cols + c;
  Cell<GDT, CH> gate[kRows];
  Cell<XDT, CH> x[kRows];
  Cell<DDT, CH> dh[kRows];
  const RowMarks m = row_marks(a, row0, lane);
#pragma unroll
  for (int r = 0; r < kRows; ++r)
    if (mine && r < m.n) {
      gate[r].load(a.gate, base + (size_t)r * a.cols);
      x[r].load(a.x, base + (size_t)r * a.cols);
      dh[r].load(a.dh, base + (size_t)r * a.cols);
    }
  float f[kRows][CH], hp[kRows][CH];      // hp: first (1 - f) x + f h0 where a sequence starts, then the state in front of the row
  float in_carry[2] = {0.f, 0.f};
  if (mine && a.carry) {
#pragma unroll
    for (int e = 0; e < CH; ++e) in_carry[e] = __ldg(a.carry + (size_t)tile * a.cols + c + e);
  }
  float h0v[kRows][CH];
#pragma unroll
  for (int r = 0; r < kRows; ++r)
#pragma unroll
    for (int e = 0; e < CH; ++e) {
      f[r][e] = 1.f;
      hp[r][e] = 0.f;
      h0v[r][e] = 0.f;
      if (mine && r < m.n) {
        float keep;
        gate_of(gate[r].get(e), &f[r][e], &keep);
        hp[r][e] = keep * x[r].get(e);
      }
    }
  if (a.h0 && m.from_h0) {
#pragma unroll
    for (int r = 0; r < kRows; ++r) {
      const int seq = __shfl_sync(0xffffffffu, m.seq, r);
      if (mine && (m.from_h0 >> r & 1)) {
#pragma unroll
        for (int e = 0; e < CH; ++e) load_any<1>(a.h0, a.h0dt, (size_t)seq * a.cols + c + e, &h0v[r][e]);
      }
    }
  }
  // the state: the warps' pairs, then every row's predecessor
  float A[2] = {1.f, 1.f}, B[2] = {0.f, 0.f};
#pragma unroll
  for (int r = 0; r < kRows; ++r) {
    const bool fresh = m.fresh >> r & 1;
#pragma unroll
    for (int e = 0; e < CH; ++e) {
      A[e] *= f[r][e];
      B[e] = fmaf(f[r][e], fresh ? h0v[r][e] : B[e], hp[r][e]);
    }
  }
  sh.ab[warp][lane] = make_float4(A[0], A[1], B[0], B[1]);
  if (lane == 0) sh.fresh[warp] = m.fresh;
  __syncthreads();
  {
    const float2 in = through(sh, lane, 0, warp, 1, make_float2(in_carry[0], in_carry[1]));
    float h[2] = {in.x, in.y};
#pragma unroll
    for (int r = 0; r < kRows; ++r) {
      const bool fresh = m.fresh >> r & 1;
#pragma unroll
      for (int e = 0; e < CH; ++e) {
        const float before = fresh ? h0v[r][e] : h[e];
        h[e] = fmaf(f[r][e], before, hp[r][e]);
        hp[r][e] = before;
      }
    }
  }
  __syncthreads();           // the pairs of the state have been read
  // the gradient, against time: e -> f (dh + e)
  A[0] = A[1] = 1.f;
  B[0] = B[1] = 0.f;
#pragma unroll
  for (int r = kRows - 1; r >= 0; --r) {
    const bool fresh = m.fresh >> r & 1;
#pragma unroll
    for (int e = 0; e < CH; ++e) {
      const float g = mine && r < m.n ? dh[r].get(e) : 0.f;
      A[e] *= f[r][e];
      B[e] = fresh ? 0.f : f[r][e] * (g + B[e]);
    }
  }
  sh.ab[warp][lane] = make_float4(A[0], A[1], B[0], B[1]);
  __syncthreads();
  if (warp == kWarps - 1) {
    float2 in = make_float2(0.f, 0.f);
    if (a.counter) {
      bool closed;
      const float4 ab = fold_tile(sh, lane, -1, &closed);
      in = look_back(a, tile, group, lane, ab, closed, true, 1);
    }
    sh.in[lane] = in;
  }
  __syncthreads();
  const float2 in = through(sh, lane, kWarps - 1, warp, -1, sh.in[lane]);
  float d[2] = {in.x, in.y};
#pragma unroll
  for (int r = kRows - 1; r >= 0; --r) {
    const bool fresh = m.fresh >> r & 1;
    float dx[2], dz[2];
#pragma unroll
    for (int e = 0; e < CH; ++e) {
      if (mine && r < m.n) {
        float ff, keep;
        gate_of(gate[r].get(e), &ff, &keep);     // 1 - f once more: cheaper than the registers that would keep it
        d[e] += dh[r].get(e);
        dx[e] = d[e] * keep;
        dz[e] = d[e] * (hp[r][e] - x[r].get(e)) * (ff * keep);
        d[e] = ff * d[e];
      }
    }
    if (mine && r < m.n) {
      if (a.dx) store_cell<CH>(a.dx, a.dxdt, base + (size_t)r * a.cols, dx);
      if (a.dgate) store_cell<CH>(a.dgate, a.dgdt, base + (size_t)r * a.cols, dz);
    }
    if (fresh) {
      if (a.dh0) {
        const int row = row0 + r, seq = row / a.length;
        if (row - seq * a.length == 0) {         // a sequence's first row: what reaches its initial state (nothing past a reset)
          const bool reaches = m.from_h0 >> r & 1;
          float g[2] = {reaches ? d[0] : 0.f, reaches ? d[1] : 0.f};
          if (mine) store_cell<CH>(a.dh0, a.dh0dt, (size_t)seq * a.cols + c, g);
        }
      }
      d[0] = d[1] = 0.f;
    }
  }
}

int columns_per_lane(int64_t cols) { return cols % 2 == 0 ? 2 : 1; }    // pairs of columns are aligned in every row

struct Scratch { size_t flag, pair, end, bytes; };
Scratch scratch_layout(int64_t rows, int64_t cols) {
  const int64_t slots = (rows + kScanTileRows - 1) / kScanTileRows * ((cols + 32 * columns_per_lane(cols) - 1) / (32 * columns_per_lane(cols)));
  auto up = [](size_t b) { return (b + 255) & ~(size_t)255; };
  Scratch s;
  s.flag = 256;
  s.pair = s.flag + up((size_t)slots * sizeof(int));
  s.end = s.pair + up((size_t)slots * 32 * sizeof(float4));
  s.bytes = s.end + up((size_t)slots * 32 * sizeof(float2));
  return s;
}

// everything that forward and gradient share; clears the look-back's counter and flags
cudaError_t scan_args(const StepRun& r, bool backward, ScanArgs* out) {
  const Shape& sh = r.mems[r.s.rd[sc::GATE]].shape;
  ScanArgs& a = *out;
  a.gate = r.rd(sc::GATE); a.x = r.rd(sc::X); a.h0 = r.rd(sc::H0); a.reset = reinterpret_cast<const int*>(r.rd(sc::RESET));
  a.gdt = r.rd_type(sc::GATE); a.xdt = r.rd_type(sc::X); a.h0dt = r.rd_type(sc::H0);
  a.rows = (int)sh.d[0];
  a.cols = (int)sh.d[1];
  a.length = (int)(sh.d[0] / (int64_t)r.s.attr);
  a.tiles = (a.rows + kScanTileRows - 1) / kScanTileRows;
  const int per_group = 32 * columns_per_lane(a.cols);
  a.groups = (a.cols + per_group - 1) / per_group;
  a.status = r.status;
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
  if ((int64_t)a.tiles * a.groups > 0x7fffffffLL) return cudaErrorInvalidConfiguration;
  // tiles that all begin with a sequence need no other tile
  if (a.tiles == 1 || kScanTileRows % a.length == 0) return cudaSuccess;
  const Scratch s = scratch_layout(a.rows, a.cols);
  char* p = r.ws + r.s.scratch_off;
  a.counter = reinterpret_cast<unsigned*>(p);
  a.flag = reinterpret_cast<int*>(p + s.flag);
  a.pair = reinterpret_cast<float4*>(p + s.pair);
  a.end = reinterpret_cast<float2*>(p + s.end);
  return cudaMemsetAsync(p, 0, s.pair, reinterpret_cast<cudaStream_t>(r.stream));
}

template <int GDT, int XDT>
void launch_fwd(const ScanArgs& a, cudaStream_t st) {
  const unsigned grid = (unsigned)a.tiles * a.groups;
  if (columns_per_lane(a.cols) == 2) scan_kernel<GDT, XDT, 2><<<grid, kThreads, 0, st>>>(a);
  else scan_kernel<GDT, XDT, 1><<<grid, kThreads, 0, st>>>(a);
}
template <int GDT, int XDT, int DDT>
void launch_bwd(const ScanArgs& a, cudaStream_t st) {
  const unsigned grid = (unsigned)a.tiles * a.groups;
  if (columns_per_lane(a.cols) == 2) scan_bwd_kernel<GDT, XDT, DDT, 2><<<grid, kThreads, 0, st>>>(a);
  else scan_bwd_kernel<GDT, XDT, DDT, 1><<<grid, kThreads, 0, st>>>(a);
}

}  // namespace

size_t scan_scratch_bytes(int64_t rows, int64_t cols) { return scratch_layout(rows, cols).bytes; }

cudaError_t launch_scan(const StepRun& r) {
  ScanArgs a{};
  cudaStream_t st = reinterpret_cast<cudaStream_t>(r.stream);
  const cudaError_t e = scan_args(r, false, &a);
  if (e != cudaSuccess) return e;
  if (a.gdt == DRAGON_F32) a.xdt == DRAGON_F32 ? launch_fwd<DRAGON_F32, DRAGON_F32>(a, st) : launch_fwd<DRAGON_F32, DRAGON_BF16>(a, st);
  else a.xdt == DRAGON_F32 ? launch_fwd<DRAGON_BF16, DRAGON_F32>(a, st) : launch_fwd<DRAGON_BF16, DRAGON_BF16>(a, st);
  return cudaGetLastError();
}

cudaError_t launch_scan_bwd(const StepRun& r) {
  ScanArgs a{};
  cudaStream_t st = reinterpret_cast<cudaStream_t>(r.stream);
  const cudaError_t e = scan_args(r, true, &a);
  if (e != cudaSuccess) return e;
#define DRAGON_SB(G, X) (a.dhdt == DRAGON_F32 ? launch_bwd<G, X, DRAGON_F32>(a, st) : launch_bwd<G, X, DRAGON_BF16>(a, st))
  if (a.gdt == DRAGON_F32) a.xdt == DRAGON_F32 ? DRAGON_SB(DRAGON_F32, DRAGON_F32) : DRAGON_SB(DRAGON_F32, DRAGON_BF16);
  else a.xdt == DRAGON_F32 ? DRAGON_SB(DRAGON_BF16, DRAGON_F32) : DRAGON_SB(DRAGON_BF16, DRAGON_BF16);
#undef DRAGON_SB
  return cudaGetLastError();
}

}  // namespace dragon
