// Gated linear recurrence over packed sequences, and its gradient.
//   h[t] = f[t] h[t-1] + (1 - f[t]) x[t],  f = sigmoid(gate);   h[-1] = the sequence's row of h0 (or 0); a row with reset
//   starts from 0.
//   D[t] = dh[t] + e[t],  e[t-1] = f[t] D[t] (0 from a row that starts afresh);  dx = (1 - f) D,
//   dgate = D (h[t-1] - x) f (1 - f),  dh0 = f[0] D[0].
// Bound: bytes.  A recurrence h -> f h + b composes: rows r..s act on the state in front of them as h -> A h + B with A the
// product of the f and B the state they reach from 0.  A tile is kScanTileRows rows x 64 columns; each warp of a CTA folds
// its rows into (A, B) from registers, the warps' pairs are folded through shared memory, and the state in front of the
// tile comes from the tiles before it: a tile publishes its (A, B) as soon as it has it and its end state once it knows its
// start; a tile looks back over published pairs until it meets an end state.  Everything is read once and written once,
// whatever the number of sequences: a long one is spread over the whole GPU.  Tiles are handed out by a counter in time
// order, so a tile waits only for tiles that are running or done; the wait is bounded (DRAGON_ERR_TIMEOUT).
// Published words need no flags and no fences: the exchange area is filled with a bit pattern that no arithmetic
// produces (a NaN other than the canonical one) before the launch, and a word that differs from it is there.
// A row that starts afresh cuts the chain by selection, not by a factor of 0: what is in front of it cannot reach it, NaN
// or not.  The state is fp32; the gradient recomputes it from the state in front of each tile, which the forward keeps.
#include <algorithm>

#include "device_util.h"
#include "plan.h"

namespace dragon {
namespace {

// The forward folds 16 rows a warp (4 CTAs of 4 warps per SM, next tile's rows loading), the gradient, which holds three
// tensors' rows and five values per element, 8 (2 CTAs of 8 warps).  Measured on 65536 x 1024 bf16: forward 4 x 16 rows
// 160 us, 8 x 8 178, 8 x 16 (tiles of 128) 154; gradient 8 x 8 320, 16 x 8 (tiles of 128) 347.
constexpr int kFwdWarps = 4, kBwdWarps = 8, kFwdCtas = 4, kBwdCtas = 2;
template <int W> constexpr int rows_per_warp() { return kScanTileRows / W; }
constexpr long long kWaitBudgetCycles = 4000000000LL;   // about two seconds
constexpr unsigned kAbsent = 0xffffffffu;          // an exchange word that has not been written

struct ScanArgs {
  const void *gate, *x, *h0, *dh;
  const int* reset;
  void *h, *dgate, *dx, *dh0;
  float* carry;            // state in front of each tile
  int gdt, xdt, h0dt, dhdt, hdt, dgdt, dxdt, dh0dt;
  int rows, cols, length;  // length: rows per sequence
  int tiles, groups;       // tiles of kScanTileRows rows, groups of 32 * CH columns
  unsigned* counter;       // tickets (starts at kAbsent)
  uint4* pair;             // exchange area: per tile and group 32 lanes' pairs (A, A', B, B'), null if no tile needs another
  uint2* end;              // ... and end states
  int *status, *status_clear;
};

// CH neighbouring columns as they are in memory; DT -1: a type known at run time
template <int DT, int CH> struct Cell;
template <> struct Cell<DRAGON_BF16, 2> {
  unsigned u;
  __device__ __forceinline__ void load(const char* p, int) { u = __ldg(reinterpret_cast<const unsigned*>(p)); }
  __device__ __forceinline__ float get(int e) const { return e ? bf16_high(u) : bf16_low(u); }
};
template <> struct Cell<DRAGON_F32, 2> {
  float2 u;
  __device__ __forceinline__ void load(const char* p, int) { u = __ldg(reinterpret_cast<const float2*>(p)); }
  __device__ __forceinline__ float get(int e) const { return e ? u.y : u.x; }
};
template <> struct Cell<DRAGON_BF16, 1> {
  unsigned short u;
  __device__ __forceinline__ void load(const char* p, int) { u = __ldg(reinterpret_cast<const unsigned short*>(p)); }
  __device__ __forceinline__ float get(int) const { return bf16_low(u); }
};
template <> struct Cell<DRAGON_F32, 1> {
  float u;
  __device__ __forceinline__ void load(const char* p, int) { u = __ldg(reinterpret_cast<const float*>(p)); }
  __device__ __forceinline__ float get(int) const { return u; }
};
template <int CH> struct Cell<-1, CH> {
  float u[CH];
  __device__ __forceinline__ void load(const char* p, int dtype) {
    if (dtype == DRAGON_F32) {
      Cell<DRAGON_F32, CH> c;
      c.load(p, dtype);
      for (int e = 0; e < CH; ++e) u[e] = c.get(e);
    } else {
      Cell<DRAGON_BF16, CH> c;
      c.load(p, dtype);
      for (int e = 0; e < CH; ++e) u[e] = c.get(e);
    }
  }
  __device__ __forceinline__ float get(int e) const { return u[e]; }
};
template <int DT> __device__ __forceinline__ int element_bytes(int dtype) { return (DT >= 0 ? DT : dtype) == DRAGON_F32 ? 4 : 2; }
template <int DT, int CH> __device__ __forceinline__ void store_cell(char* p, int dtype, const float* v) {
  if ((DT >= 0 ? DT : dtype) == DRAGON_F32) {
    if (CH == 2) *reinterpret_cast<float2*>(p) = make_float2(v[0], v[CH - 1]);
    else *reinterpret_cast<float*>(p) = v[0];
  } else {
    if (CH == 2) *reinterpret_cast<unsigned*>(p) = bf16_pair(v[0], v[CH - 1]);
    else *reinterpret_cast<unsigned short*>(p) = bf16_one(v[0]);
  }
}

// f and 1 - f = exp(-z) f, each to full relative precision (two units or so); exp(-z) is kept finite, a NaN stays one
__device__ __forceinline__ void gate_of(float z, float* f, float* keep) {
  float u = -z * 1.4426950408889634f, t;
  asm("min.NaN.f32 %0, %1, 0f42FC0000;" : "=f"(u) : "f"(u));      // 126
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(t) : "f"(u));
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(*f) : "f"(1.f + t));
  *keep = t * *f;
}

// which of a warp's rows exist, start afresh, and start from h0: lane r looks at row r
struct RowMarks {
  int n;                     // rows of the warp inside the tensor
  unsigned fresh, from_h0;   // bit r
  int seq;                   // this lane's row: its sequence
};
template <int W> __device__ __forceinline__ RowMarks row_marks(const ScanArgs& a, int row0, int lane) {
  constexpr int kRows = rows_per_warp<W>();
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

__device__ __forceinline__ void put(uint4* p, float4 v) {
  asm volatile("st.relaxed.gpu.global.v4.b32 [%0], {%1, %2, %3, %4};" ::"l"(p), "r"(__float_as_uint(v.x)), "r"(__float_as_uint(v.y)), "r"(__float_as_uint(v.z)),
               "r"(__float_as_uint(v.w)) : "memory");
}
__device__ __forceinline__ void put(uint2* p, float2 v) {
  asm volatile("st.relaxed.gpu.global.v2.b32 [%0], {%1, %2};" ::"l"(p), "r"(__float_as_uint(v.x)), "r"(__float_as_uint(v.y)) : "memory");
}
__device__ __forceinline__ uint4 look(const uint4* p) {
  uint4 v;
  asm volatile("ld.relaxed.gpu.global.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p) : "memory");
  return v;
}
__device__ __forceinline__ uint2 look(const uint2* p) {
  uint2 v;
  asm volatile("ld.relaxed.gpu.global.v2.b32 {%0, %1}, [%2];" : "=r"(v.x), "=r"(v.y) : "l"(p) : "memory");
  return v;
}
// Every value that is published goes through this: an arithmetic result is never kAbsent (NaNs come out canonical)
__device__ __forceinline__ float computed(float v) { return __fadd_rn(v, 0.f); }

// What one warp (2 columns a lane) hands on for its tile, and what it finds in front of it.  dir -1: the state, from the
// tiles before it; +1: the gradient, from the tiles behind it.  `closed`: a row of the tile starts afresh, so the end
// state is B whatever comes in.
__device__ __forceinline__ size_t slot_of(const ScanArgs& a, int tile, int group, int lane) { return ((size_t)tile * a.groups + group) * 32 + lane; }
__device__ __forceinline__ void publish_pair(const ScanArgs& a, int tile, int group, int lane, float4 ab, bool closed, int last) {
  const size_t s = slot_of(a, tile, group, lane);
  if (closed || tile == last) put(a.end + s, make_float2(computed(ab.z), computed(ab.w)));
  else put(a.pair + s, make_float4(computed(ab.x), computed(ab.y), computed(ab.z), computed(ab.w)));
}
__device__ __forceinline__ float2 look_back(const ScanArgs& a, int tile, int group, int lane, int dir, int last) {
  constexpr int kAhead = 4;                        // tiles looked at together
  float2 in = make_float2(0.f, 0.f);
  float4 acc = make_float4(1.f, 1.f, 0.f, 0.f);    // the tiles between the one looked at and this one
  int at = tile + dir;
  const long long t0 = clock64();
  for (bool done = tile == last; !done;) {
    uint4 p[kAhead];
    uint2 e[kAhead];
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      const int t = dir < 0 ? max(at - i, last) : min(at + i, last);
      const size_t s = slot_of(a, t, group, lane);
      p[i] = look(a.pair + s);
      e[i] = look(a.end + s);
    }
    bool moving = true;
    int moved = 0;
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      const bool has_end = e[i].x != kAbsent && e[i].y != kAbsent;
      const bool has_pair = p[i].x != kAbsent && p[i].y != kAbsent && p[i].z != kAbsent && p[i].w != kAbsent;
      if (moving && !done && has_end) {
        in = make_float2(fmaf(acc.x, __uint_as_float(e[i].x), acc.z), fmaf(acc.y, __uint_as_float(e[i].y), acc.w));
        done = true;
      }
      moving = moving && !done && has_pair;        // (the last tile has an end state and no pair: nothing moves past it)
      if (moving) {
        acc.z = fmaf(acc.x, __uint_as_float(p[i].z), acc.z);
        acc.w = fmaf(acc.y, __uint_as_float(p[i].w), acc.w);
        acc.x *= __uint_as_float(p[i].x);
        acc.y *= __uint_as_float(p[i].y);
        ++moved;
      }
    }
    at += dir * moved;
    if (!done && moved == 0 && clock64() - t0 > kWaitBudgetCycles) {
      atomicExch(a.status, DRAGON_ERR_TIMEOUT);
      done = true;
    }
  }
  __syncwarp();
  return in;
}
__device__ __forceinline__ void publish_end(const ScanArgs& a, int tile, int group, int lane, float4 ab, float2 in) {
  put(a.end + slot_of(a, tile, group, lane), make_float2(computed(fmaf(ab.x, in.x, ab.z)), computed(fmaf(ab.y, in.y, ab.w))));
}

template <int W> struct TileShared {
  float4 ab[W][32];          // each warp's pair (A, A', B, B')
  unsigned fresh[W];         // whether one of its rows starts afresh
  float2 in[32];             // the state in front of the tile
  unsigned ticket;
};

// fold of warps [w0, w1) in time order (dir 1) or against it, applied to `in`
template <int W> __device__ __forceinline__ float2 through(const TileShared<W>& sh, int lane, int w0, int w1, int dir, float2 in) {
#pragma unroll 4
  for (int w = w0; w != w1; w += dir) {
    const float4 p = sh.ab[w][lane];
    in = sh.fresh[w] ? make_float2(p.z, p.w) : make_float2(fmaf(p.x, in.x, p.z), fmaf(p.y, in.y, p.w));
  }
  return in;
}
// the tile's own pair and whether it is closed
template <int W> __device__ __forceinline__ float4 fold_tile(const TileShared<W>& sh, int lane, int dir, bool* closed) {
  float4 ab = make_float4(1.f, 1.f, 0.f, 0.f);
  *closed = false;
#pragma unroll 8
  for (int i = 0; i < W; ++i) {
    const int w = dir > 0 ? i : W - 1 - i;
    const float4 p = sh.ab[w][lane];
    if (sh.fresh[w]) { ab = make_float4(0.f, 0.f, p.z, p.w); *closed = true; }
    else ab = make_float4(ab.x * p.x, ab.y * p.y, fmaf(p.x, ab.z, p.z), fmaf(p.y, ab.w, p.w));
  }
  return ab;
}

// Tiles in the order they are handed out.  With an exchange area the counter decides (it starts at kAbsent, so the first
// ticket is 0 after the increment); without one any order will do.
__device__ __forceinline__ unsigned next_ticket(const ScanArgs& a, unsigned now) { return a.pair ? atomicAdd(a.counter, 1u) + 1u : now + gridDim.x; }

// initial states of the rows that start a sequence: h0v[r] for the bits of m.from_h0
template <int CH, int kRows>
__device__ __forceinline__ void load_h0(const ScanArgs& a, const RowMarks& m, int c, float (*v)[CH]) {
#pragma unroll
  for (int r = 0; r < kRows; ++r) {
    const size_t at = (size_t)__shfl_sync(0xffffffffu, m.seq, r) * a.cols + c;
    const bool want = m.from_h0 >> r & 1;
#pragma unroll
    for (int e = 0; e < CH; ++e) {
      v[r][e] = 0.f;
      if (want && a.h0dt == DRAGON_F32) v[r][e] = __ldg(reinterpret_cast<const float*>(a.h0) + at + e);
      if (want && a.h0dt == DRAGON_BF16) v[r][e] = bf16_low(__ldg(reinterpret_cast<const unsigned short*>(a.h0) + at + e));
    }
  }
}

// One tile's rows of one warp as they come from memory; rows behind the tensor repeat its last one
template <int DT, int CH, int N, int kRows> struct TileRows {
  Cell<DT, CH> v[N][kRows];
  __device__ __forceinline__ void load(const ScanArgs& a, int row0, int c) {
    const void* src[3] = {a.gate, a.x, a.dh};
    const int dt[3] = {a.gdt, a.xdt, a.dhdt};
    const size_t at = (size_t)min(row0, a.rows - 1) * a.cols + c;
    const bool whole = row0 + kRows <= a.rows;
#pragma unroll
    for (int k = 0; k < N; ++k) {
      const int es = element_bytes<DT>(dt[k]);
      const char* p = reinterpret_cast<const char*>(src[k]) + at * es;
      const size_t step = (size_t)a.cols * es;
      if (whole) {
#pragma unroll
        for (int r = 0; r < kRows; ++r, p += step) v[k][r].load(p, dt[k]);
      } else {
#pragma unroll
        for (int r = 0; r < kRows; ++r) { v[k][r].load(p, dt[k]); if (row0 + r + 1 < a.rows) p += step; }
      }
    }
  }
};

// a ticket's tile, counted with or against time, and its column group
struct Place {
  int tile, group;
  template <bool kReverse> static __device__ __forceinline__ Place of(const ScanArgs& a, unsigned ticket) {
    const unsigned t = ticket / (unsigned)a.groups;
    return {kReverse ? a.tiles - 1 - (int)t : (int)t, (int)(ticket - t * a.groups)};
  }
};

// Persistent CTAs.  While a tile's warp 0 looks back, the next tile's rows are on their way.
template <int DT, int CH>
__global__ void __launch_bounds__(kFwdWarps * 32, kFwdCtas) scan_kernel(const ScanArgs a) {
  constexpr int kRows = rows_per_warp<kFwdWarps>(), kThreads = kFwdWarps * 32;
  __shared__ TileShared<kFwdWarps> sh;
  if (a.status_clear && blockIdx.x == 0 && threadIdx.x == 0) *a.status_clear = 0;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const unsigned n = (unsigned)a.tiles * a.groups;
  unsigned ticket = blockIdx.x;
  if (a.pair) {
    if (threadIdx.x == 0) sh.ticket = next_ticket(a, 0);
    __syncthreads();
    ticket = sh.ticket;
  }
  TileRows<DT, CH, 2, kRows> rows;
  Place next = Place::of<false>(a, ticket);
  auto load_next = [&] { rows.load(a, next.tile * kScanTileRows + warp * kRows, min((next.group * 32 + lane) * CH, a.cols - CH)); };
  if (ticket < n) load_next();
  while (ticket < n) {
    const int tile = next.tile, group = next.group;
    const int c0 = (group * 32 + lane) * CH, row0 = tile * kScanTileRows + warp * kRows;
    const bool mine = c0 < a.cols;
    const int c = min(c0, a.cols - CH);
    const RowMarks m = row_marks<kFwdWarps>(a, row0, lane);
    float f[kRows][CH], b[kRows][CH];
#pragma unroll
    for (int r = 0; r < kRows; ++r)
#pragma unroll
      for (int e = 0; e < CH; ++e) {
        float keep;
        gate_of(rows.v[0][r].get(e), &f[r][e], &keep);
        b[r][e] = keep * rows.v[1][r].get(e);
      }
    if (m.n < kRows) {       // rows behind the tensor pass the state on
#pragma unroll
      for (int r = 0; r < kRows; ++r)
#pragma unroll
        for (int e = 0; e < CH; ++e)
          if (r >= m.n) { f[r][e] = 1.f; b[r][e] = 0.f; }
    }
    if (a.h0 && m.from_h0) {
      float v[kRows][CH];
      load_h0<CH, kRows>(a, m, c, v);
#pragma unroll
      for (int r = 0; r < kRows; ++r)
#pragma unroll
        for (int e = 0; e < CH; ++e)
          if (m.from_h0 >> r & 1) b[r][e] = fmaf(f[r][e], v[r][e], b[r][e]);
    }
    float A[2] = {1.f, 1.f}, B[2] = {0.f, 0.f};
    if (m.fresh == 0) {
#pragma unroll
      for (int r = 0; r < kRows; ++r)
#pragma unroll
        for (int e = 0; e < CH; ++e) { A[e] *= f[r][e]; B[e] = fmaf(f[r][e], B[e], b[r][e]); }
    } else {
#pragma unroll
      for (int r = 0; r < kRows; ++r)
#pragma unroll
        for (int e = 0; e < CH; ++e) B[e] = (m.fresh >> r & 1) ? b[r][e] : fmaf(f[r][e], B[e], b[r][e]);
    }
    sh.ab[warp][lane] = make_float4(A[0], A[1], B[0], B[1]);
    if (lane == 0) sh.fresh[warp] = m.fresh;
    if (threadIdx.x == kThreads - 1) sh.ticket = next_ticket(a, ticket);
    __syncthreads();
    ticket = sh.ticket;
    next = Place::of<false>(a, ticket);
    bool closed = true;
    float4 ab;
    if (warp == 0 && a.pair) {
      ab = fold_tile(sh, lane, 1, &closed);
      publish_pair(a, tile, group, lane, ab, closed, 0);
    }
    if (ticket < n) load_next();
    if (warp == 0) {
      float2 in = make_float2(0.f, 0.f);
      if (a.pair && !(m.fresh & 1)) in = look_back(a, tile, group, lane, -1, 0);
      if (a.pair && !closed && tile != 0) publish_end(a, tile, group, lane, ab, in);
      sh.in[lane] = in;
      if (a.carry && mine) {
        float* p = a.carry + (size_t)tile * a.cols + c;
        p[0] = in.x;
        if (CH == 2) p[1] = in.y;
      }
    }
    __syncthreads();
    if (a.h) {
      const float2 in = through(sh, lane, 0, warp, 1, sh.in[lane]);
      float h[2] = {in.x, in.y};
      const int es = element_bytes<DT>(a.hdt);
      char* p = reinterpret_cast<char*>(a.h) + ((size_t)row0 * a.cols + c) * es;
      const size_t step = (size_t)a.cols * es;
      if (m.fresh == 0 && m.n == kRows) {
#pragma unroll
        for (int r = 0; r < kRows; ++r, p += step) {
#pragma unroll
          for (int e = 0; e < CH; ++e) h[e] = fmaf(f[r][e], h[e], b[r][e]);
          if (mine) store_cell<DT, CH>(p, a.hdt, h);
        }
      } else {
#pragma unroll
        for (int r = 0; r < kRows; ++r, p += step) {
#pragma unroll
          for (int e = 0; e < CH; ++e) h[e] = (m.fresh >> r & 1) ? b[r][e] : fmaf(f[r][e], h[e], b[r][e]);
          if (mine && r < m.n) store_cell<DT, CH>(p, a.hdt, h);
        }
      }
    }
    __syncthreads();         // the pairs and the state have been read
  }
}

template <int DT, int CH>
__global__ void __launch_bounds__(kBwdWarps * 32, kBwdCtas) scan_bwd_kernel(const ScanArgs a) {
  constexpr int kWarps = kBwdWarps, kRows = rows_per_warp<kBwdWarps>();
  __shared__ TileShared<kBwdWarps> sh, back;
  if (a.status_clear && blockIdx.x == 0 && threadIdx.x == 0) *a.status_clear = 0;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const unsigned n = (unsigned)a.tiles * a.groups;
  unsigned ticket = blockIdx.x;
  if (a.pair) {
    if (threadIdx.x == 0) sh.ticket = next_ticket(a, 0);
    __syncthreads();
    ticket = sh.ticket;
  }
  const bool plain_out = a.dx && a.dgate && a.dxdt == DRAGON_F32 && a.dgdt == DRAGON_F32;
  while (ticket < n) {
    const Place at = Place::of<true>(a, ticket);      // tickets against time
    const int tile = at.tile, group = at.group;
    const int c0 = (group * 32 + lane) * CH, row0 = tile * kScanTileRows + warp * kRows;
    const bool mine = c0 < a.cols;
    const int c = min(c0, a.cols - CH);
    TileRows<DT, CH, 3, kRows> rows;
    rows.load(a, row0, c);
    float carry[2] = {0.f, 0.f};
#pragma unroll
    for (int e = 0; e < CH; ++e) carry[e] = __ldg(a.carry + (size_t)tile * a.cols + c + e);
    const RowMarks m = row_marks<kBwdWarps>(a, row0, lane);
    const bool plain = m.n == kRows && m.fresh == 0;
    float f[kRows][CH], keep[kRows][CH], hp[kRows][CH];      // hp: the state in front of the row
#pragma unroll
    for (int r = 0; r < kRows; ++r)
#pragma unroll
      for (int e = 0; e < CH; ++e) gate_of(rows.v[0][r].get(e), &f[r][e], &keep[r][e]);
    if (m.n < kRows) {       // rows behind the tensor pass the state and the gradient on
#pragma unroll
      for (int r = 0; r < kRows; ++r)
#pragma unroll
        for (int e = 0; e < CH; ++e)
          if (r >= m.n) { f[r][e] = 1.f; keep[r][e] = 0.f; }
    }
    // pairs of the state and of the gradient e -> f (dh + e)
    float A[2] = {1.f, 1.f}, B[2] = {0.f, 0.f}, E[2] = {0.f, 0.f};
    if (plain) {
#pragma unroll
      for (int r = 0; r < kRows; ++r)
#pragma unroll
        for (int e = 0; e < CH; ++e) { A[e] *= f[r][e]; B[e] = fmaf(f[r][e], B[e], keep[r][e] * rows.v[1][r].get(e)); }
#pragma unroll
      for (int r = kRows - 1; r >= 0; --r)
#pragma unroll
        for (int e = 0; e < CH; ++e) E[e] = f[r][e] * (rows.v[2][r].get(e) + E[e]);
    } else {
#pragma unroll
      for (int r = 0; r < kRows; ++r)
#pragma unroll
        for (int e = 0; e < CH; ++e) hp[r][e] = 0.f;         // for now: h0 where a sequence starts
      if (a.h0 && m.from_h0) load_h0<CH, kRows>(a, m, c, hp);
#pragma unroll
      for (int r = 0; r < kRows; ++r)
#pragma unroll
        for (int e = 0; e < CH; ++e) {
          A[e] *= f[r][e];
          const float kx = r < m.n ? keep[r][e] * rows.v[1][r].get(e) : 0.f;
          B[e] = fmaf(f[r][e], (m.fresh >> r & 1) ? hp[r][e] : B[e], kx);
        }
#pragma unroll
      for (int r = kRows - 1; r >= 0; --r)
#pragma unroll
        for (int e = 0; e < CH; ++e) {
          const float g = f[r][e] * (rows.v[2][r].get(e) + E[e]);
          E[e] = r >= m.n || (m.fresh >> r & 1) ? 0.f : g;
        }
    }
    sh.ab[warp][lane] = make_float4(A[0], A[1], B[0], B[1]);
    back.ab[warp][lane] = make_float4(A[0], A[1], E[0], E[1]);
    if (lane == 0) sh.fresh[warp] = back.fresh[warp] = m.fresh;
    if (threadIdx.x == 0) sh.ticket = next_ticket(a, ticket);
    __syncthreads();
    ticket = sh.ticket;
    if (warp == kWarps - 1) {
      float2 in = make_float2(0.f, 0.f);
      if (a.pair) {
        bool closed;
        const float4 ab = fold_tile(back, lane, -1, &closed);
        publish_pair(a, tile, group, lane, ab, closed, a.tiles - 1);
        in = look_back(a, tile, group, lane, 1, a.tiles - 1);
        if (!closed && tile != a.tiles - 1) publish_end(a, tile, group, lane, ab, in);
      }
      back.in[lane] = in;
    }
    {
      const float2 in = through(sh, lane, 0, warp, 1, make_float2(carry[0], carry[1]));
      float h[2] = {in.x, in.y};
#pragma unroll
      for (int r = 0; r < kRows; ++r)
#pragma unroll
        for (int e = 0; e < CH; ++e) {
          if (!plain && (m.fresh >> r & 1)) h[e] = hp[r][e];
          hp[r][e] = h[e];
          h[e] = fmaf(f[r][e], h[e], keep[r][e] * rows.v[1][r].get(e));
        }
    }
    __syncthreads();
    const float2 in = through(back, lane, kWarps - 1, warp, -1, back.in[lane]);
    float d[2] = {in.x, in.y};
    if (plain && plain_out) {
      const size_t step = (size_t)a.cols * 4, at_last = ((size_t)(row0 + kRows - 1) * a.cols + c) * 4;
      char *px = reinterpret_cast<char*>(a.dx) + at_last, *pg = reinterpret_cast<char*>(a.dgate) + at_last;
#pragma unroll
      for (int r = kRows - 1; r >= 0; --r, px -= step, pg -= step) {
        float dx[2], dz[2];
#pragma unroll
        for (int e = 0; e < CH; ++e) {
          d[e] += rows.v[2][r].get(e);
          dx[e] = d[e] * keep[r][e];
          d[e] *= f[r][e];
          dz[e] = dx[e] * f[r][e] * (hp[r][e] - rows.v[1][r].get(e));
        }
        if (mine) { store_cell<DRAGON_F32, CH>(px, DRAGON_F32, dx); store_cell<DRAGON_F32, CH>(pg, DRAGON_F32, dz); }
      }
    } else {
#pragma unroll
      for (int r = kRows - 1; r >= 0; --r) {
        if (r >= m.n) continue;
        float dx[2], dz[2];
#pragma unroll
        for (int e = 0; e < CH; ++e) {
          d[e] += rows.v[2][r].get(e);
          dx[e] = d[e] * keep[r][e];
          d[e] *= f[r][e];
          dz[e] = dx[e] * f[r][e] * (hp[r][e] - rows.v[1][r].get(e));
        }
        if (mine) {
          const size_t i = (size_t)(row0 + r) * a.cols + c;
          if (a.dx) store_cell<-1, CH>(reinterpret_cast<char*>(a.dx) + i * element_bytes<-1>(a.dxdt), a.dxdt, dx);
          if (a.dgate) store_cell<-1, CH>(reinterpret_cast<char*>(a.dgate) + i * element_bytes<-1>(a.dgdt), a.dgdt, dz);
        }
        if (m.fresh >> r & 1) {
          if (a.dh0) {
            const int row = row0 + r, seq = row / a.length;
            if (row - seq * a.length == 0) {         // a sequence's first row: what reaches its initial state (nothing past a reset)
              const bool reaches = m.from_h0 >> r & 1;
              float g[2] = {reaches ? d[0] : 0.f, reaches ? d[1] : 0.f};
              if (mine) store_cell<-1, CH>(reinterpret_cast<char*>(a.dh0) + ((size_t)seq * a.cols + c) * element_bytes<-1>(a.dh0dt), a.dh0dt, g);
            }
          }
          d[0] = d[1] = 0.f;
        }
      }
    }
    __syncthreads();         // the pairs and the states have been read
  }
}

// One row per sequence (a decoding step): nothing to scan, every element by itself
template <int DT, int CH>
__global__ void __launch_bounds__(256) scan_step_kernel(const ScanArgs a) {
  if (a.status_clear && blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0) *a.status_clear = 0;
  const int c = (blockIdx.x * 256 + threadIdx.x) * CH;
  if (c >= a.cols) return;
  for (int row = blockIdx.y; row < a.rows; row += gridDim.y) {
    const size_t at = (size_t)row * a.cols + c;
    Cell<DT, CH> z, x;
    Cell<-1, CH> h0;
    z.load(reinterpret_cast<const char*>(a.gate) + at * element_bytes<DT>(a.gdt), a.gdt);
    x.load(reinterpret_cast<const char*>(a.x) + at * element_bytes<DT>(a.xdt), a.xdt);
    if (a.h0) h0.load(reinterpret_cast<const char*>(a.h0) + at * element_bytes<-1>(a.h0dt), a.h0dt);
    const bool from_h0 = a.h0 && !(a.reset && __ldg(a.reset + row) != 0);
    float h[CH];
#pragma unroll
    for (int e = 0; e < CH; ++e) {
      float f, keep;
      gate_of(z.get(e), &f, &keep);
      h[e] = keep * x.get(e);
      if (from_h0) h[e] = fmaf(f, h0.get(e), h[e]);
    }
    store_cell<DT, CH>(reinterpret_cast<char*>(a.h) + at * element_bytes<DT>(a.hdt), a.hdt, h);
  }
}

int columns_per_lane(int64_t cols) { return cols % 2 == 0 ? 2 : 1; }    // pairs of columns are aligned in every row

struct Scratch { size_t pair, end, bytes; };
Scratch scratch_layout(int64_t rows, int64_t cols) {
  const int64_t slots = (rows + kScanTileRows - 1) / kScanTileRows * ((cols + 32 * columns_per_lane(cols) - 1) / (32 * columns_per_lane(cols)));
  Scratch s;
  s.pair = 256;            // the counter stands in front
  s.end = s.pair + (size_t)slots * 32 * sizeof(uint4);
  s.bytes = s.end + (size_t)slots * 32 * sizeof(uint2);
  return s;
}

// everything that forward and gradient share; fills the exchange area
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
  if ((int64_t)a.tiles * a.groups > 0x3fffffffLL) return cudaErrorInvalidConfiguration;
  // tiles that all begin with a sequence need no other tile
  if (a.tiles == 1 || kScanTileRows % a.length == 0) return cudaSuccess;
  const Scratch s = scratch_layout(a.rows, a.cols);
  char* p = r.ws + r.s.scratch_off;
  a.counter = reinterpret_cast<unsigned*>(p);
  a.pair = reinterpret_cast<uint4*>(p + s.pair);
  a.end = reinterpret_cast<uint2*>(p + s.end);
  return cudaMemsetAsync(p, 0xff, s.bytes, reinterpret_cast<cudaStream_t>(r.stream));
}

template <int DT>
void launch_fwd(const ScanArgs& a, int sm_count, cudaStream_t st) {
  if (a.length == 1 && !a.carry) {
    const int per = columns_per_lane(a.cols);
    const dim3 grid((a.cols + 256 * per - 1) / (256 * per), std::min(a.rows, 32768));
    if (per == 2) scan_step_kernel<DT, 2><<<grid, 256, 0, st>>>(a);
    else scan_step_kernel<DT, 1><<<grid, 256, 0, st>>>(a);
    return;
  }
  const unsigned grid = std::min((unsigned)a.tiles * a.groups, (unsigned)(sm_count * kFwdCtas));
  if (columns_per_lane(a.cols) == 2) scan_kernel<DT, 2><<<grid, kFwdWarps * 32, 0, st>>>(a);
  else scan_kernel<DT, 1><<<grid, kFwdWarps * 32, 0, st>>>(a);
}
template <int DT>
void launch_bwd(const ScanArgs& a, int sm_count, cudaStream_t st) {
  const unsigned grid = std::min((unsigned)a.tiles * a.groups, (unsigned)(sm_count * kBwdCtas));
  if (columns_per_lane(a.cols) == 2) scan_bwd_kernel<DT, 2><<<grid, kBwdWarps * 32, 0, st>>>(a);
  else scan_bwd_kernel<DT, 1><<<grid, kBwdWarps * 32, 0, st>>>(a);
}

}  // namespace

size_t scan_scratch_bytes(int64_t rows, int64_t cols) { return scratch_layout(rows, cols).bytes; }

cudaError_t launch_scan(const StepRun& r) {
  ScanArgs a{};
  cudaStream_t st = reinterpret_cast<cudaStream_t>(r.stream);
  const cudaError_t e = scan_args(r, false, &a);
  if (e != cudaSuccess) return e;
  const bool same = a.gdt == a.xdt && (!a.h || a.hdt == a.gdt);
  if (!same) launch_fwd<-1>(a, r.sm_count, st);
  else if (a.gdt == DRAGON_F32) launch_fwd<DRAGON_F32>(a, r.sm_count, st);
  else launch_fwd<DRAGON_BF16>(a, r.sm_count, st);
  return cudaGetLastError();
}

cudaError_t launch_scan_bwd(const StepRun& r) {
  ScanArgs a{};
  cudaStream_t st = reinterpret_cast<cudaStream_t>(r.stream);
  const cudaError_t e = scan_args(r, true, &a);
  if (e != cudaSuccess) return e;
  const bool same = a.gdt == a.xdt && a.dhdt == a.gdt;
  if (!same) launch_bwd<-1>(a, r.sm_count, st);
  else if (a.gdt == DRAGON_F32) launch_bwd<DRAGON_F32>(a, r.sm_count, st);
  else launch_bwd<DRAGON_BF16>(a, r.sm_count, st);
  return cudaGetLastError();
}

}  // namespace dragon
