// Gated linear recurrence over packed sequences, and its gradient.
//   h[t] = f[t] h[t-1] + (1 - f[t]) x[t],  f = sigmoid(gate);   h[-1] = the sequence's row of h0 (or 0); a row with reset
//   starts from 0.
//   D[t] = dh[t] + e[t],  e[t-1] = f[t] D[t] (0 from a row that starts afresh);  dx = (1 - f) D,
//   dgate = D (h[t-1] - x) f (1 - f),  dh0 = f[0] D[0].
// Bound: bytes.  A recurrence h -> f h + b composes: rows r..s act on the state in front of them as h -> A h + B with A the
// product of the f and B the state they reach from 0.  A tile is kScanTileRows rows x 64 columns; each warp of a CTA folds
// its rows into (A, B) from registers, the warps' pairs are folded through shared memory, and the state in front of the
// tile comes from the tiles before it.  Tiles form runs of 32: every tile publishes its (A, B) as soon as it has it; a tile
// reads those of the tiles before it in its run (the warps share them, all loads in flight together), and the state in front
// of the run, which the last tile of the run before published.  What is added to what is fixed by the tile's place alone, so
// every run of the kernel gives the same bits; a long sequence passes 1/32 of its tiles one after another.  Everything is
// read once and written once, whatever the number of sequences: a long one is spread over the whole GPU.  Tiles are handed
// out by a counter in the order of the chain, so a tile waits only for tiles that are running or done; the wait is bounded
// (DRAGON_ERR_TIMEOUT).  Published words need no flags and no fences: the exchange area is filled with a bit pattern that no
// arithmetic produces (a NaN other than the canonical one) before the launch, and a word that differs from it is there.
// A row that starts afresh cuts the chain by selection, not by a factor of 0: what is in front of it cannot reach it, NaN
// or not.  The state is fp32; the gradient recomputes it from the state in front of each tile, which the forward keeps.
#include <algorithm>
#include <cstdlib>

#include "device_util.h"
#include "plan.h"

namespace dragon {
namespace {

// The forward folds 16 rows a warp (3 CTAs of 4 warps per SM, the next tile's rows on their way in registers), the gradient,
// which holds three tensors' rows and three values per element, 8 (2 CTAs of 8 warps; the next tile's rows on their way to
// L2).  Measured on 65536 x 1024 bf16, one sequence (and 1024 of them, where no tile needs another): forward 169 us (104),
// gradient 295 (247); the bytes alone: 61, 143.  Other shapes, when the gate took three instructions less (forward 164 (98),
// gradient 295 (241)): 4 CTAs and their spills 175 (112), 8 x 8 rows 199 (117), folding one tile ahead of the one that waits 242
// (143: the second tile's registers cost more than the wait), the gradient without the next tile asked for 337 (258).
constexpr int kFwdWarps = 4, kBwdWarps = 8, kBwdCtas = 2;
template <int CH> constexpr int kFwdCtas = CH == 2 ? 3 : 4;      // per SM, as registers allow
template <int W> constexpr int rows_per_warp() { return kScanTileRows / W; }
constexpr long long kWaitBudgetCycles = 4000000000LL;   // about two seconds
constexpr unsigned kAbsent = 0xffffffffu;          // an exchange word that has not been written
constexpr unsigned kClosed = 0xfffffffeu;          // in the place of A: a row of the tile starts afresh, its end state is B whatever comes in
constexpr int kRun = 32;                           // tiles of a run

struct ScanArgs {
  const void *gate, *x, *h0, *dh;
  const int* reset;
  void *h, *dgate, *dx, *dh0;
  float* carry;            // state in front of each tile
  int gdt, xdt, h0dt, dhdt, hdt, dgdt, dxdt, dh0dt;
  int rows, cols, length;  // length: rows per sequence
  int tiles, groups;       // tiles of kScanTileRows rows, groups of 32 * CH columns
  unsigned* counter;       // tickets (starts at kAbsent)
  uint4* pair;             // exchange area: per tile (in the chain's order) and group 32 lanes' pairs (A, A', B, B'), null if no tile needs another
  uint2* start;            // ... and per run and group the state in front of it
  int *status, *status_clear;
  long long wait_budget;   // clock cycles
  int withhold;            // failure-detection test: the chain's first tile publishes nothing
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

// CH neighbouring columns' values; pairs go through the packed instructions (each half rounded as the scalar one rounds)
template <int CH> struct Vec { float v[CH]; };
template <int CH> __device__ __forceinline__ Vec<CH> splat(float x) { Vec<CH> r; for (int e = 0; e < CH; ++e) r.v[e] = x; return r; }
__device__ __forceinline__ unsigned long long packed(const Vec<2>& a) { unsigned long long r; asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a.v[0]), "f"(a.v[1])); return r; }
__device__ __forceinline__ Vec<2> unpacked(unsigned long long a) { Vec<2> r; asm("mov.b64 {%0, %1}, %2;" : "=f"(r.v[0]), "=f"(r.v[1]) : "l"(a)); return r; }
__device__ __forceinline__ Vec<2> mul(const Vec<2>& a, const Vec<2>& b) { unsigned long long r; asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(packed(a)), "l"(packed(b))); return unpacked(r); }
__device__ __forceinline__ Vec<2> add(const Vec<2>& a, const Vec<2>& b) { unsigned long long r; asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(packed(a)), "l"(packed(b))); return unpacked(r); }
__device__ __forceinline__ Vec<2> fma(const Vec<2>& a, const Vec<2>& b, const Vec<2>& c) {
  unsigned long long r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(packed(a)), "l"(packed(b)), "l"(packed(c)));
  return unpacked(r);
}
__device__ __forceinline__ Vec<1> mul(const Vec<1>& a, const Vec<1>& b) { return {{__fmul_rn(a.v[0], b.v[0])}}; }
__device__ __forceinline__ Vec<1> add(const Vec<1>& a, const Vec<1>& b) { return {{__fadd_rn(a.v[0], b.v[0])}}; }
__device__ __forceinline__ Vec<1> fma(const Vec<1>& a, const Vec<1>& b, const Vec<1>& c) { return {{__fmaf_rn(a.v[0], b.v[0], c.v[0])}}; }

// f = 1 / (1 + exp(-z)) and 1 - f = exp(-z) f, each within 10 units of 2^-24 of itself: exp(-z) = 2^u (1 + w) with u the rounded
// product -z log2(e) and w what it leaves out times ln 2 (its residue, exact, and z times the part of log2(e) that fp32 does
// not hold; without it the error grows to |z| units); 2^u is good to 4 units, the reciprocal to 2, three more roundings.  z is
// kept in [-87, 104], where exp(-z) and f are normal numbers or 0 and nothing is infinite; a NaN stays one.  Two columns at a
// time this is three instructions an element more than the rounded product alone: 65536 x 1024 bf16 forward 169 us for 165,
// forward and gradient 463 for 456.
constexpr float kLog2eHi = 1.44269502162933349609375f, kLog2eLo = 1.9259629911266175e-8f, kLn2 = 0.693147180559945309f;
template <int CH> __device__ __forceinline__ void gate_of(Vec<CH> z, Vec<CH>* f, Vec<CH>* keep) {
#pragma unroll
  for (int e = 0; e < CH; ++e) {
    asm("max.NaN.f32 %0, %1, 0fC2AE0000;" : "=f"(z.v[e]) : "f"(z.v[e]));      // -87
    asm("min.NaN.f32 %0, %1, 0f42D00000;" : "=f"(z.v[e]) : "f"(z.v[e]));      // 104
  }
  const Vec<CH> u = mul(z, splat<CH>(-kLog2eHi)), w = fma(z, splat<CH>(kLog2eLo), fma(z, splat<CH>(kLog2eHi), u));
  Vec<CH> t;
#pragma unroll
  for (int e = 0; e < CH; ++e) asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(t.v[e]) : "f"(u.v[e]));
  t = fma(t, mul(w, splat<CH>(-kLn2)), t);
  const Vec<CH> d = add(t, splat<CH>(1.f));
#pragma unroll
  for (int e = 0; e < CH; ++e) asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(f->v[e]) : "f"(d.v[e]));
  *keep = mul(t, *f);
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

// `order`: a tile's place in the chain (its number, or counted from the end for the gradient)
__device__ __forceinline__ size_t slot_of(const ScanArgs& a, int order, int group, int lane) { return ((size_t)order * a.groups + group) * 32 + lane; }
__device__ __forceinline__ void publish_pair(const ScanArgs& a, int order, int group, int lane, float4 ab, bool closed) {
  if (a.withhold && order == 0) return;
  const float none = __uint_as_float(kClosed);
  put(a.pair + slot_of(a, order, group, lane), make_float4(closed ? none : computed(ab.x), closed ? none : computed(ab.y), computed(ab.z), computed(ab.w)));
}
// the state behind a run's last tile, for the next run
__device__ __forceinline__ void publish_start(const ScanArgs& a, int order, int group, int lane, float2 v) {
  if (order % kRun == kRun - 1) put(a.start + slot_of(a, order / kRun + 1, group, lane), make_float2(computed(v.x), computed(v.y)));
}
__device__ __forceinline__ bool out_of_time(const ScanArgs& a, long long t0) {
  if (clock64() - t0 <= a.wait_budget) return false;
  atomicExch(a.status, DRAGON_ERR_TIMEOUT);
  return true;
}

// what the warps of a CTA exchange; kCopies: tiles whose pairs are alive at a time
template <int W, int kCopies> struct TileShared {
  float4 ab[kCopies][W][32];     // each warp's pair (A, A', B, B')
  unsigned fresh[kCopies][W];    // its rows that start afresh
  unsigned ticket[kCopies];
  float4 seg[W][32];             // the pairs of the run's tiles in front of this one, folded by each warp's share
  bool seg_closed[W];
};

// This warp's share of the run's tiles in front of tile `order`: their pairs, folded in order (waits for them)
// kAhead: loads in flight together (the forward over fp32 rows has registers for half of them: 95 us for 107 on 16384 x 2048)
template <int kAhead, int W, int K> __device__ __forceinline__ void fold_run(const ScanArgs& a, TileShared<W, K>& sh, int order, int group, int warp, int lane) {
  constexpr int kShare = kRun / W;
  const int first = order / kRun * kRun + warp * kShare, n = min(kShare, order - first);
  float4 ab = make_float4(1.f, 1.f, 0.f, 0.f);
  bool closed = false;
#pragma unroll 1
  for (int i0 = 0; i0 < n; i0 += kAhead) {
    uint4 p[kAhead];
    const long long t0 = clock64();
    for (;;) {
      bool all = true;
#pragma unroll
      for (int i = 0; i < kAhead; ++i) p[i] = look(a.pair + slot_of(a, first + min(i0 + i, n - 1), group, lane));
#pragma unroll
      for (int i = 0; i < kAhead; ++i) all = all && p[i].x != kAbsent && p[i].y != kAbsent && p[i].z != kAbsent && p[i].w != kAbsent;
      if (__all_sync(0xffffffffu, all) || out_of_time(a, t0)) break;
    }
    __syncwarp();
#pragma unroll
    for (int i = 0; i < kAhead; ++i)
      if (i0 + i < n) {
        const float4 q = make_float4(__uint_as_float(p[i].x), __uint_as_float(p[i].y), __uint_as_float(p[i].z), __uint_as_float(p[i].w));
        if (p[i].x == kClosed) { ab = q; closed = true; }      // (closed for all columns or for none)
        else ab = make_float4(ab.x * q.x, ab.y * q.y, fmaf(q.x, ab.z, q.z), fmaf(q.y, ab.w, q.w));
      }
  }
  sh.seg[warp][lane] = ab;
  if (lane == 0) sh.seg_closed[warp] = closed;
}
// the first look at the state in front of the run, sent for before the pairs
__device__ __forceinline__ uint2 early_start(const ScanArgs& a, int order, int group, int lane) {
  return order < kRun ? make_uint2(0, 0) : look(a.start + slot_of(a, order / kRun, group, lane));
}
// ... and, after a barrier, the state in front of tile `order` (u: the first look)
template <int W, int K> __device__ __forceinline__ float2 state_in_front(const ScanArgs& a, const TileShared<W, K>& sh, int order, int group, int lane, uint2 u) {
  float2 v = make_float2(0.f, 0.f);
  const int run = order / kRun;
  bool cut = run == 0;
#pragma unroll
  for (int w = 0; w < W; ++w) cut = cut || sh.seg_closed[w];
  if (!cut) {
    const uint2* from = a.start + slot_of(a, run, group, lane);
    const long long t0 = clock64();
    while ((u.x == kAbsent || u.y == kAbsent) && !out_of_time(a, t0)) u = look(from);
    __syncwarp();
    v = make_float2(__uint_as_float(u.x), __uint_as_float(u.y));
  }
#pragma unroll
  for (int w = 0; w < W; ++w) {
    const float4 p = sh.seg[w][lane];
    v = sh.seg_closed[w] ? make_float2(p.z, p.w) : make_float2(fmaf(p.x, v.x, p.z), fmaf(p.y, v.y, p.w));
  }
  return v;
}

// fold of warps [w0, w1) in time order (dir 1) or against it, applied to `in`
__device__ __forceinline__ float2 through(const float4 (*ab)[32], const unsigned* fresh, int lane, int w0, int w1, int dir, float2 in) {
#pragma unroll 4
  for (int w = w0; w != w1; w += dir) {
    const float4 p = ab[w][lane];
    in = fresh[w] ? make_float2(p.z, p.w) : make_float2(fmaf(p.x, in.x, p.z), fmaf(p.y, in.y, p.w));
  }
  return in;
}
// the tile's own pair and whether it is closed
template <int W> __device__ __forceinline__ float4 fold_tile(const float4 (*abs)[32], const unsigned* fresh, int lane, int dir, bool* closed) {
  float4 ab = make_float4(1.f, 1.f, 0.f, 0.f);
  *closed = false;
#pragma unroll
  for (int i = 0; i < W; ++i) {
    const int w = dir > 0 ? i : W - 1 - i;
    const float4 p = abs[w][lane];
    if (fresh[w]) { ab = make_float4(0.f, 0.f, p.z, p.w); *closed = true; }
    else ab = make_float4(ab.x * p.x, ab.y * p.y, fmaf(p.x, ab.z, p.z), fmaf(p.y, ab.w, p.w));
  }
  return ab;
}

// Tiles in the order they are handed out.  With an exchange area the counter decides (it starts at kAbsent, so the first
// ticket is 0 after the increment); without one any order will do.
__device__ __forceinline__ unsigned take_tickets(const ScanArgs& a, unsigned count) { return atomicAdd(a.counter, count) + 1u; }

// initial states of the rows that start a sequence: v[r] for the bits of m.from_h0, else 0
template <int CH, int kRows>
__device__ __forceinline__ void load_h0(const ScanArgs& a, const RowMarks& m, int c, Vec<CH> (&v)[kRows]) {
#pragma unroll
  for (int r = 0; r < kRows; ++r) {
    const size_t at = (size_t)__shfl_sync(0xffffffffu, m.seq, r) * a.cols + c;
    const bool want = a.h0 && (m.from_h0 >> r & 1);
#pragma unroll
    for (int e = 0; e < CH; ++e) {
      v[r].v[e] = 0.f;
      if (want && a.h0dt == DRAGON_F32) v[r].v[e] = __ldg(reinterpret_cast<const float*>(a.h0) + at + e);
      if (want && a.h0dt == DRAGON_BF16) v[r].v[e] = bf16_low(__ldg(reinterpret_cast<const unsigned short*>(a.h0) + at + e));
    }
  }
}

// One tile's rows of one warp, of N tensors, as they come from memory; rows behind the tensor repeat its last one
template <int DT, int CH, int N, int kRows> struct TileRows {
  Cell<DT, CH> v[N][kRows];
  __device__ __forceinline__ Vec<CH> get(int k, int r) const {
    Vec<CH> x;
#pragma unroll
    for (int e = 0; e < CH; ++e) x.v[e] = v[k][r].get(e);
    return x;
  }
  // asks L2 for the warp's rows of a tile that comes later: columns [c0, c0 + 32 CH) of kRows rows, in quarters
  static __device__ __forceinline__ void ask(const ScanArgs& a, int row0, int c0, int lane) {
    const void* src[3] = {a.gate, a.x, a.dh};
    const int dt[3] = {a.gdt, a.xdt, a.dhdt};
    const int c = min(c0 + (lane & 3) * 8 * CH, a.cols - 1);
#pragma unroll
    for (int r0 = 0; r0 < kRows; r0 += 8) {
      const size_t at = (size_t)min(row0 + r0 + (lane >> 2), a.rows - 1) * a.cols + c;
#pragma unroll
      for (int k = 0; k < N; ++k)
        asm volatile("prefetch.global.L2 [%0];" ::"l"(reinterpret_cast<const char*>(src[k]) + at * element_bytes<DT>(dt[k])));
    }
  }
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

// A tile between its fold and its output: f and b = (1 - f) x (+ f h0 where a sequence starts) of a thread's rows
template <int CH, int kRows> struct Folded {
  Vec<CH> f[kRows], b[kRows];
  unsigned fresh;      // rows that start afresh
  int n;               // rows inside the tensor
  Place at;
};

// Persistent CTAs.  While a tile waits for what is in front of it, the next tile's rows are on their way.
template <int DT, int CH>
__global__ void __launch_bounds__(kFwdWarps * 32, kFwdCtas<CH>) scan_kernel(const ScanArgs a) {
  constexpr int W = kFwdWarps, kRows = rows_per_warp<W>();
  __shared__ TileShared<W, 3> sh;
  if (a.status_clear && blockIdx.x == 0 && threadIdx.x == 0) *a.status_clear = 0;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const unsigned n = (unsigned)a.tiles * a.groups;
  unsigned ticket = blockIdx.x;          // of the tile whose rows are on their way
  if (a.pair) {
    if (threadIdx.x == 0) sh.ticket[0] = take_tickets(a, 1);
    __syncthreads();
    ticket = sh.ticket[0];
    __syncthreads();
  }
  TileRows<DT, CH, 2, kRows> rows;
  auto load = [&] {
    if (ticket >= n) return;
    const Place p = Place::of<false>(a, ticket);
    rows.load(a, p.tile * kScanTileRows + warp * kRows, min((p.group * 32 + lane) * CH, a.cols - CH));
  };
  auto column = [&](const Place& p) { return min((p.group * 32 + lane) * CH, a.cols - CH); };
  // the rows that have come become a folded tile; the next ones are sent for
  auto fold = [&](Folded<CH, kRows>& o, int copy) {
    o.at = Place::of<false>(a, ticket);
    const RowMarks m = row_marks<W>(a, o.at.tile * kScanTileRows + warp * kRows, lane);
    o.fresh = m.fresh;
    o.n = m.n;
#pragma unroll
    for (int r = 0; r < kRows; ++r) {
      Vec<CH> keep;
      gate_of(rows.get(0, r), &o.f[r], &keep);
      o.b[r] = mul(keep, rows.get(1, r));
    }
    if (m.n < kRows) {       // rows behind the tensor pass the state on
#pragma unroll
      for (int r = 0; r < kRows; ++r)
        if (r >= m.n) { o.f[r] = splat<CH>(1.f); o.b[r] = splat<CH>(0.f); }
    }
    if (a.h0 && m.from_h0) {
      Vec<CH> v[kRows];
      load_h0<CH, kRows>(a, m, column(o.at), v);
#pragma unroll
      for (int r = 0; r < kRows; ++r)
        if (m.from_h0 >> r & 1) o.b[r] = fma(o.f[r], v[r], o.b[r]);
    }
    Vec<CH> A = splat<CH>(1.f), B = splat<CH>(0.f);
    if (m.fresh == 0) {
#pragma unroll
      for (int r = 0; r < kRows; ++r) { A = mul(A, o.f[r]); B = fma(o.f[r], B, o.b[r]); }
    } else {
#pragma unroll
      for (int r = 0; r < kRows; ++r) B = (m.fresh >> r & 1) ? o.b[r] : fma(o.f[r], B, o.b[r]);
    }
    sh.ab[copy][warp][lane] = make_float4(A.v[0], A.v[CH - 1], B.v[0], B.v[CH - 1]);
    if (lane == 0) sh.fresh[copy][warp] = m.fresh;
    if (threadIdx.x == W * 32 - 1) sh.ticket[copy] = a.pair ? take_tickets(a, 1) : ticket + gridDim.x;
    __syncthreads();
    ticket = sh.ticket[copy];
    load();
    if (a.pair && warp == 0) {
      bool closed;
      const float4 ab = fold_tile<W>(sh.ab[copy], sh.fresh[copy], lane, 1, &closed);
      publish_pair(a, o.at.tile, o.at.group, lane, ab, closed);
      if (closed) publish_start(a, o.at.tile, o.at.group, lane, make_float2(ab.z, ab.w));
    }
  };
  // a folded tile's state in front, end state and output
  auto finish = [&](const Folded<CH, kRows>& o, int copy) {
    float2 front = make_float2(0.f, 0.f);
    if (a.pair) {
      const bool open = !(sh.fresh[copy][0] & 1);         // the tile's first row goes on from the tile before
      if (open) {
        const uint2 u = early_start(a, o.at.tile, o.at.group, lane);
        fold_run<DT == DRAGON_BF16 ? kRun / W : kRun / W / 2>(a, sh, o.at.tile, o.at.group, warp, lane);
        __syncthreads();
        front = state_in_front(a, sh, o.at.tile, o.at.group, lane, u);
      }
      if (warp == 0 && o.at.tile % kRun == kRun - 1) {
        bool closed;
        const float4 ab = fold_tile<W>(sh.ab[copy], sh.fresh[copy], lane, 1, &closed);
        if (!closed) publish_start(a, o.at.tile, o.at.group, lane, make_float2(fmaf(ab.x, front.x, ab.z), fmaf(ab.y, front.y, ab.w)));
      }
    }
    const int c = column(o.at), row0 = o.at.tile * kScanTileRows + warp * kRows;
    const bool mine = (o.at.group * 32 + lane) * CH < a.cols;
    if (warp == 0 && a.carry && mine) {
      float* p = a.carry + (size_t)o.at.tile * a.cols + c;
      p[0] = front.x;
      if (CH == 2) p[1] = front.y;
    }
    if (!a.h) return;
    const float2 in = through(sh.ab[copy], sh.fresh[copy], lane, 0, warp, 1, front);
    Vec<CH> h;
    h.v[0] = in.x;
    h.v[CH - 1] = CH == 2 ? in.y : in.x;
    const int es = element_bytes<DT>(a.hdt);
    char* p = reinterpret_cast<char*>(a.h) + ((size_t)row0 * a.cols + c) * es;
    const size_t step = (size_t)a.cols * es;
    if (o.fresh == 0 && o.n == kRows) {
#pragma unroll
      for (int r = 0; r < kRows; ++r, p += step) {
        h = fma(o.f[r], h, o.b[r]);
        if (mine) store_cell<DT, CH>(p, a.hdt, h.v);
      }
    } else {
#pragma unroll
      for (int r = 0; r < kRows; ++r, p += step) {
        h = (o.fresh >> r & 1) ? o.b[r] : fma(o.f[r], h, o.b[r]);
        if (mine && r < o.n) store_cell<DT, CH>(p, a.hdt, h.v);
      }
    }
  };
  // three copies of the pairs in turn: a copy is written again only behind two barriers that follow its last use
  load();
  Folded<CH, kRows> tile;
  for (int copy = 0; ticket < n; copy = copy == 2 ? 0 : copy + 1) {
    fold(tile, copy);
    finish(tile, copy);
  }
}

template <int DT, int CH>
__global__ void __launch_bounds__(kBwdWarps * 32, kBwdCtas) scan_bwd_kernel(const ScanArgs a) {
  constexpr int W = kBwdWarps, kRows = rows_per_warp<W>();
  __shared__ TileShared<W, 2> sh;        // copy 0: the state's pairs, copy 1: the gradient's
  if (a.status_clear && blockIdx.x == 0 && threadIdx.x == 0) *a.status_clear = 0;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const unsigned n = (unsigned)a.tiles * a.groups;
  const bool plain_out = a.dx && a.dgate && a.dxdt == DRAGON_F32 && a.dgdt == DRAGON_F32;
  unsigned ticket = blockIdx.x;
  if (a.pair) {
    if (threadIdx.x == 0) sh.ticket[0] = take_tickets(a, 1);
    __syncthreads();
    ticket = sh.ticket[0];
    __syncthreads();
  }
  while (ticket < n) {
    const Place at = Place::of<true>(a, ticket);      // tickets against time
    const int tile = at.tile, group = at.group, order = a.tiles - 1 - tile;
    const int c0 = (group * 32 + lane) * CH, row0 = tile * kScanTileRows + warp * kRows;
    const bool mine = c0 < a.cols;
    const int c = min(c0, a.cols - CH);
    TileRows<DT, CH, 3, kRows> rows;
    rows.load(a, row0, c);
    float carry[2] = {0.f, 0.f};
#pragma unroll
    for (int e = 0; e < CH; ++e) carry[e] = __ldg(a.carry + (size_t)tile * a.cols + c + e);
    const RowMarks m = row_marks<W>(a, row0, lane);
    const bool plain = m.n == kRows && m.fresh == 0;
    Vec<CH> f[kRows], keep[kRows], hp[kRows];      // hp: the state in front of the row
#pragma unroll
    for (int r = 0; r < kRows; ++r) gate_of(rows.get(0, r), &f[r], &keep[r]);
    if (m.n < kRows) {       // rows behind the tensor pass the state and the gradient on
#pragma unroll
      for (int r = 0; r < kRows; ++r)
        if (r >= m.n) { f[r] = splat<CH>(1.f); keep[r] = splat<CH>(0.f); }
    }
    // pairs of the state and of the gradient e -> f (dh + e)
    Vec<CH> A = splat<CH>(1.f), B = splat<CH>(0.f), E = splat<CH>(0.f);
    if (plain) {
#pragma unroll
      for (int r = 0; r < kRows; ++r) { A = mul(A, f[r]); B = fma(f[r], B, mul(keep[r], rows.get(1, r))); }
#pragma unroll
      for (int r = kRows - 1; r >= 0; --r) E = mul(f[r], add(rows.get(2, r), E));
    } else {
      load_h0<CH, kRows>(a, m, c, hp);         // for now: h0 where a sequence starts
#pragma unroll
      for (int r = 0; r < kRows; ++r) {
        A = mul(A, f[r]);
        B = fma(f[r], (m.fresh >> r & 1) ? hp[r] : B, r < m.n ? mul(keep[r], rows.get(1, r)) : splat<CH>(0.f));
      }
#pragma unroll
      for (int r = kRows - 1; r >= 0; --r) {
        if (r < m.n) E = mul(f[r], add(rows.get(2, r), E));
        if (m.fresh >> r & 1) E = splat<CH>(0.f);
      }
    }
    sh.ab[0][warp][lane] = make_float4(A.v[0], A.v[CH - 1], B.v[0], B.v[CH - 1]);
    sh.ab[1][warp][lane] = make_float4(A.v[0], A.v[CH - 1], E.v[0], E.v[CH - 1]);
    if (lane == 0) sh.fresh[0][warp] = m.fresh;
    if (threadIdx.x == 0) sh.ticket[0] = a.pair ? take_tickets(a, 1) : ticket + gridDim.x;
    __syncthreads();
    ticket = sh.ticket[0];
    if (ticket < n) {        // (registers hold one tile only: the next one comes as far as L2)
      const Place next = Place::of<true>(a, ticket);
      TileRows<DT, CH, 3, kRows>::ask(a, next.tile * kScanTileRows + warp * kRows, next.group * 32 * CH, lane);
    }
    bool closed = false;
    float4 ab;
    uint2 u = make_uint2(0, 0);
    if (a.pair) {
      u = early_start(a, order, group, lane);
      if (warp == W - 1) {
        ab = fold_tile<W>(sh.ab[1], sh.fresh[0], lane, -1, &closed);
        publish_pair(a, order, group, lane, ab, closed);
        if (closed) publish_start(a, order, group, lane, make_float2(ab.z, ab.w));
      }
      fold_run<kRun / W>(a, sh, order, group, warp, lane);
    }
    {
      const float2 in = through(sh.ab[0], sh.fresh[0], lane, 0, warp, 1, make_float2(carry[0], carry[1]));
      Vec<CH> h;
      h.v[0] = in.x;
      h.v[CH - 1] = CH == 2 ? in.y : in.x;
#pragma unroll
      for (int r = 0; r < kRows; ++r) {
        if (!plain && (m.fresh >> r & 1)) h = hp[r];
        hp[r] = h;
        h = fma(f[r], h, mul(keep[r], rows.get(1, r)));
      }
    }
    float2 front = make_float2(0.f, 0.f);
    if (a.pair) {
      __syncthreads();
      front = state_in_front(a, sh, order, group, lane, u);
      if (warp == W - 1 && !closed) publish_start(a, order, group, lane, make_float2(fmaf(ab.x, front.x, ab.z), fmaf(ab.y, front.y, ab.w)));
    }
    const float2 in = through(sh.ab[1], sh.fresh[0], lane, W - 1, warp, -1, front);
    Vec<CH> d;
    d.v[0] = in.x;
    d.v[CH - 1] = CH == 2 ? in.y : in.x;
    const Vec<CH> minus = splat<CH>(-1.f);
    if (plain && plain_out) {
      const size_t step = (size_t)a.cols * 4, at_last = ((size_t)(row0 + kRows - 1) * a.cols + c) * 4;
      char *px = reinterpret_cast<char*>(a.dx) + at_last, *pg = reinterpret_cast<char*>(a.dgate) + at_last;
#pragma unroll
      for (int r = kRows - 1; r >= 0; --r, px -= step, pg -= step) {
        d = add(d, rows.get(2, r));
        const Vec<CH> dx = mul(d, keep[r]), dz = mul(mul(dx, f[r]), fma(rows.get(1, r), minus, hp[r]));
        d = mul(d, f[r]);
        if (mine) { store_cell<DRAGON_F32, CH>(px, DRAGON_F32, dx.v); store_cell<DRAGON_F32, CH>(pg, DRAGON_F32, dz.v); }
      }
    } else {
#pragma unroll
      for (int r = kRows - 1; r >= 0; --r) {
        if (r >= m.n) continue;
        d = add(d, rows.get(2, r));
        const Vec<CH> dx = mul(d, keep[r]), dz = mul(mul(dx, f[r]), fma(rows.get(1, r), minus, hp[r]));
        d = mul(d, f[r]);
        if (mine) {
          const size_t i = (size_t)(row0 + r) * a.cols + c;
          if (a.dx) store_cell<-1, CH>(reinterpret_cast<char*>(a.dx) + i * element_bytes<-1>(a.dxdt), a.dxdt, dx.v);
          if (a.dgate) store_cell<-1, CH>(reinterpret_cast<char*>(a.dgate) + i * element_bytes<-1>(a.dgdt), a.dgdt, dz.v);
        }
        if (m.fresh >> r & 1) {
          if (a.dh0) {
            const int row = row0 + r, seq = row / a.length;
            if (row - seq * a.length == 0) {         // a sequence's first row: what reaches its initial state (nothing past a reset)
              const Vec<CH> g = (m.from_h0 >> r & 1) ? d : splat<CH>(0.f);
              if (mine) store_cell<-1, CH>(reinterpret_cast<char*>(a.dh0) + ((size_t)seq * a.cols + c) * element_bytes<-1>(a.dh0dt), a.dh0dt, g.v);
            }
          }
          d = splat<CH>(0.f);
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
    Vec<CH> v, f, keep;
#pragma unroll
    for (int e = 0; e < CH; ++e) v.v[e] = z.get(e);
    gate_of(v, &f, &keep);
#pragma unroll
    for (int e = 0; e < CH; ++e) {
      h[e] = keep.v[e] * x.get(e);
      if (from_h0) h[e] = fmaf(f.v[e], h0.get(e), h[e]);
    }
    store_cell<DT, CH>(reinterpret_cast<char*>(a.h) + at * element_bytes<DT>(a.hdt), a.hdt, h);
  }
}

int columns_per_lane(int64_t cols) { return cols % 2 == 0 ? 2 : 1; }    // pairs of columns are aligned in every row

struct Scratch { size_t pair, start, bytes; };
Scratch scratch_layout(int64_t rows, int64_t cols) {
  const int64_t tiles = (rows + kScanTileRows - 1) / kScanTileRows, per_group = 32 * columns_per_lane(cols), groups = (cols + per_group - 1) / per_group;
  Scratch s;
  s.pair = 256;            // the counter stands in front
  s.start = s.pair + (size_t)(tiles * groups) * 32 * sizeof(uint4);
  s.bytes = s.start + (size_t)((tiles / kRun + 1) * groups) * 32 * sizeof(uint2);
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
  a.wait_budget = kWaitBudgetCycles;
  // failure-detection test only: a short budget and a first tile that publishes nothing
  if (const char* e = std::getenv("DRAGON_SCAN_WAIT_BUDGET")) { const long long b = std::atoll(e); if (b > 0) a.wait_budget = std::min(b, kWaitBudgetCycles); }
  if (const char* e = std::getenv("DRAGON_SCAN_WITHHOLD")) a.withhold = e[0] == '1';
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
  a.start = reinterpret_cast<uint2*>(p + s.start);
  return cudaMemsetAsync(p, 0xff, s.bytes, reinterpret_cast<cudaStream_t>(r.stream));
}

template <int DT> cudaError_t launch_fwd(const ScanArgs& a, int sm_count, cudaStream_t st) {
  const bool two = columns_per_lane(a.cols) == 2;
  if (a.length == 1 && !a.carry) {
    const int per = two ? 2 : 1;
    const dim3 grid((a.cols + 256 * per - 1) / (256 * per), std::min(a.rows, 32768));
    if (two) scan_step_kernel<DT, 2><<<grid, 256, 0, st>>>(a);
    else scan_step_kernel<DT, 1><<<grid, 256, 0, st>>>(a);
    return cudaGetLastError();
  }
  const unsigned n = (unsigned)a.tiles * a.groups;
  if (two) scan_kernel<DT, 2><<<std::min(n, (unsigned)(sm_count * kFwdCtas<2>)), kFwdWarps * 32, 0, st>>>(a);
  else scan_kernel<DT, 1><<<std::min(n, (unsigned)(sm_count * kFwdCtas<1>)), kFwdWarps * 32, 0, st>>>(a);
  return cudaGetLastError();
}
template <int DT> cudaError_t launch_bwd(const ScanArgs& a, int sm_count, cudaStream_t st) {
  const unsigned grid = std::min((unsigned)a.tiles * a.groups, (unsigned)(sm_count * kBwdCtas));
  if (columns_per_lane(a.cols) == 2) scan_bwd_kernel<DT, 2><<<grid, kBwdWarps * 32, 0, st>>>(a);
  else scan_bwd_kernel<DT, 1><<<grid, kBwdWarps * 32, 0, st>>>(a);
  return cudaGetLastError();
}

}  // namespace

size_t scan_scratch_bytes(int64_t rows, int64_t cols) { return scratch_layout(rows, cols).bytes; }

cudaError_t launch_scan(const StepRun& r) {
  ScanArgs a{};
  cudaStream_t st = reinterpret_cast<cudaStream_t>(r.stream);
  const cudaError_t e = scan_args(r, false, &a);
  if (e != cudaSuccess) return e;
  const bool same = a.gdt == a.xdt && (!a.h || a.hdt == a.gdt);
  return !same ? launch_fwd<-1>(a, r.sm_count, st) : a.gdt == DRAGON_F32 ? launch_fwd<DRAGON_F32>(a, r.sm_count, st) : launch_fwd<DRAGON_BF16>(a, r.sm_count, st);
}

cudaError_t launch_scan_bwd(const StepRun& r) {
  ScanArgs a{};
  cudaStream_t st = reinterpret_cast<cudaStream_t>(r.stream);
  const cudaError_t e = scan_args(r, true, &a);
  if (e != cudaSuccess) return e;
  const bool same = a.gdt == a.xdt && a.dhdt == a.gdt;
  return !same ? launch_bwd<-1>(a, r.sm_count, st) : a.gdt == DRAGON_F32 ? launch_bwd<DRAGON_F32>(a, r.sm_count, st) : launch_bwd<DRAGON_BF16>(a, r.sm_count, st);
}

}  // namespace dragon
