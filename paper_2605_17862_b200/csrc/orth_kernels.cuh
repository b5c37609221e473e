// Orthogonalised updates: Newton-Schulz products over a list of matrices (sm_100a).
//
//   X = M / (|M| + eps);  steps times:  A = X X^T,  P = a I + b A + c A^2,  X <- P X;   out = scale X
//
// (X^T X and X P for a matrix with more rows than columns.)  A singular value s of X becomes a s + b s^3 + c s^5 in each step.
//
// Numbers.  The steps amplify small singular values, and with them whatever rounding has put there: by up to a^steps (485 for
// five steps of 3.4445).  In bf16 the rounding of X in the first steps comes out as 1 % of the result and, where a few strong directions
// stand above the others, as 10 % and more.  So X, A and P are held in fp16 under powers of two that keep them just below its largest
// number (11 bits, everything down to 2^-29 of the largest normal): an eighth of bf16's rounding at the same rate.  X has a second
// plane of what the rounding left (together 22 bits) while the steps still ahead amplify by 32 or more, and P X then takes both.  The
// rounding of A and P multiplies what is there and averages out over their elements, but for a shorter side of up to 16: one plane
// takes 2 x 31, 2 x 600, 3 x 300 and 4 x 3,000 matrices 0.5 % off one time in a hundred and 0.9 % at most, 16 x 300 0.26 % and 17 x 40 0.30 %
// (of which 0.17 % are a bf16 result's own rounding), whatever the longer side.  There A and P have two planes: 0.22 % at most from
// 257 columns on.  Results in fp32, and matrices so short that X's roundings do not average out either (16 x 256: 2 x 17 0.43 % off
// otherwise, 0.26 % as built), have two planes throughout, three products each.
// The scales follow from a bound on the largest singular value in each step, which the host takes from the coefficients for a
// largest one of 1.  Where eps makes it less, 2^-lift or below, X is held 2^lift higher (A 4^lift), and lift falls from step to step by as
// much as the bound says that the step may amplify: a norm far below eps keeps its bits.
//
// Everything lies in one workspace in panels of 64 columns ([panel][rows][64], rows and columns padded with zeros to 64), so that one
// tensor map serves every operand, along its rows or across them, and tiles need no edges.  A and A^2 are symmetric: only the
// tiles on and below the diagonal are computed and stored, and what lies above is read across out of those below.
#pragma once

#include "tensor_core.cuh"

namespace fopd {

// What has two planes: nothing but X in some steps; A and P; X too, throughout.
enum OrthHeld : uint8_t { kOrthPlain, kOrthSquare, kOrthFull };

struct OrthMatrix {
  const void *data;
  void *out;
  int64_t pitch, out_pitch;
  int rows, cols;      // of the matrix
  int rp, cp, mp;      // padded to 64; mp: the shorter side
  int x[2], x_lo;      // workspace rows (of 64 elements) where X starts (two in turn), and from its first plane to the second
  int a, p, m_lo;      // the same for A and P
  uint32_t two_planes; // bit k: X of step k has its second plane
  int space;           // workspace rows of all of it
  int sym_tile, x_tile;  // first tile of the matrix
  int norm_block, norm_blocks, load_block;
  float scale;
  uint8_t dtype, out_dtype, tall;
  OrthHeld held;
  __host__ __device__ __forceinline__ bool square() const { return held >= kOrthSquare; }
  __host__ __device__ __forceinline__ bool full() const { return held == kOrthFull; }
};

constexpr int kOrthThreads = 256;
// Blocks of 64 that an accumulator adds up where the result is fp32, and in A^2, whose terms the rest of the polynomial nearly cancels:
// with every block of that taken out a result is 3.1e-6 off instead of 4.9e-6 (fp32 products 2.6e-6 to 3.2e-6) for 1.5 % of the time, with every
// block of all three 2.8e-6 for 5 %.
constexpr int kOrthChunk = 2, kOrthPolyChunk = 1;

struct OrthNorm {
  float factor;  // 2^lift / ((|M| + eps) 2^e)
  int lift;      // |M| / (|M| + eps) in [2^-(lift + 1), 2^-lift]
};
struct OrthWorkspace {
  OrthNorm *norm;      // per matrix
  int *lifted;         // whether any has a lift above 0
  int *done;           // per matrix: units of finished tiles (one for each epilogue warp); behind the last one the tiles claimed
  double *partial;     // per block of the norm
  __half *planes;
};

// The list travels as a kernel parameter (at most 32,764 bytes), in sizes so that short lists are quick to hand over: all that
// the products' tiles need of it comes through the constant cache, which waiting for other tiles' results leaves alone.
template <int N>
struct OrthTable {
  int n;
  int norm_chunk;  // elements to a block of the norm
  int load_cols;   // columns, by 64 rows, to a block of the load
  OrthMatrix m[N];
};

// The entry whose range (by `first`) holds i.
template <class First>
__device__ __forceinline__ int find_entry(int n, int i, First first) {
  int lo = 0, hi = n - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) / 2;
    if (first(mid) <= i) lo = mid;
    else hi = mid - 1;
  }
  return lo;
}

__device__ __forceinline__ float load_element(const void *p, int64_t i, int dtype) {
  return dtype == FOPD_BF16 ? Elem<FOPD_BF16>::load1(p, i) : Elem<FOPD_F32>::load1(p, i);
}

__device__ __forceinline__ double block_sum(double s, double *scratch) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
  if ((threadIdx.x & 31) == 0) scratch[threadIdx.x >> 5] = s;
  __syncthreads();
  double t = 0.0;
  for (int w = 0; w < kOrthThreads / 32; ++w) t += scratch[w];
  __syncthreads();
  return t;
}

// Sums of squares in fp64, a block to 16,384 elements (4,096 for short lists).
template <int N>
__global__ void __launch_bounds__(kOrthThreads) orth_norm_kernel(const __grid_constant__ OrthTable<N> tab, OrthWorkspace ws) {
  __shared__ double scratch[kOrthThreads / 32];
  grid_wait();
  const int k = find_entry(tab.n, (int)blockIdx.x, [&](int j) { return tab.m[j].norm_block; });
  const OrthMatrix &m = tab.m[k];
  const int64_t all = (int64_t)m.rows * m.cols, from = (int64_t)((int)blockIdx.x - m.norm_block) * tab.norm_chunk;
  const int64_t to = from + tab.norm_chunk < all ? from + tab.norm_chunk : all;
  double s = 0.0;
  const int size = m.dtype == FOPD_BF16 ? 2 : 4, per = 16 / size;
  const bool dense = m.rows == 1 || m.pitch == m.cols;
  if (dense && ((uintptr_t)m.data & 15) == 0) {  // (chunks start at whole vectors)
    const char *base = static_cast<const char *>(m.data);
#pragma unroll 4
    for (int64_t i = from + threadIdx.x * per; i + per <= to; i += kOrthThreads * per) {
      const uint4 v = *reinterpret_cast<const uint4 *>(base + i * size);
      if (m.dtype == FOPD_BF16) {
        float x[8];
        Elem<FOPD_BF16>::unpack(v, x);
#pragma unroll
        for (int e = 0; e < 8; ++e) s = fma((double)x[e], (double)x[e], s);
      } else {
        float x[4];
        Elem<FOPD_F32>::unpack(v, x);
#pragma unroll
        for (int e = 0; e < 4; ++e) s = fma((double)x[e], (double)x[e], s);
      }
    }
    const int64_t tail = from + (to - from) / per * per + threadIdx.x;
    if (tail < to) {
      const double x = load_element(base, tail, m.dtype);
      s = fma(x, x, s);
    }
  } else {
    for (int64_t i = from + threadIdx.x; i < to; i += kOrthThreads) {
      const int64_t r = i / m.cols;
      const double x = load_element(m.data, r * m.pitch + (i - r * m.cols), m.dtype);
      s = fma(x, x, s);
    }
  }
  s = block_sum(s, scratch);
  if (threadIdx.x == 0) ws.partial[blockIdx.x] = s;
  if (threadIdx.x == 0 && blockIdx.x == 0) *ws.lifted = 0;
}

__device__ __forceinline__ void split_half(float x, __half &hi, __half &lo) {
  hi = __float2half_rn(x);
  lo = __float2half_rn(x - __half2float(hi));
}

// Into the workspace times 2^e, with 2^e |M| in [2^14, 2^15): no element leaves fp16's range, and bf16 ones are exact down to 2^-24.
// A block takes 64 rows x 256 columns (64 for short lists) and forms the norm from the partial sums itself (in order).
template <int N>
__global__ void __launch_bounds__(kOrthThreads) orth_load_kernel(const __grid_constant__ OrthTable<N> tab, OrthWorkspace ws, float eps,
                                                                 int32_t *status) {
  __shared__ double scratch[kOrthThreads / 32];
  grid_wait();
  const int k = find_entry(tab.n, (int)blockIdx.x, [&](int j) { return tab.m[j].load_block; });
  const OrthMatrix &m = tab.m[k];
  const int block = (int)blockIdx.x - m.load_block;
  double s = 0.0;
  for (int i = threadIdx.x; i < m.norm_blocks; i += kOrthThreads) s += ws.partial[m.norm_block + i];
  __shared__ double scale_of_block;
  __shared__ int exponent_of_block;
  s = block_sum(s, scratch);
  const double norm = sqrt(s);
  const bool finite = norm <= 1.7e308;
  if (threadIdx.x == 0) {
    int e = 0;
    if (finite && norm > 0.0) {
      frexp(norm, &e);  // norm in [2^(e-1), 2^e)
      e = 15 - e;
    }
    exponent_of_block = finite ? e : 0;
    scale_of_block = finite ? ldexp(1.0, e) : __longlong_as_double(0x7ff8000000000000ll);
  }
  __syncthreads();
  const double scale = scale_of_block;
  const int e = exponent_of_block;
  if (block == 0 && threadIdx.x == 0) {
    OrthNorm of = {finite ? 0.f : __int_as_float(0x7fffffff), 0};
    if (finite && norm > 0.0) {
      const double with_eps = norm + (double)eps;
      int a, b;
      const double f = frexp(norm, &a), g = frexp(with_eps, &b);
      of.lift = max(0, b - a - (f >= g ? 1 : 0));
      of.factor = (float)(1.0 / ldexp(with_eps, e - of.lift));
    }
    ws.norm[k] = of;
    if (of.lift > 0) *ws.lifted = 1;
    ws.done[k] = 0;
    if (k == 0) ws.done[tab.n] = 0;
    if (!finite && status) atomicOr(status, FOPD_DEV_NONFINITE);
  }
  const int col_blocks = (m.cp + tab.load_cols - 1) / tab.load_cols;
  const int row0 = block / col_blocks * 64, col0 = block % col_blocks * tab.load_cols;
  const int size = m.dtype == FOPD_BF16 ? 2 : 4;
  const bool two = m.two_planes & 1;
  const bool aligned = (((uintptr_t)m.data | (uintptr_t)(m.rows > 1 ? m.pitch * size : 0)) & 15) == 0;
  const float f = (float)scale;  // (2^e may be beyond fp32 for the smallest matrices: then in fp64)
  const bool in_range = e > -126 && e < 126;
#pragma unroll 4
  for (int u = threadIdx.x; u < 64 * (tab.load_cols / 8); u += kOrthThreads) {
    const int c = col0 + (u / 64 / 8) * 64 + (u & 7) * 8, r = row0 + ((u >> 3) & 63);
    if (c >= m.cp) continue;
    float x[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    if (r < m.rows) {
      const int64_t at = r * m.pitch + c;
      if (aligned && c + 8 <= m.cols) {
        const char *p = static_cast<const char *>(m.data) + at * size;
        if (m.dtype == FOPD_BF16) Elem<FOPD_BF16>::unpack(*reinterpret_cast<const uint4 *>(p), x);
        else {
          float y[4];
          Elem<FOPD_F32>::unpack(*reinterpret_cast<const uint4 *>(p), y);
#pragma unroll
          for (int q = 0; q < 4; ++q) x[q] = y[q];
          Elem<FOPD_F32>::unpack(*reinterpret_cast<const uint4 *>(p + 16), y);
#pragma unroll
          for (int q = 0; q < 4; ++q) x[4 + q] = y[q];
        }
      } else {
#pragma unroll
        for (int q = 0; q < 8; ++q)
          if (c + q < m.cols) x[q] = load_element(m.data, at + q, m.dtype);
      }
    }
    __half hi[8], lo[8];
#pragma unroll
    for (int q = 0; q < 8; ++q) split_half(in_range ? x[q] * f : (float)((double)x[q] * scale), hi[q], lo[q]);
    const int64_t row = (int64_t)m.x[0] + (int64_t)(c / 64) * m.rp + r;
    *reinterpret_cast<uint4 *>(ws.planes + row * 64 + (c & 63)) = *reinterpret_cast<uint4 *>(hi);
    if (two) *reinterpret_cast<uint4 *>(ws.planes + (row + m.x_lo) * 64 + (c & 63)) = *reinterpret_cast<uint4 *>(lo);
  }
}

// ------------------------------------------------------------------ the products
// All steps of all matrices in one launch.  Tiles are numbered step by step and in a step phase by phase over the whole list; one
// that needs the results of the phase before waits for that phase of its own matrix only, so that the tail of one matrix's phase runs
// beside the other matrices' tiles, and a phase of a single matrix costs a signal through the L2 instead of a launch.
// Large lists are bound by the tensor pipe (14 matrices of two blocks of width 2,048: 81 to 83 % busy, 2.64 to 2.75 ms); small ones by the
// chain of three phases a step, each 6 to 16 us from the first load to the last count (256 x 1,024 in fp32: 157 us for five steps, norm and load 15 of them).
enum OrthPhase { kOrthGram = 0, kOrthPoly = 1, kOrthApply = 2 };
constexpr int kOrthMostSteps = 16;

// Factors of one step (powers of two but for the coefficients).  Values in the workspace are X 2^ex, A 2^ea, P 2^ep, but for the lift.
struct OrthStep {
  float gram;                   // from X's products to A's scale (first step: on top of the norm's factor squared)
  float poly_a, poly_b, poly_c; // P = a I + b A + c A^2, from A's values and A's products to P's scale
  float apply;                  // from P X to the next X's scale; last step: to 1 (first step: on top of the norm's factor)
  int fall;                     // what is left of the lift in this step: its first value less this, at least 0
};

template <int kCtas, int kN, int N>
struct OrthJob {
  static constexpr bool kFp16 = true, kTurns = true, kClaimed = true;
  static constexpr int kRows = kCtas * 128;
  static_assert(kN == kRows, "symmetric tiles");
  struct Params {
    CUtensorMap boxes, boxes_along, rows_out;
    OrthWorkspace ws;
    OrthStep step[kOrthMostSteps];
    OrthTable<N> tab;
    int steps;
    int sym_tiles, x_tiles;  // of the list, in each step
    int32_t *status;
  };
  struct Ticket {
    int i;
    int of;        // matrix, step and phase
    int row, col;  // of the tile
    static __device__ __forceinline__ int pack(int k, int step, int phase) { return k << 8 | step << 2 | phase; }
    __device__ __forceinline__ int k() const { return of >> 8; }
    __device__ __forceinline__ int step() const { return of >> 2 & 63; }
    __device__ __forceinline__ int phase() const { return of & 3; }
    __device__ __forceinline__ int row0() const { return row * kRows; }
    __device__ __forceinline__ int col0() const { return col * kN; }
  };
  const Params &p;
  uint32_t staged_turn = 0;  // parity of this warp's copies into its staging buffers
  uint32_t order_turn = 1;   // and of the storing thread's handing them back
  int first_lift = 0;        // of the tile's matrix
  const bool lifted;         // (as a rule none is, and tiles are spared the reading: with it and ldexpf it was 2 % of small lists' time)
  __device__ explicit OrthJob(const Params &params) : p(params), lifted(*params.ws.lifted != 0) {}
  __device__ int64_t tiles() const { return (int64_t)p.steps * (2 * p.sym_tiles + p.x_tiles); }
  __device__ int32_t *status() const { return p.status; }
  __device__ int *counter() const { return p.ws.done + p.tab.n; }
  __device__ __forceinline__ bool last(const Ticket &o) const { return o.step() + 1 == p.steps; }
  __device__ __forceinline__ Ticket ticket(int i) const {
    Ticket o;
    o.i = i;
    const int per = 2 * p.sym_tiles + p.x_tiles, step = i / per;
    int t = i - step * per;
    const int phase = t < p.sym_tiles ? kOrthGram : t < 2 * p.sym_tiles ? kOrthPoly : kOrthApply;
    t -= phase * p.sym_tiles;
    int k;
    const OrthMatrix *tab = p.tab.m;
    if (phase == kOrthApply) {
      k = find_entry(p.tab.n, t, [&](int j) { return tab[j].x_tile; });
      t -= tab[k].x_tile;
      const int across = (tab[k].cp + kN - 1) / kN;
      o.row = t / across;
      o.col = t % across;
    } else {
      k = find_entry(p.tab.n, t, [&](int j) { return tab[j].sym_tile; });
      t -= tab[k].sym_tile;
      int r = (int)((sqrtf(8.f * t + 1.f) - 1.f) * 0.5f);
      while (r * (r + 1) / 2 > t) --r;
      while ((r + 1) * (r + 2) / 2 <= t) ++r;
      o.row = r;
      o.col = t - r * (r + 1) / 2;
    }
    o.of = Ticket::pack(k, step, phase);
    return o;
  }
  // Units of a matrix's tiles before this phase.
  __device__ __forceinline__ int units_before(const Ticket &o, const OrthMatrix &m) const {
    const int s = (m.mp + kN - 1) / kN, sym = s * (s + 1) / 2, x = ((m.rp + kRows - 1) / kRows) * ((m.cp + kN - 1) / kN);
    return kCtas * kEpilogueWarps * (o.step() * (2 * sym + x) + o.phase() * sym);
  }
  __device__ __forceinline__ bool ready(const Ticket &o, long long limit) const {
    const int want = units_before(o, p.tab.m[o.k()]);
    const int *done = p.ws.done + o.k();
    if (load_acquire(done) < want) {
      const long long t0 = clock64();
      while (load_acquire(done) < want)
        if (clock64() - t0 > limit) return false;
    }
    fence_async_global();  // (the copies that follow are of another proxy than the load)
    return true;
  }
  __device__ __forceinline__ void tile(const Ticket &o, int cta, Tile &t) const {
    const OrthMatrix &m = p.tab.m[o.k()];
    const int row0 = o.row0() + cta * 128, col0 = o.col0() + cta * (kN / kCtas);
    const bool x_two = m.two_planes >> o.step() & 1;
    const int x = m.x[o.step() & 1];
    // along: rows of the operand are rows of the plane; across: they are its columns
    const auto along = [&](int y, int pitch, int r, int lo) { return Operand{&p.boxes_along, 0, y + r, 0, pitch, 0, 128, lo, false}; };
    const auto across = [&](int y, int pitch, int r, int lo) { return Operand{&p.boxes, 0, y + r / 64 * pitch, 0, 64, 0, pitch, lo, true}; };
    // a symmetric operand: rows `r` of the tile that starts at `first`
    const auto symmetric = [&](int y, int r, int first, Operand &op, Turn &turn) {
      op = along(y, m.mp, r, m.m_lo);
      turn = {(first + kN) / 64, &p.boxes, y + r / 64 * m.mp, m.mp};
    };
    t.a_turn = t.b_turn = {1 << 30, &p.boxes, 0, 0};
    t.a_lo = t.b_lo = 0;
    t.passes = 1;
    t.chunk = m.full() ? kOrthChunk : kLongChunk;
    if (o.phase() == kOrthGram) {
      t.a = m.tall ? across(x, m.rp, row0, m.x_lo) : along(x, m.rp, row0, m.x_lo);
      t.b = m.tall ? across(x, m.rp, col0, m.x_lo) : along(x, m.rp, col0, m.x_lo);
      t.k_blocks = (m.tall ? m.rp : m.cp) / 64;
      if (m.full() && x_two) t.passes = 3, t.b_lo = 1, t.a_lo = 2;
    } else if (o.phase() == kOrthPoly) {
      symmetric(m.a, row0, o.row0(), t.a, t.a_turn);
      symmetric(m.a, col0, o.col0(), t.b, t.b_turn);
      t.k_blocks = m.mp / 64;
      if (m.square()) t.passes = 3, t.b_lo = 1, t.a_lo = 2;
      if (m.full()) t.chunk = kOrthPolyChunk;
    } else {
      t.k_blocks = m.mp / 64;
      uint32_t p_lo = 0, x_lo = 0;  // (the small terms first)
      if (m.square()) p_lo = 1u << (t.passes++ - 1);
      if (x_two) x_lo = 1u << (t.passes++ - 1);
      if (m.tall) {
        t.a = along(x, m.rp, row0, m.x_lo);
        symmetric(m.p, col0, o.col0(), t.b, t.b_turn);
        t.a_lo = x_lo, t.b_lo = p_lo;
      } else {
        symmetric(m.p, row0, o.row0(), t.a, t.a_turn);
        t.b = across(x, m.rp, col0, m.x_lo);
        t.a_lo = p_lo, t.b_lo = x_lo;
      }
    }
  }

  __device__ __forceinline__ const CUtensorMap *store_map() const { return &p.rows_out; }
  __device__ __forceinline__ int *done_counts() const { return p.ws.done; }
  // This warp's staging buffers are free.
  __device__ __forceinline__ bool buffers(const Accumulator &acc) {
    return __all_sync(0xffffffffu, mbar_wait_bounded(acc.order_empty, order_turn, kLongWaitCycles));
  }
  __device__ __forceinline__ void order(const Accumulator &acc, int which, int y, int z, int units) {
    fence_async_shared();
    __syncwarp();
    if (acc.lane == 0) {
      asm volatile("st.shared.v4.s32 [%0], {%1, %2, %3, %4};" ::"r"(acc.order), "r"(which), "r"(y), "r"(z), "r"(units) : "memory");
      mbar_arrive(acc.order_full);
    }
    order_turn ^= 1;
  }
  __device__ __forceinline__ bool finish(const Accumulator &acc) {
    const bool ok = buffers(acc);
    order(acc, -1, -1, -1, 0);
    return ok;
  }
  // 64 columns of this warp's rows into a staging buffer: the values, or what their rounding leaves.
  __device__ __forceinline__ void stage(const Accumulator &acc, int buf, const float *v, bool lo) {
    stage_box(acc.staging + buf * kStageBufBytes, acc.lane, [&](int j) {
      __half2 h = __floats2half2_rn(v[2 * j], v[2 * j + 1]);
      if (lo) h = __floats2half2_rn(v[2 * j] - __low2float(h), v[2 * j + 1] - __high2float(h));
      return *reinterpret_cast<uint32_t *>(&h);
    });
  }
  // All of a tile's columns (up to two panels) to one or two planes of a matrix at row y of its first panel, `pitch` rows to a panel;
  // panels beyond `have` do not exist.
  __device__ __forceinline__ bool put(const Ticket &o, const Accumulator &acc, const float (&v)[kN / 2], int have, int y, int pitch,
                                      bool two, int lo) {
    constexpr int kPanels = kN / 128;
    if constexpr (kPanels == 1) {  // both planes in one round
      if (!buffers(acc)) return false;
      if (have > 0) {
        stage(acc, 0, v, false);
        if (two) stage(acc, 1, v, true);
      }
      order(acc, o.k(), have > 0 ? y : -1, have > 0 && two ? y + lo : -1, 1);
    } else {
      for (int plane = 0; plane < (two ? 2 : 1); ++plane) {
        if (!buffers(acc)) return false;
        if (have > 0) stage(acc, 0, v, plane);
        if (have > 1) stage(acc, 1, v + 64, plane);
        const int at = y + plane * lo;
        order(acc, o.k(), have > 0 ? at : -1, have > 1 ? at + pitch : -1, plane == (two ? 1 : 0));
      }
    }
    return true;
  }

  // A plane of A's values at a warp's part of a tile of P: up to two panels into the staging buffers.
  __device__ __forceinline__ int square_panels(const OrthMatrix &m, int row0, int col0) const {
    return row0 >= m.mp ? 0 : max(0, min(kN / 128, (m.mp - col0) / 64));
  }
  __device__ __forceinline__ void stage_square(const Ticket &o, const OrthMatrix &m, int cta, const Accumulator &acc, int plane) {
    const int row0 = o.row0() + cta * 128 + acc.warp * 32, col0 = o.col0() + acc.half * (kN / 2);
    const int panels = square_panels(m, row0, col0);
    if (acc.lane != 0 || panels == 0) return;
    mbar_expect_tx(acc.staged, panels * kStageBufBytes);
    for (int c = 0; c < panels; ++c)
      tma_load<1>(acc.staging + c * kStageBufBytes, &p.rows_out, 0, m.a + plane * m.m_lo + (col0 / 64 + c) * m.mp + row0, acc.staged);
  }
  __device__ __forceinline__ bool prefetch(const Ticket &o, int cta, const Accumulator &acc, long long limit) {
    if (lifted) first_lift = p.ws.norm[o.k()].lift;
    if (o.phase() != kOrthPoly) return true;
    const bool ok = __all_sync(0xffffffffu, ready(o, limit)) && buffers(acc);
    if (ok) stage_square(o, p.tab.m[o.k()], cta, acc, 0);
    return ok;
  }
  __device__ __forceinline__ int lift(int step) const { return max(0, first_lift - p.step[step].fall); }
  // (e <= 0; below 2^-126 taken for that)
  static __device__ __forceinline__ float power_of_two(int e) { return __int_as_float((max(e, -126) + 127) << 23); }
  __device__ __forceinline__ bool epilogue(const Ticket &o, int cta, const Accumulator &acc, float (&v)[kN / 2]) {
    const OrthMatrix &m = p.tab.m[o.k()];
    const int row0 = o.row0() + cta * 128 + acc.warp * 32, col0 = o.col0() + acc.half * (kN / 2);
    return o.phase() == kOrthApply ? put_x(o, m, row0, col0, acc, v) : put_square(o, m, cta, row0, col0, acc, v);
  }
  __device__ __forceinline__ bool put_x(const Ticket &o, const OrthMatrix &m, int row0, int col0, const Accumulator &acc, float (&v)[kN / 2]) {
    constexpr int kCols = kN / 2;
    float f = (o.step() == 0 ? p.ws.norm[o.k()].factor : 1.f) * p.step[o.step()].apply * (last(o) ? m.scale : 1.f);
    const int down = lift(o.step()) - (last(o) ? 0 : lift(o.step() + 1));
    f = f * power_of_two(-(down / 2)) * power_of_two(down / 2 - down);
#pragma unroll
    for (int j = 0; j < kCols; ++j) v[j] *= f;
    if (last(o)) {
      if (!buffers(acc)) return false;
      const int rows = min(32, m.rows - row0);
      const int64_t at = row0 * m.out_pitch + col0;
      if (m.out_dtype == FOPD_F32) {
#pragma unroll
        for (int c = 0; c < kCols; c += 32)
          put_rows_out<FOPD_F32>(acc.staging, acc.lane, v + c, static_cast<float *>(m.out) + at + c, m.out_pitch, rows,
                                 min(32, m.cols - col0 - c), false);
      } else {
#pragma unroll
        for (int c = 0; c < kCols; c += 64)
          put_rows_out<FOPD_BF16>(acc.staging, acc.lane, v + c, static_cast<__nv_bfloat16 *>(m.out) + at + c, m.out_pitch, rows,
                                  min(64, m.cols - col0 - c), false);
      }
      return true;
    }
    return put(o, acc, v, row0 >= m.rp ? 0 : max(0, (m.cp - col0) / 64), m.x[(o.step() + 1) & 1] + col0 / 64 * m.rp + row0, m.rp,
               m.two_planes >> (o.step() + 1) & 1, m.x_lo);
  }
  __device__ __forceinline__ bool put_square(const Ticket &o, const OrthMatrix &m, int cta, int row0, int col0, const Accumulator &acc,
                                             float (&v)[kN / 2]) {
    constexpr int kCols = kN / 2;
    const OrthStep &step = p.step[o.step()];
    const int panels = square_panels(m, row0, col0);
    float f = step.poly_c, poly_b = step.poly_b;
    if (o.phase() == kOrthGram) {
      const float s = o.step() == 0 ? p.ws.norm[o.k()].factor : 1.f;
      f = step.gram * s * s;
    } else {
      f *= power_of_two(-4 * lift(o.step()));
      poly_b *= power_of_two(-2 * lift(o.step()));
    }
#pragma unroll
    for (int j = 0; j < kCols; ++j) v[j] *= f;
    if (o.phase() == kOrthPoly && panels > 0) {
      for (int plane = 0; plane < (m.square() ? 2 : 1); ++plane) {
        if (plane) {
          __syncwarp();  // (the first plane has been read by all lanes)
          stage_square(o, m, cta, acc, 1);
        }
        const bool here = mbar_wait_bounded(acc.staged, staged_turn, kLongWaitCycles);
        if (!__all_sync(0xffffffffu, here)) return false;
        staged_turn ^= 1;
#pragma unroll
        for (int c = 0; c < kCols; c += 64) {
          if (c / 64 >= panels) continue;
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const uint4 w = lds_vector(acc.staging + (c / 64) * kStageBufBytes + acc.lane * 128 + ((j ^ (acc.lane & 7)) * 16));
            const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const float2 a = __half22float2(*reinterpret_cast<const __half2 *>(&u[e]));
              v[c + 8 * j + 2 * e] = fmaf(poly_b, a.x, v[c + 8 * j + 2 * e]);
              v[c + 8 * j + 2 * e + 1] = fmaf(poly_b, a.y, v[c + 8 * j + 2 * e + 1]);
            }
          }
        }
      }
      __syncwarp();  // (before the buffers are written again)
      const int d = row0 + acc.lane - col0;
      if (d >= 0 && d < kCols) {
#pragma unroll
        for (int j = 0; j < kCols; ++j) v[j] += j == d ? step.poly_a : 0.f;
      }
    }
    return put(o, acc, v, panels, (o.phase() == kOrthGram ? m.a : m.p) + col0 / 64 * m.mp + row0, m.mp, m.square(), m.m_lo);
  }
};

}  // namespace fopd
