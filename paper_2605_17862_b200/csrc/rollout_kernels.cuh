// Drawing tokens from rows of logits and verifying drafted tokens (fopd_draw_tokens,
// fopd_verify_draft).
//
// Which token comes out has to be that of exact arithmetic, and a running sum over 150,000
// probabilities in fp32 is off by more than many of them.  Evaluating every exponential in fp64 is
// not an option either (the fp64 pipe takes 5 logits per cycle and SM, memory brings 12).  So the
// sweeps run in fp32 with a bound on their error, and a decision that lies within it is made again in
// fp64: a few per cent of the draws.
//
// A row is cut into parts of 128 16-byte vectors, four for each lane of a warp, and a few parts make a
// slot; a cluster of C CTAs shares a row (or a pair of rows), C such that few rows still fill the GPU.
// A search goes over the CTAs' sums, the owner's slot sums and the elements of one slot.
#pragma once

#include <cooperative_groups.h>

#include "common.cuh"

namespace fopd {

namespace cg = cooperative_groups;

constexpr int kRollThreads = 256;
constexpr int kRollWarps = kRollThreads / 32;
constexpr int kLoadVecs = 4;        // 16-byte vectors of a part per lane of a warp, in flight together
constexpr int kPartVecs = 32 * kLoadVecs;
constexpr int kStages = 2;          // parts of a warp on their way to shared memory
constexpr int kSlots = 256;         // slots per CTA
constexpr int kRollMaxCluster = 8;
constexpr int kDrawList = 4;        // CTAs that share a row in the second launch of a draw: clusters of four pack onto the SMs,
constexpr int kFinishList = 8;      // of eight they leave some empty; but a finish has three passes to make one after another
constexpr int kRollResident = 592;  // CTAs of these kernels that 148 SMs hold at once (64 registers),
constexpr int kRollWhole = 296;     // and of those with the fp64 part in them (128 registers)

enum DraftKind { kDraftNone = 0, kDraftCertain = 1, kDraftRows = 2, kDraftBest = 3 };
enum PosState { kAccept = 0, kReject = 1, kOpen = 2, kBadRow = 3, kBadUniform = 4, kEnd = 5, kBadToken = 6 };

// What a sweep of one row leaves: its maximum, the sum of exponentials behind it, or the index of the best.
struct RowSum {
  float m;
  int32_t best;
  double z;
};

struct Position {
  RowSum t, q;  // the target's row and the draft's
  float lp;     // log p of the drafted token
  int32_t state;
};

// Rows (sequences) to be decided in fp64 by a later launch.
struct LaterEntry {
  int32_t unit;
  float m;   // the row's sum and number (draws)
  double z, v;
};
constexpr int32_t kUnset = 0x7f7f7f7f;  // what one memset leaves in all counters of a call
__device__ __forceinline__ int32_t since_unset(int32_t x) { return (int32_t)((uint32_t)x - (uint32_t)kUnset); }
struct Later {
  int32_t count, pad[7];  // count starts at kUnset
  LaterEntry e[1];  // as many as there are rows
};
// What a launch of a draw or of a finish does: everything; the fp32 part, putting off what it does not decide; the fp64
// part of what was put off.
enum Mode { kWhole = 0, kFirst = 1, kSecond = 2 };

struct RolloutDev {
  const char *target, *draft;
  const int32_t *drafted, *n_draft;
  const double *uniform;
  int64_t vocab, n_parts;
  int64_t tseq, trow, dseq, drow;  // bytes
  int32_t B, K;
  int kind;            // DraftKind
  int span;            // parts per slot
  float ct, cd;        // log2(e) / temperature in fp32
  double ct64, cd64;
  double eps;          // relative error of a row's fp32 sum (and of a weight)
  Position *pos;       // [B, K + 1]
  Later *later;        // kFirst, kSecond
  int32_t *stop;       // [B] the lowest position known not to be accepted, or NULL: nobody looks
  int32_t *next;       // [B] kUnset + the next position to sweep, or NULL: the grid has a cluster for each
  int32_t *tokens;
  float *logprob;
  uint8_t *mask;
  int32_t *n_accepted;
  int32_t *status;
};

template <int DT>
constexpr int kPartElems = kPartVecs *Elem<DT>::kPerVec;

__device__ __forceinline__ float warp_max(float x) {
  float r;
  asm volatile("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(x));
  return r;
}
__device__ __forceinline__ double warp_sum(double x) {
#pragma unroll
  for (int off = 16; off > 0; off >>= 1) x += __shfl_xor_sync(0xffffffffu, x, off);
  return x;
}
__device__ __forceinline__ double warp_scan(double x) {  // inclusive
#pragma unroll
  for (int off = 1; off < 32; off <<= 1) {
    const double y = __shfl_up_sync(0xffffffffu, x, off);
    if ((threadIdx.x & 31) >= off) x += y;
  }
  return x;
}
// 1 / T from log2(e) / T
__device__ __forceinline__ double inv_temperature(double c) { return 0.69314718055994530942 * c; }

// ---- loads ------------------------------------------------------------------------------------------

__device__ __forceinline__ uint4 ld_row(const void *p) {
  uint4 v;
  asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];"
               : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w)
               : "l"(p));
  return v;
}

// Vector i of a row; what lies behind the vocabulary reads as -infinity.
template <int DT>
__device__ __forceinline__ uint4 row_vec(const char *row, int64_t i, int64_t V) {
  using E = Elem<DT>;
  constexpr int P = E::kPerVec;
  const int64_t left = V - i * P;
  if (left >= P) return ld_row(reinterpret_cast<const uint4 *>(row) + i);
  float x[P];
#pragma unroll
  for (int k = 0; k < P; ++k) x[k] = k < left ? E::load1(row, i * P + k) : -INFINITY;
  return E::pack(x);
}

// Asynchronous copies of n times 32 vectors of a row, from vector i0 on, to where the lane that asks for them will read
// them.
template <int DT, int N>
__device__ __forceinline__ void copy_vecs(uint4 *to, const char *row, int64_t i0, int64_t V) {
  const int lane = threadIdx.x & 31;
  if ((i0 + 32 * N) * Elem<DT>::kPerVec <= V) {
    const uint4 *p = reinterpret_cast<const uint4 *>(row) + i0 + lane;
    const uint32_t at = (uint32_t)__cvta_generic_to_shared(to + lane);
#pragma unroll
    for (int v = 0; v < N; ++v)
      asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(at + v * 512), "l"(p + v * 32) : "memory");
  } else {
#pragma unroll
    for (int v = 0; v < N; ++v) to[v * 32 + lane] = row_vec<DT>(row, i0 + v * 32 + lane, V);
  }
}
__device__ __forceinline__ void copies_asked() { asm volatile("cp.async.commit_group;" ::: "memory"); }
__device__ __forceinline__ void oldest_copy() { asm volatile("cp.async.wait_group %0;" ::"n"(kStages - 1) : "memory"); }

// ---- 2^y in fp64 ------------------------------------------------------------------------------------

// For every element of a row that is decided in fp64: y rounded to sixteenths, 2^{j/16} from a table in shared memory
// (sixteen entries lie in sixteen banks) and 1 + f g(f), g the Chebyshev fit of degree four to (2^f - 1) / f on
// |f| <= 1/32: error 1e-14, and exactly 1 for the maximum, so that even rows are summed without rounding.  The high word
// of the table's entry j is less by j << 16, so that adding n << 16 for y = n / 16 makes it 2^{n/16}.
//
// A weight whose y rounds to below -900 is exactly 0 (n = -1023 * 16 takes entry 0 and leaves no bit of it).  The cut is
// made here, at the element, and nowhere else: all levels of a search (CTAs, runs of slots, slots, vectors, elements) ask
// for a sum above 0, and since what is added up is 0 or above 2^-1000, where nothing underflows, a sum above 0 has a part
// above 0.  A cut applied to the sums would find regions that pass it without an element that does.  (92 -> 94 us for 64
// verifications with a row in fp64; setting the power or the polynomial to zero instead: 99, 106.)
constexpr int kCutSixteenths = -900 * 16;
__constant__ double kSixteenths[16] = {
    1.0, 1.0442737824274138, 1.0905077326652577, 1.1387886347566916, 1.189207115002721, 1.241857812073484,
    1.2968395546510096, 1.3542555469368927, 1.4142135623730951, 1.4768261459394993, 1.5422108254079407,
    1.6104903319492543, 1.681792830507429, 1.7562521603732995, 1.8340080864093424, 1.9152065613971474};
__device__ __forceinline__ void fill_exp64(double *tab) {
  if (threadIdx.x < 16) {
    const double x = kSixteenths[threadIdx.x];
    tab[threadIdx.x] = __hiloint2double(__double2hiint(x) - ((int)threadIdx.x << 16), __double2loint(x));
  }
}
// A weight is the product of the two; x is the element, m its row's maximum.  The difference is cut off at about -1000 / c
// (`least`: the high word of that; of two negative numbers the larger word is the lower one), beyond the weights' cut.
struct Weight64 {
  double p, scale;
};
__device__ __forceinline__ Weight64 weight64(float x, double m, double c, uint32_t least, const double *tab) {
  constexpr double kRound = 6755399441055744.0 / 16;  // 1.5 * 2^52 / 16: adding it rounds to sixteenths
  const double e0 = (double)x - m;
  const double d = __hiloint2double((int)min((uint32_t)__double2hiint(e0), least), __double2loint(e0));
  const double t = fma(d, c, kRound);
  const double f = fma(d, c, kRound - t);
  const int sixteenths = __double2loint(t), n = sixteenths < kCutSixteenths ? -1023 * 16 : sixteenths;
  double p = 0.0013333744338239965;
  p = fma(p, f, 0.009618317140580765);
  p = fma(p, f, 0.05550410866027587);
  p = fma(p, f, 0.24022650691319414);
  p = fma(p, f, 0.6931471805599453);
  p = fma(p, f, 1.0);
  const double e = tab[n & 15];
  return {p, __hiloint2double(__double2hiint(e) + (n << 16), __double2loint(e))};
}
__device__ __forceinline__ uint32_t least_of(double c) { return (uint32_t)__double2hiint(-1000.0 / c); }

// The same without a table, for a value here and there: y rounded to a whole number, eleven terms, |f| <= 1/2: 1e-14.
__device__ __forceinline__ double exp64(double d, double c) {
  constexpr double kRound = 6755399441055744.0;  // 1.5 * 2^52
  const double t = fma(d, c, kRound);
  const double f = fma(d, c, kRound - t);
  double p = 4.4455382718708116e-10;
  p = fma(p, f, 7.054911620801123e-9);
  p = fma(p, f, 1.01780860092397e-7);
  p = fma(p, f, 1.321548679014431e-6);
  p = fma(p, f, 1.5252733804059841e-5);
  p = fma(p, f, 1.540353039338161e-4);
  p = fma(p, f, 1.3333558146428443e-3);
  p = fma(p, f, 9.618129107628477e-3);
  p = fma(p, f, 5.550410866482158e-2);
  p = fma(p, f, 2.4022650695910072e-1);
  p = fma(p, f, 6.931471805599453e-1);
  p = fma(p, f, 1.0);
  p = __hiloint2double(__double2hiint(p) + (__double2loint(t) << 20), __double2loint(p));
  return d * c >= -1000.0 ? p : 0.0;  // (not a number counts as nothing: the sum it belongs to tells)
}
// ---- sweeps -----------------------------------------------------------------------------------------

// Two fp32 in one register pair: one instruction works on both.
using f32x2 = unsigned long long;
__device__ __forceinline__ f32x2 pair(float lo, float hi) {
  f32x2 r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
  return r;
}
__device__ __forceinline__ void split(f32x2 x, float &lo, float &hi) {
  asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(x));
}
__device__ __forceinline__ f32x2 add2(f32x2 a, f32x2 b) {
  f32x2 r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ f32x2 mul2(f32x2 a, f32x2 b) {
  f32x2 r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ f32x2 fma2(f32x2 a, f32x2 b, f32x2 c) {
  f32x2 r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
__device__ __forceinline__ f32x2 exp2_2(f32x2 y) {
  float lo, hi;
  split(y, lo, hi);
  return pair(ex2(lo), ex2(hi));
}
// Element pairs of a vector.
template <int DT>
__device__ __forceinline__ void unpack2(const uint4 &v, f32x2 (&x)[Elem<DT>::kPerVec / 2]) {
  float f[Elem<DT>::kPerVec];
  Elem<DT>::unpack(v, f);
#pragma unroll
  for (int k = 0; k < Elem<DT>::kPerVec / 2; ++k) x[k] = pair(f[2 * k], f[2 * k + 1]);
}
template <int N>
__device__ __forceinline__ f32x2 tree_sum2(f32x2 (&x)[N]) {
#pragma unroll
  for (int n = N / 2; n > 0; n >>= 1)
#pragma unroll
    for (int k = 0; k < n; ++k) x[k] = add2(x[k], x[k + n]);
  return x[0];
}
__device__ __forceinline__ float both(f32x2 x) {
  float lo, hi;
  split(x, lo, hi);
  return lo + hi;
}

// Largest element of some vectors, without unpacking bf16.
__device__ __forceinline__ uint32_t max_bf16x2(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("max.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
template <int DT, int N>
__device__ __forceinline__ float max_vecs(const uint4 (&raw)[N]) {
  if (DT == FOPD_BF16) {
    uint32_t m = 0xff80ff80u;
#pragma unroll
    for (int v = 0; v < N; ++v)
      m = max_bf16x2(m, max_bf16x2(max_bf16x2(raw[v].x, raw[v].y), max_bf16x2(raw[v].z, raw[v].w)));
    return fmaxf(__uint_as_float(m << 16), __uint_as_float(m & 0xffff0000u));
  }
  float m = -INFINITY;
#pragma unroll
  for (int v = 0; v < N; ++v)
    m = max3(max3(m, __uint_as_float(raw[v].x), __uint_as_float(raw[v].y)), __uint_as_float(raw[v].z), __uint_as_float(raw[v].w));
  return m;
}

__device__ __forceinline__ RowSum nothing() { return {-INFINITY, INT32_MAX, 0.0}; }

// Rows whose max c is beyond this: its rounding in fp32 is no longer small (or max is infinite: NaN).  Out of line:
// hardly any row comes here.
constexpr float kFar = 1 << 20;
template <int DT>
__device__ __noinline__ double far_sum(uint4 raw, float m, float c) {
  double z = 0.0;
  float x[Elem<DT>::kPerVec];
  Elem<DT>::unpack(raw, x);
#pragma unroll
  for (int k = 0; k < Elem<DT>::kPerVec; ++k) z += (double)ex2((x[k] - m) * c);
  return z;
}

// A sum of weights 2^{x c - mc}, mc = fl(m c), with what fl() took away put back (tiny unless the logits are far from zero).
__device__ __forceinline__ double put_back(float s, float m, float c, float mc) {
  const float took = m == -INFINITY ? 0.f : fmaf(m, c, -mc);
  return fabsf(took) < 1.2e-4f ? (double)fmaf(-took * kLn2, s, s) : (double)s * exp64(-(double)took, 1.0);
}

// A lane's sum of 2^{(x - m) c} over its vectors of a part.  The exponent is x c - fl(m c) in one fused multiply-add; what
// fl() took away is the same for all elements and put back at the end.
template <int DT>
__device__ __forceinline__ double lane_sum(const uint4 (&raw)[kLoadVecs], float m, float c) {
  constexpr int P = Elem<DT>::kPerVec;
  const float mc = m == -INFINITY ? 0.f : m * c;
  if (fabsf(mc) <= kFar) {
    const f32x2 c2 = pair(c, c), mc2 = pair(-mc, -mc);
    f32x2 sums[kLoadVecs];
#pragma unroll
    for (int v = 0; v < kLoadVecs; ++v) {
      f32x2 x[P / 2];
      unpack2<DT>(raw[v], x);
#pragma unroll
      for (int k = 0; k < P / 2; ++k) x[k] = exp2_2(fma2(x[k], c2, mc2));
      sums[v] = tree_sum2<P / 2>(x);
    }
    return put_back(both(tree_sum2<kLoadVecs>(sums)), m, c, mc);
  }
  double z = 0.0;
#pragma unroll
  for (int v = 0; v < kLoadVecs; ++v) z += far_sum<DT>(raw[v], m, c);
  return z;
}

// Sums of a row, part after part: {max, sum 2^{(x - max) c}} with the maximum the warp's and the sum the lane's own.
// -infinity everywhere gives {-inf, 0}; a NaN or +inf makes the sum NaN.
template <int DT>
__device__ __forceinline__ void add_part(RowSum &acc, const uint4 (&raw)[kLoadVecs], float c, double c64) {
  const float m = warp_max(max_vecs<DT>(raw));
  if (m > acc.m) {
    if (acc.m != -INFINITY) acc.z *= exp64((double)acc.m - m, c64);
    acc.m = m;
  }
  acc.z += lane_sum<DT>(raw, acc.m, c);
}

__device__ __forceinline__ float max_nan(float a, float b) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}

// {max, lowest index of it} so far, in every lane; a NaN anywhere gives NaN.
template <int DT>
__device__ __forceinline__ void add_best(RowSum &acc, const uint4 (&raw)[kLoadVecs], int64_t part) {
  using E = Elem<DT>;
  constexpr int P = E::kPerVec;
  float m = -INFINITY;
#pragma unroll
  for (int v = 0; v < kLoadVecs; ++v) {
    float x[P];
    E::unpack(raw[v], x);
#pragma unroll
    for (int k = 0; k < P; ++k) m = max_nan(m, x[k]);
  }
  if (__any_sync(0xffffffffu, isnan(m))) {
    acc.m = NAN;
    return;
  }
  const float top = warp_max(m);
  if (!(top > acc.m)) return;  // (earlier parts hold lower indices; a NaN stays)
  int32_t at = INT32_MAX;
  if (m == top) {
#pragma unroll
    for (int v = kLoadVecs - 1; v >= 0; --v) {
      float x[P];
      E::unpack(raw[v], x);
#pragma unroll
      for (int k = P - 1; k >= 0; --k)
        if (x[k] == top) at = (int32_t)((part * kPartVecs + v * 32 + (threadIdx.x & 31)) * P + k);
    }
  }
  acc.best = (int32_t)__reduce_min_sync(0xffffffffu, at);
  acc.m = top;
}

// A warp's sweep over the slots first, first + step, ... below end of a row, `parts` parts each.  The next kStages parts
// are on their way to the warp's corner of shared memory while one is worked on: with registers as their landing place
// an SM had 64 KB in flight, which was not enough (4.9 TB/s).  flush(slot, acc) closes a slot.
template <int DT, bool kBest, class Flush>
__device__ __forceinline__ void sweep(RowSum &acc, const char *row, int64_t V, int64_t first, int64_t end, int64_t step,
                                      int parts, float c, double c64, uint4 *ring, Flush flush) {
  if (first >= end) return;
  const int lane = threadIdx.x & 31;
  int64_t ahead = first;  // the next part to ask for: slot and part in it
  int ahead_p = 0;
#pragma unroll
  for (int k = 0; k < kStages; ++k) {
    if (ahead < end) copy_vecs<DT, kLoadVecs>(ring + k * kPartVecs, row, (ahead * parts + ahead_p) * kPartVecs, V);
    copies_asked();
    if (++ahead_p == parts) {
      ahead_p = 0;
      ahead += step;
    }
  }
  uint4 *stage = ring;
  for (int64_t slot = first; slot < end; slot += step) {
#pragma unroll 1
    for (int p = 0; p < parts; ++p) {
      oldest_copy();
      uint4 raw[kLoadVecs];
#pragma unroll
      for (int v = 0; v < kLoadVecs; ++v) raw[v] = stage[v * 32 + lane];
      if (ahead < end) copy_vecs<DT, kLoadVecs>(stage, row, (ahead * parts + ahead_p) * kPartVecs, V);
      copies_asked();
      if (++ahead_p == parts) {
        ahead_p = 0;
        ahead += step;
      }
      stage = stage + kPartVecs == ring + kStages * kPartVecs ? ring : stage + kPartVecs;
      if (kBest) add_best<DT>(acc, raw, slot * parts + p);
      else add_part<DT>(acc, raw, c, c64);
    }
    flush(slot, acc);
  }
}

// The lanes' parts of a row as one, in every lane (2^y in fp64: its error stays out of the bound).
__device__ __forceinline__ double part_of(const RowSum &a, float m, double c) {
  return a.m == m ? a.z : a.z * exp64((double)a.m - m, c);
}
__device__ __forceinline__ RowSum warp_merge(const RowSum &a, double c) {
  const float m = warp_max(a.m);
  return {m, 0, warp_sum(part_of(a, m, c))};
}
__device__ __forceinline__ RowSum warp_merge_best(RowSum a) {
#pragma unroll
  for (int off = 16; off > 0; off >>= 1) {
    const float m = __shfl_xor_sync(0xffffffffu, a.m, off);
    const int32_t at = __shfl_xor_sync(0xffffffffu, a.best, off);
    const bool keep = isnan(a.m) || (!isnan(m) && (a.m > m || (a.m == m && a.best <= at)));
    if (!keep) {
      a.m = m;
      a.best = at;
    }
  }
  return a;
}

// (a sum is 0 or above 2^-1000, and compared with that rather than 0: 8.3 against 8.8 us for a row, 21 against 22.5 us for
// four drafts)
__device__ __forceinline__ bool is_distribution(const RowSum &r) {
  return r.m > -INFINITY && r.m < INFINITY && r.z > 0x1p-1000 && r.z < INFINITY;
}

// ---- weights ----------------------------------------------------------------------------------------

// Weights of the distribution a token is drawn from, a vector of elements at a time: e^{t} of the target's row, without
// one element (`without` >= 0), or max(p - q, 0) (`rest`).
template <int DT>
struct Weights {
  static constexpr int P = Elem<DT>::kPerVec;
  const char *t, *q;  // rows
  int64_t V;
  bool rest;
  int32_t without;
  RowSum ts, qs;
  float ct, cd;
  double ct64, cd64;
  const double *tab;
  // derived
  float mct, mcd, a, b;  // fl(max c); 2^{what fl() took} / sum
  uint32_t least_t, least_q;
  double ia, ib;         // 1 / sum

  __device__ __forceinline__ void derive() {
    mct = ts.m * ct;
    least_t = least_of(ct64);
    if (rest) {
      a = (float)(exp64(-(double)fmaf(ts.m, ct, -mct), 1.0) / ts.z);
      ia = 1.0 / ts.z;
      mcd = qs.m * cd;
      b = (float)(exp64(-(double)fmaf(qs.m, cd, -mcd), 1.0) / qs.z);
      least_q = least_of(cd64);
      ib = 1.0 / qs.z;
    }
  }
  // fp32's exponent cannot be formed (see add_part)
  __device__ __forceinline__ bool beyond() const { return !(fabsf(mct) <= kFar) || (rest && !(fabsf(mcd) <= kFar)); }

  __device__ __forceinline__ void take_away(int64_t i, uint4 &rt) const {  // a logit becomes -infinity
    if (without >= 0 && without / P == i) {
      float x[P];
      Elem<DT>::unpack(rt, x);
#pragma unroll
      for (int k = 0; k < P; ++k) x[k] = k == without % P ? -INFINITY : x[k];
      rt = Elem<DT>::pack(x);
    }
  }
  template <bool kRest>
  __device__ __forceinline__ double fast_sum(const uint4 &rt, const uint4 &rq) const {
    f32x2 w[P / 2];
    const f32x2 c2 = pair(ct, ct), m2 = pair(-mct, -mct);
    unpack2<DT>(rt, w);
#pragma unroll
    for (int k = 0; k < P / 2; ++k) w[k] = exp2_2(fma2(w[k], c2, m2));
    if (kRest) {
      const f32x2 d2 = pair(cd, cd), n2 = pair(-mcd, -mcd), a2 = pair(a, a), b2 = pair(-b, -b);
      f32x2 x[P / 2];
      unpack2<DT>(rq, x);
#pragma unroll
      for (int k = 0; k < P / 2; ++k) {
        float lo, hi;
        split(fma2(w[k], a2, mul2(exp2_2(fma2(x[k], d2, n2)), b2)), lo, hi);
        w[k] = pair(fmaxf(lo, 0.f), fmaxf(hi, 0.f));
      }
    }
    return (double)both(tree_sum2<P / 2>(w));
  }
  // (both products are rounded alike: equal rows leave exactly nothing)
  __device__ __forceinline__ double difference(const Weight64 &p, const Weight64 &r) const {
    const double d = __dsub_rn(__dmul_rn(__dmul_rn(p.p, p.scale), ia), __dmul_rn(__dmul_rn(r.p, r.scale), ib));
    const int keep = ~(__double2hiint(d) >> 31);
    return __hiloint2double(__double2hiint(d) & keep, __double2loint(d) & keep);
  }
  template <bool kRest>
  __device__ __forceinline__ double exact_sum(const uint4 &rt, const uint4 &rq) const {
    float x[P], y[P];
    Elem<DT>::unpack(rt, x);
    if (kRest) Elem<DT>::unpack(rq, y);
    double s = 0.0;
#pragma unroll
    for (int k = 0; k < P; ++k) {
      const Weight64 p = weight64(x[k], ts.m, ct64, least_t, tab);
      if (kRest) s += difference(p, weight64(y[k], qs.m, cd64, least_q, tab));
      else s = fma(p.p, p.scale, s);
    }
    return s;
  }
  template <bool kExact, bool kRest>
  __device__ __forceinline__ double sum(const uint4 &rt, const uint4 &rq) const {
    return kExact ? exact_sum<kRest>(rt, rq) : fast_sum<kRest>(rt, rq);
  }
  // one element's weight from its logits, in fp64 or in fp32
  template <bool kExact>
  __device__ __forceinline__ double element(float x, float y) const {
    if (kExact) {
      const Weight64 p = weight64(x, ts.m, ct64, least_t, tab);
      return rest ? difference(p, weight64(y, qs.m, cd64, least_q, tab)) : p.p * p.scale;
    }
    const float p = ex2(fmaf(x, ct, -mct));
    return rest ? (double)fmaxf(fmaf(p, a, -b * ex2(fmaf(y, cd, -mcd))), 0.f) : (double)p;
  }
};

// ---- a CTA's and a cluster's tools ------------------------------------------------------------------

__device__ __forceinline__ void roll_sync(cg::cluster_group &cl) {
  if (cl.num_blocks() > 1) cl.sync();
  else __syncthreads();
}

// A CTA's shared memory may be written by another one once it runs: each says so as it starts, and all wait for the
// others before the first such write, where that is hidden behind loads (starting late costs nothing then).
__device__ __forceinline__ void say_started(cg::cluster_group &cl) {
  if (cl.num_blocks() > 1) asm volatile("barrier.cluster.arrive.relaxed;" ::: "memory");
}
__device__ __forceinline__ void all_started(cg::cluster_group &cl) {
  if (cl.num_blocks() > 1) asm volatile("barrier.cluster.wait.acquire;" ::: "memory");
}

struct ExactSums {
  double t, q;  // of a target's row and of a draft's
};

// CTAs of a cluster write into one another's shared memory before a barrier of the cluster and read their own behind
// it; so a CTA may leave when it has passed its last barrier.
struct RollShared {
  uint4 ring[kRollWarps][kStages * kPartVecs];
  double tz[kSlots];  // slot sums of this CTA, relative to 2^{tm c} where they come from the sweep
  float tm[kSlots];
  double scan[kRollWarps];
  double tab[16];
  RowSum part[2][kRollWarps];
  RowSum pub[2][kRollMaxCluster];  // the CTAs' totals, by parity of the exchange
  ExactSums sums[2][kRollMaxCluster * kRollWarps];  // the warps' exact sums, by parity
  RowSum total;
  double before, goal;
  int64_t slot;
  uint4 found[2];  // the vectors that hold the element found, and its logit
  float logit;
  int32_t owner, result, thread, unsure, stop, take[2];
};

// This CTA's slots of a row: [lo, hi) of ceil(n_parts / span), contiguous and in rank order.
struct Slots {
  int64_t lo, hi;
};
__device__ __forceinline__ Slots my_slots(const RolloutDev &d, int rank, int size) {
  const int64_t n = (d.n_parts + d.span - 1) / d.span, per = (n + size - 1) / size;
  const int64_t lo = rank * per, hi = lo + per;
  return {lo < n ? lo : n, hi < n ? hi : n};
}

// Inclusive scan over the CTA's threads; the warps' sums stay in scan[] until the next call.
__device__ __forceinline__ double cta_scan(double x, double *scan) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  x = warp_scan(x);
  __syncthreads();
  if (lane == 31) scan[warp] = x;
  __syncthreads();
  double before = 0.0;
#pragma unroll
  for (int w = 0; w < kRollWarps; ++w)
    if (w < warp) before += scan[w];
  return before + x;
}

constexpr int32_t kUnsure = -2;  // within the bound, or another CTA's

// The element of slot `slot` whose running sum (starting at `before`) passes `goal`; where rounding leaves none, the
// last one with a weight.  Same result in every thread; its logit is left in sh.logit.
template <int DT, bool kExact>
__device__ int32_t cta_find(const Weights<DT> &w, const RolloutDev &d, int64_t slot, double before, double goal,
                            double bound, RollShared &sh) {
  constexpr int P = Weights<DT>::P;
  if (threadIdx.x == 0) sh.result = kUnsure;
  const int64_t vec0 = slot * d.span * kPartVecs, vecs = min((int64_t)d.span, d.n_parts - slot * d.span) * kPartVecs;
  const int64_t rounds = (vecs + kRollThreads - 1) / kRollThreads;  // a vector for each thread
  int64_t last = 0;  // the last round with a weight, and the running sum before it
  double last_before = before;
  for (int64_t s = 0; s <= rounds; ++s) {
    const bool back = s == rounds;  // no round passes: the last weight it is
    const int64_t o = (back ? last : s) * kRollThreads + threadIdx.x, i = vec0 + o;
    if (back) before = last_before;
    double sum = 0.0;
    uint4 rt, rq;
    if (o < vecs) {
      rt = row_vec<DT>(w.t, i, d.vocab);
      w.take_away(i, rt);
      if (w.rest) {
        rq = row_vec<DT>(w.q, i, d.vocab);
        sum = w.template sum<kExact, true>(rt, rq);
      } else {
        sum = w.template sum<kExact, false>(rt, rq);
      }
    }
    const double incl = before + cta_scan(sum, sh.scan);
    const bool here = sum > 0.0 && (back || incl > goal);
    if (threadIdx.x == 0) sh.thread = back ? -1 : kRollThreads;
    if (!__syncthreads_or(here)) {
      if (__syncthreads_or(sum > 0.0)) {
        last = s;
        last_before = before;
      }
#pragma unroll
      for (int k = 0; k < kRollWarps; ++k) before += sh.scan[k];
      continue;
    }
    if (here && back) atomicMax(&sh.thread, (int)threadIdx.x);
    else if (here) atomicMin(&sh.thread, (int)threadIdx.x);
    __syncthreads();
    if (sh.thread >> 5 == (int)threadIdx.x >> 5) {  // its warp: a lane for each element
      const int lane = threadIdx.x & 31;
      if (sh.thread == (int)threadIdx.x) {
        sh.found[0] = rt;
        sh.found[1] = w.rest ? rq : rt;
      }
      __syncwarp();
      const float logit = lane < P ? Elem<DT>::load1(&sh.found[0], lane) : 0.f;
      const double x = lane < P ? w.template element<kExact>(logit, Elem<DT>::load1(&sh.found[1], lane)) : 0.0;
      const int from = sh.thread & 31;
      const double before_vec = __shfl_sync(0xffffffffu, incl - sum, from), after = before_vec + warp_scan(x);
      const int64_t vec = __shfl_sync(0xffffffffu, i, from);
      const unsigned pass = __ballot_sync(0xffffffffu, x > 0.0 && after > goal),
                     has = __ballot_sync(0xffffffffu, x > 0.0);
      const int at = pass ? __ffs(pass) - 1 : 31 - __clz(has);
      if (lane == at && (kExact || (goal - (after - x) > bound && after - goal > bound))) {
        sh.result = (int32_t)(vec * P + at);
        sh.logit = logit;
      }
    }
    break;
  }
  __syncthreads();
  return sh.result;
}

// Search over the cluster.  On entry this CTA's slots have their sums in sh.tz: relative to 2^{tm c} (kRelative: w then
// gets the row's sum) or all to one reference.  The CTAs exchange their totals; the owner of the goal looks through its
// slots, then through one slot's elements.  Returns the token (-1: none) in the owner's threads, elsewhere kUnsure, the total
// and whether the cluster is to do it again in fp64 in all threads.
template <int DT, bool kExact, bool kRelative>
__device__ __forceinline__ int32_t cluster_search(cg::cluster_group &cl, Weights<DT> &w, const RolloutDev &d, Slots sl, double v,
                                  double bound_rel, double bound_abs, int parity, RollShared &sh, RowSum *total,
                                  bool *again) {
  const int rank = (int)cl.block_rank(), size = (int)cl.num_blocks();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int n = (int)(sl.hi - sl.lo);
  if (warp == 0) {
    // a lane takes a run of slots
    const int per = (n + 31) / 32, lo = min(n, lane * per), hi = min(n, lo + per);
    RowSum own = {0.f, 0, 0.0};
    if (kRelative) {
      own.m = -INFINITY;
      for (int t = lo; t < hi; ++t) own.m = fmaxf(own.m, sh.tm[t]);
      own.m = warp_max(own.m);
    }
    double s = 0.0;
    for (int t = lo; t < hi; ++t) {
      double x = sh.tz[t];
      if (kRelative) sh.tz[t] = x = part_of({sh.tm[t], 0, x}, own.m, d.ct64);
      s += x;
    }
    const double incl = warp_scan(s);
    own.z = __shfl_sync(0xffffffffu, incl, 31);
    RowSum all = own;
    // (rounded down: a sum in fp64 is above that exactly if it is above v times the total)
    double goal = __dmul_rd(v, own.z), before = 0.0, scale = 1.0;
    int owner = 0;
    if (size > 1) {
      if (lane < size) *cl.map_shared_rank(&sh.pub[parity][rank], lane) = own;
      cl.sync();
      const RowSum mine = lane < size ? sh.pub[parity][lane] : nothing();
      all.m = warp_max(mine.m);
      const double part = part_of(mine, all.m, d.ct64), run = warp_scan(part);
      all.z = __shfl_sync(0xffffffffu, run, 31);
      goal = __dmul_rd(v, all.z);
      const unsigned pass = __ballot_sync(0xffffffffu, part > 0.0 && run > goal),
                     has = __ballot_sync(0xffffffffu, part > 0.0);
      owner = pass ? __ffs(pass) - 1 : has ? 31 - __clz(has) : 0;
      before = __shfl_sync(0xffffffffu, run - part, owner);
      scale = part_of({own.m, 0, 1.0}, all.m, d.ct64);
    }
    if (lane == 0) {
      sh.total = all;
      sh.owner = owner;
      sh.goal = goal;
    }
    if (owner == rank && is_distribution(all)) {  // the first run that passes, or the last one with a weight
      const unsigned pass = __ballot_sync(0xffffffffu, s * scale > 0.0 && before + scale * incl > goal),
                     has = __ballot_sync(0xffffffffu, s * scale > 0.0);
      if (lane == (pass ? __ffs(pass) - 1 : has ? 31 - __clz(has) : 0)) {
        double run = before + scale * (incl - s), at = run;
        int slot = lo;
        for (int t = lo; t < hi; ++t) {
          const double x = sh.tz[t] * scale;
          if (x > 0.0) {
            slot = t;
            at = run;
            if (run + x > goal) break;
          }
          run += x;
        }
        sh.slot = sl.lo + slot;
        sh.before = at;
      }
    }
  } else if (size > 1) {
    cl.sync();
  }
  __syncthreads();
  *total = sh.total;
  int32_t token = kUnsure;
  const bool good = is_distribution(*total), mine = good && sh.owner == rank;
  if (mine) {
    const double bound = bound_rel * total->z + bound_abs;
    double scale = 1.0;
    if (kRelative) {  // the slots' sums are free of the rounding of max c; the elements' weights all carry it
      w.ts = *total;
      w.derive();
      scale = exp64((double)fmaf(w.ts.m, w.ct, -w.mct), 1.0);
    }
    if (!kRelative || !w.beyond())
      token = cta_find<DT, kExact>(w, d, sh.slot, sh.before * scale, sh.goal * scale, bound * scale, sh);
    if (kExact && token == kUnsure) token = -1;  // (a positive total has an element: said, should it ever not be so)
  }
  *again = false;
  if (!kExact) {
    if (size == 1) {
      *again = good && token == kUnsure;
    } else {
      if (mine && (int)threadIdx.x < size) *cl.map_shared_rank(&sh.unsure, threadIdx.x) = token == kUnsure;
      cl.sync();
      *again = good && sh.unsure;
    }
  }
  return token;
}

// Slot sums of the weights, relative to one reference.  As in sweep(), the next vectors are on their way meanwhile; a
// stage holds two of the target's and two of the draft's for each lane.
template <int DT, bool kExact, bool kRest>
__device__ __forceinline__ void cta_sums(const Weights<DT> &w, const RolloutDev &d, Slots sl, RollShared &sh) {
  static_assert(kLoadVecs == 4, "two vectors of each row fill a stage");
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, steps = d.span * (kPartVecs / 64);
  uint4 *ring = sh.ring[warp], *stage = ring;
  int64_t ahead = sl.lo + warp;
  int ahead_u = 0;
  const auto ask = [&](uint4 *to) {
    if (ahead < sl.hi) {
      const int64_t i0 = (ahead * steps + ahead_u) * 64;
      copy_vecs<DT, 2>(to, w.t, i0, w.V);
      if (kRest) copy_vecs<DT, 2>(to + 64, w.q, i0, w.V);
    }
    copies_asked();
    if (++ahead_u == steps) {
      ahead_u = 0;
      ahead += kRollWarps;
    }
  };
#pragma unroll
  for (int k = 0; k < kStages; ++k) ask(ring + k * kPartVecs);
  for (int64_t slot = sl.lo + warp; slot < sl.hi; slot += kRollWarps) {
    double s = 0.0;
#pragma unroll 1
    for (int u = 0; u < steps; ++u) {
      oldest_copy();
#pragma unroll(kExact ? 1 : 2)
      for (int v = 0; v < 2; ++v) {
        uint4 rt = stage[v * 32 + lane], rq = rt;
        if (kRest) rq = stage[64 + v * 32 + lane];
        else w.take_away((slot * steps + u) * 64 + v * 32 + lane, rt);
        s += w.template sum<kExact, kRest>(rt, rq);
      }
      ask(stage);
      stage = stage + kPartVecs == ring + kStages * kPartVecs ? ring : stage + kPartVecs;
    }
    s = warp_sum(s);
    if (lane == 0) sh.tz[slot - sl.lo] = s;
  }
  __syncthreads();
}

// The sums of exponentials of a target's row and, with q, of a draft's in fp64, over the cluster, in every thread.
// parity alternates from call to call.
template <int DT, bool kBoth>
__device__ __forceinline__ ExactSums cta_exact_pair(const Weights<DT> &w, const RolloutDev &d, Slots sl, RollShared &sh) {
  constexpr int P = Weights<DT>::P;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  uint4 *ring = sh.ring[warp], *stage = ring;
  const int64_t end = min(sl.hi * d.span, d.n_parts) * (kPartVecs / 64);  // in steps of 64 vectors
  int64_t ahead = sl.lo * d.span * (kPartVecs / 64) + warp;
  const auto ask = [&](uint4 *to) {
    if (ahead < end) {
      copy_vecs<DT, 2>(to, w.t, ahead * 64, w.V);
      if (kBoth) copy_vecs<DT, 2>(to + 64, w.q, ahead * 64, w.V);
    }
    copies_asked();
    ahead += kRollWarps;
  };
#pragma unroll
  for (int k = 0; k < kStages; ++k) ask(ring + k * kPartVecs);
  ExactSums s = {0.0, 0.0};
#pragma unroll 1
  for (int64_t at = sl.lo * d.span * (kPartVecs / 64) + warp; at < end; at += kRollWarps) {
    oldest_copy();
#pragma unroll 1
    for (int v = 0; v < 2; ++v) {
      float x[P], y[P];
      Elem<DT>::unpack(stage[v * 32 + lane], x);
      if (kBoth) Elem<DT>::unpack(stage[64 + v * 32 + lane], y);
#pragma unroll
      for (int k = 0; k < P; ++k) {
        const Weight64 p = weight64(x[k], w.ts.m, w.ct64, w.least_t, w.tab);
        s.t = fma(p.p, p.scale, s.t);
        if (kBoth) {
          const Weight64 r = weight64(y[k], w.qs.m, w.cd64, w.least_q, w.tab);
          s.q = fma(r.p, r.scale, s.q);
        }
      }
    }
    ask(stage);
    stage = stage + kPartVecs == ring + kStages * kPartVecs ? ring : stage + kPartVecs;
  }
  s.t = warp_sum(s.t);
  if (kBoth) s.q = warp_sum(s.q);
  return s;
}
template <int DT>
__device__ __noinline__ ExactSums cluster_exact_sums(cg::cluster_group &cl, const char *trow, float tm, const char *qrow,
                                                     float qm, const RolloutDev &d, Slots sl, int &parity,
                                                     RollShared &sh) {
  Weights<DT> w = {};
  w.t = trow;
  w.q = qrow;
  w.V = d.vocab;
  w.ts = {tm, 0, 1.0};
  w.qs = {qm, 0, 1.0};
  w.ct64 = d.ct64;
  w.cd64 = d.cd64;
  w.least_t = least_of(d.ct64);
  w.least_q = qrow ? least_of(d.cd64) : 0;
  w.tab = sh.tab;
  const ExactSums mine = qrow ? cta_exact_pair<DT, true>(w, d, sl, sh) : cta_exact_pair<DT, false>(w, d, sl, sh);
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, size = (int)cl.num_blocks();
  if (lane < size) cl.map_shared_rank(&sh.sums[parity][0], lane)[cl.block_rank() * kRollWarps + warp] = mine;
  roll_sync(cl);
  ExactSums s = {0.0, 0.0};
  for (int k = lane; k < size * kRollWarps; k += 32) {
    s.t += sh.sums[parity][k].t;
    s.q += sh.sums[parity][k].q;
  }
  parity ^= 1;
  return {warp_sum(s.t), warp_sum(s.q)};
}

// The sum of a row without its largest element `at`, in every lane of a warp.  Beside a weight of 1 the fp32 sum of its
// lane's vectors has lost what the others weigh (2^-24 of the whole); all other sums are free of it and have been added up
// in fp64.  So that lane's sum is formed again, a lane for each of its elements and in the same order (lane_sum's trees),
// taken out of the row's, and put back without the element.  (Out of line: 61.5 us for 64 sequences with drafts, inlined
// 62.5.)
template <int DT>
__device__ __noinline__ double sum_beside(const char *row, int64_t V, int32_t at, const RowSum &r, float c) {
  constexpr int P = Elem<DT>::kPerVec;
  const float mc = r.m * c;
  if (!(fabsf(mc) <= kFar)) return fmax(r.z - 1.0, 0.0);  // (far_sum adds weight by weight in fp64)
  const int e = (threadIdx.x & 31) % (kLoadVecs * P);
  const int64_t vec = at / P, i = (vec / kPartVecs * kPartVecs + vec % 32 + e / P * 32) * P + e % P;
  float with = i < V ? ex2(fmaf(Elem<DT>::load1(row, i), c, -mc)) : 0.f, without = i == at ? 0.f : with;
  const auto add = [&](int off) {
    with += __shfl_xor_sync(0xffffffffu, with, off);
    without += __shfl_xor_sync(0xffffffffu, without, off);
  };
#pragma unroll
  for (int off = P / 2; off > 1; off >>= 1) add(off);
#pragma unroll
  for (int off = kLoadVecs / 2 * P; off >= P; off >>= 1) add(off);
  add(1);
  return fmax(r.z - put_back(with, r.m, c, mc) + put_back(without, r.m, c, mc), 0.0);
}
// log p of element `at` of a row from its logit and the row's sum, by a warp: the difference in fp64, the log's error is
// 1e-6 of it.  Towards p = 1 the row's sum is hardly more than 1 and its log no larger than its error: above 0.8 it comes
// from the rest (about 1 us; below, the sum's error is 1e-6 of the log at most).
template <int DT>
__device__ __forceinline__ float log_prob(const char *row, int64_t V, int32_t at, float logit, const RowSum &r, float c, double c64) {
  if (logit == r.m && r.z < 1.25) return 0.f - log1pf((float)sum_beside<DT>(row, V, at, r, c));
  return (float)(((double)logit - r.m) * inv_temperature(c64) - (double)logf((float)r.z));
}

// ---- draws: a cluster per row -----------------------------------------------------------------------

// With more rows than fit at once a row that fp32 does not decide waits for the second launch, where kDrawList CTAs share
// it: one CTA alone takes tens of microseconds for it in fp64, and a few of those held up the end of the grid (278 us
// against 240 for 4,096 rows of 151,936).
template <int DT, bool kBest, int kMode>
__global__ void __launch_bounds__(kRollThreads, kMode == kFirst ? 4 : 2) draw_kernel(const __grid_constant__ RolloutDev d) {
  __shared__ RollShared sh;
  cg::cluster_group cl = cg::this_cluster();
  const int rank = (int)cl.block_rank(), size = (int)cl.num_blocks();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const Slots sl = my_slots(d, rank, size);
  say_started(cl);
  asm volatile("griddepcontrol.launch_dependents;");
  if (kMode != kFirst) {
    fill_exp64(sh.tab);
    __syncthreads();
  }
  if (kMode == kSecond) {
    all_started(cl);
    asm volatile("griddepcontrol.wait;" ::: "memory");
  }
  const int64_t count = kMode == kSecond ? since_unset(d.later->count) : d.B, step = gridDim.x / size;
  int parity = 0;
  for (int64_t k = blockIdx.x / size; k < count; k += step) {
    const int64_t n = kMode == kSecond ? d.later->e[k].unit : k;
    const char *row = d.target + n * d.tseq;
    const double v = kBest ? 0.0 : kMode == kSecond ? d.later->e[k].v : d.uniform[n];
    RowSum acc = nothing();
    if (kMode != kSecond)
      sweep<DT, kBest>(acc, row, d.vocab, sl.lo + warp, sl.hi, kRollWarps, d.span, d.ct, d.ct64, sh.ring[warp],
                       [&](int64_t slot, RowSum &r) {
                         if (kBest) return;
                         r.z = warp_sum(r.z);
                         if (lane == 0) {
                           sh.tm[slot - sl.lo] = r.m;
                           sh.tz[slot - sl.lo] = r.z;
                         }
                         r = nothing();
                       });
    if (kMode != kSecond) all_started(cl);  // (one row to a cluster)
    int32_t token = kUnsure;
    float lp = 0.f;
    bool good;
    int bits = FOPD_DEV_BAD_LOGITS;
    if (kBest) {
      if (lane == 0) sh.part[0][warp] = acc;
      __syncthreads();
      if (warp == 0) {
        const RowSum r = warp_merge_best(lane < kRollWarps ? sh.part[0][lane] : nothing());
        if (lane < size) *cl.map_shared_rank(&sh.pub[0][rank], lane) = r;
      }
      roll_sync(cl);
      RowSum r = nothing();
      if (warp == 0) r = warp_merge_best(lane < size ? sh.pub[0][lane] : nothing());
      good = r.m > -INFINITY && r.m < INFINITY;  // (warp 0)
      if (rank == 0 && good) token = r.best;
    } else {
      const bool v_ok = v >= 0.0 && v < 1.0;
      Weights<DT> w = {};
      w.t = row;
      w.V = d.vocab;
      w.without = -1;
      w.ct = d.ct;
      w.ct64 = d.ct64;
      w.tab = sh.tab;
      RowSum total;
      bool again = true;
      if (kMode == kSecond) {
        total = {d.later->e[k].m, 0, d.later->e[k].z};
      } else {
        __syncthreads();
        token = cluster_search<DT, false, true>(cl, w, d, sl, v_ok ? v : 0.0, 2 * d.eps, 0.0, parity, sh, &total, &again);
        parity ^= 1;
      }
      good = is_distribution(total) && v_ok;
      if (is_distribution(total)) bits = FOPD_DEV_BAD_UNIFORM;
      if (again && good) {
        if (kMode == kFirst) {
          if (rank == 0 && threadIdx.x == 0) d.later->e[since_unset(atomicAdd(&d.later->count, 1))] = {(int32_t)n, total.m, total.z, v};
          continue;
        }
        w.ts = total;
        w.derive();
        cta_sums<DT, true, false>(w, d, sl, sh);
        RowSum exact_total;
        bool never;
        token = cluster_search<DT, true, false>(cl, w, d, sl, v, 0.0, 0.0, parity, sh, &exact_total, &never);
        parity ^= 1;
      }
      if (good && token >= 0 && warp == 0) lp = log_prob<DT>(row, d.vocab, token, sh.logit, total, d.ct, d.ct64);
    }
    if (threadIdx.x == 0 && (good ? token != kUnsure : rank == 0)) {  // the CTA that has the token, or the first one
      if (!good) token = -1;
      d.tokens[n] = token;
      if (d.logprob) d.logprob[n] = lp;
      if (d.mask) d.mask[n] = token >= 0 ? 1 : 0;
      if (token < 0 && d.status) atomicOr(d.status, good ? FOPD_DEV_BAD_LOGITS : bits);
    }
    if (threadIdx.x == 0 && rank == 0 && d.n_accepted) d.n_accepted[n] = 0;
    if (k + step < count) roll_sync(cl);  // the next row writes what this one has read
  }
}

// ---- verification -----------------------------------------------------------------------------------

__device__ __forceinline__ int32_t drafts_of(const RolloutDev &d, int32_t b) {
  const int32_t n = d.n_draft ? d.n_draft[b] : d.K;
  return n < 0 ? 0 : n > d.K ? d.K : n;
}

// What the decision on a draft needs besides the rows' sums, asked for before the sweep.
struct Draft {
  int32_t x;
  double u;
  float t, q;  // logits
  bool there;
};
template <int DT>
__device__ __forceinline__ Draft draft_of(const RolloutDev &d, int32_t b, int32_t j, int32_t n, const char *trow,
                                          const char *qrow) {
  Draft r = {-1, 0.0, 0.f, 0.f, false};
  if (j < n) {
    r.x = d.drafted[(int64_t)b * d.K + j];
    r.u = d.uniform[(int64_t)b * (d.K + 1) + j];
    r.there = r.x >= 0 && r.x < d.vocab;
    if (r.there) {
      r.t = Elem<DT>::load1(trow, r.x);
      if (d.kind == kDraftRows) r.q = Elem<DT>::load1(qrow, r.x);
    }
  }
  return r;
}
// Decides on one position (a warp, all lanes alike).
template <int DT>
__device__ __forceinline__ void judge(const RolloutDev &d, const Draft &r, const char *trow, bool last, bool target_best, Position &o) {
  o.lp = 0.f;
  o.state = is_distribution(o.t) ? kEnd : kBadRow;
  if (o.state == kBadRow || last) return;
  if (!r.there) {
    o.state = kBadToken;
  } else if (target_best) {
    o.state = r.x == o.t.best ? kAccept : kReject;
  } else if (!(r.u >= 0.0 && r.u < 1.0)) {
    o.state = kBadUniform;
  } else {
    const double p = exp64((double)r.t - o.t.m, d.ct64) / o.t.z;
    double q = 1.0;
    if (d.kind == kDraftRows) q = exp64((double)r.q - o.q.m, d.cd64) / o.q.z;
    else if (d.kind == kDraftBest) q = r.x == o.q.best ? 1.0 : 0.0;
    const double uq = r.u * q;
    o.state = fabs(uq - p) < 4 * d.eps * fmax(uq, p) ? kOpen : uq < p ? kAccept : kReject;
    if (o.state != kReject) o.lp = log_prob<DT>(trow, d.vocab, r.x, r.t, o.t, d.ct, d.ct64);
  }
  if ((d.kind == kDraftRows || d.kind == kDraftBest) && o.state != kBadUniform && !is_distribution(o.q)) o.state = kBadRow;
}

// Whether a position is to be swept: its sequence has it, and no rejection before it is known.  One thread looks for all
// CTAs of the cluster (the value may change between two looks).
__device__ __forceinline__ bool wanted(cg::cluster_group &cl, const RolloutDev &d, int32_t b, int32_t j, RollShared &sh) {
  if (!d.stop || j == 0) return j <= drafts_of(d, b);
  if (cl.block_rank() == 0 && threadIdx.x == 0) {
    const int32_t known = *(volatile const int32_t *)(d.stop + b);
    for (unsigned r = 0; r < cl.num_blocks(); ++r)
      *cl.map_shared_rank(&sh.take[0], r) = j <= drafts_of(d, b) && known >= j;
  }
  roll_sync(cl);
  return sh.take[0];
}

// The next position for a cluster that stays: of the sequence it is at, else of one of the 31 behind it.  {b, j} in
// sh.take; j = -1: nothing is left there, or other clusters have it (one that takes a position comes back to the same
// sequence, so no sequence is left with work and without a cluster).
__device__ __forceinline__ void take_next(cg::cluster_group &cl, const RolloutDev &d, int32_t b, RollShared &sh) {
  if (cl.block_rank() == 0 && threadIdx.x < 32) {
    const int lane = threadIdx.x;
    const int32_t at = (int32_t)(((int64_t)b + lane) % d.B);
    int32_t take_b = b, take_j = -1;
    for (int tries = 0; tries < 4; ++tries) {
      int32_t left = -1;  // the last position that may be wanted
      if (lane < d.B) left = min(drafts_of(d, at), *(volatile const int32_t *)(d.stop + at));
      const bool some = lane < d.B && since_unset(*(volatile const int32_t *)(d.next + at)) <= left;
      const unsigned has = __ballot_sync(0xffffffffu, some);
      if (!has) break;
      const int from = __ffs(has) - 1;
      int32_t j = -1;
      if (lane == from) {
        j = since_unset(atomicAdd(d.next + at, 1));
        if (j > left) j = -1;
      }
      take_j = __shfl_sync(0xffffffffu, j, from);
      take_b = __shfl_sync(0xffffffffu, at, from);
      if (take_j >= 0) break;
    }
    if (lane < (int)cl.num_blocks()) {
      int32_t *to = cl.map_shared_rank(&sh.take[0], lane);
      to[0] = take_b;
      to[1] = take_j;
    }
  }
  roll_sync(cl);
}

// One position: sums of the target's and the draft's row in one stream of parts, and the decision.
template <int DT, bool kBest>
__device__ __forceinline__ void sweep_position(cg::cluster_group &cl, const RolloutDev &d, int32_t b, int32_t j,
                                               RollShared &sh) {
  const int rank = (int)cl.block_rank(), size = (int)cl.num_blocks();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int32_t n = drafts_of(d, b);
  const char *trow = d.target + b * d.tseq + j * d.trow, *qrow = d.draft + b * d.dseq + j * d.drow;
  const bool q_best = d.kind == kDraftBest, want_q = j < n && (d.kind == kDraftRows || q_best);
  const int64_t total = want_q ? 2 * d.n_parts : d.n_parts, step = size * kRollWarps;
  uint4 *ring = sh.ring[warp], *stage = ring;
  int64_t ahead = rank * kRollWarps + warp;
  const auto ask = [&](uint4 *to) {
    if (ahead < total) {
      const bool of_q = ahead >= d.n_parts;
      copy_vecs<DT, kLoadVecs>(to, of_q ? qrow : trow, (of_q ? ahead - d.n_parts : ahead) * kPartVecs, d.vocab);
    }
    copies_asked();
    ahead += step;
  };
#pragma unroll
  for (int k = 0; k < kStages; ++k) ask(ring + k * kPartVecs);
  if (!d.stop) all_started(cl);  // (with d.stop they have met before)
  Draft draft = {};
  if (rank == 0 && warp == 0) draft = draft_of<DT>(d, b, j, n, trow, qrow);
  RowSum t = nothing(), q = nothing();  // (q holds the row being swept, then the draft's)
  bool in_q = false;
#pragma unroll 1
  for (int64_t part = rank * kRollWarps + warp; part < total; part += step) {
    const bool of_q = part >= d.n_parts;
    if (of_q && !in_q) {
      t = q;
      q = nothing();
      in_q = true;
    }
    oldest_copy();
    uint4 raw[kLoadVecs];
#pragma unroll
    for (int v = 0; v < kLoadVecs; ++v) raw[v] = stage[v * 32 + lane];
    ask(stage);
    stage = stage + kPartVecs == ring + kStages * kPartVecs ? ring : stage + kPartVecs;
    if (kBest || (of_q && q_best)) add_best<DT>(q, raw, of_q ? part - d.n_parts : part);
    else add_part<DT>(q, raw, of_q ? d.cd : d.ct, of_q ? d.cd64 : d.ct64);
  }
  if (!in_q) {
    t = q;
    q = nothing();
  }
  if (!kBest) t.z = warp_sum(t.z);
  if (!q_best) q.z = warp_sum(q.z);
  if (lane == 0) {
    sh.part[0][warp] = t;
    sh.part[1][warp] = q;
  }
  __syncthreads();
  if (warp == 0) {
    t = lane < kRollWarps ? sh.part[0][lane] : nothing();
    q = lane < kRollWarps ? sh.part[1][lane] : nothing();
    t = kBest ? warp_merge_best(t) : warp_merge(t, d.ct64);
    if (want_q) q = q_best ? warp_merge_best(q) : warp_merge(q, d.cd64);
    if (lane == 0 && size > 1) {
      *cl.map_shared_rank(&sh.pub[0][rank], 0) = t;
      *cl.map_shared_rank(&sh.pub[1][rank], 0) = q;
    }
  }
  if (size > 1) {
    cl.sync();
    if (rank == 0 && warp == 0) {
      t = lane < size ? sh.pub[0][lane] : nothing();
      q = lane < size ? sh.pub[1][lane] : nothing();
      t = kBest ? warp_merge_best(t) : warp_merge(t, d.ct64);
      if (want_q) q = q_best ? warp_merge_best(q) : warp_merge(q, d.cd64);
    }
  }
  if (rank == 0 && warp == 0) {
    Position o;
    if (kBest) t.z = 1.0;
    if (q_best) q.z = 1.0;
    o.t = t;
    o.q = q;
    judge<DT>(d, draft, trow, j == n, kBest, o);
    if (lane == 0) d.pos[(int64_t)b * (d.K + 1) + j] = o;
    if (lane == 0 && d.stop && j < n && o.state != kAccept && o.state != kOpen) atomicMin(d.stop + b, j);
  }
}

// A cluster per position, earlier positions of all sequences first.  With d.stop (more positions than fit at once) a
// position behind a rejection that is known by then is left out.  With d.next (many more) clusters stay and take one
// position after another.
template <int DT, bool kBest>
__global__ void __launch_bounds__(kRollThreads, 4) verify_sweep_kernel(const __grid_constant__ RolloutDev d) {
  __shared__ RollShared sh;
  asm volatile("griddepcontrol.launch_dependents;");  // the finish may be set up beside the last positions
  cg::cluster_group cl = cg::this_cluster();
  say_started(cl);
  const int64_t id = blockIdx.x / cl.num_blocks();
  int32_t b = (int32_t)(id % d.B);
  if (d.stop) all_started(cl);  // (else hidden in the sweep)
  if (!d.next) {
    const int32_t j = (int32_t)(id / d.B);
    if (wanted(cl, d, b, j, sh)) sweep_position<DT, kBest>(cl, d, b, j, sh);
    else if (!d.stop) all_started(cl);
    return;
  }
  for (;;) {
    take_next(cl, d, b, sh);
    const int32_t j = sh.take[1];
    b = sh.take[0];
    if (j < 0) return;
    sweep_position<DT, kBest>(cl, d, b, j, sh);
    roll_sync(cl);  // what this round has read is written in the next one
  }
}

// One sequence of the finish, by a cluster.
template <int DT, bool kBest, int kMode>
__device__ __forceinline__ void finish_sequence(cg::cluster_group &cl, const RolloutDev &d, int32_t b, RollShared &sh) {
  using E = Elem<DT>;
  const int rank = (int)cl.block_rank(), size = (int)cl.num_blocks();
  const int32_t n = drafts_of(d, b), W = d.K + 1;
  int bits = d.n_draft && d.n_draft[b] != n ? FOPD_DEV_BAD_LENGTH : 0;
  const Position *pos = d.pos + (int64_t)b * W;
  const Slots sl = my_slots(d, rank, size);
  const int32_t limit = d.stop && d.stop[b] < n ? d.stop[b] : n;  // positions behind it may have been left out

  int32_t j = 0;
  int state, parity = 0;
  for (int32_t from = 0;; from = j + 1) {
    if (threadIdx.x == 0) sh.stop = limit;
    __syncthreads();
    for (int32_t k = from + threadIdx.x; k < limit; k += kRollThreads)
      if (pos[k].state != kAccept) {
        atomicMin(&sh.stop, k);
        break;
      }
    __syncthreads();
    j = sh.stop;
    __syncthreads();
    state = pos[j].state;
    if (kBest || state != kOpen) break;
    if (kMode == kFirst) {
      if (rank == 0 && threadIdx.x == 0) d.later->e[since_unset(atomicAdd(&d.later->count, 1))].unit = b;
      return;
    }
    const int32_t x = d.drafted[(int64_t)b * d.K + j];
    const char *trow = d.target + b * d.tseq + j * d.trow, *qrow = d.draft + b * d.dseq + j * d.drow;
    const bool rows = d.kind == kDraftRows;
    const ExactSums z = cluster_exact_sums<DT>(cl, trow, pos[j].t.m, rows ? qrow : nullptr, pos[j].q.m, d, sl, parity, sh);
    // u q < p with both sums on the other side: where the weights and sums are exact (even rows), so is this, since
    // a product rounded down is below a number exactly if the product is.  (kDraftBest: q is 1, or 0 and then never open)
    const double wp = exp64((double)E::load1(trow, x) - pos[j].t.m, d.ct64);
    const double wq = rows ? exp64((double)E::load1(qrow, x) - pos[j].q.m, d.cd64) : 1.0;
    if (!(__dmul_rd(d.uniform[(int64_t)b * W + j], wq * z.t) < wp * (rows ? z.q : 1.0))) {
      state = kReject;
      break;
    }
  }

  int32_t token = kUnsure;  // in the threads that know it
  float lp = 0.f;
  bool there = false;       // a token comes out
  const double v = d.uniform[(int64_t)b * W + d.K];
  if (state == kBadToken) bits |= FOPD_DEV_BAD_TOKEN;
  if (state == kBadRow) {
    bits |= FOPD_DEV_BAD_LOGITS;
    if (j < n && is_distribution(pos[j].t) && (uint32_t)d.drafted[(int64_t)b * d.K + j] >= (uint64_t)d.vocab)
      bits |= FOPD_DEV_BAD_TOKEN;
  } else if (state == kBadUniform) {
    bits |= FOPD_DEV_BAD_UNIFORM;
  } else if (kBest) {
    if (rank == 0) token = pos[j].t.best;
    there = true;
  } else if (!(v >= 0.0 && v < 1.0)) {
    bits |= FOPD_DEV_BAD_UNIFORM;
  } else {
    there = true;
    const RowSum t32 = pos[j].t, q32 = pos[j].q;
    Weights<DT> w = {};
    w.t = d.target + b * d.tseq + j * d.trow;
    w.q = d.draft + b * d.dseq + j * d.drow;
    w.V = d.vocab;
    w.rest = j < n && d.kind == kDraftRows;
    w.without = j == n ? -1 : d.kind == kDraftBest ? q32.best : d.kind == kDraftCertain ? d.drafted[(int64_t)b * d.K + j] : -1;
    w.ct = d.ct;
    w.cd = d.cd;
    w.ct64 = d.ct64;
    w.cd64 = d.cd64;
    w.tab = sh.tab;
    RowSum total;
    int turn = 0;  // two searches in a row exchange in different places: what one has left may still be read in the next
    for (int round = 0; round < 2; ++round) {  // the second one only where p - q is zero everywhere
      bool again = true;
      w.ts = t32;
      w.qs = q32;
      w.derive();
      if (kMode != kSecond && !w.beyond()) {
        if (w.rest) cta_sums<DT, false, true>(w, d, sl, sh);
        else cta_sums<DT, false, false>(w, d, sl, sh);
        // p - q: both rows' weights and both their sums are off; else the row's whole sum counts, with what was taken away
        // (and up to a twentieth for the rounding of max c, which these weights carry)
        token = cluster_search<DT, false, false>(cl, w, d, sl, v, 0.0, w.rest ? 9 * d.eps : 2.1 * d.eps * t32.z, turn, sh,
                                                 &total, &again);
        turn ^= 1;
        if (!is_distribution(total)) again = true;
      }
      if (!again) break;
      if (kMode == kFirst) {
        if (rank == 0 && threadIdx.x == 0) d.later->e[since_unset(atomicAdd(&d.later->count, 1))].unit = b;
        return;
      }
      if (w.rest) {
        const ExactSums z = cluster_exact_sums<DT>(cl, w.t, w.ts.m, w.q, w.qs.m, d, sl, parity, sh);
        w.ts.z = z.t;
        w.qs.z = z.q;
        w.derive();
        cta_sums<DT, true, true>(w, d, sl, sh);
      } else {
        cta_sums<DT, true, false>(w, d, sl, sh);
      }
      bool never;
      token = cluster_search<DT, true, false>(cl, w, d, sl, v, 0.0, 0.0, turn, sh, &total, &never);
      turn ^= 1;
      if (is_distribution(total)) break;
      w.rest = false;
      w.without = -1;
    }
    if (token >= 0 && threadIdx.x < 32) lp = log_prob<DT>(w.t, d.vocab, token, sh.logit, t32, d.ct, d.ct64);
  }
  const int64_t at = (int64_t)b * W;
  if (token != kUnsure && threadIdx.x == 0) {
    d.tokens[at + j] = token;
    if (d.logprob) d.logprob[at + j] = lp;
    if (d.mask) d.mask[at + j] = token >= 0 ? 1 : 0;
    if (token < 0 && d.status) atomicOr(d.status, FOPD_DEV_BAD_LOGITS);
  }
  if (rank == 0) {
    if (bits && threadIdx.x == 0 && d.status) atomicOr(d.status, bits);
    if (d.n_accepted && threadIdx.x == 0) d.n_accepted[b] = j;
    for (int32_t k = threadIdx.x; k < W; k += kRollThreads) {
      if (k == j && there) continue;
      d.tokens[at + k] = k < j ? d.drafted[(int64_t)b * d.K + k] : -1;
      if (d.logprob) d.logprob[at + k] = k < j ? pos[k].lp : 0.f;
      if (d.mask) d.mask[at + k] = k < j ? 1 : 0;
    }
  }
}

// A cluster per sequence: the first position that is not accepted (an open one is settled in fp64), the new token,
// the outputs.  Modes as for draws.
template <int DT, bool kBest, int kMode>
__global__ void __launch_bounds__(kRollThreads, kMode == kFirst ? 4 : 2) verify_finish_kernel(const __grid_constant__ RolloutDev d) {
  __shared__ RollShared sh;
  cg::cluster_group cl = cg::this_cluster();
  say_started(cl);
  if (!kBest && kMode != kFirst) fill_exp64(sh.tab);
  asm volatile("griddepcontrol.launch_dependents;");
  all_started(cl);
  asm volatile("griddepcontrol.wait;" ::: "memory");  // the sweep's positions are there, or the list
  const int size = (int)cl.num_blocks();
  const int64_t count = kMode == kSecond ? since_unset(d.later->count) : d.B, step = gridDim.x / size;
  for (int64_t k = blockIdx.x / size; k < count; k += step) {
    finish_sequence<DT, kBest, kMode>(cl, d, kMode == kSecond ? d.later->e[k].unit : (int32_t)k, sh);
    if (k + step < count) roll_sync(cl);  // the next one writes what this one has read
  }
}

}  // namespace fopd
