// Drawing tokens from rows of logits and verifying drafted tokens (fopd_draw_tokens,
// fopd_verify_draft).
//
// Which token comes out has to be that of exact arithmetic, and a running sum over 150,000
// probabilities in fp32 is off by more than many of them.  Evaluating every exponential in fp64 is
// not an option either (the fp64 pipe takes 5 logits per cycle and SM, memory brings 12).  So the
// sweeps run in fp32 with a bound on their error, and a decision that lies within it is made again in
// fp64: a few per cent of the draws.
//
// A row is cut into tiles of 256 16-byte vectors, one warp each; a cluster of C CTAs shares a row (or
// a pair of rows), C such that few rows still fill the GPU.  A search goes over the CTAs' sums, the
// owner's tile sums and the elements of one tile.
#pragma once

#include <cooperative_groups.h>

#include "common.cuh"

namespace fopd {

namespace cg = cooperative_groups;

constexpr int kRollThreads = 256;
constexpr int kRollWarps = kRollThreads / 32;
constexpr int kTileVecs = 8;        // 16-byte vectors of a tile per lane of a warp
constexpr int kTileSlots = 512;     // tiles per CTA; a longer row takes `span` tiles a slot
constexpr int kRollMaxCluster = 8;
constexpr int kRollResident = 592;  // CTAs of these kernels that 148 SMs hold at once (64 registers)

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

struct RolloutDev {
  const char *target, *draft;
  const int32_t *drafted, *n_draft;
  const double *uniform;
  int64_t vocab, n_tiles;
  int64_t tseq, trow, dseq, drow;  // bytes
  int32_t B, K;
  int kind;         // DraftKind
  int span;         // tiles per slot
  float ct, cd;     // log2(e) / temperature in fp32
  double ct64, cd64;
  double eps;       // relative error of a row's fp32 sum (and of a weight)
  Position *pos;    // [B, K + 1]
  int32_t *stop;    // [B] the lowest position known not to be accepted, or NULL: nobody looks
  int32_t *tokens;
  float *logprob;
  uint8_t *mask;
  int32_t *n_accepted;
  int32_t *status;
};

template <int DT>
struct TileShape {
  static constexpr int kElems = 32 * kTileVecs * Elem<DT>::kPerVec;
  static_assert(32 * kTileVecs == kRollThreads, "a tile is one vector for each thread of a CTA");
};

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

template <int DT>
__device__ __forceinline__ void load_tile(uint4 (&raw)[kTileVecs], const char *row, int64_t tile, int64_t V) {
  const int64_t i0 = tile * (32 * kTileVecs) + (threadIdx.x & 31);
  if ((tile + 1) * TileShape<DT>::kElems <= V) {
    const uint4 *p = reinterpret_cast<const uint4 *>(row) + i0;
#pragma unroll
    for (int v = 0; v < kTileVecs; ++v) raw[v] = ld_row(p + v * 32);
  } else {
#pragma unroll
    for (int v = 0; v < kTileVecs; ++v) raw[v] = row_vec<DT>(row, i0 + v * 32, V);
  }
}

// ---- fp32 sums --------------------------------------------------------------------------------------

template <int N>
__device__ __forceinline__ float tree_sum(float (&x)[N]) {
#pragma unroll
  for (int n = N / 2; n > 0; n >>= 1)
#pragma unroll
    for (int k = 0; k < n; ++k) x[k] += x[k + n];
  return x[0];
}

__device__ __forceinline__ float max_nan(float a, float b) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}

// {max, lowest index of it} of one tile, in every lane; a NaN anywhere gives NaN.
template <int DT>
__device__ __forceinline__ RowSum tile_best(const char *row, int64_t tile, int64_t V) {
  using E = Elem<DT>;
  constexpr int P = E::kPerVec;
  uint4 raw[kTileVecs];
  load_tile<DT>(raw, row, tile, V);
  float m = -INFINITY;
#pragma unroll
  for (int v = 0; v < kTileVecs; ++v) {
    float x[P];
    E::unpack(raw[v], x);
#pragma unroll
    for (int k = 0; k < P; ++k) m = max_nan(m, x[k]);
  }
  if (__any_sync(0xffffffffu, isnan(m))) return {NAN, INT32_MAX, 1.0};
  const float top = warp_max(m);
  int32_t at = INT32_MAX;
  if (m == top) {
#pragma unroll
    for (int v = kTileVecs - 1; v >= 0; --v) {
      float x[P];
      E::unpack(raw[v], x);
#pragma unroll
      for (int k = P - 1; k >= 0; --k)
        if (x[k] == top) at = (int32_t)((tile * (32 * kTileVecs) + v * 32 + (threadIdx.x & 31)) * P + k);
    }
  }
  return {top, (int32_t)__reduce_min_sync(0xffffffffu, at), 1.0};
}

// Sums of a row, tile after tile: {max, sum 2^{(x - max) c}} with the maximum the warp's and the sum the lane's own.
// The exponent is x c - fl(max c) in one fused multiply-add; what fl() took away is the same for all elements and put
// back at the end.  -infinity everywhere gives {-inf, 0}; a NaN or +inf makes the sum NaN.
template <int DT>
__device__ __forceinline__ void add_tile(RowSum &acc, const char *row, int64_t tile, int64_t V, float c, double c64) {
  using E = Elem<DT>;
  constexpr int P = E::kPerVec;
  uint4 raw[kTileVecs];
  load_tile<DT>(raw, row, tile, V);
  float m = -INFINITY;
#pragma unroll
  for (int v = 0; v < kTileVecs; ++v) {
    float x[P];
    E::unpack(raw[v], x);
    m = fmaxf(m, max_of<P>(x));
  }
  m = warp_max(m);
  if (m > acc.m) {
    acc.z = acc.m == -INFINITY ? acc.z : acc.z * exp2(((double)acc.m - m) * c64);
    acc.m = m;
  }
  m = acc.m;
  const float mc = m == -INFINITY ? 0.f : m * c;
  double z = 0.0;
  if (fabsf(mc) <= 1e38f) {
#pragma unroll
    for (int v = 0; v < kTileVecs; ++v) {
      float x[P];
      E::unpack(raw[v], x);
#pragma unroll
      for (int k = 0; k < P; ++k) x[k] = ex2(fmaf(x[k], c, -mc));
      z += (double)tree_sum<P>(x);
    }
    if (m != -INFINITY) z *= (double)ex2(-fmaf(m, c, -mc));
  } else {  // max c is beyond fp32 (or max is infinite: NaN)
    for (int v = 0; v < kTileVecs; ++v) {
      float x[P];
      E::unpack(raw[v], x);
#pragma unroll
      for (int k = 0; k < P; ++k) x[k] = ex2((x[k] - m) * c);
      z += (double)tree_sum<P>(x);
    }
  }
  acc.z += z;
}

// Two parts of a row as one.  (2^y in fp64: a few hundred merges a row, and their error stays out of the bound.)
__device__ __forceinline__ RowSum merge(const RowSum &a, const RowSum &b, double c) {
  if (b.m == -INFINITY && !isnan(b.z)) return a;
  if (a.m == -INFINITY && !isnan(a.z)) return b;
  if (a.m >= b.m) return {a.m, a.best, a.z + b.z * exp2(((double)b.m - a.m) * c)};
  return {b.m, b.best, b.z + a.z * exp2(((double)a.m - b.m) * c)};  // (NaN maxima: is_distribution sees them)
}
__device__ __forceinline__ RowSum merge_best(const RowSum &a, const RowSum &b) {
  const bool first = isnan(a.m) || (!isnan(b.m) && (a.m > b.m || (a.m == b.m && a.best <= b.best)));
  return first ? a : b;
}
__device__ __forceinline__ RowSum nothing() { return {-INFINITY, INT32_MAX, 0.0}; }

__device__ __forceinline__ RowSum shfl_xor(const RowSum &a, int lanes) {
  return {__shfl_xor_sync(0xffffffffu, a.m, lanes), __shfl_xor_sync(0xffffffffu, a.best, lanes),
          __shfl_xor_sync(0xffffffffu, a.z, lanes)};
}
template <bool kBest>
__device__ __forceinline__ RowSum warp_merge(RowSum a, double c) {
#pragma unroll
  for (int off = 16; off > 0; off >>= 1) a = kBest ? merge_best(a, shfl_xor(a, off)) : merge(a, shfl_xor(a, off), c);
  return a;
}

__device__ __forceinline__ bool is_distribution(const RowSum &r) {
  return r.m > -INFINITY && r.m < INFINITY && r.z > 0.0 && r.z < INFINITY;
}

// ---- fp64 weights -----------------------------------------------------------------------------------

// 2^{(x - m) c}: the exponent rounded to sixteenths, 2^{j/16} from a table in shared memory (sixteen entries lie in
// sixteen banks) and six terms of the Taylor series of 2^f, |f| <= 1/32: error below 1e-15.
struct Exp64 {
  const double *tab;
  __device__ __forceinline__ double operator()(float x, double m, double c, float least) const {
    constexpr double kRound = 6755399441055744.0 / 16;  // 1.5 * 2^52 / 16: adding it rounds to sixteenths
    const double d = (double)x - m;
    const double t = fma(d, c, kRound);
    const double f = fma(d, c, kRound - t);
    const int n = __double2loint(t);
    double p = 1.5403530393381608e-4;
    p = fma(p, f, 1.3333558146428443e-3);
    p = fma(p, f, 9.6181291076284772e-3);
    p = fma(p, f, 5.5504108664821580e-2);
    p = fma(p, f, 2.4022650695910071e-1);
    p = fma(p, f, 6.9314718055994531e-1);
    p = fma(p, f, 1.0);
    p *= tab[n & 15];
    p = __hiloint2double(__double2hiint(p) + ((n >> 4) << 20), __double2loint(p));
    return x >= least ? p : 0.0;  // 2^-1000 and less is nothing (and -infinity has no f)
  }
};
__device__ __forceinline__ void fill_exp64(double *tab) {
  if (threadIdx.x < 16) tab[threadIdx.x] = exp2((double)threadIdx.x / 16.0);
}
__device__ __forceinline__ float least_of(float m, double c) { return (float)((double)m - 1000.0 / c); }

// Weights of the distribution a token is drawn from, a vector of elements at a time.
enum WeightKind { kWPlain = 0, kWWithout = 1, kWRest = 2 };
template <int DT>
struct Weights {
  static constexpr int P = Elem<DT>::kPerVec;
  const char *t, *q;  // rows
  int64_t V;
  int kind;           // WeightKind
  int32_t without;    // kWWithout: the element of which everything is taken away
  RowSum ts, qs;
  float ct, cd;
  double ct64, cd64;
  // derived
  float mct, mcd, a, b;  // fl(max c); 2^{what fl() took} / sum
  float least_t, least_q;
  double ia, ib;         // 1 / sum
  Exp64 e;

  __device__ __forceinline__ void derive() {
    mct = ts.m * ct;
    a = kind == kWRest ? (float)((double)ex2(-fmaf(ts.m, ct, -mct)) / ts.z) : 1.f;
    least_t = least_of(ts.m, ct64);
    ia = 1.0 / ts.z;
    if (kind == kWRest) {
      mcd = qs.m * cd;
      b = (float)((double)ex2(-fmaf(qs.m, cd, -mcd)) / qs.z);
      least_q = least_of(qs.m, cd64);
      ib = 1.0 / qs.z;
    }
  }
  // fp32's exponent cannot be formed (see tile_sum)
  __device__ __forceinline__ bool beyond() const {
    return !(fabsf(mct) <= 1e38f) || (kind == kWRest && !(fabsf(mcd) <= 1e38f));
  }

  __device__ __forceinline__ void fast(int64_t i, const uint4 &rt, const uint4 &rq, float (&w)[P]) const {
    float x[P];
    Elem<DT>::unpack(rt, x);
#pragma unroll
    for (int k = 0; k < P; ++k) w[k] = ex2(fmaf(x[k], ct, -mct));
    if (kind == kWRest) {
      Elem<DT>::unpack(rq, x);
#pragma unroll
      for (int k = 0; k < P; ++k) w[k] = fmaxf(fmaf(w[k], a, -b * ex2(fmaf(x[k], cd, -mcd))), 0.f);
    } else if (kind == kWWithout) {
#pragma unroll
      for (int k = 0; k < P; ++k)
        if (i * P + k == without) w[k] = 0.f;
    }
  }
  __device__ __forceinline__ void exact(int64_t i, const uint4 &rt, const uint4 &rq, double (&w)[P]) const {
    float x[P];
    Elem<DT>::unpack(rt, x);
#pragma unroll
    for (int k = 0; k < P; ++k) w[k] = e(x[k], ts.m, ct64, least_t);
    if (kind == kWRest) {
      Elem<DT>::unpack(rq, x);
#pragma unroll
      for (int k = 0; k < P; ++k)  // (both products rounded alike: equal rows leave exactly nothing)
        w[k] = fmax(__dsub_rn(__dmul_rn(w[k], ia), __dmul_rn(e(x[k], qs.m, cd64, least_q), ib)), 0.0);
    } else if (kind == kWWithout) {
#pragma unroll
      for (int k = 0; k < P; ++k)
        if (i * P + k == without) w[k] = 0.0;
    }
  }
  // sum of a vector's weights, in fp64 from the vector up
  template <bool kExact>
  __device__ __forceinline__ double vec_sum(int64_t i) const {
    const uint4 rt = row_vec<DT>(t, i, V), rq = kind == kWRest ? row_vec<DT>(q, i, V) : make_uint4(0, 0, 0, 0);
    if (kExact) {
      double w[P], s = 0.0;
      exact(i, rt, rq, w);
#pragma unroll
      for (int k = 0; k < P; ++k) s += w[k];
      return s;
    }
    float w[P];
    fast(i, rt, rq, w);
    return (double)tree_sum<P>(w);
  }
};

// ---- a CTA's and a cluster's tools ------------------------------------------------------------------

struct RollShared {
  double tz[kTileSlots];  // tile sums of this CTA
  float tm[kTileSlots];
  double scan[kRollWarps];
  double tab[16];
  RowSum part[2][kRollWarps];
  RowSum pub[2][2];       // what other CTAs of the cluster read: [exchange parity][row]
  double before, goal;
  int64_t slot;
  int32_t owner, result, flag[2];
};

// This CTA's slots of a row: [lo, hi) of ceil(n_tiles / span), contiguous and in rank order.
struct Slots {
  int64_t lo, hi;
};
__device__ __forceinline__ Slots my_slots(const RolloutDev &d, int rank, int size) {
  const int64_t n = (d.n_tiles + d.span - 1) / d.span, per = (n + size - 1) / size;
  const int64_t lo = rank * per, hi = lo + per;
  return {lo < n ? lo : n, hi < n ? hi : n};
}

// Inclusive scan over the CTA's threads.
__device__ __forceinline__ double cta_scan(double x, double *scan) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
  for (int off = 1; off < 32; off <<= 1) {
    const double y = __shfl_up_sync(0xffffffffu, x, off);
    if (lane >= off) x += y;
  }
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

// The element of tiles [tile0, tile0 + span) whose running sum (starting at `before`) passes `goal`; where rounding
// leaves none, the last one with a weight.  Same result in every thread.
template <int DT, bool kExact>
__device__ int32_t cta_find(const Weights<DT> &w, const RolloutDev &d, int64_t tile0, double before, double goal,
                            double bound, RollShared &sh) {
  constexpr int P = Weights<DT>::P;
  if (threadIdx.x == 0) sh.result = kUnsure;
  const int64_t tiles = min((int64_t)d.span, d.n_tiles - tile0);
  int64_t last = 0;  // the last tile with a weight, and the running sum before it
  double last_before = before;
  for (int64_t s = 0; s <= tiles; ++s) {
    const bool back = s == tiles;  // no tile passes: the last weight it is
    const int64_t i = (tile0 + (back ? last : s)) * kRollThreads + threadIdx.x;
    if (back) before = last_before;
    double x[P], sum = 0.0;
    const uint4 rt = row_vec<DT>(w.t, i, d.vocab),
                rq = w.kind == kWRest ? row_vec<DT>(w.q, i, d.vocab) : make_uint4(0, 0, 0, 0);
    if (kExact) {
      w.exact(i, rt, rq, x);
    } else {
      float y[P];
      w.fast(i, rt, rq, y);
#pragma unroll
      for (int k = 0; k < P; ++k) x[k] = (double)y[k];
    }
#pragma unroll
    for (int k = 0; k < P; ++k) sum += x[k];
    const double incl = before + cta_scan(sum, sh.scan);
    const bool here = sum > 0.0 && (back || incl > goal);
    if (!__syncthreads_or(here)) {
      if (__syncthreads_or(sum > 0.0)) {
        last = s;
        last_before = before;
      }
#pragma unroll
      for (int k = 0; k < kRollWarps; ++k) before += sh.scan[k];
      continue;
    }
    if (threadIdx.x == 0) sh.flag[0] = back ? -1 : kRollThreads;
    __syncthreads();
    if (here && back) atomicMax(&sh.flag[0], (int)threadIdx.x);
    else if (here) atomicMin(&sh.flag[0], (int)threadIdx.x);
    __syncthreads();
    if (sh.flag[0] == (int)threadIdx.x) {
      double run = incl - sum, at_before = run, at_after = run;
      int32_t at = kUnsure;
#pragma unroll
      for (int k = 0; k < P; ++k) {
        if (x[k] > 0.0 && (at < 0 || at_after <= goal)) {
          at = (int32_t)(i * P + k);
          at_before = run;
          at_after = run + x[k];
        }
        run += x[k];
      }
      if (kExact || (goal - at_before > bound && at_after - goal > bound)) sh.result = at;
    }
    break;
  }
  __syncthreads();
  return sh.result;
}

// Search over the cluster.  On entry this CTA's slots have their sums in sh.tz relative to 2^{tm c} (or all to the same
// reference: relative false).  The CTAs exchange their totals; the owner of the goal looks through its slots, then its
// tile.  Returns the token in the owner's threads and elsewhere kUnsure; *total in all.  Whether the cluster is to do
// it again in fp64 comes back in *again.  One cluster barrier before the search and, in fp32, one behind it; the other
// CTAs' shared memory may still be read after the last one.  kRelative: w gets the row's sum.
template <int DT, bool kExact, bool kRelative>
__device__ int32_t cluster_search(cg::cluster_group &cl, Weights<DT> &w, const RolloutDev &d, Slots sl, double v,
                                  double bound_rel, double bound_abs, int parity, RollShared &sh, RowSum *total,
                                  bool *again) {
  const int rank = (int)cl.block_rank(), size = (int)cl.num_blocks();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int n = (int)(sl.hi - sl.lo);
  if (warp == 0) {
    RowSum r = nothing();
    if (kRelative) {
      for (int t = lane; t < n; t += 32) r = merge(r, RowSum{sh.tm[t], 0, sh.tz[t]}, d.ct64);
      r = warp_merge<false>(r, d.ct64);
    } else {
      double s = 0.0;
      for (int t = lane; t < n; t += 32) s += sh.tz[t];
      r = {0.f, 0, warp_sum(s)};
    }
    if (lane == 0) sh.pub[parity][0] = r;
  }
  cl.sync();
  if (warp == 0) {
    RowSum mine = nothing();
    if (lane < size) mine = *cl.map_shared_rank(&sh.pub[parity][0], lane);
    const RowSum all = warp_merge<false>(mine, d.ct64);
    const double part = lane < size && mine.z > 0.0 ? mine.z * exp2(((double)mine.m - all.m) * d.ct64) : 0.0;
    double incl = part;
#pragma unroll
    for (int off = 1; off < 32; off <<= 1) {
      const double y = __shfl_up_sync(0xffffffffu, incl, off);
      if (lane >= off) incl += y;
    }
    double sum = __shfl_sync(0xffffffffu, incl, 31);
    const double goal = v * sum;
    if (isnan(all.z)) sum = all.z;
    const unsigned pass = __ballot_sync(0xffffffffu, part > 0.0 && incl > goal), has = __ballot_sync(0xffffffffu, part > 0.0);
    const int owner = pass ? __ffs(pass) - 1 : has ? 31 - __clz(has) : 0;
    const double before = __shfl_sync(0xffffffffu, incl - part, owner);
    if (lane == 0) {
      sh.pub[parity][1] = {all.m, 0, sum};
      sh.owner = owner;
      sh.goal = goal;
      sh.before = before;
    }
    __syncwarp();
    if (owner == rank && is_distribution({all.m, 0, sum})) {  // this CTA's slots
      double run = before;
      int64_t slot = -1, last = -1;
      double at = run, last_at = run;
      for (int base = 0; base < n && slot < 0; base += 32) {
        const int t = base + lane;
        const double x = t < n && sh.tz[t] > 0.0
                             ? sh.tz[t] * (kRelative ? exp2(((double)sh.tm[t] - all.m) * d.ct64) : 1.0) : 0.0;
        double in = x;
#pragma unroll
        for (int off = 1; off < 32; off <<= 1) {
          const double y = __shfl_up_sync(0xffffffffu, in, off);
          if (lane >= off) in += y;
        }
        const unsigned p = __ballot_sync(0xffffffffu, x > 0.0 && run + in > goal), h = __ballot_sync(0xffffffffu, x > 0.0);
        const int l = p ? __ffs(p) - 1 : h ? 31 - __clz(h) : -1;
        const double b = __shfl_sync(0xffffffffu, run + in - x, l < 0 ? 0 : l);
        if (p) {
          slot = base + l;
          at = b;
        } else if (h) {
          last = base + l;
          last_at = b;
        }
        run += __shfl_sync(0xffffffffu, in, 31);
      }
      if (lane == 0) {
        sh.slot = sl.lo + (slot >= 0 ? slot : last);
        sh.before = slot >= 0 ? at : last_at;
      }
    }
  }
  __syncthreads();
  *total = sh.pub[parity][1];
  int32_t token = kUnsure;
  const bool good = is_distribution(*total);
  if (good && sh.owner == rank) {
    if (kRelative) {
      w.ts = *total;
      w.derive();
    }
    const double bound = bound_rel * total->z + bound_abs;
    token = cta_find<DT, kExact>(w, d, sh.slot * d.span, sh.before, sh.goal, bound, sh);
    if (threadIdx.x == 0) sh.flag[1] = token == kUnsure;
  }
  *again = false;
  if (!kExact) {
    cl.sync();
    if (good) *again = *cl.map_shared_rank(&sh.flag[1], sh.owner) != 0;
  }
  return token;
}

// Slot sums of the weights in fp32 or fp64, relative to one reference.
template <int DT, bool kExact>
__device__ __forceinline__ void cta_slot_sums(const Weights<DT> &w, const RolloutDev &d, Slots sl, RollShared &sh) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  for (int64_t t = sl.lo + warp; t < sl.hi; t += kRollWarps) {
    double s = 0.0;
    const int64_t end = min((t + 1) * d.span, d.n_tiles);
    for (int64_t tile = t * d.span; tile < end; ++tile)
#pragma unroll
      for (int v = 0; v < kTileVecs; ++v) s += w.template vec_sum<kExact>(tile * kRollThreads + v * 32 + lane);
    s = warp_sum(s);
    if (lane == 0) sh.tz[t - sl.lo] = s;
  }
  __syncthreads();
}

// A row's sum of exponentials in fp64, over the cluster, in every thread.
template <int DT>
__device__ double cluster_exact_sum(cg::cluster_group &cl, const char *row, float m, double c, const RolloutDev &d,
                                    Slots sl, RollShared &sh) {
  Weights<DT> w = {};
  w.t = row;
  w.V = d.vocab;
  w.kind = kWPlain;
  w.ts = {m, 0, 1.0};
  w.ct64 = c;
  w.least_t = least_of(m, c);
  w.e.tab = sh.tab;
  cta_slot_sums<DT, true>(w, d, sl, sh);
  if (threadIdx.x < 32) {
    double s = 0.0;
    for (int t = threadIdx.x; t < (int)(sl.hi - sl.lo); t += 32) s += sh.tz[t];
    s = warp_sum(s);
    if (threadIdx.x == 0) sh.pub[0][0].z = s;
  }
  cl.sync();
  double s = 0.0;
  for (unsigned k = 0; k < cl.num_blocks(); ++k) s += cl.map_shared_rank(&sh.pub[0][0], k)->z;
  cl.sync();  // the sums have been read
  return s;
}

// 1 / T from log2(e) / T
__device__ __forceinline__ double inv_temperature(double c) { return 0.69314718055994530942 * c; }

// ---- draws: a cluster per row -----------------------------------------------------------------------

template <int DT, bool kBest>
__global__ void __launch_bounds__(kRollThreads, 4) draw_kernel(const __grid_constant__ RolloutDev d) {
  __shared__ RollShared sh;
  cg::cluster_group cl = cg::this_cluster();
  const int rank = (int)cl.block_rank(), size = (int)cl.num_blocks();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int64_t n = blockIdx.x / size;
  const char *row = d.target + n * d.tseq;
  const Slots sl = my_slots(d, rank, size);
  RowSum best = nothing();
  for (int64_t t = sl.lo + warp; t < sl.hi; t += kRollWarps) {
    RowSum r = nothing();
    const int64_t end = min((t + 1) * d.span, d.n_tiles);
    for (int64_t tile = t * d.span; tile < end; ++tile) {
      if (kBest) best = merge_best(best, tile_best<DT>(row, tile, d.vocab));
      else add_tile<DT>(r, row, tile, d.vocab, d.ct, d.ct64);
    }
    if (!kBest) {
      r.z = warp_sum(r.z);
      if (lane == 0) {
        sh.tm[t - sl.lo] = r.m;
        sh.tz[t - sl.lo] = r.z;
      }
    }
  }
  if (kBest) {
    if (lane == 0) sh.part[0][warp] = best;
    __syncthreads();
    if (warp == 0) {
      const RowSum r = warp_merge<true>(lane < kRollWarps ? sh.part[0][lane] : nothing(), 0.0);
      if (lane == 0) sh.pub[0][0] = r;
    }
    cl.sync();
    if (rank == 0 && warp == 0) {
      const RowSum r = warp_merge<true>(lane < size ? *cl.map_shared_rank(&sh.pub[0][0], lane) : nothing(), 0.0);
      if (lane == 0) {
        const bool good = r.m > -INFINITY && r.m < INFINITY;
        d.tokens[n] = good ? r.best : -1;
        if (d.logprob) d.logprob[n] = 0.f;
        if (d.mask) d.mask[n] = good ? 1 : 0;
        if (d.n_accepted) d.n_accepted[n] = 0;
        if (!good && d.status) atomicOr(d.status, FOPD_DEV_BAD_LOGITS);
      }
    }
    cl.sync();  // nobody leaves while its shared memory is read
    return;
  }
  fill_exp64(sh.tab);
  __syncthreads();
  const double v = d.uniform[n];
  const bool v_ok = v >= 0.0 && v < 1.0;
  Weights<DT> w = {};
  w.t = row;
  w.V = d.vocab;
  w.kind = kWPlain;
  w.without = -1;
  w.ct = d.ct;
  w.ct64 = d.ct64;
  w.e.tab = sh.tab;
  RowSum total;
  bool again;
  int32_t token = cluster_search<DT, false, true>(cl, w, d, sl, v_ok ? v : 0.0, 2 * d.eps, 0.0, 0, sh, &total, &again);
  const bool good = is_distribution(total) && v_ok;
  const double z = total.z;
  if (again && good) {
    w.ts = total;
    w.derive();
    cta_slot_sums<DT, true>(w, d, sl, sh);
    RowSum exact_total;
    bool never;
    token = cluster_search<DT, true, false>(cl, w, d, sl, v, 0.0, 0.0, 1, sh, &exact_total, &never);
  }
  if (good && token >= 0 && threadIdx.x == 0) {
    d.tokens[n] = token;
    if (d.logprob)
      d.logprob[n] = (float)(((double)Elem<DT>::load1(row, token) - total.m) * inv_temperature(d.ct64) - log(z));
  }
  if (!good && rank == 0 && threadIdx.x == 0) {
    d.tokens[n] = -1;
    if (d.logprob) d.logprob[n] = 0.f;
    if (d.status) atomicOr(d.status, is_distribution(total) ? FOPD_DEV_BAD_UNIFORM : FOPD_DEV_BAD_LOGITS);
  }
  if (rank == 0 && threadIdx.x == 0) {
    if (d.mask) d.mask[n] = good ? 1 : 0;
    if (d.n_accepted) d.n_accepted[n] = 0;
  }
  cl.sync();  // nobody leaves while its shared memory is read
}

// ---- verification -----------------------------------------------------------------------------------

__device__ __forceinline__ int32_t drafts_of(const RolloutDev &d, int32_t b) {
  const int32_t n = d.n_draft ? d.n_draft[b] : d.K;
  return n < 0 ? 0 : n > d.K ? d.K : n;
}

// Decides on one position from its rows' sums.
template <int DT>
__device__ __forceinline__ void judge(const RolloutDev &d, int32_t b, int32_t j, int32_t n, bool target_best, Position &o) {
  using E = Elem<DT>;
  o.lp = 0.f;
  o.state = is_distribution(o.t) ? kEnd : kBadRow;
  if (o.state == kBadRow || j == n) return;
  const int32_t x = d.drafted[(int64_t)b * d.K + j];
  const double u = d.uniform[(int64_t)b * (d.K + 1) + j];
  if (x < 0 || x >= d.vocab) {
    o.state = kBadToken;
  } else if (target_best) {
    o.state = x == o.t.best ? kAccept : kReject;
  } else if (!(u >= 0.0 && u < 1.0)) {
    o.state = kBadUniform;
  } else {
    const double y = ((double)E::load1(d.target + b * d.tseq + j * d.trow, x) - o.t.m) * inv_temperature(d.ct64);
    const double p = exp(y) / o.t.z;
    o.lp = (float)(y - log(o.t.z));
    double q = 1.0;
    if (d.kind == kDraftRows)
      q = exp(((double)E::load1(d.draft + b * d.dseq + j * d.drow, x) - o.q.m) * inv_temperature(d.cd64)) / o.q.z;
    else if (d.kind == kDraftBest)
      q = x == o.q.best ? 1.0 : 0.0;
    const double uq = u * q;
    o.state = fabs(uq - p) < 4 * d.eps * fmax(uq, p) ? kOpen : uq < p ? kAccept : kReject;
  }
  if ((d.kind == kDraftRows || d.kind == kDraftBest) && o.state != kBadUniform && !is_distribution(o.q)) o.state = kBadRow;
}

// A cluster per position, earlier positions of all sequences first: sums of the target's and the draft's row, and the
// decision.  With d.stop (one CTA a position, more positions than fit at once) a position behind a rejection that is
// known by then is left out.
template <int DT, bool kBest>
__global__ void __launch_bounds__(kRollThreads, 4) verify_sweep_kernel(const __grid_constant__ RolloutDev d) {
  __shared__ RollShared sh;
  cg::cluster_group cl = cg::this_cluster();
  const int rank = (int)cl.block_rank(), size = (int)cl.num_blocks();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int64_t id = blockIdx.x / size;
  const int32_t j = (int32_t)(id / d.B), b = (int32_t)(id % d.B);
  const int32_t n = drafts_of(d, b);
  if (j > n) return;  // (all CTAs of the cluster alike)
  // (one thread looks: the value may change between two looks)
  if (d.stop && __syncthreads_or(threadIdx.x == 0 && *(volatile const int32_t *)(d.stop + b) < j)) return;
  const char *trow = d.target + b * d.tseq + j * d.trow, *qrow = d.draft + b * d.dseq + j * d.drow;
  const bool want_q = j < n && (d.kind == kDraftRows || d.kind == kDraftBest);
  RowSum t = nothing(), q = nothing();
  for (int64_t tile = rank * kRollWarps + warp; tile < d.n_tiles; tile += size * kRollWarps) {
    if (kBest) t = merge_best(t, tile_best<DT>(trow, tile, d.vocab));
    else add_tile<DT>(t, trow, tile, d.vocab, d.ct, d.ct64);
  }
  if (want_q) {
    if (d.kind == kDraftBest)
      for (int64_t tile = rank * kRollWarps + warp; tile < d.n_tiles; tile += size * kRollWarps)
        q = merge_best(q, tile_best<DT>(qrow, tile, d.vocab));
    else
      for (int64_t tile = rank * kRollWarps + warp; tile < d.n_tiles; tile += size * kRollWarps)
        add_tile<DT>(q, qrow, tile, d.vocab, d.cd, d.cd64);
  }
  if (!kBest) t.z = warp_sum(t.z);
  if (d.kind == kDraftRows) q.z = warp_sum(q.z);
  if (lane == 0) {
    sh.part[0][warp] = t;
    sh.part[1][warp] = q;
  }
  __syncthreads();
  const bool q_best = d.kind == kDraftBest;
  if (warp == 0) {
    t = lane < kRollWarps ? sh.part[0][lane] : nothing();
    q = lane < kRollWarps ? sh.part[1][lane] : nothing();
    t = kBest ? warp_merge<true>(t, 0.0) : warp_merge<false>(t, d.ct64);
    if (want_q) q = q_best ? warp_merge<true>(q, 0.0) : warp_merge<false>(q, d.cd64);
    if (lane == 0) {
      sh.pub[0][0] = t;
      sh.pub[0][1] = q;
    }
  }
  if (size > 1) {
    cl.sync();
    if (rank == 0 && warp == 0) {
      t = lane < size ? *cl.map_shared_rank(&sh.pub[0][0], lane) : nothing();
      q = lane < size ? *cl.map_shared_rank(&sh.pub[0][1], lane) : nothing();
      t = kBest ? warp_merge<true>(t, 0.0) : warp_merge<false>(t, d.ct64);
      if (want_q) q = q_best ? warp_merge<true>(q, 0.0) : warp_merge<false>(q, d.cd64);
    }
  }
  if (rank == 0 && threadIdx.x == 0) {
    Position o;
    if (kBest) t.z = 1.0;
    if (q_best) q.z = 1.0;
    o.t = t;
    o.q = q;
    judge<DT>(d, b, j, n, kBest, o);
    d.pos[(int64_t)b * (d.K + 1) + j] = o;
    if (d.stop && j < n && o.state != kAccept && o.state != kOpen) atomicMin(d.stop + b, j);
  }
  if (size > 1) cl.sync();
}

// A cluster per sequence: the first position that is not accepted (an open one is settled in fp64), the new token,
// the outputs.
template <int DT, bool kBest>
__global__ void __launch_bounds__(kRollThreads, 2) verify_finish_kernel(const __grid_constant__ RolloutDev d) {
  using E = Elem<DT>;
  __shared__ RollShared sh;
  __shared__ int stop;
  cg::cluster_group cl = cg::this_cluster();
  const int rank = (int)cl.block_rank(), size = (int)cl.num_blocks();
  const int32_t b = blockIdx.x / size;
  const int32_t n = drafts_of(d, b), W = d.K + 1;
  int bits = d.n_draft && d.n_draft[b] != n ? FOPD_DEV_BAD_LENGTH : 0;
  const Position *pos = d.pos + (int64_t)b * W;
  const Slots sl = my_slots(d, rank, size);
  if (!kBest) fill_exp64(sh.tab);
  const int32_t limit = d.stop && d.stop[b] < n ? d.stop[b] : n;  // positions behind it may have been left out

  int32_t j = 0;
  int state;
  for (int32_t from = 0;; from = j + 1) {
    if (threadIdx.x == 0) stop = limit;
    __syncthreads();
    for (int32_t k = from + threadIdx.x; k < limit; k += kRollThreads)
      if (pos[k].state != kAccept) {
        atomicMin(&stop, k);
        break;
      }
    __syncthreads();
    j = stop;
    __syncthreads();
    state = pos[j].state;
    if (kBest || state != kOpen) break;
    const int64_t at = (int64_t)b * d.K + j;
    const int32_t x = d.drafted[at];
    const char *trow = d.target + b * d.tseq + j * d.trow, *qrow = d.draft + b * d.dseq + j * d.drow;
    const double p = exp(((double)E::load1(trow, x) - pos[j].t.m) * inv_temperature(d.ct64)) /
                     cluster_exact_sum<DT>(cl, trow, pos[j].t.m, d.ct64, d, sl, sh);
    double q = 1.0;  // (kDraftBest: or 0 and then never open)
    if (d.kind == kDraftRows)
      q = exp(((double)E::load1(qrow, x) - pos[j].q.m) * inv_temperature(d.cd64)) /
          cluster_exact_sum<DT>(cl, qrow, pos[j].q.m, d.cd64, d, sl, sh);
    if (!(d.uniform[(int64_t)b * W + j] * q < p)) {
      state = kReject;
      break;
    }
  }

  int32_t token = -1;  // in the threads that know it
  float lp = 0.f;
  const double v = d.uniform[(int64_t)b * W + d.K];
  bool there = false;  // a token comes out
  if (state == kBadToken) bits |= FOPD_DEV_BAD_TOKEN;
  if (state == kBadRow) {
    bits |= FOPD_DEV_BAD_LOGITS;
    if (j < n && is_distribution(pos[j].t) && (uint32_t)d.drafted[(int64_t)b * d.K + j] >= (uint64_t)d.vocab)
      bits |= FOPD_DEV_BAD_TOKEN;
  } else if (state == kBadUniform) bits |= FOPD_DEV_BAD_UNIFORM;
  else if (kBest) {
    token = rank == 0 ? pos[j].t.best : -1;
    there = true;
  } else if (!(v >= 0.0 && v < 1.0)) bits |= FOPD_DEV_BAD_UNIFORM;
  else {
    there = true;
    Weights<DT> w = {};
    w.t = d.target + b * d.tseq + j * d.trow;
    w.q = d.draft + b * d.dseq + j * d.drow;
    w.V = d.vocab;
    w.kind = j == n ? kWPlain : d.kind == kDraftRows ? kWRest : kWWithout;
    w.without = j == n ? -1 : d.kind == kDraftBest ? pos[j].q.best : d.kind == kDraftCertain ? d.drafted[(int64_t)b * d.K + j] : -1;
    w.ts = pos[j].t;
    w.qs = pos[j].q;
    w.ct = d.ct;
    w.cd = d.cd;
    w.ct64 = d.ct64;
    w.cd64 = d.cd64;
    w.e.tab = sh.tab;
    const RowSum t32 = w.ts, q32 = w.qs;
    RowSum total;
    for (int round = 0; round < 2; ++round) {  // the second one only where p - q is zero everywhere
      bool again = true;
      w.ts = t32;
      w.qs = q32;
      w.derive();
      if (!w.beyond()) {
        cta_slot_sums<DT, false>(w, d, sl, sh);
        // p - q: both rows' weights and both their sums are off; else the row's sum as a whole counts, without what was
        // taken away
        token = cluster_search<DT, false, false>(cl, w, d, sl, v, 0.0, w.kind == kWRest ? 8 * d.eps : 2 * d.eps * t32.z, 0, sh,
                                                 &total, &again);
        if (!is_distribution(total)) again = true;
      }
      if (again) {
        if (w.kind == kWRest) {
          w.ts.z = cluster_exact_sum<DT>(cl, w.t, w.ts.m, d.ct64, d, sl, sh);
          w.qs.z = cluster_exact_sum<DT>(cl, w.q, w.qs.m, d.cd64, d, sl, sh);
          w.derive();
        }
        cta_slot_sums<DT, true>(w, d, sl, sh);
        bool never;
        token = cluster_search<DT, true, false>(cl, w, d, sl, v, 0.0, 0.0, 1, sh, &total, &never);
        cl.sync();
        if (!is_distribution(total)) {  // nothing left
          w.kind = kWPlain;
          continue;
        }
      }
      break;
    }
    if (token >= 0 && threadIdx.x == 0)
      lp = (float)(((double)E::load1(w.t, token) - t32.m) * inv_temperature(d.ct64) - log(t32.z));
  }
  const int64_t at = (int64_t)b * W;
  if (token >= 0 && threadIdx.x == 0) {
    d.tokens[at + j] = token;
    if (d.logprob) d.logprob[at + j] = lp;
    if (d.mask) d.mask[at + j] = 1;
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
  cl.sync();  // nobody leaves while its shared memory is read
}

}  // namespace fopd
