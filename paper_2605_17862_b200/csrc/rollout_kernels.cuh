// Drawing tokens from rows of logits and verifying drafted tokens (fopd_draw_tokens,
// fopd_verify_draft; a draw is a verification without drafts).
//
// Two kernels.  rollout_tiles_kernel sweeps every row that may be needed: a warp takes a tile of a
// row and leaves the tile's maximum and sum of exponentials.  rollout_finish_kernel, one CTA per
// sequence, merges the tiles of each position, finds the first draft that is not accepted and draws
// the new token by a search over tile sums and then inside one tile.
//
// Which token comes out has to be that of exact arithmetic, and a running sum over 150,000
// probabilities in fp32 is off by more than many of them.  So the fp32 results come with a bound, and
// a decision that lies within it is made again in fp64.
#pragma once

#include "common.cuh"

namespace fopd {

constexpr int kTileWarps = 8;       // warps of a CTA of the tile sweep, one tile each
constexpr int kTileVecs = 8;        // 16-byte vectors of a tile per lane
constexpr int kFinishThreads = 512;
constexpr int kFinishWarps = kFinishThreads / 32;

// Error of the fp32 sums, relative to a row's whole sum.  An exponent (x - max) log2(e)/T is three roundings,
// |y| 2^-22.4, off, so e^y by up to 24 * 1.3e-7 = 3.1e-6 where y > -24 (what lies below weighs 2^-24 each); ex2 adds
// 2^-22, a lane's sum of 64 terms and the warp's five levels 69 * 2^-24 = 4.1e-6.  Both v * total and a running sum
// carry it: 2 * 7.5e-6 < 2^-15.  For p - q both rows do.
constexpr double kSumBound = 1.0 / (1 << 15);
// Error of u q against p, relative to the larger: two sums of 7.5e-6 and two exponentials in fp64.
constexpr double kTestBound = 1.0 / (1 << 15);

enum DraftKind { kDraftNone = 0, kDraftCertain = 1, kDraftRows = 2, kDraftBest = 3 };
enum PosState { kAccept = 0, kReject = 1, kOpen = 2, kBadRow = 3, kBadUniform = 4, kEnd = 5, kBadToken = 6 };

struct RolloutDev {
  const char *target, *draft;
  const int32_t *drafted, *n_draft;
  const double *uniform;
  int64_t vocab, n_tiles;
  int64_t tseq, trow, dseq, drow;  // bytes
  int32_t B, K;
  int kind;        // DraftKind
  int best;        // the target's temperature is 0
  float ct, cd;    // log2(e) / temperature, fp32
  double it, id;   // 1 / temperature
  float2 *part;    // [B (K + 1) + B K, n_tiles]: {max, sum}, or {max, index} for a row of which only the best is wanted
  double *tsum;    // [B, n_tiles]
  struct Position *pos;  // [B, K + 1]
};

struct Position {
  float m;       // maximum of the target's row
  int32_t state;
  double z;      // sum of exponentials behind it
  float lp;      // log p of the drafted token
  int32_t best;
};

template <int DT>
struct TileShape {
  static constexpr int kElems = 32 * kTileVecs * Elem<DT>::kPerVec;
};

// Vector i of a row; what lies behind the vocabulary reads as -infinity.
template <int DT>
__device__ __forceinline__ uint4 row_vec(const char *row, int64_t i, int64_t V) {
  using E = Elem<DT>;
  constexpr int P = E::kPerVec;
  const int64_t left = V - i * P;
  if (left >= P) return ld_stream(reinterpret_cast<const uint4 *>(row) + i);
  float x[P];
#pragma unroll
  for (int k = 0; k < P; ++k) x[k] = k < left ? E::load1(row, i * P + k) : -INFINITY;
  return E::pack(x);
}

__device__ __forceinline__ float warp_max(float x) {
  float r;
  asm volatile("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(x));
  return r;
}
template <class T>
__device__ __forceinline__ T warp_sum(T x) {
#pragma unroll
  for (int off = 16; off > 0; off >>= 1) x += __shfl_xor_sync(0xffffffffu, x, off);
  return x;
}

// {max, sum e^{(x - max) / T}} of one tile, in every lane.  A tile of -infinity gives {-inf, 0}; a NaN or +inf makes the
// sum NaN.
template <int DT>
__device__ __forceinline__ float2 tile_sum(const char *row, int64_t tile, int64_t V, float c) {
  using E = Elem<DT>;
  constexpr int P = E::kPerVec;
  const int lane = threadIdx.x & 31;
  uint4 raw[kTileVecs];
#pragma unroll
  for (int v = 0; v < kTileVecs; ++v) raw[v] = row_vec<DT>(row, (tile * kTileVecs + v) * 32 + lane, V);
  float m = -INFINITY;
#pragma unroll
  for (int v = 0; v < kTileVecs; ++v) {
    float x[P];
    E::unpack(raw[v], x);
    m = fmaxf(m, max_of<P>(x));
  }
  m = warp_max(m);
  const float ref = m == -INFINITY ? 0.f : m;
  float z = 0.f;
#pragma unroll
  for (int v = 0; v < kTileVecs; ++v) {
    float x[P];
    E::unpack(raw[v], x);
#pragma unroll
    for (int k = 0; k < P; ++k) z += ex2((x[k] - ref) * c);
  }
  return make_float2(m, warp_sum(z));
}

// {max, lowest index of it} of one tile, in every lane; NaN anywhere gives {NaN, -1}.
template <int DT>
__device__ __forceinline__ float2 tile_best(const char *row, int64_t tile, int64_t V) {
  using E = Elem<DT>;
  constexpr int P = E::kPerVec;
  const int lane = threadIdx.x & 31;
  float m = -INFINITY;
  int32_t at = INT32_MAX;
  bool nan = false;
  for (int v = 0; v < kTileVecs; ++v) {
    const int64_t i = (tile * kTileVecs + v) * 32 + lane;
    float x[P];
    E::unpack(row_vec<DT>(row, i, V), x);
    for (int k = 0; k < P; ++k) {
      nan |= isnan(x[k]);
      if (x[k] > m) {
        m = x[k];
        at = (int32_t)(i * P + k);
      }
    }
  }
  nan = __any_sync(0xffffffffu, nan);
  const float top = warp_max(m);
  at = m == top ? at : INT32_MAX;
  at = __reduce_min_sync(0xffffffffu, at);
  return nan ? make_float2(NAN, __int_as_float(-1)) : make_float2(top, __int_as_float(at));
}

__device__ __forceinline__ int32_t drafts_of(const RolloutDev &d, int32_t b) {
  if (d.K == 0) return 0;
  const int32_t n = d.n_draft ? d.n_draft[b] : d.K;
  return n < 0 ? 0 : n > d.K ? d.K : n;
}

// Tile sweep: items are (row, group of kTileWarps tiles), target rows first.
template <int DT>
__global__ void __launch_bounds__(kTileWarps * 32) rollout_tiles_kernel(RolloutDev d, int64_t n_items) {
  const int64_t groups = (d.n_tiles + kTileWarps - 1) / kTileWarps;
  const int64_t n_target = (int64_t)d.B * (d.K + 1);
  for (int64_t item = blockIdx.x; item < n_items; item += gridDim.x) {
    const int64_t r = item / groups, tile = (item % groups) * kTileWarps + (threadIdx.x >> 5);
    if (tile >= d.n_tiles) continue;
    const char *row;
    bool best;
    float c;
    if (r < n_target) {
      const int32_t b = (int32_t)(r / (d.K + 1)), j = (int32_t)(r % (d.K + 1));
      if (j > drafts_of(d, b)) continue;
      row = d.target + b * d.tseq + j * d.trow;
      best = d.best;
      c = d.ct;
    } else {
      const int32_t b = (int32_t)((r - n_target) / d.K), j = (int32_t)((r - n_target) % d.K);
      if (j >= drafts_of(d, b)) continue;
      row = d.draft + b * d.dseq + j * d.drow;
      best = d.kind == kDraftBest;
      c = d.cd;
    }
    const float2 p = best ? tile_best<DT>(row, tile, d.vocab) : tile_sum<DT>(row, tile, d.vocab, c);
    if ((threadIdx.x & 31) == 0) d.part[r * d.n_tiles + tile] = p;
  }
}

// ---- a CTA's tools ----------------------------------------------------------------------------------

// Inclusive scan of one value per thread; every thread also gets all of them through sh[].
__device__ __forceinline__ void block_scan(double x, double *sh) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  __shared__ double tot[kFinishWarps];
#pragma unroll
  for (int off = 1; off < 32; off <<= 1) {
    const double y = __shfl_up_sync(0xffffffffu, x, off);
    if (lane >= off) x += y;
  }
  __syncthreads();  // sh and tot are free again
  if (lane == 31) tot[warp] = x;
  __syncthreads();
  double before = 0.0;
  for (int w = 0; w < warp; ++w) before += tot[w];
  sh[threadIdx.x] = before + x;
  __syncthreads();
}

__device__ __forceinline__ double block_sum(double x, double *sh) {
  block_scan(x, sh);
  return sh[kFinishThreads - 1];
}

// Weights of the distribution a token is drawn from, element by element.  fp32: with a row's rounded sums; fp64: exact.
enum WeightKind { kWPlain = 0, kWWithout = 1, kWRest = 2 };
template <int DT>
struct Weights {
  const char *t, *q;  // rows
  int kind;           // WeightKind
  int32_t without;    // kWWithout: the element of which everything is taken away
  float ct, cd, mt, mq;
  double it, id, zt, zq;  // 1 / T and the sums (fp32's or fp64's own)
  __device__ __forceinline__ double fast(int64_t i) const {
    const float p = ex2((Elem<DT>::load1(t, i) - mt) * ct);
    if (kind == kWRest) {
      const double r = p / zt - ex2((Elem<DT>::load1(q, i) - mq) * cd) / zq;
      return r > 0.0 ? r : 0.0;
    }
    return kind == kWWithout && i == without ? 0.0 : (double)p;
  }
  __device__ __forceinline__ double exact(int64_t i) const {
    const double p = exp(((double)Elem<DT>::load1(t, i) - mt) * it);
    if (kind == kWRest) {
      const double r = p / zt - exp(((double)Elem<DT>::load1(q, i) - mq) * id) / zq;
      return r > 0.0 ? r : 0.0;
    }
    return kind == kWWithout && i == without ? 0.0 : p;
  }
  template <bool kExact>
  __device__ __forceinline__ double at(int64_t i) const {
    return kExact ? exact(i) : fast(i);
  }
};

template <int DT>
__device__ double block_exact_sum(const char *row, float m, double it, int64_t V, double *sh) {
  double s = 0.0;
  for (int64_t i = threadIdx.x; i < V; i += kFinishThreads) s += exp(((double)Elem<DT>::load1(row, i) - m) * it);
  return block_sum(s, sh);
}

template <int DT, bool kExact>
__device__ void block_tile_sums(const Weights<DT> &w, int64_t V, int64_t n_tiles, double *tsum) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  for (int64_t t = warp; t < n_tiles; t += kFinishWarps) {
    double s = 0.0;
    const int64_t lo = t * TileShape<DT>::kElems, hi = min(V, lo + TileShape<DT>::kElems);
    for (int64_t i = lo + lane; i < hi; i += 32) s += w.template at<kExact>(i);
    s = warp_sum(s);
    if (lane == 0) tsum[t] = s;
  }
  __syncthreads();
}

constexpr int32_t kNobody = -1;  // no weight at all
constexpr int32_t kUnsure = -2;  // within the bound

// The first element whose running sum passes v times the total.  bound: absolute error of the sums (0: none).
template <int DT, bool kExact>
__device__ int32_t block_search(const Weights<DT> &w, int64_t V, int64_t n_tiles, const double *tsum, double v,
                                double bound, double *sh) {
  __shared__ int first, last;
  __shared__ int64_t found_tile;
  __shared__ double found_before;
  __shared__ int32_t result;
  // the tile
  const int64_t per = (n_tiles + kFinishThreads - 1) / kFinishThreads;
  const int64_t lo = threadIdx.x * per, hi = min(n_tiles, lo + per);
  double s = 0.0;
  for (int64_t t = lo; t < hi; ++t) s += tsum[t];
  block_scan(s, sh);
  const double total = sh[kFinishThreads - 1];
  if (!(total > 0.0)) return bound > 0.0 ? kUnsure : kNobody;
  const double goal = v * total;
  if (threadIdx.x == 0) {
    first = kFinishThreads;
    last = 0;
    result = kUnsure;
  }
  __syncthreads();
  if (s > 0.0) {
    atomicMax(&last, (int)threadIdx.x);
    if (sh[threadIdx.x] > goal) atomicMin(&first, (int)threadIdx.x);
  }
  __syncthreads();
  const int own = first < kFinishThreads ? first : last;
  if ((int)threadIdx.x == own) {
    double before = own ? sh[own - 1] : 0.0;
    int64_t at = lo, t = lo;
    double at_before = before;
    for (; t < hi; ++t) {
      if (tsum[t] > 0.0) {
        at = t;
        at_before = before;
        if (before + tsum[t] > goal) break;
      }
      before += tsum[t];
    }
    found_tile = at;
    found_before = at_before;
  }
  __syncthreads();
  // the element
  constexpr int kEach = TileShape<DT>::kElems / kFinishThreads;
  static_assert(kEach * kFinishThreads == TileShape<DT>::kElems, "a tile divides among the threads");
  const int64_t base = found_tile * TileShape<DT>::kElems + threadIdx.x * kEach;
  const double start = found_before;
  double x[kEach];
  s = 0.0;
#pragma unroll
  for (int k = 0; k < kEach; ++k) {
    x[k] = base + k < V ? w.template at<kExact>(base + k) : 0.0;
    s += x[k];
  }
  block_scan(s, sh);
  if (threadIdx.x == 0) {
    first = kFinishThreads;
    last = 0;
  }
  __syncthreads();
  if (s > 0.0) {
    atomicMax(&last, (int)threadIdx.x);
    if (start + sh[threadIdx.x] > goal) atomicMin(&first, (int)threadIdx.x);
  }
  __syncthreads();
  if ((int)threadIdx.x == (first < kFinishThreads ? first : last)) {
    double before = start + (threadIdx.x ? sh[threadIdx.x - 1] : 0.0);
    int32_t at = kUnsure;
    double at_before = before, at_after = before;
#pragma unroll
    for (int k = 0; k < kEach; ++k) {
      if (x[k] > 0.0 && (at < 0 || at_after <= goal)) {
        at = (int32_t)(base + k);
        at_before = before;
        at_after = before + x[k];
      }
      before += x[k];
    }
    const bool sure = !(bound > 0.0) || (goal - at_before > bound && at_after - goal > bound);
    result = sure ? at : kUnsure;
  }
  __syncthreads();
  return result;
}

// {max, sum} of a row from its tiles, in every lane; m is NaN or infinite, or z is NaN, for a row without a
// distribution.
__device__ __forceinline__ void merge_tiles(const float2 *part, int64_t n_tiles, float c, float &m, double &z) {
  const int lane = threadIdx.x & 31;
  m = -INFINITY;
  for (int64_t t = lane; t < n_tiles; t += 32) m = fmaxf(m, part[t].x);
  m = warp_max(m);
  z = 0.0;
  for (int64_t t = lane; t < n_tiles; t += 32) z += (double)(part[t].y * ex2((part[t].x - m) * c));
  z = warp_sum(z);
}
__device__ __forceinline__ void merge_best(const float2 *part, int64_t n_tiles, float &m, int32_t &at) {
  const int lane = threadIdx.x & 31;
  m = -INFINITY;
  at = INT32_MAX;
  bool nan = false;
  for (int64_t t = lane; t < n_tiles; t += 32) {
    nan |= isnan(part[t].x);
    if (part[t].x > m) {
      m = part[t].x;
      at = __float_as_int(part[t].y);
    }
  }
  const float top = warp_max(m);
  at = m == top ? at : INT32_MAX;
  at = __reduce_min_sync(0xffffffffu, at);
  m = __any_sync(0xffffffffu, nan) ? NAN : top;
}
__device__ __forceinline__ bool is_distribution(float m, double z) {
  return m > -INFINITY && m < INFINITY && z > 0.0 && z < INFINITY;
}

// One position of one sequence, by a warp.
template <int DT>
__device__ __forceinline__ void judge(const RolloutDev &d, int32_t b, int32_t j, int32_t n) {
  using E = Elem<DT>;
  Position &out = d.pos[(int64_t)b * (d.K + 1) + j];
  const float2 *part = d.part + ((int64_t)b * (d.K + 1) + j) * d.n_tiles;
  const char *row = d.target + b * d.tseq + j * d.trow;
  float m;
  double z = 1.0;
  int32_t best = 0;
  if (d.best) merge_best(part, d.n_tiles, m, best);
  else merge_tiles(part, d.n_tiles, d.ct, m, z);
  int state = is_distribution(m, z) ? kEnd : kBadRow;
  float lp = 0.f;
  if (state == kEnd && j < n) {
    const int64_t at = (int64_t)b * d.K + j;
    const int32_t x = d.drafted[at];
    const double u = d.uniform[(int64_t)b * (d.K + 1) + j];
    if (x < 0 || x >= d.vocab) state = kBadToken;
    else if (d.best) state = x == best ? kAccept : kReject;
    else if (!(u >= 0.0 && u < 1.0)) state = kBadUniform;
    else {
      const double y = ((double)E::load1(row, x) - m) * d.it;
      const double p = exp(y) / z;
      lp = (float)(y - log(z));
      double q = 1.0;
      const float2 *qpart = d.part + ((int64_t)d.B * (d.K + 1) + at) * d.n_tiles;
      if (d.kind == kDraftRows) {
        float mq;
        double zq;
        merge_tiles(qpart, d.n_tiles, d.cd, mq, zq);
        q = exp(((double)E::load1(d.draft + b * d.dseq + j * d.drow, x) - mq) * d.id) / zq;
        if (!is_distribution(mq, zq)) state = kBadRow;
      } else if (d.kind == kDraftBest) {
        float mq;
        int32_t bq;
        merge_best(qpart, d.n_tiles, mq, bq);
        q = x == bq ? 1.0 : 0.0;
        if (!is_distribution(mq, 1.0)) state = kBadRow;
      }
      if (state == kEnd) {
        const double uq = u * q;
        state = fabs(uq - p) < kTestBound * fmax(uq, p) ? kOpen : uq < p ? kAccept : kReject;
      }
    }
  }
  if ((threadIdx.x & 31) == 0) {
    out.m = m;
    out.z = z;
    out.state = state;
    out.lp = lp;
    out.best = best;
  }
}

template <int DT>
__global__ void __launch_bounds__(kFinishThreads)
    rollout_finish_kernel(RolloutDev d, int32_t *tokens, float *logprob, uint8_t *mask, int32_t *n_accepted,
                          int32_t *status) {
  using E = Elem<DT>;
  __shared__ double sh[kFinishThreads];
  __shared__ int stop;
  const int32_t b = blockIdx.x;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int32_t n = drafts_of(d, b), W = d.K + 1;
  int bits = d.n_draft && d.K > 0 && d.n_draft[b] != n ? FOPD_DEV_BAD_LENGTH : 0;
  Position *pos = d.pos + (int64_t)b * W;
  for (int32_t j = warp; j <= n; j += kFinishWarps) judge<DT>(d, b, j, n);
  __syncthreads();

  // the first position that is not accepted; an open one is settled in fp64
  int32_t from = 0, j;
  for (;;) {
    if (threadIdx.x == 0) stop = n;
    __syncthreads();
    for (int32_t k = from + threadIdx.x; k < n; k += kFinishThreads)
      if (pos[k].state != kAccept) {
        atomicMin(&stop, k);
        break;
      }
    __syncthreads();
    j = stop;
    __syncthreads();
    if (pos[j].state != kOpen) break;
    const int64_t at = (int64_t)b * d.K + j;
    const int32_t x = d.drafted[at];
    const char *row = d.target + b * d.tseq + j * d.trow;
    const double p =
        exp(((double)E::load1(row, x) - pos[j].m) * d.it) / block_exact_sum<DT>(row, pos[j].m, d.it, d.vocab, sh);
    double q = 1.0;
    if (d.kind == kDraftRows) {
      const char *qrow = d.draft + b * d.dseq + j * d.drow;
      float mq;
      double zq;
      merge_tiles(d.part + ((int64_t)d.B * W + at) * d.n_tiles, d.n_tiles, d.cd, mq, zq);
      q = exp(((double)E::load1(qrow, x) - mq) * d.id) / block_exact_sum<DT>(qrow, mq, d.id, d.vocab, sh);
    }  // (kDraftBest: q = 1, or 0 and never open)
    const bool ok = d.uniform[(int64_t)b * W + j] * q < p;
    __syncthreads();
    if (threadIdx.x == 0) pos[j].state = ok ? kAccept : kReject;
    __syncthreads();
    from = j;
  }

  // the new token
  const int state = pos[j].state;
  int32_t token = -1;
  float lp = 0.f;
  const double v = d.uniform[(int64_t)b * W + d.K];
  if (state == kBadRow) bits |= FOPD_DEV_BAD_LOGITS;
  else if (state == kBadUniform) bits |= FOPD_DEV_BAD_UNIFORM;
  else {
    if (state == kBadToken) bits |= FOPD_DEV_BAD_TOKEN;
    if (d.best) token = pos[j].best;
    else if (!(v >= 0.0 && v < 1.0)) bits |= FOPD_DEV_BAD_UNIFORM;
    else {
      Weights<DT> w;
      w.t = d.target + b * d.tseq + j * d.trow;
      w.q = nullptr;
      w.kind = kWPlain;
      w.without = -1;
      w.ct = d.ct;
      w.cd = d.cd;
      w.it = d.it;
      w.id = d.id;
      w.mt = pos[j].m;
      w.zt = pos[j].z;
      w.mq = 0.f;
      w.zq = 1.0;
      const float2 *part = d.part + ((int64_t)b * W + j) * d.n_tiles;
      double *tsum = d.tsum + b * d.n_tiles;
      if (j < n) {  // rejected
        const int64_t at = (int64_t)b * d.K + j;
        const float2 *qpart = d.part + ((int64_t)d.B * W + at) * d.n_tiles;
        if (d.kind == kDraftCertain) {
          w.kind = kWWithout;
          w.without = d.drafted[at];
        } else if (d.kind == kDraftBest) {
          float mq;
          w.kind = kWWithout;
          merge_best(qpart, d.n_tiles, mq, w.without);
          if (!is_distribution(mq, 1.0)) bits |= FOPD_DEV_BAD_LOGITS;  // (a bad token hid it)
        } else if (d.kind == kDraftRows) {
          w.kind = kWRest;
          w.q = d.draft + b * d.dseq + j * d.drow;
          merge_tiles(qpart, d.n_tiles, d.cd, w.mq, w.zq);
          if (!is_distribution(w.mq, w.zq)) bits |= FOPD_DEV_BAD_LOGITS;
        }
      }
      if (!(bits & FOPD_DEV_BAD_LOGITS)) {
        const double z32 = w.zt, zq32 = w.zq;
        for (int round = 0; round < 2; ++round) {  // the second one only where p - q is zero everywhere
          double bound;
          w.zt = z32;
          w.zq = zq32;
          if (w.kind == kWRest) {
            block_tile_sums<DT, false>(w, d.vocab, d.n_tiles, tsum);
            bound = 2 * kSumBound;
          } else {
            for (int64_t t = threadIdx.x; t < d.n_tiles; t += kFinishThreads) {
              double s = (double)(part[t].y * ex2((part[t].x - w.mt) * w.ct));
              if (w.kind == kWWithout && w.without / TileShape<DT>::kElems == t && w.without >= 0)
                s = fmax(0.0, s - (double)ex2((E::load1(w.t, w.without) - w.mt) * w.ct));
              tsum[t] = s;
            }
            bound = kSumBound * z32;
            __syncthreads();
          }
          token = block_search<DT, false>(w, d.vocab, d.n_tiles, tsum, v, bound, sh);
          if (token == kUnsure) {
            __syncthreads();
            if (w.kind == kWRest) {
              w.zt = block_exact_sum<DT>(w.t, w.mt, w.it, d.vocab, sh);
              w.zq = block_exact_sum<DT>(w.q, w.mq, w.id, d.vocab, sh);
            }
            block_tile_sums<DT, true>(w, d.vocab, d.n_tiles, tsum);
            token = block_search<DT, true>(w, d.vocab, d.n_tiles, tsum, v, 0.0, sh);
          }
          if (token != kNobody) break;
          w.kind = kWPlain;
          __syncthreads();
        }
        lp = (float)(((double)E::load1(w.t, token) - w.mt) * w.it - log(z32));
      }
    }
  }
  if (bits && threadIdx.x == 0 && status) atomicOr(status, bits);
  for (int32_t k = threadIdx.x; k < W; k += kFinishThreads) {
    const int64_t at = (int64_t)b * W + k;
    const bool there = k < j || (k == j && token >= 0);
    tokens[at] = k < j ? d.drafted[(int64_t)b * d.K + k] : k == j ? token : -1;
    if (logprob) logprob[at] = k < j ? pos[k].lp : k == j && token >= 0 ? lp : 0.f;
    if (mask) mask[at] = there ? 1 : 0;
  }
  if (n_accepted && threadIdx.x == 0) n_accepted[b] = j;
}

}  // namespace fopd
