// Norm and clipping of a set of tensors: sum of squares over all of them, then every element
// times min(1, max_norm / norm).  Both are streams over memory; the set's table travels in the
// kernel parameters, so a call needs no device-side table, no copy and no allocation.
#pragma once

#include "common.cuh"

namespace fopd {

constexpr int kClipThreads = 256;
constexpr int kClipTileBytes = 32768;  // a CTA's piece of a row of a tensor
constexpr int kClipVecs = 8;           // 16-byte vectors of a tile per thread, in flight together
constexpr int kClipMaxGrid = 592;      // CTAs that stay, four to an SM; their partial sums fit the workspace
static_assert(kClipTileBytes == kClipThreads * kClipVecs * 16, "a full tile is one round of loads");
constexpr int kClipTicket = 1;         // ws[1]: counter of finished CTAs (left at zero by every launch)
constexpr int kClipPartials = 8;       // ws[8 ..]: partial sums, one per CTA
static_assert(kClipPartials + kClipMaxGrid <= FOPD_GRAD_WS, "the workspace holds the partial sums");

// A tensor in a launch's table: 32 bytes, since handing over a launch's parameters takes the host 0.5 us per KB.  One
// whose rows lie apart takes a second entry.
enum ClipKind : uint8_t { kClipDense = 0, kClipRows = 1, kClipShortRows = 2, kClipMore = 3 };
struct ClipEntry {
  const char *data;
  char *out;
  int64_t cols;    // elements of a row; of the whole tensor where it is dense
  uint32_t tile0;  // first tile of this tensor in the launch
  uint8_t kind;    // kClipRows: each row is cut into tiles; kClipShortRows: a tile is a few whole rows
  uint8_t dtype;
  uint16_t pad;
};
struct ClipMore {  // in the place of the entry behind a tensor with rows
  int64_t rows, row_stride;  // (elements)
  int64_t per;               // tiles of a row, or rows of a tile
  uint32_t tile0;            // the same as its tensor's
  uint8_t kind, dtype;
  uint16_t pad;
};
static_assert(sizeof(ClipEntry) == 32 && sizeof(ClipMore) == 32, "one size");

template <int N>
struct ClipTable {
  int64_t n_tiles;
  int32_t n;
  int32_t in_place;  // every tensor's out is its data
  ClipEntry e[N];
};

// The tensor a tile belongs to: the last one whose first tile is not behind it.
template <int N>
__device__ __forceinline__ int find_entry(const ClipTable<N> &t, uint32_t tile) {
  int lo = 0, hi = t.n - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (t.e[mid].tile0 <= tile) lo = mid;
    else hi = mid - 1;
  }
  return t.e[lo].kind == kClipMore ? lo - 1 : lo;
}

// A tile: n elements in a row from element `off` of the tensor on, or (rows > 0) rows of n elements `stride` apart.
struct ClipTile {
  int64_t off, stride;
  int n, rows;
};
template <int N>
__device__ __forceinline__ ClipTile tile_range(const ClipTable<N> &t, int i, uint32_t tile) {
  const ClipEntry &e = t.e[i];
  const int per = kClipTileBytes / (e.dtype == FOPD_BF16 ? 2 : 4);
  const int64_t local = tile - e.tile0;
  if (e.kind == kClipDense) return {local * per, 0, (int)min((int64_t)per, e.cols - local * per), 0};
  const ClipMore &m = reinterpret_cast<const ClipMore &>(t.e[i + 1]);
  if (e.kind == kClipShortRows) {
    const int64_t row = local * m.per;
    return {row * m.row_stride, m.row_stride, (int)e.cols, (int)min(m.per, m.rows - row)};
  }
  const int64_t row = local / m.per, piece = local % m.per;
  return {row * m.row_stride + piece * per, 0, (int)min((int64_t)per, e.cols - piece * per), 0};
}

// (an ordinary load: what the norm has read last the scaling finds in the L2, and it was faster there too)
__device__ __forceinline__ uint4 ld_keep(const void *p) {
  return *reinterpret_cast<const uint4 *>(p);
}

// Sum of squares of n elements at p, per thread, in fp64 (|g| up to 3e38: its square is out of fp32's range).
template <int DT>
__device__ __forceinline__ double vec_squares(const uint4 &v) {
  constexpr int P = Elem<DT>::kPerVec;
  float x[P];
  Elem<DT>::unpack(v, x);
  double s = 0.0, r = 0.0;
#pragma unroll
  for (int k = 0; k < P; k += 2) {
    s = fma((double)x[k], (double)x[k], s);
    r = fma((double)x[k + 1], (double)x[k + 1], r);
  }
  return s + r;
}
template <int DT>
__device__ __forceinline__ double tile_squares(const char *p, const ClipTile &r) {
  using E = Elem<DT>;
  constexpr int P = E::kPerVec;
  const int n = r.n;
  if (r.rows > 0) {  // rows too short for vectors
    double s = 0.0;
    for (int i = threadIdx.x; i < r.rows * n; i += kClipThreads) {
      const double x = (double)E::load1(p, (i / n) * r.stride + i % n);
      s = fma(x, x, s);
    }
    return s;
  }
  // elements before the first 16-byte boundary, whole vectors, the rest
  int head = (int)(((16 - (reinterpret_cast<uintptr_t>(p) & 15)) & 15) / E::kBytes);
  if (head > n) head = n;
  const int nvec = (n - head) / P;
  const uint4 *v = reinterpret_cast<const uint4 *>(p + (size_t)head * E::kBytes);
  double s = 0.0;
  uint4 a[kClipVecs];
#pragma unroll
  for (int u = 0; u < kClipVecs; ++u) {
    const int i = threadIdx.x + u * kClipThreads;
    a[u] = i < nvec ? ld_keep(v + i) : make_uint4(0, 0, 0, 0);
  }
#pragma unroll
  for (int u = 0; u < kClipVecs; ++u) s += vec_squares<DT>(a[u]);
  const int tail0 = head + nvec * P;
  const int k = (int)threadIdx.x < head ? (int)threadIdx.x : tail0 + ((int)threadIdx.x - head);
  if (k < n) {
    const double x = (double)E::load1(p, k);
    s = fma(x, x, s);
  }
  return s;
}

// grid <= kClipMaxGrid.  The CTAs' partial sums go to the workspace; the last CTA to finish adds them in the order
// of the CTAs.  set != 0: ws[0] = the sum, else ws[0] += it.
template <int N>
__global__ void __launch_bounds__(kClipThreads, 4)
    grad_norm_kernel(const __grid_constant__ ClipTable<N> t, double *ws, int set, float *norm, int32_t *status) {
  __shared__ double sh[kClipThreads];
  __shared__ int last;
  asm volatile("griddepcontrol.launch_dependents;");
  double s = 0.0;
  for (int64_t tile = blockIdx.x; tile < t.n_tiles; tile += gridDim.x) {
    const int i = find_entry(t, (uint32_t)tile);
    const ClipEntry &e = t.e[i];
    const ClipTile r = tile_range(t, i, (uint32_t)tile);
    s += e.dtype == FOPD_BF16 ? tile_squares<FOPD_BF16>(e.data + r.off * 2, r) : tile_squares<FOPD_F32>(e.data + r.off * 4, r);
  }
  sh[threadIdx.x] = s;
  __syncthreads();
  for (int off = kClipThreads / 2; off > 0; off >>= 1) {
    if ((int)threadIdx.x < off) sh[threadIdx.x] += sh[threadIdx.x + off];
    __syncthreads();
  }
  unsigned long long *ticket = reinterpret_cast<unsigned long long *>(ws + kClipTicket);
  if (threadIdx.x == 0) {
    ws[kClipPartials + blockIdx.x] = sh[0];
    __threadfence();
    last = atomicAdd(ticket, 1ull) == gridDim.x - 1;
  }
  __syncthreads();
  if (!last) return;
  __threadfence();
  double v = 0.0;
  for (int i = threadIdx.x; i < (int)gridDim.x; i += kClipThreads) v += __ldcg(ws + kClipPartials + i);
  sh[threadIdx.x] = v;
  __syncthreads();
  for (int off = kClipThreads / 2; off > 0; off >>= 1) {
    if ((int)threadIdx.x < off) sh[threadIdx.x] += sh[threadIdx.x + off];
    __syncthreads();
  }
  if (threadIdx.x == 0) {
    const double total = set ? sh[0] : ws[FOPD_GRAD_WS_SUM] + sh[0];
    ws[FOPD_GRAD_WS_SUM] = total;
    *ticket = 0;
    if (norm) norm[0] = (float)sqrt(total);
    if (status && !(total <= 1.7976931348623157e308)) atomicOr(status, FOPD_DEV_NONFINITE);
  }
}

// coef of a sum of squares (see fopd_grad_scale); 1 where the norm is not finite.
__device__ __forceinline__ double clip_coef(double sum, float max_norm) {
  const double norm = sqrt(sum);
  return norm > (double)max_norm && norm <= 1.7976931348623157e308 ? (double)max_norm / norm : 1.0;
}

// The scaling by a coefficient below fp32's normal numbers, where that has few bits or none: products in fp64, rounded
// once.  Out of line, and element by element: hardly any set comes here.
template <int N>
__device__ __noinline__ void scale_tiny(const ClipTable<N> &t, double c) {
  for (int64_t tile = blockIdx.x; tile < t.n_tiles; tile += gridDim.x) {
    const int k = find_entry(t, (uint32_t)tile);
    const ClipEntry &e = t.e[k];
    const ClipTile r = tile_range(t, k, (uint32_t)tile);
    const int n = (r.rows > 0 ? r.rows : 1) * r.n;
    for (int i = threadIdx.x; i < n; i += kClipThreads) {
      const int64_t at = r.off + (i / r.n) * r.stride + i % r.n;
      if (e.dtype == FOPD_BF16)
        reinterpret_cast<__nv_bfloat16 *>(e.out)[at] = __double2bfloat16((double)Elem<FOPD_BF16>::load1(e.data, at) * c);
      else
        reinterpret_cast<float *>(e.out)[at] = (float)((double)Elem<FOPD_F32>::load1(e.data, at) * c);
    }
  }
}

template <int DT>
__device__ __forceinline__ void tile_scale(const char *p, char *o, const ClipTile &r, float c) {
  using E = Elem<DT>;
  constexpr int P = E::kPerVec;
  const int n = r.n;
  if (r.rows > 0) {
    for (int i = threadIdx.x; i < r.rows * n; i += kClipThreads) {
      const int64_t at = (i / n) * r.stride + i % n;
      E::store1(o, at, E::load1(p, at) * c);
    }
    return;
  }
  if (((reinterpret_cast<uintptr_t>(p) ^ reinterpret_cast<uintptr_t>(o)) & 15) != 0) {  // no common vector boundary
    for (int i = threadIdx.x; i < n; i += kClipThreads) E::store1(o, i, E::load1(p, i) * c);
    return;
  }
  int head = (int)(((16 - (reinterpret_cast<uintptr_t>(p) & 15)) & 15) / E::kBytes);
  if (head > n) head = n;
  const int nvec = (n - head) / P;
  const uint4 *v = reinterpret_cast<const uint4 *>(p + (size_t)head * E::kBytes);
  uint4 *w = reinterpret_cast<uint4 *>(o + (size_t)head * E::kBytes);
  uint4 a[kClipVecs];
#pragma unroll
  for (int u = 0; u < kClipVecs; ++u) {
    const int i = threadIdx.x + u * kClipThreads;
    if (i < nvec) a[u] = ld_keep(v + i);
  }
#pragma unroll
  for (int u = 0; u < kClipVecs; ++u) {
    const int i = threadIdx.x + u * kClipThreads;
    if (i < nvec) {
      float x[P];
      E::unpack(a[u], x);
#pragma unroll
      for (int k = 0; k < P; ++k) x[k] *= c;
      st_stream(w + i, E::pack(x));
    }
  }
  const int tail0 = head + nvec * P;
  const int k = (int)threadIdx.x < head ? (int)threadIdx.x : tail0 + ((int)threadIdx.x - head);
  if (k < n) E::store1(o, k, E::load1(p, k) * c);
}

template <int N>
__global__ void __launch_bounds__(kClipThreads, 4)
    grad_scale_kernel(const __grid_constant__ ClipTable<N> t, const double *ws, float max_norm, float *norm,
                      float *coef, int32_t *status) {
  asm volatile("griddepcontrol.wait;" ::: "memory");  // the norm kernel's sum (launched early behind it)
  const double sum = ws[FOPD_GRAD_WS_SUM];
  const float c = (float)clip_coef(sum, max_norm);
  if (blockIdx.x == 0 && threadIdx.x == 0) {
    if (norm) norm[0] = (float)sqrt(sum);
    if (coef) coef[0] = c;
    if (status && !(sum <= 1.7976931348623157e308)) atomicOr(status, FOPD_DEV_NONFINITE);
  }
  if (c == 1.f && t.in_place) return;
  if (c < 0x1p-126f) {
    scale_tiny(t, clip_coef(sum, max_norm));
    return;
  }
  // from the end: what the norm has read last may still be in the L2
  for (int64_t tile = t.n_tiles - 1 - blockIdx.x; tile >= 0; tile -= gridDim.x) {
    const int i = find_entry(t, (uint32_t)tile);
    const ClipEntry &e = t.e[i];
    if (c == 1.f && e.out == e.data) continue;
    const ClipTile r = tile_range(t, i, (uint32_t)tile);
    if (e.dtype == FOPD_BF16) tile_scale<FOPD_BF16>(e.data + r.off * 2, e.out + r.off * 2, r, c);
    else tile_scale<FOPD_F32>(e.data + r.off * 4, e.out + r.off * 4, r, c);
  }
}

}  // namespace fopd
