// Gradient norm and clipping: argument checks, the set's table, launches.
#include <vector>

#include "clip_kernels.cuh"
#include "host_common.cuh"
#include "host_ranges.cuh"

using namespace fopd;

namespace {

// Tensors of one launch: the table is a kernel parameter (at most 32,764 bytes), in sizes so that small sets are quick to
// hand over.
constexpr int kLargestTable = 1000;

int check_tensors(const fopd_tensor *t, int32_t n, const double *ws) {
  if (n < 0) return FOPD_ERR_SIZE;
  if (!ws || (n > 0 && !t)) return FOPD_ERR_NULL;
  if (!aligned16(ws)) return FOPD_ERR_ALIGN;
  for (int32_t i = 0; i < n; ++i) {
    if (t[i].dtype != FOPD_BF16 && t[i].dtype != FOPD_F32) return FOPD_ERR_DTYPE;
    const int64_t most = (int64_t)1 << 42, esz = t[i].dtype == FOPD_BF16 ? 2 : 4;
    if (t[i].rows < 0 || t[i].cols < 0 || t[i].rows > most || t[i].cols > most) return FOPD_ERR_SIZE;
    if (t[i].rows == 0 || t[i].cols == 0) continue;
    if (t[i].rows > 1 && (t[i].row_stride < t[i].cols || t[i].row_stride > most / t[i].rows)) return FOPD_ERR_SIZE;
    if (!t[i].data) return FOPD_ERR_NULL;
    if ((uintptr_t)t[i].data % esz != 0 || (uintptr_t)t[i].out % esz != 0) return FOPD_ERR_ALIGN;
  }
  return FOPD_OK;
}

// Whether a written range meets another one (its own tensor's data exactly in place excepted).
int check_overlap(const fopd_tensor *t, int32_t n) {
  std::vector<Range> in, out;
  in.reserve(n);
  for (int32_t i = 0; i < n; ++i) {
    if (t[i].rows == 0 || t[i].cols == 0) continue;
    const uintptr_t esz = t[i].dtype == FOPD_BF16 ? 2 : 4;
    const bool in_place = !t[i].out || t[i].out == t[i].data;
    in.push_back(range_of(t[i].data, t[i].rows, t[i].cols, t[i].row_stride, esz, i, in_place));
    if (!in_place) out.push_back(range_of(t[i].out, t[i].rows, t[i].cols, t[i].row_stride, esz, i, true));
  }
  return check_ranges(in, out);
}

// Fills a launch's table from tensors [*next, n) as far as they go; empty ones are left out.
template <int N>
void fill_table(const fopd_tensor *t, int32_t n, int32_t *next, ClipTable<N> *tab) {
  tab->n = 0;
  tab->n_tiles = 0;
  tab->in_place = 1;
  for (; *next < n; ++*next) {
    const fopd_tensor &x = t[*next];
    if (x.rows == 0 || x.cols == 0) continue;
    const bool dense = x.rows == 1 || x.row_stride == x.cols;
    if (tab->n + (dense ? 1 : 2) > N || tab->n_tiles > (int64_t)1 << 30) return;  // (one tensor has at most 2^30 tiles)
    ClipEntry &e = tab->e[tab->n++];
    const int esz = x.dtype == FOPD_BF16 ? 2 : 4, per = kClipTileBytes / esz;
    e.data = static_cast<const char *>(x.data);
    e.out = static_cast<char *>(x.out ? x.out : const_cast<void *>(x.data));
    e.cols = dense ? x.rows * x.cols : x.cols;
    e.tile0 = (uint32_t)tab->n_tiles;
    e.dtype = (uint8_t)x.dtype;
    e.pad = 0;
    if (e.out != e.data) tab->in_place = 0;
    if (dense) {
      e.kind = kClipDense;
      tab->n_tiles += (e.cols + per - 1) / per;
      continue;
    }
    ClipMore &m = reinterpret_cast<ClipMore &>(tab->e[tab->n++]);
    m.rows = x.rows;
    m.row_stride = x.row_stride;
    m.tile0 = e.tile0;
    m.kind = kClipMore;
    m.dtype = e.dtype;
    m.pad = 0;
    if (x.cols * 8 <= per) {  // eight rows and more in a tile
      e.kind = kClipShortRows;
      m.per = per / x.cols;
      tab->n_tiles += (x.rows + m.per - 1) / m.per;
    } else {
      e.kind = kClipRows;
      m.per = (x.cols + per - 1) / per;
      tab->n_tiles += x.rows * m.per;
    }
  }
}

unsigned clip_grid(int64_t n_tiles) {
  return (unsigned)(n_tiles < 1 ? 1 : n_tiles < kClipMaxGrid ? n_tiles : kClipMaxGrid);
}

template <int N>
int launch_norm_table(const ClipTable<N> &tab, double *ws, int set, float *norm, int32_t *status, cudaStream_t st) {
  grad_norm_kernel<N><<<clip_grid(tab.n_tiles), kClipThreads, 0, st>>>(tab, ws, set, norm, status);
  return launch_ok();
}
template <int N>
int launch_norm(const fopd_tensor *t, int32_t n, double *ws, int set, float *norm, int32_t *status, cudaStream_t st) {
  ClipTable<N> tab;
  int32_t next = 0;
  do {
    fill_table<N>(t, n, &next, &tab);
    const int rc = launch_norm_table<N>(tab, ws, set, norm, status, st);
    if (rc != FOPD_OK) return rc;
    set = 0;
  } while (next < n);
  return FOPD_OK;
}

// early: set up while the norm kernel before it is still running (it waits for it itself).
template <int N>
int launch_scale_table(const ClipTable<N> &tab, const double *ws, float max_norm, float *norm, float *coef,
                       int32_t *status, cudaStream_t st, bool early) {
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(clip_grid(tab.n_tiles));
  cfg.blockDim = dim3(kClipThreads);
  cfg.stream = st;
  cfg.attrs = attr;
  cfg.numAttrs = early ? 1 : 0;
  if (cudaLaunchKernelEx(&cfg, grad_scale_kernel<N>, tab, ws, max_norm, norm, coef, status) != cudaSuccess) {
    (void)cudaGetLastError();
    return FOPD_ERR_CUDA;
  }
  return FOPD_OK;
}
template <int N>
int launch_scale(const fopd_tensor *t, int32_t n, const double *ws, float max_norm, float *norm, float *coef,
                 int32_t *status, cudaStream_t st) {
  ClipTable<N> tab;
  int32_t next = 0;
  do {
    fill_table<N>(t, n, &next, &tab);
    const int rc = launch_scale_table<N>(tab, ws, max_norm, norm, coef, status, st, false);
    if (rc != FOPD_OK) return rc;
  } while (next < n);
  return FOPD_OK;
}

template <int N>
int launch_both(const fopd_tensor *t, int32_t n, double *ws, float max_norm, float *norm, float *coef, int32_t *status,
                cudaStream_t st) {
  ClipTable<N> tab;
  int32_t next = 0;
  fill_table<N>(t, n, &next, &tab);
  if (next == n) {  // all in one table
    const int rc = launch_norm_table<N>(tab, ws, 1, nullptr, nullptr, st);
    return rc != FOPD_OK ? rc : launch_scale_table<N>(tab, ws, max_norm, norm, coef, status, st, true);
  }
  const int rc = launch_norm<N>(t, n, ws, 1, nullptr, nullptr, st);
  return rc != FOPD_OK ? rc : launch_scale<N>(t, n, ws, max_norm, norm, coef, status, st);
}

// The smallest table for n tensors (most of which are dense).
#define FOPD_CLIP_TABLE(n, CALL)          \
  ((n) <= 16    ? CALL(16)                 \
   : (n) <= 48  ? CALL(48)                 \
   : (n) <= 112 ? CALL(112)                \
   : (n) <= 256 ? CALL(256)                \
                : CALL(kLargestTable))

int check_scale(const fopd_tensor *t, int32_t n, const double *ws, float max_norm) {
  const int rc = check_tensors(t, n, ws);
  if (rc != FOPD_OK) return rc;
  if (!std::isfinite(max_norm) || !(max_norm > 0.f)) return FOPD_ERR_PARAM;
  try {
    return check_overlap(t, n);
  } catch (...) {  // host memory for the ranges
    return FOPD_ERR_CUDA;
  }
}

}  // namespace

extern "C" {

int fopd_grad_norm(const fopd_tensor *tensors, int32_t n_tensors, double *ws, float *norm, int32_t *status,
                   void *stream) {
  const int rc = check_tensors(tensors, n_tensors, ws);
  if (rc != FOPD_OK) return rc;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
#define CALL(N) launch_norm<N>(tensors, n_tensors, ws, 0, norm, status, st)
  return FOPD_CLIP_TABLE(n_tensors, CALL);
#undef CALL
}

int fopd_grad_scale(const fopd_tensor *tensors, int32_t n_tensors, double *ws, float max_norm, float *norm,
                    float *coef, int32_t *status, void *stream) {
  const int rc = check_scale(tensors, n_tensors, ws, max_norm);
  if (rc != FOPD_OK) return rc;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
#define CALL(N) launch_scale<N>(tensors, n_tensors, ws, max_norm, norm, coef, status, st)
  return FOPD_CLIP_TABLE(n_tensors, CALL);
#undef CALL
}

int fopd_grad_clip(const fopd_tensor *tensors, int32_t n_tensors, double *ws, float max_norm, float *norm,
                   float *coef, int32_t *status, void *stream) {
  const int rc = check_scale(tensors, n_tensors, ws, max_norm);
  if (rc != FOPD_OK) return rc;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
#define CALL(N) launch_both<N>(tensors, n_tensors, ws, max_norm, norm, coef, status, st)
  return FOPD_CLIP_TABLE(n_tensors, CALL);
#undef CALL
}

}  // extern "C"
