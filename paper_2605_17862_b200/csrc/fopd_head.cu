// Log-probs from hidden states and head weights, and their gradient: argument checks, workspaces, launches.
#include "head_kernels.cuh"
#include "host_ranges.cuh"
#include "tensor_host.cuh"

using namespace fopd;

namespace {

constexpr int64_t kPieceBytes = (int64_t)1 << 29;   // gradient of the logits kept at a time
constexpr int64_t kPartBytes = (int64_t)1 << 29;    // rows' pieces (8 bytes to 128 tokens) kept at a time
constexpr int64_t kLogprobRows = 32768;             // rows they are of at most
constexpr int64_t kSumBytes = (int64_t)256 << 20;   // sums of d_hidden, where the vocabulary is cut into splits

int check_head(const fopd_head *h) {
  if (!h) return FOPD_ERR_NULL;
  if (h->dtype != FOPD_BF16) return FOPD_ERR_DTYPE;
  if (h->n_rows < 0 || h->vocab <= 0 || h->dim <= 0 || h->n_rows > 1 << 27 || h->vocab > 1 << 30 || h->dim > 1 << 20) return FOPD_ERR_SIZE;
  if ((h->n_rows > 1 && h->hidden_stride < h->dim) || (h->vocab > 1 && h->weight_stride < h->dim)) return FOPD_ERR_SIZE;
  if (h->hidden_stride > (int64_t)1 << 32 || h->weight_stride > (int64_t)1 << 32) return FOPD_ERR_SIZE;
  if (h->n_rows == 0) return FOPD_OK;
  if (!h->hidden || !h->weight || !h->tokens) return FOPD_ERR_NULL;
  if (!aligned16(h->hidden) || !aligned16(h->weight) || (h->n_rows > 1 && h->hidden_stride % 8 != 0) ||
      (h->vocab > 1 && h->weight_stride % 8 != 0))
    return FOPD_ERR_ALIGN;
  return FOPD_OK;
}

// Where a tensor of the call lies.  Rows that share no element with those of another are apart, also in columns of one wider matrix.
struct Place {
  Range at;
  bool there;
};
Place place(const void *p, int64_t rows, int64_t cols, int64_t stride, int64_t size) {
  if (!p || rows <= 0) return {{}, false};
  return {range_of(p, rows, cols, stride, (uintptr_t)size, 0, false), true};
}
Place vector_at(const void *p, int64_t n, int64_t size) { return place(p, 1, n, n, size); }
bool meet(const Place &a, const Place &b) {
  if (!a.there || !b.there || a.at.hi <= b.at.lo || b.at.hi <= a.at.lo) return false;
  return a.at.lo <= b.at.lo ? !disjoint_columns(a.at, b.at) : !disjoint_columns(b.at, a.at);
}
// Whether an output meets one of the arrays that every call reads.
bool meets_inputs(const fopd_head *h, const Place &p) {
  return meet(p, place(h->hidden, h->n_rows, h->dim, h->hidden_stride, 2)) || meet(p, place(h->weight, h->vocab, h->dim, h->weight_stride, 2)) ||
         meet(p, vector_at(h->tokens, h->n_rows, 4)) || meet(p, vector_at(h->mask, h->n_rows, 1));
}

// (an error is this call's alone: the next one's is not to find it)
int clear_rows(void *p, int64_t pitch, int64_t width, int64_t rows, cudaStream_t st) {
  if (cudaMemset2DAsync(p, (size_t)pitch, 0, (size_t)width, (size_t)rows, st) == cudaSuccess) return FOPD_OK;
  (void)cudaGetLastError();
  return FOPD_ERR_CUDA;
}

struct Temporary {
  char *base = nullptr;
  cudaStream_t st;
  explicit Temporary(cudaStream_t s) : st(s) {}
  int take(int64_t bytes) { return scratch_alloc(reinterpret_cast<void **>(&base), (size_t)bytes, st); }
  int give(int rc) {
    if (!base || cudaFreeAsync(base, st) == cudaSuccess) return rc;
    (void)cudaGetLastError();
    return rc == FOPD_OK ? FOPD_ERR_CUDA : rc;
  }
};

// The rows of a call and where their hidden states are: the caller's, or with a mask a compacted copy.
struct Prepared {
  HeadRows rows;
  const void *hidden_at;
  int64_t hidden_rows, hidden_pitch;
  CUtensorMap hidden_along, weight_along;  // boxes for products along the dimensions
};
int operand_map(CUtensorMap *map, const void *at, int64_t dim, int64_t rows, int64_t pitch, int box_rows) {
  return make_map(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, at, dim, rows, pitch * 2, 64, box_rows);
}
int64_t weight_pitch(const fopd_head *h) { return h->vocab > 1 ? h->weight_stride : round_up(h->dim, 8); }
struct RowParts {
  int64_t index = 0, active = 0, copy = 0;
};
RowParts row_parts(const fopd_head *h, Layout *lay) {
  RowParts r;
  if (!h->mask) return r;
  r.index = lay->take(h->n_rows * 4);
  r.active = lay->take(4);
  r.copy = lay->take(round_up(h->n_rows, 64) * round_up(h->dim, 8) * 2);
  return r;
}
int prepare_rows(const fopd_head *h, const RowParts &at, char *base, const float *coef, float *logprob, float *lse, int32_t *status,
                 cudaStream_t st, Prepared *out) {
  out->rows = {(int)h->n_rows, 0, nullptr, nullptr};
  const void *hidden = h->hidden;
  int64_t rows = h->n_rows, pitch = h->n_rows > 1 ? h->hidden_stride : round_up(h->dim, 8);
  if (h->mask) {
    int *index = reinterpret_cast<int *>(base + at.index), *active = reinterpret_cast<int *>(base + at.active);
    __nv_bfloat16 *copy = reinterpret_cast<__nv_bfloat16 *>(base + at.copy);
    const int64_t per = round_up((rows + kCompactBlocks - 1) / kCompactBlocks, 8);
    const int rc = launch_early(head_compact_kernel, dim3((unsigned)((rows + per - 1) / per)), kCompactThreads, st, h->mask, h->tokens, coef,
                                (int)rows, (int)per, h->vocab, static_cast<const __nv_bfloat16 *>(h->hidden), pitch, (int)h->dim,
                                (int)round_up(h->dim, 8), copy, index, active, logprob, lse, status);
    if (rc != FOPD_OK) return rc;
    rows = round_up(h->n_rows, 64);
    out->rows.index = index;
    out->rows.active = active;
    hidden = copy;
    pitch = round_up(h->dim, 8);
  }
  out->hidden_at = hidden;
  out->hidden_rows = rows;
  out->hidden_pitch = pitch;
  const int rc = operand_map(&out->hidden_along, hidden, h->dim, rows, pitch, 2 * kBoxRows);
  return rc != FOPD_OK ? rc : operand_map(&out->weight_along, h->weight, h->dim, h->vocab, weight_pitch(h), 2 * kBoxRows);
}

// The same from row `first` on, `n` rows at most.
int rows_from(const fopd_head *h, int64_t first, int64_t n, Prepared *pre) {
  if (first == 0 && n >= h->n_rows) return FOPD_OK;
  pre->rows.first = (int)first;
  pre->rows.n = (int)(h->n_rows - first < n ? h->n_rows - first : n);
  return operand_map(&pre->hidden_along, static_cast<const char *>(pre->hidden_at) + first * pre->hidden_pitch * 2, h->dim,
                     pre->hidden_rows - first, pre->hidden_pitch, 2 * kBoxRows);
}

template <int kCtas, int kN>
int run_logprob(const fopd_head *h, float *logprob, float *lse, int32_t *status, int sms, cudaStream_t st) {
  constexpr int64_t kRows = kCtas * 128;
  const int64_t v_tiles = (h->vocab + kN - 1) / kN;
  const int64_t fit = kPartBytes / (16 * v_tiles) / kRows * kRows, at_a_time = fit < kRows ? kRows : fit < kLogprobRows ? fit : kLogprobRows;
  const int64_t pitch = round_up(h->n_rows < at_a_time ? h->n_rows : at_a_time, kRows);
  Layout lay;
  const RowParts parts = row_parts(h, &lay);
  const int64_t part = lay.take(2 * v_tiles * pitch * 8), logit = lay.take(pitch * 4);
  Temporary tmp(st);
  int rc = tmp.take(lay.bytes);
  if (rc != FOPD_OK) return rc;
  Prepared pre;
  rc = prepare_rows(h, parts, tmp.base, nullptr, logprob, lse, status, st, &pre);
  for (int64_t first = 0; rc == FOPD_OK && first < h->n_rows; first += at_a_time) {
    rc = rows_from(h, first, at_a_time, &pre);
    if (rc != FOPD_OK) break;
    typename LogprobJob<kCtas, kN>::Params p;
    p.hidden = pre.hidden_along;
    p.weight = pre.weight_along;
    p.l = {nullptr, nullptr, pre.rows, h->vocab, (int)((h->dim + 63) / 64), 0, (int)v_tiles, kCtas == 1 ? kFewRowsChunk : kLogitChunk};
    p.tokens = h->tokens;
    p.part = reinterpret_cast<float2 *>(tmp.base + part);
    p.token_logit = reinterpret_cast<float *>(tmp.base + logit);
    p.pitch = (int)pitch;
    p.status = status;
    rc = launch_product<kCtas, kN, LogprobJob<kCtas, kN>>(p, (pre.rows.n + kRows - 1) / kRows * v_tiles, sms, st);
    if (rc == FOPD_OK)
      rc = launch_early(head_join_kernel, dim3((unsigned)((pre.rows.n + 3) / 4)), kJoinThreads, st, pre.rows, (const float2 *)p.part,
                        (const float *)p.token_logit, 2 * (int)v_tiles, (int)pitch, h->tokens, h->vocab, logprob, lse, status);
  }
  return tmp.give(rc);
}

struct GradOut {
  void *d_hidden;
  int64_t d_hidden_stride;
  void *d_weight;
  int64_t d_weight_stride;
  int32_t d_weight_dtype, add;
};

template <int kCtas, int kN>
int run_grad(const fopd_head *h, const float *logprob, const float *lse, const float *coef, const GradOut &o, int32_t *status, int sms,
             cudaStream_t st) {
  constexpr int kRows = kCtas * 128;
  const int64_t pitch = round_up(h->n_rows, kRows);
  const int planes = o.d_weight && o.d_weight_dtype == FOPD_F32 ? 2 : 1;
  // pieces of the vocabulary, alike, of whole tiles of both products that cut it
  constexpr int64_t kUnit = kN > kRows ? kN : kRows;
  int64_t piece = kPieceBytes / (pitch * 2 * planes) / kUnit * kUnit;
  if (piece < kUnit) piece = kUnit;
  const int64_t n_pieces = (h->vocab + piece - 1) / piece;
  piece = round_up((h->vocab + n_pieces - 1) / n_pieces, kUnit);
  const int64_t panels = piece / 64, lo = planes > 1 ? panels * pitch : 0;
  if (panels * pitch * planes >= (int64_t)1 << 31) return FOPD_ERR_SIZE;  // (n_rows beyond 2^28)

  // splits of d_hidden's contraction: no tile longer than a quarter of a CTA's share of the piece's work, where the sums fit
  const int64_t d_tiles = (h->dim + kN - 1) / kN, h_tiles = pitch / kRows * d_tiles, w_tiles = piece / kRows * d_tiles;
  const int64_t share = ((o.d_hidden ? h_tiles * panels : 0) + (o.d_weight ? w_tiles * planes * ((h->n_rows + 63) / 64) : 0)) / (sms / kCtas);
  int64_t split_panels = share / 4 > 16 ? share / 4 : 16;
  const int64_t sum_pitch = round_up(h->dim, 32), sum_each = pitch * sum_pitch * 4;
  int64_t splits = (panels + split_panels - 1) / split_panels;
  if (splits > kSumBytes / sum_each) splits = kSumBytes / sum_each;
  if (splits < 1) splits = 1;
  split_panels = (panels + splits - 1) / splits;
  splits = (panels + split_panels - 1) / split_panels;
  if (!o.d_hidden) splits = 0;

  Layout lay;
  const RowParts parts = row_parts(h, &lay);
  const int64_t g_at = lay.take(panels * pitch * planes * 128), sum_at = lay.take(splits * sum_each);
  Temporary tmp(st);
  int rc = tmp.take(lay.bytes);
  if (rc != FOPD_OK) return rc;
  Prepared pre;
  rc = prepare_rows(h, parts, tmp.base, coef, nullptr, nullptr, status, st, &pre);
  typename GradLogitsJob<kCtas, kN>::Params g;
  typename HeadGradsJob<kCtas, kN>::Params q;
  if (rc == FOPD_OK) rc = operand_map(&q.hidden, pre.hidden_at, h->dim, pre.hidden_rows, pre.hidden_pitch, kBoxRows);
  if (rc == FOPD_OK) rc = operand_map(&q.weight, h->weight, h->dim, h->vocab, weight_pitch(h), kBoxRows);
  if (rc == FOPD_OK)
    rc = make_map(&g.panels_out, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, tmp.base + g_at, 64, panels * pitch * planes, 128, 64, 32);
  if (rc == FOPD_OK)
    rc = make_map(&q.panels, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, tmp.base + g_at, 64, panels * pitch * planes, 128, 64, kBoxRows);
  // (a box ends at a multiple of 16 bytes: rows that do not would be written beyond their end)
  q.d_weight_boxes = o.d_weight && !o.add && h->dim * (o.d_weight_dtype == FOPD_F32 ? 4 : 2) % 16 == 0;
  if (rc == FOPD_OK && q.d_weight_boxes) {
    const bool f32 = o.d_weight_dtype == FOPD_F32;
    const int64_t size = f32 ? 4 : 2, stride = h->vocab > 1 ? o.d_weight_stride : round_up(h->dim, 16 / size);
    rc = make_map(&q.d_weight_out, f32 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, o.d_weight, h->dim, h->vocab,
                  stride * size, 128 / (int)size, 32);
  }
  if (rc == FOPD_OK)
    rc = make_map(&q.panels_along, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, tmp.base + g_at, 64, panels * pitch * planes, 128, 64, 2 * kBoxRows);
  if (rc == FOPD_OK && o.d_hidden && h->mask)
    rc = clear_rows(o.d_hidden, (h->n_rows > 1 ? o.d_hidden_stride : h->dim) * 2, h->dim * 2, h->n_rows, st);
  if (rc == FOPD_OK) {
    g.hidden = pre.hidden_along;
    g.weight = pre.weight_along;
    g.tokens = h->tokens;
    g.logprob = logprob;
    g.lse = lse;
    g.coef = coef;
    g.pitch = q.pitch = (int)pitch;
    g.lo = q.lo = (int)lo;
    g.status = q.status = status;
    q.rows = pre.rows;
    q.vocab = h->vocab;
    q.dim = (int)h->dim;
    q.splits = (int)splits;
    q.split_panels = (int)split_panels;
    q.sum = reinterpret_cast<float *>(tmp.base + sum_at);
    q.sum_pitch = (int)sum_pitch;
    q.d_weight = o.d_weight;
    q.d_weight_pitch = o.d_weight_stride;
    q.d_weight_f32 = o.d_weight_dtype == FOPD_F32;
    q.add = o.add;
    for (int64_t v0 = 0; rc == FOPD_OK && v0 < h->vocab; v0 += piece) {
      const int64_t count = h->vocab - v0 < piece ? h->vocab - v0 : piece;
      // (for bf16 gradients the logits' own last bits do not show: one accumulator)
      g.l = {nullptr, nullptr, pre.rows, h->vocab, (int)((h->dim + 63) / 64), (int)(v0 / kN), (int)((count + kN - 1) / kN),
             !lo ? kLongChunk : kCtas == 1 ? kFewRowsChunk : kGradChunk};
      q.v0 = v0;
      q.v_count = (int)count;
      q.first = v0 == 0;
      rc = launch_product<kCtas, kN, GradLogitsJob<kCtas, kN>>(g, pitch / kRows * g.l.v_tiles, sms, st);
      if (rc == FOPD_OK)
        rc = launch_product<kCtas, kN, HeadGradsJob<kCtas, kN>>(q, splits * h_tiles + (o.d_weight ? (count + kRows - 1) / kRows * d_tiles : 0), sms, st);
    }
  }
  if (rc == FOPD_OK && o.d_hidden) {
    const bool many = splits >= 8;
    const int dims = many ? 128 : 1024;
    rc = launch_early(many ? head_hidden_kernel<8> : head_hidden_kernel<1>,
                      dim3(row_grid(h->n_rows), (unsigned)((h->dim + dims - 1) / dims)), 256, st, pre.rows, (const float *)q.sum, (int)splits,
                      (int)pitch, (int)sum_pitch, h->tokens, logprob, coef, static_cast<const __nv_bfloat16 *>(h->weight), h->weight_stride,
                      h->vocab, (int)h->dim, o.d_hidden_stride, static_cast<__nv_bfloat16 *>(o.d_hidden));
  }
  return tmp.give(rc);
}

}  // namespace

extern "C" {

int fopd_head_logprob(const fopd_head *h, float *logprob, float *lse, int32_t *status, void *stream) {
  int rc = check_head(h);
  if (rc != FOPD_OK || h->n_rows == 0) return rc;
  if (!logprob) return FOPD_ERR_NULL;
  const Place lp = vector_at(logprob, h->n_rows, 4), ls = vector_at(lse, h->n_rows, 4);
  if (meets_inputs(h, lp) || meets_inputs(h, ls) || meet(lp, ls)) return FOPD_ERR_ALIAS;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  int sms = 0;
  rc = current_sms(&sms);
  if (rc != FOPD_OK) return rc;
  return h->n_rows <= 128 ? run_logprob<1, 256>(h, logprob, lse, status, sms, st) : run_logprob<2, 256>(h, logprob, lse, status, sms, st);
}

int fopd_head_grad(const fopd_head *h, const float *logprob, const float *lse, const float *coef, void *d_hidden,
                   int64_t d_hidden_stride, void *d_weight, int64_t d_weight_stride, int32_t d_weight_dtype, int32_t add_d_weight,
                   int32_t *status, void *stream) {
  int rc = check_head(h);
  if (rc != FOPD_OK) return rc;
  if (!d_hidden && !d_weight) return FOPD_ERR_NULL;
  if (d_weight && d_weight_dtype != FOPD_BF16 && d_weight_dtype != FOPD_F32) return FOPD_ERR_DTYPE;
  const int64_t wsize = d_weight_dtype == FOPD_F32 ? 4 : 2;
  if (d_hidden && h->n_rows > 1 && d_hidden_stride < h->dim) return FOPD_ERR_SIZE;
  if (d_weight && h->vocab > 1 && d_weight_stride < h->dim) return FOPD_ERR_SIZE;
  if (d_hidden_stride > (int64_t)1 << 32 || d_weight_stride > (int64_t)1 << 32) return FOPD_ERR_SIZE;
  if (!aligned16(d_hidden) || !aligned16(d_weight) || (d_hidden && h->n_rows > 1 && d_hidden_stride % 8 != 0) ||
      (d_weight && h->vocab > 1 && d_weight_stride * wsize % 16 != 0))
    return FOPD_ERR_ALIGN;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (h->n_rows == 0) {  // no row: the weights' gradient is zero
    return d_weight && !add_d_weight ? clear_rows(d_weight, (h->vocab > 1 ? d_weight_stride : h->dim) * wsize, h->dim * wsize, h->vocab, st)
                                     : FOPD_OK;
  }
  if (!logprob || !lse || !coef) return FOPD_ERR_NULL;
  const Place dh = place(d_hidden, h->n_rows, h->dim, d_hidden_stride, 2), dw = place(d_weight, h->vocab, h->dim, d_weight_stride, wsize);
  for (const float *in : {logprob, lse, coef})
    if (meet(dh, vector_at(in, h->n_rows, 4)) || meet(dw, vector_at(in, h->n_rows, 4))) return FOPD_ERR_ALIAS;
  if (meets_inputs(h, dh) || meets_inputs(h, dw) || meet(dh, dw)) return FOPD_ERR_ALIAS;
  int sms = 0;
  rc = current_sms(&sms);
  if (rc != FOPD_OK) return rc;
  const GradOut o = {d_hidden, d_hidden_stride, d_weight, d_weight_stride, d_weight_dtype, add_d_weight ? 1 : 0};
  return h->n_rows <= 128 ? run_grad<1, 256>(h, logprob, lse, coef, o, status, sms, st)
                          : run_grad<2, 256>(h, logprob, lse, coef, o, status, sms, st);
}

}  // extern "C"
