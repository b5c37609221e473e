// Token drawing and draft verification: argument checks, the temporary, launches.
#include "host_common.cuh"
#include "rollout_kernels.cuh"

using namespace fopd;

namespace {

bool temperature_ok(float t) { return t == 0.f || (t >= 1.f / 1024 && t <= 1024.f); }

template <int DT>
int launch_rollout(RolloutDev d, int32_t *tokens, float *logprob, uint8_t *mask, int32_t *n_accepted, int32_t *status,
                   cudaStream_t st) {
  d.n_tiles = (d.vocab + TileShape<DT>::kElems - 1) / TileShape<DT>::kElems;
  const bool draft_rows = d.kind == kDraftRows || d.kind == kDraftBest;
  const int64_t positions = (int64_t)d.B * (d.K + 1);
  const int64_t rows = positions + (draft_rows ? (int64_t)d.B * d.K : 0);
  const size_t part_bytes = ((size_t)rows * d.n_tiles * sizeof(float2) + 255) & ~size_t(255);
  const size_t tsum_bytes = ((size_t)d.B * d.n_tiles * sizeof(double) + 255) & ~size_t(255);
  char *tmp = nullptr;
  int rc = scratch_alloc(reinterpret_cast<void **>(&tmp), part_bytes + tsum_bytes + positions * sizeof(Position), st);
  if (rc != FOPD_OK) return rc;
  d.part = reinterpret_cast<float2 *>(tmp);
  d.tsum = reinterpret_cast<double *>(tmp + part_bytes);
  d.pos = reinterpret_cast<Position *>(tmp + part_bytes + tsum_bytes);
  const int64_t items = rows * ((d.n_tiles + kTileWarps - 1) / kTileWarps);
  rollout_tiles_kernel<DT><<<(unsigned)(items < kMaxGrid ? items : kMaxGrid), kTileWarps * 32, 0, st>>>(d, items);
  rc = launch_ok();
  if (rc == FOPD_OK) {
    rollout_finish_kernel<DT><<<(unsigned)d.B, kFinishThreads, 0, st>>>(d, tokens, logprob, mask, n_accepted, status);
    rc = launch_ok();
  }
  if (cudaFreeAsync(tmp, st) != cudaSuccess) rc = FOPD_ERR_CUDA;
  return rc;
}

}  // namespace

extern "C" {

int fopd_verify_draft(const fopd_draft *d, int32_t *tokens, float *logprob, uint8_t *mask, int32_t *n_accepted,
                      int32_t *status, void *stream) {
  if (!d) return FOPD_ERR_NULL;
  if (d->dtype != FOPD_BF16 && d->dtype != FOPD_F32) return FOPD_ERR_DTYPE;
  if (d->B < 0 || d->K < 0 || d->K >= (1 << 20) || d->vocab <= 0 || d->vocab > (int64_t)1 << 30) return FOPD_ERR_SIZE;
  const int64_t esz = d->dtype == FOPD_BF16 ? 2 : 4, most = (int64_t)1 << 40;
  if (d->target_row_stride < 0 || d->target_seq_stride < 0 || d->target_row_stride > most || d->target_seq_stride > most ||
      (d->K > 0 && d->target_row_stride < d->vocab))
    return FOPD_ERR_SIZE;
  const bool rows = d->draft && d->K > 0;
  if (rows && (d->draft_row_stride < 0 || d->draft_seq_stride < 0 || d->draft_row_stride > most ||
               d->draft_seq_stride > most || (d->K > 1 && d->draft_row_stride < d->vocab)))
    return FOPD_ERR_SIZE;
  if (!temperature_ok(d->temperature) || (rows && !temperature_ok(d->draft_temperature))) return FOPD_ERR_PARAM;
  if (d->B == 0) return FOPD_OK;
  if (!d->target || !d->uniform || !tokens || (d->K > 0 && !d->tokens)) return FOPD_ERR_NULL;
  if (!aligned16(d->target) || (d->K > 0 && (d->target_row_stride * esz) % 16 != 0) ||
      (d->B > 1 && (d->target_seq_stride * esz) % 16 != 0))
    return FOPD_ERR_ALIGN;
  if (rows && (!aligned16(d->draft) || (d->K > 1 && (d->draft_row_stride * esz) % 16 != 0) ||
               (d->B > 1 && (d->draft_seq_stride * esz) % 16 != 0)))
    return FOPD_ERR_ALIGN;
  RolloutDev r = {};
  r.target = static_cast<const char *>(d->target);
  r.draft = static_cast<const char *>(d->draft);
  r.drafted = d->tokens;
  r.n_draft = d->n_draft;
  r.uniform = d->uniform;
  r.vocab = d->vocab;
  r.tseq = d->target_seq_stride * esz;
  r.trow = d->target_row_stride * esz;
  r.dseq = d->draft_seq_stride * esz;
  r.drow = d->draft_row_stride * esz;
  r.B = d->B;
  r.K = d->K;
  r.best = d->temperature == 0.f;
  // a target without temperature never asks for the draft's probabilities: x is accepted if it is the best token
  r.kind = d->K == 0 || r.best ? kDraftNone : !d->draft ? kDraftCertain : d->draft_temperature == 0.f ? kDraftBest : kDraftRows;
  r.it = r.best ? 0.0 : 1.0 / (double)d->temperature;
  r.id = r.kind == kDraftRows ? 1.0 / (double)d->draft_temperature : 0.0;
  r.ct = (float)(r.it * 1.4426950408889634);
  r.cd = (float)(r.id * 1.4426950408889634);
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  return d->dtype == FOPD_BF16 ? launch_rollout<FOPD_BF16>(r, tokens, logprob, mask, n_accepted, status, st)
                               : launch_rollout<FOPD_F32>(r, tokens, logprob, mask, n_accepted, status, st);
}

int fopd_draw_tokens(const void *logits, const double *uniform, int64_t n_rows, int64_t vocab, int64_t row_stride,
                     int32_t dtype, float temperature, int32_t *tokens, float *logprob, int32_t *status,
                     void *stream) {
  if (dtype != FOPD_BF16 && dtype != FOPD_F32) return FOPD_ERR_DTYPE;
  if (n_rows < 0 || n_rows > INT32_MAX || vocab <= 0 || row_stride < vocab) return FOPD_ERR_SIZE;
  fopd_draft d = {};
  d.target = logits;
  d.uniform = uniform;
  d.vocab = vocab;
  d.target_seq_stride = row_stride;
  d.target_row_stride = row_stride;
  d.B = (int32_t)n_rows;
  d.dtype = dtype;
  d.temperature = temperature;
  if (n_rows > 0 && (row_stride * (dtype == FOPD_BF16 ? 2 : 4)) % 16 != 0) return FOPD_ERR_ALIGN;
  return fopd_verify_draft(&d, tokens, logprob, nullptr, nullptr, status, stream);
}

}  // extern "C"
