// Token drawing and draft verification: argument checks, the temporary, launches.
#include "host_common.cuh"
#include "rollout_kernels.cuh"

using namespace fopd;

namespace {

bool temperature_ok(double t) { return t == 0.0 || (t >= 1.0 / 1024 && t <= 1024.0); }

// CTAs that share a row, a position or a sequence: as many as keep `units` clusters of them within `most` CTAs.
int cluster_for(int64_t units, int most) {
  int c = kRollMaxCluster;
  while (c > 1 && units * c > most) c /= 2;
  return c;
}

// early: the kernel may be set up while the one before it on the stream is still running (it waits for it itself).
template <class Kernel>
int launch_clusters(Kernel kernel, const RolloutDev &d, int64_t units, int c, cudaStream_t st, bool early = false) {
  if (units * c > INT32_MAX) return FOPD_ERR_SIZE;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = c;
  attr[0].val.clusterDim.y = 1;
  attr[0].val.clusterDim.z = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(units * c));
  cfg.blockDim = dim3(kRollThreads);
  cfg.stream = st;
  cfg.attrs = attr;
  cfg.numAttrs = early ? 2 : 1;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  if (cudaLaunchKernelEx(&cfg, kernel, d) != cudaSuccess) {
    (void)cudaGetLastError();
    return FOPD_ERR_CUDA;
  }
  return FOPD_OK;
}

// Parts of a row, and how many of them share a slot when c CTAs have the row between them: one where warps are to have
// few parts each, two (one vector of a slot for each thread of the search) where a CTA has a row of its own.
template <int DT>
void set_parts(RolloutDev *d, int c) {
  d->n_parts = (d->vocab + kPartElems<DT> - 1) / kPartElems<DT>;
  const int64_t slots = (int64_t)c * kSlots, least = (d->n_parts + slots - 1) / slots;
  d->span = (int)(least > 2 ? least : c > 1 ? least : 2);
}

// Relative error of a row's fp32 sum and of one weight.  An exponent y = x c - max c is off by the rounding of c (known
// here) and its own (2^-24 |y|).  The mean of |y| over the distribution is its entropy less its min-entropy in bits, at
// most (1 - s) log2(s (V - 1) / (1 - s)) for some s: 0.74 log2 V covers V <= 2^18, 0.82 log2 V all up to 2^30.  An ex2
// (2^-22) and six roundings (2^-24) come on top.
double sum_error(int64_t vocab, float c, double c64) {
  const double bits = std::log2((double)vocab), y = (vocab <= (1 << 18) ? 0.74 : 0.82) * bits + 0.5;
  return 0.6932 * (5.97e-8 + std::fabs((double)c - c64) / c64) * y + 6.2e-7;
}

size_t later_bytes(int64_t units) { return sizeof(Later) + (size_t)units * sizeof(LaterEntry); }
int64_t list_clusters(int64_t units, int c) { return units < kRollWhole / c ? units : kRollWhole / c; }
// Two launches (Mode) for more rows or sequences than clusters of c of the whole kernel fit at once.
bool two_launches(int64_t units, int c) { return units * c > kRollWhole; }

template <int DT>
int launch_draw(RolloutDev d, cudaStream_t st) {
  int c = cluster_for(d.B, kRollResident);
  set_parts<DT>(&d, c);
  if (d.ct64 == 0.0) return launch_clusters(draw_kernel<DT, true, kFirst>, d, d.B, c, st);
  if (!two_launches(d.B, kDrawList)) {
    c = cluster_for(d.B, kRollWhole);
    set_parts<DT>(&d, c);
    return launch_clusters(draw_kernel<DT, false, kWhole>, d, d.B, c, st);
  }
  int rc = scratch_alloc(reinterpret_cast<void **>(&d.later), later_bytes(d.B), st);
  if (rc != FOPD_OK) return rc;
  if (cudaMemsetAsync(d.later, kUnset & 0xff, sizeof(int32_t), st) != cudaSuccess) rc = FOPD_ERR_CUDA;
  if (rc == FOPD_OK) rc = launch_clusters(draw_kernel<DT, false, kFirst>, d, d.B, c, st);
  set_parts<DT>(&d, kDrawList);
  if (rc == FOPD_OK)
    rc = launch_clusters(draw_kernel<DT, false, kSecond>, d, list_clusters(d.B, kDrawList), kDrawList, st, true);
  if (cudaFreeAsync(d.later, st) != cudaSuccess) rc = FOPD_ERR_CUDA;
  return rc;
}

template <int DT>
int launch_verify(RolloutDev d, cudaStream_t st) {
  const bool best = d.ct64 == 0.0;
  const int64_t positions = (int64_t)d.B * (d.K + 1);
  const int64_t parts = (d.vocab + kPartElems<DT> - 1) / kPartElems<DT>;
  // Up to four times what fits at once, a cluster per position (rows of unequal need are then shared out evenly); more
  // positions: clusters that stay, so few that a rejection is known before much behind it has been swept.
  bool stay = positions > 4 * kRollResident;
  int c = stay ? cluster_for(d.B, kRollResident) : cluster_for(positions, 2 * kRollResident);
  while (c > 1 && parts * 2 < c * kRollWarps * 2) c /= 2;  // a few parts for each warp
  const int cf = best ? 1 : cluster_for(d.B, kRollResident);
  const bool look = positions * c > kRollResident;  // later positions start when earlier ones have been decided
  int64_t clusters = positions;
  if (stay) clusters = d.B * ((kRollResident / c + d.B - 1) / d.B);
  const bool two = !best && two_launches(d.B, kFinishList);
  const size_t pos_bytes = ((size_t)positions * sizeof(Position) + 255) & ~size_t(255);
  const size_t stop_bytes = look ? ((size_t)d.B * sizeof(int32_t) + 255) & ~size_t(255) : 0;
  const size_t next_bytes = stay ? stop_bytes : 0;
  char *tmp = nullptr;
  int rc = scratch_alloc(reinterpret_cast<void **>(&tmp), pos_bytes + stop_bytes + next_bytes + (two ? later_bytes(d.B) : 0), st);
  if (rc != FOPD_OK) return rc;
  d.pos = reinterpret_cast<Position *>(tmp);
  if (look) d.stop = reinterpret_cast<int32_t *>(tmp + pos_bytes);
  if (stay) d.next = reinterpret_cast<int32_t *>(tmp + pos_bytes + stop_bytes);
  if (two) d.later = reinterpret_cast<Later *>(tmp + pos_bytes + stop_bytes + next_bytes);
  // all counters in one go
  const size_t unset = stop_bytes + next_bytes + (two ? sizeof(int32_t) : 0);
  if (unset && cudaMemsetAsync(tmp + pos_bytes, kUnset & 0xff, unset, st) != cudaSuccess) rc = FOPD_ERR_CUDA;
  set_parts<DT>(&d, c);
  if (rc == FOPD_OK)
    rc = best ? launch_clusters(verify_sweep_kernel<DT, true>, d, clusters, c, st)
              : launch_clusters(verify_sweep_kernel<DT, false>, d, clusters, c, st);
  set_parts<DT>(&d, cf);
  if (rc == FOPD_OK)
    rc = best  ? launch_clusters(verify_finish_kernel<DT, true, kFirst>, d, d.B, cf, st, true)
         : two ? launch_clusters(verify_finish_kernel<DT, false, kFirst>, d, d.B, cf, st, true)
               : launch_clusters(verify_finish_kernel<DT, false, kWhole>, d, d.B, cf, st, true);
  if (rc == FOPD_OK && two) {
    set_parts<DT>(&d, kFinishList);
    rc = launch_clusters(verify_finish_kernel<DT, false, kSecond>, d, list_clusters(d.B, kFinishList), kFinishList, st, true);
  }
  if (cudaFreeAsync(tmp, st) != cudaSuccess) rc = FOPD_ERR_CUDA;
  return rc;
}

struct Span {
  const void *p;
  int64_t bytes;
};
// Whether an output lies on tokens, counts or numbers that are read: CTAs read these while others write those.
bool outputs_meet_inputs(const fopd_draft *d, const int32_t *tokens, const float *logprob, const uint8_t *mask,
                         const int32_t *n_accepted) {
  const int64_t B = d->B, W = (int64_t)d->K + 1;
  const Span in[] = {{d->uniform, B * W * 8}, {d->K > 0 ? d->tokens : nullptr, B * d->K * 4}, {d->K > 0 ? d->n_draft : nullptr, B * 4}};
  const Span out[] = {{tokens, B * W * 4}, {logprob, B * W * 4}, {mask, B * W}, {n_accepted, B * 4}};
  for (const Span &i : in)
    for (const Span &o : out) {
      const uintptr_t a = (uintptr_t)i.p, b = (uintptr_t)o.p;
      if (a && b && a < b + (uintptr_t)o.bytes && b < a + (uintptr_t)i.bytes) return true;
    }
  return false;
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
  if (outputs_meet_inputs(d, tokens, logprob, mask, n_accepted)) return FOPD_ERR_ALIAS;
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
  r.tokens = tokens;
  r.logprob = logprob;
  r.mask = mask;
  r.n_accepted = n_accepted;
  r.status = status;
  // a target without temperature never asks for the draft's probabilities: x is accepted if it is the best token
  const bool best = d->temperature == 0.0;
  r.kind = best || d->K == 0 ? kDraftNone : !d->draft ? kDraftCertain : d->draft_temperature == 0.0 ? kDraftBest : kDraftRows;
  r.ct64 = best ? 0.0 : 1.4426950408889634074 / d->temperature;
  r.cd64 = r.kind == kDraftRows ? 1.4426950408889634074 / d->draft_temperature : 0.0;
  r.ct = (float)r.ct64;
  r.cd = (float)r.cd64;
  if (!best) r.eps = sum_error(d->vocab, r.ct, r.ct64);
  if (r.kind == kDraftRows) r.eps = std::fmax(r.eps, sum_error(d->vocab, r.cd, r.cd64));
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const bool bf16 = d->dtype == FOPD_BF16;
  if (d->K == 0) return bf16 ? launch_draw<FOPD_BF16>(r, st) : launch_draw<FOPD_F32>(r, st);
  return bf16 ? launch_verify<FOPD_BF16>(r, st) : launch_verify<FOPD_F32>(r, st);
}

int fopd_draw_tokens(const void *logits, const double *uniform, int64_t n_rows, int64_t vocab, int64_t row_stride,
                     int32_t dtype, double temperature, int32_t *tokens, float *logprob, int32_t *status,
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
