// Log-probs of tokens and their gradient from hidden states and the weights of the vocabulary head (sm_100a).
//
//   z_nv = h_n . w_v,   lse_n = log sum_v e^{z_nv},   logprob_n = z_{n,y_n} - lse_n
//   G_nv = coef_n (e^{z_nv - lse_n} - [v = y_n]),   d_hidden = G W,   d_weight = G^T H
//
// The logits live in TMEM only: a tile of 256 (128) rows x 256 tokens is reduced by its epilogue to each row's maximum and sum,
// or turned into the tile of G that the two products behind it read.  G is kept for a piece of the vocabulary at a time, in
// bf16 and in panels of 64 columns, which both products read as they are: d_hidden along the columns, d_weight along the rows.
#pragma once

#include "tensor_core.cuh"

namespace fopd {

// The rows a call works on: all n of them, or the *active first ones of a compacted copy.
struct HeadRows {
  int n;
  const int *active;  // DEVICE count, or NULL: n
  const int *index;   // compacted row -> row of the caller's, or NULL: the same
  __device__ __forceinline__ int count() const { return active ? *active : n; }
  __device__ __forceinline__ int row(int i) const { return index ? index[i] : i; }
};

// ------------------------------------------------------------------ rows that count, one after another
// The kernel of one CTA that numbers them (and clears the others' results), then the copies of their hidden states.
constexpr int kHeadIndexThreads = 1024;
__global__ void __launch_bounds__(kHeadIndexThreads) head_index_kernel(const uint8_t *mask, const int32_t *tokens, const float *coef,
                                                                       int n, int64_t vocab, int *index, int *active,
                                                                       float *logprob, float *lse, int32_t *status) {
  __shared__ int warp_sum[kHeadIndexThreads / 32];
  __shared__ int base, bad;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  if (threadIdx.x == 0) base = bad = 0;
  __syncthreads();
  for (int at = 0; at < n; at += kHeadIndexThreads) {
    const int i = at + threadIdx.x;
    bool on = i < n && mask[i] != 0;
    if (on && (uint32_t)tokens[i] >= (uint64_t)vocab) {
      on = false;
      bad = 1;
    }
    if (on && coef && coef[i] == 0.f) on = false;
    const uint32_t vote = __ballot_sync(0xffffffffu, on);
    if (lane == 0) warp_sum[warp] = __popc(vote);
    __syncthreads();
    int before = base;
    for (int w = 0; w < warp; ++w) before += warp_sum[w];
    if (on) index[before + __popc(vote & ((1u << lane) - 1))] = i;
    if (i < n && !on) {
      if (logprob) logprob[i] = 0.f;
      if (lse) lse[i] = 0.f;
    }
    __syncthreads();
    if (threadIdx.x == kHeadIndexThreads - 1) base = before + __popc(vote);
    __syncthreads();
  }
  if (threadIdx.x == 0) {
    *active = base;
    if (bad && status) atomicOr(status, FOPD_DEV_BAD_TOKEN);
  }
}

// A warp per row of the copy; rows up to the next multiple of 64 are cleared, for products along the rows.
__global__ void __launch_bounds__(256) head_gather_kernel(const __nv_bfloat16 *hidden, int64_t pitch, const int *index,
                                                          const int *active, int dim, int copy_pitch, __nv_bfloat16 *copy) {
  const int r = blockIdx.x * 8 + (threadIdx.x >> 5), n = *active;
  if (r >= (n + 63) / 64 * 64) return;
  const __nv_bfloat16 *src = r < n ? hidden + (int64_t)index[r] * pitch : nullptr;
  __nv_bfloat16 *dst = copy + (int64_t)r * copy_pitch;
  for (int d = (threadIdx.x & 31) * 8; d < dim; d += 256) {
    if (d + 8 <= dim) *reinterpret_cast<uint4 *>(dst + d) = src ? *reinterpret_cast<const uint4 *>(src + d) : make_uint4(0, 0, 0, 0);
    else
      for (int e = d; e < dim; ++e) dst[e] = src ? src[e] : __float2bfloat16_rn(0.f);
  }
}

// ------------------------------------------------------------------ tiles of logits
constexpr int kLogitChunk = 8;  // blocks of 64 dimensions that a matrix instruction's accumulator adds up
struct LogitTiles {
  const CUtensorMap *hidden, *weight;
  HeadRows rows;
  int64_t vocab;
  int k_blocks;      // of 64 hidden dimensions
  int v_tile0, v_tiles;
};
// Tiles run over the rows first, in groups of 4,096 rows (a group's hidden states and the weights in flight stay in the L2).
template <int kCtas, int kN>
__device__ __forceinline__ void logit_tile_at(const LogitTiles &l, int n_rows, int64_t i, int &row0, int64_t &col0) {
  constexpr int kRows = kCtas * 128, kGroup = 4096 / kRows;
  const int m_tiles = (n_rows + kRows - 1) / kRows;
  const int64_t per = (int64_t)kGroup * l.v_tiles;
  const int g = (int)(i / per), in_group = min(kGroup, m_tiles - g * kGroup);
  const int64_t r = i - g * per;
  row0 = (g * kGroup + (int)(r % in_group)) * kRows;
  col0 = (l.v_tile0 + r / in_group) * kN;
}
template <int kCtas, int kN>
__device__ __forceinline__ int64_t logit_tiles(const LogitTiles &l, int n_rows) {
  return (int64_t)((n_rows + kCtas * 128 - 1) / (kCtas * 128)) * l.v_tiles;
}
template <int kCtas, int kN>
__device__ __forceinline__ void logit_tile(const LogitTiles &l, int n_rows, int64_t i, int cta, Tile &t) {
  int row0;
  int64_t col0;
  logit_tile_at<kCtas, kN>(l, n_rows, i, row0, col0);
  t.a = {l.hidden, 0, row0 + cta * 128, 64, 0, 0, 128, 0, false};
  t.b = {l.weight, 0, (int)col0 + cta * (kN / kCtas), 64, 0, 0, 128, 0, false};
  t.k_blocks = l.k_blocks;
  t.chunk = kLogitChunk;
  t.passes = 1;
  t.a_lo = t.b_lo = 0;
}

// ------------------------------------------------------------------ log-probs
// A tile's epilogue: two threads per row, each the maximum and the sum of exponentials of 128 logits (exponents as in RowSweep), the
// stored token's left out of the sum: the log-prob of a nearly certain token comes from the others' sum.
template <int kCtas, int kN>
struct LogprobJob {
  static constexpr bool kFp16 = false, kTurns = false, kClaimed = false;
  using Ticket = TileNumber;
  struct Params {
    CUtensorMap hidden, weight;
    LogitTiles l;
    const int32_t *tokens;
    float2 *part;  // [2 v_tiles][pitch]
    float *token_logit;
    int pitch;
    int32_t *status;
  };
  const Params &p;
  LogitTiles l;
  int n;
  __device__ explicit LogprobJob(const Params &params) : p(params), l(params.l), n(params.l.rows.count()) {
    l.hidden = &p.hidden;
    l.weight = &p.weight;
  }
  __device__ int64_t tiles() const { return logit_tiles<kCtas, kN>(l, n); }
  __device__ int32_t *status() const { return p.status; }
  __device__ __forceinline__ void tile(Ticket ticket, int cta, Tile &t) const { logit_tile<kCtas, kN>(l, n, ticket.i, cta, t); }
  __device__ __forceinline__ void epilogue(Ticket ticket, int cta, const Accumulator &acc, float (&z)[kN / 2]) const {
    constexpr int kCols = kN / 2;
    int row0;
    int64_t v0;
    logit_tile_at<kCtas, kN>(l, n, ticket.i, row0, v0);
    v0 += acc.half * kCols;
    const int row = row0 + cta * 128 + acc.warp * 32 + acc.lane;
    const int y = row < n ? p.tokens[l.rows.row(row)] : -1;
    if (v0 + kCols > l.vocab) {
      const int have = (int)max((int64_t)0, l.vocab - v0);
#pragma unroll
      for (int j = 0; j < kCols; ++j)
        if (j >= have) z[j] = -INFINITY;
    }
    const int64_t mine = (int64_t)y - v0;
    if (mine >= 0 && mine < kCols && y < l.vocab) {
      float zy = 0.f;
#pragma unroll
      for (int j = 0; j < kCols; ++j)
        if (j == (int)mine) {
          zy = z[j];
          z[j] = -INFINITY;
        }
      p.token_logit[row] = zy;
    }
    float m = kNegBig;
#pragma unroll
    for (int j = 0; j < kCols; j += 2) m = max3(m, z[j], z[j + 1]);
    const float c = fmaxf(m * kLog2e, kNegBig);  // (a half behind the last token has no logit)
    float s[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int j = 0; j < kCols; ++j) s[j & 3] += ex2(fmaf(z[j], kLog2e, -c));
    const float sum = (s[0] + s[1]) + (s[2] + s[3]), fix = -fmaf(m, kLog2e, -c) * kLn2;
    if (row < n) p.part[(v0 / kCols) * p.pitch + row] = make_float2(m, __fmaf_rn(sum, fix, sum));
  }
};

// Joins the pieces of 32 rows: 32 threads to a row's pieces, then in a fixed order; exponentials fp32, sums and logs fp64.
__global__ void __launch_bounds__(1024) head_join_kernel(HeadRows rows, const float2 *part, const float *token_logit, int pieces,
                                                         int pitch, const int32_t *tokens, int64_t vocab, float *logprob,
                                                         float *lse, int32_t *status) {
  __shared__ float sm[32][33];
  __shared__ double ss[32][33];
  const int n = rows.count(), tx = threadIdx.x & 31, ty = threadIdx.x >> 5, r = blockIdx.x * 32 + tx;
  if (blockIdx.x * 32 >= n) return;
  float m = kNegBig;
  double s = 0.0;
  if (r < n)
    for (int v = ty; v < pieces; v += 32) {
      const float2 q = part[(int64_t)v * pitch + r];
      if (q.x > m) {
        s *= (double)ex2((m - q.x) * kLog2e);
        m = q.x;
      }
      s += (double)(q.y * ex2((q.x - m) * kLog2e));
    }
  sm[ty][tx] = m;
  ss[ty][tx] = s;
  __syncthreads();
  if (ty != 0 || r >= n) return;
  const int row = rows.row(r), y = tokens[row];
  if (y < 0 || y >= vocab) {  // (without a mask rows are not sorted out beforehand)
    logprob[row] = 0.f;
    if (lse) lse[row] = 0.f;
    if (status) atomicOr(status, FOPD_DEV_BAD_TOKEN);
    return;
  }
  const float zy = token_logit[r];
  m = zy;
  for (int k = 0; k < 32; ++k) m = fmaxf(m, sm[k][tx]);
  double rest = 0.0;
  for (int k = 0; k < 32; ++k) rest += ss[k][tx] * exp((double)sm[k][tx] - (double)m);
  const double d = (double)zy - (double)m, t = exp(d);
  logprob[row] = (float)(t > rest ? -log1p(rest / t) : d - log(rest + t));
  if (lse) lse[row] = (float)((double)m + log(rest + t));
}

// ------------------------------------------------------------------ gradient of the logits, a piece of the vocabulary
// G goes to panels: [panel of 64 columns][pitch rows][64], bf16; a second plane of what the rounding left where the weights'
// gradient is wanted in fp32.  One rounding to bf16 (2^-9 at most) is what a matrix instruction takes; it is of the size of the
// bf16 results' own.
template <int kCtas, int kN>
struct GradLogitsJob {
  static constexpr bool kFp16 = false, kTurns = false, kClaimed = false;
  using Ticket = TileNumber;
  struct Params {
    CUtensorMap hidden, weight, panels_out;
    LogitTiles l;
    const int32_t *tokens;
    const float *logprob, *lse, *coef;
    int pitch;      // rows of a panel
    int lo;         // rows from one plane to the other, 0: one plane
    int32_t *status;
  };
  const Params &p;
  LogitTiles l;
  int n;
  Staging staging;
  __device__ explicit GradLogitsJob(const Params &params) : p(params), l(params.l), n(params.l.rows.count()) {
    l.hidden = &p.hidden;
    l.weight = &p.weight;
  }
  __device__ int64_t tiles() const { return logit_tiles<kCtas, kN>(l, n); }
  __device__ int32_t *status() const { return p.status; }
  __device__ __forceinline__ void tile(Ticket ticket, int cta, Tile &t) const { logit_tile<kCtas, kN>(l, n, ticket.i, cta, t); }
  __device__ __forceinline__ void epilogue(Ticket ticket, int cta, const Accumulator &acc, float (&g)[kN / 2]) {
    constexpr int kCols = kN / 2;
    int row0;
    int64_t v0;
    logit_tile_at<kCtas, kN>(l, n, ticket.i, row0, v0);
    v0 += acc.half * kCols;
    row0 += cta * 128 + acc.warp * 32;
    const int row = row0 + acc.lane;
    float lse = 0.f, coef = 0.f, at_token = 0.f;
    int y = -1;
    if (row < n) {
      const int r = l.rows.row(row);
      y = p.tokens[r];
      if (y >= 0 && y < l.vocab) {
        lse = p.lse[r];
        coef = p.coef[r];
        at_token = coef * expm1f(p.logprob[r]);  // p - 1 without the cancellation
      } else {
        y = -1;
        if (p.status && v0 == 0) atomicOr(p.status, FOPD_DEV_BAD_TOKEN);
      }
    }
    const bool live = coef != 0.f;
#pragma unroll
    for (int j = 0; j < kCols; ++j) g[j] = live ? coef * ex2((g[j] - lse) * kLog2e) : 0.f;
    const int64_t mine = (int64_t)y - v0;
    if (live && mine >= 0 && mine < kCols) {
      const int at = (int)mine;
#pragma unroll
      for (int j = 0; j < kCols; ++j) asm("{\n.reg .pred p;\nsetp.eq.s32 p, %1, %2;\nselp.f32 %0, %3, %0, p;\n}" : "+f"(g[j]) : "r"(at), "r"(j), "f"(at_token));
    }
    if (v0 + kCols > l.vocab) {
      const int have = (int)max((int64_t)0, l.vocab - v0);
#pragma unroll
      for (int j = 0; j < kCols; ++j)
        if (j >= have) g[j] = 0.f;
    }
    const int panel0 = (int)((v0 - (int64_t)l.v_tile0 * kN) / 64);
    const auto put = [&](const float *g, int c) {
      for (int plane = 0; plane < (v0 + c >= l.vocab ? 0 : p.lo ? 2 : 1); ++plane) {
        const uint32_t at = staging.next(acc);
        stage_box(at, acc.lane, [&](int j) {
          const float a = g[2 * j], b = g[2 * j + 1];
          __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
          if (plane) h = __floats2bfloat162_rn(a - __low2float(h), b - __high2float(h));
          return *reinterpret_cast<uint32_t *>(&h);
        });
        staging.send(acc, &p.panels_out, 0, (panel0 + c / 64) * p.pitch + row0 + plane * p.lo, at);
      }
    };
    put(g, 0);
    if (kCols > 64) put(g + 64, 64);
  }
};

// ------------------------------------------------------------------ gradients of hidden states and weights
// d_hidden's tiles run along the piece's columns, cut into `splits` where there are too few of them, and are added up in fp32
// (in the workspace, in a fixed order); d_weight's run along the rows and are finished.
template <int kCtas, int kN>
struct HeadGradsJob {
  static constexpr bool kFp16 = false, kTurns = false, kClaimed = false;
  using Ticket = TileNumber;
  struct Params {
    CUtensorMap hidden, weight, panels, panels_along;
    HeadRows rows;
    int64_t vocab, v0;   // first column of the piece
    int dim, v_count;    // columns of the piece
    int pitch, lo;       // of a panel; from plane to plane
    int splits;          // 0: no d_hidden
    int split_panels;    // panels to a split
    int first;           // the first piece sets, the others add
    float *sum;          // [splits][pitch][sum_pitch]
    int sum_pitch;
    void *d_weight;      // or NULL
    int64_t d_weight_pitch;
    int d_weight_f32, add;
    int32_t *status;
  };
  static constexpr int kRows = kCtas * 128;
  const Params &p;
  int n, m_tiles, d_tiles, v_tiles;
  int64_t n_hidden;
  __device__ explicit HeadGradsJob(const Params &params) : p(params), n(params.rows.count()) {
    m_tiles = (n + kRows - 1) / kRows;
    d_tiles = (p.dim + kN - 1) / kN;
    v_tiles = (p.v_count + kRows - 1) / kRows;
    n_hidden = (int64_t)p.splits * m_tiles * d_tiles;
  }
  __device__ int64_t tiles() const { return n_hidden + (p.d_weight ? (int64_t)v_tiles * d_tiles : 0); }
  __device__ int32_t *status() const { return p.status; }
  // hidden: (split, row0, d0); weight: (-1, row of the piece, d0)
  __device__ __forceinline__ void at(int64_t i, int &split, int &row0, int &d0) const {
    if (i < n_hidden) {
      split = (int)(i / ((int64_t)m_tiles * d_tiles));
      const int r = (int)(i - (int64_t)split * m_tiles * d_tiles);
      row0 = r / d_tiles * kRows;
      d0 = r % d_tiles * kN;
    } else {
      i -= n_hidden;
      split = -1;
      row0 = (int)(i / d_tiles) * kRows;
      d0 = (int)(i % d_tiles) * kN;
    }
  }
  __device__ __forceinline__ void tile(Ticket ticket, int cta, Tile &t) const {
    int split, row0, d0;
    at(ticket.i, split, row0, d0);
    row0 += cta * 128;
    d0 += cta * (kN / kCtas);
    if (split >= 0) {
      const int panels = (p.v_count + 63) / 64, first = split * p.split_panels;
      t.a = {&p.panels_along, 0, first * p.pitch + row0, 0, p.pitch, 0, 128, 0, false};
      t.b = {&p.weight, d0, (int)p.v0 + first * 64, 0, 64, 64, 0, 0, true};
      t.k_blocks = max(0, min(p.split_panels, panels - first));
      t.chunk = 0;
      t.passes = 1;
      t.a_lo = 0;
    } else {
      t.a = {&p.panels, 0, row0 / 64 * p.pitch, 0, 64, 0, p.pitch, p.lo, true};
      t.b = {&p.hidden, d0, 0, 0, 64, 64, 0, 0, true};
      t.k_blocks = (n + 63) / 64;
      t.chunk = p.lo ? kLogitChunk : 0;
      t.passes = p.lo ? 2 : 1;
      t.a_lo = p.lo ? 1 : 0;  // (the small terms first)
    }
    t.b_lo = 0;
  }
  __device__ __forceinline__ void epilogue(Ticket ticket, int cta, const Accumulator &acc, float (&g)[kN / 2]) const {
    int split, row0, d0;
    at(ticket.i, split, row0, d0);
    d0 += acc.half * (kN / 2);
    const int row = row0 + cta * 128 + acc.warp * 32 + acc.lane;
    if (split >= 0) {
      if (row >= n) return;
      float *out = p.sum + ((int64_t)split * p.pitch + row) * p.sum_pitch + d0;
#pragma unroll
      for (int j = 0; j < kN / 2; j += 4) {
        if (d0 + j >= p.dim) continue;  // (sum_pitch is a multiple of 32)
        float4 *q = reinterpret_cast<float4 *>(out + j);
        float4 v = make_float4(g[j], g[j + 1], g[j + 2], g[j + 3]);
        if (!p.first) {
          const float4 o = *q;
          v.x += o.x, v.y += o.y, v.z += o.z, v.w += o.w;
        }
        *q = v;
      }
      return;
    }
    if (row >= p.v_count) return;
    const int64_t at = (p.v0 + row) * p.d_weight_pitch + d0;
    char *out = static_cast<char *>(p.d_weight);
    if (p.d_weight_f32) store_row<FOPD_F32, kN / 2>(out + at * 4, g, d0, p.dim, p.add);
    else store_row<FOPD_BF16, kN / 2>(out + at * 2, g, d0, p.dim, p.add);
  }
};

// d_hidden from the splits' sums, added in order, rows back in their places.  What the rounding to bf16 left of the token's own
// entry of G, as a rule by far the largest of its row, is added here in fp32 (one row of the weights per row).
__global__ void __launch_bounds__(128) head_hidden_kernel(HeadRows rows, const float *sum, int splits, int pitch, int sum_pitch,
                                                          const int32_t *tokens, const float *logprob, const float *coef,
                                                          const __nv_bfloat16 *weight, int64_t weight_pitch, int64_t vocab, int dim,
                                                          int64_t out_pitch, __nv_bfloat16 *out) {
  const int n = rows.count();
  for (int r = blockIdx.x; r < n; r += gridDim.x) {
    const int row = rows.row(r), y = tokens[row];
    const bool known = y >= 0 && y < vocab;
    const float c = known ? coef[row] : 0.f, g = c != 0.f ? c * expm1f(logprob[row]) : 0.f;
    const float left = g - __bfloat162float(__float2bfloat16_rn(g));
    const __nv_bfloat16 *w = weight + (known ? y : 0) * weight_pitch;
    __nv_bfloat16 *o = out + (int64_t)row * out_pitch;
    for (int d = threadIdx.x * 8; d < dim; d += 128 * 8) {
      float x[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
      for (int s = 0; s < splits; ++s) {
        const float4 *q = reinterpret_cast<const float4 *>(sum + ((int64_t)s * pitch + r) * sum_pitch + d);
        const float4 a = q[0], b = q[1];
        x[0] += a.x, x[1] += a.y, x[2] += a.z, x[3] += a.w, x[4] += b.x, x[5] += b.y, x[6] += b.z, x[7] += b.w;
      }
      if (d + 8 <= dim) {
        if (left != 0.f) {
          float v[8];
          Elem<FOPD_BF16>::unpack(*reinterpret_cast<const uint4 *>(w + d), v);
#pragma unroll
          for (int e = 0; e < 8; ++e) x[e] = fmaf(left, v[e], x[e]);
        }
        *reinterpret_cast<uint4 *>(o + d) = Elem<FOPD_BF16>::pack(x);
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (d + e < dim) o[d + e] = __float2bfloat16_rn(left != 0.f ? fmaf(left, __bfloat162float(w[d + e]), x[e]) : x[e]);
      }
    }
  }
}

}  // namespace fopd
