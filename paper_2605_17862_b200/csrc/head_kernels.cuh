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

// The rows a launch works on: n from `first` on, or as many of those as there are among the *active first ones of a compacted copy.
struct HeadRows {
  int n, first;
  const int *active;  // DEVICE count, or NULL
  const int *index;   // compacted row -> row of the caller's, or NULL: the same
  __device__ __forceinline__ int count() const { return active ? max(0, min(n, *active - first)) : n; }
  __device__ __forceinline__ int row(int i) const { return index ? index[first + i] : first + i; }
};

// ------------------------------------------------------------------ rows that count, one after another
// Numbers the rows that count, copies their hidden states into place and clears the others' results, in one launch: a block takes
// `per` rows and counts those before them itself (nine bytes to a row, from the L2; at most 512 blocks do so).
constexpr int kCompactThreads = 256, kCompactBlocks = 512;
__global__ void __launch_bounds__(kCompactThreads) head_compact_kernel(const uint8_t *mask, const int32_t *tokens, const float *coef,
                                                                       int n, int per, int64_t vocab, const __nv_bfloat16 *hidden,
                                                                       int64_t pitch, int dim, int copy_pitch, __nv_bfloat16 *copy,
                                                                       int *index, int *active, float *logprob, float *lse,
                                                                       int32_t *status) {
  __shared__ int sums[kCompactThreads / 32], list[kCompactThreads];
  grid_wait();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const auto counts = [&](int i) {  // (all three are asked for at once)
    const bool on = mask[i] != 0, known = (uint32_t)tokens[i] < (uint64_t)vocab, weighs = coef ? coef[i] != 0.f : true;
    return on & known & weighs;
  };
  const auto sum_of = [&](int x) {  // over the block
    x = __reduce_add_sync(0xffffffffu, x);
    __syncthreads();
    if (lane == 0) sums[warp] = x;
    __syncthreads();
    int s = 0;
    for (int w = 0; w < kCompactThreads / 32; ++w) s += sums[w];
    return s;
  };
  const int first = blockIdx.x * per, end = min(n, first + per);
  int before = 0;
#pragma unroll 4
  for (int i = threadIdx.x; i < first; i += kCompactThreads) before += counts(i);
  before = sum_of(before);
  const auto copy_row = [&](int from, int to) {  // a warp
    const __nv_bfloat16 *src = from >= 0 ? hidden + (int64_t)from * pitch : nullptr;
    __nv_bfloat16 *dst = copy + (int64_t)to * copy_pitch;
#pragma unroll 4
    for (int d = lane * 8; d < dim; d += 256) {
      if (d + 8 <= dim) *reinterpret_cast<uint4 *>(dst + d) = src ? *reinterpret_cast<const uint4 *>(src + d) : make_uint4(0, 0, 0, 0);
      else
        for (int e = d; e < dim; ++e) dst[e] = src ? src[e] : __float2bfloat16_rn(0.f);
    }
  };
  for (int at = first; at < end; at += kCompactThreads) {
    const int i = at + threadIdx.x;
    const bool on = i < end && counts(i);
    const uint32_t vote = __ballot_sync(0xffffffffu, on);
    const int all = sum_of(lane == 0 ? __popc(vote) : 0);
    int place = before + __popc(vote & ((1u << lane) - 1));
    for (int w = 0; w < warp; ++w) place += sums[w];
    if (on) {
      index[place] = i;
      list[place - before] = i;
    }
    if (i < end && !on) {
      if (logprob) logprob[i] = 0.f;
      if (lse) lse[i] = 0.f;
      if (status && mask[i] != 0 && (uint32_t)tokens[i] >= (uint64_t)vocab) atomicOr(status, FOPD_DEV_BAD_TOKEN);
    }
    __syncthreads();
    for (int j = warp; j < all; j += kCompactThreads / 32) copy_row(list[j], before + j);
    before += all;
  }
  if (end == n && first < n) {  // the last block: the count, and zeros up to the next 64 rows, for products along the rows
    if (threadIdx.x == 0) *active = before;
    for (int r = before + warp; r < (before + 63) / 64 * 64; r += kCompactThreads / 32) copy_row(-1, r);
  }
}

// ------------------------------------------------------------------ tiles of logits
constexpr int kLogitChunk = 8;   // for logits whose error is to stay that of fp32 sums: 512 dimensions
constexpr int kGradChunk = 16;   // for those behind a weights' gradient in fp32, next to the 2^-17 that two planes leave
// Tiles of one CTA, up to 128 rows, wait for the weights and not for the tensor pipe: 1.5 % of the time for log-probs of large logits 5.4e-7 off
// instead of 1.6e-6 (fp32 products: 6.1e-7, 1 x 32,000 x 1,024).  With pairs it would be 45 %.
constexpr int kFewRowsChunk = 2;
struct LogitTiles {
  const CUtensorMap *hidden, *weight;
  HeadRows rows;
  int64_t vocab;
  int k_blocks;      // of 64 hidden dimensions
  int v_tile0, v_tiles;
  int chunk;         // blocks that a matrix instruction's accumulator adds up
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
  t.chunk = l.chunk;
  t.passes = 1;
  t.a_lo = t.b_lo = 0;
}

// ------------------------------------------------------------------ log-probs
// A tile's epilogue: two threads per row, each the maximum and the sum of exponentials of 128 logits (exponents as in RowSweep), the
// stored token's left out of the sum: the log-prob of a nearly certain token comes from the others' sum.
// 4,096 x 151,936 x 2,048: 1.83 to 1.89 ms, the tensor pipe's rate; 48 rows: 106 us, reading the weights at 5.9 TB/s (128 rows a tile, three
// stages of 48 KB on each SM in flight).
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
  int n, y = -1;  // this thread's row's token
  __device__ explicit LogprobJob(const Params &params) : p(params), l(params.l), n(params.l.rows.count()) {
    l.hidden = &p.hidden;
    l.weight = &p.weight;
  }
  __device__ int64_t tiles() const { return logit_tiles<kCtas, kN>(l, n); }
  __device__ int32_t *status() const { return p.status; }
  __device__ __forceinline__ void tile(Ticket ticket, int cta, Tile &t) const { logit_tile<kCtas, kN>(l, n, ticket.i, cta, t); }
  __device__ __forceinline__ void prefetch(Ticket ticket, int cta, const Accumulator &acc) {
    int row0;
    int64_t v0;
    logit_tile_at<kCtas, kN>(l, n, ticket.i, row0, v0);
    const int row = row0 + cta * 128 + acc.warp * 32 + acc.lane;
    y = row < n ? p.tokens[l.rows.row(row)] : -1;
  }
  __device__ __forceinline__ void epilogue(Ticket ticket, int cta, const Accumulator &acc, float (&z)[kN / 2]) const {
    constexpr int kCols = kN / 2;
    int row0;
    int64_t v0;
    logit_tile_at<kCtas, kN>(l, n, ticket.i, row0, v0);
    v0 += acc.half * kCols;
    const int row = row0 + cta * 128 + acc.warp * 32 + acc.lane;
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

// Joins the pieces of four rows: 64 threads to a row, merged in a fixed order; a row's last step in fp64.
constexpr int kJoinThreads = 256;
__global__ void __launch_bounds__(kJoinThreads) head_join_kernel(HeadRows rows, const float2 *part, const float *token_logit, int pieces,
                                                                 int pitch, const int32_t *tokens, int64_t vocab, float *logprob,
                                                                 float *lse, int32_t *status) {
  __shared__ float2 shared[kJoinThreads / 32][4];
  grid_wait();
  const int n = rows.count(), k = threadIdx.x & 3, r = blockIdx.x * 4 + k, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  if (blockIdx.x * 4 >= n) return;
  float m = kNegBig, s = 0.f;
  const auto merge = [&](float om, float os) {
    const float top = fmaxf(m, om);
    s = __fmaf_rn(s, ex2((m - top) * kLog2e), __fmul_rn(os, ex2((om - top) * kLog2e)));
    m = top;
  };
  constexpr int kAhead = 5;  // loads in flight
  for (int v = threadIdx.x >> 2; v < pieces; v += kAhead * (kJoinThreads / 4)) {
    float2 q[kAhead];
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
      const int w = v + j * (kJoinThreads / 4);
      q[j] = w < pieces && r < n ? part[(int64_t)w * pitch + r] : make_float2(kNegBig, 0.f);
    }
    float top = m;
#pragma unroll
    for (int j = 0; j < kAhead; ++j) top = fmaxf(top, q[j].x);
    s *= ex2((m - top) * kLog2e);
#pragma unroll
    for (int j = 0; j < kAhead; ++j) s = fmaf(q[j].y, ex2((q[j].x - top) * kLog2e), s);
    m = top;
  }
#pragma unroll
  for (int o = 4; o < 32; o <<= 1) merge(__shfl_xor_sync(0xffffffffu, m, o), __shfl_xor_sync(0xffffffffu, s, o));
  if (lane < 4) shared[warp][lane] = make_float2(m, s);
  __syncthreads();
  if (threadIdx.x >= 4 || r >= n) return;
  const int row = rows.row(r), y = tokens[row];
  if (y < 0 || y >= vocab) {  // (without a mask rows are not sorted out beforehand)
    logprob[row] = 0.f;
    if (lse) lse[row] = 0.f;
    if (status) atomicOr(status, FOPD_DEV_BAD_TOKEN);
    return;
  }
  m = kNegBig, s = 0.f;
  for (int w = 0; w < kJoinThreads / 32; ++w) merge(shared[w][k].x, shared[w][k].y);
  const float zy = token_logit[r], top = fmaxf(m, zy);
  const double d = (double)zy - (double)top, t = exp(d), rest = (double)s * exp((double)m - (double)top);
  logprob[row] = (float)(t > rest ? -log1p(rest / t) : d - log(rest + t));
  if (lse) lse[row] = (float)((double)top + log(rest + t));
}

// ------------------------------------------------------------------ gradient of the logits, a piece of the vocabulary
// G goes to panels: [panel of 64 columns][pitch rows][64], bf16; a second plane of what the rounding left where the weights'
// gradient is wanted in fp32.  One rounding to bf16 (2^-8 of an entry at most) is what a matrix instruction takes; it is of the size
// of the bf16 results' own.  Each tile's boxes go out by TMA while the next one's products run: 4,096 x 151,936 x 2,048 in 1.6 ms, the tensor pipe
// 91 to 92 % busy.
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
  int y = -1;  // this thread's row: token, lse, coefficient, entry of G at the token
  float lse = 0.f, coef = 0.f, at_token = 0.f;
  __device__ explicit GradLogitsJob(const Params &params) : p(params), l(params.l), n(params.l.rows.count()) {
    l.hidden = &p.hidden;
    l.weight = &p.weight;
  }
  __device__ int64_t tiles() const { return logit_tiles<kCtas, kN>(l, n); }
  __device__ int32_t *status() const { return p.status; }
  __device__ __forceinline__ void tile(Ticket ticket, int cta, Tile &t) const { logit_tile<kCtas, kN>(l, n, ticket.i, cta, t); }
  __device__ __forceinline__ void prefetch(Ticket ticket, int cta, const Accumulator &acc) {
    int row0;
    int64_t v0;
    logit_tile_at<kCtas, kN>(l, n, ticket.i, row0, v0);
    const int row = row0 + cta * 128 + acc.warp * 32 + acc.lane;
    lse = coef = at_token = 0.f;
    y = -1;
    if (row >= n) return;
    const int r = l.rows.row(row), token = p.tokens[r];
    const float c = p.coef[r], lp = p.logprob[r], z = p.lse[r];
    if (token >= 0 && token < l.vocab) {
      y = token;
      lse = z;
      coef = c;
      at_token = c * expm1f(lp);  // p - 1 without the cancellation
    } else if (p.status && v0 == 0 && acc.half == 0) {
      atomicOr(p.status, FOPD_DEV_BAD_TOKEN);
    }
  }
  __device__ __forceinline__ void epilogue(Ticket ticket, int cta, const Accumulator &acc, float (&g)[kN / 2]) {
    constexpr int kCols = kN / 2;
    int row0;
    int64_t v0;
    logit_tile_at<kCtas, kN>(l, n, ticket.i, row0, v0);
    v0 += acc.half * kCols;
    row0 += cta * 128 + acc.warp * 32;
    // coef e^{z - lse} with the exponent in one fused multiply-add; the rounding of lse log2(e), the same for the whole row, goes into the
    // coefficient.  Rows without one: an exponential of zero.
    const bool live = coef != 0.f;
    const float c = live ? lse * kLog2e : 1e30f, scale = live ? coef * (1.f - fmaf(lse, kLog2e, -c) * kLn2) : 0.f;
#pragma unroll
    for (int j = 0; j < kCols; ++j) g[j] = scale * ex2(fmaf(g[j], kLog2e, -c));
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
    static_assert(kCols == 128, "two panels");
    put(g, 0);
    put(g + 64, 64);
  }
};

// ------------------------------------------------------------------ gradients of hidden states and weights
// d_hidden's tiles run along the piece's columns, cut into `splits` where there are too few of them, and are added up in fp32
// (in the workspace, in a fixed order); d_weight's run along the rows and are finished.  Both in one launch, the long tiles first:
// 4,096 x 151,936 x 2,048 in 3.3 ms of products at 88 to 90 % of the tensor pipe; with 100 rows, where d_hidden alone would be four tiles,
// 33 us for 32,000 x 1,024.
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
    CUtensorMap d_weight_out;  // boxes of 32 rows x 128 bytes
    int d_weight_boxes;        // it is stored by way of those
    void *d_weight;      // or NULL
    int64_t d_weight_pitch;
    int d_weight_f32, add;
    int32_t *status;
  };
  static constexpr int kRows = kCtas * 128;
  const Params &p;
  Staging staging;
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
      t.chunk = kLongChunk;
      t.passes = 1;
      t.a_lo = 0;
    } else {
      t.a = {&p.panels, 0, row0 / 64 * p.pitch, 0, 64, 0, p.pitch, p.lo, true};
      t.b = {&p.hidden, d0, 0, 0, 64, 64, 0, 0, true};
      t.k_blocks = (n + 63) / 64;
      t.chunk = p.lo ? kLogitChunk : kLongChunk;
      t.passes = p.lo ? 2 : 1;
      t.a_lo = p.lo ? 1 : 0;  // (the small terms first)
    }
    t.b_lo = 0;
  }
  __device__ __forceinline__ void prefetch(Ticket, int, const Accumulator &) const {}
  __device__ __forceinline__ void epilogue(Ticket ticket, int cta, const Accumulator &acc, float (&g)[kN / 2]) {
    int split, row0, d0;
    at(ticket.i, split, row0, d0);
    d0 += acc.half * (kN / 2);
    const int row = row0 + cta * 128 + acc.warp * 32 + acc.lane;
    if (split >= 0) {  // (sum_pitch is a multiple of 32)
      const uint32_t at = staging.idle(acc);
      float *out = p.sum + ((int64_t)split * p.pitch + row - acc.lane) * p.sum_pitch + d0;
#pragma unroll
      for (int c = 0; c < kN / 2; c += 32)
        put_rows_out<FOPD_F32>(at, acc.lane, g + c, out + c, p.sum_pitch, min(32, n - (row - acc.lane)), d0 + c < p.dim ? 32 : 0, !p.first);
      return;
    }
    if (p.d_weight_boxes) {  // (rows and columns that do not exist are left out by the copy)
      const int64_t row_out = p.v0 + row - acc.lane;
      if (row - acc.lane >= p.v_count) return;
      const auto send = [&](const float *v, int d) {  // 128 bytes of each row
        if (d >= p.dim) return;
        const uint32_t at = staging.next(acc);
        if (p.d_weight_f32) stage_box(at, acc.lane, [&](int j) { return __float_as_uint(v[j]); });
        else
          stage_box(at, acc.lane, [&](int j) {
            const __nv_bfloat162 h = __floats2bfloat162_rn(v[2 * j], v[2 * j + 1]);
            return *reinterpret_cast<const uint32_t *>(&h);
          });
        staging.send(acc, &p.d_weight_out, d, (int)row_out, at);
      };
      static_assert(kN == 256, "four boxes of 32 columns, two of 64");
      if (p.d_weight_f32) {
        send(g, d0);
        send(g + 32, d0 + 32);
        send(g + 64, d0 + 64);
        send(g + 96, d0 + 96);
      } else {
        send(g, d0);
        send(g + 64, d0 + 64);
      }
      return;
    }
    const uint32_t at = staging.idle(acc);
    const int rows = min(32, p.v_count - (row - acc.lane));
    const int64_t first = (p.v0 + row - acc.lane) * p.d_weight_pitch + d0;
    if (p.d_weight_f32) {
#pragma unroll
      for (int c = 0; c < kN / 2; c += 32)
        put_rows_out<FOPD_F32>(at, acc.lane, g + c, static_cast<float *>(p.d_weight) + first + c, p.d_weight_pitch, rows, min(32, p.dim - d0 - c), p.add);
    } else {
#pragma unroll
      for (int c = 0; c < kN / 2; c += 64)
        put_rows_out<FOPD_BF16>(at, acc.lane, g + c, static_cast<__nv_bfloat16 *>(p.d_weight) + first + c, p.d_weight_pitch, rows,
                                min(64, p.dim - d0 - c), p.add);
    }
  }
};

// d_hidden from the splits' sums, rows back in their places: a thread takes four dimensions of a row and the splits in order, or where
// there are many, one of eight threads an eighth of them in order.  What the rounding to bf16 left of the token's own entry of G, as a
// rule by far the largest of its row, is added here in fp32 (one row of the weights per row).
template <int kGroups>
__global__ void __launch_bounds__(256) head_hidden_kernel(HeadRows rows, const float *sum, int splits, int pitch, int sum_pitch,
                                                          const int32_t *tokens, const float *logprob, const float *coef,
                                                          const __nv_bfloat16 *weight, int64_t weight_pitch, int64_t vocab, int dim,
                                                          int64_t out_pitch, __nv_bfloat16 *out) {
  constexpr int kLanes = 256 / kGroups;
  __shared__ float4 part[kGroups][kLanes];
  grid_wait();
  const int lane = threadIdx.x % kLanes, group = threadIdx.x / kLanes, n = rows.count(), d = (blockIdx.y * kLanes + lane) * 4;
  const int per = (splits + kGroups - 1) / kGroups, first = group * per, end = min(splits, first + per);
  for (int r = blockIdx.x; r < n; r += gridDim.x) {
    float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
    if (d < dim) {
      const float4 *q = reinterpret_cast<const float4 *>(sum + ((int64_t)first * pitch + r) * sum_pitch + d);
#pragma unroll 4
      for (int s = first; s < end; ++s, q += (int64_t)pitch * sum_pitch / 4) {
        const float4 a = *q;
        x.x += a.x, x.y += a.y, x.z += a.z, x.w += a.w;
      }
    }
    if constexpr (kGroups > 1) {
      part[group][lane] = x;
      __syncthreads();
      for (int g = 1; group == 0 && g < kGroups && g * per < splits; ++g) {
        const float4 a = part[g][lane];
        x.x += a.x, x.y += a.y, x.z += a.z, x.w += a.w;
      }
    }
    if (group == 0 && d < dim) {
      const int row = rows.row(r), y = tokens[row];
      const bool known = y >= 0 && y < vocab;
      const float c = known ? coef[row] : 0.f, g = c != 0.f ? c * expm1f(logprob[row]) : 0.f;
      const float left = g - __bfloat162float(__float2bfloat16_rn(g));
      const __nv_bfloat16 *w = weight + (known ? y : 0) * weight_pitch + d;
      __nv_bfloat16 *o = out + (int64_t)row * out_pitch + d;
      float v[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (d + e < dim && left != 0.f) v[e] = fmaf(left, __bfloat162float(w[e]), v[e]);
      if (d + 4 <= dim) {
        const __nv_bfloat162 a = __floats2bfloat162_rn(v[0], v[1]), b = __floats2bfloat162_rn(v[2], v[3]);
        *reinterpret_cast<uint2 *>(o) = make_uint2(*reinterpret_cast<const uint32_t *>(&a), *reinterpret_cast<const uint32_t *>(&b));
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (d + e < dim) o[e] = __float2bfloat16_rn(v[e]);
      }
    }
    if constexpr (kGroups > 1) __syncthreads();
  }
}

}  // namespace fopd
