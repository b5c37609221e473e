// Orthogonalised updates: argument checks, scales, workspaces, launches.
#include <algorithm>
#include <vector>

#include "host_ranges.cuh"
#include "orth_kernels.cuh"
#include "tensor_host.cuh"

using namespace fopd;

namespace {

constexpr int kMostSteps = kOrthMostSteps;
constexpr int kGroup = 240;                               // matrices of one table
constexpr int64_t kGroupBytes = (int64_t)1 << 30;         // workspace of one group, unless a single matrix takes more
constexpr int64_t kFewAcross = 16, kFewAlong = 256;       // sides up to which roundings do not average out
constexpr float kLoud = 32.f;                             // amplification ahead from which X keeps its second plane

int check_matrices(const fopd_matrix *t, int32_t n) {
  if (n < 0) return FOPD_ERR_SIZE;
  if (n > 0 && !t) return FOPD_ERR_NULL;
  for (int32_t i = 0; i < n; ++i) {
    const fopd_matrix &m = t[i];
    if ((m.dtype != FOPD_BF16 && m.dtype != FOPD_F32) || (m.out_dtype != FOPD_BF16 && m.out_dtype != FOPD_F32)) return FOPD_ERR_DTYPE;
    if (!std::isfinite(m.scale)) return FOPD_ERR_PARAM;
    const int64_t most = (int64_t)1 << 24;
    if (m.rows < 0 || m.cols < 0 || m.rows > most || m.cols > most) return FOPD_ERR_SIZE;
    if (m.rows == 0 || m.cols == 0) continue;
    if (m.rows > 1 && (m.row_stride < m.cols || m.out_stride < m.cols || m.row_stride > (int64_t)1 << 32 || m.out_stride > (int64_t)1 << 32))
      return FOPD_ERR_SIZE;
    // (workspace rows of 64 elements are counted in 31 bits: four planes of the matrix and of its shorter side's square)
    const int64_t rp = round_up(m.rows, 64), cp = round_up(m.cols, 64), mp = std::min(rp, cp);
    if (4 * (rp * cp + mp * mp) / 64 > (int64_t)1 << 30) return FOPD_ERR_SIZE;
    if (!m.data || !m.out) return FOPD_ERR_NULL;
    if ((uintptr_t)m.data % (m.dtype == FOPD_BF16 ? 2 : 4) != 0 || (uintptr_t)m.out % (m.out_dtype == FOPD_BF16 ? 2 : 4) != 0)
      return FOPD_ERR_ALIGN;
  }
  return FOPD_OK;
}

int check_outputs(const fopd_matrix *t, int32_t n) {
  std::vector<Range> in, out;
  in.reserve(n);
  for (int32_t i = 0; i < n; ++i) {
    const fopd_matrix &m = t[i];
    if (m.rows == 0 || m.cols == 0) continue;
    const bool in_place = m.out == m.data && m.dtype == m.out_dtype && (m.rows == 1 || m.row_stride == m.out_stride);
    in.push_back(range_of(m.data, m.rows, m.cols, m.row_stride, m.dtype == FOPD_BF16 ? 2 : 4, i, in_place));
    if (!in_place) out.push_back(range_of(m.out, m.rows, m.cols, m.out_stride, m.out_dtype == FOPD_BF16 ? 2 : 4, i, true));
  }
  return check_ranges(in, out);
}

// The scales of every step from a bound on the largest singular value before it.
struct Scales {
  OrthStep step[kMostSteps];
  uint32_t loud;  // bit k: the steps from k on amplify by kLoud or more
};
int exponent_below(double bound) {  // bound * 2^e in (2^14, 2^15]
  int e = 0;
  const double f = std::frexp(bound, &e);
  return 15 - (f == 0.5 ? e - 1 : e);
}
int make_scales(const float *coefficients, int32_t steps, Scales *s) {
  double most = 1.0;  // |M| / (|M| + eps) <= 1
  int ex = 0, fall = 0;
  double ahead = 1.0;
  s->loud = 0;
  for (int k = steps - 1; k >= 0; --k) {
    ahead *= std::fabs((double)coefficients[3 * k]);
    if (ahead >= kLoud) s->loud |= 1u << k;
  }
  for (int k = 0; k < steps; ++k) {
    const double a = coefficients[3 * k], b = coefficients[3 * k + 1], c = coefficients[3 * k + 2], l = most * most;
    if (!std::isfinite(a) || !std::isfinite(b) || !std::isfinite(c)) return FOPD_ERR_PARAM;
    // largest |a + b x + c x^2| for x in [0, l], largest |s (a + b s^2 + c s^4)| for s in [0, most]
    const auto poly = [&](double x) { return a + x * (b + x * c); };
    double p = std::max(std::fabs(poly(0.0)), std::fabs(poly(l))), next = most * std::fabs(poly(l));
    if (c != 0.0 && -b / (2 * c) > 0.0 && -b / (2 * c) < l) p = std::max(p, std::fabs(poly(-b / (2 * c))));
    const double disc = 9 * b * b - 20 * a * c;  // a + 3 b x + 5 c x^2 = 0
    double roots[2] = {-1.0, -1.0};
    if (c != 0.0 && disc >= 0.0) {
      roots[0] = (-3 * b + std::sqrt(disc)) / (10 * c);
      roots[1] = (-3 * b - std::sqrt(disc)) / (10 * c);
    } else if (c == 0.0 && b != 0.0) {
      roots[0] = -a / (3 * b);
    }
    for (double x : roots)
      if (x > 0.0 && x < l) next = std::max(next, std::sqrt(x) * std::fabs(poly(x)));
    p = std::max(p, 1e-6);
    next = std::max(next, 1e-6) * 1.001;  // (the scales leave a factor of two above it)
    if (p > 1e6 || next > 1e6) return FOPD_ERR_PARAM;
    const int ea = exponent_below(l), ep = exponent_below(p), ex_next = k + 1 < steps ? exponent_below(next) : 0;
    OrthStep &o = s->step[k];
    o.gram = (float)std::ldexp(1.0, k == 0 ? ea : ea - 2 * ex);
    o.poly_a = (float)std::ldexp(a, ep);
    o.poly_b = (float)std::ldexp(b, ep - ea);
    o.poly_c = (float)std::ldexp(c, ep - 2 * ea);
    o.apply = (float)std::ldexp(1.0, (k == 0 ? 0 : -ex) - ep + ex_next);
    // (singular values of at most 2^-lift most come out at most p times as large, and have room up to next)
    o.fall = fall;
    fall += std::max(0, (int)std::ceil(std::log2(most * p / next)));
    ex = ex_next;
    most = next;
  }
  return FOPD_OK;
}

// One matrix's entry but for where it starts.
OrthMatrix describe(const fopd_matrix &m, const Scales &s, int32_t steps) {
  OrthMatrix o = {};
  o.data = m.data;
  o.out = m.out;
  o.pitch = m.rows > 1 ? m.row_stride : m.cols;
  o.out_pitch = m.rows > 1 ? m.out_stride : m.cols;
  o.rows = (int)m.rows;
  o.cols = (int)m.cols;
  o.rp = (int)round_up(m.rows, 64);
  o.cp = (int)round_up(m.cols, 64);
  o.tall = m.rows > m.cols;
  o.mp = o.tall ? o.cp : o.rp;
  o.scale = m.scale;
  o.dtype = (uint8_t)m.dtype;
  o.out_dtype = (uint8_t)m.out_dtype;
  // (the roundings of a few numbers do not average out, and a singular value that passes 1.15 on its way makes three times of them: A
  // and P have as many as the shorter side says, X as both)
  const bool thin = std::min(m.rows, m.cols) <= kFewAcross, few = thin && std::max(m.rows, m.cols) <= kFewAlong;
  o.held = m.out_dtype == FOPD_F32 || few ? kOrthFull : thin ? kOrthSquare : kOrthPlain;
  const uint32_t all = (1u << steps) - 1;
  o.two_planes = o.full() ? all : s.loud & all;
  if (m.dtype == FOPD_BF16) o.two_planes &= ~1u;  // (bf16 values are whole in the first plane)
  const int64_t x = (int64_t)o.rp * o.cp / 64, a = (int64_t)o.mp * o.mp / 64;
  uint32_t in_turn[2] = {0, 0};
  for (int k = 0; k < steps; ++k) in_turn[k & 1] |= o.two_planes >> k & 1;
  int64_t at = 0;
  o.x_lo = (int)x;
  for (int k = 0; k < 2; ++k) {
    o.x[k] = (int)at;
    at += x * (1 + in_turn[k]);
  }
  o.m_lo = (int)a;
  o.a = (int)at;
  at += a * (1 + o.square());
  o.p = (int)at;
  at += a * (1 + o.square());
  o.space = (int)at;
  return o;
}

// The launches of one group.
struct Group {
  OrthWorkspace ws;
  CUtensorMap boxes, boxes_along, rows_out;
  int norm_blocks, load_blocks, norm_chunk, load_cols;
  int64_t sym_tiles, x_tiles;
  bool pairs;  // tiles of 256 x 256 on pairs of CTAs
};
template <int N>
int run_table(const std::vector<OrthMatrix> &g, const Group &o, const Scales &s, int32_t steps, float eps, int32_t *status, int sms,
              cudaStream_t st) {
  OrthTable<N> tab;
  tab.n = (int)g.size();
  tab.norm_chunk = o.norm_chunk;
  tab.load_cols = o.load_cols;
  std::copy(g.begin(), g.end(), tab.m);
  int rc = launch_early(orth_norm_kernel<N>, dim3((unsigned)o.norm_blocks), kOrthThreads, st, tab, o.ws);
  if (rc == FOPD_OK) rc = launch_early(orth_load_kernel<N>, dim3((unsigned)o.load_blocks), kOrthThreads, st, tab, o.ws, eps, status);
  if (rc != FOPD_OK) return rc;
  const auto run = [&](auto p, auto launch) {
    p.boxes = o.boxes;
    p.boxes_along = o.boxes_along;
    p.rows_out = o.rows_out;
    p.ws = o.ws;
    std::copy(s.step, s.step + steps, p.step);
    p.tab = tab;
    p.steps = steps;
    p.sym_tiles = (int)o.sym_tiles;
    p.x_tiles = (int)o.x_tiles;
    p.status = status;
    return launch(p, std::max(o.x_tiles, o.sym_tiles), sms, st);
  };
  using Pairs = OrthJob<2, 256, N>;
  using Single = OrthJob<1, 128, N>;
  return o.pairs ? run(typename Pairs::Params(), launch_product<2, 256, Pairs>) : run(typename Single::Params(), launch_product<1, 128, Single>);
}

// Tiles of 256 x 256 on pairs of CTAs, or of 128 x 128 on single ones?  In units of a pair's time for 256 x 256 x 64 products a single one's
// 128 x 128 x 64 take 0.6 (where sums are taken out every other block 0.43: four accumulators hide that better than two).  Small tiles
// waste less at the edges and are more in number; a phase takes as long as its share on each CTA, and no less than one tile.
bool pairs_pay(const std::vector<OrthMatrix> &g, int sms) {
  double cost[2];
  for (int v = 0; v < 2; ++v) {
    const int tile = v ? 256 : 128, slots = v ? sms / 2 : sms;
    double units[3] = {0, 0, 0}, longest[3] = {0, 0, 0};
    for (const OrthMatrix &m : g) {
      const double t = (m.mp + tile - 1) / tile, n_sym = t * (t + 1) / 2, n_x = (double)((m.rp + tile - 1) / tile) * ((m.cp + tile - 1) / tile);
      const double unit = v ? 1.0 : m.full() ? 0.43 : 0.6, other = m.tall ? m.rp : m.cp;
      const double each[3] = {other / 64 * (m.full() ? 3 : 1) * unit, m.mp / 64 * (m.square() ? 3 : 1) * unit,
                              m.mp / 64 * (m.full() ? 3 : m.square() ? 2 : 1) * unit};
      for (int k = 0; k < 3; ++k) {
        units[k] += (k < 2 ? n_sym : n_x) * each[k];
        longest[k] = std::max(longest[k], each[k]);
      }
    }
    cost[v] = 0;
    for (int k = 0; k < 3; ++k) cost[v] += std::max(units[k] / slots, longest[k]);
  }
  return cost[1] <= cost[0];
}

int run_group(std::vector<OrthMatrix> &g, const Scales &s, int32_t steps, float eps, int32_t *status, int sms, cudaStream_t st) {
  // the largest first: their phases take longest, and the small ones' tiles fill what is left
  std::stable_sort(g.begin(), g.end(), [](const OrthMatrix &a, const OrthMatrix &b) { return (int64_t)a.rp * a.cp > (int64_t)b.rp * b.cp; });
  // (short lists in small blocks: their norm and load are latencies)
  int64_t elements = 0;
  for (const OrthMatrix &m : g) elements += (int64_t)m.rows * m.cols;
  const bool small = elements < (int64_t)1 << 22;
  const int norm_chunk = small ? 4096 : 16384, load_cols = small ? 64 : 256;
  int64_t at = 0, norm_blocks = 0, load_blocks = 0;
  for (size_t i = 0; i < g.size(); ++i) {
    OrthMatrix &m = g[i];
    m.x[0] += (int)at, m.x[1] += (int)at, m.a += (int)at, m.p += (int)at;
    at += m.space;
    m.norm_block = (int)norm_blocks;
    m.norm_blocks = (int)(((int64_t)m.rows * m.cols + norm_chunk - 1) / norm_chunk);
    norm_blocks += m.norm_blocks;
    m.load_block = (int)load_blocks;
    load_blocks += (int64_t)(m.rp / 64) * ((m.cp + load_cols - 1) / load_cols);
  }
  const int tile = pairs_pay(g, sms) ? 256 : 128;
  int64_t sym_tiles = 0, x_tiles = 0;
  for (OrthMatrix &m : g) {
    const int64_t t = (m.mp + tile - 1) / tile;
    m.sym_tile = (int)sym_tiles;
    m.x_tile = (int)x_tiles;
    sym_tiles += t * (t + 1) / 2;
    x_tiles += ((int64_t)(m.rp + tile - 1) / tile) * ((m.cp + tile - 1) / tile);
  }
  Layout lay;
  const int64_t planes = lay.take(at * 128), norm = lay.take((int64_t)(g.size() * sizeof(OrthNorm))), lifted = lay.take(4),
                done = lay.take(((int64_t)g.size() + 1) * 4), partial = lay.take(norm_blocks * 8);
  char *base = nullptr;
  int rc = scratch_alloc(reinterpret_cast<void **>(&base), (size_t)lay.bytes, st);
  if (rc != FOPD_OK) return rc;
  Group o;
  o.ws = {reinterpret_cast<OrthNorm *>(base + norm), reinterpret_cast<int *>(base + lifted), reinterpret_cast<int *>(base + done),
          reinterpret_cast<double *>(base + partial), reinterpret_cast<__half *>(base + planes)};
  o.norm_blocks = (int)norm_blocks;
  o.load_blocks = (int)load_blocks;
  o.norm_chunk = norm_chunk;
  o.load_cols = load_cols;
  o.sym_tiles = sym_tiles;
  o.x_tiles = x_tiles;
  o.pairs = tile == 256;
  rc = make_map(&o.boxes, CU_TENSOR_MAP_DATA_TYPE_FLOAT16, o.ws.planes, 64, at, 128, 64, kBoxRows);
  if (rc == FOPD_OK) rc = make_map(&o.rows_out, CU_TENSOR_MAP_DATA_TYPE_FLOAT16, o.ws.planes, 64, at, 128, 64, 32);
  if (rc == FOPD_OK) rc = make_map(&o.boxes_along, CU_TENSOR_MAP_DATA_TYPE_FLOAT16, o.ws.planes, 64, at, 128, 64, 2 * kBoxRows);
  if (rc == FOPD_OK) {
    const size_t n = g.size();
    rc = n <= 8    ? run_table<8>(g, o, s, steps, eps, status, sms, st)
         : n <= 64 ? run_table<64>(g, o, s, steps, eps, status, sms, st)
                   : run_table<kGroup>(g, o, s, steps, eps, status, sms, st);
  }
  if (cudaFreeAsync(base, st) == cudaSuccess) return rc;
  (void)cudaGetLastError();
  return rc == FOPD_OK ? FOPD_ERR_CUDA : rc;
}

}  // namespace

extern "C" {

int fopd_orthogonalise(const fopd_matrix *matrices, int32_t n, const float *coefficients, int32_t steps, float eps, int32_t *status,
                       void *stream) {
  int rc = check_matrices(matrices, n);
  if (rc != FOPD_OK) return rc;
  if (!coefficients) return FOPD_ERR_NULL;
  if (steps < 1 || steps > kMostSteps || !std::isfinite(eps) || eps < 0.f) return FOPD_ERR_PARAM;
  Scales s;
  rc = make_scales(coefficients, steps, &s);
  if (rc != FOPD_OK) return rc;
  try {
    rc = check_outputs(matrices, n);
    if (rc != FOPD_OK) return rc;
    int sms = 0;
    std::vector<OrthMatrix> group;
    int64_t total = 0;
    for (int32_t i = 0; i < n; ++i) {
      if (matrices[i].rows == 0 || matrices[i].cols == 0) continue;
      if (sms == 0 && (rc = current_sms(&sms)) != FOPD_OK) return rc;
      const OrthMatrix m = describe(matrices[i], s, steps);
      if (!group.empty() && ((int)group.size() == kGroup || (total + m.space) * 128 > kGroupBytes)) {
        rc = run_group(group, s, steps, eps, status, sms, static_cast<cudaStream_t>(stream));
        if (rc != FOPD_OK) return rc;
        group.clear();
        total = 0;
      }
      group.push_back(m);
      total += m.space;
    }
    return group.empty() ? FOPD_OK : run_group(group, s, steps, eps, status, sms, static_cast<cudaStream_t>(stream));
  } catch (...) {  // host memory for the table
    return FOPD_ERR_CUDA;
  }
}

}  // extern "C"
