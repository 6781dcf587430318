// Orthogonalised updates: X = G / (|G| + eps), then X <- a X + (b A + c A^2) X with A = X X^T, some steps of it
// (Newton-Schulz: an odd polynomial of X that takes its singular values towards one), for a batch of matrices; and the
// update of the TT cores by it, slice by slice, with momentum.
#include <math.h>
#include <string.h>

#include "tt_gemm_device.h"
#include "tt_ortho_slice.h"

namespace {
using namespace ttg;

size_t pad256(size_t n) { return (n + 255) & ~(size_t)255; }

struct Steps {
  int n;
  const float *c;  // HOST [n][3]
};
struct Mats {
  long long batch;
  int rows, cols;
  long long b_step, r_step;
};

// ---- norm and scaling ------------------------------------------------------------------------------
// Sums of squares in 64 bits: neither 1e-25 nor 1e25 leaves the range, and the scale is not what limits the result.
constexpr int kMaxParts = 1024;
int parts_of(long long elems) {
  long long p = (elems + 4095) / 4096;
  return (int)(p < 1 ? 1 : p > kMaxParts ? kMaxParts : p);
}
// the place of element e of a matrix (a 64-bit division costs as much as the rest)
__device__ __forceinline__ long long place_of(const Mats &m, long long e, bool small) {
  const long long r = small ? (long long)((unsigned)e / (unsigned)m.cols) : e / m.cols;
  return r * m.r_step + (e - r * m.cols);
}
__device__ __forceinline__ double block_sum(double s) {
  __shared__ double red[TT_BLOCK];
  red[threadIdx.x] = s;
  __syncthreads();
  for (int o = TT_BLOCK / 2; o > 0; o >>= 1) {
    if ((int)threadIdx.x < o) red[threadIdx.x] += red[threadIdx.x + o];
    __syncthreads();
  }
  return red[0];
}

template <class T>
__global__ void __launch_bounds__(TT_BLOCK) k_sum_squares(const T *__restrict__ g, Mats m, int parts, double *__restrict__ partial) {
  const long long z = blockIdx.x / (unsigned)parts;
  const int p = (int)(blockIdx.x % (unsigned)parts);
  const long long elems = (long long)m.rows * m.cols;
  const bool small = elems < 2147483648LL;
  double s = 0;
  for (long long e = (long long)p * TT_BLOCK + threadIdx.x; e < elems; e += (long long)parts * TT_BLOCK) {
    const double v = (double)to_f32(g[z * m.b_step + place_of(m, e, small)]);
    s += v * v;
  }
  s = block_sum(s);
  if (threadIdx.x == 0) partial[z * parts + p] = s;
}

// x = g * s in fp32, packed.  A matrix whose squares do not sum to a number is NaN as a whole.
template <class T>
__global__ void __launch_bounds__(TT_BLOCK) k_scale_in(const T *__restrict__ g, Mats m, int parts, const double *__restrict__ partial, float eps,
                                                       float *__restrict__ x) {
  const long long z = blockIdx.x / (unsigned)parts;
  const int p = (int)(blockIdx.x % (unsigned)parts);
  const long long elems = (long long)m.rows * m.cols;
  const bool small = elems < 2147483648LL;
  double sum = 0;
  for (int i = threadIdx.x; i < parts; i += TT_BLOCK) sum += partial[z * parts + i];
  sum = block_sum(sum);
  double scale = 1.0 / (sqrt(sum) + (double)eps);
  if (!(sum <= 1.7976931348623157e308)) scale = (double)NAN;
  for (long long e = (long long)p * TT_BLOCK + threadIdx.x; e < elems; e += (long long)parts * TT_BLOCK)
    x[z * elems + e] = (float)((double)to_f32(g[z * m.b_step + place_of(m, e, small)]) * scale);
}

// The three products of a step, without their operands' addresses.  For results in 16 bits two bf16 parts of each operand are
// multiplied (16 bits of significand: five steps take errors up 485 times at most, in a few directions), for fp32 three.  A and B are
// symmetric: the tiles on one side of the diagonal are computed.  Measured, 4096 x 2048 bf16: 1.27 ms a
// call among others; under the profiler, where launches do not follow each other closely, 1.40 ms: norm and scaling 35 us, a step 83 + 15 for A, 46 + 15 for B,
// 115 for X (900 to 980 TFLOP/s of bf16 products).  512 x 128 fp32: 158 us, bound by four launches a step of 4 to 10 us.
struct Products {
  TTGemm gram, square, move;
};
Products products(const Mats &m, int dtype) {
  const bool tall = m.rows > m.cols;
  const int side = tall ? m.cols : m.rows;
  const long long elems = (long long)m.rows * m.cols, sq = (long long)side * side;
  Products p;
  TTGemm g;
  memset(&g, 0, sizeof(g));
  g.dtype = g.out_dtype = TT_F32;
  g.mode = TT_GEMM_BATCH;
  g.batch = (int)m.batch;
  g.alpha = 1.f;
  g.parts = dtype == TT_F32 ? 3 : 2;
  // A = X X^T, or X^T X
  p.gram = g;
  p.gram.symmetric = 1;
  p.gram.a_kc = p.gram.b_kc = tall ? 0 : 1;
  p.gram.M = p.gram.N = side; p.gram.K = tall ? m.rows : m.cols;
  p.gram.lda = p.gram.ldb = m.cols; p.gram.a_step = p.gram.b_step = elems;
  p.gram.ldo = side; p.gram.o_step = sq;
  // B = b A + c A A (A is symmetric)
  p.square = g;
  p.square.symmetric = 1;
  p.square.a_kc = p.square.b_kc = 1;
  p.square.M = p.square.N = p.square.K = side;
  p.square.lda = p.square.ldb = p.square.ldo = p.square.ldr = side;
  p.square.a_step = p.square.b_step = p.square.o_step = p.square.r_step = sq;
  // X <- a X + B X, or a X + X B (B is symmetric)
  p.move = g;
  p.move.a_kc = 1; p.move.b_kc = tall ? 1 : 0;
  p.move.M = m.rows; p.move.N = m.cols; p.move.K = side;
  p.move.lda = side; p.move.a_step = tall ? elems : sq;
  p.move.ldb = m.cols; p.move.b_step = tall ? sq : elems;
  p.move.ldr = p.move.ldo = m.cols; p.move.r_step = p.move.o_step = elems;
  return p;
}

struct Scratch {
  size_t partial, x0, x1, a, b, pieces, total;
};
Scratch scratch(long long batch, long long rows, long long cols, int dtype) {
  Scratch w;
  const long long elems = rows * cols, side = rows < cols ? rows : cols;
  memset(&w, 0, sizeof(w));
  if (ttk_slices_serves(side, rows < cols ? cols : rows)) {  // these need none
    w.total = 256;
    return w;
  }
  w.partial = 0;
  w.x0 = pad256((size_t)batch * parts_of(elems) * 8);
  w.x1 = w.x0 + pad256((size_t)batch * elems * 4);
  w.a = w.x1 + pad256((size_t)batch * elems * 4);
  w.b = w.a + pad256((size_t)batch * side * side * 4);
  w.pieces = w.b + pad256((size_t)batch * side * side * 4);
  Mats m = {batch, (int)rows, (int)cols, 0, 0};
  const Products p = products(m, dtype);
  const size_t n[3] = {ttk_gemm_partial_bytes(p.gram), ttk_gemm_partial_bytes(p.square), ttk_gemm_partial_bytes(p.move)};
  w.total = w.pieces + (n[0] > n[1] ? (n[0] > n[2] ? n[0] : n[2]) : (n[1] > n[2] ? n[1] : n[2]));
  return w;
}

template <class T>
tt_status scale_in(const void *g, const Mats &m, float eps, char *ws, const Scratch &w, hipStream_t s) {
  const int parts = parts_of((long long)m.rows * m.cols);
  const unsigned blocks = (unsigned)(m.batch * parts);
  hipLaunchKernelGGL(k_sum_squares<T>, dim3(blocks), dim3(TT_BLOCK), 0, s, (const T *)g, m, parts, (double *)(ws + w.partial));
  hipLaunchKernelGGL(k_scale_in<T>, dim3(blocks), dim3(TT_BLOCK), 0, s, (const T *)g, m, parts, (const double *)(ws + w.partial), eps,
                     (float *)(ws + w.x0));
  return tt_launch_status();
}

// The iteration.  X, A and B stay in fp32 (the polynomial takes small singular values up 485 times in five steps, and with them
// the rounding errors that they carry).
tt_status iterate(const Mats &m, const Steps &steps, int out_dtype, void *out, long long o_step, long long ldo, char *ws, const Scratch &w,
                  hipStream_t s) {
  const bool tall = m.rows > m.cols;
  float *x = (float *)(ws + w.x0), *y = (float *)(ws + w.x1), *A = (float *)(ws + w.a), *B = (float *)(ws + w.b);
  Products p = products(m, out_dtype);
  for (int i = 0; i < steps.n; ++i) {
    const float ca = steps.c[3 * i], cb = steps.c[3 * i + 1], cc = steps.c[3 * i + 2];
    p.gram.a = p.gram.b = x;
    p.gram.out = A;
    tt_status st = ttk_gemm(p.gram, ws + w.pieces, s);
    if (st != TT_OK) return st;
    p.square.a = p.square.b = p.square.res = A;
    p.square.out = B;
    p.square.alpha = cc; p.square.beta = cb;
    st = ttk_gemm(p.square, ws + w.pieces, s);
    if (st != TT_OK) return st;
    p.move.a = tall ? x : B;
    p.move.b = tall ? B : x;
    p.move.res = x;
    p.move.beta = ca;
    p.move.out = y;
    if (i + 1 == steps.n) {
      p.move.out = out; p.move.ldo = ldo; p.move.o_step = o_step;
      p.move.out_dtype = out_dtype;
    }
    st = ttk_gemm(p.move, ws + w.pieces, s);
    if (st != TT_OK) return st;
    float *t = x; x = y; y = t;
  }
  return TT_OK;
}

bool steps_ok(int steps, const float *coefficients, float eps) {
  if (steps < 1 || steps > TT_ORTHO_MAX_STEPS || !coefficients || !(eps >= 0.f)) return false;
  for (int i = 0; i < 3 * steps; ++i)
    if (!isfinite(coefficients[i])) return false;
  return true;
}
bool size_ok(int64_t batch, int64_t rows, int64_t cols) {
  if (rows < 1 || cols < 1 || batch < 0 || rows > TT_ORTHO_MAX_SIDE || cols > TT_ORTHO_MAX_SIDE) return false;
  const int64_t side = rows < cols ? rows : cols, most = (int64_t)1 << 36;
  if (batch > most / (rows * cols) || batch > most / (side * side)) return false;
  if (ttk_slices_serves(side, rows < cols ? cols : rows)) return batch <= TT_MAX_WORKGROUPS / 4;
  // a matrix is one of a grid's second side (and is cut along K only where there are few); the norm's launch has all parts of all matrices
  return batch <= 65535 && batch * parts_of(rows * cols) <= TT_MAX_WORKGROUPS &&
         batch * tt_ceil_div(rows, 64) * tt_ceil_div(cols, 64) <= TT_MAX_WORKGROUPS;
}

// ---- TT cores --------------------------------------------------------------------------------------
// Core k is [r][n][d r'] in memory; its slices i are r x (d r') matrices (core 0: d x r').  Packed: [i][r][d r'].
struct CoreDims {
  int r, n, c;  // stored order [r][n][c]
};
__device__ __forceinline__ long long packed_of(const CoreDims &d, long long e) {
  const long long row = e / d.c;  // r index * n + i
  const int a = (int)(row / d.n);
  return ((row - (long long)a * d.n) * d.r + a) * d.c + (e - row * d.c);
}
__global__ void __launch_bounds__(TT_BLOCK) k_core_momentum(CoreDims d, const float *__restrict__ grad, float *__restrict__ mom, float mu, int nesterov,
                                                            float *__restrict__ packed) {
  const long long total = (long long)d.r * d.n * d.c, stride = (long long)gridDim.x * blockDim.x;
  for (long long e = (long long)blockIdx.x * blockDim.x + threadIdx.x; e < total; e += stride) {
    const float g = grad[e], m = mu * mom[e] + g;
    mom[e] = m;
    packed[packed_of(d, e)] = nesterov ? g + mu * m : m;
  }
}
__global__ void __launch_bounds__(TT_BLOCK) k_core_apply(CoreDims d, float *__restrict__ core, const float *__restrict__ packed, float lr) {
  const long long total = (long long)d.r * d.n * d.c, stride = (long long)gridDim.x * blockDim.x;
  for (long long e = (long long)blockIdx.x * blockDim.x + threadIdx.x; e < total; e += stride) core[e] -= lr * packed[packed_of(d, e)];
}

// A batch of matrices that the kernels of one launch serve.
TTSlices slices_of(const Mats &m, int dtype, const Steps &steps, float eps) {
  const bool tall = m.rows > m.cols;
  TTSlices p;
  memset(&p, 0, sizeof(p));
  p.dtype = dtype;
  p.shorter = tall ? m.cols : m.rows;
  p.longer = tall ? m.rows : m.cols;
  p.batch = m.batch;
  p.eps = eps;
  p.steps = steps.n;
  memcpy(p.c, steps.c, sizeof(float) * 3 * steps.n);
  return p;
}

bool table_ok(const tt_table *t) {
  if (t->r[0] != 1 || t->r[3] != 1) return false;
  for (int k = 0; k < 3; ++k)
    if (t->n[k] < 1 || t->d[k] < 1 || t->r[k + 1] < 1 || t->r[k + 1] > 128 || t->d[k] > 4096) return false;
  return (int64_t)t->d[0] * t->r[1] <= 4096 && (int64_t)t->d[1] * t->r[2] <= 4096 && (int64_t)t->d[2] * t->r[2] <= 4096;
}
// slices of core k
Mats slices(const tt_table *t, int k) {
  Mats m;
  m.batch = t->n[k];
  m.rows = k == 0 ? t->d[0] : t->r[k];
  m.cols = k == 0 ? t->r[1] : t->d[k] * t->r[k + 1];
  m.r_step = m.cols;
  m.b_step = (long long)m.rows * m.cols;
  return m;
}
size_t core_elems(const Mats &m) { return (size_t)m.batch * m.b_step; }

}  // namespace

extern "C" size_t tt_orthogonalize_workspace_bytes(const tt_matrices *m) {
  if (!m || m->dtype < TT_F32 || m->dtype > TT_F16 || !size_ok(m->batch, m->rows, m->cols)) return 0;
  return m->batch == 0 ? 256 : scratch(m->batch, m->rows, m->cols, m->dtype).total;
}

extern "C" tt_status tt_orthogonalize(const tt_matrices *m, const void *g, void *out, int steps, const float *coefficients, float eps, void *workspace,
                                      size_t workspace_bytes, void *stream) {
  if (!m || m->dtype < TT_F32 || m->dtype > TT_F16 || !steps_ok(steps, coefficients, eps)) return TT_ERR_INVALID_ARG;
  if (!size_ok(m->batch, m->rows, m->cols)) return TT_ERR_SHAPE;
  if (m->batch == 0) return TT_OK;
  if (!g || !out) return TT_ERR_INVALID_ARG;
  const uintptr_t low = m->dtype == TT_F32 ? 3 : 1;
  if (((uintptr_t)g | (uintptr_t)out) & low) return TT_ERR_INVALID_ARG;
  Mats in;
  in.batch = m->batch; in.rows = (int)m->rows; in.cols = (int)m->cols;
  in.r_step = m->row_step ? m->row_step : m->cols;
  in.b_step = m->batch_step ? m->batch_step : in.r_step * m->rows;
  const long long ldo = m->out_row_step ? m->out_row_step : m->cols, o_step = m->out_batch_step ? m->out_batch_step : ldo * m->rows;
  if (in.r_step < m->cols || ldo < m->cols || in.b_step < 0 || o_step < ldo * (m->rows - 1) + m->cols) return TT_ERR_SHAPE;
  if (g == out && ((m->rows > 1 && in.r_step != ldo) || (m->batch > 1 && in.b_step != o_step))) return TT_ERR_INVALID_ARG;  // in place, from other places
  const Scratch w = scratch(m->batch, m->rows, m->cols, m->dtype);
  if (!workspace || ((uintptr_t)workspace & 255) != 0 || workspace_bytes < w.total) return TT_ERR_WORKSPACE;
  hipStream_t s = (hipStream_t)stream;
  char *ws = (char *)workspace;
  if (ttk_slices_serves(m->rows < m->cols ? m->rows : m->cols, m->rows < m->cols ? m->cols : m->rows)) {
    const bool tall = m->rows > m->cols;
    TTSlices p = slices_of(in, m->dtype, Steps{steps, coefficients}, eps);
    p.in = g; p.in_b = in.b_step; p.in_s = tall ? 1 : in.r_step; p.in_l = tall ? in.r_step : 1;
    p.out = out; p.out_b = o_step; p.out_s = tall ? 1 : ldo; p.out_l = tall ? ldo : 1;
    return ttk_slices(&p, 1, s);
  }
  tt_status st = m->dtype == TT_F32    ? scale_in<float>(g, in, eps, ws, w, s)
                 : m->dtype == TT_BF16 ? scale_in<ttg::bf16>(g, in, eps, ws, w, s)
                                       : scale_in<ttg::f16>(g, in, eps, ws, w, s);
  if (st != TT_OK) return st;
  return iterate(in, Steps{steps, coefficients}, m->dtype, out, o_step, ldo, ws, w, s);
}

extern "C" size_t tt_core_ortho_workspace_bytes(const tt_table *table) {
  if (!table || !table_ok(table)) return 0;
  size_t most = 0;
  for (int k = 0; k < 3; ++k) {
    const Mats m = slices(table, k);
    if (!size_ok(m.batch, m.rows, m.cols)) return 0;
    const bool served = ttk_slices_serves(m.rows < m.cols ? m.rows : m.cols, m.rows < m.cols ? m.cols : m.rows);
    const size_t n = scratch(m.batch, m.rows, m.cols, TT_F32).total + (served ? 0 : 2 * pad256(core_elems(m) * 4));
    if (n > most) most = n;
  }
  return most;
}

extern "C" tt_status tt_core_ortho_update(const tt_table *table, const float *const dcore[3], float *const momentum[3], float lr, float mu, int nesterov,
                                          int steps, const float *coefficients, float eps, void *workspace, size_t workspace_bytes, void *stream) {
  if (!table || !dcore || !momentum || !steps_ok(steps, coefficients, eps)) return TT_ERR_INVALID_ARG;
  if (!table_ok(table)) return TT_ERR_SHAPE;
  for (int k = 0; k < 3; ++k)
    if (!table->core[k] || !dcore[k] || !momentum[k] || (((uintptr_t)table->core[k] | (uintptr_t)dcore[k] | (uintptr_t)momentum[k]) & 3))
      return TT_ERR_INVALID_ARG;
  const size_t need = tt_core_ortho_workspace_bytes(table);
  if (need == 0) return TT_ERR_SHAPE;
  if (!workspace || ((uintptr_t)workspace & 255) != 0 || workspace_bytes < need) return TT_ERR_WORKSPACE;
  hipStream_t s = (hipStream_t)stream;
  TTSlices jobs[3];  // the cores whose slices stay on chip go into one launch, core 1 first
  int n = 0;
  const int order[3] = {1, 0, 2};
  for (int i = 0; i < 3; ++i) {
    const int k = order[i];
    const Mats m = slices(table, k);
    const Scratch w = scratch(m.batch, m.rows, m.cols, TT_F32);
    char *ws = (char *)workspace;
    float *u = (float *)(ws + w.total), *o = (float *)(ws + w.total + pad256(core_elems(m) * 4));
    CoreDims d;
    d.r = k == 0 ? 1 : m.rows; d.n = (int)m.batch; d.c = k == 0 ? m.rows * m.cols : m.cols;
    long long blocks = ((long long)core_elems(m) + TT_BLOCK - 1) / TT_BLOCK;
    if (blocks > 8192) blocks = 8192;
    const float *grad = dcore[k];
    float *mom = momentum[k], *core = table->core[k];
    const float rate = (float)((double)lr * sqrt(m.rows > m.cols ? (double)m.rows / m.cols : 1.0));
    const bool tall = m.rows > m.cols;
    if (ttk_slices_serves(tall ? m.cols : m.rows, tall ? m.rows : m.cols)) {
      TTSlices &p = jobs[n++];
      p = slices_of(m, TT_F32, Steps{steps, coefficients}, eps);
      const long long row = k == 0 ? m.cols : (long long)m.batch * m.cols;  // between a slice's rows; slices are a row apart, in core 0 whole
      p.in = grad; p.out = core; p.mom = mom;
      p.in_b = p.out_b = k == 0 ? m.b_step : m.cols;
      p.in_s = p.out_s = tall ? 1 : row;
      p.in_l = p.out_l = tall ? row : 1;
      p.mu = mu; p.rate = rate; p.nesterov = nesterov;
      continue;
    }
    hipLaunchKernelGGL(k_core_momentum, dim3((unsigned)blocks), dim3(TT_BLOCK), 0, s, d, grad, mom, mu, nesterov, u);
    tt_status st = scale_in<float>(u, m, eps, ws, w, s);
    if (st == TT_OK) st = iterate(m, Steps{steps, coefficients}, TT_F32, o, m.b_step, m.r_step, ws, w, s);
    if (st != TT_OK) return st;
    hipLaunchKernelGGL(k_core_apply, dim3((unsigned)blocks), dim3(TT_BLOCK), 0, s, d, core, (const float *)o, rate);
    st = tt_launch_status();
    if (st != TT_OK) return st;
  }
  return ttk_slices(jobs, n, s);
}
