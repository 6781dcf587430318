// The product behind the pooled rows: out = act(x W^T + bias) + residual with one weight, or a weight per group of rows
// (the tables of a fused table, experts), and its gradients.  C entry points; the products themselves are tt_gemm.hip.
#include <string.h>

#include "tt_gemm_device.h"

namespace {
using namespace ttg;

size_t pad256(size_t n) { return (n + 255) & ~(size_t)255; }
size_t elem(int dtype) { return dtype == TT_F32 ? 4 : 2; }

tt_status check(const tt_dense *op) {
  if (!op) return TT_ERR_INVALID_ARG;
  if (op->dtype < TT_F32 || op->dtype > TT_F16 || op->activation < TT_ACT_NONE || op->activation > TT_ACT_SIGMOID) return TT_ERR_INVALID_ARG;
  if (op->rows < 0 || op->groups < 0) return TT_ERR_INVALID_ARG;
  if (op->in_dim < 1 || op->out_dim < 1 || op->in_dim > TT_DENSE_MAX_DIM || op->out_dim > TT_DENSE_MAX_DIM || op->groups > TT_DENSE_MAX_GROUPS ||
      op->rows >= 2147483647LL - 2 * TT_DENSE_MAX_GROUPS)
    return TT_ERR_SHAPE;
  if (op->groups > 0 && !op->offsets) return TT_ERR_INVALID_ARG;
  const int64_t ld[5] = {op->ld_x, op->ld_dx, op->ld_out, op->ld_residual, op->ld_grad};
  for (int i = 0; i < 5; ++i)
    if (ld[i] != 0 && (ld[i] < (i < 2 ? op->in_dim : op->out_dim) || ld[i] > ((int64_t)1 << 40))) return TT_ERR_SHAPE;
  return TT_OK;
}
bool aligned(const void *p, int dtype) { return ((uintptr_t)p & (elem(dtype) - 1)) == 0; }
long long step(int64_t ld, int dim) { return ld ? ld : dim; }

// dz = grad * act'(pre), rounded to the operands' type: the matrix cores take it in that type.  A rounding of half a step of
// each term, in sums whose result is rounded by as much.
template <class T>
__global__ void __launch_bounds__(TT_BLOCK) k_act_grad(const T *__restrict__ grad, long long ldg, const T *__restrict__ pre, T *__restrict__ dz,
                                                       long long rows, int n, int act) {
  const int per = (n + 7) / 8;
  const long long total = rows * per, stride = (long long)gridDim.x * blockDim.x;
  for (long long e = (long long)blockIdx.x * blockDim.x + threadIdx.x; e < total; e += stride) {
    const long long r = total < 2147483648LL ? (long long)((unsigned)e / (unsigned)per) : e / per;  // (a 64-bit division costs as much as the rest)
    const int c = (int)(e - r * per) * 8, valid = n - c;
    float v[8], z[8];
    load_n<T, 8>(grad + r * ldg + c, valid, v);
    load_n<T, 8>(pre + r * n + c, valid, z);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] *= slope_of<T>(z[i], act);
    store_n<T, 8>(dz + r * n + c, valid, v);
  }
}

template <class T>
tt_status act_grad(const tt_dense *op, const void *grad, const void *pre, void *dz, hipStream_t s) {
  const long long total = op->rows * ((op->out_dim + 7) / 8);
  long long blocks = (total + TT_BLOCK - 1) / TT_BLOCK;
  if (blocks > 16384) blocks = 16384;
  const long long ldg = step(op->ld_grad, op->out_dim);
  hipLaunchKernelGGL(k_act_grad<T>, dim3((unsigned)blocks), dim3(TT_BLOCK), 0, s, (const T *)grad, ldg, (const T *)pre, (T *)dz, (long long)op->rows,
                     (int)op->out_dim, (int)op->activation);
  return tt_launch_status();
}

void describe(const tt_dense *op, TTGemm *g) {
  memset(g, 0, sizeof(*g));
  g->dtype = g->out_dtype = op->dtype;
  g->batch = op->groups > 0 ? op->groups : 1;
  g->offsets = op->offsets;
  g->zero_rest = op->zero_rest;
  g->alpha = g->beta = 1.f;
  g->parts = 3;
}

// The products of a call, without their operands' addresses.
TTGemm of_out(const tt_dense *op) {  // x W^T
  TTGemm g;
  describe(op, &g);
  g.a_kc = g.b_kc = 1;
  g.mode = op->groups > 0 ? TT_GEMM_RAGGED_M : TT_GEMM_BATCH;
  g.M = (int)op->rows; g.N = op->out_dim; g.K = op->in_dim;
  g.lda = step(op->ld_x, op->in_dim);
  g.ldb = op->in_dim; g.b_step = (long long)op->out_dim * op->in_dim;
  g.ldo = step(op->ld_out, op->out_dim);
  g.bias_step = op->out_dim;
  g.ldr = step(op->ld_residual, op->out_dim);
  g.ldp = op->out_dim;
  g.act = op->activation;
  return g;
}
TTGemm of_dx(const tt_dense *op, long long ldz) {  // dz W
  TTGemm g;
  describe(op, &g);
  g.a_kc = 1; g.b_kc = 0;
  g.mode = op->groups > 0 ? TT_GEMM_RAGGED_M : TT_GEMM_BATCH;
  g.M = (int)op->rows; g.N = op->in_dim; g.K = op->out_dim;
  g.lda = ldz;
  g.ldb = op->in_dim; g.b_step = (long long)op->out_dim * op->in_dim;
  g.ldo = step(op->ld_dx, op->in_dim);
  return g;
}
TTGemm of_dw(const tt_dense *op, long long ldz, bool column) {  // dz^T x, or one column of dz^T dz
  TTGemm g;
  describe(op, &g);
  g.a_kc = g.b_kc = 0;
  g.mode = op->groups > 0 ? TT_GEMM_RAGGED_K : TT_GEMM_BATCH;
  g.M = op->out_dim; g.N = column ? 1 : op->in_dim; g.K = (int)op->rows;
  g.like_N = op->in_dim;
  g.lda = ldz;
  g.ldb = column ? ldz : step(op->ld_x, op->in_dim);
  g.ldo = g.N; g.o_step = (long long)op->out_dim * g.N;
  g.rs_step = op->out_dim;
  return g;
}

struct Scratch {
  size_t dz, column, pieces, total;  // byte offsets
};
Scratch scratch(const tt_dense *op, bool backward) {
  Scratch w = {0, 0, 0, 0};
  size_t most = ttk_gemm_partial_bytes(of_out(op));
  if (backward) {
    if (op->activation != TT_ACT_NONE) w.total += pad256((size_t)op->rows * op->out_dim * elem(op->dtype));
    w.column = w.total;
    w.total += pad256((size_t)(op->groups > 0 ? op->groups : 1) * op->out_dim * elem(op->dtype));
    const TTGemm products[3] = {of_dx(op, op->out_dim), of_dw(op, op->out_dim, false), of_dw(op, op->out_dim, true)};
    most = 0;
    for (int i = 0; i < 3; ++i) {
      const size_t n = ttk_gemm_partial_bytes(products[i]);
      if (n > most) most = n;
    }
  }
  w.pieces = w.total;
  w.total += most;
  return w;
}

}  // namespace

extern "C" size_t tt_dense_workspace_bytes(const tt_dense *op, int backward) {
  if (check(op) != TT_OK) return 0;
  return scratch(op, backward != 0).total;
}

extern "C" tt_status tt_dense_forward(const tt_dense *op, const void *x, const void *w, const void *bias, const void *residual, void *out, void *pre,
                                      void *workspace, size_t workspace_bytes, void *stream) {
  const tt_status st = check(op);
  if (st != TT_OK) return st;
  if (op->rows == 0) return TT_OK;
  if (!x || !w || !out) return TT_ERR_INVALID_ARG;
  if (!aligned(x, op->dtype) || !aligned(w, op->dtype) || !aligned(bias, op->dtype) || !aligned(residual, op->dtype) || !aligned(out, op->dtype) ||
      !aligned(pre, op->dtype))
    return TT_ERR_INVALID_ARG;
  // outputs over inputs that other workgroups still read; a residual that shares out's memory is read where it is written
  if (out == x || out == w || out == bias || (pre && (pre == x || pre == w || pre == bias || pre == residual || pre == out))) return TT_ERR_INVALID_ARG;
  if (out == residual && op->rows > 1 && step(op->ld_out, op->out_dim) != step(op->ld_residual, op->out_dim)) return TT_ERR_INVALID_ARG;
  const Scratch need = scratch(op, false);
  if (need.total && (!workspace || ((uintptr_t)workspace & 255) != 0 || workspace_bytes < need.total)) return TT_ERR_WORKSPACE;
  TTGemm g = of_out(op);
  g.a = x; g.b = w; g.out = out;
  g.bias = bias; g.res = residual; g.pre = pre;
  return ttk_gemm(g, workspace ? (char *)workspace + need.pieces : nullptr, (hipStream_t)stream);
}

extern "C" tt_status tt_dense_backward(const tt_dense *op, const void *x, const void *w, const void *pre, const void *grad_out, void *dx, void *dw,
                                       void *dbias, void *workspace, size_t workspace_bytes, void *stream) {
  tt_status st = check(op);
  if (st != TT_OK) return st;
  const bool some = op->rows > 0, bent = op->activation != TT_ACT_NONE;
  if (!dx && !dw && !dbias) return TT_OK;
  if (some && (!grad_out || (dw && !x) || (dx && !w) || (bent && !pre))) return TT_ERR_INVALID_ARG;
  const void *ptrs[7] = {x, w, pre, grad_out, dx, dw, dbias};
  for (int i = 0; i < 7; ++i) {
    if (!aligned(ptrs[i], op->dtype)) return TT_ERR_INVALID_ARG;
    for (int j = 4; j < 7; ++j)  // outputs over inputs
      if (i < 4 && ptrs[j] && ptrs[i] == ptrs[j]) return TT_ERR_INVALID_ARG;
  }
  const Scratch need = scratch(op, true);
  if (!workspace || ((uintptr_t)workspace & 255) != 0 || workspace_bytes < need.total) return TT_ERR_WORKSPACE;
  hipStream_t s = (hipStream_t)stream;
  char *ws = (char *)workspace;
  const void *dz = grad_out;
  long long ldz = step(op->ld_grad, op->out_dim);
  if (bent && some) {
    st = op->dtype == TT_F32    ? act_grad<float>(op, grad_out, pre, ws + need.dz, s)
         : op->dtype == TT_BF16 ? act_grad<ttg::bf16>(op, grad_out, pre, ws + need.dz, s)
                                : act_grad<ttg::f16>(op, grad_out, pre, ws + need.dz, s);
    if (st != TT_OK) return st;
    dz = ws + need.dz;
    ldz = op->out_dim;
  }
  if (dx && some) {
    TTGemm g = of_dx(op, ldz);
    g.a = dz; g.b = w; g.out = dx;
    st = ttk_gemm(g, ws + need.pieces, s);
    if (st != TT_OK) return st;
  }
  if (dw || dbias) {  // the sums of dz's columns come beside a product: where that is not asked for, of a single column, into scratch
    TTGemm g = of_dw(op, ldz, !dw);
    g.a = dz; g.b = dw ? x : dz;
    g.out = dw ? dw : ws + need.column;
    g.rowsum = dbias;
    st = ttk_gemm(g, ws + need.pieces, s);
  }
  return st;
}
