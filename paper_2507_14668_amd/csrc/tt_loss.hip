// Softmax cross entropy against a catalogue, and its gradients, in pieces of the classes.
#include <string.h>

#include "tt_gemm_device.h"
#include "tt_loss.h"

namespace {
using namespace ttg;

typedef TTLossRows Rows;

// One workgroup: places in the order of the rows.  In the backward also each place's lse, hot and share of the loss's gradient.
constexpr int SCAN = 512;
__global__ void __launch_bounds__(SCAN) k_loss_rows(const int64_t *labels, long long rows, int classes, long long ignored, int reduce, const float2 *of_rows,
                                                    const float *grad, int apart, int half, int negative, float *loss, float2 *zeros, Rows w) {
  __shared__ int tmp[SCAN / 64 + 1];
  __shared__ float tops[SCAN / 64];
  int places = 0;
  constexpr int EACH = 8;  // rows of a thread at a time
  for (long long r0 = 0; r0 < rows; r0 += SCAN * EACH) {
    const long long r1 = r0 + threadIdx.x * EACH;
    int64_t label[EACH];
    int mine = 0;
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
      label[i] = r1 + i < rows ? labels[r1 + i] : ignored;
      mine += label[i] != ignored;
    }
    int total, at = places + tt_block_excl_scan_n<SCAN>(mine, tmp, &total);
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
      const long long r = r1 + i;
      const bool counts = label[i] != ignored;
      if (r < rows) w.at[r] = counts ? at : -1;
      if (zeros && r < rows && !counts) {
        zeros[r] = float2{0.f, 0.f};
        if (loss) loss[r] = 0.f;
      }
      if (!counts) continue;
      w.of[at] = (int32_t)r;
      w.label[at] = label[i] >= 0 && label[i] < classes ? (int32_t)label[i] : -1;
      if (of_rows) {
        const float2 s = of_rows[r];
        w.lse[at] = negative ? -s.x : s.x;
        w.hot[at] = expm1f(-s.y);
      }
      ++at;
    }
    places += total;
  }
  if (threadIdx.x == 0) {
    w.offsets[0] = 0;
    w.offsets[1] = places;
  }
  if (!of_rows) return;
  __syncthreads();
  const float all = reduce == TT_REDUCE_NONE ? 0.f : reduce == TT_REDUCE_MEAN && places > 0 ? grad[0] / (float)places : grad[0];
  float top = 0.f;  // the largest finite share: what fp16 asks for
  if (half && reduce == TT_REDUCE_NONE) {
#pragma unroll 4
    for (int i = threadIdx.x; i < places; i += SCAN) {
      const float g = fabsf(grad[w.of[i]]);
      top = g < INFINITY && g > top ? g : top;
    }
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor(top, o, 64));
  if ((threadIdx.x & 63) == 0) tops[threadIdx.x >> 6] = top;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < SCAN / 64; ++i) top = fmaxf(top, tops[i]);
  // fp32 products take G as it is.  Else (`apart`: 16 bits, and short rows) a share that all rows have is left for the end (rounded into each term it would be the same error in
  // all of them); shares of their own are part of G, in fp16 times the power of two that takes the largest to 2^13 .. 2^14, as far as that and its
  // inverse are normal numbers.  2^13 for the same reason: fp16 has a short range.
  const bool own = reduce == TT_REDUCE_NONE;
  float scale = 1.f, back = 1.f;
  if (own && half && top > 0.f) {
    int e = (int)(__float_as_uint(top) >> 23);
    e = e < 14 ? 14 : e > 240 ? 240 : e;
    scale = __uint_as_float((unsigned)(127 + 13 + 127 - e) << 23);
    back = __uint_as_float((unsigned)(e - 13) << 23);
  }
  const float raised = half ? TT_LOSS_RAISE : 1.f;  // (a bf16 G has the range, and its sums need theirs: of rows near 1e38 they would overflow)
  if (apart && !own) back = places > 0 ? all / raised : 0.f;
  if (threadIdx.x == 0) w.back[0] = back;
#pragma unroll 4
  for (int i = threadIdx.x; i < places; i += SCAN) {
    const float share = own ? grad[w.of[i]] : all;
    w.share[i] = share;
    w.weight[i] = apart && !own ? raised : scale * share;
  }
  if (negative && threadIdx.x < TT_LOSS_STEP && places + (int)threadIdx.x < (places + TT_LOSS_STEP - 1) / TT_LOSS_STEP * TT_LOSS_STEP) {
    w.lse[places + threadIdx.x] = -INFINITY;  // up to a whole step: rows that add nothing
    w.label[places + threadIdx.x] = -1;
    w.weight[places + threadIdx.x] = 0.f;
  }
}

// x's rows that count next to each other, `ld` apart (padded with zeros), zeros behind the last one.
template <class T> __global__ void __launch_bounds__(TT_BLOCK) k_loss_gather(const T *x, long long ld_x, long long rows, int dim, Rows w, T *to, int ld) {
  constexpr int C = 16 / sizeof(T);
  const long long places = w.offsets[1];
  const int per = (ld + C - 1) / C;
  for (long long e = (long long)blockIdx.x * TT_BLOCK + threadIdx.x; e < rows * per; e += (long long)gridDim.x * TT_BLOCK) {
    const long long i = e / per;
    const int c = (int)(e - i * per) * C;
    float v[C] = {};
    if (i < places) load_n<T, C>(x + w.of[i] * ld_x + c, dim - c, v);
    store_n<T, C>(to + i * ld + c, ld - c, v);
  }
}

// The pieces of fp32 logits that went through memory: of each place's COLUMNS of them the pair that a tile of the product gives else, and the label's
// logit; a wavefront each.  z: [rows][ld], 16-byte aligned rows.
constexpr int COLUMNS = 1024;
__global__ void __launch_bounds__(TT_BLOCK) k_loss_pairs(const float *__restrict__ z, long long ld, long long rows, int n, int first, Rows w, float2 *stats,
                                                         float *picked) {
  const long long i = (long long)blockIdx.x * (TT_BLOCK / 64) + (threadIdx.x >> 6);
  if (i >= w.offsets[1]) return;
  const int lane = threadIdx.x & 63, label = w.label[i] - first;
  for (int t = (int)blockIdx.y; t * COLUMNS < n; t += (int)gridDim.y) {
    const int c0 = t * COLUMNS + 4 * lane;
    f32x4 v[COLUMNS / 256];
    float top = -INFINITY, sum = 0.f;
#pragma unroll
    for (int k = 0; k < COLUMNS / 256; ++k) {
      const int c = c0 + 256 * k;
      float a[4] = {0.f, 0.f, 0.f, 0.f};
      if (c < n) load4(z + i * ld + c, n - c, a);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        v[k][e] = c + e < n ? a[e] : -INFINITY;
        if (c + e == label && c + e < n) {  // (in no sum: row_of_loss)
          picked[i] = a[e];
          v[k][e] = -INFINITY;
        }
        top = fmaxf(top, v[k][e]);
      }
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor(top, o, 64));
    const float base = top == -INFINITY ? 0.f : top;
#pragma unroll
    for (int k = 0; k < COLUMNS / 256; ++k)
#pragma unroll
      for (int e = 0; e < 4; ++e) sum += __expf(v[k][e] - base);
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) sum += __shfl_xor(sum, o, 64);
    if (lane == 0) stats[t * rows + i] = float2{top, sum};
  }
}
// ... and G in their place, zeros in the rows that do not count and in columns n .. padded - 1.
__global__ void __launch_bounds__(TT_BLOCK) k_loss_softmax(float *z, long long ld, long long rows, int n, int padded, int first, Rows w) {
  const long long places = w.offsets[1];
  const int per = padded / 4;
  for (long long e = (long long)blockIdx.x * TT_BLOCK + threadIdx.x; e < rows * per; e += (long long)gridDim.x * TT_BLOCK) {
    const long long i = e / per;
    const int c = (int)(e - i * per) * 4;
    float *at = z + i * ld + c;
    float v[4] = {0.f, 0.f, 0.f, 0.f};
    if (i < places) {
      load4(at, n - c, v);
      const float lse = w.lse[i], grad = w.weight[i];
      const int label = w.label[i] - first - c;
#pragma unroll
      for (int k = 0; k < 4; ++k) v[k] = k < n - c ? grad * (k == label ? w.hot[i] : __expf(v[k] - lse)) : 0.f;
    }
    store4(at, 4, v);
  }
}

// A piece's tiles into each place's running pair (largest logit, sum of exp(logit - it)), sixteen places a workgroup and sixteen runs of the tiles;
// of the last piece the row's lse and loss.
__global__ void __launch_bounds__(TT_BLOCK) k_loss_fold(const float2 *__restrict__ stats, int tiles, long long rows, int first, int last, Rows w, float2 *run,
                                                        const float *picked, float2 *each, float *loss) {
  __shared__ float2 part[TT_BLOCK];
  const int lane = threadIdx.x & 15, seg = threadIdx.x >> 4, per = (tiles + 15) / 16;
  const long long i = (long long)blockIdx.x * 16 + lane, places = w.offsets[1];
  float2 s = {-INFINITY, 0.f};
  if (i < places) {
    const int end = (seg + 1) * per < tiles ? (seg + 1) * per : tiles;
#pragma unroll 4
    for (int t = seg * per; t < end; ++t) s = join_stats(s, stats[t * rows + i]);
  }
  part[threadIdx.x] = s;
  __syncthreads();
  if (seg != 0 || i >= places) return;
  for (int k = 1; k < 16; ++k) s = join_stats(s, part[16 * k + lane]);
  if (!first) s = join_stats(run[i], s);
  if (!last) {
    run[i] = s;
    return;
  }
  const int r = w.of[i];
  each[r] = w.label[i] < 0 ? float2{NAN, NAN} : row_of_loss(s, picked[i]);
  if (loss) loss[r] = each[r].y;
}
// One workgroup: the sum or the mean, in 64 bits.
__global__ void __launch_bounds__(SCAN) k_loss_sum(const float2 *each, long long rows, Rows w, int reduce, float *loss) {
  __shared__ double sums[SCAN / 64];
  double s = 0;
#pragma unroll 8
  for (long long r = threadIdx.x; r < rows; r += SCAN) s += (double)each[r].y;
  s = wave_sum64(s);
  if ((threadIdx.x & 63) == 0) sums[threadIdx.x >> 6] = s;
  __syncthreads();
  if (threadIdx.x != 0) return;
  s = 0;
  for (int i = 0; i < SCAN / 64; ++i) s += sums[i];
  const int64_t places = w.offsets[1];
  loss[0] = (float)(reduce == TT_REDUCE_MEAN && places > 0 ? s / (double)places : s);
}

// dx from its sums in the order of the places; zeros in rows that do not count
template <class T> __global__ void __launch_bounds__(TT_BLOCK) k_loss_dx(const float *acc, int ld_acc, int cuts, long long rows, int dim, Rows w, T *dx, long long ld) {
  const int per = (dim + 3) / 4;
  const float back = w.back[0];
  for (long long e = (long long)blockIdx.x * TT_BLOCK + threadIdx.x; e < rows * per; e += (long long)gridDim.x * TT_BLOCK) {
    const long long r = e / per;
    const int c = (int)(e - r * per) * 4, at = w.at[r];
    float v[4] = {0.f, 0.f, 0.f, 0.f};
    if (at >= 0) {
#pragma unroll 4
      for (int k = 0; k < cuts; ++k) {
        float t[4];
        load4(acc + (k * rows + at) * ld_acc + c, dim - c, t);
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] += t[i];
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] *= back;  // (which may be infinite: not times the zeros of the others)
    }
    store4(dx + r * ld + c, dim - c, v);
  }
}
// Rows of W with zeros up to a multiple of 8.
template <class T> __global__ void __launch_bounds__(TT_BLOCK) k_loss_pad(const T *w, long long rows, int dim, T *to, int ld) {
  const int per = ld / 8;
  for (long long e = (long long)blockIdx.x * TT_BLOCK + threadIdx.x; e < rows * per; e += (long long)gridDim.x * TT_BLOCK) {
    const long long r = e / per;
    const int c = (int)(e - r * per) * 8;
    float v[8];
    load_n<T, 8>(w + r * dim + c, dim - c, v);
    store_n<T, 8>(to + r * ld + c, 8, v);
  }
}
template <class T> __global__ void __launch_bounds__(TT_BLOCK) k_loss_clear(T *p, long long n) {
  for (long long i = (long long)blockIdx.x * TT_BLOCK + threadIdx.x; i < n; i += (long long)gridDim.x * TT_BLOCK) p[i] = from_f32<T>(0.f);
}

// ---- host ------------------------------------------------------------------------------------------
size_t pad256(size_t n) { return (n + 255) & ~(size_t)255; }
size_t elem(int dtype) { return dtype == TT_F32 ? 4 : 2; }
bool aligned(const void *p, size_t size) { return ((uintptr_t)p & (size - 1)) == 0; }

tt_status check(const tt_loss *op) {
  if (!op || op->dtype < TT_F32 || op->dtype > TT_F16 || op->reduce < TT_REDUCE_NONE || op->reduce > TT_REDUCE_MEAN || op->rows < 0) return TT_ERR_INVALID_ARG;
  if (op->dim < 1 || op->dim > TT_DENSE_MAX_DIM || op->classes < 1 || op->classes > TT_LOSS_MAX_CLASSES || op->rows >= 2147483647LL - 2 * TT_DENSE_MAX_GROUPS)
    return TT_ERR_SHAPE;
  const int64_t ld[2] = {op->ld_x, op->ld_dx};
  for (int i = 0; i < 2; ++i)
    if (ld[i] != 0 && (ld[i] < op->dim || ld[i] > ((int64_t)1 << 40))) return TT_ERR_SHAPE;
  return TT_OK;
}

bool stored(const tt_loss *op);
// Classes of a piece, whole tiles of 256: of a forward one the statistics, of a backward one G (and of both logits that go through memory) has
// `room` bytes, about half of what the last-level cache holds, so that the products that read a piece find it there.
#ifndef TT_LOSS_ROOM
#define TT_LOSS_ROOM (128 << 20)
#endif
long long piece_of(const tt_loss *op, bool backward) {
  const long long each = backward || stored(op) ? op->rows * (long long)elem(op->dtype) : tt_ceil_div(op->rows * 8, 64);
  long long most = (long long)TT_LOSS_ROOM / (each > 0 ? each : 1) / 256 * 256;
  if (most < 256) most = 256;
  const long long pieces = (op->classes + most - 1) / most;
  return ((op->classes + pieces - 1) / pieces + 255) / 256 * 256;
}
bool narrow(const tt_loss *op) { return ttk_narrow_serves(op->dim); }
// 16-bit rows of a W whose length is no multiple of 8 elements are copied to ones that are, a piece at a time, so that the large tiles serve: the copy costs
// four bytes an element at 4.5 TB/s, the tiles save the difference between 330 and 1100 TFLOP/s in every product; 1001 rows of 479 against
// 50001 classes 111 us with it, 178 without.  Few rows do not pay for it.
#ifndef TT_LOSS_COPY_ROWS
#define TT_LOSS_COPY_ROWS 256
#endif
bool copies(const tt_loss *op) { return op->dtype != TT_F32 && !narrow(op) && (op->dim & 7) && op->rows >= TT_LOSS_COPY_ROWS; }
int padded(const tt_loss *op) { return narrow(op) ? ttk_narrow_padded(op->dim) : (op->dim + 7) & ~7; }

void describe(const tt_loss *op, TTGemm *g) {
  memset(g, 0, sizeof(*g));
  g->dtype = g->out_dtype = op->dtype;
  g->batch = 1;
  g->alpha = g->beta = 1.f;
  g->parts = 3;
  g->large = op->dtype == TT_F32;
}
TTGemm of_logits(const tt_loss *op, int classes, bool backward, long long ldg) {  // rows that count by W of a piece
  TTGemm g;
  describe(op, &g);
  g.a_kc = g.b_kc = 1;
  g.mode = TT_GEMM_RAGGED_M;
  g.M = (int)op->rows; g.N = classes; g.K = copies(op) ? padded(op) : op->dim;
  g.lda = padded(op); g.ldb = g.K; g.ldo = ldg;
  g.epilogue = backward ? TT_GEMM_SOFTMAX : TT_GEMM_STATS;
  g.zero_rest = backward;
  g.n_padded = (classes + 7) & ~7;
  return g;
}
// The logits of a piece, or its G, in fp32 as an ordinary product that all rows take part in (zeros behind the last one that counts).
TTGemm of_stored(const tt_loss *op, int classes, long long ldz) {
  TTGemm g;
  describe(op, &g);
  g.a_kc = g.b_kc = 1;
  g.M = (int)op->rows; g.N = classes; g.K = op->dim;
  g.lda = padded(op); g.ldb = op->dim; g.ldo = ldz;
  return g;
}
// Whether fp32 logits go through memory: where few tiles leave most compute units without one, which the ordinary product cuts along its sums, and for the
// few rows that have a kernel of their own.  The loss alone, through memory / in the tiles' own statistics, us: 1000 rows of 4096 against 500 classes 87 / 154, 300 x
// 4096 x 2000 97 / 143, 70 x 2000 x 30000 144 / 224, 16 x 4096 x 30000 163 / 229.  (In 16 bits the steps are four times as fast, and a rounded logit would not do.)
bool stored(const tt_loss *op) {
  if (op->dtype != TT_F32 || narrow(op) || op->rows < 1) return false;
  const long long most = (long long)TT_LOSS_ROOM / (op->rows * 4);  // (a piece has so many, and 256 at least)
  const TTGemm g = of_stored(op, op->classes < most ? op->classes : most < 256 ? 256 : (int)most, 0);
  return ttk_gemm_rows_serves(g) || ttk_gemm_partial_bytes(g) > 0;
}
// G W: few tiles of dx over many classes are cut into `cuts` equal members, whole steps of 64 classes, whose sums stand side by side until
// the end; what is left over is a product of its own.  4000 rows of 513 (48 tiles of 256) against 16384 classes in fp16 250 us whole, 108 in
// five; 2000 x 256 (8 tiles) against 33536 in bf16 98 whole (in tiles of 64, by four), 67 in sixteen.
#ifndef TT_LOSS_CUT
#define TT_LOSS_CUT 1024  // classes of a member at least
#endif
int cuts_of(const tt_loss *op) {
  const int e = op->dtype == TT_F32 ? 128 : 256;
  const long long tiles = (long long)tt_ceil_div(op->rows, e) * tt_ceil_div(op->dim, e), want = op->dtype == TT_F32 ? 512 : 256;
  if (op->rows <= 128 || tiles * 2 > want) return 1;
  long long cuts = want / tiles;
  const long long piece = piece_of(op, true), most = (piece < op->classes ? piece : op->classes) / TT_LOSS_CUT;
  if (cuts > most) cuts = most;
  return (int)(cuts < 1 ? 1 : cuts > 16 ? 16 : cuts);
}
TTGemm of_dx(const tt_loss *op, int classes, int members, long long ldg) {
  TTGemm g;
  describe(op, &g);
  g.a_kc = 1; g.b_kc = 0;
  g.batch = members;
  g.M = (int)op->rows; g.N = copies(op) ? padded(op) : op->dim; g.K = classes;
  g.lda = ldg; g.ldb = g.ldo = g.N;
  g.a_step = classes; g.b_step = (long long)classes * g.ldb;
  g.a_padded = 1;
  g.epilogue = TT_GEMM_ACC;
  return g;
}
TTGemm of_dw(const tt_loss *op, int classes, long long ldg, bool column) {  // G^T x, or one column of G^T G
  TTGemm g;
  describe(op, &g);
  g.a_kc = g.b_kc = 0;
  g.M = classes; g.N = column ? 1 : op->dim; g.K = (int)op->rows;
  g.like_N = op->dim;
  g.lda = ldg; g.ldb = column ? ldg : padded(op); g.ldo = g.N;
  g.a_padded = g.b_padded = 1;
  g.epilogue = TT_GEMM_SCALED;
  return g;
}

struct Scratch {
  size_t of, at, label, lse, share, weight, hot, back, offsets, x, stats, run, picked, grads, acc, column, pieces, parts, starts, copy, total;
};
size_t stored_bytes(const tt_loss *op, long long piece) {
  const int first = (int)(piece < op->classes ? piece : op->classes), last = (int)(op->classes - (op->classes - 1) / piece * piece);
  const size_t a = ttk_gemm_partial_bytes(of_stored(op, first, piece)), b = ttk_gemm_partial_bytes(of_stored(op, last, piece));
  return a > b ? a : b;
}
Scratch scratch(const tt_loss *op, bool backward) {
  Scratch w = {};
  const size_t rows = (size_t)op->rows, whole = rows + TT_LOSS_STEP, es = elem(op->dtype);
  const long long piece = piece_of(op, backward);
  TTNarrow n = {};
  n.dtype = op->dtype;
  n.dim = op->dim;
  n.padded = padded(op);
  n.classes = op->classes;
  n.rows = op->rows;
  auto take = [&](size_t &at, size_t bytes) {
    at = w.total;
    w.total += pad256(bytes);
  };
  take(w.of, rows * 4);
  take(w.at, rows * 4);
  take(w.label, whole * 4);
  take(w.back, 4);
  take(w.offsets, 16);
  const size_t each = narrow(op) && op->dtype == TT_F32 ? 6 : es;  // (three planes of 16 bits)
  take(w.x, rows * padded(op) * each);
  if (copies(op)) take(w.copy, (size_t)(piece < op->classes ? piece : op->classes) * padded(op) * es);
  if (narrow(op)) {
    take(w.starts, ((size_t)op->classes + TT_LOSS_STEP) * 4);
    take(w.copy, (size_t)op->classes * padded(op) * each);  // (whether it is used is known with w's address only)
  }
  if (!backward) {
    take(w.stats, narrow(op) ? ttk_narrow_stats_bytes(n) : (size_t)tt_ceil_div(piece, 64) * rows * 8);
    take(w.run, rows * 8);
    take(w.picked, rows * 4);
    if (stored(op)) {
      take(w.grads, rows * piece * 4);
      take(w.pieces, stored_bytes(op, piece));
    }
    return w;
  }
  take(w.lse, whole * 4);
  take(w.share, rows * 4);
  take(w.weight, whole * 4);
  take(w.hot, whole * 4);
  if (narrow(op)) {
    take(w.parts, ttk_narrow_parts_bytes(n));
    return w;
  }
  take(w.grads, rows * piece * es);
  take(w.acc, (size_t)cuts_of(op) * rows * (copies(op) ? padded(op) : op->dim) * 4);
  take(w.column, (size_t)piece * es);
  size_t most = stored(op) ? stored_bytes(op, piece) : 0;
  const int last = (int)(op->classes - (op->classes - 1) / piece * piece);
  for (int i = 0; i < 2; ++i) {
    const int n = i ? last : (int)(piece < op->classes ? piece : op->classes);
    const int cuts = cuts_of(op), each = n / cuts / 64 * 64;
    const size_t whole = ttk_gemm_partial_bytes(cuts > 1 && each > 0 ? of_dx(op, each, cuts, piece) : of_dx(op, n, 1, piece));
    const size_t rest = cuts > 1 && each > 0 && n > each * cuts ? ttk_gemm_partial_bytes(of_dx(op, n - each * cuts, 1, piece)) : 0;
    const size_t need[3] = {whole > rest ? whole : rest, ttk_gemm_partial_bytes(of_dw(op, n, piece, false)),
                            ttk_gemm_partial_bytes(of_dw(op, n, piece, true))};
    for (int k = 0; k < 3; ++k) most = need[k] > most ? need[k] : most;
  }
  take(w.pieces, most);
  return w;
}
Rows rows_of(char *ws, const Scratch &w) {
  return TTLossRows{(int32_t *)(ws + w.of), (int32_t *)(ws + w.at), (int32_t *)(ws + w.label), (float *)(ws + w.lse), (float *)(ws + w.share), (float *)(ws + w.weight),
                    (float *)(ws + w.hot), (float *)(ws + w.back), (int64_t *)(ws + w.offsets)};
}
TTNarrow narrow_of(const tt_loss *op, const void *x, const void *w, const void *bias, char *ws, const Scratch &need) {
  const bool as_it_is = op->dtype != TT_F32 && op->dim == padded(op) && aligned(w, 16);
  return TTNarrow{op->dtype, op->dim, padded(op), op->classes, op->rows, x, op->ld_x ? op->ld_x : op->dim, w, bias, rows_of(ws, need), ws + need.x,
                  as_it_is ? nullptr : ws + need.copy, (float *)(ws + need.starts)};
}
unsigned grid_of(long long items) {
  const long long blocks = (items + TT_BLOCK - 1) / TT_BLOCK;
  return (unsigned)(blocks < 1 ? 1 : blocks > 16384 ? 16384 : blocks);
}
template <class T> tt_status gather(const tt_loss *op, const void *x, const Rows &r, void *to, hipStream_t s) {
  const int ld = padded(op), dim = op->dim;
  const long long rows = op->rows, ld_x = op->ld_x ? op->ld_x : op->dim;
  hipLaunchKernelGGL(k_loss_gather<T>, dim3(grid_of(rows * tt_ceil_div(ld, 16 / (int)sizeof(T)))), dim3(TT_BLOCK), 0, s, (const T *)x, ld_x, rows, dim, r,
                     (T *)to, ld);
  return tt_launch_status();
}
template <class T> tt_status write_dx(const tt_loss *op, const float *acc, const Rows &r, void *dx, hipStream_t s) {
  const int dim = op->dim, ld_acc = copies(op) ? padded(op) : op->dim, cuts = cuts_of(op);
  const long long rows = op->rows, ld = op->ld_dx ? op->ld_dx : op->dim;
  hipLaunchKernelGGL(k_loss_dx<T>, dim3(grid_of(rows * tt_ceil_div(dim, 4))), dim3(TT_BLOCK), 0, s, acc, ld_acc, cuts, rows, dim, r, (T *)dx, ld);
  return tt_launch_status();
}
template <class T> tt_status pad(const tt_loss *op, const void *w, int classes, void *to, hipStream_t s) {
  const int dim = op->dim, ld = padded(op);
  const long long rows = classes;
  hipLaunchKernelGGL(k_loss_pad<T>, dim3(grid_of(rows * (ld / 8))), dim3(TT_BLOCK), 0, s, (const T *)w, rows, dim, (T *)to, ld);
  return tt_launch_status();
}
template <class T> tt_status clear(void *p, long long n, hipStream_t s) {
  hipLaunchKernelGGL(k_loss_clear<T>, dim3(grid_of(n)), dim3(TT_BLOCK), 0, s, (T *)p, n);
  return tt_launch_status();
}
// The logits of n classes from c on, fp32, in `grads`.
tt_status logits(const tt_loss *op, char *ws, const Scratch &need, const void *w, const void *bias, long long c, int n, long long piece, hipStream_t s) {
  TTGemm g = of_stored(op, n, piece);
  g.a = ws + need.x;
  g.b = (const float *)w + c * op->dim;
  g.bias = bias ? (const float *)bias + c : nullptr;
  g.out = ws + need.grads;
  return ttk_gemm(g, ws + need.pieces, s);
}
#define TT_BY_TYPE(call, dtype, ...) \
  ((dtype) == TT_F32 ? call<float>(__VA_ARGS__) : (dtype) == TT_BF16 ? call<ttg::bf16>(__VA_ARGS__) : call<ttg::f16>(__VA_ARGS__))

}  // namespace

extern "C" size_t tt_cross_entropy_workspace_bytes(const tt_loss *op, int backward) {
  if (check(op) != TT_OK) return 0;
  return scratch(op, backward != 0).total;
}

extern "C" tt_status tt_cross_entropy_forward(const tt_loss *op, const void *x, const void *w, const void *bias, const int64_t *labels, float *loss, float *stats,
                                              void *workspace, size_t workspace_bytes, void *stream) {
  tt_status st = check(op);
  if (st != TT_OK) return st;
  const bool some = op->rows > 0, whole = op->reduce != TT_REDUCE_NONE;
  if (!some && !whole) return TT_OK;
  const size_t es = elem(op->dtype);
  if (!loss || (some && (!x || !w || !labels || !stats))) return TT_ERR_INVALID_ARG;
  const void *ptrs[6] = {x, w, bias, labels, loss, stats};
  const size_t sizes[6] = {es, es, es, 8, 4, 8};
  for (int i = 0; i < 6; ++i) {
    if (!aligned(ptrs[i], sizes[i])) return TT_ERR_INVALID_ARG;
    for (int j = 4; j < 6; ++j)
      if (i < j && ptrs[j] && ptrs[i] == ptrs[j]) return TT_ERR_INVALID_ARG;
  }
  const Scratch need = scratch(op, false);
  if (!workspace || ((uintptr_t)workspace & 255) != 0 || workspace_bytes < need.total) return TT_ERR_WORKSPACE;
  hipStream_t s = (hipStream_t)stream;
  char *ws = (char *)workspace;
  const Rows r = rows_of(ws, need);
  const long long rows = op->rows, ignored = op->ignore_index, piece = piece_of(op, false);
  const int classes = op->classes, reduce = op->reduce;
  float2 *each = (float2 *)stats;
  float *losses = whole ? nullptr : loss;
  hipLaunchKernelGGL(k_loss_rows, dim3(1), dim3(SCAN), 0, s, labels, rows, classes, ignored, reduce, (const float2 *)nullptr, (const float *)nullptr, 0, 0, 0, losses, each, r);
  if ((st = tt_launch_status()) != TT_OK) return st;
  if (some) {
    if (!narrow(op) && (st = TT_BY_TYPE(gather, op->dtype, op, x, r, ws + need.x, s)) != TT_OK) return st;
    float2 *run = (float2 *)(ws + need.run);
    if (narrow(op)) {
      const TTNarrow n = narrow_of(op, x, w, bias, ws, need);
      if ((st = ttk_narrow_take(n, s)) != TT_OK) return st;
      if ((st = ttk_narrow_stats(n, (float *)(ws + need.stats), (float *)(ws + need.picked), stats, losses, s)) != TT_OK) return st;
    }
    for (long long c = 0; c < classes && !narrow(op); c += piece) {
      const int n = (int)(classes - c < piece ? classes - c : piece);
      const int first = c == 0, last = c + n == classes;
      int tiles;
      if (stored(op)) {
        float *z = (float *)(ws + need.grads);
        if ((st = logits(op, ws, need, w, bias, c, n, piece, s)) != TT_OK) return st;
        tiles = tt_ceil_div(n, COLUMNS);
        hipLaunchKernelGGL(k_loss_pairs, dim3((unsigned)tt_ceil_div(rows, TT_BLOCK / 64), (unsigned)(tiles < 65535 ? tiles : 65535)), dim3(TT_BLOCK), 0, s, (const float *)z, piece,
                           rows, n, (int)c, r, (float2 *)(ws + need.stats), (float *)(ws + need.picked));
        if ((st = tt_launch_status()) != TT_OK) return st;
      } else {
        TTGemm g = of_logits(op, n, false, 0);
        g.a = ws + need.x;
        g.b = (const char *)w + (size_t)c * op->dim * es;
        if (copies(op)) {
          if ((st = TT_BY_TYPE(pad, op->dtype, op, g.b, n, ws + need.copy, s)) != TT_OK) return st;
          g.b = ws + need.copy;
        }
        g.bias = bias ? (const char *)bias + (size_t)c * es : nullptr;
        g.offsets = r.offsets;
        g.stats = (float *)(ws + need.stats);
        g.picked = (float *)(ws + need.picked);
        g.labels = r.label;
        g.first = (int)c;
        if ((st = ttk_gemm(g, nullptr, s)) != TT_OK) return st;
        tiles = tt_ceil_div(n, ttk_gemm_tile(g));
      }
      hipLaunchKernelGGL(k_loss_fold, dim3((unsigned)tt_ceil_div(rows, 16)), dim3(TT_BLOCK), 0, s, (const float2 *)(ws + need.stats), tiles, rows, first, last, r, run,
                         (const float *)(ws + need.picked), each, losses);
    }
  }
  if (whole) hipLaunchKernelGGL(k_loss_sum, dim3(1), dim3(SCAN), 0, s, (const float2 *)each, rows, r, reduce, loss);
  return tt_launch_status();
}

extern "C" tt_status tt_cross_entropy_backward(const tt_loss *op, const void *x, const void *w, const void *bias, const int64_t *labels, const float *stats,
                                               const float *grad_loss, void *dx, void *dw, void *dbias, void *workspace, size_t workspace_bytes,
                                               void *stream) {
  tt_status st = check(op);
  if (st != TT_OK) return st;
  if (!dx && !dw && !dbias) return TT_OK;
  const bool some = op->rows > 0;
  const size_t es = elem(op->dtype);
  if (some && (!x || !w || !labels || !stats || !grad_loss)) return TT_ERR_INVALID_ARG;
  const void *ptrs[9] = {x, w, bias, labels, stats, grad_loss, dx, dw, dbias};
  const size_t sizes[9] = {es, es, es, 8, 8, 4, es, es, es};
  for (int i = 0; i < 9; ++i) {
    if (!aligned(ptrs[i], sizes[i])) return TT_ERR_INVALID_ARG;
    for (int j = 6; j < 9; ++j)
      if (i < j && ptrs[j] && ptrs[i] == ptrs[j]) return TT_ERR_INVALID_ARG;
  }
  hipStream_t s = (hipStream_t)stream;
  if (!some) {
    if (dw && (st = TT_BY_TYPE(clear, op->dtype, dw, (long long)op->classes * op->dim, s)) != TT_OK) return st;
    return dbias ? TT_BY_TYPE(clear, op->dtype, dbias, (long long)op->classes, s) : TT_OK;
  }
  const Scratch need = scratch(op, true);
  if (!workspace || ((uintptr_t)workspace & 255) != 0 || workspace_bytes < need.total) return TT_ERR_WORKSPACE;
  char *ws = (char *)workspace;
  const Rows r = rows_of(ws, need);
  const long long rows = op->rows, ignored = op->ignore_index, piece = piece_of(op, true);
  const int classes = op->classes, reduce = op->reduce, apart = op->dtype != TT_F32 || narrow(op), half = op->dtype == TT_F16, negative = narrow(op);
  hipLaunchKernelGGL(k_loss_rows, dim3(1), dim3(SCAN), 0, s, labels, rows, classes, ignored, reduce, (const float2 *)stats, grad_loss, apart, half, negative, (float *)nullptr, (float2 *)nullptr, r);
  if ((st = tt_launch_status()) != TT_OK) return st;
  if (!narrow(op) && (st = TT_BY_TYPE(gather, op->dtype, op, x, r, ws + need.x, s)) != TT_OK) return st;
  if (narrow(op)) {
    const TTNarrow n = narrow_of(op, x, w, bias, ws, need);
    float *parts = (float *)(ws + need.parts);
    if ((st = ttk_narrow_take(n, s)) != TT_OK) return st;
    if (dx && (st = ttk_narrow_dx(n, parts, dx, op->ld_dx ? op->ld_dx : op->dim, s)) != TT_OK) return st;
    return dw || dbias ? ttk_narrow_dw(n, reduce == TT_REDUCE_NONE, parts, dw, dbias, s) : TT_OK;
  }
  for (long long c = 0; c < classes; c += piece) {
    const int n = (int)(classes - c < piece ? classes - c : piece);
    const char *wc = (const char *)w + (size_t)c * op->dim * es;
    if (copies(op)) {
      if ((st = TT_BY_TYPE(pad, op->dtype, op, wc, n, ws + need.copy, s)) != TT_OK) return st;
      wc = ws + need.copy;
    }
    if (stored(op)) {
      if ((st = logits(op, ws, need, w, bias, c, n, piece, s)) != TT_OK) return st;
      const int to = (n + 7) & ~7;
      hipLaunchKernelGGL(k_loss_softmax, dim3(grid_of(rows * (to / 4))), dim3(TT_BLOCK), 0, s, (float *)(ws + need.grads), piece, rows, n, to, (int)c, r);
      if ((st = tt_launch_status()) != TT_OK) return st;
    } else {
      TTGemm g = of_logits(op, n, true, piece);
      g.a = ws + need.x;
      g.b = wc;
      g.bias = bias ? (const char *)bias + (size_t)c * es : nullptr;
      g.offsets = r.offsets;
      g.out = ws + need.grads;
      g.labels = r.label;
      g.lse = r.lse;
      g.row_grad = r.weight;
      g.hot = r.hot;
      g.first = (int)c;
      if ((st = ttk_gemm(g, nullptr, s)) != TT_OK) return st;
    }
    if (dx) {
      const int cuts = cuts_of(op), size = n / cuts / 64 * 64, members = cuts > 1 && size > 0 ? cuts : 1, whole = members > 1 ? size : n;
      for (int i = 0; i < 2; ++i) {
        const int from = i ? whole * members : 0, classes_of = i ? n - from : whole;
        if (classes_of == 0) continue;
        TTGemm d = of_dx(op, classes_of, i ? 1 : members, piece);
        d.a = ws + need.grads + (size_t)from * es;
        d.b = wc + (size_t)from * d.ldb * es;
        d.acc = (float *)(ws + need.acc);
        d.acc_add = c > 0 || i;
        if ((st = ttk_gemm(d, ws + need.pieces, s)) != TT_OK) return st;
      }
    }
    if (dw || dbias) {  // as in the dense operators: the sums of G's columns come beside a product
      TTGemm d = of_dw(op, n, piece, !dw);
      d.a = ws + need.grads;
      d.b = dw ? ws + need.x : ws + need.grads;
      d.out = dw ? (char *)dw + (size_t)c * op->dim * es : ws + need.column;
      d.rowsum = dbias ? (char *)dbias + (size_t)c * es : nullptr;
      d.scale = r.back;
      if ((st = ttk_gemm(d, ws + need.pieces, s)) != TT_OK) return st;
    }
  }
  return dx ? TT_BY_TYPE(write_dx, op->dtype, op, (const float *)(ws + need.acc), r, dx, s) : TT_OK;
}
