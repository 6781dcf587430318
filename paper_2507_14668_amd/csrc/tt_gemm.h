// Matrix products with an epilogue, shared by the dense operators (tt_dense.hip) and the orthogonalised update
// (tt_ortho.hip).  Internal; the C ABI is include/tt_emb.h.
//
//   out[m][n] = act(alpha * sum_k A(m, k) B(n, k) + bias[n]) + beta * res[m][n]
//
// An operand is stored either K-contiguous, [row][k], or row-contiguous, [k][row]; `lda` / `ldb` are the elements between
// two stored rows.  One description covers one product, a batch at a fixed step, and groups of rows given by offsets.
#pragma once

#include "tt_internal.h"

#define TT_GEMM_BATCH 0     // member z at z * step of every operand
#define TT_GEMM_RAGGED_M 1  // rows [start(z), end(z)) of A, res and out belong to group z, whose B and bias are at z * step
#define TT_GEMM_RAGGED_K 2  // group z sums over the stored rows [start(z), end(z)) of A and B; its out is at z * step

// What becomes of the sums z = alpha * sum + bias of a tile, beside what the fields bias, pre, act and res say (PLAIN); the others
// are the softmax loss's (tt_loss.hip), each for the layouts that it needs: rows of z by K-contiguous operands, ACC with a
// row-contiguous B, SCALED with both row-contiguous.
#define TT_GEMM_PLAIN 0
#define TT_GEMM_STATS 1    // nothing is stored but, of each row's columns in the tile, the largest z and the sum of exp(z - it), the label's z apart
#define TT_GEMM_SOFTMAX 2  // out = (n is the label ? hot[m] : exp(z - lse[m])) * row_grad[m], zeros in columns N .. n_padded - 1
#define TT_GEMM_ACC 3      // acc[m][n] = z, plus what is there if acc_add, in fp32
#define TT_GEMM_SCALED 4   // out and rowsum times *scale

struct TTGemm {
  int dtype, out_dtype;        // of the operands, bias, res; of out
  int a_kc, b_kc;              // 1: K-contiguous
  int mode;
  const void *a, *b;
  void *out;
  long long lda, ldb, ldo, a_step, b_step, o_step;
  int like_N;                  // not 0: tiles and pieces are chosen as for this N
  int M, N, K;                 // RAGGED_M: M rows in all; RAGGED_K: K stored rows in all
  int batch;                   // members or groups
  const int64_t *offsets;      // DEVICE [batch + 1], ragged modes
  int symmetric;               // BATCH: out is symmetric (A and B are one operand, res is symmetric): half its tiles are computed
  int zero_rest;               // RAGGED_M: rows of out outside every group are cleared (else left as they were)
  const void *bias;            // [N], nullable
  const void *res;             // nullable
  void *pre;                   // nullable: alpha * sum + bias, rounded, [M][N]
  void *rowsum;                // nullable, RAGGED_K and BATCH: sum_k A(m, k), [M] per member
  long long bias_step, ldr, r_step, ldp, p_step, rs_step;
  int act;
  float alpha, beta;
  int epilogue;                // TT_GEMM_PLAIN ...
  int large;                   // tiles of 128 also where those are few but their sums can be cut into pieces for the whole card
  int a_padded;                // 16-bit A whose rows go on with zeros (K-contiguous) or anything (else) up to a multiple of 8
  int b_padded;                // the same of a row-contiguous B whose rows go on with anything
  float *stats;                // STATS: pairs [column tile][M]
  float *picked;               // STATS: [M]
  const int32_t *labels;       // STATS, SOFTMAX: [M], first + the label's column; others are no column's
  int first;
  const float *lse, *row_grad; // SOFTMAX: [M]
  const float *hot;            // SOFTMAX: [M], the label's softmax less one
  int n_padded;                // SOFTMAX
  float *acc;                  // ACC: [batch][M][N], fp32
  int acc_add;
  const float *scale;          // SCALED: DEVICE
  int parts;                   // fp32 operands: bf16 parts of each that are multiplied (3: fp32's precision, 2: 16 bits)
};

// relu in fp32: which side of its kink a result lies on decides whole rows of gradients, so results that rounding could have taken to the
// other side are formed again in 64 bits (settle_signs in tt_gemm_device.h).
__host__ __device__ inline bool ttk_gemm_settles(const TTGemm &g) { return g.dtype == TT_F32 && g.act == TT_ACT_RELU; }
// A piece of a cut product: sums [M][N], then sums of A's rows [M]; with settled signs also squares of A's rows [M] and of B's [N].
__host__ __device__ inline long long ttk_gemm_piece_floats(const TTGemm &g) {
  return (long long)g.M * (g.N + 1LL) + (ttk_gemm_settles(g) ? (long long)g.M + g.N : 0);
}

// Long sums over few tiles of out are cut into pieces of K that run side by side; the pieces' sums go to `partial` and a
// second launch adds them in order.  How many follows from types and sizes alone, so that a caller's workspace query knows.
size_t ttk_gemm_partial_bytes(const TTGemm &g);  // 0: not cut (addresses are not looked at: enough for any)
// Enqueues the product.  partial: ttk_gemm_partial_bytes(g) bytes of DEVICE memory, 256-byte aligned.
tt_status ttk_gemm(const TTGemm &g, void *partial, hipStream_t s);

int ttk_gemm_tile(const TTGemm &g);  // the side of its tiles: the columns of a tile of stats

// Rows of a group from which its sum is cut, for tiles of e x e (RAGGED_K); `least` steps of bk at least.
int ttk_gemm_chunk(const TTGemm &g, int e, int bk, int least);
size_t ttk_gemm_chunk_bytes(const TTGemm &g, int chunk);  // of the pieces' sums
tt_status ttk_gemm_join_groups(const TTGemm &g, int chunk, int bk, const float *partial, hipStream_t s);
// Large 16-bit products on aligned operands (tt_gemm_direct.hip); ttk_gemm passes them on.
bool ttk_gemm_direct_serves(const TTGemm &g);
int ttk_gemm_direct_chunk(const TTGemm &g);  // 0: nothing is cut
size_t ttk_gemm_direct_bytes(const TTGemm &g);
tt_status ttk_gemm_direct(const TTGemm &g, void *partial, hipStream_t s);
// Few rows with a K-contiguous weight (tt_gemm_rows.hip); likewise.
bool ttk_gemm_rows_serves(const TTGemm &g);
tt_status ttk_gemm_rows(const TTGemm &g, hipStream_t s);
