// Softmax cross entropy, shared by its two ways: pieces of the classes through the matrix products (tt_loss.hip), and rows of up
// to 128 16-bit elements without a stored gradient of the logits (tt_loss_narrow.hip).  Internal; the C ABI is include/tt_emb.h.
#pragma once

#include "tt_internal.h"

// Rows that count stand next to each other in the work: the products leave the others out, and whatever those hold (padding
// may hold anything) meets nothing.
struct TTLossRows {
  int32_t *of, *at;         // [rows]: row of each place, place of each row (-1: does not count)
  int32_t *label;           // [rows] of each place; -1: no class
  float *lse;               // [rows] of each place: backward
  float *share;             // [rows]: what the loss's gradient gives each place
  float *weight;            // [rows]: what G is formed with instead of it
  float *back;              // [1]: what that is multiplied by at the end
  int64_t *offsets;         // {0, places}
};

struct TTNarrow {
  int dtype, dim, padded, classes;
  long long rows;
  const void *x;            // rows that count, `padded` (64 or 128) apart, zeros behind dim and behind the last one
  const void *w, *bias;     // of the call
  TTLossRows r;
};

bool ttk_narrow_serves(int dtype, int dim);
int ttk_narrow_padded(int dim);
// Runs of the classes that a row's statistics and dx come in, and runs of the rows that dW comes in.
int ttk_narrow_runs(long long rows, int classes);
int ttk_narrow_row_runs(long long rows, int classes);
// stats: pairs [run][rows] of each row's largest logit, about, and the sum of exp(logit - it)
tt_status ttk_narrow_stats(const TTNarrow &n, float *stats, hipStream_t s);
tt_status ttk_narrow_picked(const TTNarrow &n, float *picked, hipStream_t s);
// parts: sums [run][rows][padded] of exp(z - lse) W, times 2^13
tt_status ttk_narrow_dx(const TTNarrow &n, float *parts, void *dx, long long ld_dx, hipStream_t s);
// parts: [row run][classes][padded + 1], only where there are several
tt_status ttk_narrow_dw(const TTNarrow &n, bool shares, float *parts, void *dw, void *dbias, hipStream_t s);
