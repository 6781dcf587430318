// Softmax cross entropy, shared by its two ways: pieces of the classes through the matrix products (tt_loss.hip), and rows of up
// to 128 elements without a stored gradient of the logits (tt_loss_narrow.hip).  Internal; the C ABI is include/tt_emb.h.
#pragma once

#include "tt_internal.h"

// Rows that count stand next to each other in the work: the products leave the others out, and whatever those hold (padding
// may hold anything) meets nothing.
struct TTLossRows {
  int32_t *of, *at;         // [rows]: row of each place, place of each row (-1: does not count)
  int32_t *label;           // [rows] of each place; -1: no class
  float *lse;               // [rows] of each place: backward.  (Short rows: of, label, lse and weight up to whole steps.)
  float *share;             // [rows]: what the loss's gradient gives each place
  float *weight;            // [rows]: what G is formed with instead of it
  float *hot;               // [rows]: the label's softmax less one
  float *back;              // [1]: what that is multiplied by at the end
  int64_t *offsets;         // {0, places}
};

#define TT_LOSS_STEP 32
#define TT_LOSS_RAISE 8192.f  // what a G without its shares is formed with in fp16, whose range is short

struct TTNarrow {
  int dtype, dim, padded, classes;
  long long rows;
  const void *of_call;      // x of the call, its rows `ld` apart
  long long ld;
  const void *w, *bias;     // of the call
  TTLossRows r;             // lse: its negative
  void *x;                  // rows that count, `padded` (64 or 128) apart, zeros behind dim and behind the last one; fp32: three planes [rows][padded] of their parts
  void *copy;               // the same of w; null if w is that
  float *starts;            // [classes], and up to whole steps of TT_LOSS_STEP
};

// A row's lse and loss from the label's logit and the statistics of the other classes: m, a logit among them that the largest exceeds by little (-infinity: there is none), and s, the
// sum of exp(logit - m).  Where the label's is above, the loss is log1p of what the others have beside it, and keeps its relative precision down to the smallest numbers; else both
// terms are of one sign.  So it is never below zero.
__device__ __forceinline__ float2 row_of_loss(float2 others, float label) {
  if (!(label < INFINITY)) return float2{NAN, NAN};
  if (label > others.x) {
    const float loss = log1pf(others.y * expf(others.x - label));
    return float2{label + loss, loss};
  }
  const float more = logf(others.y + expf(label - others.x));
  return float2{others.x + more, (others.x - label) + more};
}

bool ttk_narrow_serves(int dim);
int ttk_narrow_padded(int dim);
size_t ttk_narrow_stats_bytes(const TTNarrow &n);  // (sizes alone are looked at)
size_t ttk_narrow_parts_bytes(const TTNarrow &n);
tt_status ttk_narrow_take(const TTNarrow &n, hipStream_t s);  // writes x, copy and starts: before the others
// picked: [rows]; each: the rows' pairs (lse, loss); loss: the losses again, or null
tt_status ttk_narrow_stats(const TTNarrow &n, float *stats, float *picked, float *each, float *loss, hipStream_t s);
tt_status ttk_narrow_dx(const TTNarrow &n, float *parts, void *dx, long long ld_dx, hipStream_t s);
tt_status ttk_narrow_dw(const TTNarrow &n, bool shares, float *parts, void *dw, void *dbias, hipStream_t s);
