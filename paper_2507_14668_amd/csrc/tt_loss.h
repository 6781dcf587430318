// Softmax cross entropy, shared by its two ways: pieces of the classes through the matrix products (tt_loss.hip), and rows of up
// to 128 16-bit elements without a stored gradient of the logits (tt_loss_narrow.hip).  Internal; the C ABI is include/tt_emb.h.
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
  float *back;              // [1]: what that is multiplied by at the end
  int64_t *offsets;         // {0, places}
};

#define TT_LOSS_STEP 32

#ifdef __HIPCC__
// What place i's row has for its loss and lse: s is its largest logit (or one near it) and the sum of exp(logit - that).
__device__ __forceinline__ void ttk_loss_of(const TTLossRows &w, long long i, float2 s, float picked, float *loss, float *lse) {
  const bool bad = w.label[i] < 0;
  const int r = w.of[i];
  lse[r] = bad ? NAN : s.x + logf(s.y);
  // (the difference of the logits first: near a loss of zero lse less the label's logit would be lse's rounding)
  loss[r] = bad ? NAN : (s.x - picked) + logf(s.y);
}
#endif

struct TTNarrow {
  int dtype, dim, padded, classes;
  long long rows;
  const void *x;            // rows that count, `padded` (64 or 128) apart, zeros behind dim and behind the last one
  const void *w, *bias;     // of the call
  TTLossRows r;             // lse: its negative
  float *starts;            // [classes], and up to whole steps of TT_LOSS_STEP
  void *copy;               // [classes][padded]; null if w is that
};

bool ttk_narrow_serves(int dtype, int dim);
int ttk_narrow_padded(int dim);
size_t ttk_narrow_stats_bytes(const TTNarrow &n);  // (sizes alone are looked at)
size_t ttk_narrow_parts_bytes(const TTNarrow &n);
tt_status ttk_narrow_classes(const TTNarrow &n, hipStream_t s);  // writes starts and copy: before the others
tt_status ttk_narrow_stats(const TTNarrow &n, float *stats, float *loss, float *lse, hipStream_t s);
tt_status ttk_narrow_dx(const TTNarrow &n, float *parts, void *dx, long long ld_dx, hipStream_t s);
tt_status ttk_narrow_dw(const TTNarrow &n, bool shares, float *parts, void *dw, void *dbias, hipStream_t s);
