// Orthogonalised updates of batches of small matrices, one launch for the whole iteration (tt_ortho_slice.hip).
#pragma once

#include "tt_gemm.h"

#define TT_SLICE_MAX_STEPS TT_ORTHO_MAX_STEPS

// Matrix z: element (s, l) of its short and its long side at z * b_step + s * s_step + l * l_step.
struct TTSlices {
  int dtype;                       // of in and out; the core update is fp32
  int shorter, longer;
  long long batch;
  const void *in;
  long long in_b, in_s, in_l;
  void *out;
  long long out_b, out_s, out_l;
  // core update (mom != null): in is the gradient, out the core; mom has the gradient's steps
  float *mom;
  float mu, rate;                  // out -= rate * result
  int nesterov;
  float eps;
  int steps;
  float c[3 * TT_SLICE_MAX_STEPS];
};

bool ttk_slices_serves(long long shorter, long long longer);
tt_status ttk_slices(const TTSlices *p, int n, hipStream_t s);  // n <= 3 batches of one dtype side by side
