// Routing of rows to experts: scores, choice, weights and their gradient, and the experts' order of the choices.
#include "tt_gemm_device.h"

namespace {
using namespace ttg;
typedef unsigned long long u64;

struct Route {  // of a call, by value to the kernels
  const void *logits;
  const float *bias, *grad;
  int64_t *experts;
  float *weights;
  void *dlogits;
  long long rows, ld, ldd;
  int num, k, groups, top_groups, group_size, group_mul;
  int sigmoid, renorm;
  float scale;
};

// ---- reductions and reads over the LANES (16 or 64) of a row ---------------------------------------
__device__ __forceinline__ int row_lane(int lanes) { return threadIdx.x & (lanes - 1); }
template <int LANES> __device__ __forceinline__ int from_lane(int v, int lane) {  // lane: the same in all of the row's
  if constexpr (LANES == 64) return __builtin_amdgcn_readlane(v, lane);
  else return __shfl(v, (threadIdx.x & 63 & ~(LANES - 1)) | lane, 64);
}
template <int LANES> __device__ __forceinline__ u64 ballot_of(bool p) {  // of the row's lanes
  if constexpr (LANES == 64) return __ballot(p);
  else return __ballot(p) >> (threadIdx.x & 63 & ~(LANES - 1)) & ((1ull << LANES) - 1);
}
// Neighbours within rows of 16 lanes, then across those, without LDS; the last lane has the result.
template <int CTRL, int ROWS> __device__ __forceinline__ unsigned max_dpp(unsigned v) {
  const unsigned t = (unsigned)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, ROWS, 0xf, false);
  return t > v ? t : v;
}
template <int LANES> __device__ __forceinline__ unsigned max_of(unsigned v) {
  v = max_dpp<0x111, 0xf>(v);  // from 1, 2, 4, 8 lanes before
  v = max_dpp<0x112, 0xf>(v);
  v = max_dpp<0x114, 0xf>(v);
  v = max_dpp<0x118, 0xf>(v);
  if constexpr (LANES == 64) {
    v = max_dpp<0x142, 0xa>(v);  // the ends of rows 0 and 2 to rows 1 and 3
    v = max_dpp<0x143, 0xc>(v);  // the end of row 1 to rows 2 and 3
  }
  return (unsigned)from_lane<LANES>((int)v, LANES - 1);
}
template <int LANES> __device__ __forceinline__ float largest_of(float v) {  // NaN does not count
#pragma unroll
  for (int o = LANES / 2; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor(v, o, 64));
  return v;
}
template <int LANES> __device__ __forceinline__ float sum_of(float v) {
#pragma unroll
  for (int o = LANES / 2; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
  return v;
}
template <int LANES> __device__ __forceinline__ double sum_of(double v) {
#pragma unroll
  for (int o = LANES / 2; o > 0; o >>= 1) {
    const long long b = __builtin_bit_cast(long long, v);
    const int lo = __shfl((int)b, (threadIdx.x & 63) ^ o, 64), hi = __shfl((int)(b >> 32), (threadIdx.x & 63) ^ o, 64);
    v += __builtin_bit_cast(double, ((long long)hi << 32) | (unsigned)lo);
  }
  return v;
}
// The order of numbers as that of unsigned integers: -infinity and masked ones 0 (there is no choice), NaN the largest.
__device__ __forceinline__ u64 key_of(double c) {
  if (c != c) return ~0ull;
  if (c == -INFINITY) return 0;
  const long long b = __builtin_bit_cast(long long, c + 0.0);  // (-0 is 0)
  return b < 0 ? ~(u64)b : (u64)b | 0x8000000000000000ull;
}
__device__ __forceinline__ double value_of(u64 key) {  // of keys other than 0; ~0 is a NaN as it is
  return __builtin_bit_cast(double, (long long)(key >> 63 ? key & 0x7fffffffffffffffull : ~key));
}
// The row's lane with the largest key, the first of them; its key is `best`.
template <int LANES> __device__ __forceinline__ int pick(u64 key, u64 &best) {
  const unsigned hi = (unsigned)(key >> 32), top = max_of<LANES>(hi);
  u64 lanes = ballot_of<LANES>(hi == top);
  unsigned low;
  if (__ballot(__popcll(lanes) > 1)) {  // (of any row of the wavefront)
    low = max_of<LANES>(hi == top ? (unsigned)key : 0u);
    lanes = ballot_of<LANES>(hi == top && (unsigned)key == low);
  } else {
    low = (unsigned)from_lane<LANES>((int)(unsigned)key, __ffsll(lanes) - 1);
  }
  best = (u64)top << 32 | low;
  return __ffsll(lanes) - 1;
}
template <int LANES> __device__ __forceinline__ double read_lane64(double v, int lane) {
  const long long b = __builtin_bit_cast(long long, v);
  const unsigned lo = (unsigned)from_lane<LANES>((int)b, lane), hi = (unsigned)from_lane<LANES>((int)(b >> 32), lane);
  return __builtin_bit_cast(double, (long long)((u64)hi << 32 | lo));
}

// The lane's EL logits, experts EL lane .. + EL - 1 (-infinity behind the last one).
template <class T, int LANES, int EL> __device__ __forceinline__ void load_logits(const Route &p, long long row, float z[EL]) {
  const int first = EL * row_lane(LANES), valid = p.num - first;
  const T *src = (const T *)p.logits + row * p.ld + first;
  if constexpr (EL >= 4) {
    load_n<T, EL>(src, valid, z);
  } else {
#pragma unroll
    for (int i = 0; i < EL; ++i) z[i] = i < valid ? to_f32(src[i]) : 0.f;
  }
#pragma unroll
  for (int i = 0; i < EL; ++i) z[i] = i < valid ? z[i] : -INFINITY;
}

constexpr int ROUTE_WAVES = 4;

// LANES lanes take a row (16: up to 64 experts and 16 choices, four rows a wavefront; 64: all others): scores in 64 bits, then choice after choice the largest
// key of all lanes.  16384 rows of 256 experts, sigmoid, four of eight groups, eight choices 37 us: the 64-bit exp and division, and about 60 instructions a
// choice.  65536 rows of 64 experts and four choices 21 us; the call with the order 57 us by 64 lanes a row, 43 by 16.
template <class T, int LANES, int EL, bool GROUPS> __global__ void __launch_bounds__(64 * ROUTE_WAVES) k_route(Route p) {
  static_assert(!GROUPS || LANES == 64, "groups");
  constexpr int PER = 64 / LANES;  // rows a wavefront
  __shared__ u64 room[GROUPS ? ROUTE_WAVES : 1][GROUPS ? 64 * EL : 1];
  const int lane = row_lane(LANES), wave = threadIdx.x >> 6, first = EL * lane;
  float bias[EL];
#pragma unroll
  for (int i = 0; i < EL; ++i) bias[i] = p.bias && first + i < p.num ? p.bias[first + i] : 0.f;
  for (long long r0 = ((long long)blockIdx.x * ROUTE_WAVES + wave) * PER; r0 < p.rows; r0 += (long long)gridDim.x * ROUTE_WAVES * PER) {
    const bool live = r0 + (threadIdx.x & 63) / LANES < p.rows;
    const long long r = live ? r0 + (threadIdx.x & 63) / LANES : p.rows - 1;
    float z[EL];
    double s[EL];
    load_logits<T, LANES, EL>(p, r, z);
    if (p.sigmoid) {
#pragma unroll
      for (int i = 0; i < EL; ++i) s[i] = 1.0 / (1.0 + exp(-(double)z[i]));
    } else {
      float top = z[0];
#pragma unroll
      for (int i = 1; i < EL; ++i) top = fmaxf(top, z[i]);
      top = largest_of<LANES>(top);
      if (top == -INFINITY) top = 0.f;
      double sum = 0;
#pragma unroll
      for (int i = 0; i < EL; ++i) {
        s[i] = exp((double)z[i] - (double)top);
        sum += s[i];
      }
      sum = sum_of<LANES>(sum);
      const double inv = sum == 0 ? 0.0 : 1.0 / sum;
#pragma unroll
      for (int i = 0; i < EL; ++i) s[i] *= inv;
    }
    u64 key[EL];
#pragma unroll
    for (int i = 0; i < EL; ++i) key[i] = z[i] == -INFINITY ? 0 : key_of(s[i] + (double)bias[i]);
    if constexpr (GROUPS) {
      // each group's two best, by 64 / groups lanes (a power of two of them) and then by those together
#pragma unroll
      for (int i = 0; i < EL; ++i) room[wave][first + i] = key[i];
      tt_wave_lds_order();
      int per = 1;
      while (2 * per * p.groups <= 64) per *= 2;
      const int g = lane / per;
      u64 a = 0, b = 0;  // the best and the next
      if (g < p.groups)
        for (int e = lane % per; e < p.group_size; e += per) {
          const u64 x = room[wave][g * p.group_size + e];
          b = x > a ? a : x > b ? x : b;
          a = x > a ? x : a;
        }
      for (int o = 1; o < per; o *= 2) {
        const u64 x = (u64)(unsigned)__shfl((int)(a >> 32), lane ^ o, 64) << 32 | (unsigned)__shfl((int)a, lane ^ o, 64);
        const u64 y = (u64)(unsigned)__shfl((int)(b >> 32), lane ^ o, 64) << 32 | (unsigned)__shfl((int)b, lane ^ o, 64);
        const u64 least = x < a ? x : a, next = y > b ? y : b;
        a = x > a ? x : a;
        b = least > next ? least : next;
      }
      u64 strength = 0;
      if (g < p.groups && lane % per == 0 && a) strength = key_of(value_of(a) + (b ? value_of(b) : 0.0));
      if (a && strength == 0) strength = 1;  // (a sum beyond the range of numbers is still a group)
      if (lane % per != 0 || g >= p.groups) strength = 0;
      u64 keep = 0;
      for (int t = 0; t < p.top_groups; ++t) {
        u64 best;
        const int l = pick<64>(strength, best);
        if (best == 0) break;
        keep |= 1ull << (l / per);
        strength = lane == l ? 0 : strength;
      }
#pragma unroll
      for (int i = 0; i < EL; ++i) key[i] = (keep >> (((first + i) * p.group_mul) >> 20 & 63)) & 1 ? key[i] : 0;
      tt_wave_lds_order();
    }
    int mine = -1;  // lane j has choice j
    double score = 0;
    for (int j = 0; j < p.k; ++j) {
      u64 best = key[0];
      int at = 0;
#pragma unroll
      for (int i = 1; i < EL; ++i) {
        at = key[i] > best ? i : at;
        best = key[i] > best ? key[i] : best;
      }
      double sc = s[0];
#pragma unroll
      for (int i = 1; i < EL; ++i) sc = at == i ? s[i] : sc;
      u64 top;
      const int l = pick<LANES>(best, top), which = from_lane<LANES>(at, l);
      sc = read_lane64<LANES>(sc, l);
      if (lane == j && top != 0) {  // (0: none is left)
        mine = EL * l + which;
        score = sc;
      }
#pragma unroll
      for (int i = 0; i < EL; ++i) key[i] = lane == l && which == i ? 0 : key[i];
    }
    if (p.renorm) {
      const double sum = sum_of<LANES>(score);
      score = sum == 0 ? 0.0 : score / sum;
    }
    if (live && lane < p.k) {
      p.experts[r * p.k + lane] = mine;
      p.weights[r * p.k + lane] = (float)((double)p.scale * score);
    }
  }
}

// dz = s (ds - sum ds s) (softmax) or ds s (1 - s), with ds of the chosen experts from the gradients g of their weights, in 64 bits as the scores are: those of
// chosen experts may be far below what fp32 holds.  Renormalised weights w = s / sum s have the gradient t = w (g - sum g w) beside them, which no small sum is divided into:
// dz = t (softmax: the chosen scores' share of all others cancels) or t (1 - s).  Only softmax weights as they are need every expert's exp.
// 16384 rows of 256 experts, eight choices: 15 us (sigmoid) to 20 (softmax), where the bytes take 7; renormalised sigmoid 17.5, in fp32 14.9.
template <class T, int LANES, int EL> __global__ void __launch_bounds__(64 * ROUTE_WAVES) k_route_backward(Route p) {
  constexpr int PER = 64 / LANES;
  __shared__ float room[ROUTE_WAVES * PER][LANES * EL];
  const int lane = row_lane(LANES), wave = threadIdx.x >> 6, first = EL * lane;
  float *logits_of = room[threadIdx.x / LANES];
  for (long long r0 = ((long long)blockIdx.x * ROUTE_WAVES + wave) * PER; r0 < p.rows; r0 += (long long)gridDim.x * ROUTE_WAVES * PER) {
    const bool live = r0 + (threadIdx.x & 63) / LANES < p.rows;
    const long long r = live ? r0 + (threadIdx.x & 63) / LANES : p.rows - 1;
    float z[EL];
    load_logits<T, LANES, EL>(p, r, z);
    const int64_t asked = lane < p.k ? p.experts[r * p.k + lane] : -1;
    const int mine = asked >= 0 && asked < p.num ? (int)asked : -1;
    const double g = mine >= 0 ? (double)p.scale * (double)p.grad[r * p.k + lane] : 0.0;
#pragma unroll
    for (int i = 0; i < EL; ++i) logits_of[first + i] = z[i];
    tt_wave_lds_order();
    const float chosen = mine >= 0 ? logits_of[mine] : -INFINITY;
    tt_wave_lds_order();
    double s = 0, inv = 0, each[EL] = {};  // the chosen expert's score; softmax: one over the sum, and without renormalising the lane's exponentials
    float top = 0.f;
    if (p.sigmoid) {
      s = mine >= 0 ? 1.0 / (1.0 + exp(-(double)chosen)) : 0.0;
    } else {
      top = z[0];
#pragma unroll
      for (int i = 1; i < EL; ++i) top = fmaxf(top, z[i]);
      top = largest_of<LANES>(top);
      if (top == -INFINITY) top = 0.f;
      double sum = 0;
      if (p.renorm) {  // (it only says whether scores are zero in 64 bits, or not numbers)
        float about = 0.f;
#pragma unroll
        for (int i = 0; i < EL; ++i) about += expf(z[i] - top);
        sum = sum_of<LANES>(about);
      } else {
#pragma unroll
        for (int i = 0; i < EL; ++i) {
          each[i] = exp((double)z[i] - (double)top);
          sum += each[i];
        }
        sum = sum_of<LANES>(sum);
      }
      inv = sum == 0 ? 0.0 : 1.0 / sum;
      s = mine >= 0 ? exp((double)chosen - (double)top) * inv : 0.0;
    }
    double t;
    if (p.renorm) {
      const double total = sum_of<LANES>(s), w = total == 0 ? 0.0 : s / total;
      t = w * (g - sum_of<LANES>(g * w));
    } else {
      t = g * s;
    }
    if (p.sigmoid) t *= 1.0 / (1.0 + exp((double)chosen));
    if (mine < 0) t = 0;
    const double dot = p.sigmoid || p.renorm ? 0.0 : sum_of<LANES>(t);
    double d[EL];
#pragma unroll
    for (int i = 0; i < EL; ++i) d[i] = p.sigmoid ? 0.0 : p.renorm ? 0.0 * inv : -(each[i] * inv) * dot;
    for (int j = 0; j < p.k; ++j) {  // one after the other: an expert named twice gets both
      const int e = from_lane<LANES>(mine, j) - first;
      const double tj = read_lane64<LANES>(t, j);
#pragma unroll
      for (int i = 0; i < EL; ++i) d[i] += e == i ? tj : 0.0;
    }
    if (!live) continue;
    float out[EL];
#pragma unroll
    for (int i = 0; i < EL; ++i) out[i] = (float)d[i];
    T *to = (T *)p.dlogits + r * p.ldd + first;
    const int valid = p.num - first;
    if constexpr (EL >= 4) {
      store_n<T, EL>(to, valid, out);
    } else {
#pragma unroll
      for (int i = 0; i < EL; ++i)
        if (i < valid) to[i] = from_f32<T>(out[i]);
    }
  }
}

// ---- the experts' order: a counting sort that keeps the order of the choices of an expert ----------
// A workgroup takes a tile of choices, a wavefront a run of it.  Counts of each run, and where the runs of an expert start, are in LDS; then each run
// deals its choices 64 at a time, those of one expert by the number of lanes before (ballots over the bits of the number).  131072 choices of 256
// experts 20 us in three launches (count, sums over the tiles, deal), a few in one of 2.7.
constexpr int ORDER_THREADS = 512, ORDER_WAVES = ORDER_THREADS / 64, ORDER_TILE = 8 * ORDER_THREADS;
constexpr int ORDER_ONE = 16 * ORDER_THREADS;  // choices that one workgroup takes in a launch of its own

__device__ __forceinline__ int expert_at(const int64_t *experts, long long i, long long end, int num) {
  if (i >= end) return -1;
  const int64_t e = experts[i];
  return e >= 0 && e < num ? (int)e : -1;
}
// hist[wave][e]: counts of the wavefront's run [lo, hi)
__device__ __forceinline__ void count_runs(const int64_t *experts, long long lo, long long hi, int num, int *hist) {
  for (int i = threadIdx.x; i < ORDER_WAVES * num; i += ORDER_THREADS) hist[i] = 0;
  __syncthreads();
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  for (long long i = lo + lane; i < hi; i += 64) {
    const int e = expert_at(experts, i, hi, num);
    if (e >= 0) atomicAdd(&hist[wave * num + e], 1);
  }
  __syncthreads();
}
// Exclusive sums of count[0 .. num) in place (num <= 1024: two a thread); returns the sum of all.
__device__ __forceinline__ int scan_counts(int *count, int num, int *tmp) {
  const int e = 2 * threadIdx.x;
  const int a = e < num ? count[e] : 0, b = e + 1 < num ? count[e + 1] : 0;
  int total;
  const int before = tt_block_excl_scan_n<ORDER_THREADS>(a + b, tmp, &total);
  if (e < num) count[e] = before;
  if (e + 1 < num) count[e + 1] = before + a;
  __syncthreads();
  return total;
}
// Places of the wavefront's run; hist[wave][e] is the next place of expert e.
__device__ __forceinline__ void deal_run(const int64_t *experts, long long lo, long long hi, int num, int *hist, int32_t *slots, int32_t *sources) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  for (long long i0 = lo; i0 < hi; i0 += 64) {
    const long long i = i0 + lane;
    const int e = expert_at(experts, i, hi, num);
    u64 peers = __ballot(e >= 0);
    for (int b = 1; b < num; b *= 2) {
      const bool set = e & b;
      const u64 with = __ballot(set);
      peers &= set ? with : ~with;
    }
    int at = -1;
    if (e >= 0) {
      const int rank = __popcll(peers & ((1ull << lane) - 1));
      at = hist[wave * num + e] + rank;
    }
    tt_wave_lds_order();
    if (e >= 0 && (peers >> lane) == 1) hist[wave * num + e] = at + 1;  // the last of them
    tt_wave_lds_order();
    if (i < hi) slots[i] = at;
    if (at >= 0) sources[at] = (int32_t)i;
  }
}

__global__ void __launch_bounds__(ORDER_THREADS) k_order_one(const int64_t *experts, int n, int num, int64_t *offsets, int32_t *slots, int32_t *sources) {
  __shared__ int hist[ORDER_WAVES * TT_ROUTE_MAX_EXPERTS], starts[TT_ROUTE_MAX_EXPERTS], tmp[ORDER_WAVES + 1];
  const int wave = threadIdx.x >> 6, per = ((n + ORDER_THREADS - 1) / ORDER_THREADS) * 64;
  const long long lo = (long long)wave * per < n ? (long long)wave * per : n, hi = lo + per < n ? lo + per : n;
  count_runs(experts, lo, hi, num, hist);
  for (int e = threadIdx.x; e < num; e += ORDER_THREADS) {
    int sum = 0;
    for (int w = 0; w < ORDER_WAVES; ++w) sum += hist[w * num + e];
    starts[e] = sum;
  }
  __syncthreads();
  const int total = scan_counts(starts, num, tmp);
  for (int e = threadIdx.x; e < num; e += ORDER_THREADS) {
    offsets[e] = starts[e];
    int at = starts[e];
    for (int w = 0; w < ORDER_WAVES; ++w) {
      const int c = hist[w * num + e];
      hist[w * num + e] = at;
      at += c;
    }
  }
  if (threadIdx.x == 0) offsets[num] = total;
  for (int i = total + threadIdx.x; i < n; i += ORDER_THREADS) sources[i] = -1;
  __syncthreads();
  deal_run(experts, lo, hi, num, hist, slots, sources);
}

__device__ __forceinline__ void run_of(long long n, long long &lo, long long &hi) {
  lo = (long long)blockIdx.x * ORDER_TILE + (threadIdx.x >> 6) * (ORDER_TILE / ORDER_WAVES);
  hi = lo + ORDER_TILE / ORDER_WAVES;
  lo = lo < n ? lo : n;
  hi = hi < n ? hi : n;
}
__global__ void __launch_bounds__(ORDER_THREADS) k_order_count(const int64_t *experts, long long n, int num, int32_t *counts) {
  __shared__ int hist[ORDER_WAVES * TT_ROUTE_MAX_EXPERTS];
  long long lo, hi;
  run_of(n, lo, hi);
  count_runs(experts, lo, hi, num, hist);
  for (int e = threadIdx.x; e < num; e += ORDER_THREADS) {
    int sum = 0;
    for (int w = 0; w < ORDER_WAVES; ++w) sum += hist[w * num + e];
    counts[(long long)blockIdx.x * num + e] = sum;
  }
}
// counts[tile][e] -> the sums of the tiles before, totals[e]; 64 experts a workgroup, the tiles in eight runs
__global__ void __launch_bounds__(ORDER_THREADS) k_order_scan(int32_t *counts, long long tiles, int num, int32_t *totals) {
  __shared__ int sums[ORDER_WAVES][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, e = (int)blockIdx.x * 64 + lane;
  const long long per = (tiles + ORDER_WAVES - 1) / ORDER_WAVES, lo = wave * per, hi = lo + per < tiles ? lo + per : tiles;
  int sum = 0;
  if (e < num) {
#pragma unroll 4
    for (long long t = lo; t < hi; ++t) sum += counts[t * num + e];
  }
  sums[wave][lane] = sum;
  __syncthreads();
  int before = 0, total = 0;
  for (int w = 0; w < ORDER_WAVES; ++w) {
    before += w < wave ? sums[w][lane] : 0;
    total += sums[w][lane];
  }
  if (e >= num) return;
  for (long long t = lo; t < hi; ++t) {
    const int c = counts[t * num + e];
    counts[t * num + e] = before;
    before += c;
  }
  if (wave == 0) totals[e] = total;
}
__global__ void __launch_bounds__(ORDER_THREADS) k_order_deal(const int64_t *experts, long long n, int num, const int32_t *counts, const int32_t *totals,
                                                              int64_t *offsets, int32_t *slots, int32_t *sources) {
  __shared__ int hist[ORDER_WAVES * TT_ROUTE_MAX_EXPERTS], starts[TT_ROUTE_MAX_EXPERTS], tmp[ORDER_WAVES + 1];
  long long lo, hi;
  run_of(n, lo, hi);
  for (int e = threadIdx.x; e < num; e += ORDER_THREADS) starts[e] = totals[e];
  __syncthreads();
  const int total = scan_counts(starts, num, tmp);
  count_runs(experts, lo, hi, num, hist);
  for (int e = threadIdx.x; e < num; e += ORDER_THREADS) {
    if (blockIdx.x == 0) offsets[e] = starts[e];
    int at = starts[e] + counts[(long long)blockIdx.x * num + e];
    for (int w = 0; w < ORDER_WAVES; ++w) {
      const int c = hist[w * num + e];
      hist[w * num + e] = at;
      at += c;
    }
  }
  if (blockIdx.x == 0 && threadIdx.x == 0) offsets[num] = total;
  const long long end = (long long)(blockIdx.x + 1) * ORDER_TILE < n ? (long long)(blockIdx.x + 1) * ORDER_TILE : n;
  for (long long i = (long long)blockIdx.x * ORDER_TILE + threadIdx.x; i < end; i += ORDER_THREADS)
    if (i >= total) sources[i] = -1;
  __syncthreads();
  deal_run(experts, lo, hi, num, hist, slots, sources);
}

// ---- host ------------------------------------------------------------------------------------------
const long long kMostPlaces = 2147483647LL - 2 * TT_DENSE_MAX_GROUPS;  // rows that tt_dense takes

tt_status check(const tt_route *op) {
  if (!op || op->dtype < TT_F32 || op->dtype > TT_F16 || (op->scores != TT_SCORES_SOFTMAX && op->scores != TT_SCORES_SIGMOID) || op->rows < 0)
    return TT_ERR_INVALID_ARG;
  if ((op->renormalize != 0 && op->renormalize != 1) || !(fabsf(op->scale) < INFINITY)) return TT_ERR_INVALID_ARG;
  if (op->experts < 1 || op->experts > TT_ROUTE_MAX_EXPERTS || op->groups < 1 || op->groups > TT_ROUTE_MAX_GROUPS || op->experts % op->groups != 0 ||
      op->top_groups < 1 || op->top_groups > op->groups)
    return TT_ERR_SHAPE;
  if (op->choices < 1 || op->choices > TT_ROUTE_MAX_CHOICES || op->choices > op->experts / op->groups * op->top_groups) return TT_ERR_SHAPE;
  if (op->rows >= kMostPlaces / op->choices) return TT_ERR_SHAPE;
  const int64_t ld[2] = {op->ld_logits, op->ld_dlogits};
  for (int i = 0; i < 2; ++i)
    if (ld[i] != 0 && (ld[i] < op->experts || ld[i] > ((int64_t)1 << 40))) return TT_ERR_SHAPE;
  return TT_OK;
}
bool aligned(const void *p, size_t size) { return ((uintptr_t)p & (size - 1)) == 0; }
size_t elem(int dtype) { return dtype == TT_F32 ? 4 : 2; }

Route describe(const tt_route *op) {
  Route p = {};
  p.rows = op->rows;
  p.ld = op->ld_logits ? op->ld_logits : op->experts;
  p.ldd = op->ld_dlogits ? op->ld_dlogits : op->experts;
  p.num = op->experts;
  p.k = op->choices;
  p.groups = op->groups;
  p.top_groups = op->top_groups;
  p.group_size = op->experts / op->groups;
  p.group_mul = ((1 << 20) + p.group_size - 1) / p.group_size;  // e / group_size = e * this >> 20 for e < 1024
  p.sigmoid = op->scores == TT_SCORES_SIGMOID;
  p.renorm = op->renormalize;
  p.scale = op->scale;
  return p;
}
template <class T, int LANES, int EL> void launch_el(const Route &p, bool backward, hipStream_t s) {
  constexpr int ROWS = ROUTE_WAVES * 64 / LANES;
  long long blocks = (p.rows + ROWS - 1) / ROWS;
  if (blocks > 8192) blocks = 8192;
  const dim3 grid((unsigned)blocks), block(64 * ROUTE_WAVES);
  if (backward) {
    hipLaunchKernelGGL((k_route_backward<T, LANES, EL>), grid, block, 0, s, p);
    return;
  }
  if constexpr (LANES == 64) {
    if (p.top_groups < p.groups) {
      hipLaunchKernelGGL((k_route<T, LANES, EL, true>), grid, block, 0, s, p);
      return;
    }
  }
  hipLaunchKernelGGL((k_route<T, LANES, EL, false>), grid, block, 0, s, p);
}
template <class T> tt_status launch(const Route &p, bool backward, hipStream_t s) {
  const int el = tt_ceil_div(p.num, 64);
  if (p.num <= 64 && p.k <= 16 && (backward || p.top_groups == p.groups)) {
    if (p.num <= 16) launch_el<T, 16, 1>(p, backward, s);
    else if (p.num <= 32) launch_el<T, 16, 2>(p, backward, s);
    else launch_el<T, 16, 4>(p, backward, s);
  } else if (el <= 1) launch_el<T, 64, 1>(p, backward, s);
  else if (el <= 2) launch_el<T, 64, 2>(p, backward, s);
  else if (el <= 4) launch_el<T, 64, 4>(p, backward, s);
  else if (el <= 8) launch_el<T, 64, 8>(p, backward, s);
  else launch_el<T, 64, 16>(p, backward, s);
  return tt_launch_status();
}
tt_status launch(int dtype, const Route &p, bool backward, hipStream_t s) {
  return dtype == TT_F32 ? launch<float>(p, backward, s) : dtype == TT_BF16 ? launch<ttg::bf16>(p, backward, s) : launch<ttg::f16>(p, backward, s);
}

}  // namespace

extern "C" tt_status tt_route_forward(const tt_route *op, const void *logits, const float *bias, int64_t *experts, float *weights, void *stream) {
  const tt_status st = check(op);
  if (st != TT_OK) return st;
  if (op->rows == 0) return TT_OK;
  if (!logits || !experts || !weights || !aligned(logits, elem(op->dtype)) || !aligned(bias, 4) || !aligned(experts, 8) || !aligned(weights, 4))
    return TT_ERR_INVALID_ARG;
  if ((void *)experts == logits || (void *)experts == (void *)bias || (void *)weights == logits || (const float *)weights == bias || (void *)experts == (void *)weights)
    return TT_ERR_INVALID_ARG;
  Route p = describe(op);
  p.logits = logits;
  p.bias = bias;
  p.experts = experts;
  p.weights = weights;
  return launch(op->dtype, p, false, (hipStream_t)stream);
}

extern "C" tt_status tt_route_backward(const tt_route *op, const void *logits, const int64_t *experts, const float *grad_weights, void *dlogits,
                                       void *stream) {
  const tt_status st = check(op);
  if (st != TT_OK) return st;
  if (op->rows == 0) return TT_OK;
  if (!logits || !experts || !grad_weights || !dlogits || !aligned(logits, elem(op->dtype)) || !aligned(dlogits, elem(op->dtype)) || !aligned(experts, 8) ||
      !aligned(grad_weights, 4))
    return TT_ERR_INVALID_ARG;
  if (dlogits == logits || dlogits == (const void *)experts || dlogits == (const void *)grad_weights) return TT_ERR_INVALID_ARG;
  Route p = describe(op);
  p.logits = logits;
  p.experts = const_cast<int64_t *>(experts);
  p.grad = grad_weights;
  p.dlogits = dlogits;
  return launch(op->dtype, p, true, (hipStream_t)stream);
}

extern "C" size_t tt_expert_order_workspace_bytes(int64_t n, int32_t num_experts) {
  if (n <= ORDER_ONE || n > kMostPlaces || num_experts < 1 || num_experts > TT_ROUTE_MAX_EXPERTS) return 0;
  return (((size_t)tt_ceil_div(n, ORDER_TILE) + 1) * num_experts * 4 + 255) & ~(size_t)255;
}

extern "C" tt_status tt_expert_order(const int64_t *experts, int64_t n, int32_t num_experts, int64_t *offsets, int32_t *slots, int32_t *sources,
                                     void *workspace, size_t workspace_bytes, void *stream) {
  if (n < 0) return TT_ERR_INVALID_ARG;
  if (n > kMostPlaces || num_experts < 1 || num_experts > TT_ROUTE_MAX_EXPERTS) return TT_ERR_SHAPE;
  if (!offsets || (n > 0 && (!experts || !slots || !sources))) return TT_ERR_INVALID_ARG;
  if (!aligned(experts, 8) || !aligned(offsets, 8) || !aligned(slots, 4) || !aligned(sources, 4)) return TT_ERR_INVALID_ARG;
  if ((const int64_t *)offsets == experts || (n > 0 && (slots == sources || (void *)slots == (void *)offsets || (void *)sources == (void *)offsets ||
                                                        (const void *)slots == experts || (const void *)sources == experts)))
    return TT_ERR_INVALID_ARG;
  hipStream_t s = (hipStream_t)stream;
  if (n <= ORDER_ONE) {
    const int count = (int)n, num = num_experts;
    hipLaunchKernelGGL(k_order_one, dim3(1), dim3(ORDER_THREADS), 0, s, experts, count, num, offsets, slots, sources);
    return tt_launch_status();
  }
  const size_t need = tt_expert_order_workspace_bytes(n, num_experts);
  if (!workspace || ((uintptr_t)workspace & 255) != 0 || workspace_bytes < need) return TT_ERR_WORKSPACE;
  const int tiles = tt_ceil_div(n, ORDER_TILE), num = num_experts;
  const long long count = n, many = tiles;
  int32_t *counts = (int32_t *)workspace, *totals = counts + (long long)tiles * num_experts;
  hipLaunchKernelGGL(k_order_count, dim3((unsigned)tiles), dim3(ORDER_THREADS), 0, s, experts, count, num, counts);
  hipLaunchKernelGGL(k_order_scan, dim3((unsigned)tt_ceil_div(num, 64)), dim3(ORDER_THREADS), 0, s, counts, many, num, totals);
  hipLaunchKernelGGL(k_order_deal, dim3((unsigned)tiles), dim3(ORDER_THREADS), 0, s, experts, count, num, (const int32_t *)counts, (const int32_t *)totals,
                     offsets, slots, sources);
  return tt_launch_status();
}

extern "C" tt_status tt_route_order(const tt_route *op, const void *logits, const float *bias, int64_t *experts, float *weights, int64_t *offsets, int32_t *slots,
                                    int32_t *sources, void *workspace, size_t workspace_bytes, void *stream) {
  tt_status st = check(op);
  if (st != TT_OK) return st;
  const int64_t n = op->rows * op->choices;
  // what the second call would refuse is refused before the first one has begun
  if (!offsets || !aligned(offsets, 8) || (n > 0 && (!slots || !sources || !aligned(slots, 4) || !aligned(sources, 4)))) return TT_ERR_INVALID_ARG;
  const void *outs[5] = {experts, weights, offsets, slots, sources};
  for (int i = 0; i < 5; ++i) {
    if (outs[i] && (outs[i] == logits || outs[i] == (const void *)bias)) return TT_ERR_INVALID_ARG;
    for (int j = 0; j < i; ++j)
      if (outs[i] && outs[i] == outs[j]) return TT_ERR_INVALID_ARG;
  }
  const size_t need = tt_expert_order_workspace_bytes(n, op->experts);
  if (need && (!workspace || ((uintptr_t)workspace & 255) != 0 || workspace_bytes < need)) return TT_ERR_WORKSPACE;
  st = tt_route_forward(op, logits, bias, experts, weights, stream);
  return st == TT_OK ? tt_expert_order(experts, n, op->experts, offsets, slots, sources, workspace, workspace_bytes, stream) : st;
}
