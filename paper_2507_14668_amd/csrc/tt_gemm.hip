// Matrix products with an epilogue on the matrix cores (fp32, bf16, fp16 operands; fp32 sums).
#include "tt_gemm_device.h"

namespace {
using namespace ttg;


// ---- operands into LDS -----------------------------------------------------------------------------
// A step of the product takes BK values of K.  An operand's tile of E = 128 or 64 rows is held in LDS as 16-bit parts, one plane of
// E x BK after the other: K-contiguous operands [row][k], row-contiguous ones [k][row] (read with the transposing read, so that neither
// is transposed on its way).  16-bit operands are one plane of themselves with BK = 64; fp32 operands are split into
// bf16 parts on their way from registers to LDS (tt_split_bf16), BK = 32.
template <class T> struct Step { static constexpr int BK = sizeof(T) == 2 ? 64 : 32; };

// 16-byte pieces of a plane are spread over the banks: in an LDS row of 64 or 128 bytes (K-contiguous) by the tile's row, so that
// eight neighbouring rows at one k meet every bank once; in a row of 2 E bytes (row-contiguous) pairs of pieces by k, so that the four
// rows of a transposing read do.
template <bool KC, int BK> __device__ __forceinline__ int piece_at(int row, int k8) {  // element offset of elements [row][8 k8 ..]
  if constexpr (BK == 64) return row * 64 + ((k8 ^ (row & 7)) << 3);
  else return row * 32 + ((k8 ^ ((row >> 1) & 3)) << 3);
}
template <int E> __device__ __forceinline__ int cross_at(int k, int row) {  // [k][row]
  return k * E + ((((row >> 4) ^ (k & (E / 16 - 1))) << 4) | (row & 15));
}

// Eight elements of an operand that are neighbours in memory, as a thread carries them from memory to LDS.
template <class T> struct Unit;
template <> struct Unit<float> { f32x4 a, b; };
template <> struct Unit<bf16> { u16x8 v; };
template <> struct Unit<f16> { u16x8 v; };
// `valid` of them exist.  A row of 8 and more has its last ones by a load that ends with them (one at a time, the lanes at the end of
// a row had the whole step wait for them).
template <class T> __device__ __forceinline__ Unit<T> load_unit(const T *p, int valid, bool long_row) {
  Unit<T> u;
  if (long_row && valid > 0 && valid < 8) {
    const int by = 8 - valid;
    unsigned d[sizeof(T) * 2];
    if constexpr (sizeof(T) == 4) {
      u.a = *reinterpret_cast<const typename Vec<float>::v4 *>(p - by);
      u.b = *reinterpret_cast<const typename Vec<float>::v4 *>(p - by + 4);
    } else {
      u.v = *reinterpret_cast<const typename Vec<T>::v16b *>(p - by);
    }
    if constexpr (sizeof(T) == 4) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        d[i] = __float_as_uint(u.a[i]);
        d[4 + i] = __float_as_uint(u.b[i]);
      }
#pragma unroll
      for (int s = 1; s < 8; s *= 2)
#pragma unroll
        for (int i = 0; i < 8; ++i) d[i] = (by & s) ? (i + s < 8 ? d[i + s] : 0u) : d[i];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        u.a[i] = __uint_as_float(d[i]);
        u.b[i] = __uint_as_float(d[4 + i]);
      }
    } else {
      typedef unsigned u4 __attribute__((ext_vector_type(4)));
      const u4 w = __builtin_bit_cast(u4, u.v);
#pragma unroll
      for (int i = 0; i < 4; ++i) d[i] = w[i];
      if (by & 1) {
#pragma unroll
        for (int i = 0; i < 4; ++i) d[i] = (d[i] >> 16) | (i < 3 ? d[i + 1] << 16 : 0u);
      }
#pragma unroll
      for (int s = 1; s < 4; s *= 2)
#pragma unroll
        for (int i = 0; i < 4; ++i) d[i] = (by & (2 * s)) ? (i + s < 4 ? d[i + s] : 0u) : d[i];
      u.v = __builtin_bit_cast(u16x8, u4{d[0], d[1], d[2], d[3]});
    }
    return u;
  }
  if constexpr (sizeof(T) == 4) {
    u.a = u.b = f32x4{0.f, 0.f, 0.f, 0.f};
    if (valid >= 8) {
      u.a = *reinterpret_cast<const typename Vec<float>::v4 *>(p);
      u.b = *reinterpret_cast<const typename Vec<float>::v4 *>(p + 4);
    } else if (valid > 0) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if (i < valid) u.a[i] = p[i];
        if (i + 4 < valid) u.b[i] = p[i + 4];
      }
    }
  } else {
    u.v = u16x8{0, 0, 0, 0, 0, 0, 0, 0};
    if (valid >= 8) u.v = *reinterpret_cast<const typename Vec<T>::v16b *>(p);
    else if (valid > 0) {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (i < valid) u.v[i] = __builtin_bit_cast(unsigned short, p[i]);
    }
  }
  return u;
}

// The units of one operand that a thread carries, step after step.
template <class T, bool KC, int E> struct Carrier {
  static constexpr int BK = Step<T>::BK, N = E * BK / 8 / TT_BLOCK;
  const T *p[N];
  int valid[N];
  bool long_row, whole;  // whole: all rows of the tile are there
  long long step;
  __device__ __forceinline__ void start(const T *base, long long ld, int row0, int rows, int k_first, int k_end) {
    whole = rows - row0 >= E;
    long_row = (KC ? k_end - k_first : rows - row0) >= 8;
    step = KC ? BK : (long long)BK * ld;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int u = threadIdx.x + i * TT_BLOCK;
      if constexpr (KC) {
        const int r = row0 + u / (BK / 8);
        valid[i] = r < rows ? 8 : 0;
        p[i] = base + (long long)(r < rows ? r : 0) * ld + k_first + (u % (BK / 8)) * 8;
      } else {
        const int c = row0 + (u % (E / 8)) * 8, left = rows - c;
        valid[i] = left >= 8 ? 8 : (left > 0 ? left : 0);
        p[i] = base + (long long)(k_first + u / (E / 8)) * ld + (left > 0 ? c : 0);
      }
    }
  }
  // the units of the step at k0 (K: the end), and on to the next step
  __device__ __forceinline__ void load(Unit<T> u[N], int k0, int K) {
    if (whole && K - k0 >= BK) {  // the same for all lanes, and most steps
#pragma unroll
      for (int i = 0; i < N; ++i) {
        if constexpr (sizeof(T) == 4) {
          u[i].a = *reinterpret_cast<const typename Vec<float>::v4 *>(p[i]);
          u[i].b = *reinterpret_cast<const typename Vec<float>::v4 *>(p[i] + 4);
        } else {
          u[i].v = *reinterpret_cast<const typename Vec<T>::v16b *>(p[i]);
        }
        p[i] += step;
      }
      return;
    }
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int n = threadIdx.x + i * TT_BLOCK;
      const int left = K - k0 - (KC ? (n % (BK / 8)) * 8 : n / (E / 8));
      u[i] = load_unit<T>(p[i], KC ? (left < valid[i] ? left : valid[i]) : (left > 0 ? valid[i] : 0), long_row);
      p[i] += step;
    }
  }
  template <int P> __device__ __forceinline__ void store(const Unit<T> u[N], unsigned short *lds) const {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int n = threadIdx.x + i * TT_BLOCK;
      const int o = KC ? piece_at<KC, BK>(n / (BK / 8), n % (BK / 8)) : cross_at<E>(n / (E / 8), (n % (E / 8)) * 8);
      if constexpr (sizeof(T) == 2) {
        *reinterpret_cast<u16x8 *>(lds + o) = u[i].v;
      } else {
        typedef unsigned u4 __attribute__((ext_vector_type(4)));
        unsigned h[4], m[4], l[4];
        tt_split_bf16(u[i].a[0], u[i].a[1], h[0], m[0], l[0]);
        tt_split_bf16(u[i].a[2], u[i].a[3], h[1], m[1], l[1]);
        tt_split_bf16(u[i].b[0], u[i].b[1], h[2], m[2], l[2]);
        tt_split_bf16(u[i].b[2], u[i].b[3], h[3], m[3], l[3]);
        *reinterpret_cast<u4 *>(lds + o) = u4{h[0], h[1], h[2], h[3]};
        *reinterpret_cast<u4 *>(lds + E * BK + o) = u4{m[0], m[1], m[2], m[3]};
        if constexpr (P == 3) *reinterpret_cast<u4 *>(lds + 2 * E * BK + o) = u4{l[0], l[1], l[2], l[3]};
      }
    }
  }
  // unsplit, for the fp32 instructions: [row][32 + 4] or [k][128 + 4] floats
  static constexpr int LD32 = KC ? 36 : E + 4, SIZE32 = (KC ? E : 32) * LD32;
  __device__ __forceinline__ void store32(const Unit<T> u[N], float *lds) const {
    if constexpr (sizeof(T) == 4) {
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const int n = threadIdx.x + i * TT_BLOCK;
        float *d = lds + (KC ? (n / (BK / 8)) * LD32 + (n % (BK / 8)) * 8 : (n / (E / 8)) * LD32 + (n % (E / 8)) * 8);
        *reinterpret_cast<f32x4 *>(d) = u[i].a;
        *reinterpret_cast<f32x4 *>(d + 4) = u[i].b;
      }
    }
  }
};

// The lane's eight elements of rows r0 .. r0 + 15 at k = 32 s + 8 (lane / 16) + i
template <bool KC, int BK, int E> __device__ __forceinline__ u16x8 frag(const unsigned short *lds, int r0, int s) {
  const int lane = threadIdx.x & 63, q = lane >> 4, j = lane & 15;
  if constexpr (KC) return *reinterpret_cast<const u16x8 *>(lds + piece_at<KC, BK>(r0 + j, 4 * s + q));
  const int k = 32 * s + 8 * q + (j >> 2), c = r0 + 4 * (j & 3);
  const u16x4 x = lds_read_tr(lds + cross_at<E>(k, c)), y = lds_read_tr(lds + cross_at<E>(k + 4, c));
  return __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7);
}
template <bool KC, int LD32> __device__ __forceinline__ f32x4 frag32(const float *lds, int r0, int h) {  // k = 16 h + 4 (lane / 16) + i
  const int lane = threadIdx.x & 63, q = lane >> 4, j = lane & 15;
  if constexpr (KC) return *reinterpret_cast<const f32x4 *>(lds + (r0 + j) * LD32 + 16 * h + 4 * q);
  f32x4 v;
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = lds[(16 * h + 4 * q + i) * LD32 + r0 + j];
  return v;
}

// ---- the tile kernel -------------------------------------------------------------------------------
// E x E of out per workgroup (E = 128, or 64 where there are few tiles), four wavefronts of a quarter each, any size, row step and alignment down to the element's; elements
// outside are zeros.  The product is formed as out^T (B's rows are the instruction's M side), so that a lane's four results are
// neighbours in a row of out.
// P planes: 1 (16-bit operands), 2 or 3 (fp32 operands in bf16 parts).  Three parts hold all 24 bits; of the nine products
// the six with hi * hi, hi * mid, hi * lo and mid * mid count, the rest is below 2^-24 of the product.  What parts cannot do:
// infinities, NaN and numbers that round to a bf16 infinity give NaN sums, products below 2^-92 lose parts to underflow, and so do
// numbers below 2^-100 by themselves.  A tile with a sum that is not finite, or with one so small that such a loss would
// count beside operands that have it, is done again with the fp32 instruction.  (P = 2 is for operands that are scaled to at most one, with no such products that count.)
// Measured: fp32 4096 x 4096 x 1024 188 us (183 TFLOP/s, 1100 of bf16 products; the fp32 instruction's rate is 154), 106496 x 128 x 128 39 us (22 by
// its bytes), 2 % of both for the largest number; two parts 2048 x 4096 x 2048 106 us (975 of bf16 products).  Without the matrix instructions the first took 169 of 198,
// without the split of P = 2 the last 93 of 106: splitting, LDS and barriers bound it.  Loads two or four steps ahead in registers, and two buffers for P = 2, are no faster.
template <class T, class O, int P, bool AKC, bool BKC, int E>
__global__ void __launch_bounds__(TT_BLOCK, 2) k_gemm(TTGemm g, int m_tiles, int n_tiles, int split, int chunk, float *partial) {
  typedef Carrier<T, AKC, E> CA;
  typedef Carrier<T, BKC, E> CB;
    constexpr int BK = Step<T>::BK, PLANE = E * BK, F = E / 32, BUF = P == 1 ? 2 : 1;  // fp32's planes fill the LDS of two workgroups with one buffer (two planes: two buffers are no faster)
  constexpr int HALVES = 2 * BUF * P * PLANE, REDO = P == 3 ? 2 * (CA::SIZE32 + CB::SIZE32) : 0,
                FINISH = 8 * finish_floats<F, 2>();
  __shared__ __align__(16) unsigned short lds[HALVES > REDO ? (HALVES > FINISH ? HALVES : FINISH) : (REDO > FINISH ? REDO : FINISH)];
  __shared__ int flags[4];
  __shared__ float ends[4][2];
  constexpr bool SETTLES = P == 3 && AKC && BKC;
  __shared__ float norms_a[SETTLES ? E : 1], norms_b[SETTLES ? E : 1];  // sums of squares of A's and B's rows
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int members = (int)gridDim.y / split, cut = (int)blockIdx.y / members;  // which piece of K
  unsigned mt, nt;
  tile_order(blockIdx.x, (unsigned)m_tiles, (unsigned)n_tiles, g.symmetric, mt, nt);
  Place w;
  w.n0 = (int)nt * E;
  w.k_lo = 0;
  w.k_hi = g.K;
  float *piece = nullptr;
  if (g.mode == TT_GEMM_RAGGED_M) {
    const int there = find_tile<E>(g.offsets, g.batch, g.M, (int)mt, w.z, w.lo, w.hi);
    if (w.z < 0) {
      if (g.zero_rest) clear_rest<O>(g, w.lo, w.hi, (int)mt - there, m_tiles - there, w.n0, E);
      return;
    }
  } else {
    w.z = (int)blockIdx.y - cut * members;
    w.lo = (int)mt * E;
    w.hi = g.M < w.lo + E ? g.M : w.lo + E;
    if (g.mode == TT_GEMM_RAGGED_K) {
      int pieces = 1, number = 0;
      find_slot(g.offsets, g.batch, g.K, chunk, BK, (int)blockIdx.y, w.z, w.k_lo, w.k_hi, pieces, number);
      if (w.z < 0) return;
      if (pieces > 1) piece = partial + number * ttk_gemm_piece_floats(g);
    }
  }
  if (split > 1) {  // whole steps to each piece
    piece = partial + ((long long)cut * g.batch + w.z) * ttk_gemm_piece_floats(g);
    const int steps = (w.k_hi - w.k_lo + BK - 1) / BK, per = (steps + split - 1) / split;
    const long long a = (long long)w.k_lo + (long long)cut * per * BK, b = a + (long long)per * BK;
    if (a < w.k_hi) w.k_lo = (int)a;
    else w.k_lo = w.k_hi;
    if (b < w.k_hi) w.k_hi = (int)b;
  }
  const bool by_member = g.mode == TT_GEMM_BATCH;
  const T *a = (const T *)g.a + (by_member ? w.z * g.a_step : 0), *b = (const T *)g.b + (g.mode != TT_GEMM_RAGGED_K ? w.z * g.b_step : 0);
  const int K = w.k_hi;
  CA ca;
  CB cb;
  ca.start(a, g.lda, w.lo, w.hi, w.k_lo, K);
  cb.start(b, g.ldb, w.n0, g.N, w.k_lo, K);
  Unit<T> ua[CA::N], ub[CB::N];
  const int wm = (wave >> 1) * (E / 2), wn = (wave & 1) * (E / 2);
  f32x4 acc[F][F] = {}, rs[F] = {};  // [m][n]; sums of A's rows
  const bool sums = g.rowsum && w.n0 == 0;
  const bool settles = SETTLES && ttk_gemm_settles(g);
  float squares_a[CA::N] = {}, squares_b[CB::N] = {};  // of the rows that the thread carries (its units are of one row each, all along K)
  auto measure = [&]() {
    if constexpr (SETTLES) {
      if (settles) {
#pragma unroll
        for (int i = 0; i < CA::N; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            squares_a[i] = fmaf(ua[i].a[e], ua[i].a[e], fmaf(ua[i].b[e], ua[i].b[e], squares_a[i]));
            squares_b[i] = fmaf(ub[i].a[e], ub[i].a[e], fmaf(ub[i].b[e], ub[i].b[e], squares_b[i]));
          }
      }
    }
  };
  float large = 0.f;  // the largest number of both operands
  auto note = [&](const Unit<T> *u, int n) {
    if constexpr (P == 3) {
#pragma unroll
      for (int i = 0; i < n; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) large = tt_max3_abs(large, u[i].a[e], u[i].b[e]);
    }
  };
  // the smallest number that is not zero, as twice its bits less one
  auto note_small = [&](const Unit<T> *u, int n, unsigned &small) {
    if constexpr (P == 3) {
#pragma unroll
      for (int i = 0; i < n; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const unsigned x = 2 * __float_as_uint(u[i].a[e]) - 1, y = 2 * __float_as_uint(u[i].b[e]) - 1;
          small = x < small ? x : small;
          small = y < small ? y : small;
        }
    }
  };
  auto plane_a = [&](int buf, int p) { return lds + (buf * 2 * P + p) * PLANE; };
  auto plane_b = [&](int buf, int p) { return lds + (buf * 2 * P + P + p) * PLANE; };
  auto multiply = [&](int buf) {
#pragma unroll
    for (int s = 0; s < BK / 32; ++s) {
      u16x8 fa[F][P];
#pragma unroll
      for (int x = 0; x < F; ++x)
#pragma unroll
        for (int p = 0; p < P; ++p) fa[x][p] = frag<AKC, BK, E>(plane_a(buf, p), wm + 16 * x, s);
#pragma unroll
      for (int y = 0; y < F; ++y) {
        u16x8 fb[P];
#pragma unroll
        for (int p = 0; p < P; ++p) fb[p] = frag<BKC, BK, E>(plane_b(buf, p), wn + 16 * y, s);
        if constexpr (P == 1) {
#pragma unroll
          for (int x = 0; x < F; ++x) acc[x][y] = mma(T(), fb[0], fa[x][0], acc[x][y]);
        } else {  // the smallest terms first
#pragma unroll
          for (int d = P - 1; d >= 0; --d)
#pragma unroll
            for (int p = 0; p <= d; ++p)
#pragma unroll
              for (int x = 0; x < F; ++x) acc[x][y] = mma(bf16(), fb[d - p], fa[x][p], acc[x][y]);
        }
      }
      if (sums) {
        unsigned short one = 0x3f80;  // of bf16
        if constexpr (std::is_same<T, f16>::value) one = 0x3c00;
        const u16x8 ones = {one, one, one, one, one, one, one, one};
#pragma unroll
        for (int x = 0; x < F; ++x)
#pragma unroll
          for (int p = P - 1; p >= 0; --p) {
            if constexpr (P == 1) rs[x] = mma(T(), ones, fa[x][0], rs[x]);
            else rs[x] = mma(bf16(), ones, fa[x][p], rs[x]);
          }
      }
    }
  };
  if (w.k_lo < K) {
    ca.load(ua, w.k_lo, K);
    cb.load(ub, w.k_lo, K);
    if constexpr (BUF == 2) {
      ca.template store<P>(ua, plane_a(0, 0));
      cb.template store<P>(ub, plane_b(0, 0));
    }
    int buf = 0;
    for (int k0 = w.k_lo; k0 < K; k0 += BK) {
      const bool more = k0 + BK < K;
      __syncthreads();  // two buffers: this step's tiles are whole, and nobody reads the other buffer any more
      if constexpr (BUF == 1) {
        measure();
        note(ua, CA::N);
        note(ub, CB::N);
        ca.template store<P>(ua, plane_a(0, 0));
        cb.template store<P>(ub, plane_b(0, 0));
        __syncthreads();
      }
      if (more) {
        ca.load(ua, k0 + BK, K);
        cb.load(ub, k0 + BK, K);
      }
      multiply(buf);
      if constexpr (BUF == 2) {
        buf ^= 1;
        if (more) {
          ca.template store<P>(ua, plane_a(buf, 0));
          cb.template store<P>(ub, plane_b(buf, 0));
        }
      }
    }
  }
  if constexpr (P == 3) {
    // A number below 2^-100 loses less than 2^-125 of itself to parts that are no normal numbers: nothing to a sum of more than 2^-98 K times
    // the largest number.  That is below 2^-80 unless there are large numbers; smaller sums are of rows of zeros, mostly.
    const float terms = (float)(K - w.k_lo);
    bool odd = false;
    float least = INFINITY;  // of the sums
#pragma unroll
    for (int x = 0; x < F; ++x) {
      const bool in = w.lo + wm + 16 * x + (lane & 15) < w.hi;
#pragma unroll
      for (int y = 0; y < F; ++y)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float v = fabsf(acc[x][y][i]);
          odd |= !(v < INFINITY);
          if (in && w.n0 + wn + 16 * y + 4 * (lane >> 4) + i < g.N && v < least) least = v;
        }
      if (sums) {  // (sums of A's rows are of products with one)
        odd |= !(fabsf(rs[x][0]) < INFINITY);
        if (in && fabsf(rs[x][0]) < least) least = fabsf(rs[x][0]);
        large = tt_max3_abs(large, large, 1.f);
      }
    }
    // what any lane of the workgroup has seen
    auto any = [&](int mine) {
      const int all = (__ballot(mine & 1) ? 1 : 0) | (__ballot(mine & 2) ? 2 : 0) | (__ballot(mine & 4) ? 4 : 0);
      __syncthreads();
      if (lane == 0) flags[wave] = all;
      __syncthreads();
      return flags[0] | flags[1] | flags[2] | flags[3];
    };
    const int found = any((odd ? 1 : 0) | (least < 0x1p-80f ? 2 : 0) | (large * terms > 0x1p18f ? 4 : 0));
    bool redo = found & 1, look = found & 2;
    if (found == 4) {
#pragma unroll
      for (int o = 1; o < 64; o <<= 1) {
        const float x = __shfl(least, lane ^ o, 64), y = __shfl(large, lane ^ o, 64);
        least = x < least ? x : least;
        large = y > large ? y : large;
      }
      if (lane == 0) {
        ends[wave][0] = least;
        ends[wave][1] = large;
      }
      __syncthreads();
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        least = ends[i][0] < least ? ends[i][0] : least;
        large = ends[i][1] > large ? ends[i][1] : large;
      }
      look = least < 0x1p-98f * terms * large;
    }
    if (look && !redo) {  // whether small operands are the reason takes another look at them
      unsigned small_a = ~0u, small_b = ~0u;
      ca.start(a, g.lda, w.lo, w.hi, w.k_lo, K);
      cb.start(b, g.ldb, w.n0, g.N, w.k_lo, K);
      for (int k0 = w.k_lo; k0 < K; k0 += BK) {
        ca.load(ua, k0, K);
        cb.load(ub, k0, K);
        note_small(ua, CA::N, small_a);
        note_small(ub, CB::N, small_b);
      }
      unsigned ea = small_a == ~0u ? 255 : small_a >> 24, eb = small_b == ~0u ? 255 : small_b >> 24;  // exponents
#pragma unroll
      for (int o = 1; o < 64; o <<= 1) {
        const unsigned x = (unsigned)__shfl((int)ea, lane ^ o, 64), y = (unsigned)__shfl((int)eb, lane ^ o, 64);
        ea = x < ea ? x : ea;
        eb = y < eb ? y : eb;
      }
      __syncthreads();
      if (lane == 0) flags[wave] = (int)(ea << 8 | eb);
      __syncthreads();
      ea = eb = 255;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const unsigned x = (unsigned)flags[i] >> 8, y = (unsigned)flags[i] & 255;
        ea = x < ea ? x : ea;
        eb = y < eb ? y : eb;
      }
      // the smallest product is below 2^-92 if the exponents' sum (each 127 too many) is; parts themselves are whole down to 2^-100
      redo = ea < 27 || eb < 27 || ((found & 2) && (int)(ea + eb) - 254 < -92);
    }
    if (redo) {
      float *l32a = reinterpret_cast<float *>(lds), *l32b = l32a + CA::SIZE32;
#pragma unroll
      for (int x = 0; x < F; ++x) {
        rs[x] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int y = 0; y < F; ++y) acc[x][y] = f32x4{0.f, 0.f, 0.f, 0.f};
      }
      ca.start(a, g.lda, w.lo, w.hi, w.k_lo, K);
      cb.start(b, g.ldb, w.n0, g.N, w.k_lo, K);
      for (int k0 = w.k_lo; k0 < K; k0 += BK) {
        ca.load(ua, k0, K);
        cb.load(ub, k0, K);
        __syncthreads();
        ca.store32(ua, l32a);
        cb.store32(ub, l32b);
        __syncthreads();
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          f32x4 fa[F];
#pragma unroll
          for (int x = 0; x < F; ++x) fa[x] = frag32<AKC, CA::LD32>(l32a, wm + 16 * x, h);
#pragma unroll
          for (int y = 0; y < F; ++y) {
            const f32x4 fb = frag32<BKC, CB::LD32>(l32b, wn + 16 * y, h);
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
              for (int x = 0; x < F; ++x) acc[x][y] = __builtin_amdgcn_mfma_f32_16x16x4f32(fb[i], fa[x][i], acc[x][y], 0, 0, 0);
          }
          if (sums)
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
              for (int x = 0; x < F; ++x) rs[x] = __builtin_amdgcn_mfma_f32_16x16x4f32(1.f, fa[x][i], rs[x], 0, 0, 0);
        }
      }
    }
  }
  if constexpr (SETTLES) {
    if (settles) {
      constexpr int PER = BK / 8;  // lanes of a row
#pragma unroll
      for (int i = 0; i < CA::N; ++i) {
#pragma unroll
        for (int o = 1; o < PER; o *= 2) {
          squares_a[i] += __shfl(squares_a[i], lane ^ o, 64);
          squares_b[i] += __shfl(squares_b[i], lane ^ o, 64);
        }
        const int r = ((int)threadIdx.x + i * TT_BLOCK) / PER;
        if (lane % PER == 0) {
          norms_a[r] = squares_a[i];
          norms_b[r] = squares_b[i];
          if (piece) {
            float *rows = piece + (long long)g.M * (g.N + 1LL);
            if (w.n0 == 0 && w.lo + r < w.hi) rows[w.lo + r] = squares_a[i];
            if (w.lo == 0 && w.n0 + r < g.N) rows[g.M + w.n0 + r] = squares_b[i];
          }
        }
      }
    }
  }
  const int q = lane >> 4, j = lane & 15;
  if (sums && wn == 0 && q == 0) {
#pragma unroll
    for (int x = 0; x < F; ++x) {
      const int m = w.lo + wm + 16 * x + j;
      if (m >= w.hi) continue;
      if (piece) piece[(long long)g.M * g.N + m] = rs[x][0];
      else ((O *)g.rowsum)[w.z * g.rs_step + m] = from_f32<O>(rs[x][0]);
    }
  }
  __syncthreads();  // nobody reads the operands any more
  float *room = reinterpret_cast<float *>(lds) + wave * finish_floats<F, 2>();
  const bool mirror = g.symmetric && mt != nt;
  if (piece) finish_tile<T, float, F, F, 2, false>(as_piece(g, piece), 0, w.lo + wm, w.hi, w.n0 + wn, acc, room, mirror);
  else finish_tile<T, O, F, F, 2, false>(g, w.z, w.lo + wm, w.hi, w.n0 + wn, acc, room, mirror, settles ? norms_a + wm : nullptr,
                                                  settles ? norms_b + wn : nullptr);
}

// The pieces of a cut product, added in order; four columns of a row per thread.
template <class T, class O> __device__ __forceinline__ void join_pieces(const TTGemm &g, int z, int pieces, const float *p, long long step) {
  const int per = (g.N + 3) / 4;
  const long long total = (long long)g.M * per;
  const int lane = threadIdx.x & 63;
  for (long long e0 = (long long)blockIdx.x * TT_BLOCK + (threadIdx.x - lane); e0 < total + g.M; e0 += (long long)gridDim.x * TT_BLOCK) {
    const long long e = e0 + lane;  // (whole wavefronts, for settle_signs)
    if (e >= total && e < total + g.M && g.rowsum) {
      const long long m = e - total;
      float s = 0.f;
      for (int i = 0; i < pieces; ++i) s += p[i * step + (long long)g.M * g.N + m];
      ((O *)g.rowsum)[z * g.rs_step + m] = from_f32<O>(s);
    }
    if (e0 >= total) continue;
    const int m = e < total ? (int)(e / per) : 0, n = e < total ? (int)(e - (long long)m * per) * 4 : 0;
    const int valid = e >= total ? 0 : g.N - n < 4 ? g.N - n : 4;
    f32x4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
    for (int i = 0; i < pieces; ++i) {
      float t[4];
      load4(p + i * step + (long long)m * g.N + n, valid, t);
#pragma unroll
      for (int c = 0; c < 4; ++c) s[c] += t[c];
    }
    float v[4] = {s[0], s[1], s[2], s[3]};
    if constexpr (std::is_same<T, float>::value && std::is_same<O, float>::value) {
      if (ttk_gemm_settles(g)) {
        const float none[4] = {0.f, 0.f, 0.f, 0.f};  // (bias is in v)
        float a = 0.f, b[4] = {0.f, 0.f, 0.f, 0.f};
        for (int i = 0; i < pieces; ++i) {
          const float *rows = p + i * step + (long long)g.M * (g.N + 1LL);
          float t[4];
          a += rows[m];
          load4(rows + g.M + n, valid, t);
#pragma unroll
          for (int c = 0; c < 4; ++c) b[c] += t[c];
        }
        float bias[4] = {0.f, 0.f, 0.f, 0.f};
        if (g.bias) load4((const float *)g.bias + z * g.bias_step + n, valid, bias);
        settle_signs<4>(g, z, m, n, valid, v, bias, a, b);
        if (valid > 0) finish<T, O, 4>(g, z, m, n, valid, v, none);
        continue;
      }
    }
    if (valid > 0) finish<T, O, 4>(g, z, m, n, valid, v);
  }
}
template <class T, class O> __global__ void __launch_bounds__(TT_BLOCK) k_join(TTGemm g, int split, const float *__restrict__ partial) {
  const int z = (int)blockIdx.y;
  join_pieces<T, O>(g, z, split, partial + z * ttk_gemm_piece_floats(g), g.batch * ttk_gemm_piece_floats(g));
}
template <class T> __global__ void __launch_bounds__(TT_BLOCK) k_join_groups(TTGemm g, int chunk, int bk, const float *__restrict__ partial) {
  int z = (int)blockIdx.y, lo = 0, hi = 0, pieces = 1, first = 0;
  find_slot(g.offsets, g.batch, g.K, chunk, bk, -1, z, lo, hi, pieces, first);
  if (z >= 0) join_pieces<T, T>(g, z, pieces, partial + first * ttk_gemm_piece_floats(g), ttk_gemm_piece_floats(g));
}

// ---- host ------------------------------------------------------------------------------------------
// Tiles of 128 from which they are taken.  These / tiles of 64, us: fp32 4096 x 2048 x 512 (512 tiles) 57 / 71 and its gradients 69 / 87 and
// 72 / 93, 2048 x 2048 x 512 (256) 45 / 38, 42 / 49 and 43 / 51, 2048 x 1024 x 1024 (128) 46 / 44; fp16 2048 x 2048 x 520 18 / 15, 26 / 28 and
// 26 / 30, 2048 x 1024 x 1024 27 / 15.
#ifndef TT_GEMM_LARGE_TILES
#define TT_GEMM_LARGE_TILES 256
#endif
struct Shape {
  int e, split, chunk;
  long long m_tiles, n_tiles, members;
};
Shape shape_of(const TTGemm &g) {
  Shape h;
  const int bk = g.dtype == TT_F32 ? 32 : 64;
  // (as for N = like_N: sums of A's rows beside one column have the bits of those beside all)
  auto tiles = [&](int e) {
    // every group ends in at most one part tile; one more for the rows outside the groups
    h.m_tiles = g.mode == TT_GEMM_RAGGED_M ? (long long)tt_ceil_div(g.M, e) + g.batch + 1 : tt_ceil_div(g.M, e);
    h.n_tiles = tt_ceil_div(g.N, e);
    h.members = g.mode == TT_GEMM_RAGGED_M ? 1 : g.batch;
    h.e = e;
    const long long n = (long long)tt_ceil_div(g.M, e) * tt_ceil_div(g.like_N ? g.like_N : g.N, e) * h.members;
    return n;
  };
  long long n = tiles(128);
  if (n < TT_GEMM_LARGE_TILES) n = tiles(64);
  if (g.symmetric) n = (n + h.members * h.m_tiles) / 2;
  // two workgroups and more run on a compute unit: long sums in pieces up to 512 workgroups in all, of eight steps at least
  // (of four where even so most compute units have none)
  h.split = 1;
  h.chunk = 0;
  if (g.mode == TT_GEMM_BATCH) {
    const long long steps = tt_ceil_div(g.K, bk);
    long long split = 512 / n;
    const long long least = n * (steps / 4) <= 128 ? 4 : 8;
    if (split > steps / least) split = steps / least;
    if (split > 64) split = 64;
    if (split > 1) h.split = (int)split;
  } else if (g.mode == TT_GEMM_RAGGED_K) {
    h.chunk = ttk_gemm_chunk(g, h.e, bk, h.e == 64 ? 8 : 32);
    if (g.like_N && g.N != g.like_N) {  // (cut as the whole product of aligned operands would be)
      TTGemm whole = g;
      whole.N = g.like_N;
      whole.b = g.a;
      whole.ldb = 8;
      if (ttk_gemm_direct_serves(whole)) h.chunk = ttk_gemm_direct_chunk(whole);
    }
    h.members = tt_ceil_div(g.K, h.chunk) + g.batch;  // slots
  }
  return h;
}

template <class T, class O, int P, int E> void launch_e(const TTGemm &g, const Shape &h, float *part, hipStream_t s) {
  const long long per_member = g.symmetric ? h.n_tiles * (h.n_tiles + 1) / 2 : h.m_tiles * h.n_tiles;
  const dim3 grid((unsigned)per_member, (unsigned)(h.members * h.split));
  const int mti = (int)h.m_tiles, nti = (int)h.n_tiles, split = h.split, chunk = h.chunk;
  if (g.a_kc && g.b_kc) hipLaunchKernelGGL((k_gemm<T, O, P, true, true, E>), grid, dim3(TT_BLOCK), 0, s, g, mti, nti, split, chunk, part);
  else if (g.a_kc) hipLaunchKernelGGL((k_gemm<T, O, P, true, false, E>), grid, dim3(TT_BLOCK), 0, s, g, mti, nti, split, chunk, part);
  else hipLaunchKernelGGL((k_gemm<T, O, P, false, false, E>), grid, dim3(TT_BLOCK), 0, s, g, mti, nti, split, chunk, part);
}
unsigned join_blocks(const TTGemm &g) {
  long long blocks = ((long long)g.M * ((g.N + 3) / 4) + g.M + TT_BLOCK - 1) / TT_BLOCK;
  return (unsigned)(blocks > 4096 ? 4096 : blocks);
}
template <class T, class O, int P> tt_status launch(const TTGemm &g, void *partial, hipStream_t s) {
  const Shape h = shape_of(g);
  if (h.m_tiles * h.n_tiles > TT_MAX_WORKGROUPS || h.m_tiles * h.n_tiles * h.members * h.split > TT_MAX_WORKGROUPS || h.members * h.split > 65535)
    return TT_ERR_SHAPE;
  if ((h.split > 1 || h.chunk) && !partial) return TT_ERR_WORKSPACE;
  float *part = (float *)partial;
  if (h.e == 128) launch_e<T, O, P, 128>(g, h, part, s);
  else launch_e<T, O, P, 64>(g, h, part, s);
  if (h.split > 1) {
    const int split = h.split;
    hipLaunchKernelGGL((k_join<T, O>), dim3(join_blocks(g), (unsigned)h.members), dim3(TT_BLOCK), 0, s, g, split, (const float *)part);
  }
  const tt_status st = tt_launch_status();
  return st == TT_OK && h.chunk ? ttk_gemm_join_groups(g, h.chunk, g.dtype == TT_F32 ? 32 : 64, part, s) : st;
}

}  // namespace

// About as many workgroups as run at once, and pieces long enough that writing and adding their sums does not count: a tile of 256
// costs as much as 24 steps of it.
int ttk_gemm_chunk(const TTGemm &g, int e, int bk, int least) {
  const long long tiles = (long long)tt_ceil_div(g.M, e) * tt_ceil_div(g.like_N ? g.like_N : g.N, e), steps = tt_ceil_div(g.K, bk);
  long long per = (steps * tiles + 511) / 512;
  if (per < least) per = least;
  if (per < steps / 16384) per = steps / 16384;  // slots are a grid's second side
  const long long chunk = per * bk;
  return (int)(chunk > 1073741824LL ? 1073741824LL : chunk);
}
size_t ttk_gemm_chunk_bytes(const TTGemm &g, int chunk) {
  // groups of several pieces have fewer than 2 rows / chunk each, the rest none
  const long long slots = 2 * ((long long)g.K / chunk);
  return ((size_t)slots * ttk_gemm_piece_floats(g) * 4 + 255) & ~(size_t)255;
}
tt_status ttk_gemm_join_groups(const TTGemm &g, int chunk, int bk, const float *partial, hipStream_t s) {
  const int most = g.K / chunk < g.batch ? g.K / chunk : g.batch;  // groups that can have two pieces
  if (most < 1) return TT_OK;
  const dim3 grid(join_blocks(g), (unsigned)most);
  if (g.dtype == TT_F32) hipLaunchKernelGGL(k_join_groups<float>, grid, dim3(TT_BLOCK), 0, s, g, chunk, bk, partial);
  else if (g.dtype == TT_BF16) hipLaunchKernelGGL(k_join_groups<ttg::bf16>, grid, dim3(TT_BLOCK), 0, s, g, chunk, bk, partial);
  else hipLaunchKernelGGL(k_join_groups<ttg::f16>, grid, dim3(TT_BLOCK), 0, s, g, chunk, bk, partial);
  return tt_launch_status();
}

size_t ttk_gemm_partial_bytes(const TTGemm &g) {
  if (g.M < 1 || g.N < 1 || g.batch < 1 || ttk_gemm_rows_serves(g)) return 0;
  const Shape h = shape_of(g);
  if (h.chunk) {
    const size_t a = ttk_gemm_chunk_bytes(g, h.chunk), b = ttk_gemm_direct_bytes(g);
    return a > b ? a : b;
  }
  return h.split < 2 ? 0 : (((size_t)h.split * g.batch * ttk_gemm_piece_floats(g) * 4) + 255) & ~(size_t)255;
}

tt_status ttk_gemm(const TTGemm &g, void *partial, hipStream_t s) {
  if (g.M < 1 || g.N < 1 || g.batch < 1) return TT_OK;
  if (!g.a_kc && g.b_kc) return TT_ERR_INVALID_ARG;  // no caller needs it
  if (ttk_gemm_rows_serves(g)) return ttk_gemm_rows(g, s);
  if (ttk_gemm_direct_serves(g)) return ttk_gemm_direct(g, partial, s);
  if (g.dtype == TT_BF16 && g.out_dtype == TT_BF16) return launch<ttg::bf16, ttg::bf16, 1>(g, partial, s);
  if (g.dtype == TT_F16 && g.out_dtype == TT_F16) return launch<ttg::f16, ttg::f16, 1>(g, partial, s);
  if (g.dtype != TT_F32) return TT_ERR_INVALID_ARG;
  if (g.parts == 3 && g.out_dtype == TT_F32) return launch<float, float, 3>(g, partial, s);
  if (g.parts == 2 && g.out_dtype == TT_F32) return launch<float, float, 2>(g, partial, s);
  if (g.parts == 2 && g.out_dtype == TT_BF16) return launch<float, ttg::bf16, 2>(g, partial, s);
  if (g.parts == 2 && g.out_dtype == TT_F16) return launch<float, ttg::f16, 2>(g, partial, s);
  return TT_ERR_INVALID_ARG;
}
