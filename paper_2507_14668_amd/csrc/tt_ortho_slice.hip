// Newton-Schulz steps on small matrices that stay on chip from the first to the last step: read once, written once.
#include <string.h>

#include "tt_gemm_device.h"
#include "tt_ortho_slice.h"

namespace {
using namespace ttg;

// The value that is to be orthogonalised at (z, s, l); in the core update the momentum is brought up to date on the way.
template <class T> __device__ __forceinline__ float take(const TTSlices &p, long long z, int s, int l) {
  const long long e = z * p.in_b + s * p.in_s + l * p.in_l;
  const float g = to_f32(((const T *)p.in)[e]);
  if (!p.mom) return g;
  const float m = p.mu * p.mom[e] + g;
  p.mom[e] = m;
  return p.nesterov ? g + p.mu * m : m;
}
template <class T> __device__ __forceinline__ void give(const TTSlices &p, long long z, int s, int l, float v) {
  T *o = (T *)p.out + z * p.out_b + s * p.out_s + l * p.out_l;
  if (!p.mom) *o = from_f32<T>(v);
  else *o = from_f32<T>(to_f32(*o) - p.rate * v);
}
// C neighbours along l (ALONG_L) or along s from (s, l) on, in one access where they all exist and lie next to each other.
template <class T, int C, bool ALONG_L> __device__ __forceinline__ void take_n(const TTSlices &p, long long z, int s, int l, float v[C]) {
  const long long e = z * p.in_b + s * p.in_s + l * p.in_l;
  const bool whole = ALONG_L ? s < p.shorter && l + C <= p.longer : s + C <= p.shorter && l < p.longer;
  if constexpr (C == 4) {
    if (whole && (ALONG_L ? p.in_l : p.in_s) == 1) {
      load4((const T *)p.in + e, 4, v);
      if (p.mom) {
        float m[4];
        load4(p.mom + e, 4, m);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          m[i] = p.mu * m[i] + v[i];
          v[i] = p.nesterov ? v[i] + p.mu * m[i] : m[i];
        }
        store4(p.mom + e, 4, m);
      }
      return;
    }
  }
#pragma unroll
  for (int i = 0; i < C; ++i) {
    const int si = ALONG_L ? s : s + i, li = ALONG_L ? l + i : l;
    v[i] = si < p.shorter && li < p.longer ? take<T>(p, z, si, li) : 0.f;
  }
}
template <class T, int C, bool ALONG_L> __device__ __forceinline__ void give_n(const TTSlices &p, long long z, int s, int l, float v[C]) {
  const long long e = z * p.out_b + s * p.out_s + l * p.out_l;
  const bool whole = ALONG_L ? s < p.shorter && l + C <= p.longer : s + C <= p.shorter && l < p.longer;
  if constexpr (C == 4) {
    if (whole && (ALONG_L ? p.out_l : p.out_s) == 1) {
      T *o = (T *)p.out + e;
      if (p.mom) {
        float m[4];
        load4(o, 4, m);
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = m[i] - p.rate * v[i];
      }
      store4(o, 4, v);
      return;
    }
  }
#pragma unroll
  for (int i = 0; i < C; ++i) {
    const int si = ALONG_L ? s : s + i, li = ALONG_L ? l + i : l;
    if (si < p.shorter && li < p.longer) give<T>(p, z, si, li, v[i]);
  }
}
// 1 / (norm + eps); NaN for a sum of squares that is no number or infinite, so that the whole matrix is NaN
__device__ __forceinline__ double scale_of(double sum, float eps) {
  return sum <= 1.7976931348623157e308 ? 1.0 / (sqrt(sum) + (double)eps) : (double)NAN;
}

// ---- short side up to 8: a wavefront per matrix, all in registers -----------------------------------
// Lane l has the columns l, l + 64, ... of the long side; A is summed over the lanes and every lane has all of it.  Bound by the
// reads and writes, and by latency where there are few matrices: 5 steps of 10 sums over the wavefront for a 4 x 64 slice, 9 us for 342 of them.
template <class T, int S, int LC> __device__ __forceinline__ void slices_small(const TTSlices &p, long long z) {
  const int lane = threadIdx.x & 63;
  if (z >= p.batch) return;
  float x[LC][S];
  double sum = 0;
#pragma unroll
  for (int c = 0; c < LC; ++c)
#pragma unroll
    for (int s = 0; s < S; ++s) {
      const int l = lane + 64 * c;
      x[c][s] = s < p.shorter && l < p.longer ? take<T>(p, z, s, l) : 0.f;
      sum += (double)x[c][s] * x[c][s];
    }
  const double scale = scale_of(wave_sum64(sum), p.eps);
#pragma unroll
  for (int c = 0; c < LC; ++c)
#pragma unroll
    for (int s = 0; s < S; ++s) x[c][s] = s < p.shorter && lane + 64 * c < p.longer ? (float)((double)x[c][s] * scale) : 0.f;
  for (int i = 0; i < p.steps; ++i) {
    const float a = p.c[3 * i], b = p.c[3 * i + 1], q = p.c[3 * i + 2];
    float A[S][S];
#pragma unroll
    for (int s = 0; s < S; ++s)
#pragma unroll
      for (int t = s; t < S; ++t) {
        float v = 0.f;
#pragma unroll
        for (int c = 0; c < LC; ++c) v = fmaf(x[c][s], x[c][t], v);
        A[s][t] = A[t][s] = tt_wave_sum(v);
      }
    float B[S][S];
#pragma unroll
    for (int s = 0; s < S; ++s)
#pragma unroll
      for (int t = s; t < S; ++t) {
        float v = 0.f;
#pragma unroll
        for (int k = 0; k < S; ++k) v = fmaf(A[s][k], A[k][t], v);
        B[s][t] = B[t][s] = fmaf(b, A[s][t], q * v);
      }
#pragma unroll
    for (int c = 0; c < LC; ++c) {
      float y[S];
#pragma unroll
      for (int s = 0; s < S; ++s) {
        float v = 0.f;
#pragma unroll
        for (int k = 0; k < S; ++k) v = fmaf(B[s][k], x[c][k], v);
        y[s] = fmaf(a, x[c][s], v);
      }
#pragma unroll
      for (int s = 0; s < S; ++s) x[c][s] = y[s];
    }
  }
#pragma unroll
  for (int c = 0; c < LC; ++c)
#pragma unroll
    for (int s = 0; s < S; ++s)
      if (s < p.shorter && lane + 64 * c < p.longer) give<T>(p, z, s, lane + 64 * c, x[c][s]);
}

// ---- short side up to 64, long side up to 512: a workgroup of eight wavefronts per matrix ------------
// Each wavefront keeps 16 CT columns of X in registers, as results of the matrix instruction: lane (q, j) has rows 16 t + 4 q + i of
// column j of each 16 x 16 tile.  Columns are dealt so that a lane's are neighbours in memory (their order does not matter to X X^T).  fp32 products are six products of bf16 parts, as in tt_gemm.hip; X is at most one in norm,
// so nothing over- or underflows that counts.
//   A = X X^T: K runs over columns, of which a lane has one, so X's parts go through LDS, 32 columns at a time, [column][row], and come
//     back by the transposing read.  Each wavefront sums over its own columns; the eight sums are added in order.
//   B = b A + c A A: 16 x 16 tiles dealt to the wavefronts.
//   X <- a X + B X: K runs over rows: a lane's own rows are its operand as they are, in the order 16 t + 4 q + i of K, in
//     which B is read too.
// Measured: 342 slices of 64 x 512 (and 684 of 4 x 64) with momentum and the update of the cores 164 us, 42 of it reading and writing (228 MB: 47 us
// at 4.9 TB/s with nothing else).  A workgroup takes a compute unit (150 KB of LDS, 256 registers), so 342 slices go in two rounds of
// 256, the second a third full, and 12 us a step; of a step 5 us are X, 5 B and the adding of A's sums, which wait for LDS and barriers.
template <int MT, int CT> struct Mid {
  static constexpr int ROWS = 16 * MT, TILES = MT * (MT + 1) / 2;
  static constexpr int XP = MT == 4 ? 80 : MT == 2 ? 48 : 16;  // halves between columns: four of them meet different banks
  static constexpr int XPLANE = 32 * XP, REGION = 3 * XPLANE;  // of a wavefront: three parts of 32 columns, then its sums
  static constexpr int MP = ROWS + 8, MPLANE = ROWS * MP;      // A and B: [row][k]
  static constexpr int HALVES = 8 * REGION + 3 * MPLANE;
  static_assert(REGION * 2 >= TILES * 1024 && 8 * REGION >= 3 * MPLANE, "sums and B take the place of X's parts");
};

__device__ __forceinline__ void split4(const f32x4 &v, u16x4 &h, u16x4 &m, u16x4 &l) {
  unsigned a[3], b[3];
  tt_split_bf16(v[0], v[1], a[0], a[1], a[2]);
  tt_split_bf16(v[2], v[3], b[0], b[1], b[2]);
  typedef unsigned u2 __attribute__((ext_vector_type(2)));
  h = __builtin_bit_cast(u16x4, u2{a[0], b[0]});
  m = __builtin_bit_cast(u16x4, u2{a[1], b[1]});
  l = __builtin_bit_cast(u16x4, u2{a[2], b[2]});
}
__device__ __forceinline__ u16x8 join(u16x4 x, u16x4 y) { return __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7); }
// d += a b from three parts each, the smallest products first
__device__ __forceinline__ f32x4 mma3(const u16x8 a[3], const u16x8 b[3], f32x4 d) {
#pragma unroll
  for (int s = 2; s >= 0; --s)
#pragma unroll
    for (int x = 0; x <= s; ++x) d = mma(bf16(), a[x], b[s - x], d);
  return d;
}

template <class T, int MT, int CT> __device__ __forceinline__ void slices_mid(const TTSlices &p, long long z, unsigned short *lds, double *norms) {
  typedef Mid<MT, CT> G;
  constexpr int KS = (MT + 1) / 2;  // steps of 32 over the short side
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, q = lane >> 4, j = lane & 15;
  unsigned short *region = lds + wave * G::REGION, *pa = lds + 8 * G::REGION, *pb = lds;
  const int l0 = (wave * 16 + j) * CT;  // the lane's columns are l0 + c
  f32x4 x[MT][CT];
  if (p.in_l == 1) {
#pragma unroll
    for (int t = 0; t < MT; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float v[CT];
        take_n<T, CT, true>(p, z, 16 * t + 4 * q + i, l0, v);
#pragma unroll
        for (int c = 0; c < CT; ++c) x[t][c][i] = v[c];
      }
  } else {
#pragma unroll
    for (int t = 0; t < MT; ++t)
#pragma unroll
      for (int c = 0; c < CT; ++c) {
        float v[4];
        take_n<T, 4, false>(p, z, 16 * t + 4 * q, l0 + c, v);
        x[t][c] = f32x4{v[0], v[1], v[2], v[3]};
      }
  }
  double sum = 0;
#pragma unroll
  for (int t = 0; t < MT; ++t)
#pragma unroll
    for (int c = 0; c < CT; ++c)
#pragma unroll
      for (int i = 0; i < 4; ++i) sum += (double)x[t][c][i] * x[t][c][i];
  sum = wave_sum64(sum);
  if (lane == 0) norms[wave] = sum;
  __syncthreads();
  sum = 0;
#pragma unroll
  for (int w = 0; w < 8; ++w) sum += norms[w];
  const double scale = scale_of(sum, p.eps);
#pragma unroll
  for (int t = 0; t < MT; ++t)
#pragma unroll
    for (int c = 0; c < CT; ++c)
#pragma unroll
      for (int i = 0; i < 4; ++i) x[t][c][i] = (float)((double)x[t][c][i] * scale);  // (zeros outside: of a matrix that is NaN they are NaN too, and not stored)

  // rows 16 t .. + 15 of A or B: lane (q, j) has row j at k = 32 s + 4 q + i and 32 s + 16 + 4 q + i
  auto read = [&](const unsigned short *base, int t, int s, u16x8 f[3]) {
#pragma unroll
    for (int part = 0; part < 3; ++part) {
      const unsigned short *r = base + part * G::MPLANE + (16 * t + j) * G::MP + 32 * s + 4 * q;
      const u16x4 lo = *reinterpret_cast<const u16x4 *>(r);
      u16x4 hi = {0, 0, 0, 0};
      if constexpr (MT > 1) hi = *reinterpret_cast<const u16x4 *>(r + 16);
      f[part] = join(lo, hi);
    }
  };
  for (int step = 0; step < p.steps; ++step) {
    const float ca = p.c[3 * step], cb = p.c[3 * step + 1], cc = p.c[3 * step + 2];
    // ---- A, of the wavefront's own columns
    f32x4 sums[G::TILES] = {};
#pragma unroll
    for (int c = 0; c < CT; c += 2) {
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int t = 0; t < MT; ++t) {
          u16x4 part[3];
          split4(x[t][c + h], part[0], part[1], part[2]);
#pragma unroll
          for (int n = 0; n < 3; ++n) *reinterpret_cast<u16x4 *>(region + n * G::XPLANE + (16 * h + j) * G::XP + 16 * t + 4 * q) = part[n];
        }
      tt_wave_lds_order();
      u16x8 f[MT][3];
#pragma unroll
      for (int t = 0; t < MT; ++t)
#pragma unroll
        for (int n = 0; n < 3; ++n) {
          const unsigned short *r = region + n * G::XPLANE + (8 * q + (j >> 2)) * G::XP + 16 * t + 4 * (j & 3);
          f[t][n] = join(lds_read_tr(r), lds_read_tr(r + 4 * G::XP));
        }
      tt_wave_lds_order();
      int n = 0;
#pragma unroll
      for (int a = 0; a < MT; ++a)
#pragma unroll
        for (int b = a; b < MT; ++b, ++n) sums[n] = mma3(f[b], f[a], sums[n]);  // lane (q, j): row 16 a + j, columns 16 b + 4 q + i
      __builtin_amdgcn_sched_barrier(0);  // (one pair of column tiles after the other: with both at once the registers do not suffice)
    }
#pragma unroll
    for (int n = 0; n < G::TILES; ++n) *reinterpret_cast<f32x4 *>(reinterpret_cast<float *>(region) + n * 256 + lane * 4) = sums[n];
    __syncthreads();
    for (int e = threadIdx.x; e < G::TILES * 64; e += 512) {
      const int n = e >> 6, el = e & 63, eq = el >> 4, ej = el & 15;
      f32x4 v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int w = 0; w < 8; ++w) v += *reinterpret_cast<const f32x4 *>(reinterpret_cast<const float *>(lds + w * G::REGION) + n * 256 + el * 4);
      int a = 0, b = n;
      while (b >= MT - a) {  // tile n is (a, a + b)
        b -= MT - a;
        ++a;
      }
      b += a;
      u16x4 part[3];
      split4(v, part[0], part[1], part[2]);
#pragma unroll
      for (int m = 0; m < 3; ++m) {
        *reinterpret_cast<u16x4 *>(pa + m * G::MPLANE + (16 * a + ej) * G::MP + 16 * b + 4 * eq) = part[m];
        if (a != b)
#pragma unroll
          for (int i = 0; i < 4; ++i) pa[m * G::MPLANE + (16 * b + 4 * eq + i) * G::MP + 16 * a + ej] = part[m][i];
      }
    }
    __syncthreads();
    // ---- B
    for (int n = wave; n < MT * MT; n += 8) {
      const int a = n / MT, b = n % MT;
      f32x4 v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int s = 0; s < KS; ++s) {
        u16x8 fa[3], fb[3];
        read(pa, a, s, fa);
        read(pa, b, s, fb);
        v = mma3(fb, fa, v);  // row 16 a + j, columns 16 b + 4 q + i
      }
      const unsigned short *own = pa + (16 * a + j) * G::MP + 16 * b + 4 * q;
      const u16x4 h = *reinterpret_cast<const u16x4 *>(own), m = *reinterpret_cast<const u16x4 *>(own + G::MPLANE),
                  l = *reinterpret_cast<const u16x4 *>(own + 2 * G::MPLANE);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float A = (__uint_as_float((unsigned)l[i] << 16) + __uint_as_float((unsigned)m[i] << 16)) + __uint_as_float((unsigned)h[i] << 16);
        v[i] = fmaf(cb, A, cc * v[i]);
      }
      u16x4 part[3];
      split4(v, part[0], part[1], part[2]);
#pragma unroll
      for (int k = 0; k < 3; ++k) *reinterpret_cast<u16x4 *>(pb + k * G::MPLANE + (16 * a + j) * G::MP + 16 * b + 4 * q) = part[k];
    }
    __syncthreads();
    // ---- X
#pragma unroll
    for (int c = 0; c < CT; c += 2) {
      u16x8 f[2][KS][3];
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int s = 0; s < KS; ++s) {
          u16x4 lo[3], hi[3] = {};
          split4(x[2 * s][c + h], lo[0], lo[1], lo[2]);
          if constexpr (MT > 1) split4(x[2 * s + 1][c + h], hi[0], hi[1], hi[2]);
#pragma unroll
          for (int n = 0; n < 3; ++n) f[h][s][n] = join(lo[n], hi[n]);
        }
#pragma unroll
      for (int t = 0; t < MT; ++t) {
        f32x4 v[2] = {};
#pragma unroll
        for (int s = 0; s < KS; ++s) {
          u16x8 fb[3];
          read(pb, t, s, fb);
#pragma unroll
          for (int h = 0; h < 2; ++h) v[h] = mma3(fb, f[h][s], v[h]);  // rows 16 t + 4 q + i of column j
        }
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int i = 0; i < 4; ++i) x[t][c + h][i] = fmaf(ca, x[t][c + h][i], v[h][i]);
        __builtin_amdgcn_sched_barrier(0);
      }
    }
    __syncthreads();  // B is read no more: X's parts take its place
  }
  if (p.out_l == 1) {
#pragma unroll
    for (int t = 0; t < MT; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float v[CT];
#pragma unroll
        for (int c = 0; c < CT; ++c) v[c] = x[t][c][i];
        give_n<T, CT, true>(p, z, 16 * t + 4 * q + i, l0, v);
      }
  } else {
#pragma unroll
    for (int t = 0; t < MT; ++t)
#pragma unroll
      for (int c = 0; c < CT; ++c) {
        float v[4] = {x[t][c][0], x[t][c][1], x[t][c][2], x[t][c][3]};
        give_n<T, 4, false>(p, z, 16 * t + 4 * q, l0 + c, v);
      }
  }
}

// ---- launches --------------------------------------------------------------------------------------
// A batch with a short side above 8 and two of smaller matrices in one launch, in workgroups of 512 threads: the small slices of a
// table's cores 0 and 2 run beside the last slices of core 1, which has the launch's length.
struct Jobs {
  TTSlices mid, small[2];
  int mid_blocks, small_blocks;  // of the first small batch
};
template <class T> __device__ __forceinline__ void small_job(const TTSlices &p, int block) {
  const long long z = (long long)block * 8 + (threadIdx.x >> 6);
  if (p.shorter <= 4) {
    if (p.longer <= 64) slices_small<T, 4, 1>(p, z);
    else if (p.longer <= 128) slices_small<T, 4, 2>(p, z);
    else slices_small<T, 4, 8>(p, z);
  } else {
    if (p.longer <= 128) slices_small<T, 8, 2>(p, z);
    else slices_small<T, 8, 8>(p, z);
  }
}
template <class T, int MT, int CT> __global__ void __launch_bounds__(512, 1) k_slices(Jobs jobs) {
  __shared__ __align__(16) unsigned short lds[Mid<MT, CT>::HALVES];
  __shared__ double norms[8];
  int block = (int)blockIdx.x;
  if (block < jobs.mid_blocks) {
    slices_mid<T, MT, CT>(jobs.mid, block, lds, norms);
    return;
  }
  block -= jobs.mid_blocks;
  if (block < jobs.small_blocks) small_job<T>(jobs.small[0], block);
  else small_job<T>(jobs.small[1], block - jobs.small_blocks);
}

template <class T> tt_status launch(const TTSlices *p, int n, hipStream_t s) {
  Jobs jobs;
  for (int first = 0; first < n;) {  // each launch: as many as fit of those that follow each other
    int mids = 0, smalls = 0, next = first;
    long long blocks = 0;
    memset(&jobs, 0, sizeof(jobs));
    for (; next < n; ++next) {
      const TTSlices &q = p[next];
      const long long b = q.shorter > 8 ? q.batch : (q.batch + 7) / 8;
      if (b > TT_MAX_WORKGROUPS / 4) return TT_ERR_SHAPE;
      if (q.shorter > 8) {
        if (mids || smalls) break;
        jobs.mid = q;
        jobs.mid_blocks = (int)b;
        ++mids;
      } else {
        if (smalls == 2 || blocks + b > TT_MAX_WORKGROUPS / 2) break;
        jobs.small[smalls++] = q;
        if (smalls == 1) jobs.small_blocks = (int)b;
      }
      blocks += b;
    }
    first = next;
    const int tall = mids ? jobs.mid.shorter : 0, wide = mids ? jobs.mid.longer : 0;
    const dim3 grid((unsigned)blocks), block(512);
    if (blocks == 0) continue;
    if (tall <= 16 && wide <= 256) hipLaunchKernelGGL((k_slices<T, 1, 2>), grid, block, 0, s, jobs);
    else if (tall <= 16) hipLaunchKernelGGL((k_slices<T, 1, 4>), grid, block, 0, s, jobs);
    else if (tall <= 32 && wide <= 256) hipLaunchKernelGGL((k_slices<T, 2, 2>), grid, block, 0, s, jobs);
    else if (tall <= 32) hipLaunchKernelGGL((k_slices<T, 2, 4>), grid, block, 0, s, jobs);
    else if (wide <= 256) hipLaunchKernelGGL((k_slices<T, 4, 2>), grid, block, 0, s, jobs);
    else hipLaunchKernelGGL((k_slices<T, 4, 4>), grid, block, 0, s, jobs);
    const tt_status st = tt_launch_status();
    if (st != TT_OK) return st;
  }
  return TT_OK;
}

}  // namespace

bool ttk_slices_serves(long long shorter, long long longer) { return shorter <= 64 && longer <= 512; }

tt_status ttk_slices(const TTSlices *p, int n, hipStream_t s) {
  if (n < 1) return TT_OK;
  return p->dtype == TT_F32 ? launch<float>(p, n, s) : p->dtype == TT_BF16 ? launch<ttg::bf16>(p, n, s) : launch<ttg::f16>(p, n, s);
}
