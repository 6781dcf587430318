// Products of few rows with a K-contiguous weight: the weight is read once, straight into registers.
#include "tt_gemm_device.h"

namespace {
using namespace ttg;

// 16 columns of out and up to 16 MT rows per workgroup; its eight wavefronts take chunks of K in turn and add their sums in order at the
// end.  A lane reads 16 bytes of a weight row (16 rows, 64 bytes of each, an instruction), which is the matrix instruction's operand as it is;
// no LDS, so that two chunks of every wavefront, 64 KB on a compute unit, are on their way at once.  Bound by reading
// the weight: one token through 4096 x 4096 in bf16 8.3 us (4.0 TB/s), in tiles of 64 x 64 cut along K and joined 14.7; 48 rows through
// 1024 x 4096 7.4 us, 100 rows in 26 groups through 128 x 512 6.6, one fp32 row through 128 x 512 3.7 (a launch).
// fp32 goes through the fp32 instruction, whose rate such products do not reach.
constexpr int WAVES = 8, THREADS = 64 * WAVES;
template <class T> struct Chunk { static constexpr int E = 16 / sizeof(T), LOADS = 4, K = LOADS * 4 * E; };  // a load: 4 E values of K

template <class T> struct Piece { typedef u16x8 type; };
template <> struct Piece<float> { typedef f32x4 type; };

template <class T> __device__ __forceinline__ typename Piece<T>::type load_piece(const T *p, int left) {  // left: values from p on
  constexpr int E = Chunk<T>::E;
  typename Piece<T>::type v;
  if (left >= E) {
    const typename Vec<T>::v16b r = *reinterpret_cast<const typename Vec<T>::v16b *>(p);
#pragma unroll
    for (int i = 0; i < E; ++i) v[i] = r[i];
    return v;
  }
#pragma unroll
  for (int i = 0; i < E; ++i) {
    if constexpr (sizeof(T) == 4) v[i] = i < left ? p[i] : 0.f;
    else v[i] = i < left ? __builtin_bit_cast(unsigned short, p[i]) : (unsigned short)0;
  }
  return v;
}
template <class T> __device__ __forceinline__ f32x4 multiply(const typename Piece<T>::type &a, const typename Piece<T>::type &b, f32x4 c) {
  if constexpr (sizeof(T) == 4) {
#pragma unroll
    for (int i = 0; i < 4; ++i) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[i], b[i], c, 0, 0, 0);
    return c;
  } else {
    return mma(T(), a, b, c);
  }
}

template <class T, int MT> __global__ void __launch_bounds__(THREADS) k_gemm_rows(TTGemm g, int m_tiles, int n_tiles) {
  typedef Chunk<T> C;
  typedef typename Piece<T>::type P;
  __shared__ __align__(16) float sums[WAVES * MT * 256];
  constexpr bool F32 = sizeof(T) == 4;
  __shared__ __align__(16) float norms_a[F32 ? WAVES * MT * 16 : 4], norms_b[F32 ? WAVES * 16 : 4];  // for settle_signs: squares of every wavefront's part of K
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, q = lane >> 4, j = lane & 15;
  const int n0 = (int)(blockIdx.x % (unsigned)n_tiles) * 16, mt = (int)(blockIdx.x / (unsigned)n_tiles);
  int z, lo, hi;
  if (g.mode == TT_GEMM_RAGGED_M) {
    const int there = find_tile<16 * MT>(g.offsets, g.batch, g.M, mt, z, lo, hi);
    if (z < 0) {
      if (g.zero_rest && threadIdx.x < 256) clear_rest<T>(g, lo, hi, mt - there, m_tiles - there, n0, 16);
      return;
    }
  } else {
    z = (int)blockIdx.y;
    lo = mt * 16 * MT;
    hi = g.M < lo + 16 * MT ? g.M : lo + 16 * MT;
  }
  // rows outside: a row inside, whose results are not stored
  const T *b = (const T *)g.b + z * g.b_step + (long long)(n0 + j < g.N ? n0 + j : g.N - 1) * g.ldb + q * C::E;
  const T *a[MT];
#pragma unroll
  for (int x = 0; x < MT; ++x) {
    const int m = lo + 16 * x + j;
    a[x] = (const T *)g.a + (g.mode == TT_GEMM_BATCH ? z * g.a_step : 0) + (long long)(m < hi ? m : hi - 1) * g.lda + q * C::E;
  }
  f32x4 acc[MT] = {};
  P fb[2][C::LOADS], fa[2][MT][C::LOADS];
  const int K = g.K, skip = WAVES * C::K;
  auto load = [&](P (&lb)[C::LOADS], P (&la)[MT][C::LOADS], int k0) {
#pragma unroll
    for (int i = 0; i < C::LOADS; ++i) {
      const int k = k0 + i * 4 * C::E, left = K - k - q * C::E;
      lb[i] = load_piece<T>(b + k, left);
#pragma unroll
      for (int x = 0; x < MT; ++x) la[x][i] = load_piece<T>(a[x] + k, left);
    }
  };
  const bool settles = F32 && ttk_gemm_settles(g);
  float squares_a[MT] = {}, squares_b = 0.f;  // of the lane's values of rows j
  const int first = wave * C::K;
  if (first < K) load(fb[0], fa[0], first);
  if (first + skip < K) load(fb[1], fa[1], first + skip);
  for (int k0 = first; k0 < K; k0 += 2 * skip) {
#pragma unroll
    for (int d = 0; d < 2; ++d) {
      if (k0 + d * skip >= K) break;
#pragma unroll
      for (int i = 0; i < C::LOADS; ++i)
#pragma unroll
        for (int x = 0; x < MT; ++x) acc[x] = multiply<T>(fb[d][i], fa[d][x][i], acc[x]);  // lane (q, j): row j, columns 4 q + i
      if constexpr (F32) {
        if (settles) {
#pragma unroll
          for (int i = 0; i < C::LOADS; ++i)
#pragma unroll
            for (int e = 0; e < C::E; ++e) {
              squares_b = fmaf(fb[d][i][e], fb[d][i][e], squares_b);
#pragma unroll
              for (int x = 0; x < MT; ++x) squares_a[x] = fmaf(fa[d][x][i][e], fa[d][x][i][e], squares_a[x]);
            }
        }
      }
      if (k0 + (d + 2) * skip < K) load(fb[d], fa[d], k0 + (d + 2) * skip);
    }
  }
#pragma unroll
  for (int x = 0; x < MT; ++x) *reinterpret_cast<f32x4 *>(sums + (wave * MT + x) * 256 + lane * 4) = acc[x];
  if constexpr (F32) {
    if (settles) {
#pragma unroll
      for (int o = 16; o < 64; o *= 2) {
        squares_b += __shfl(squares_b, lane ^ o, 64);
#pragma unroll
        for (int x = 0; x < MT; ++x) squares_a[x] += __shfl(squares_a[x], lane ^ o, 64);
      }
      if (q == 0) {
        norms_b[wave * 16 + j] = squares_b;
#pragma unroll
        for (int x = 0; x < MT; ++x) norms_a[(wave * MT + x) * 16 + j] = squares_a[x];
      }
    }
  }
  __syncthreads();
  for (int e = threadIdx.x; e < MT * 64; e += THREADS) {
    f32x4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int v = 0; v < WAVES; ++v) s += *reinterpret_cast<const f32x4 *>(sums + v * MT * 256 + e * 4);
    const int m = lo + 16 * (e >> 6) + (e & 15), n = n0 + 4 * ((e >> 4) & 3);
    float v[4] = {s[0], s[1], s[2], s[3]};
    if constexpr (F32) {
      if (settles) {  // (a wavefront has a whole turn of this loop or none)
        const float none[4] = {0.f, 0.f, 0.f, 0.f};  // (bias is in v)
        float sa = 0.f, sb[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
          sa += norms_a[(w * MT + (e >> 6)) * 16 + (e & 15)];
#pragma unroll
          for (int i = 0; i < 4; ++i) sb[i] += norms_b[w * 16 + 4 * ((e >> 4) & 3) + i];
        }
        const int valid = m < hi ? (g.N - n < 4 ? g.N - n : 4) : 0;
        float bias[4] = {0.f, 0.f, 0.f, 0.f};
        if (g.bias) load4((const float *)g.bias + z * g.bias_step + n, valid, bias);
        settle_signs<4>(g, z, m, n, valid, v, bias, sa, sb);
        if (valid > 0) finish<T, T, 4>(g, z, m, n, valid, v, none);
        continue;
      }
    }
    if (m < hi && n < g.N) finish<T, T, 4>(g, z, m, n, g.N - n < 4 ? g.N - n : 4, v);
  }
}

template <class T, int MT> tt_status launch(const TTGemm &g, hipStream_t s) {
  const long long n_tiles = tt_ceil_div(g.N, 16), members = g.mode == TT_GEMM_RAGGED_M ? 1 : g.batch;
  const long long m_tiles = g.mode == TT_GEMM_RAGGED_M ? (long long)tt_ceil_div(g.M, 16 * MT) + g.batch + 1 : tt_ceil_div(g.M, 16 * MT);
  if (m_tiles * n_tiles > TT_MAX_WORKGROUPS / 2 || m_tiles * n_tiles * members > TT_MAX_WORKGROUPS / 2 || members > 65535) return TT_ERR_SHAPE;
  const int mti = (int)m_tiles, nti = (int)n_tiles;
  hipLaunchKernelGGL((k_gemm_rows<T, MT>), dim3((unsigned)(m_tiles * n_tiles), (unsigned)members), dim3(THREADS), 0, s, g, mti, nti);
  return tt_launch_status();
}
template <class T> tt_status launch_t(const TTGemm &g, hipStream_t s) {
  // rows of a group of the average size, in RAGGED_M
  const int rows = g.mode == TT_GEMM_RAGGED_M ? tt_ceil_div(g.M, g.batch) : g.M;
  return rows <= 16 ? launch<T, 1>(g, s) : rows <= 32 ? launch<T, 2>(g, s) : launch<T, 4>(g, s);
}

}  // namespace

// Up to 32 rows (of a group of the average size) always; more while there are few workgroups and the rows that each of them reads are
// short.  These / tiles, us: bf16 16 x 512 x 512 3.4 / 8.3, 64 x 4096 x 1024 7.5 / 11.8, 256 x 512 x 512 4.9 / 8.8, 128 x 1024 x 1024 7.0 / 9.5,
// 96 x 4096 x 1024 11.8 / 12.7, 64 x 4096 x 4096 21.7 / 17.1, 128 x 4096 x 4096 41 / 22; fp32 64 x 512 x 512 8.0 / 10.8, 128 x 1024 x 1024 14.4 / 15.0.
#ifndef TT_GEMM_FEW_ROWS
#define TT_GEMM_FEW_ROWS 32
#endif
bool ttk_gemm_rows_serves(const TTGemm &g) {
  if (g.out_dtype != g.dtype || !g.a_kc || !g.b_kc || g.rowsum || g.symmetric || g.mode == TT_GEMM_RAGGED_K || g.parts == 2 || g.epilogue != TT_GEMM_PLAIN) return false;
  const int rows = g.mode == TT_GEMM_RAGGED_M ? tt_ceil_div(g.M, g.batch) : g.M;
  if (rows <= TT_GEMM_FEW_ROWS) return true;
  const long long bytes = (long long)g.K * (g.dtype == TT_F32 ? 4 : 2), groups = (long long)tt_ceil_div(rows, 64) * tt_ceil_div(g.N, 16) * g.batch;
  return TT_GEMM_FEW_ROWS > 0 && rows <= 256 && bytes <= 4096 && groups <= 256;
}
tt_status ttk_gemm_rows(const TTGemm &g, hipStream_t s) {
  return g.dtype == TT_F32 ? launch_t<float>(g, s) : g.dtype == TT_BF16 ? launch_t<ttg::bf16>(g, s) : launch_t<ttg::f16>(g, s);
}
