// Device kernels of the orthogonalised updates.
//
// For every matrix of a unit, with r = min(rows, cols), c = max(rows, cols)
// and the working matrix X [r][c] (the stored one, or its transpose):
//
//   source   u of the call (the update itself; a worker's momentum step; the
//            outer step's Nesterov direction) and its sums of squares
//   load     X = u / ||u||_F, and X^T
//   gram     A = X X^T              } steps times, each a launch over the
//   square   polynomial of A        } tiles of all matrices
//   update   X <- (polynomial) X    }
//   apply    the call's outputs from O = X
//
// Numerics.  The products run on the fp16 matrix cores with fp32 sums.  Two
// things keep them near 32 bits of X at that price:
//  * X is held to 22 bits as the sum of two fp16 values (high + low).  The
//    term a X of an iteration uses both; a product uses the high half
//    (EDIT_ORTHO_FAST), or high*high + high*low + low*high (EDIT_ORTHO_FULL).
//  * A is taken about its mean diagonal s = ||X||_F^2 / r: with R = A - sI,
//      a + b A + c A^2 = (a + bs + cs^2) + (b + 2cs) R + c R^2
//    for any s.  Once the singular values are near one, R is small where A is
//    near I, and what fp16 rounds off R is small with it; b A + c A^2 would
//    cancel to a third of its terms.  Only s must be the same in the three
//    products, so it is computed once per iteration and stored.
// Error of O against 64 bits: 1e-4 to 1e-3 with FAST over Gaussian, low-rank
// and power-law spectra (1e-3 to 4e-2 if X itself were rounded to fp16, 1e-2
// to 9e-2 in bf16), and that of a 32-bit iteration with FULL.
#include "edit_ortho_internal.h"

namespace edit {
namespace {

typedef _Float16 half8 __attribute__((ext_vector_type(8)));
typedef _Float16 half4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
typedef float float2_t __attribute__((ext_vector_type(2)));

// ------------------------------------------------------- elements of a unit

constexpr int kVec = 8;  // elements per thread and step of the streaming passes

__device__ __forceinline__ float widen_bf16(uint32_t h) { return __uint_as_float(h << 16); }

__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
  const float2_t f = {a, b};
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(f, bf16x2_t));  // RNE
}

template <bool BF16>
__device__ __forceinline__ float load_one(const void* p, int64_t i) {
  if constexpr (BF16)
    return widen_bf16(static_cast<const uint16_t*>(p)[i]);
  else
    return static_cast<const float*>(p)[i];
}

template <bool BF16>
__device__ __forceinline__ void store_one(void* p, int64_t i, float x) {
  if constexpr (BF16)
    static_cast<uint16_t*>(p)[i] = static_cast<uint16_t>(pack_bf16(x, 0.f));
  else
    static_cast<float*>(p)[i] = x;
}

// Elements i .. i+7 (i a multiple of 8, the unit 16-byte aligned) of which
// [lo, hi) are in range.
template <bool BF16>
__device__ __forceinline__ void load_vec(const void* p, int64_t i, int lo, int hi, float (&x)[kVec]) {
  if (lo == 0 && hi == kVec) {
    if constexpr (BF16) {
      const u32x4 w = *reinterpret_cast<const u32x4*>(static_cast<const uint16_t*>(p) + i);
#pragma unroll
      for (int e = 0; e < kVec; ++e) x[e] = __uint_as_float((e & 1) ? (w[e >> 1] & 0xffff0000u) : (w[e >> 1] << 16));
    } else {
      const f32x4* q = reinterpret_cast<const f32x4*>(static_cast<const float*>(p) + i);
      const f32x4 a = q[0], b = q[1];
#pragma unroll
      for (int e = 0; e < 4; ++e) x[e] = a[e], x[e + 4] = b[e];
    }
  } else {
#pragma unroll
    for (int e = 0; e < kVec; ++e) x[e] = e >= lo && e < hi ? load_one<BF16>(p, i + e) : 0.f;
  }
}

template <bool BF16>
__device__ __forceinline__ void store_vec(void* p, int64_t i, int lo, int hi, const float (&x)[kVec]) {
  if (lo == 0 && hi == kVec) {
    if constexpr (BF16) {
      u32x4 w;
#pragma unroll
      for (int e = 0; e < 4; ++e) w[e] = pack_bf16(x[2 * e], x[2 * e + 1]);
      *reinterpret_cast<u32x4*>(static_cast<uint16_t*>(p) + i) = w;
    } else {
      f32x4* q = reinterpret_cast<f32x4*>(static_cast<float*>(p) + i);
      q[0] = f32x4{x[0], x[1], x[2], x[3]};
      q[1] = f32x4{x[4], x[5], x[6], x[7]};
    }
  } else {
#pragma unroll
    for (int e = 0; e < kVec; ++e)
      if (e >= lo && e < hi) store_one<BF16>(p, i + e, x[e]);
  }
}

// Sum over a block in a fixed order; every thread calls it and gets the sum.
template <int kThreads>
__device__ __forceinline__ double block_sum(double x) {
  __shared__ double red[kThreads / 64];
#pragma unroll
  for (int m = 32; m >= 1; m >>= 1) x += __shfl_xor(x, m, 64);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = x;
  __syncthreads();
  double s = red[0];
#pragma unroll
  for (int w = 1; w < kThreads / 64; ++w) s += red[w];
  return s;
}

// ------------------------------------------------------------- source pass

struct RepPtrs {
  void* p[EDIT_MAX_K];
};

struct OrthoArgs {
  const void* x;
  void* out;
  float* momentum;
  float* theta;
  float* u;
  const UnitRecord* rec;
  int32_t workers;
  int32_t nesterov;
  double mu, keep, lr;
};

// One chunk per block: the call's update u, its sum of squares, and what the
// call stores on the way (the momentum; the outer step's u, and the whole
// step of elements that belong to no matrix).  Bound by memory.
template <int SOURCE, bool BF16>
__global__ __launch_bounds__(kOrthoStreamThreads) void ortho_source_kernel(OrthoArgs a, RepPtrs reps,
                                                                          const OrthoMat* __restrict__ mats,
                                                                          const OrthoChunk* __restrict__ chunks) {
  const OrthoChunk ch = chunks[blockIdx.x];
  double sum = 0.0;
  const int64_t first = ch.begin / kVec;
  const int64_t last = (ch.end + kVec - 1) / kVec;
  for (int64_t v = first + threadIdx.x; v < last; v += kOrthoStreamThreads) {
    const int64_t i = v * kVec;
    const int lo = ch.begin > i ? static_cast<int>(ch.begin - i) : 0;
    const int hi = ch.end < i + kVec ? static_cast<int>(ch.end - i) : kVec;
    if constexpr (SOURCE == kSourcePlain) {
      float x[kVec];
      load_vec<BF16>(a.x, i, lo, hi, x);
#pragma unroll
      for (int e = 0; e < kVec; ++e) sum = fma(static_cast<double>(x[e]), static_cast<double>(x[e]), sum);
    } else if constexpr (SOURCE == kSourceLocal) {
      float g[kVec], m[kVec];
      load_vec<BF16>(a.x, i, lo, hi, g);
      load_vec<false>(a.momentum, i, lo, hi, m);
#pragma unroll
      for (int e = 0; e < kVec; ++e) {
        m[e] = static_cast<float>(fma(a.mu, static_cast<double>(m[e]), static_cast<double>(g[e])));
        const double u = a.nesterov ? fma(a.mu, static_cast<double>(m[e]), static_cast<double>(g[e])) : m[e];
        sum = fma(u, u, sum);
      }
      store_vec<false>(a.momentum, i, lo, hi, m);
    } else {
      // b' = rho b - D and u = rho b' - D, D = sum_j c_j (r_j - theta); a
      // rollback moves nothing (u = 0 leaves the matrices where they are)
      const UnitRecord* rec = a.rec;
      const bool rollback = rec->rollback;
      float th[kVec], b[kVec], u[kVec];
      load_vec<false>(a.theta, i, lo, hi, th);
#pragma unroll
      for (int e = 0; e < kVec; ++e) u[e] = 0.f;
      if (!rollback) {
        double d[kVec];
        load_vec<false>(a.momentum, i, lo, hi, b);
#pragma unroll
        for (int e = 0; e < kVec; ++e) d[e] = 0.0;
        if (rec->use_deltas) {
          for (int j = 0; j < a.workers; ++j) {
            const double c = rec->coef[j];
            const int s = __builtin_amdgcn_readfirstlane(rec->src[j]);
            float x[kVec];
            load_vec<BF16>(reps.p[s], i, lo, hi, x);
#pragma unroll
            for (int e = 0; e < kVec; ++e)
              d[e] = fma(c, static_cast<double>(x[e]) - static_cast<double>(th[e]), d[e]);
          }
        }
#pragma unroll
        for (int e = 0; e < kVec; ++e) {
          const double bn = fma(a.mu, static_cast<double>(b[e]), -d[e]);
          const double step = fma(a.mu, bn, -d[e]);
          b[e] = static_cast<float>(bn);
          u[e] = static_cast<float>(step);
          if (ch.mat < 0) th[e] = static_cast<float>(static_cast<double>(th[e]) - a.lr * step);
        }
        store_vec<false>(a.momentum, i, lo, hi, b);
      }
      if (ch.mat < 0) {
        if (!rollback) store_vec<false>(a.theta, i, lo, hi, th);
        for (int j = 0; j < a.workers; ++j) store_vec<BF16>(reps.p[j], i, lo, hi, th);
      } else {
        store_vec<false>(a.u, i, lo, hi, u);
#pragma unroll
        for (int e = 0; e < kVec; ++e)
          if (e >= lo && e < hi) sum = fma(static_cast<double>(u[e]), static_cast<double>(u[e]), sum);
      }
    }
  }
  if (ch.mat < 0) return;
  sum = block_sum<kOrthoStreamThreads>(sum);
  if (threadIdx.x == 0) mats[ch.mat].norm_part[ch.slot] = sum;
}

// --------------------------------------------------------------- load pass

__device__ __forceinline__ void split(float v, _Float16& hi, _Float16& lo) {
  hi = static_cast<_Float16>(v);
  lo = static_cast<_Float16>(v - static_cast<float>(hi));
}

// One 64 x 64 tile of a stored matrix per block: X = u / ||u|| at kScaleX,
// written in the stored orientation and, through LDS, transposed.
template <int SOURCE, bool BF16, bool FULL>
__global__ __launch_bounds__(kOrthoStreamThreads) void ortho_load_kernel(OrthoArgs a, const OrthoMat* __restrict__ mats,
                                                                        const OrthoTile* __restrict__ tiles) {
  constexpr int T = kOrthoLoadTile;
  __shared__ uint32_t lds[T][T + 1];  // high half in the low 16 bits
  const OrthoTile t = tiles[blockIdx.x];
  const OrthoMat& mt = mats[t.mat];
  double sum = 0.0;
  for (int i = threadIdx.x; i < mt.chunks; i += kOrthoStreamThreads) sum += mt.norm_part[i];
  sum = block_sum<kOrthoStreamThreads>(sum);
  // sums of squares of fp32 values neither overflow nor vanish in fp64, nor does their root's inverse
  const double inv = sum > 0.0 ? kScaleX / sqrt(sum) : (sum == 0.0 ? 0.0 : sum);
  const int tx = threadIdx.x & 63, ty = threadIdx.x >> 6;
  const int row0 = t.m * T, col0 = t.n * T;
  _Float16* nat_hi = mt.tall ? mt.t[0][0] : mt.x[0];
  _Float16* nat_lo = mt.tall ? mt.t[0][1] : mt.x[1];
  _Float16* tr_hi = mt.tall ? mt.x[0] : mt.t[0][0];
  _Float16* tr_lo = mt.tall ? mt.x[1] : mt.t[0][1];
  const int64_t ld_nat = mt.tall ? mt.ldr : mt.ldc;
  const int64_t ld_tr = mt.tall ? mt.ldc : mt.ldr;
  // X^T needs its low half in the products only
  const bool nat_has_lo = FULL || !mt.tall;
  const bool tr_has_lo = FULL || mt.tall;
  for (int y = ty; y < T; y += kOrthoStreamThreads / 64) {
    const int row = row0 + y, col = col0 + tx;
    float v = 0.f;
    if (row < mt.rows && col < mt.cols) {
      const int64_t i = mt.offset + static_cast<int64_t>(row) * mt.cols + col;
      double u;
      if constexpr (SOURCE == kSourcePlain) {
        u = load_one<BF16>(a.x, i);
      } else if constexpr (SOURCE == kSourceLocal) {
        const double m = a.momentum[i];
        u = a.nesterov ? fma(a.mu, m, static_cast<double>(load_one<BF16>(a.x, i))) : m;
      } else {
        u = a.u[i];
      }
      v = static_cast<float>(u * inv);
      _Float16 hi, lo;
      split(v, hi, lo);
      nat_hi[row * ld_nat + col] = hi;
      if (nat_has_lo) nat_lo[row * ld_nat + col] = lo;
      lds[y][tx] = __builtin_bit_cast(uint16_t, hi) | static_cast<uint32_t>(__builtin_bit_cast(uint16_t, lo)) << 16;
    }
  }
  __syncthreads();
  for (int y = ty; y < T; y += kOrthoStreamThreads / 64) {
    const int col = col0 + y, row = row0 + tx;
    if (row < mt.rows && col < mt.cols) {
      const uint32_t w = lds[tx][y];
      tr_hi[col * ld_tr + row] = __builtin_bit_cast(_Float16, static_cast<uint16_t>(w));
      if (tr_has_lo) tr_lo[col * ld_tr + row] = __builtin_bit_cast(_Float16, static_cast<uint16_t>(w >> 16));
    }
  }
}

// ---------------------------------------------------------------- products

// Product C[m][n] = sum_k P[m][k] Q[n][k] over the tiles of all matrices, both
// operands row by row along k:
//   gram    P = Q = X          C -> R = C - sI                (symmetric)
//   square  P = Q = R          C -> (b + 2cs) R + c C         (symmetric)
//   update  P = X^T, Q = poly  C -> X^T' = (a + bs + cs^2) X^T + C
// Symmetric products take the tiles with m >= n and store each twice.
struct ProductArgs {
  double a, b, c;
  int32_t from, first, last;
};

template <int PRODUCT, bool FULL, int BM, int BN, int WM, int WN, int BK>
struct ProductShape {
  static constexpr int kWaves = (BM / WM) * (BN / WN);
  static constexpr int kThreads = kWaves * 64;
  static constexpr int kHalves = FULL ? 2 : 1;
  static constexpr int kRowBytes = BK * 2;
  static constexpr int kChunks = kRowBytes / 16;            // 16-byte chunks of a row
  static constexpr int kStage = (BM + BN) * kRowBytes * kHalves;
  static constexpr int kRowsPerLoad = 1024 / kRowBytes;     // rows that a wave's load fills
  static constexpr int kLoadsP = BM / kRowsPerLoad / kWaves;
  static constexpr int kLoadsQ = BN / kRowsPerLoad / kWaves;
};

// LDS holds rows of BK values; the 16-byte chunks of a row are permuted by
// its number, so that the 16 rows that a wave reads at once lie in different
// banks.
template <int CHUNKS>
__device__ __forceinline__ int chunk_swizzle(int row) {
  return CHUNKS == 8 ? (row & 7) : ((row >> 1) & 3);
}

// 16 bytes a lane from global memory to LDS, no register in between: lane l's
// go to `lds` + 16 l.  The compiler keeps nothing in m0 here (no indirect
// register access, no messages); with its own builtin it would wait for the
// load before any other read of LDS.
__device__ __forceinline__ void load_to_lds(uint32_t lds, const void* base, uint32_t offset) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2"
               :
               : "s"(lds), "v"(offset), "s"(base)
               : "memory");
}

template <int PRODUCT, bool FULL, int BM, int BN, int WM, int WN, int BK>
__global__ __launch_bounds__((ProductShape<PRODUCT, FULL, BM, BN, WM, WN, BK>::kThreads)) void ortho_product_kernel(
    const OrthoMat* __restrict__ mats, const OrthoTile* __restrict__ tiles, ProductArgs args, float* __restrict__ out) {
  using S = ProductShape<PRODUCT, FULL, BM, BN, WM, WN, BK>;
  __shared__ __align__(128) char smem[2 * S::kStage];
  const OrthoTile t = tiles[blockIdx.x];
  if (t.mat < 0) return;
  const OrthoMat& mt = mats[t.mat];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);

  // s of this iteration: the mean of A's diagonal, ||X||^2 / r (1 / r at first)
  double s;
  if constexpr (PRODUCT == kProductGram) {
    if (args.first) {
      s = 1.0;
    } else {
      s = 0.0;
      for (int i = threadIdx.x; i < mt.x_tiles; i += S::kThreads) s += mt.x_part[i];
      s = block_sum<S::kThreads>(s);
    }
    s /= mt.r;
    if (t.m == 0 && t.n == 0 && threadIdx.x == 0) *mt.shift = s;
  } else {
    s = *mt.shift;
  }

  const _Float16* p[2];
  const _Float16* q[2];
  int ld, rows_p, rows_q;
  if constexpr (PRODUCT == kProductGram) {
    p[0] = q[0] = mt.x[0], p[1] = q[1] = mt.x[1];
    ld = mt.ldc, rows_p = rows_q = mt.r;
  } else if constexpr (PRODUCT == kProductSquare) {
    p[0] = q[0] = mt.g[0], p[1] = q[1] = mt.g[1];
    ld = mt.ldr, rows_p = rows_q = mt.r;
  } else {
    p[0] = mt.t[args.from][0], p[1] = mt.t[args.from][1];
    q[0] = mt.q[0], q[1] = mt.q[1];
    ld = mt.ldr, rows_p = mt.c, rows_q = mt.r;
  }

  // Byte offsets of this lane's loads.  Rows past the end read the last one:
  // what they give is not stored.
  uint32_t off_p[S::kLoadsP], off_q[S::kLoadsQ];
  const int lrow = lane / S::kChunks, lchunk = lane % S::kChunks;
#pragma unroll
  for (int i = 0; i < S::kLoadsP; ++i) {
    const int row = (wave + i * S::kWaves) * S::kRowsPerLoad + lrow;
    const int g = min(t.m * BM + row, rows_p - 1);
    off_p[i] = (static_cast<uint32_t>(g) * static_cast<uint32_t>(ld)) * 2u +
               16u * (lchunk ^ chunk_swizzle<S::kChunks>(row));
  }
#pragma unroll
  for (int i = 0; i < S::kLoadsQ; ++i) {
    const int row = (wave + i * S::kWaves) * S::kRowsPerLoad + lrow;
    const int g = min(t.n * BN + row, rows_q - 1);
    off_q[i] = (static_cast<uint32_t>(g) * static_cast<uint32_t>(ld)) * 2u +
               16u * (lchunk ^ chunk_swizzle<S::kChunks>(row));
  }

  const uint32_t lds0 = static_cast<uint32_t>(
      reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) char*)(smem)));  // byte offset in LDS
  constexpr int kPBytes = BM * S::kRowBytes, kQBytes = BN * S::kRowBytes;
  auto fetch = [&](int stage, int k) {
    const uint32_t at = lds0 + stage * S::kStage;
#pragma unroll
    for (int h = 0; h < S::kHalves; ++h) {
#pragma unroll
      for (int i = 0; i < S::kLoadsP; ++i)
        load_to_lds(at + h * kPBytes + (wave + i * S::kWaves) * 1024, p[h] + k * BK, off_p[i]);
#pragma unroll
      for (int i = 0; i < S::kLoadsQ; ++i)
        load_to_lds(at + S::kHalves * kPBytes + h * kQBytes + (wave + i * S::kWaves) * 1024, q[h] + k * BK, off_q[i]);
    }
  };

  constexpr int FM = WM / 16, FN = WN / 16;
  const int wm = (wave % (BM / WM)) * WM, wn = (wave / (BM / WM)) * WN;
  f32x4 acc[FM][FN];
#pragma unroll
  for (int i = 0; i < FM; ++i)
#pragma unroll
    for (int j = 0; j < FN; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};

  const int frow = lane & 15, fchunk = lane >> 4;
  const int steps = ld / BK;
  fetch(0, 0);
  for (int k = 0; k < steps; ++k) {
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();  // stage k has landed for all waves, and all have read stage k - 1
    if (k + 1 < steps) fetch((k + 1) & 1, k + 1);
    const char* st = smem + (k & 1) * S::kStage;
#pragma unroll
    for (int kk = 0; kk < BK / 32; ++kk) {
      half8 pf[S::kHalves][FM], qf[S::kHalves][FN];
#pragma unroll
      for (int h = 0; h < S::kHalves; ++h) {
#pragma unroll
        for (int i = 0; i < FM; ++i) {
          const int row = wm + i * 16 + frow;
          pf[h][i] = *reinterpret_cast<const half8*>(
              st + h * kPBytes + row * S::kRowBytes + 16 * ((kk * 4 + fchunk) ^ chunk_swizzle<S::kChunks>(row)));
        }
#pragma unroll
        for (int j = 0; j < FN; ++j) {
          const int row = wn + j * 16 + frow;
          qf[h][j] = *reinterpret_cast<const half8*>(
              st + S::kHalves * kPBytes + h * kQBytes + row * S::kRowBytes +
              16 * ((kk * 4 + fchunk) ^ chunk_swizzle<S::kChunks>(row)));
        }
      }
#pragma unroll
      for (int i = 0; i < FM; ++i)
#pragma unroll
        for (int j = 0; j < FN; ++j) {
          acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(pf[0][i], qf[0][j], acc[i][j], 0, 0, 0);
          if constexpr (FULL) {
            acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(pf[0][i], qf[1][j], acc[i][j], 0, 0, 0);
            acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(pf[1][i], qf[0][j], acc[i][j], 0, 0, 0);
          }
        }
    }
  }

  // Lane l holds C[m .. m+3][n] of each 16 x 16 block: m = 4 (l / 16), n = l mod 16.
  const int m0 = t.m * BM + wm + 4 * (lane >> 4), n0 = t.n * BN + wn + (lane & 15);
  if constexpr (PRODUCT != kProductUpdate) {
    const int r = mt.r;
    const int64_t ldr = mt.ldr;
    _Float16* dst_hi = PRODUCT == kProductGram ? mt.g[0] : mt.q[0];
    _Float16* dst_lo = PRODUCT == kProductGram ? mt.g[1] : mt.q[1];
    // the polynomial's low half goes into products only
    constexpr bool kLow = PRODUCT == kProductGram || FULL;
    const float shift = static_cast<float>(s * kScaleA);
    const float lin = static_cast<float>(args.b + 2.0 * args.c * s);
    const float quad = static_cast<float>(args.c) / kScaleA;
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
      for (int j = 0; j < FN; ++j) {
        const int n = n0 + j * 16;
        if (n >= r) continue;
        half4 hi, lo;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int m = m0 + i * 16 + e;
          float v = 0.f;
          if (m < r) {
            if constexpr (PRODUCT == kProductGram) {
              v = acc[i][j][e] * (kScaleA / (kScaleX * kScaleX));
              if (m == n) v -= shift;
            } else {
              // R is symmetric: read along the row that is stored contiguously
              const int64_t at = n * ldr + m;
              v = lin * (static_cast<float>(mt.g[0][at]) + static_cast<float>(mt.g[1][at])) + quad * acc[i][j][e];
            }
          }
          _Float16 h, l;
          split(v, h, l);
          hi[e] = h, lo[e] = l;
          if (m < r && t.m != t.n) {
            dst_hi[m * ldr + n] = h;
            if constexpr (kLow) dst_lo[m * ldr + n] = l;
          }
        }
        const int m = m0 + i * 16;
        if (m + 3 < r) {
          *reinterpret_cast<half4*>(dst_hi + n * ldr + m) = hi;
          if constexpr (kLow) *reinterpret_cast<half4*>(dst_lo + n * ldr + m) = lo;
        } else {
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (m + e < r) {
              dst_hi[n * ldr + m + e] = hi[e];
              if constexpr (kLow) dst_lo[n * ldr + m + e] = lo[e];
            }
        }
      }
  } else {
    const int r = mt.r, c = mt.c;
    const int64_t ldr = mt.ldr, ldc = mt.ldc;
    _Float16* to_hi = mt.t[args.from ^ 1][0];
    _Float16* to_lo = mt.t[args.from ^ 1][1];
    const float keep = static_cast<float>(args.a + args.b * s + args.c * s * s);
    float sq = 0.f;
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
      for (int j = 0; j < FN; ++j) {
        const int n = n0 + j * 16, m = m0 + i * 16;  // X[n][m .. m+3]
        if (n >= r) continue;
        const int64_t at = n * ldc + m;
        half4 hi, lo;
        float v[4];
        const bool whole = m + 3 < c;
        if (whole) {
          hi = *reinterpret_cast<const half4*>(mt.x[0] + at);
          lo = *reinterpret_cast<const half4*>(mt.x[1] + at);
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          v[e] = 0.f;
          if (m + e < c) {
            const float x = whole ? static_cast<float>(hi[e]) + static_cast<float>(lo[e])
                                  : static_cast<float>(mt.x[0][at + e]) + static_cast<float>(mt.x[1][at + e]);
            v[e] = keep * x + acc[i][j][e] * (1.f / kScaleA);
          }
        }
        if (args.last) {
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (m + e < c) {
              const int64_t o = mt.tall ? static_cast<int64_t>(m + e) * mt.cols + n
                                        : static_cast<int64_t>(n) * mt.cols + m + e;
              out[mt.offset + o] = v[e] * (1.f / kScaleX);
            }
        } else {
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            sq += v[e] * v[e];
            _Float16 h, l;
            split(v[e], h, l);
            hi[e] = h, lo[e] = l;
            if (m + e < c) {
              to_hi[(m + e) * ldr + n] = h;
              if constexpr (FULL) to_lo[(m + e) * ldr + n] = l;
              if (!whole) mt.x[0][at + e] = h, mt.x[1][at + e] = l;
            }
          }
          if (whole) {
            *reinterpret_cast<half4*>(mt.x[0] + at) = hi;
            *reinterpret_cast<half4*>(mt.x[1] + at) = lo;
          }
        }
      }
    if (!args.last) {
      const double sum = block_sum<S::kThreads>(static_cast<double>(sq) / (static_cast<double>(kScaleX) * kScaleX));
      if (threadIdx.x == 0) mt.x_part[t.slot] = sum;
    }
  }
}

// -------------------------------------------------------------- apply pass

// One chunk of a matrix per block: the call's outputs from O, which is fp32 in
// the stored order.  Bound by memory.
template <int SOURCE, bool BF16>
__global__ __launch_bounds__(kOrthoStreamThreads) void ortho_apply_kernel(OrthoArgs a, RepPtrs reps,
                                                                         const OrthoMat* __restrict__ mats,
                                                                         const OrthoChunk* __restrict__ chunks) {
  const OrthoChunk ch = chunks[blockIdx.x];
  if (ch.mat < 0) return;
  const double step = a.lr * mats[ch.mat].scale;
  const int64_t first = ch.begin / kVec;
  const int64_t last = (ch.end + kVec - 1) / kVec;
  for (int64_t v = first + threadIdx.x; v < last; v += kOrthoStreamThreads) {
    const int64_t i = v * kVec;
    const int lo = ch.begin > i ? static_cast<int>(ch.begin - i) : 0;
    const int hi = ch.end < i + kVec ? static_cast<int>(ch.end - i) : kVec;
    float o[kVec];
    load_vec<false>(a.u, i, lo, hi, o);
    if constexpr (SOURCE == kSourcePlain) {
      store_vec<BF16>(a.out, i, lo, hi, o);
    } else if constexpr (SOURCE == kSourceLocal) {
      float p[kVec];
      load_vec<BF16>(a.out, i, lo, hi, p);
#pragma unroll
      for (int e = 0; e < kVec; ++e)
        p[e] = static_cast<float>(fma(a.keep, static_cast<double>(p[e]), -step * static_cast<double>(o[e])));
      store_vec<BF16>(a.out, i, lo, hi, p);
    } else {
      float th[kVec];
      load_vec<false>(a.theta, i, lo, hi, th);
      if (!a.rec->rollback) {
#pragma unroll
        for (int e = 0; e < kVec; ++e)
          th[e] = static_cast<float>(fma(-step, static_cast<double>(o[e]), static_cast<double>(th[e])));
        store_vec<false>(a.theta, i, lo, hi, th);
      }
      for (int j = 0; j < a.workers; ++j) store_vec<BF16>(reps.p[j], i, lo, hi, th);
    }
  }
}

OrthoArgs args_of(const OrthoCall& c) {
  return {c.x, c.out, c.momentum, c.theta, c.u, c.rec, c.workers, c.nesterov, c.mu, c.keep, c.lr};
}

RepPtrs reps_of(const OrthoCall& c) {
  RepPtrs r = {};
  for (int j = 0; j < c.workers; ++j) r.p[j] = c.reps[j];
  return r;
}

template <int PRODUCT, bool FULL, int BM, int BN, int WM, int WN, int BK>
hipError_t launch_product(const OrthoMat* mats, const OrthoTiles& tiles, const ProductArgs& args, float* out,
                          hipStream_t stream) {
  using S = ProductShape<PRODUCT, FULL, BM, BN, WM, WN, BK>;
  ortho_product_kernel<PRODUCT, FULL, BM, BN, WM, WN, BK>
      <<<tiles.count, S::kThreads, 0, stream>>>(mats, tiles.tile, args, out);
  return hipGetLastError();
}

template <int PRODUCT>
hipError_t launch_product_of(bool full, const OrthoMat* mats, const OrthoTiles& tiles, const ProductArgs& args,
                             float* out, hipStream_t stream) {
  if (full) return launch_product<PRODUCT, true, 128, 128, 64, 64, 32>(mats, tiles, args, out, stream);
  return launch_product<PRODUCT, false, 128, 128, 64, 64, 64>(mats, tiles, args, out, stream);
}

}  // namespace

hipError_t launch_ortho_source(const OrthoCall& call, const OrthoMat* mats, const OrthoChunk* chunks, int count,
                               hipStream_t stream) {
  if (count == 0) return hipSuccess;
  const OrthoArgs a = args_of(call);
  const RepPtrs r = reps_of(call);
#define EDIT_SOURCE(S, B) ortho_source_kernel<S, B><<<count, kOrthoStreamThreads, 0, stream>>>(a, r, mats, chunks)
  switch (call.source) {
    case kSourcePlain: call.bf16 ? EDIT_SOURCE(kSourcePlain, true) : EDIT_SOURCE(kSourcePlain, false); break;
    case kSourceLocal: call.bf16 ? EDIT_SOURCE(kSourceLocal, true) : EDIT_SOURCE(kSourceLocal, false); break;
    case kSourceOuter: call.bf16 ? EDIT_SOURCE(kSourceOuter, true) : EDIT_SOURCE(kSourceOuter, false); break;
  }
#undef EDIT_SOURCE
  return hipGetLastError();
}

hipError_t launch_ortho_load(bool full, const OrthoCall& call, const OrthoMat* mats, const OrthoTile* tiles, int count,
                             hipStream_t stream) {
  if (count == 0) return hipSuccess;
  const OrthoArgs a = args_of(call);
#define EDIT_LOAD(S, B)                                                                            \
  (full ? ortho_load_kernel<S, B, true><<<count, kOrthoStreamThreads, 0, stream>>>(a, mats, tiles) \
        : ortho_load_kernel<S, B, false><<<count, kOrthoStreamThreads, 0, stream>>>(a, mats, tiles))
  switch (call.source) {
    case kSourcePlain: call.bf16 ? EDIT_LOAD(kSourcePlain, true) : EDIT_LOAD(kSourcePlain, false); break;
    case kSourceLocal: call.bf16 ? EDIT_LOAD(kSourceLocal, true) : EDIT_LOAD(kSourceLocal, false); break;
    case kSourceOuter: EDIT_LOAD(kSourceOuter, false); break;  // u is fp32
  }
#undef EDIT_LOAD
  return hipGetLastError();
}

hipError_t launch_ortho_product(OrthoProduct product, bool full, int side, const OrthoMat* mats, const OrthoTiles& tiles,
                                const OrthoCoef& coef, int from, bool first, bool last, float* u, hipStream_t stream) {
  if (tiles.count == 0) return hipSuccess;
  if (side != 128) return hipErrorInvalidValue;
  const ProductArgs args = {coef.a, coef.b, coef.c, from, first, last};
  switch (product) {
    case kProductGram: return launch_product_of<kProductGram>(full, mats, tiles, args, u, stream);
    case kProductSquare: return launch_product_of<kProductSquare>(full, mats, tiles, args, u, stream);
    case kProductUpdate: return launch_product_of<kProductUpdate>(full, mats, tiles, args, u, stream);
  }
  return hipErrorInvalidValue;
}

hipError_t launch_ortho_apply(const OrthoCall& call, const OrthoMat* mats, const OrthoChunk* chunks, int count,
                              hipStream_t stream) {
  if (count == 0) return hipSuccess;
  const OrthoArgs a = args_of(call);
  const RepPtrs r = reps_of(call);
#define EDIT_APPLY(S, B) ortho_apply_kernel<S, B><<<count, kOrthoStreamThreads, 0, stream>>>(a, r, mats, chunks)
  switch (call.source) {
    case kSourcePlain: call.bf16 ? EDIT_APPLY(kSourcePlain, true) : EDIT_APPLY(kSourcePlain, false); break;
    case kSourceLocal: call.bf16 ? EDIT_APPLY(kSourceLocal, true) : EDIT_APPLY(kSourceLocal, false); break;
    case kSourceOuter: call.bf16 ? EDIT_APPLY(kSourceOuter, true) : EDIT_APPLY(kSourceOuter, false); break;
  }
#undef EDIT_APPLY
  return hipGetLastError();
}

}  // namespace edit
