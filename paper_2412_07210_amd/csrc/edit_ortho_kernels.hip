// Device kernels of the orthogonalised updates.
//
// For every matrix of a unit, with r = min(rows, cols), c = max(rows, cols)
// and the working matrix X [r][c] (the stored one, or its transpose):
//
//   source   u of the call (the update itself; a worker's momentum step; the
//            outer step's Nesterov direction) and its sums of squares
//   load     X = u / ||u||_F
//   gram     A = X X^T               } steps times, each a launch over the
//   square   F = a I + b A + c A^2   } tiles of all matrices
//   update   X <- F X                }
//   apply    the call's outputs from O = X
//
// Numerics.  The products run on the fp16 matrix cores with fp32 sums.  Two
// things keep them near 32 bits of X at that price:
//  * X is held to 22 bits as the sum of two fp16 values (high + low).  A
//    product takes the high halves (EDIT_ORTHO_FAST), and the low half of X
//    enters the next X times F's mean diagonal; or it takes high*high +
//    high*low + low*high (EDIT_ORTHO_FULL).
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

// How the halves of a matrix lie in memory.  The 128 bytes of a cache line are
// what one row of a slab takes, so that a load asks the L2 for whole lines:
//   FAST  high and low halves in arrays of their own, 64 high ones a line
//   FULL  one array, 32 columns' high halves and then their low ones a line
template <bool FULL>
struct Layout {
  __device__ static int64_t pitch(int ld) { return FULL ? 2 * static_cast<int64_t>(ld) : ld; }
  __device__ static int64_t at(int row, int col, int ld) {  // of a high half; the low one: see low()
    return row * pitch(ld) + (FULL ? 2 * (col & ~31) + (col & 31) : col);
  }
  template <typename T>
  __device__ static T* low(T* hi, T* lo) {  // the array of low halves
    return FULL ? hi + 32 : lo;
  }
};

// A pointer read from a table, which the compiler would take for one to any
// memory (and wait for LDS on each use).
template <typename T>
__device__ __forceinline__ T* as_global(T* p) {
  return (T*)(__attribute__((address_space(1))) T*)p;
}

// One 64 x 64 tile of a stored matrix per block: X^T = u / ||u|| at kScaleX,
// through LDS where that transposes.
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
  using L = Layout<FULL>;
  _Float16* x_hi = as_global(mt.t[0][0]);
  _Float16* x_lo = L::low(x_hi, as_global(mt.t[0][1]));
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
      if (mt.tall) {  // X^T is the stored matrix
        const int64_t at = L::at(row, col, mt.ldr);
        x_hi[at] = hi;
        x_lo[at] = lo;
      } else {
        lds[y][tx] = __builtin_bit_cast(uint16_t, hi) | static_cast<uint32_t>(__builtin_bit_cast(uint16_t, lo)) << 16;
      }
    }
  }
  if (mt.tall) return;
  __syncthreads();
  for (int y = ty; y < T; y += kOrthoStreamThreads / 64) {
    const int col = col0 + y, row = row0 + tx;
    if (row < mt.rows && col < mt.cols) {
      const uint32_t w = lds[tx][y];
      const int64_t at = L::at(col, row, mt.ldr);
      x_hi[at] = __builtin_bit_cast(_Float16, static_cast<uint16_t>(w));
      x_lo[at] = __builtin_bit_cast(_Float16, static_cast<uint16_t>(w >> 16));
    }
  }
}

// ---------------------------------------------------------------- products

// Product C[p][q] = sum_k P[p][k] Q[q][k] over the tiles of all matrices:
//   gram    P = Q = X, read from X^T          C -> R = C - sI          (symmetric)
//   square  P = Q = R                         C -> F = (b + 2cs) R + c C, FULL: + (a + bs + cs^2) I   (symmetric)
//   update  P = F, Q = X^T                    C^T -> X^T of the next iteration
// X lives as X^T only, so an iteration reads and writes one array of the
// matrix's size: the gram product reads its operands across the rows of LDS
// (the transposing LDS reads of gfx950).  The term (a + bs + cs^2) X is part of
// F X with FULL; with FAST F's diagonal would round it to 11 bits, so the
// update product takes it from the operand tiles as they pass through LDS, and
// the low half of X in its epilogue.  Symmetric products take the tiles with
// p >= q and store each twice.
struct ProductArgs {
  double a, b, c;
  int32_t from, first, last;
};

// LDS holds two slabs of both operands: 64 values of k (FAST), or 32 with both
// halves (FULL); 128 bytes for each of the operands' rows either way.
template <bool FULL, int BP, int BQ, int WP, int WQ>
struct ProductShape {
  static constexpr int kSlabK = FULL ? 32 : 64;
  static constexpr int kWaves = (BP / WP) * (BQ / WQ);
  static constexpr int kThreads = kWaves * 64;
  static constexpr int kBytesP = BP * 128, kBytesQ = BQ * 128;
  static constexpr int kSlab = kBytesP + kBytesQ;
  static constexpr int kLoadsP = kBytesP / 1024 / kWaves;  // of a wave, 1 KB each
  static constexpr int kLoadsQ = kBytesQ / 1024 / kWaves;
  static_assert(kLoadsP * kWaves * 1024 == kBytesP && kLoadsQ * kWaves * 1024 == kBytesQ, "whole loads");
  static_assert(kOrthoPad % kSlabK == 0, "whole slabs");
  static_assert(2 * kSlab <= 160 * 1024 - 256, "two slabs, and the sums of block_sum");
  static_assert(!FULL || WP >= WQ, "the order of the reads");
};

// How an operand lies in a slab and is read from it: 16 lanes at a time, lane l
// for row `side` + l of the tile unless said otherwise.
enum Reading {
  kAlong,   // an operand's row is a slab row: a lane reads 16 bytes of it
  kBlocks,  // the same, lane l for row side + 8 (l / 4) + l mod 4: with side + 4,
            // a lane of the product's results gets eight neighbours of a column
  kAcross,  // a value of k is a slab row: four lanes read 32 bytes of it, and the
            // 16 lanes exchange theirs (the transposing read of gfx950)
};

// A slab's rows of 16-byte chunks are permuted within a row by its number, so
// that what a wave reads in one cycle (256 bytes) lies in different banks.
template <Reading READING, int CHUNKS>
__device__ __forceinline__ int chunk_swizzle(int row, int chunk) {
  if constexpr (READING == kAlong) return chunk ^ ((row >> 1) & 7);  // 16 rows from a multiple of 16 on
  if constexpr (READING == kBlocks) return chunk ^ (((row >> 1) & 1) | ((row >> 2) & 6));
  // rows 0..3 and 8..11, or 4..7 and 12..15, of sixteen
  if constexpr (CHUNKS >= 16) return chunk ^ (((row & 3) | ((row >> 1) & 4)) << 1);
  return chunk ^ ((((row >> 1) & 1) | ((row >> 2) & 2)) << 1);
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

// The byte offsets of a lane's loads of a tile's first slab: `rows` x `ld` is
// the operand.  Rows (along k) or columns (across) past its end read the last
// ones; what they give is not stored.
template <Reading READING, bool FULL, int SIDE, int WAVES, int LOADS>
__device__ __forceinline__ void tile_offsets(uint32_t (&off)[LOADS], int side0, int rows, int ld, int wave, int lane) {
  constexpr bool ACROSS = READING == kAcross;
  constexpr int kChunks = !ACROSS ? 8 : FULL ? SIDE / 4 : SIDE / 8;
  constexpr int kRowsPerLoad = 64 / kChunks;
  const int pitch = static_cast<int>(Layout<FULL>::pitch(ld));
#pragma unroll
  for (int i = 0; i < LOADS; ++i) {
    const int row = (wave + i * WAVES) * kRowsPerLoad + lane / kChunks;
    const int chunk = chunk_swizzle<READING, kChunks>(row, lane % kChunks);
    const int g = ACROSS ? row : min(side0 + row, rows - 1);
    const int col = ACROSS ? min((FULL ? 2 * side0 : side0) + 8 * chunk, pitch - 8) : 8 * chunk;
    off[i] = (static_cast<uint32_t>(g) * static_cast<uint32_t>(pitch) + static_cast<uint32_t>(col)) * 2u;
  }
}

typedef __fp16 fp16x4 __attribute__((__vector_size__(8)));

// A lane's eight values of its row of a slab's operand: of FAST's k = 32 part +
// 8 (lane / 16) .., of FULL's k = 8 (lane / 16) .. and half `part`.
template <Reading READING, bool FULL, int SIDE>
__device__ __forceinline__ half8 read_operand(const char* slab, int side, int part, int lane) {
  if constexpr (READING == kAcross) {
    // 16 lanes give four rows of 16 values and get four values of 16 columns
    constexpr int kChunks = FULL ? SIDE / 4 : SIDE / 8;
    half8 out;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int row = (FULL ? 0 : 32 * part) + 8 * (lane >> 4) + 4 * h + ((lane & 15) >> 2);
      const int col = (side >> 3) + ((lane & 3) >> 1);  // in chunks of one half
      const int chunk = chunk_swizzle<kAcross, kChunks>(row, FULL ? 2 * (col & ~3) + 4 * part + (col & 3) : col);
      const char* at = slab + (row * kChunks + chunk) * 16 + 8 * (lane & 1);
      const half4 v = __builtin_bit_cast(
          half4, __builtin_amdgcn_ds_read_tr16_b64_v4f16((__attribute__((address_space(3))) fp16x4*)(at)));
#pragma unroll
      for (int e = 0; e < 4; ++e) out[4 * h + e] = v[e];
    }
    return out;
  } else {
    const int row = side + (READING == kBlocks ? 2 * (lane & 12) + (lane & 3) : lane & 15);
    return *reinterpret_cast<const half8*>(slab + row * 128 +
                                           chunk_swizzle<READING, 8>(row, 4 * part + (lane >> 4)) * 16);
  }
}

// All of the wave's loads into LDS have landed and its reads of LDS are done,
// for every wave of the block.  The wait is the builtin one, which the compiler
// counts: with scalar loads outstanding it could only wait for all reads of LDS
// at each use of one.
__device__ __forceinline__ void slab_barrier() {
  asm volatile("" : : : "memory");
  __builtin_amdgcn_s_waitcnt(0x0070);  // vmcnt(0) lgkmcnt(0)
  __builtin_amdgcn_s_barrier();
  asm volatile("" : : : "memory");
}

// The 4 x 4 transpose of what four neighbouring lanes hold: lane q of each
// quad gives v[e] = element (e, q) and gets (q, e).
template <int CTRL>
__device__ __forceinline__ uint32_t quad_move(uint32_t x) {
  return static_cast<uint32_t>(__builtin_amdgcn_mov_dpp(static_cast<int>(x), CTRL, 0xf, 0xf, true));
}
__device__ __forceinline__ void quad_transpose(uint32_t (&v)[4], int lane) {
  constexpr int kSwap1 = 1 | 0 << 2 | 3 << 4 | 2 << 6;  // lanes 1 0 3 2
  constexpr int kSwap2 = 2 | 3 << 2 | 0 << 4 | 1 << 6;  // lanes 2 3 0 1
  const bool odd = lane & 1, high = lane & 2;
#pragma unroll
  for (int e = 0; e < 4; e += 2) {
    const uint32_t got = quad_move<kSwap1>(odd ? v[e] : v[e + 1]);
    v[e] = odd ? got : v[e];
    v[e + 1] = odd ? v[e + 1] : got;
  }
#pragma unroll
  for (int e = 0; e < 2; ++e) {
    const uint32_t got = quad_move<kSwap2>(high ? v[e] : v[e + 2]);
    v[e] = high ? got : v[e];
    v[e + 2] = high ? v[e + 2] : got;
  }
}

// A value as its (high, low) halves in 32 bits, and four of them in two rows.
__device__ __forceinline__ uint32_t pack_split(float v) {
  _Float16 hi, lo;
  split(v, hi, lo);
  return __builtin_bit_cast(uint16_t, hi) | static_cast<uint32_t>(__builtin_bit_cast(uint16_t, lo)) << 16;
}
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
template <bool LOW>
__device__ __forceinline__ void store_split(_Float16* hi, _Float16* lo, int64_t at, const uint32_t (&v)[4]) {
  *reinterpret_cast<u32x2*>(hi + at) =
      u32x2{__builtin_amdgcn_perm(v[1], v[0], 0x05040100), __builtin_amdgcn_perm(v[3], v[2], 0x05040100)};
  if constexpr (LOW)
    *reinterpret_cast<u32x2*>(lo + at) =
        u32x2{__builtin_amdgcn_perm(v[1], v[0], 0x07060302), __builtin_amdgcn_perm(v[3], v[2], 0x07060302)};
}
__device__ __forceinline__ float join(const half4& hi, const half4& lo, int e) {
  return static_cast<float>(hi[e]) + static_cast<float>(lo[e]);
}

// One tile of a product per block.  While one slab is multiplied, the loads of
// the next are under way.  A wave's operands are read a step ahead of their
// use: each register is read anew right after its last use, and the barrier
// between slabs stands before the last step of a slab, so that the first reads
// of the next one run under that step's products.
template <int PRODUCT, bool FULL, bool LAST, int BP, int BQ, int WP, int WQ>
__global__ __launch_bounds__((ProductShape<FULL, BP, BQ, WP, WQ>::kThreads),
                             2)  // waves per SIMD that the registers are budgeted for
void ortho_product_kernel(const OrthoMat* __restrict__ mats, const OrthoTile* __restrict__ tiles, ProductArgs args,
                          float* __restrict__ out) {
  using S = ProductShape<FULL, BP, BQ, WP, WQ>;
  constexpr Reading kReadP = PRODUCT == kProductGram ? kAcross : PRODUCT == kProductUpdate ? kBlocks : kAlong;
  constexpr Reading kReadQ = PRODUCT == kProductGram ? kAcross : kAlong;
  using L = Layout<FULL>;
  __shared__ __align__(256) char smem[2 * S::kSlab];
  const OrthoTile t = tiles[blockIdx.x];
  if (t.mat < 0) return;
  const OrthoMat mt = mats[t.mat];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int r = mt.r, c = mt.c, ld = mt.ldr;

  const _Float16* x_t = args.from ? mt.t[1][0] : mt.t[0][0];
  const _Float16* q = PRODUCT == kProductSquare ? mt.g[0] : x_t;
  const _Float16* p = PRODUCT == kProductUpdate ? mt.q[0] : q;
  uint32_t off_p[S::kLoadsP], off_q[S::kLoadsQ];
  tile_offsets<kReadP, FULL, BP, S::kWaves>(off_p, t.m * BP, r, ld, wave, lane);
  tile_offsets<kReadQ, FULL, BQ, S::kWaves>(off_q, t.n * BQ, PRODUCT == kProductUpdate ? c : r, ld, wave, lane);

  const uint32_t lds0 = static_cast<uint32_t>(
      reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) char*)(smem)));  // byte offset in LDS
  const int64_t step = PRODUCT == kProductGram ? S::kSlabK * L::pitch(ld) : 64;
  const int slabs = (PRODUCT == kProductGram ? (c + kOrthoPad - 1) / kOrthoPad * kOrthoPad : ld) / S::kSlabK;
  // Slab n, or of its loads those with number part mod parts.
  auto fetch = [&](int n, int part = 0, int parts = 1) {
    const uint32_t at = lds0 + (n & 1) * S::kSlab;
    const _Float16* from_p = p + n * step;
    const _Float16* from_q = q + n * step;
#pragma unroll
    for (int i = 0; i < S::kLoadsP; ++i)
      if (i % parts == part) load_to_lds(at + (wave + i * S::kWaves) * 1024, from_p, off_p[i]);
#pragma unroll
    for (int i = 0; i < S::kLoadsQ; ++i)
      if (i % parts == part) load_to_lds(at + S::kBytesP + (wave + i * S::kWaves) * 1024, from_q, off_q[i]);
  };
  fetch(0);

  // s of this iteration: the mean of A's diagonal, ||X||^2 / r (1 / r at first)
  double s;
  if constexpr (PRODUCT == kProductGram) {
    if (args.first) {
      s = 1.0;
    } else {
      s = 0.0;
      for (int i = threadIdx.x; i < mt.x_tiles; i += S::kThreads) s += as_global(mt.x_part)[i];
      s = block_sum<S::kThreads>(s);
    }
    s /= r;
    if (t.m == 0 && t.n == 0 && threadIdx.x == 0) *as_global(mt.shift) = s;
  } else {
    s = *as_global(mt.shift);
  }
  const double keep = args.a + args.b * s + args.c * s * s;

  constexpr int FP = WP / 16, FQ = WQ / 16;
  static_assert(!FULL || FP >= FQ, "the order of the reads");
  const int wp = (wave % (BP / WP)) * WP, wq = (wave / (BP / WP)) * WQ;
  f32x4 acc[FP][FQ];
#pragma unroll
  for (int i = 0; i < FP; ++i)
#pragma unroll
    for (int j = 0; j < FQ; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};

  // The update product's results: lane l holds C^T[q][p .. p+7], q = l mod 16, p
  // = 8 (l / 16), of each pair of 16 x 16 blocks.  FAST adds X's low half to
  // them, which is read ahead of the sums.
  const int p8 = t.m * BP + wp + 8 * (lane >> 4), q0 = t.n * BQ + wq + (lane & 15);
  _Float16* to_hi = as_global(args.from ? mt.t[0][0] : mt.t[1][0]);
  _Float16* to_lo = L::low(to_hi, as_global(mt.t[0][1]));  // FAST: read and written in place
  constexpr bool kLow = PRODUCT == kProductUpdate && !FULL;
  const float keep_lo = static_cast<float>(keep);
  half8 xl[kLow ? FP / 2 : 1][kLow ? FQ : 1];
  if constexpr (kLow) {
#pragma unroll
    for (int i = 0; i < FP; i += 2)
#pragma unroll
      for (int j = 0; j < FQ; ++j)
        xl[i / 2][j] = *reinterpret_cast<const half8*>(
            to_lo + L::at(min(q0 + j * 16, c - 1), min(p8 + i * 16, ld - 8), ld));
  }

  auto slab = [&](int n) { return smem + (n & 1) * S::kSlab; };
  auto read_p = [&](const char* at, int part, int i) {
    return read_operand<kReadP, FULL, BP>(at, wp + (kReadP == kBlocks ? 16 * (i & ~1) + 4 * (i & 1) : 16 * i), part, lane);
  };
  auto read_q = [&](const char* at, int part, int j) {
    return read_operand<kReadQ, FULL, BQ>(at + S::kBytesP, wq + j * 16, part, lane);
  };
  auto mul = [&](const half8& x, const half8& y, f32x4& to) {
    to = __builtin_amdgcn_mfma_f32_16x16x32_f16(x, y, to, 0, 0, 0);
  };
  // Slab n + 1 has landed, and slab n is read: slab n + 2 takes its place.
  auto next_slab = [&](int n) {
    slab_barrier();
    if (n + 2 < slabs) fetch(n + 2);
  };

  slab_barrier();
  if (slabs > 1) fetch(1);
  if constexpr (!FULL) {
    half8 pf[FP], qf[2][FQ];
#pragma unroll
    for (int j = 0; j < FQ; ++j) qf[0][j] = read_q(slab(0), 0, j);
#pragma unroll
    for (int i = 0; i < FP; ++i) pf[i] = read_p(slab(0), 0, i);
    const int own0 = t.m * BP + wp;
    const float keep_hi = static_cast<float>(keep) * kScaleA;
    for (int n = 0; n < slabs; ++n) {
      const char* at = slab(n);
      if constexpr (PRODUCT == kProductUpdate) {
        // This slab holds X^T at p = 64 n .. of all q: where that is the wave's
        // own part of C, the term (a + bs + cs^2) X of the high half goes in.
        const int d = 64 * n - own0;
        if (d > -64 && d < WP) {
#pragma unroll
          for (int i = 0; i < FP; ++i) {
            const int in_slab = 16 * (i & ~1) - d;  // of a pair's 32 values of p
            if (in_slab >= 0 && in_slab < 64)
#pragma unroll
              for (int j = 0; j < FQ; ++j) {
                const int row = wq + j * 16 + (lane & 15);
                const int chunk = chunk_swizzle<kReadQ, 8>(row, (in_slab >> 3) + (lane >> 4));
                const half4 x = *reinterpret_cast<const half4*>(at + S::kBytesP + row * 128 + chunk * 16 + 8 * (i & 1));
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[i][j][e] += keep_hi * static_cast<float>(x[e]);
              }
          }
        }
      }
#pragma unroll
      for (int kk = 0; kk < 2; ++kk) {
        if (kk == 1) next_slab(n);
        const char* next = kk == 0 ? at : slab(n + 1);  // behind the last one: read, not used
#pragma unroll
        for (int j = 0; j < FQ; ++j) qf[kk ^ 1][j] = read_q(next, kk ^ 1, j);
#pragma unroll
        for (int i = 0; i < FP; ++i) {
#pragma unroll
          for (int j = 0; j < FQ; ++j) mul(pf[i], qf[kk][j], acc[i][j]);
          pf[i] = read_p(next, kk ^ 1, i);
          __builtin_amdgcn_sched_barrier(0);
        }
      }
    }
  } else {
    half8 ph[FP], qh[FQ], pl[FP], ql[FQ];
#pragma unroll
    for (int j = 0; j < FQ; ++j) qh[j] = read_q(slab(0), 0, j);
#pragma unroll
    for (int i = 0; i < FP; ++i) ph[i] = read_p(slab(0), 0, i);
    for (int n = 0; n < slabs; ++n) {
      const char* at = slab(n);
#pragma unroll
      for (int i = 0; i < FP; ++i) {
        pl[i] = read_p(at, 1, i);
        if (i < FQ) ql[i] = read_q(at, 1, i);
#pragma unroll
        for (int j = 0; j < FQ; ++j) mul(ph[i], qh[j], acc[i][j]);
        __builtin_amdgcn_sched_barrier(0);
      }
#pragma unroll
      for (int i = 0; i < FP; ++i) {
#pragma unroll
        for (int j = 0; j < FQ; ++j) mul(pl[i], qh[j], acc[i][j]);
        __builtin_amdgcn_sched_barrier(0);
      }
      next_slab(n);
      const char* next = slab(n + 1);  // behind the last one: read, not used
#pragma unroll
      for (int j = 0; j < FQ; ++j) qh[j] = read_q(next, 0, j);
#pragma unroll
      for (int i = 0; i < FP; ++i) {
#pragma unroll
        for (int j = 0; j < FQ; ++j) mul(ph[i], ql[j], acc[i][j]);
        ph[i] = read_p(next, 0, i);
        __builtin_amdgcn_sched_barrier(0);
      }
    }
  }

  // Values behind the matrix become the zeros that its padding holds anyway.
  if constexpr (PRODUCT != kProductUpdate) {
    // Lane l holds C[p .. p+3][q] of each 16 x 16 block, p = 4 (l / 16), q = l mod 16.
    const int p0 = t.m * BP + wp + 4 * (lane >> 4);
    const int quad = lane & 3;
    const _Float16* r_hi = as_global(mt.g[0]);
    const _Float16* r_lo = L::low(r_hi, as_global<const _Float16>(mt.g[1]));
    _Float16* dst_hi = as_global(PRODUCT == kProductGram ? mt.g[0] : mt.q[0]);
    _Float16* dst_lo = L::low(dst_hi, as_global(mt.g[1]));  // the square product's only with FULL
    // F's low half goes into products only, R's into F as well
    constexpr bool kStoreLow = PRODUCT == kProductGram || FULL;
    // with FAST the update product adds the diagonal term itself, unrounded
    const float diag = PRODUCT == kProductGram ? static_cast<float>(-s * kScaleA)
                       : FULL                  ? static_cast<float>(keep * kScaleA)
                                               : 0.f;
    const float lin = static_cast<float>(args.b + 2.0 * args.c * s);
    const float quadratic = static_cast<float>(args.c) / kScaleA;
    half4 rh[2][FQ], rl[2][FQ];  // R, a row of blocks ahead
    auto read_r = [&](int i) {
#pragma unroll
      for (int j = 0; j < FQ; ++j) {  // R is symmetric
        const int64_t from = L::at(min(q0 + j * 16, r - 1), min(p0 + i * 16, ld - 4), ld);
        rh[i & 1][j] = *reinterpret_cast<const half4*>(r_hi + from);
        rl[i & 1][j] = *reinterpret_cast<const half4*>(r_lo + from);
      }
    };
    if constexpr (PRODUCT == kProductSquare) read_r(0);
#pragma unroll
    for (int i = 0; i < FP; ++i) {
      const int pp = p0 + i * 16;
      if constexpr (PRODUCT == kProductSquare)
        if (i + 1 < FP) read_r(i + 1);
#pragma unroll
      for (int j = 0; j < FQ; ++j) {
        const int qq = q0 + j * 16;
        uint32_t w[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          float v;
          if constexpr (PRODUCT == kProductGram)
            v = acc[i][j][e] * (kScaleA / (kScaleX * kScaleX));
          else
            v = lin * join(rh[i & 1][j], rl[i & 1][j], e) + quadratic * acc[i][j][e];
          if (pp + e == qq) v += diag;
          w[e] = pack_split(pp + e < r && qq < r ? v : 0.f);
        }
        if (qq < r && pp < r) store_split<kStoreLow>(dst_hi, dst_lo, L::at(qq, pp, ld), w);
        if (t.m != t.n) {
          quad_transpose(w, lane);  // C[p + l mod 4][q - l mod 4 .. + 3]
          if (pp + quad < r && qq - quad < r) store_split<kStoreLow>(dst_hi, dst_lo, L::at(pp + quad, qq - quad, ld), w);
        }
      }
    }
  } else {
    float sq = 0.f;
#pragma unroll
    for (int j = 0; j < FQ; ++j) {
      const int qq = q0 + j * 16;
#pragma unroll
      for (int i = 0; i < FP; i += 2) {
        const int pp = p8 + i * 16;  // X^T[q][p .. p+7]
        float v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          v[e] = acc[i + (e >> 2)][j][e & 3] * (1.f / kScaleA);
          if constexpr (!FULL) v[e] += keep_lo * static_cast<float>(xl[i / 2][j][e]);
          if (!(pp + e < r && qq < c)) v[e] = 0.f;
        }
        if constexpr (LAST) {
#pragma unroll
          for (int e = 0; e < 8; ++e)
            if (pp + e < r && qq < c) {
              const int64_t o = mt.tall ? static_cast<int64_t>(qq) * mt.cols + pp + e
                                        : static_cast<int64_t>(pp + e) * mt.cols + qq;
              out[mt.offset + o] = v[e] * (1.f / kScaleX);
            }
        } else {
          half8 hi, lo;
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            sq += v[e] * v[e];
            _Float16 h, l;
            split(v[e], h, l);
            hi[e] = h, lo[e] = l;
          }
          if (qq < c && pp < r) {
            const int64_t at = L::at(qq, pp, ld);
            *reinterpret_cast<half8*>(to_hi + at) = hi;
            *reinterpret_cast<half8*>(to_lo + at) = lo;
          }
        }
      }
    }
    if constexpr (!LAST) {
      const double sum = block_sum<S::kThreads>(static_cast<double>(sq) / (static_cast<double>(kScaleX) * kScaleX));
      if (threadIdx.x == 0) as_global(mt.x_part)[t.slot] = sum;
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

// ----------------------------------------------------------- small matrices

// The whole call for one matrix per block, where X and A fit into LDS
// (ortho_is_small): no launch between the products, whose latency bounds
// matrices of this size.  LDS holds X^T [c][r] and R, then F, [r][r], high and
// low halves apart, in rows of r rounded up to 32 values and eight more (rows
// then begin in different banks); what pads them is zero.  Wave w takes the
// 16 rows 16 w .. of the symmetric products, all columns, so that R and F stay
// in its registers as well, and rows 16 w + 128 t of X^T.
struct SmallCoef {
  double v[EDIT_ORTHO_MAX_STEPS][3];
};

// O of one element into the call's outputs.
template <int SOURCE, bool BF16>
__device__ __forceinline__ void apply_one(const OrthoArgs& a, const RepPtrs& reps, double step, bool rollback, int64_t i,
                                          float o) {
  if constexpr (SOURCE == kSourcePlain) {
    store_one<BF16>(a.out, i, o);
  } else if constexpr (SOURCE == kSourceLocal) {
    const double p = load_one<BF16>(a.out, i);
    store_one<BF16>(a.out, i, static_cast<float>(fma(a.keep, p, -step * static_cast<double>(o))));
  } else {
    float th = a.theta[i];
    if (!rollback) {
      th = static_cast<float>(fma(-step, static_cast<double>(o), static_cast<double>(th)));
      a.theta[i] = th;
    }
    for (int j = 0; j < a.workers; ++j) store_one<BF16>(reps.p[j], i, th);
  }
}

template <int SOURCE, bool BF16, bool FULL>
__global__ __launch_bounds__(kOrthoSmallThreads) void ortho_small_kernel(OrthoArgs a, RepPtrs reps,
                                                                        const OrthoMat* __restrict__ mats,
                                                                        SmallCoef coef, int steps) {
  constexpr int kThreads = kOrthoSmallThreads;
  constexpr int kBlocks = kOrthoSmallSide / 16;                // of a row of A
  constexpr int kRows = kOrthoSmallRows / 16 / (kThreads / 64);  // blocks of X^T's rows per wave
  __shared__ __align__(256) char smem[kOrthoSmallLds];
  const OrthoMat mt = mats[blockIdx.x];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int r = mt.r, c = mt.c, rp = (r + 31) & ~31, cp = (c + 31) & ~31;
  const int pitch = rp + 8;
  _Float16* x_hi = reinterpret_cast<_Float16*>(smem);
  _Float16* x_lo = x_hi + cp * pitch;
  _Float16* g_hi = x_lo + cp * pitch;
  _Float16* g_lo = g_hi + rp * pitch;
  const int64_t n = static_cast<int64_t>(r) * c;

  // u, its norm, and X^T = u / ||u||
  auto update_of = [&](int64_t i) -> double {
    if constexpr (SOURCE == kSourcePlain) return load_one<BF16>(a.x, i);
    if constexpr (SOURCE == kSourceOuter) return a.u[i];
    const double m = a.momentum[i];
    return a.nesterov ? fma(a.mu, m, static_cast<double>(load_one<BF16>(a.x, i))) : m;
  };
  for (int i = threadIdx.x; i < 2 * (cp + rp) * pitch / 8; i += kThreads)
    reinterpret_cast<u32x4*>(smem)[i] = u32x4{0, 0, 0, 0};
  double sum = 0.0;
  for (int64_t e = threadIdx.x; e < n; e += kThreads) {
    const int64_t i = mt.offset + e;
    if constexpr (SOURCE == kSourceLocal)
      a.momentum[i] = static_cast<float>(fma(a.mu, static_cast<double>(a.momentum[i]), static_cast<double>(load_one<BF16>(a.x, i))));
    const double u = update_of(i);
    sum = fma(u, u, sum);
  }
  sum = block_sum<kThreads>(sum);
  const double inv = sum > 0.0 ? kScaleX / sqrt(sum) : (sum == 0.0 ? 0.0 : sum);
  for (int e = threadIdx.x; e < n; e += kThreads) {
    const int row = e / mt.cols, col = e - row * mt.cols;
    _Float16 hi, lo;
    split(static_cast<float>(update_of(mt.offset + e) * inv), hi, lo);
    const int at = mt.tall ? row * pitch + col : col * pitch + row;
    x_hi[at] = hi, x_lo[at] = lo;
  }
  __syncthreads();

  const int blocks = rp / 16;
  const int l16 = lane & 15, l4 = lane >> 4;
  // eight values along k of row `row0` + l16
  auto along = [&](const _Float16* m, int row0, int k) {
    return *reinterpret_cast<const half8*>(m + (row0 + l16) * pitch + k + 8 * l4);
  };
  // eight rows from `k` + 8 l4 on of column `col0` + l16
  auto across = [&](const _Float16* m, int col0, int k) {
    half8 out;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const _Float16* at = m + (k + 8 * l4 + 4 * h + (l16 >> 2)) * pitch + col0 + 4 * (l16 & 3);
      const half4 v = __builtin_bit_cast(
          half4, __builtin_amdgcn_ds_read_tr16_b64_v4f16((__attribute__((address_space(3))) fp16x4*)(at)));
#pragma unroll
      for (int e = 0; e < 4; ++e) out[4 * h + e] = v[e];
    }
    return out;
  };
  auto mul = [&](const half8& x, const half8& y, f32x4& to) {
    to = __builtin_amdgcn_mfma_f32_16x16x32_f16(x, y, to, 0, 0, 0);
  };
  // four neighbours of row `row`, high and low halves
  auto put = [&](_Float16* hi, _Float16* lo, int row, int col, const f32x4& v) {
    half4 h, l;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      _Float16 x, y;
      split(v[e], x, y);
      h[e] = x, l[e] = y;
    }
    *reinterpret_cast<half4*>(hi + row * pitch + col) = h;
    *reinterpret_cast<half4*>(lo + row * pitch + col) = l;
  };

  float* o = reinterpret_cast<float*>(smem);  // [c][pitch], over both halves of X^T
  double s = 1.0 / r;
  for (int k = 0; k < steps; ++k) {
    const double ca = coef.v[k][0], cb = coef.v[k][1], cc = coef.v[k][2];
    const double keep = ca + cb * s + cc * s * s;
    const int p0 = 16 * wave;
    f32x4 g[kBlocks];  // lane l: [p0 + l16][16 j + 4 l4 ..], R and then F
#pragma unroll
    for (int j = 0; j < kBlocks; ++j) g[j] = f32x4{0.f, 0.f, 0.f, 0.f};
    if (wave < blocks) {
      for (int t = 0; t < cp; t += 32) {
        const half8 q = across(x_hi, p0, t);
        half8 ql;
        if constexpr (FULL) ql = across(x_lo, p0, t);
#pragma unroll
        for (int j = 0; j < kBlocks; ++j) {
          if (j >= blocks) continue;
          const half8 p = across(x_hi, 16 * j, t);
          mul(p, q, g[j]);
          if constexpr (FULL) {
            mul(p, ql, g[j]);
            mul(across(x_lo, 16 * j, t), q, g[j]);
          }
        }
      }
#pragma unroll
      for (int j = 0; j < kBlocks; ++j) {
        if (j >= blocks) continue;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int p = 16 * j + 4 * l4 + e;
          g[j][e] *= kScaleA / (kScaleX * kScaleX);
          // behind the matrix R stays zero, and F with it
          if (p == p0 + l16 && p < r) g[j][e] -= static_cast<float>(s * kScaleA);
        }
        put(g_hi, g_lo, p0 + l16, 16 * j + 4 * l4, g[j]);
      }
    }
    __syncthreads();
    f32x4 f[kBlocks];
#pragma unroll
    for (int j = 0; j < kBlocks; ++j) f[j] = f32x4{0.f, 0.f, 0.f, 0.f};
    if (wave < blocks)
      for (int t = 0; t < rp; t += 32) {
        const half8 q = along(g_hi, p0, t);
        half8 ql;
        if constexpr (FULL) ql = along(g_lo, p0, t);
#pragma unroll
        for (int j = 0; j < kBlocks; ++j) {
          if (j >= blocks) continue;
          const half8 p = along(g_hi, 16 * j, t);
          mul(p, q, f[j]);
          if constexpr (FULL) {
            mul(p, ql, f[j]);
            mul(along(g_lo, 16 * j, t), q, f[j]);
          }
        }
      }
    __syncthreads();
    if (wave < blocks) {
      const float lin = static_cast<float>(cb + 2.0 * cc * s), quadratic = static_cast<float>(cc) / kScaleA;
#pragma unroll
      for (int j = 0; j < kBlocks; ++j) {
        if (j >= blocks) continue;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          f[j][e] = lin * g[j][e] + quadratic * f[j][e];
          if (FULL && 16 * j + 4 * l4 + e == p0 + l16) f[j][e] += static_cast<float>(keep * kScaleA);
        }
        put(g_hi, g_lo, p0 + l16, 16 * j + 4 * l4, f[j]);
      }
    }
    __syncthreads();
    f32x4 x[kRows][kBlocks];  // lane l: X^T[16 (wave + 8 t) + l16][16 j + 4 l4 ..]
    const float keep_x = static_cast<float>(keep) * kScaleA;
#pragma unroll
    for (int t = 0; t < kRows; ++t) {
      const int q0 = 16 * (wave + t * (kThreads / 64));
      if (q0 >= cp) continue;
#pragma unroll
      for (int j = 0; j < kBlocks; ++j) {
        x[t][j] = f32x4{0.f, 0.f, 0.f, 0.f};
        if (j >= blocks || FULL) continue;
        // with FAST the term (a + bs + cs^2) X is taken from both halves as they are
        const int at = (q0 + l16) * pitch + 16 * j + 4 * l4;
        const half4 h = *reinterpret_cast<const half4*>(x_hi + at), l = *reinterpret_cast<const half4*>(x_lo + at);
#pragma unroll
        for (int e = 0; e < 4; ++e) x[t][j][e] = keep_x * join(h, l, e);
      }
      for (int kk = 0; kk < rp; kk += 32) {
        const half8 q = along(x_hi, q0, kk);
        half8 ql;
        if constexpr (FULL) ql = along(x_lo, q0, kk);
#pragma unroll
        for (int j = 0; j < kBlocks; ++j) {
          if (j >= blocks) continue;
          const half8 p = along(g_hi, 16 * j, kk);
          mul(p, q, x[t][j]);
          if constexpr (FULL) {
            mul(p, ql, x[t][j]);
            mul(along(g_lo, 16 * j, kk), q, x[t][j]);
          }
        }
      }
    }
    __syncthreads();
    float sq = 0.f;
#pragma unroll
    for (int t = 0; t < kRows; ++t) {
      const int q0 = 16 * (wave + t * (kThreads / 64));
      if (q0 >= cp) continue;
#pragma unroll
      for (int j = 0; j < kBlocks; ++j) {
        if (j >= blocks) continue;
        const int q = q0 + l16, p = 16 * j + 4 * l4;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          x[t][j][e] *= 1.f / kScaleA;
          if (!(p + e < r && q < c)) x[t][j][e] = 0.f;  // a NaN in the matrix would reach the padding
          sq += x[t][j][e] * x[t][j][e];
        }
        if (k + 1 < steps)
          put(x_hi, x_lo, q, p, x[t][j]);
        else  // O, where X^T was
          *reinterpret_cast<f32x4*>(o + q * pitch + p) = x[t][j];
      }
    }
    if (k + 1 < steps)
      s = block_sum<kThreads>(static_cast<double>(sq) / (static_cast<double>(kScaleX) * kScaleX)) / r;
  }
  __syncthreads();
  bool rollback = false;
  if constexpr (SOURCE == kSourceOuter) rollback = a.rec->rollback;
  const double step = a.lr * mt.scale;
  for (int e = threadIdx.x; e < n; e += kThreads) {
    const int row = e / mt.cols, col = e - row * mt.cols;
    apply_one<SOURCE, BF16>(a, reps, step, rollback, mt.offset + e,
                            o[mt.tall ? row * pitch + col : col * pitch + row] * (1.f / kScaleX));
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

template <int PRODUCT, bool FULL, int BP, int BQ, int WP, int WQ>
hipError_t launch_product(const OrthoMat* mats, const OrthoTiles& tiles, const ProductArgs& args, float* out,
                          hipStream_t stream) {
  using S = ProductShape<FULL, BP, BQ, WP, WQ>;
  if (PRODUCT == kProductUpdate && args.last)
    ortho_product_kernel<PRODUCT, FULL, PRODUCT == kProductUpdate, BP, BQ, WP, WQ>
        <<<tiles.count, S::kThreads, 0, stream>>>(mats, tiles.tile, args, out);
  else
    ortho_product_kernel<PRODUCT, FULL, false, BP, BQ, WP, WQ>
        <<<tiles.count, S::kThreads, 0, stream>>>(mats, tiles.tile, args, out);
  return hipGetLastError();
}

template <int PRODUCT, bool FULL>
hipError_t launch_product_of(int side, const OrthoMat* mats, const OrthoTiles& tiles, const ProductArgs& args,
                             float* out, hipStream_t stream) {
  if (side == 128) return launch_product<PRODUCT, FULL, 128, 128, 64, 64>(mats, tiles, args, out, stream);
  if (side == 64) return launch_product<PRODUCT, FULL, 64, 64, 32, 32>(mats, tiles, args, out, stream);
  return hipErrorInvalidValue;
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
  const ProductArgs args = {coef.a, coef.b, coef.c, from, first, last};
#define EDIT_PRODUCT(P)                                                        \
  (full ? launch_product_of<P, true>(side, mats, tiles, args, u, stream) \
        : launch_product_of<P, false>(side, mats, tiles, args, u, stream))
  switch (product) {
    case kProductGram: return EDIT_PRODUCT(kProductGram);
    case kProductSquare: return EDIT_PRODUCT(kProductSquare);
    case kProductUpdate: return EDIT_PRODUCT(kProductUpdate);
  }
#undef EDIT_PRODUCT
  return hipErrorInvalidValue;
}

hipError_t launch_ortho_small(bool full, const OrthoCall& call, const OrthoMat* mats, int count, const OrthoCoef* coef,
                              int steps, hipStream_t stream) {
  if (count == 0) return hipSuccess;
  const OrthoArgs a = args_of(call);
  const RepPtrs r = reps_of(call);
  SmallCoef sc = {};
  for (int k = 0; k < steps; ++k) sc.v[k][0] = coef[k].a, sc.v[k][1] = coef[k].b, sc.v[k][2] = coef[k].c;
#define EDIT_SMALL(S, B)                                                                                  \
  (full ? ortho_small_kernel<S, B, true><<<count, kOrthoSmallThreads, 0, stream>>>(a, r, mats, sc, steps) \
        : ortho_small_kernel<S, B, false><<<count, kOrthoSmallThreads, 0, stream>>>(a, r, mats, sc, steps))
  switch (call.source) {
    case kSourcePlain: call.bf16 ? EDIT_SMALL(kSourcePlain, true) : EDIT_SMALL(kSourcePlain, false); break;
    case kSourceLocal: call.bf16 ? EDIT_SMALL(kSourceLocal, true) : EDIT_SMALL(kSourceLocal, false); break;
    case kSourceOuter: call.bf16 ? EDIT_SMALL(kSourceOuter, true) : EDIT_SMALL(kSourceOuter, false); break;
  }
#undef EDIT_SMALL
  return hipGetLastError();
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
