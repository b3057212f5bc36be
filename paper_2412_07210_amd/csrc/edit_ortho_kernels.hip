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
//
// The last step's update product makes the call's outputs from O = X.
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
// Error of O against 64 bits, of its norm: 2e-4 to 2e-3 with FAST over
// Gaussian, low-rank (over noise) and power-law spectra of 64 rows and more (1e-3
// to 4e-2 if X itself were rounded to fp16, 1e-2 to 9e-2 in bf16); with FULL 0.6
// to 1.7 times an fp32 iteration's (1024 x 1024 Gaussian 1.7e-6 for its 3.1e-6).  Directions that X lacks gather noise, which grows by a = 3.4 a
// step: with FAST F (X - X_high) is left out, and F is -(bs + cs^2) I there, s
// = ||X||^2 / r; so an exact low rank is off by up to 5e-3, and by up to 0.25 / r
// of fewer than 64 rows (rank 1 of 512 x 512 1.2e-3, of 8 x 8 2e-2; without X's
// low half 0.15); with FULL 512 x 512 of rank 1 by 1.2e-4.
#include <type_traits>

#include "edit_ortho_device.h"

namespace edit {
namespace {

// ------------------------------------------------------------- source pass

// One chunk per block: the call's update u, its sum of squares, and what the
// call stores on the way (the momentum; the outer step's u, and the whole
// step of elements that belong to no matrix).  Bound by memory: a 1B layer's
// local step in bf16 (10 bytes an element) 94 us, 5.5 TB/s; its outer step of
// eight fp32 replicas (48 bytes) 527 us, 4.7 TB/s.
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
// through LDS where that transposes.  Eight elements a thread and access, also
// where matrices begin at odd places (then element by element).  Bound by memory:
// a 1B layer's local step in bf16 (10 bytes an element) 106 us, 4.9 TB/s.
template <int SOURCE, bool BF16, bool FULL>
__global__ __launch_bounds__(kOrthoStreamThreads) void ortho_load_kernel(OrthoArgs a, const OrthoMat* __restrict__ mats,
                                                                        const OrthoTile* __restrict__ tiles) {
  using L = Layout<FULL>;
  constexpr int T = kOrthoLoadTile;
  constexpr int kRuns = T / kVec;                          // of a row
  constexpr int kPasses = T * kRuns / kOrthoStreamThreads;
  __shared__ uint32_t lds[T][T + 1];  // high half in the low 16 bits
  const OrthoTile t = tiles[blockIdx.x];
  const OrthoMat mt = mats[t.mat];
  const int run = threadIdx.x % kRuns, line = threadIdx.x / kRuns;
  const int row0 = t.m * T, col0 = t.n * T;
  const bool vectors = (mt.offset | mt.cols) % kVec == 0;

  float x[kPasses][kVec], m[SOURCE == kSourceLocal ? kPasses : 1][kVec];
#pragma unroll
  for (int k = 0; k < kPasses; ++k) {
    const int row = row0 + line + k * (kOrthoStreamThreads / kRuns), col = col0 + run * kVec;
    const int count = row < mt.rows ? min(mt.cols - col, kVec) : 0;
    const int64_t i = mt.offset + static_cast<int64_t>(row) * mt.cols + col;
    auto read = [&](const void* from, auto bf16, float (&to)[kVec]) {
      constexpr bool B = decltype(bf16)::value;
      if (vectors && count > 0) {
        load_vec<B>(from, i, 0, kVec, to);
      } else {
#pragma unroll
        for (int e = 0; e < kVec; ++e) to[e] = e < count ? load_one<B>(from, i + e) : 0.f;
      }
    };
    if constexpr (SOURCE == kSourceOuter)
      read(a.u, std::false_type(), x[k]);
    else
      read(a.x, std::integral_constant<bool, BF16>(), x[k]);
    if constexpr (SOURCE == kSourceLocal) read(a.momentum, std::false_type(), m[k]);
  }

  double sum = 0.0;
  for (int i = threadIdx.x; i < mt.chunks; i += kOrthoStreamThreads) sum += as_global(mt.norm_part)[i];
  sum = block_sum<kOrthoStreamThreads>(sum);
  // sums of squares of fp32 values neither overflow nor vanish in fp64, nor does their root's inverse
  const double inv = sum > 0.0 ? kScaleX / sqrt(sum) : (sum == 0.0 ? 0.0 : sum);
  _Float16* x_hi = as_global(mt.t[0][0]);
  _Float16* x_lo = L::low(x_hi, as_global(mt.t[0][1]));
  // eight neighbours of a row of X^T; zeros behind r, as its padding
  auto write = [&](int q, int p, const half8& hi, const half8& lo) {
    if (q >= mt.c || p >= mt.ldr) return;
    const int64_t at = L::at(q, p, mt.ldr);
    *reinterpret_cast<half8*>(x_hi + at) = hi;
    *reinterpret_cast<half8*>(x_lo + at) = lo;
  };
#pragma unroll
  for (int k = 0; k < kPasses; ++k) {
    const int y = line + k * (kOrthoStreamThreads / kRuns);
    half8 hi, lo;
#pragma unroll
    for (int e = 0; e < kVec; ++e) {
      double u = x[k][e];
      if constexpr (SOURCE == kSourceLocal)
        u = a.nesterov ? fma(a.mu, static_cast<double>(m[k][e]), u) : static_cast<double>(m[k][e]);
      _Float16 h, l;
      split(static_cast<float>(u * inv), h, l);
      // a NaN of the norm stays out of the padding
      const bool in = row0 + y < mt.rows && col0 + run * kVec + e < mt.cols;
      hi[e] = in ? h : _Float16(0), lo[e] = in ? l : _Float16(0);
      if (!mt.tall)
        lds[y][run * kVec + e] = __builtin_bit_cast(uint16_t, _Float16(hi[e])) |
                                 static_cast<uint32_t>(__builtin_bit_cast(uint16_t, _Float16(lo[e]))) << 16;
    }
    if (mt.tall) write(row0 + y, col0 + run * kVec, hi, lo);  // X^T is the stored matrix
  }
  if (mt.tall) return;
  __syncthreads();
#pragma unroll
  for (int k = 0; k < kPasses; ++k) {
    const int y = line + k * (kOrthoStreamThreads / kRuns);
    half8 hi, lo;
#pragma unroll
    for (int e = 0; e < kVec; ++e) {
      const uint32_t w = lds[run * kVec + e][y];
      hi[e] = __builtin_bit_cast(_Float16, static_cast<uint16_t>(w));
      lo[e] = __builtin_bit_cast(_Float16, static_cast<uint16_t>(w >> 16));
    }
    write(col0 + y, row0 + run * kVec, hi, lo);
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
//
// Of a 1B layer (four matrices of 2048 x 2048, three of 2048 x 5632), by the
// operations that the symmetric products cannot do without:
//           FAST                 FULL, three products
//   gram    130 us,  810 TF/s    315 us, 1000 TF/s
//   square   80 us,  756 TF/s    194 us,  930 TF/s
//   update  264 us,  797 TF/s    533 us, 1180 TF/s
// FULL is bound by the matrix cores (a large library product reaches 1310
// TF/s).  FAST is bound by what the loads bring to LDS, about 34 bytes a clock
// and CU: the update product takes 175 us without its loads, 244 without its
// multiplications; 256 x 256 tiles, which load half as much, reach 1086 TF/s on
// 4096 x 11008.  The tiles of 64 x 64 are bound by the launch and the loads'
// latency: one block a CU takes about 5 us, and 0.4 a slab with two slabs in
// LDS (0.2 with four).
struct ProductArgs {
  double a, b, c;
  int32_t from;   // the X^T buffer read
  int32_t first;  // step
  int32_t low;    // the update product writes X's low half
  float* pieces;  // unfinished sums of a symmetric product
};

// LDS holds RING slabs of both operands: 64 values of k (FAST), or 32 with both
// halves (FULL); 128 bytes for each of the operands' rows either way.
template <bool FULL, int RING, int BP, int BQ, int WP, int WQ>
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
  static constexpr int kLoads = kLoadsP + kLoadsQ;
  static_assert((RING & (RING - 1)) == 0 && RING * kSlab <= 160 * 1024 - 256, "the slabs, and the sums of block_sum");
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
// go to `lds` + 16 l.  m0 is a reserved register, which a list of clobbers
// cannot name; the compiler writes it right before uses of its own, and these
// kernels have none (no indirect register access, no messages: in the generated
// code m0 occurs in these lines only).  With its own builtin it would wait for
// the load before any other read of LDS.
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

// All of the wave's loads into LDS but the last OUT have landed and its reads of
// LDS are done, for every wave of the block.  The wait is the builtin one, which
// the compiler counts: with scalar loads outstanding it could only wait for all
// reads of LDS at each use of one.
template <int OUT>
__device__ __forceinline__ void slab_barrier() {
  static_assert(OUT < 16, "four bits of the count");
  asm volatile("" : : : "memory");
  __builtin_amdgcn_s_waitcnt(0x0070 + OUT);  // vmcnt(OUT) lgkmcnt(0)
  __builtin_amdgcn_s_barrier();
  asm volatile("" : : : "memory");
}

// s of an iteration: the mean of A's diagonal, ||X||^2 / r (1 / r at first);
// kept for the products that follow.
template <int kThreads>
__device__ __forceinline__ double shift_of(const OrthoMat& mt, const OrthoTile& t, bool first) {
  double s = 1.0;
  if (!first) {
    s = 0.0;
    for (int i = threadIdx.x; i < mt.x_tiles; i += kThreads) s += as_global(mt.x_part)[i];
    s = block_sum<kThreads>(s);
  }
  s /= mt.r;
  if (t.m == 0 && t.n == 0 && threadIdx.x == 0) *as_global(mt.shift) = s;
  return s;
}

// The results of a symmetric product from its sums: lane l of a wave holds
// C[p .. p+3][q] of each 16 x 16 block, p = 4 (l / 16), q = l mod 16.  They go
// through LDS, so that both the tile and its mirror image leave in whole rows
// (eight bytes a lane, straight from the registers, cost a 1B layer's gram
// product a quarter of its time).  Values behind the matrix become the zeros
// that its padding holds anyway.
template <int PRODUCT, bool FULL, int BP, int BQ, int WP, int WQ>
__device__ __forceinline__ void store_symmetric(f32x4 (&acc)[WP / 16][WQ / 16], char* smem, const OrthoMat& mt,
                                                const OrthoTile& t, const ProductArgs& args, double s, int wave,
                                                int lane) {
  using L = Layout<FULL>;
  constexpr int FP = WP / 16, FQ = WQ / 16, kWaves = (BP / WP) * (BQ / WQ), kThreads = kWaves * 64;
  constexpr int kPitch = BP + 8;  // halves of a row in LDS: rows begin in different banks
  static_assert(BQ * kPitch * 2 <= 2 * ProductShape<FULL, 2, BP, BQ, WP, WQ>::kSlab, "LDS");
  const int r = mt.r, ld = mt.ldr;
  const int wp = (wave % (BP / WP)) * WP, wq = (wave / (BP / WP)) * WQ;
  const int p_tile = t.m * BP, q_tile = t.n * BQ;
  const int p0 = wp + 4 * (lane >> 4), q0 = wq + (lane & 15);  // in the tile
  if constexpr (PRODUCT == kProductGram) {
#pragma unroll
    for (int i = 0; i < FP; ++i)
#pragma unroll
      for (int j = 0; j < FQ; ++j) acc[i][j] *= kScaleA / (kScaleX * kScaleX);
  } else {
    const _Float16* r_hi = as_global(mt.g[0]);
    const float lin = static_cast<float>(args.b + 2.0 * args.c * s);
    const float quadratic = static_cast<float>(args.c) / kScaleA;
#pragma unroll
    for (int i = 0; i < FP; ++i) {
      half4 rh[FQ], rl[FULL ? FQ : 1];
#pragma unroll
      for (int j = 0; j < FQ; ++j) {  // R is symmetric
        const int64_t from = L::at(min(q_tile + q0 + j * 16, r - 1), min(p_tile + p0 + i * 16, ld - 4), ld);
        rh[j] = *reinterpret_cast<const half4*>(r_hi + from);
        if constexpr (FULL) rl[j] = *reinterpret_cast<const half4*>(r_hi + 32 + from);
      }
#pragma unroll
      for (int j = 0; j < FQ; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float x = FULL ? join(rh[j], rl[FULL ? j : 0], e) : static_cast<float>(rh[j][e]);
          acc[i][j][e] = lin * x + quadratic * acc[i][j][e];
        }
    }
  }
  // the gram product's shift; with FULL F's term (a + bs + cs^2) I, which with
  // FAST the update product adds itself, unrounded
  const bool diagonal = (PRODUCT == kProductGram || FULL) && t.m == t.n;
  const bool edge = p_tile + BP > r || q_tile + BQ > r;
  if (diagonal || edge) {
    const double keep = args.a + args.b * s + args.c * s * s;
    const float diag = diagonal ? static_cast<float>((PRODUCT == kProductGram ? -s : keep) * kScaleA) : 0.f;
#pragma unroll
    for (int i = 0; i < FP; ++i)
#pragma unroll
      for (int j = 0; j < FQ; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int p = p_tile + p0 + i * 16 + e, q = q_tile + q0 + j * 16;
          if (p == q) acc[i][j][e] += diag;
          if (!(p < r && q < r)) acc[i][j][e] = 0.f;
        }
  }
  _Float16* tile = reinterpret_cast<_Float16*>(smem);
  _Float16* dst = as_global(PRODUCT == kProductGram ? mt.g[0] : mt.q[0]);
#pragma unroll
  for (int h = 0; h < (FULL ? 2 : 1); ++h) {  // the high halves, and with FULL the low ones
    __syncthreads();
#pragma unroll
    for (int i = 0; i < FP; ++i)
#pragma unroll
      for (int j = 0; j < FQ; ++j) {
        half4 v;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          v[e] = static_cast<_Float16>(acc[i][j][e]);
          if (FULL && h == 0) acc[i][j][e] -= static_cast<float>(v[e]);
        }
        *reinterpret_cast<half4*>(tile + (q0 + j * 16) * kPitch + p0 + i * 16) = v;
      }
    __syncthreads();
    constexpr int kRowThreads = BP / 8;
#pragma unroll
    for (int row0 = 0; row0 < BQ; row0 += kThreads / kRowThreads) {
      const int q = row0 + threadIdx.x / kRowThreads, p = 8 * (threadIdx.x % kRowThreads);
      if (q_tile + q < r && p_tile + p < r)
        *reinterpret_cast<half8*>(dst + 32 * h + L::at(q_tile + q, p_tile + p, ld)) =
            *reinterpret_cast<const half8*>(tile + q * kPitch + p);
    }
    if (t.m == t.n) continue;
#pragma unroll
    for (int b = 0; b < BP / 16 * (BQ / 32); b += kWaves) {
      const int block = b + wave, p = 16 * (block % (BP / 16)), q = 32 * (block / (BP / 16)) + 8 * (lane >> 4);
      half8 v;  // eight rows q of column p + l mod 16
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const half4 x = __builtin_bit_cast(
            half4, __builtin_amdgcn_ds_read_tr16_b64_v4f16((__attribute__((address_space(3))) fp16x4*)(
                       tile + (q + 4 * k + ((lane & 15) >> 2)) * kPitch + p + 4 * (lane & 3))));
#pragma unroll
        for (int e = 0; e < 4; ++e) v[4 * k + e] = x[e];
      }
      const int row = p_tile + p + (lane & 15);
      if (row < r && q_tile + q < r) *reinterpret_cast<half8*>(dst + 32 * h + L::at(row, q_tile + q, ld)) = v;
    }
  }
}

// ------------------------------------------------------------ the call's end

// What a call does with O: its source, and the type of its parameters or replicas.
constexpr int kNoApply = -1;
constexpr int apply_of(int source, bool bf16) { return 2 * source + (bf16 ? 1 : 0); }

// The first `count` of the elements i + e stride, e < 8, of the call's outputs
// from O; VECTORS: there are eight, side by side at a multiple of eight.
template <int SOURCE, bool BF16, bool VECTORS>
__device__ __forceinline__ void apply_run(const OrthoArgs& a, const RepPtrs& reps, double step, bool rollback, int64_t i,
                                          int stride, int count, const float (&o)[kVec]) {
  auto read = [&](const void* from, auto bf16, float (&to)[kVec]) {
    constexpr bool B = decltype(bf16)::value;
    if constexpr (VECTORS) {
      load_vec<B>(from, i, 0, kVec, to);
    } else {
#pragma unroll
      for (int e = 0; e < kVec; ++e) to[e] = e < count ? load_one<B>(from, i + static_cast<int64_t>(e) * stride) : 0.f;
    }
  };
  auto write = [&](void* to, auto bf16, const float (&from)[kVec]) {
    constexpr bool B = decltype(bf16)::value;
    if constexpr (VECTORS) {
      store_vec<B>(to, i, 0, kVec, from);
    } else {
#pragma unroll
      for (int e = 0; e < kVec; ++e)
        if (e < count) store_one<B>(to, i + static_cast<int64_t>(e) * stride, from[e]);
    }
  };
  const std::integral_constant<bool, BF16> type;
  if constexpr (SOURCE == kSourcePlain) {
    write(a.out, type, o);
  } else if constexpr (SOURCE == kSourceLocal) {
    float p[kVec];
    read(a.out, type, p);
#pragma unroll
    for (int e = 0; e < kVec; ++e)
      p[e] = static_cast<float>(fma(a.keep, static_cast<double>(p[e]), -step * static_cast<double>(o[e])));
    write(a.out, type, p);
  } else {
    float th[kVec];
    read(a.theta, std::false_type(), th);
    if (!rollback) {  // otherwise theta stays, to the sign of its zeros
#pragma unroll
      for (int e = 0; e < kVec; ++e)
        th[e] = static_cast<float>(fma(-step, static_cast<double>(o[e]), static_cast<double>(th[e])));
      write(a.theta, std::false_type(), th);
    }
    for (int j = 0; j < a.workers; ++j) write(reps.p[j], type, th);
  }
}

// The last step's tile of O (in the registers of the update product) into the
// call's outputs: through LDS, 64 stored rows at a time, so that each row's
// elements are read and written side by side.
template <int APPLY, int BP, int BQ, int WP, int WQ>
__device__ __forceinline__ void apply_tile(const f32x4 (&acc)[WP / 16][WQ / 16], char* smem, const OrthoMat& mt,
                                           const OrthoTile& t, const OrthoArgs& a, const RepPtrs& reps, int wave,
                                           int lane) {
  constexpr int SOURCE = APPLY / 2;
  constexpr int kRows = 64, kThreads = (BP / WP) * (BQ / WQ) * 64;
  constexpr int kCols = BP;  // of a stored row
  constexpr int kPitch = kCols + 4;
  static_assert(BP == BQ && BP % kRows == 0 && kRows % 32 == 0, "whole blocks of results a pass");
  static_assert(kRows * kPitch * 4 <= 2 * (BP + BQ) * 128, "LDS");
  float* tile = reinterpret_cast<float*>(smem);
  const int wp = (wave % (BP / WP)) * WP, wq = (wave / (BP / WP)) * WQ;
  const int p0 = wp + 8 * (lane >> 4), q0 = wq + (lane & 15);
  const double step = a.lr * mt.scale;
  bool rollback = false;
  if constexpr (SOURCE == kSourceOuter) rollback = a.rec->rollback;
  const bool aligned = (mt.offset | mt.cols) % kVec == 0;
  const int row0 = mt.tall ? t.n * BQ : t.m * BP, col0 = mt.tall ? t.m * BP : t.n * BQ;
  for (int pass = 0; pass < BP; pass += kRows) {
    __syncthreads();
#pragma unroll
    for (int i = 0; i < WP / 16; i += 2)
#pragma unroll
      for (int j = 0; j < WQ / 16; ++j) {
        const int p = p0 + 16 * i, q = q0 + 16 * j;  // O[p .. p+7][q]
        if ((mt.tall ? wq + 16 * j : wp + 16 * i) / kRows * kRows != pass) continue;
        if (mt.tall) {
          float* to = tile + (q - pass) * kPitch + p;
          *reinterpret_cast<f32x4*>(to) = acc[i][j];
          *reinterpret_cast<f32x4*>(to + 4) = acc[i + 1][j];
        } else {
#pragma unroll
          for (int e = 0; e < 8; ++e) tile[(p + e - pass) * kPitch + q] = acc[i + (e >> 2)][j][e & 3];
        }
      }
    __syncthreads();
    constexpr bool BF16 = (APPLY & 1) != 0;
    if (aligned) {  // eight elements of a row a thread
      for (int k = threadIdx.x; k < kRows * kCols / kVec; k += kThreads) {
        const int y = k / (kCols / kVec), x = k % (kCols / kVec) * kVec;
        const int row = row0 + pass + y, col = col0 + x;
        if (row >= mt.rows || col >= mt.cols) continue;
        const f32x4 lo = *reinterpret_cast<const f32x4*>(tile + y * kPitch + x);
        const f32x4 hi = *reinterpret_cast<const f32x4*>(tile + y * kPitch + x + 4);
        const float o[kVec] = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
        apply_run<SOURCE, BF16, true>(a, reps, step, rollback,
                                      mt.offset + static_cast<int64_t>(row) * mt.cols + col, 1, kVec, o);
      }
    } else {  // rows that begin anywhere: eight rows a thread, a row's elements lane by lane
      constexpr int kStep = kThreads / kCols;
      const int x = threadIdx.x % kCols, col = col0 + x;
      if (col < mt.cols)
        for (int y = threadIdx.x / kCols; y < kRows; y += kVec * kStep) {
          const int row = row0 + pass + y;
          float o[kVec];
#pragma unroll
          for (int e = 0; e < kVec; ++e) o[e] = tile[(y + e * kStep) * kPitch + x];
          apply_run<SOURCE, BF16, false>(a, reps, step, rollback,
                                         mt.offset + static_cast<int64_t>(row) * mt.cols + col, kStep * mt.cols,
                                         (mt.rows - row + kStep - 1) / kStep, o);
        }
    }
  }
}

// One tile of a product per block.  While one slab is multiplied, the loads of
// the RING - 1 next are under way.  A wave's operands are read a step ahead of their
// use: each register is read anew right after its last use, and the barrier
// between slabs stands before the last step of a slab, so that the first reads
// of the next one run under that step's products.
template <int PRODUCT, bool FULL, int APPLY, int RING, int BP, int BQ, int WP, int WQ>
__global__ __launch_bounds__((ProductShape<FULL, RING, BP, BQ, WP, WQ>::kThreads),
                             2)  // waves per SIMD that the registers are budgeted for
void ortho_product_kernel(const OrthoMat* __restrict__ mats, const OrthoTile* __restrict__ tiles, ProductArgs args,
                          OrthoArgs call, RepPtrs reps) {
  constexpr bool LAST = APPLY != kNoApply;
  using S = ProductShape<FULL, RING, BP, BQ, WP, WQ>;
  constexpr Reading kReadP = PRODUCT == kProductGram ? kAcross : PRODUCT == kProductUpdate ? kBlocks : kAlong;
  constexpr Reading kReadQ = PRODUCT == kProductGram ? kAcross : kAlong;
  using L = Layout<FULL>;
  __shared__ __align__(256) char smem[RING * S::kSlab];
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
  const int slabs = t.end - t.begin;
  p += t.begin * step, q += t.begin * step;
  auto fetch = [&](int n) {  // slab n
    const uint32_t at = lds0 + (n & (RING - 1)) * S::kSlab;
    const _Float16* from_p = p + n * step;
    const _Float16* from_q = q + n * step;
#pragma unroll
    for (int i = 0; i < S::kLoadsP; ++i) load_to_lds(at + (wave + i * S::kWaves) * 1024, from_p, off_p[i]);
#pragma unroll
    for (int i = 0; i < S::kLoadsQ; ++i)
      load_to_lds(at + S::kBytesP + (wave + i * S::kWaves) * 1024, from_q, off_q[i]);
  };
  for (int n = 0; n < RING - 1; ++n)
    if (n < slabs) fetch(n);

  const bool piece = PRODUCT != kProductUpdate && t.slot >= 0;  // of a sum that the join pass finishes
  const double s = PRODUCT != kProductGram ? *as_global(mt.shift) : piece ? 0.0 : shift_of<S::kThreads>(mt, t, args.first);
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
  // them, which is read ahead of the sums where there are registers for it.
  const int p8 = t.m * BP + wp + 8 * (lane >> 4), q0 = t.n * BQ + wq + (lane & 15);
  _Float16* to_hi = as_global(args.from ? mt.t[0][0] : mt.t[1][0]);
  _Float16* to_lo = L::low(to_hi, as_global(mt.t[0][1]));  // FAST: read and written in place
  constexpr bool kLow = PRODUCT == kProductUpdate && !FULL && !LAST;
  const float keep_lo = static_cast<float>(keep);
  half8 xl[kLow ? FP / 2 : 1][kLow ? FQ : 1];
  auto read_low = [&] {
    if constexpr (kLow) {
#pragma unroll
      for (int i = 0; i < FP; i += 2)
#pragma unroll
        for (int j = 0; j < FQ; ++j)
          xl[i / 2][j] = *reinterpret_cast<const half8*>(
              to_lo + L::at(min(q0 + j * 16, c - 1), min(p8 + i * 16, ld - 8), ld));
    }
  };
  constexpr bool kLowFirst = FP * FQ <= 16;
  if constexpr (kLowFirst) read_low();

  auto slab = [&](int n) { return smem + (n & (RING - 1)) * S::kSlab; };
  auto read_p = [&](const char* at, int part, int i) {
    return read_operand<kReadP, FULL, BP>(at, wp + (kReadP == kBlocks ? 16 * (i & ~1) + 4 * (i & 1) : 16 * i), part, lane);
  };
  auto read_q = [&](const char* at, int part, int j) {
    return read_operand<kReadQ, FULL, BQ>(at + S::kBytesP, wq + j * 16, part, lane);
  };
  auto mul = [&](const half8& x, const half8& y, f32x4& to) {
    to = __builtin_amdgcn_mfma_f32_16x16x32_f16(x, y, to, 0, 0, 0);
  };
  // Slab n has landed.  Of the loads, which land in order, those of the RING - 2
  // slabs behind it may be out, where there are as many; others than of slabs
  // are older or make the wait longer.
  auto landed = [&](int n) {
    if (RING > 2 && n + RING - 2 < slabs)
      slab_barrier<(RING - 2) * S::kLoads>();
    else
      slab_barrier<0>();
  };
  // Slab n + 1 has landed, and slab n is read: slab n + RING takes its place.
  auto next_slab = [&](int n) {
    landed(n + 1);
    if (n + RING < slabs) fetch(n + RING);
  };

  landed(0);
  if (RING - 1 < slabs) fetch(RING - 1);
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

  if constexpr (PRODUCT != kProductUpdate) {
    if (piece) {
      f32x4* to = reinterpret_cast<f32x4*>(as_global(args.pieces)) + static_cast<int64_t>(t.slot) * (BP * BQ / 4);
#pragma unroll
      for (int i = 0; i < FP; ++i)
#pragma unroll
        for (int j = 0; j < FQ; ++j) to[(i * FQ + j) * S::kThreads + threadIdx.x] = acc[i][j];
      return;
    }
    store_symmetric<PRODUCT, FULL, BP, BQ, WP, WQ>(acc, smem, mt, t, args, s, wave, lane);
  } else {
    if constexpr (!kLowFirst) read_low();
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
          if constexpr (kLow) v[e] += keep_lo * static_cast<float>(xl[i / 2][j][e]);
          if (!LAST && !(pp + e < r && qq < c)) v[e] = 0.f;
        }
        if constexpr (LAST) {
#pragma unroll
          for (int e = 0; e < 8; ++e) acc[i + (e >> 2)][j][e & 3] = v[e] * (1.f / kScaleX);
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
            if (FULL || args.low) *reinterpret_cast<half8*>(to_lo + at) = lo;
          }
        }
      }
    }
    if constexpr (LAST) {
      apply_tile<APPLY, BP, BQ, WP, WQ>(acc, smem, mt, t, call, reps, wave, lane);
    } else {
      const double sum = block_sum<S::kThreads>(static_cast<double>(sq) / (static_cast<double>(kScaleX) * kScaleX));
      if (threadIdx.x == 0) as_global(mt.x_part)[t.slot] = sum;
    }
  }
}

// The tiles of a symmetric product whose sums were cut into pieces: the pieces
// added up in order, then the results as from a whole sum.  A block takes 64 x
// 64 of a tile, which is what a wave of the product has of a 128 x 128 one (or
// all of a 64 x 64 one), in 32 x 32 parts.  Bound by the latency of the pieces'
// loads, hence several at a time: 16 tiles of 128 x 128 in 18 pieces each took
// 26 us in a block a tile and 10 so; 136 of 64 x 64 in four take 5.4.
template <int PRODUCT, bool FULL, int SIDE>
__global__ __launch_bounds__(256) void ortho_join_kernel(const OrthoMat* __restrict__ mats,
                                                         const OrthoTile* __restrict__ tiles, ProductArgs args) {
  constexpr int kParts = SIDE / 64, kFrags = SIDE / 32;  // kFrags: 16 x 16 blocks along a wave of the product
  OrthoTile t = tiles[blockIdx.x / (kParts * kParts)];
  const int part = blockIdx.x % (kParts * kParts);
  t.m = t.m * kParts + part % kParts, t.n = t.n * kParts + part / kParts;
  if (t.m < t.n) return;  // the mirror image of another part
  const OrthoMat mt = mats[t.mat];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int from_wave = kParts == 1 ? wave : part, i0 = kParts == 1 ? 0 : 2 * (wave & 1), j0 = kParts == 1 ? 0 : 2 * (wave >> 1);
  f32x4 acc[2][2];
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int j = 0; j < 2; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  const f32x4* from = reinterpret_cast<const f32x4*>(as_global(args.pieces)) + from_wave * 64 + lane;
#pragma unroll 4
  for (int k = t.begin; k < t.end; ++k)
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int j = 0; j < 2; ++j)
        acc[i][j] += from[static_cast<int64_t>(k) * (SIDE * SIDE / 4) + ((i0 + i) * kFrags + j0 + j) * 256];
  const double s = PRODUCT == kProductGram ? shift_of<256>(mt, t, args.first) : *as_global(mt.shift);
  __shared__ __align__(256) char smem[2 * ProductShape<FULL, 2, 64, 64, 32, 32>::kSlab];
  store_symmetric<PRODUCT, FULL, 64, 64, 32, 32>(acc, smem, mt, t, args, s, wave, lane);
}

template <int PRODUCT, bool FULL, int APPLY, int RING, int BP, int BQ, int WP, int WQ>
hipError_t launch_product(const OrthoMat* mats, const OrthoTiles& tiles, const ProductArgs& args, const OrthoArgs& call,
                          const RepPtrs& reps, hipStream_t stream) {
  ortho_product_kernel<PRODUCT, FULL, APPLY, RING, BP, BQ, WP, WQ>
      <<<tiles.count, ProductShape<FULL, RING, BP, BQ, WP, WQ>::kThreads, 0, stream>>>(mats, tiles.tile, args, call, reps);
  return hipGetLastError();
}

template <int PRODUCT, bool FULL>
hipError_t launch_join(int side, const OrthoMat* mats, const OrthoTiles& tiles, const ProductArgs& args,
                       hipStream_t stream) {
  if (side == 128)
    ortho_join_kernel<PRODUCT, FULL, 128><<<4 * tiles.count, 256, 0, stream>>>(mats, tiles.tile, args);
  else if (side == 64)
    ortho_join_kernel<PRODUCT, FULL, 64><<<tiles.count, 256, 0, stream>>>(mats, tiles.tile, args);
  else
    return hipErrorInvalidValue;
  return hipGetLastError();
}

template <int PRODUCT, bool FULL, int APPLY = kNoApply>
hipError_t launch_product_of(int side, const OrthoMat* mats, const OrthoTiles& tiles, const ProductArgs& args,
                             const OrthoArgs& call, const RepPtrs& reps, hipStream_t stream) {
  if constexpr (PRODUCT == kProductUpdate && !FULL)
    if (side == 256) return launch_product<PRODUCT, FULL, APPLY, 2, 256, 256, 128, 64>(mats, tiles, args, call, reps, stream);
  if (side == 128) return launch_product<PRODUCT, FULL, APPLY, 2, 128, 128, 64, 64>(mats, tiles, args, call, reps, stream);
  if (side == 64 && tiles.few)
    return launch_product<PRODUCT, FULL, APPLY, 4, 64, 64, 32, 32>(mats, tiles, args, call, reps, stream);
  if (side == 64) return launch_product<PRODUCT, FULL, APPLY, 2, 64, 64, 32, 32>(mats, tiles, args, call, reps, stream);
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
                                const OrthoCoef& coef, int step, int steps, const OrthoCall& call, float* pieces,
                                hipStream_t stream) {
  if (tiles.count == 0) return hipSuccess;
  const ProductArgs args = {coef.a, coef.b, coef.c, step & 1, step == 0, step < steps - 2, pieces};
  const OrthoArgs a = args_of(call);
  const RepPtrs r = reps_of(call);
#define EDIT_PRODUCT(P, A)                                                        \
  (full ? launch_product_of<P, true, A>(side, mats, tiles, args, a, r, stream) \
        : launch_product_of<P, false, A>(side, mats, tiles, args, a, r, stream))
#define EDIT_JOIN(P)                                             \
  (full ? launch_join<P, true>(side, mats, tiles, args, stream) \
        : launch_join<P, false>(side, mats, tiles, args, stream))
  switch (product) {
    case kProductGram: return EDIT_PRODUCT(kProductGram, kNoApply);
    case kProductGramJoin: return EDIT_JOIN(kProductGram);
    case kProductSquareJoin: return EDIT_JOIN(kProductSquare);
    case kProductSquare: return EDIT_PRODUCT(kProductSquare, kNoApply);
    case kProductUpdate:
      if (step < steps - 1) return EDIT_PRODUCT(kProductUpdate, kNoApply);
      switch (apply_of(call.source, call.bf16)) {
        case apply_of(kSourcePlain, false): return EDIT_PRODUCT(kProductUpdate, apply_of(kSourcePlain, false));
        case apply_of(kSourcePlain, true): return EDIT_PRODUCT(kProductUpdate, apply_of(kSourcePlain, true));
        case apply_of(kSourceLocal, false): return EDIT_PRODUCT(kProductUpdate, apply_of(kSourceLocal, false));
        case apply_of(kSourceLocal, true): return EDIT_PRODUCT(kProductUpdate, apply_of(kSourceLocal, true));
        case apply_of(kSourceOuter, false): return EDIT_PRODUCT(kProductUpdate, apply_of(kSourceOuter, false));
        case apply_of(kSourceOuter, true): return EDIT_PRODUCT(kProductUpdate, apply_of(kSourceOuter, true));
      }
  }
#undef EDIT_JOIN
#undef EDIT_PRODUCT
  return hipErrorInvalidValue;
}

}  // namespace edit
