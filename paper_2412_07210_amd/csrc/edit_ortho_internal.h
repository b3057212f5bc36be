// Internal declarations of the orthogonalised updates (edit_ortho_* and
// edit_outer_step_layer_ortho), shared by edit_ortho_kernels.hip and
// edit_ortho_runtime.hip.  Not part of the public ABI.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "edit_outer.h"
#include "edit_outer_internal.h"
#include "ortho_tiles.h"

namespace edit {

// Powers of two that the fp16 operands are stored at, so that neither their
// high nor their low halves leave fp16's range: X (entries up to its largest
// singular value, about 1) at kScaleX, A - sI and the polynomial at kScaleA.
// The low half of a value v is v's rounding error, about v / 4096; fp16 keeps
// it down to 2^-24 / scale.
constexpr float kScaleX = 8192.f;
constexpr float kScaleA = 2048.f;
// The largest |sigma| and |polynomial| that the scales leave room for, with a
// factor of two for rounding (65504 / 8192 / 2 and 65504 / 2048 / 2).
constexpr double kMaxSigma = 4.0;
constexpr double kMaxPoly = 15.0;

constexpr int kOrthoPad = 64;           // leading dimensions are multiples of this (zero behind the matrix)
constexpr int kOrthoStreamThreads = 256;
constexpr int kOrthoMaxChunks = 512;    // chunks (norm partials) of one matrix
constexpr int kOrthoLoadTile = 64;      // side of the load pass's tiles

// Matrices that one block takes whole: X^T and A, high and low halves, in LDS,
// rows of r rounded up to 32 values and eight more.
constexpr int kOrthoSmallThreads = 512;
constexpr int kOrthoSmallSide = 128;   // of A
constexpr int kOrthoSmallRows = 256;   // of X^T
constexpr int kOrthoSmallLds = 148 * 1024;
constexpr int kOrthoSmallSlack = 10 * 1024;  // behind: reads of 128 columns or rows where there are fewer
constexpr int kOrthoSmallPer = 48;     // elements per thread, at most
inline bool ortho_is_small(int64_t r, int64_t c) {
  if (r > kOrthoSmallSide || c > kOrthoSmallRows || r * c > kOrthoSmallPer * kOrthoSmallThreads) return false;
  const int64_t rp = (r + 31) / 32 * 32, cp = (c + 31) / 32 * 32;
  return (cp + rp) * (rp + 8) * 4 <= kOrthoSmallLds;
}

// One matrix of a unit: r = min(rows, cols), c = max(rows, cols).  The
// working matrix X is r x c: the stored one, or its transpose where rows >
// cols.  Every array is zero behind its r columns.
struct OrthoMat {
  // High and low halves; with FULL they share the first array (Layout in the
  // kernels) and there is no second.  R and F have low halves with FULL only.
  _Float16* t[2][2];  // X^T, [buffer][half]: [c][ldr], and rows of zeros to a multiple of kOrthoPad
  _Float16* g[1];     // R = A - sI                            [r][ldr]
  _Float16* q[1];     // the update product's polynomial F     [r][ldr]
  double* norm_part;  // sums of squares of the update's chunks
  double* x_part;     // sums of squares of the X tiles of the last product
  double* shift;      // s of this iteration
  int64_t offset;     // of the matrix in the unit
  double scale;       // its factor in a step
  int32_t rows, cols, r, c, ldr;
  int32_t chunks, x_tiles;
  int32_t tall;       // rows > cols: X is the stored matrix transposed
};

// Elements [begin, end) of the unit: of matrix `mat`, partial `slot`; of no
// matrix with mat = -1.
struct OrthoChunk {
  int64_t begin, end;
  int32_t mat, slot;
};

// What the update of a call is made from.
enum OrthoSource { kSourcePlain = 0, kSourceLocal = 1, kSourceOuter = 2 };

struct OrthoCall {
  OrthoSource source;
  bool bf16;            // type of x / out, param / grad or the replicas
  const void* x;        // plain: the update;  local: the gradient
  void* out;            // plain: the result;  local: the parameters
  float* momentum;      // local, outer
  float* theta;         // outer
  float* u;             // [numel] scratch: outer's update
  void* const* reps;    // outer: K replicas (host array)
  const UnitRecord* rec;
  int32_t workers;
  int32_t nesterov;     // local
  double mu, keep, lr;  // momentum; 1 - lr * decay; step length
};

struct OrthoCoef {
  double a, b, c;
};

// Products of an iteration.
enum OrthoProduct { kProductGram = 0, kProductSquare = 1, kProductUpdate = 2, kProductGramJoin = 3, kProductSquareJoin = 4 };
// Values of k that a product takes a step.
inline int ortho_slab(bool full) { return full ? 32 : 64; }

struct OrthoTiles {
  const OrthoTile* tile;  // device
  int32_t count;
  bool few;  // of 64 x 64 tiles: four slabs in LDS
};

// Pass over the update: momentum and update of the call, and the chunks' sums of squares.
hipError_t launch_ortho_source(const OrthoCall& call, const OrthoMat* mats, const OrthoChunk* chunks, int count,
                               hipStream_t stream);
// X^T of the update over its norm.
hipError_t launch_ortho_load(bool full, const OrthoCall& call, const OrthoMat* mats, const OrthoTile* tiles, int count,
                             hipStream_t stream);
// One product of an iteration, or the join of a symmetric one's pieces;
// `side`: of its tiles.  The last step's update product makes the call's outputs.
hipError_t launch_ortho_product(OrthoProduct product, bool full, int side, const OrthoMat* mats, const OrthoTiles& tiles,
                                const OrthoCoef& coef, int step, int steps, const OrthoCall& call, float* pieces,
                                hipStream_t stream);
// The whole call but the outer step's source pass, for small matrices only, one
// per block; `widest`: the largest r.
hipError_t launch_ortho_small(bool full, const OrthoCall& call, const OrthoMat* mats, int count, int widest,
                              const OrthoCoef* coef, int steps, hipStream_t stream);
// The outer step's part of a handle: its argument check and, after the
// decision has been enqueued, the orthogonalised update (edit_ortho_runtime.hip).
edit_status_t check_ortho_unit(const edit_ortho* h, int64_t numel, int device);
edit_status_t enqueue_ortho_outer(edit_ortho* h, bool bf16, float* theta, float* momentum, void* const* replicas,
                                  int workers, const UnitRecord* rec, double lr, double rho, hipStream_t stream);

}  // namespace edit
