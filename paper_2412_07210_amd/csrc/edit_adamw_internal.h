// Internal declarations of the AdamW step (edit_adamw_*), shared by
// edit_adamw_kernels.hip and edit_adamw_runtime.hip.  Not part of the public ABI.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "edit_outer.h"
#include "lds_cap.h"

namespace edit {

// The streaming passes run blocks of one wave on a flat grid.
constexpr int kAdamThreads = 64;
constexpr int kAdamTensors = 56;                         // of one launch: its table is in the kernel arguments
constexpr int kAdamDecideThreads = 512;

// A lane of the update pass takes V consecutive elements of every buffer, U
// times, the next V beside its neighbour's: a block V * U * 64.  Eight bf16 and
// eight codes are 16 and 8 bytes; with fp32 buffers four, as 16-byte accesses
// 32 bytes apart run at half the rate.  Twice for 8-bit states, whose loads are
// short, once for fp32 ones.  us for 308M elements at the cap below: e4m3 states with
// bf16 parameters and gradients, V U = 8 1, 8 2 and 4 2, 517, 502 and 556; fp32 and
// bf16, 4 1 and 4 2, 715 and 699 (8 1 10% more); fp32 states, 4 1 and 4 2: bf16 1045 and
// 1098, fp32 1311 and 1415.  Blocks of 256 threads take 0 to 2% more.
constexpr int adamw_vec(bool param_bf16, bool grad_bf16, bool held) { return param_bf16 && grad_bf16 && held ? 8 : 4; }
constexpr int adamw_times(bool held) { return held ? 2 : 1; }
constexpr int adamw_chunk(bool param_bf16, bool grad_bf16, bool held) {
  return kAdamThreads * adamw_vec(param_bf16, grad_bf16, held) * adamw_times(held);
}
// Blocks of it that run on a CU: the mix of reads and writes runs faster with fewer
// of its loads in flight.  Registers leave room for 32, with bf16 and e4m3 states for
// 24 (20 rounded to nearest); LDS, handed out in whole pieces, for 25, 21, 18, 16, 14,
// 12 or 11.  32: no cap.  us for 308M elements uncapped, capped and (at the nearest
// numbers above and below): e4m3 states: bf16 506, none (505 at 25, 511 at 21); bf16
// and fp32 gradients 602, none (610 at 25); fp32 and bf16 724, 699 (704, 701); fp32
// 821, 787 (791, 792).  fp32 states: bf16 1089, 1040 (1047, 1047); bf16 and fp32 1187,
// 1124 (1133, 1142); fp32 and bf16 1286, 1219 (1224, 1226); fp32 1408, 1309 (1322, 1316).
constexpr int adamw_resident(bool param_bf16, bool grad_bf16, bool held) {
  if (held) return param_bf16 ? 32 : grad_bf16 ? 21 : 18;
  return param_bf16 && grad_bf16 ? 16 : param_bf16 || grad_bf16 ? 14 : 12;
}
// Conversions: a lane takes four elements once to pack (308M elements in 458 us,
// 6.75 TB/s; twice 471), twice to unpack, capped (498, 6.2 TB/s; uncapped 571, once
// 507).
constexpr int adamw_convert_times(bool pack) { return pack ? 1 : 2; }
constexpr int adamw_convert_chunk(bool pack) { return kAdamThreads * 4 * adamw_convert_times(pack); }
constexpr int kAdamUnpackResident = 18;

// The norm pass: persistent blocks that stride over chunks, a lane kAdamNormVecs
// 16-byte vectors of one, the next chunk's in flight.
constexpr int kAdamNormThreads = 256;
constexpr int kAdamNormVecs = 4;
constexpr int kAdamNormBlocksPerCu = 2;
constexpr int kAdamNormTensors = 192;                    // of one launch
// Bytes at its end that the update pass, which begins there, finds in the Infinity
// Cache: loaded through the caches, which all of it would run 12% slower by.  us of
// whole steps with 0, 96, 160, 224 and 256 MiB: 350M model fp32 1488, 1484, 1477,
// 1470, 1467; its fp32 parameters, bf16 gradients, e4m3 states 795, 787, 784, 780, 783.
constexpr int64_t kAdamNormKeep = int64_t(224) << 20;
constexpr int adamw_norm_chunk(bool bf16, int threads = kAdamNormThreads) { return threads * kAdamNormVecs * (bf16 ? 8 : 4); }
// Few gradients: one block takes them all, a wave a chunk, in one launch instead
// of two.  us of a sum, so and otherwise, of 2048 bf16 elements in each of 8 tensors
// in a graph 2.6 and 5.5; 32: 4.3 and 5.7; 64: 6.2 and 5.7, but eager 7.2 and 8.5.
constexpr int kAdamSmallThreads = 1024;
constexpr int kAdamSmallChunks = 64;

// Calls of few blocks take the decision in every block of the update pass, without
// a launch of its own.  us in a graph with a decision launch and so, without a clip
// and with one: fp32, 256 blocks 5.1 and 3.7, 9.6 and 8.3; 2048: 6.1 and 5.0, 8.6
// and 7.9; 4096: 7.2 and 7.6, 9.9 and 11.5; bf16 with e4m3 states, 512 blocks 6.7
// and 5.4, 9.5 and 8.4; 2048: 9.0 and 7.7, 11.3 and 11.1; 4096: 12.2 and 11.7, 15.7
// and 17.0.
constexpr int kAdamFusedBlocks = 2048;

// Device-resident state of a handle and what its next update pass goes by.  t, the
// steps taken, is in an array beside it: one for every block of a call that steps
// all tensors, which reads and writes its own (no block can tell whether another
// one has counted on already); they are the same between calls.
struct alignas(16) AdamRecord {
  int64_t step;      // t of the last call that was not left out
  int64_t skipped;   // calls left out because of the gradient's norm or the rate
  double norm;       // of the last call that took one
  double lr_decay;   // lr * weight_decay of this call
  uint64_t key;      // of this call's random numbers
  float clip;        // c
  float root, eps;   // 1 / sqrt(1 - beta2^t) and eps, over lr / (1 - beta1^t)
  int32_t skip;      // this call changes nothing
  int32_t tiny;      // roots of v below 2^-126 show beside eps
};

struct AdamTensor {
  void* param;
  const void* grad;
  void* m;  // fp32, or e4m3 codes
  void* v;
  float* m_scale;
  float* v_scale;
  int64_t numel;
};

struct AdamHyper {
  double beta1, beta2, eps;
};

// What a call does beside the tensors.
struct AdamCall {
  double lr;
  const double* lr_device;  // in place of lr
  double weight_decay;
  double max_norm;          // infinity: no clip
  uint64_t seed;
  const double* sums;       // S: the sum of `count` parts, in their order
  int32_t count;            // 0: there is none, and no check
};

// Block b works on the tensor whose first[] is the last one that is <= b.
struct AdamTable {
  int32_t first[64];  // beyond the tensors: more than any block
  double decay[kAdamTensors];  // in 64 bits: with lambda it may be a number of fp32 where it alone is none
  AdamTensor tensor[kAdamTensors];
  int32_t base;  // index of tensor[0] among all
};
static_assert(sizeof(AdamTable) + sizeof(AdamHyper) + sizeof(AdamCall) + 64 <= 4096, "kernel arguments");

struct AdamNormTable {
  int32_t first[kAdamNormTensors];
  int32_t chunks;
  int32_t keep;  // chunks from here on stay in the caches
  int64_t numel[kAdamNormTensors];
  const void* grad[kAdamNormTensors];
};
static_assert(sizeof(AdamNormTable) + 64 <= 4096, "kernel arguments");

// The record and t of a handle.
struct AdamState {
  AdamRecord* rec;
  int64_t* steps;
  int32_t slots;  // of steps, at least 1
};

hipError_t launch_adamw_norm(bool bf16, int blocks, const AdamNormTable& table, double* partials, hipStream_t stream);
// *out = S of few gradients, chunks of a wave.
hipError_t launch_adamw_small(bool bf16, const AdamNormTable& table, double* out, hipStream_t stream);
// out = the sum of `count` partials, in their order.
hipError_t launch_adamw_sum(const double* partials, int count, double* out, hipStream_t stream);
// The record of a call, and t.
hipError_t launch_adamw_decide(const AdamCall& call, const AdamHyper& hyper, const AdamState& state, hipStream_t stream);
// `call`: takes the decision itself; `before`: blocks of the call's tables before this one.
struct AdamKind {
  bool param_bf16, grad_bf16, held, stochastic;
};
hipError_t launch_adamw_step(const AdamKind& kind, int blocks, const AdamTable& table, const AdamHyper& hyper,
                             const AdamState& state, const AdamCall* call, int before, hipStream_t stream);
// States in the table's m and v (fp32) from or to the codes in param (of m) and grad (of v).
hipError_t launch_adamw_convert(bool pack, int blocks, const AdamTable& table, uint64_t key, hipStream_t stream);
uint64_t adamw_key(uint64_t seed, uint64_t t);

}  // namespace edit
