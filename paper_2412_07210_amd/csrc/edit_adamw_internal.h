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
// 32 bytes apart run at half the rate.  Then twice for 8-bit states, whose loads
// are short, once for fp32 ones.  us for 308M elements, V U = 8 1, 4 2 and 4 1:
// bf16 parameters and gradients with e4m3 states 506, 583 and 683; fp32 and
// bf16 800, 732 and 729 (770, 696 and 729 with the best cap); fp32 states, 4 2
// and 4 1: bf16 1148 and 1039, fp32 1506 and 1368.  Blocks of 256 threads take
// 0 to 2% more.
constexpr int adamw_vec(bool param_bf16, bool grad_bf16, bool held) { return param_bf16 && grad_bf16 && held ? 8 : 4; }
constexpr int adamw_times(bool param_bf16, bool grad_bf16, bool held) {
  return held && adamw_vec(param_bf16, grad_bf16, held) == 4 ? 2 : 1;
}
constexpr int adamw_chunk(bool param_bf16, bool grad_bf16, bool held) {
  return kAdamThreads * adamw_vec(param_bf16, grad_bf16, held) * adamw_times(param_bf16, grad_bf16, held);
}
// Blocks of it that run on a CU, of the 32 that fit: the mix of reads and writes
// runs faster with fewer of its loads in flight.  us uncapped, at 24, 20 and 16:
// e4m3 states: bf16 506, 559, 610, 724; bf16 and fp32 gradients 588, 620, 675,
// 796; fp32 and bf16 732, 696, 702, 810; fp32 809, 798, 778, 759.  fp32 states:
// bf16 1039, 1059, 1145, 1346; bf16 and fp32 1147, 1117, 1171, 1369; fp32 and
// bf16 1253, 1225, 1245, 1396; fp32 1368, 1322, 1311, 1431.
constexpr int adamw_resident(bool param_bf16, bool grad_bf16, bool held) {
  if (held) return param_bf16 ? 32 : grad_bf16 ? 24 : 16;
  return param_bf16 && grad_bf16 ? 32 : param_bf16 || grad_bf16 ? 24 : 20;
}
constexpr int kAdamConvertChunk = kAdamThreads * 8;

// The norm pass: persistent blocks that stride over chunks, a lane kAdamNormVecs
// 16-byte vectors of one, the next chunk's in flight.
constexpr int kAdamNormThreads = 256;
constexpr int kAdamNormVecs = 4;
constexpr int kAdamNormBlocksPerCu = 2;
constexpr int kAdamNormTensors = 192;                    // of one launch
constexpr int adamw_norm_chunk(bool bf16) { return kAdamNormThreads * kAdamNormVecs * (bf16 ? 8 : 4); }

// Device-resident state of a handle and what its next update pass goes by.
struct alignas(16) AdamRecord {
  int64_t step;      // t: steps taken
  int64_t skipped;   // calls left out because the gradient's norm was not finite
  double norm;       // of the last call that took one
  double lr_decay;   // lr * weight_decay of this call
  uint64_t key;      // of this call's random numbers
  float clip;        // c
  float rate;        // lr / (1 - beta1^t)
  float root;        // 1 / sqrt(1 - beta2^t)
  int32_t skip;      // this call changes nothing
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

// Block b works on the tensor whose first[] is the last one that is <= b.
struct AdamTable {
  int32_t first[64];  // beyond the tensors: more than any block
  float decay[kAdamTensors];
  AdamTensor tensor[kAdamTensors];
  int32_t base;  // index of tensor[0] among all
};
static_assert(sizeof(AdamTable) + 128 <= 4096, "kernel arguments");

struct AdamNormTable {
  int32_t first[kAdamNormTensors];
  int32_t chunks;
  int64_t numel[kAdamNormTensors];
  const void* grad[kAdamNormTensors];
};
static_assert(sizeof(AdamNormTable) + 128 <= 4096, "kernel arguments");

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
  bool check;               // S is there
};

hipError_t launch_adamw_norm(bool bf16, int blocks, const AdamNormTable& table, double* partials, hipStream_t stream);
// out = the sum of `count` partials, in their order.
hipError_t launch_adamw_sum(const double* partials, int count, double* out, hipStream_t stream);
// S from `count` partials, or from *sumsq where that is given, and the record.
hipError_t launch_adamw_decide(const double* partials, int count, const double* sumsq, const AdamCall& call,
                               const AdamHyper& hyper, AdamRecord* rec, hipStream_t stream);
hipError_t launch_adamw_step(bool param_bf16, bool grad_bf16, bool held, bool stochastic, int blocks, const AdamTable& table,
                             const AdamHyper& hyper, const AdamRecord* rec, hipStream_t stream);
// States in the table's m and v (fp32) from or to the codes in param (of m) and grad (of v).
hipError_t launch_adamw_convert(bool pack, int blocks, const AdamTable& table, uint64_t key, hipStream_t stream);
uint64_t adamw_key(uint64_t seed, uint64_t t);

}  // namespace edit
