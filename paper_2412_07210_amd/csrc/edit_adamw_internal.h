// Internal declarations of the AdamW step (edit_adamw_*), shared by
// edit_adamw_kernels.hip and edit_adamw_runtime.hip.  Not part of the public ABI.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "edit_outer.h"

namespace edit {

constexpr int kAdamThreads = 256;
constexpr int kAdamChunk = kAdamThreads * 8;              // elements of a block: whole scale blocks
constexpr int kAdamTensors = 56;                         // of one launch: its table is in the kernel arguments
constexpr int kAdamNormTensors = 192;                    // of one launch of the norm pass
constexpr int kAdamNormVecs = 4;                         // vectors of a lane and chunk of the norm pass
constexpr int kAdamNormChunk = kAdamChunk * kAdamNormVecs;
constexpr int kAdamNormBlocksPerCu = 4;
constexpr int kAdamDecideThreads = 1024;
static_assert(kAdamChunk % EDIT_ADAMW_BLOCK == 0, "a scale belongs to one block");

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
