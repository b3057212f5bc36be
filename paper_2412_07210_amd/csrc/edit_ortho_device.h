// Device code that edit_ortho_kernels.hip and edit_ortho_small.hip share: the
// elements of a unit, high and low halves, block sums, and a call's arguments.
#pragma once

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

typedef __fp16 fp16x4 __attribute__((__vector_size__(8)));

// A value as the sum of two halves.
__device__ __forceinline__ void split(float v, _Float16& hi, _Float16& lo) {
  hi = static_cast<_Float16>(v);
  lo = static_cast<_Float16>(v - static_cast<float>(hi));
}
__device__ __forceinline__ float join(const half4& hi, const half4& lo, int e) {
  return static_cast<float>(hi[e]) + static_cast<float>(lo[e]);
}

// ------------------------------------------------------- a call's arguments

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

inline OrthoArgs args_of(const OrthoCall& c) {
  return {c.x, c.out, c.momentum, c.theta, c.u, c.rec, c.workers, c.nesterov, c.mu, c.keep, c.lr};
}

inline RepPtrs reps_of(const OrthoCall& c) {
  RepPtrs r = {};
  for (int j = 0; j < c.workers; ++j) r.p[j] = c.reps[j];
  return r;
}

}  // namespace
}  // namespace edit
