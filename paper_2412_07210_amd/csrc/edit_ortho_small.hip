// The orthogonalised updates of small matrices: the whole call for one matrix
// per block, where X and A fit into LDS (ortho_is_small), with no launch
// between the products, whose latency bounds matrices of this size.
//
// LDS holds X^T [c][r] and R, then F, [r][r] (edit_ortho_kernels.hip names
// them), high and low halves apart, in rows of r rounded up to 32 values and
// eight more, which begin in different banks; what pads them is zero.  Wave w
// takes rows 16 w .. of the symmetric products, all columns, so that R and F
// stay in its registers as well, and rows 16 w and 16 w + 128 of X^T.  NB is
// the number of 16-column blocks of the widest matrix of the launch: a narrower
// one multiplies what lies behind its columns too and drops the results, which
// keeps the loops free of branches.  Bound by the chain of its steps: each
// product waits for the one before, with a barrier and the latency of LDS and of
// the matrix cores' results between.  One 128 x 128 matrix takes 49 us (66 with
// twice the operations; 124 in launches of 64 x 64 tiles), as many as there are
// CUs hardly more.
#include "edit_ortho_device.h"

namespace edit {
namespace {

struct SmallCoef {
  double v[EDIT_ORTHO_MAX_STEPS][3];
};

// Row and column of the elements threadIdx.x + t * kOrthoSmallThreads of a
// matrix, without a division each.
struct Walk {
  int row, col, rows, cols, width;
  __device__ Walk(int start, int width_) : width(width_) {
    row = start / width, col = start - row * width;
    rows = kOrthoSmallThreads / width, cols = kOrthoSmallThreads - rows * width;
  }
  __device__ void next() {
    row += rows, col += cols;
    if (col >= width) col -= width, ++row;
  }
};

template <int SOURCE, bool BF16, bool FULL, int NB>
__global__ __launch_bounds__(kOrthoSmallThreads) void ortho_small_kernel(OrthoArgs a, RepPtrs reps,
                                                                        const OrthoMat* __restrict__ mats,
                                                                        SmallCoef coef, int steps) {
  constexpr int kThreads = kOrthoSmallThreads;
  constexpr int kWaves = kThreads / 64;
  constexpr int kRows = kOrthoSmallRows / 16 / kWaves;  // blocks of X^T's rows per wave
  __shared__ __align__(256) char smem[kOrthoSmallLds + kOrthoSmallSlack];
  const OrthoMat mt = mats[blockIdx.x];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int r = mt.r, c = mt.c, n = r * c, rp = (r + 31) & ~31, cp = (c + 31) & ~31;
  const int pitch = rp + 8;
  _Float16* x_hi = reinterpret_cast<_Float16*>(smem);
  _Float16* x_lo = x_hi + cp * pitch;
  _Float16* g_hi = x_lo + cp * pitch;
  _Float16* g_lo = g_hi + rp * pitch;

  // u, its norm, and X^T = u / ||u||: each thread keeps its elements of u
  float u[kOrthoSmallPer];
#pragma unroll
  for (int t = 0; t < kOrthoSmallPer; ++t) {
    const int e = threadIdx.x + t * kThreads;
    const int64_t i = mt.offset + e;
    u[t] = 0.f;
    if (e < n) u[t] = SOURCE == kSourceOuter ? a.u[i] : load_one<BF16>(a.x, i);
  }
  if constexpr (SOURCE == kSourceLocal) {
    float m[kOrthoSmallPer];
#pragma unroll
    for (int t = 0; t < kOrthoSmallPer; ++t) {
      const int e = threadIdx.x + t * kThreads;
      m[t] = e < n ? a.momentum[mt.offset + e] : 0.f;
    }
#pragma unroll
    for (int t = 0; t < kOrthoSmallPer; ++t) {
      const int e = threadIdx.x + t * kThreads;
      const double g = u[t];
      m[t] = static_cast<float>(fma(a.mu, static_cast<double>(m[t]), g));
      if (e < n) a.momentum[mt.offset + e] = m[t];
      u[t] = a.nesterov ? static_cast<float>(fma(a.mu, static_cast<double>(m[t]), g)) : m[t];
    }
  }
  for (int i = threadIdx.x; i < 2 * (cp + rp) * pitch / 8; i += kThreads)
    reinterpret_cast<u32x4*>(smem)[i] = u32x4{0, 0, 0, 0};
  double sum = 0.0;
#pragma unroll
  for (int t = 0; t < kOrthoSmallPer; ++t) sum = fma(static_cast<double>(u[t]), static_cast<double>(u[t]), sum);
  sum = block_sum<kThreads>(sum);
  const double inv = sum > 0.0 ? kScaleX / sqrt(sum) : (sum == 0.0 ? 0.0 : sum);
  Walk at(threadIdx.x, mt.cols);
#pragma unroll
  for (int t = 0; t < kOrthoSmallPer; ++t) {
    if (threadIdx.x + t * kThreads < n) {
      _Float16 hi, lo;
      split(static_cast<float>(u[t] * inv), hi, lo);
      const int to = mt.tall ? at.row * pitch + at.col : at.col * pitch + at.row;
      x_hi[to] = hi, x_lo[to] = lo;
    }
    at.next();
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
      const _Float16* from = m + (k + 8 * l4 + 4 * h + (l16 >> 2)) * pitch + col0 + 4 * (l16 & 3);
      const half4 v = __builtin_bit_cast(
          half4, __builtin_amdgcn_ds_read_tr16_b64_v4f16((__attribute__((address_space(3))) fp16x4*)(from)));
#pragma unroll
      for (int e = 0; e < 4; ++e) out[4 * h + e] = v[e];
    }
    return out;
  };
  auto mul = [&](const half8& x, const half8& y, f32x4& to) {
    to = __builtin_amdgcn_mfma_f32_16x16x32_f16(x, y, to, 0, 0, 0);
  };
  // Four neighbours of row `row`: the high halves, and the low ones where a
  // product takes them.
  auto put = [&](_Float16* hi, int row, int col, const f32x4& v) {
    half4 h;
#pragma unroll
    for (int e = 0; e < 4; ++e) h[e] = static_cast<_Float16>(v[e]);
    *reinterpret_cast<half4*>(hi + row * pitch + col) = h;
    return h;
  };
  auto put_low = [&](_Float16* lo, int row, int col, const f32x4& v, const half4& h) {
    half4 l;
#pragma unroll
    for (int e = 0; e < 4; ++e) l[e] = static_cast<_Float16>(v[e] - static_cast<float>(h[e]));
    *reinterpret_cast<half4*>(lo + row * pitch + col) = l;
  };

  // What pads X stays zero and what pads R and F never meets the matrix's own
  // part (or the matrix is NaN altogether), so that nothing is masked.
  float* o = reinterpret_cast<float*>(smem);  // O in the end, [c][pitch], over both halves of X^T
  const int p0 = 16 * wave;
  for (int k = 0; k < steps; ++k) {
    f32x4 g[NB], f[NB];  // lane l: [p0 + l16][16 j + 4 l4 ..] of A, R and of R R
#pragma unroll
    for (int j = 0; j < NB; ++j) g[j] = f[j] = f32x4{0.f, 0.f, 0.f, 0.f};
    float trace = 0.f;
    if (wave < blocks) {
      for (int t = 0; t < cp; t += 32) {
        const half8 q = across(x_hi, p0, t);
        if constexpr (FULL) {
          const half8 ql = across(x_lo, p0, t);
#pragma unroll
          for (int j = 0; j < NB; ++j) {
            const half8 p = across(x_hi, 16 * j, t), pl = across(x_lo, 16 * j, t);
            mul(p, q, g[j]);
            mul(p, ql, g[j]);
            mul(pl, q, g[j]);
          }
        } else {
#pragma unroll
          for (int j = 0; j < NB; ++j) mul(across(x_hi, 16 * j, t), q, g[j]);
        }
      }
#pragma unroll
      for (int j = 0; j < NB; ++j) {
        g[j] *= kScaleA / (kScaleX * kScaleX);
        if (j == wave)
#pragma unroll
          for (int e = 0; e < 4; ++e) trace += 4 * l4 + e == l16 ? g[j][e] : 0.f;
      }
    }
    // s: any value would do that the three products share
    const double s = block_sum<kThreads>(trace) / (static_cast<double>(kScaleA) * r);
    const double ca = coef.v[k][0], cb = coef.v[k][1], cc = coef.v[k][2];
    const double keep = ca + cb * s + cc * s * s;
    const float shift = static_cast<float>(s * kScaleA), keep_x = static_cast<float>(keep) * kScaleA;
    if (wave < blocks) {
#pragma unroll
      for (int j = 0; j < NB; ++j) {
        if (j >= blocks) continue;
        if (j == wave)
#pragma unroll
          for (int e = 0; e < 4; ++e) g[j][e] -= 4 * l4 + e == l16 ? shift : 0.f;
        const half4 h = put(g_hi, p0 + l16, 16 * j + 4 * l4, g[j]);
        if constexpr (FULL) put_low(g_lo, p0 + l16, 16 * j + 4 * l4, g[j], h);
      }
    }
    __syncthreads();
    if (wave < blocks)
      for (int t = 0; t < rp; t += 32) {
        const half8 q = along(g_hi, p0, t);
        if constexpr (FULL) {
          const half8 ql = along(g_lo, p0, t);
#pragma unroll
          for (int j = 0; j < NB; ++j) {
            const half8 p = along(g_hi, 16 * j, t), pl = along(g_lo, 16 * j, t);
            mul(p, q, f[j]);
            mul(p, ql, f[j]);
            mul(pl, q, f[j]);
          }
        } else {
#pragma unroll
          for (int j = 0; j < NB; ++j) mul(along(g_hi, 16 * j, t), q, f[j]);
        }
      }
    __syncthreads();
    if (wave < blocks) {
      const float lin = static_cast<float>(cb + 2.0 * cc * s), quadratic = static_cast<float>(cc) / kScaleA;
#pragma unroll
      for (int j = 0; j < NB; ++j) {
        if (j >= blocks) continue;
#pragma unroll
        for (int e = 0; e < 4; ++e) f[j][e] = lin * g[j][e] + quadratic * f[j][e];
        if (FULL && j == wave)
#pragma unroll
          for (int e = 0; e < 4; ++e) f[j][e] += 4 * l4 + e == l16 ? keep_x : 0.f;
        const half4 h = put(g_hi, p0 + l16, 16 * j + 4 * l4, f[j]);
        if constexpr (FULL) put_low(g_lo, p0 + l16, 16 * j + 4 * l4, f[j], h);
      }
    }
    __syncthreads();
    f32x4 x[kRows][NB];  // lane l: X^T[16 (wave + 8 t) + l16][16 j + 4 l4 ..]
#pragma unroll
    for (int t = 0; t < kRows; ++t) {
      const int q0 = 16 * (wave + t * kWaves);
#pragma unroll
      for (int j = 0; j < NB; ++j) x[t][j] = f32x4{0.f, 0.f, 0.f, 0.f};
      if (q0 >= cp) continue;
      if constexpr (!FULL) {
        // the term (a + bs + cs^2) X, from both halves as they are
#pragma unroll
        for (int j = 0; j < NB; ++j) {
          const int from = (q0 + l16) * pitch + 16 * j + 4 * l4;
          const half4 h = *reinterpret_cast<const half4*>(x_hi + from), l = *reinterpret_cast<const half4*>(x_lo + from);
#pragma unroll
          for (int e = 0; e < 4; ++e) x[t][j][e] = keep_x * join(h, l, e);
        }
      }
      for (int kk = 0; kk < rp; kk += 32) {
        const half8 q = along(x_hi, q0, kk);
        if constexpr (FULL) {
          const half8 ql = along(x_lo, q0, kk);
#pragma unroll
          for (int j = 0; j < NB; ++j) {
            const half8 p = along(g_hi, 16 * j, kk), pl = along(g_lo, 16 * j, kk);
            mul(p, q, x[t][j]);
            mul(p, ql, x[t][j]);
            mul(pl, q, x[t][j]);
          }
        } else {
#pragma unroll
          for (int j = 0; j < NB; ++j) mul(along(g_hi, 16 * j, kk), q, x[t][j]);
        }
      }
    }
    __syncthreads();
#pragma unroll
    for (int t = 0; t < kRows; ++t) {
      const int q0 = 16 * (wave + t * kWaves);
      if (q0 >= cp) continue;
#pragma unroll
      for (int j = 0; j < NB; ++j) {
        if (j >= blocks) continue;
        x[t][j] *= 1.f / kScaleA;
        if (k + 1 < steps) {
          const half4 h = put(x_hi, q0 + l16, 16 * j + 4 * l4, x[t][j]);
          put_low(x_lo, q0 + l16, 16 * j + 4 * l4, x[t][j], h);
        } else {
          *reinterpret_cast<f32x4*>(o + (q0 + l16) * pitch + 16 * j + 4 * l4) = x[t][j];
        }
      }
    }
    __syncthreads();
  }

  bool rollback = false;
  if constexpr (SOURCE == kSourceOuter) rollback = a.rec->rollback;
  const double step = a.lr * mt.scale;
  constexpr int kBatch = 8;  // reads under way
  Walk from(threadIdx.x, mt.cols);
  for (int base = threadIdx.x; base < n; base += kBatch * kThreads) {
    float p[kBatch];
#pragma unroll
    for (int t = 0; t < kBatch; ++t) {
      const int e = base + t * kThreads;
      const int64_t i = mt.offset + e;
      p[t] = 0.f;
      if (e < n && SOURCE != kSourcePlain) p[t] = SOURCE == kSourceLocal ? load_one<BF16>(a.out, i) : a.theta[i];
    }
#pragma unroll
    for (int t = 0; t < kBatch; ++t) {
      const int e = base + t * kThreads;
      const int64_t i = mt.offset + e;
      const int row = from.row, col = from.col;
      from.next();
      if (e >= n) continue;
      const float v = o[mt.tall ? row * pitch + col : col * pitch + row] * (1.f / kScaleX);
      if constexpr (SOURCE == kSourcePlain) {
        store_one<BF16>(a.out, i, v);
      } else if constexpr (SOURCE == kSourceLocal) {
        store_one<BF16>(a.out, i,
                        static_cast<float>(fma(a.keep, static_cast<double>(p[t]), -step * static_cast<double>(v))));
      } else {
        if (!rollback) {
          p[t] = static_cast<float>(fma(-step, static_cast<double>(v), static_cast<double>(p[t])));
          a.theta[i] = p[t];
        }
        for (int j = 0; j < a.workers; ++j) store_one<BF16>(reps.p[j], i, p[t]);
      }
    }
  }
}

template <int SOURCE, bool BF16, bool FULL>
hipError_t launch_small(const OrthoCall& call, const OrthoMat* mats, int count, int widest, const SmallCoef& coef,
                        int steps, hipStream_t stream) {
  const OrthoArgs a = args_of(call);
  const RepPtrs r = reps_of(call);
#define EDIT_SMALL(NB) ortho_small_kernel<SOURCE, BF16, FULL, NB><<<count, kOrthoSmallThreads, 0, stream>>>(a, r, mats, coef, steps)
  if (widest <= 32) EDIT_SMALL(2);
  else if (widest <= 64) EDIT_SMALL(4);
  else EDIT_SMALL(8);
#undef EDIT_SMALL
  return hipGetLastError();
}

}  // namespace

hipError_t launch_ortho_small(bool full, const OrthoCall& call, const OrthoMat* mats, int count, int widest,
                              const OrthoCoef* coef, int steps, hipStream_t stream) {
  if (count == 0) return hipSuccess;
  if (steps > EDIT_ORTHO_MAX_STEPS || widest > kOrthoSmallSide) return hipErrorInvalidValue;
  SmallCoef sc = {};
  for (int k = 0; k < steps; ++k) sc.v[k][0] = coef[k].a, sc.v[k][1] = coef[k].b, sc.v[k][2] = coef[k].c;
#define EDIT_SMALL_OF(S, B)                                                     \
  (full ? launch_small<S, B, true>(call, mats, count, widest, sc, steps, stream) \
        : launch_small<S, B, false>(call, mats, count, widest, sc, steps, stream))
  switch (call.source) {
    case kSourcePlain: return call.bf16 ? EDIT_SMALL_OF(kSourcePlain, true) : EDIT_SMALL_OF(kSourcePlain, false);
    case kSourceLocal: return call.bf16 ? EDIT_SMALL_OF(kSourceLocal, true) : EDIT_SMALL_OF(kSourceLocal, false);
    case kSourceOuter: return call.bf16 ? EDIT_SMALL_OF(kSourceOuter, true) : EDIT_SMALL_OF(kSourceOuter, false);
  }
#undef EDIT_SMALL_OF
  return hipErrorInvalidValue;
}

}  // namespace edit
