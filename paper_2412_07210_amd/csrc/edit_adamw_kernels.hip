// Device kernels of the AdamW step over many tensors (include/edit_outer.h,
// "AdamW"):
//
//   adamw_norm     streams the gradients once: partial sums of g^2 in fp64;
//   adamw_sum      their sum, in a fixed order;
//   adamw_small    both for few gradients, in one block;
//   adamw_decide   the sum, the clip, whether the call is left out, the step count
//                  and the factors that the update goes by;
//   adamw_step     streams parameters, gradients and states once;
//   adamw_fused    decides and streams, for calls of few blocks;
//   adamw_convert  fp32 states to 8-bit ones and back.
//
// All of them are bound by memory.  m and v are taken in fp64 and rounded once
// to fp32, so that what is rounded to 8 bits afterwards does not depend on the
// order of operations; fp64 multiply-adds run at the rate of fp32 ones here.
#include <type_traits>

#include "edit_adamw_internal.h"

namespace edit {
namespace {

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

// The first 64 bits behind the point of sqrt(2), the last one set, and of sqrt(3).
constexpr uint64_t kMixA = 0x6A09E667F3BCC909ull, kMixB = 0xBB67AE8584CAA73Bull;

__host__ __device__ __forceinline__ uint64_t mix(uint64_t z) {
  z = (z ^ (z >> 32)) * kMixA;
  z = (z ^ (z >> 29)) * kMixB;
  return z ^ (z >> 32);
}

// 32 random bits of an element: `mixed`, its low word ^ the key's; k1: the high
// words of both.
__device__ __forceinline__ uint32_t random_word(uint32_t mixed, uint32_t k1) {
  uint32_t x = mixed * 0xBB67AE85u;
  x = __builtin_amdgcn_bitop3_b32(x, x >> 17, k1, 0x96) * 0x6A09E667u;  // x ^ (x >> 17) ^ k1
  return x ^ (x >> 15);
}
__device__ __forceinline__ uint32_t second_word(uint32_t w, uint32_t k0) {
  const uint32_t y = (w + k0) * 0x9E3779B1u;
  return y ^ (y >> 15);
}

// V elements of a buffer as they lie in memory.
template <bool BF16, int V>
struct RawOf {
  typedef u32x4 T;  // 8 bf16 or 4 fp32
  static_assert(V == (BF16 ? 8 : 4), "16 bytes, or 4 bf16");
};
template <>
struct RawOf<true, 4> {
  typedef u32x2 T;
};
template <bool BF16, int V>
using Raw = typename RawOf<BF16, V>::T;

// Elements [at, at + V) behind `base`, zeros from `left` > 0 on; FULL: all of them
// are there.  Parameters and gradients begin at any element.  `base` is the same in
// all lanes and `at` short, so that an address is one register.  Next to the end
// the elements are loaded one by one, the last one in place of those behind it, so
// that no load waits for a branch.
template <bool FULL, bool BF16, int V, bool CACHED = false>
__device__ __forceinline__ Raw<BF16, V> load_raw(const void* base, uint32_t at, uint32_t left) {
  typedef Raw<BF16, V> T;
  typedef T T_any __attribute__((aligned(BF16 ? 2 : 4)));
  typedef typename std::conditional<BF16, uint16_t, uint32_t>::type E;
  const E* p = static_cast<const E*>(base);
  if constexpr (FULL && CACHED) return *reinterpret_cast<const T_any*>(p + at);
  if constexpr (FULL) return __builtin_nontemporal_load(reinterpret_cast<const T_any*>(p + at));
  T raw = {};
#pragma unroll
  for (int e = 0; e < V; ++e) {
    const bool in = at + e < left;
    const uint32_t x = p[in ? at + e : left - 1];
    raw[BF16 ? e >> 1 : e] |= (in ? x : 0u) << (BF16 ? 16 * (e & 1) : 0);
  }
  return raw;
}
template <bool FULL, bool BF16, int V>
__device__ __forceinline__ void store_raw(void* base, uint32_t at, uint32_t left, Raw<BF16, V> raw) {
  typedef Raw<BF16, V> T_any __attribute__((aligned(BF16 ? 2 : 4)));
  typedef typename std::conditional<BF16, uint16_t, uint32_t>::type E;
  E* p = static_cast<E*>(base);
  if constexpr (FULL) {
    __builtin_nontemporal_store(raw, reinterpret_cast<T_any*>(p + at));
  } else {
#pragma unroll
    for (int e = 0; e < V; ++e)
      if (at + e < left) p[at + e] = static_cast<E>(BF16 ? raw[e >> 1] >> (16 * (e & 1)) : raw[e]);
  }
}
// Element `at` of a buffer, for all lanes.
template <bool BF16>
__device__ __forceinline__ const void* element_at(const void* base, int64_t at) {
  return static_cast<const char*>(base) + at * (BF16 ? 2 : 4);
}
template <bool BF16>
__device__ __forceinline__ void* element_at(void* base, int64_t at) {
  return static_cast<char*>(base) + at * (BF16 ? 2 : 4);
}
template <bool BF16, int V>
__device__ __forceinline__ float element(const Raw<BF16, V>& raw, int e) {
  if constexpr (BF16) return __uint_as_float((e & 1) ? (raw[e >> 1] & 0xffff0000u) : (raw[e >> 1] << 16));
  return __uint_as_float(raw[e]);
}

// V codes.
template <int V>
struct CodesOf {
  typedef unsigned int T __attribute__((ext_vector_type(V / 4)));
};
template <int V>
using Codes = typename CodesOf<V>::T;

template <bool FULL, int V>
__device__ __forceinline__ Codes<V> load_codes(const void* base, uint32_t at, uint32_t left) {
  const uint8_t* p = static_cast<const uint8_t*>(base);
  if constexpr (FULL) return __builtin_nontemporal_load(reinterpret_cast<const Codes<V>*>(p + at));
  Codes<V> raw = {};
#pragma unroll
  for (int e = 0; e < V; ++e) {
    const bool in = at + e < left;
    const uint32_t x = p[in ? at + e : left - 1];
    raw[e >> 2] |= (in ? x : 0u) << (8 * (e & 3));
  }
  return raw;
}
template <bool FULL, int V>
__device__ __forceinline__ void store_codes(void* base, uint32_t at, uint32_t left, Codes<V> raw) {
  uint8_t* p = static_cast<uint8_t*>(base);
  if constexpr (FULL) {
    __builtin_nontemporal_store(raw, reinterpret_cast<Codes<V>*>(p + at));
  } else {
#pragma unroll
    for (int e = 0; e < V; ++e)
      if (at + e < left) p[at + e] = static_cast<uint8_t>(raw[e >> 2] >> (8 * (e & 3)));
  }
}
// Index of the scale of element `at`, the last one's from `left` on.
template <bool FULL>
__device__ __forceinline__ uint32_t scale_index(uint32_t at, uint32_t left) {
  return (FULL || at < left ? at : left - 1) / EDIT_ADAMW_BLOCK;
}
template <int V>
__device__ __forceinline__ void decode(const Codes<V>& raw, float (&x)[V]) {
#pragma unroll
  for (int h = 0; h < V / 4; ++h) {
    const f32x2 a = __builtin_amdgcn_cvt_pk_f32_fp8(raw[h], false), b = __builtin_amdgcn_cvt_pk_f32_fp8(raw[h], true);
    x[4 * h] = a[0], x[4 * h + 1] = a[1], x[4 * h + 2] = b[0], x[4 * h + 3] = b[1];
  }
}

template <int CTRL>
__device__ __forceinline__ uint32_t dpp_max(uint32_t x) {
  const uint32_t y = __builtin_amdgcn_update_dpp(0, x, CTRL, 0xf, 0xf, true);
  return x > y ? x : y;
}
// Largest of the 256 / V lanes that share a scale.
template <int V>
__device__ __forceinline__ uint32_t block_max(uint32_t x) {
  static_assert(EDIT_ADAMW_BLOCK == 32 * V || EDIT_ADAMW_BLOCK == 64 * V, "half a wave or a whole one");
  x = dpp_max<0xB1>(x);   // quad_perm 1 0 3 2
  x = dpp_max<0x4E>(x);   // quad_perm 2 3 0 1
  x = dpp_max<0x141>(x);  // row_half_mirror
  x = dpp_max<0x140>(x);  // row_mirror
  const auto r = __builtin_amdgcn_permlane16_swap(x, x, false, false);
  x = max(r[0], r[1]);
  if constexpr (EDIT_ADAMW_BLOCK == 64 * V) {
    const auto s = __builtin_amdgcn_permlane32_swap(x, x, false, false);
    x = max(s[0], s[1]);
  }
  return x;
}

// The exponent field of the block's largest finite |x|, at least 8 (so that
// scale and 1 / scale are normal numbers).  SIGNED: x has a sign; v has none.
template <bool SIGNED, int V>
__device__ __forceinline__ uint32_t block_exponent(const float (&x)[V]) {
  uint32_t top = 0;
  if constexpr (SIGNED) {
    float t = 0.f;
#pragma unroll
    for (int e = 0; e < V; ++e) t = fmaxf(t, fabsf(x[e]));  // leaves a NaN out
    top = __float_as_uint(t);
  } else {
#pragma unroll
    for (int e = 0; e < V; ++e) top = max(top, __float_as_uint(x[e]));
  }
  top = block_max<V>(top);
  if (__builtin_expect(top >= 0x7f800000u, 0)) {  // all lanes of the block alike
    top = 0;
#pragma unroll
    for (int e = 0; e < V; ++e) {
      const uint32_t a = __float_as_uint(x[e]) & 0x7fffffffu;
      top = max(top, a < 0x7f800000u ? a : 0u);
    }
    top = block_max<V>(top);
  }
  return max(top >> 23, 8u);
}
__device__ __forceinline__ float scale_of(uint32_t exponent) { return __uint_as_float((exponent - 7) << 23); }

// x to 8 bits.  The conversion divides by the scale, adds the top 20 bits of its
// random operand below the last place kept and cuts: q floor(|y| / q + u).  LEAST:
// |y| is 2^-9 at least, for an x without a sign.
template <bool LEAST, int V>
__device__ __forceinline__ Codes<V> encode(const float (&x)[V], uint32_t exponent, const uint32_t (&word)[V]) {
  const float scale = scale_of(exponent);
  const uint32_t least = __float_as_uint(scale * 0x1p-9f);  // subnormal down to 2^-135; products keep those
  Codes<V> raw = {};
#pragma unroll
  for (int h = 0; h < V / 4; ++h) {
    int w;
#define EDIT_ADAMW_CODE(I)                                                             \
  {                                                                                    \
    float y = x[4 * h + I];                                                            \
    uint32_t r = word[4 * h + I];                                                      \
    if constexpr (LEAST) {                                                             \
      y = __uint_as_float(max(__float_as_uint(y), least)); /* as bits: keeps a NaN */  \
      r = __builtin_amdgcn_alignbit(r, r, 16);                                         \
    }                                                                                  \
    if constexpr (I == 0) w = r; /* any register that is free: four bytes follow */    \
    w = __builtin_amdgcn_cvt_scalef32_sr_fp8_f32(w, y, r, scale, I);                   \
  }
    EDIT_ADAMW_CODE(0) EDIT_ADAMW_CODE(1) EDIT_ADAMW_CODE(2) EDIT_ADAMW_CODE(3)
#undef EDIT_ADAMW_CODE
    raw[h] = w;
  }
  return raw;
}

// fp32 values as elements of a buffer: bf16 rounded to nearest, or to
// q floor(|x| / q + u), u the top 16 bits of `word`.
template <bool BF16, bool SR, int V>
__device__ __forceinline__ Raw<BF16, V> rounded(const float (&x)[V], const uint32_t (&word)[V]) {
  Raw<BF16, V> raw;
  if constexpr (BF16) {
#pragma unroll
    for (int e = 0; e < V; e += 2) {
      bf16x2_t h;
      if constexpr (SR) {
        h = __builtin_bit_cast(bf16x2_t, word[e]);  // any register that is free: both halves follow
        h = __builtin_amdgcn_cvt_sr_bf16_f32(h, x[e], word[e], false);
        h = __builtin_amdgcn_cvt_sr_bf16_f32(h, x[e + 1], word[e + 1], true);
      } else {
        const f32x2 f = {x[e], x[e + 1]};
        h = __builtin_convertvector(f, bf16x2_t);  // RNE
      }
      raw[e >> 1] = __builtin_bit_cast(uint32_t, h);
    }
  } else {
#pragma unroll
    for (int e = 0; e < V; ++e) raw[e] = __float_as_uint(x[e]);
  }
  return raw;
}

// Sum over the block's threads, in a fixed order, in every thread of wave 0.
template <int THREADS>
__device__ __forceinline__ double block_sum(double x) {
  __shared__ double part[THREADS / 64];
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) x += __shfl_xor(x, d);
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = x;
  __syncthreads();
  x = 0.0;
#pragma unroll
  for (int w = 0; w < THREADS / 64; ++w) x += part[w];
  return x;
}

// Every stride-th chunk from c on, below `end`, by THREADS threads; first: the
// table's, a lane three of them; CACHED: the update pass reads them again soon.
template <bool BF16, bool CACHED, int THREADS>
__device__ __forceinline__ void norm_chunks(const AdamNormTable& tab, const int (&first)[kAdamNormTensors / 64], int stride, int end,
                                            int& c, double (&sum)[2]) {
  constexpr int V = BF16 ? 8 : 4, chunk = adamw_norm_chunk(BF16, THREADS);
  const int thread = threadIdx.x % THREADS;
  static_assert(kAdamNormTensors == 192, "three words of first[] a lane");
  auto load = [&](int i, u32x4 (&raw)[kAdamNormVecs]) {
    int k = -1;
#pragma unroll
    for (int h = 0; h < kAdamNormTensors / 64; ++h) k += __popcll(__ballot(first[h] <= i));
    const int begin = __builtin_amdgcn_readlane(k < 64 ? first[0] : k < 128 ? first[1] : first[2], k & 63);
    const int64_t at = static_cast<int64_t>(i - begin) * chunk;
    const uint32_t left = static_cast<uint32_t>(min(tab.numel[k] - at, static_cast<int64_t>(chunk)));
    const void* g = element_at<BF16>(tab.grad[k], at);
    if (left == chunk) {
#pragma unroll
      for (int u = 0; u < kAdamNormVecs; ++u) raw[u] = load_raw<true, BF16, V, CACHED>(g, (u * THREADS + thread) * V, left);
    } else {
#pragma unroll
      for (int u = 0; u < kAdamNormVecs; ++u) raw[u] = load_raw<false, BF16, V>(g, (u * THREADS + thread) * V, left);
    }
  };
  if (c >= end) return;
  u32x4 raw[kAdamNormVecs];
  load(c, raw);
  for (; c < end; c += stride) {
    u32x4 next[kAdamNormVecs] = {};
    if (c + stride < end) load(c + stride, next);
#pragma unroll
    for (int u = 0; u < kAdamNormVecs; ++u) {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        if constexpr (BF16) {
          const double x = __uint_as_float(raw[u][e] << 16), y = __uint_as_float(raw[u][e] & 0xffff0000u);
          sum[0] = __builtin_fma(x, x, sum[0]);
          sum[1] = __builtin_fma(y, y, sum[1]);
        } else {
          const double x = __uint_as_float(raw[u][e]);
          sum[e & 1] = __builtin_fma(x, x, sum[e & 1]);
        }
      }
      raw[u] = next[u];
    }
  }
}

// Reads 2 or 4 bytes an element: 1.23G bf16 ones in 341 us (7.2 TB/s; where a
// chunk's tensor was looked up and its loads waited for before the next one's,
// 439).  Squares are exact in fp64.
template <bool BF16>
__global__ __launch_bounds__(kAdamNormThreads) void adamw_norm_kernel(const AdamNormTable tab, double* partials) {
  int first[kAdamNormTensors / 64];
#pragma unroll
  for (int h = 0; h < kAdamNormTensors / 64; ++h) first[h] = tab.first[64 * h + (threadIdx.x & 63)];
  double sum[2] = {0.0, 0.0};
  int c = blockIdx.x;
  norm_chunks<BF16, false, kAdamNormThreads>(tab, first, gridDim.x, min(tab.keep, tab.chunks), c, sum);
  norm_chunks<BF16, true, kAdamNormThreads>(tab, first, gridDim.x, tab.chunks, c, sum);
  const double s = block_sum<kAdamNormThreads>(sum[0] + sum[1]);
  if (threadIdx.x == 0) partials[blockIdx.x] = s;
}

__device__ __forceinline__ double sum_partials(const double* partials, int count) {
  double s = 0.0;
  for (int i = threadIdx.x; i < count; i += kAdamDecideThreads) s += partials[i];
  return block_sum<kAdamDecideThreads>(s);
}

__global__ __launch_bounds__(kAdamDecideThreads) void adamw_sum_kernel(const double* partials, int count, double* out) {
  const double s = sum_partials(partials, count);
  if (threadIdx.x == 0) *out = s;
}

// x^t by squaring: off by t roundings at most, where x^t itself vanishes beside 1.
__device__ __forceinline__ double power(double x, int64_t t) {
  double r = 1.0;
  for (; t > 0; t >>= 1, x *= x)
    if (t & 1) r *= x;
  return r;
}

// What call number t + 1 goes by, whose S is `s`; r holds the record before it.
__device__ __forceinline__ void decide(double s, int64_t t, const AdamCall& call, const AdamHyper& hyper, AdamRecord& r) {
  constexpr double largest = 1.7976931348623157e308;
  const double lr = call.lr_device ? *call.lr_device : call.lr;
  float clip = 1.f;
  r.skip = !(lr >= 0.0 && lr <= largest);  // one on the device; the host refuses such a number
  if (call.count > 0) {
    r.norm = sqrt(s);
    r.skip |= !(r.norm <= largest);
    if (!r.skip) clip = static_cast<float>(fmin(call.max_norm / (r.norm + EDIT_ADAMW_CLIP_EPS), 1.0));
  }
  if (r.skip) {
    r.skipped += 1;
    r.clip = 0.f;
  } else {
    r.step = t + 1;
    r.clip = clip;
    r.lr_decay = lr * call.weight_decay;
    // lr = 0 of either sign takes the largest numbers: a quotient of zero.  eps stays
    // above what the reciprocal takes as zero, however large lr is.
    const double most = 3.4028234663852886e38, over = lr > 0.0 ? (1.0 - power(hyper.beta1, r.step)) / lr : largest;
    const double scale = 1.0 / sqrt(1.0 - power(hyper.beta2, r.step));
    r.root = static_cast<float>(fmin(over * scale, most));
    r.eps = static_cast<float>(fmin(fmax(over * hyper.eps, 1.2e-38), most));
    // Such a root is below 2^-63: whether, over sqrt(1 - beta2^t), that is above 2^-24
    // of eps.  With an eps of 1e-8 only for beta2 next to 1.
    r.tiny = scale > hyper.eps * 0x1p39;
    r.key = mix(mix(call.seed) + static_cast<uint64_t>(r.step));
  }
}

__global__ __launch_bounds__(kAdamDecideThreads) void adamw_decide_kernel(const AdamCall call, const AdamHyper hyper,
                                                                          const AdamState state) {
  __shared__ int64_t now;
  const double s = sum_partials(call.sums, call.count);
  if (threadIdx.x == 0) {
    AdamRecord r = *state.rec;
    now = state.steps[0];
    decide(s, now, call, hyper, r);
    *state.rec = r;
    if (!r.skip) now = r.step;
  }
  __syncthreads();
  const int64_t t = now;
  for (int i = threadIdx.x; i < state.slots; i += kAdamDecideThreads) state.steps[i] = t;
}

template <bool BF16>
__global__ __launch_bounds__(kAdamSmallThreads) void adamw_small_kernel(const AdamNormTable tab, double* out) {
  int first[kAdamNormTensors / 64];
#pragma unroll
  for (int h = 0; h < kAdamNormTensors / 64; ++h) first[h] = tab.first[64 * h + (threadIdx.x & 63)];
  double sum[2] = {0.0, 0.0};
  int c = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  norm_chunks<BF16, true, 64>(tab, first, kAdamSmallThreads / 64, tab.chunks, c, sum);
  const double s = block_sum<kAdamSmallThreads>(sum[0] + sum[1]);
  if (threadIdx.x == 0) *out = s;
}

// Which tensor, and where in it, a block works.  Blocks are taken from the
// table's end: the norm pass has just read it, and the Infinity Cache still holds
// its gradients.
struct Place {
  int k;       // index of the tensor in the table
  int64_t at;  // first element of the block
};
__device__ __forceinline__ Place place_of(const AdamTable& tab, int chunk) {
  const int b = gridDim.x - 1 - blockIdx.x, first = tab.first[threadIdx.x];
  Place p;
  p.k = __popcll(__ballot(first <= b)) - 1;
  p.at = static_cast<int64_t>(b - __builtin_amdgcn_readlane(first, p.k)) * chunk;
  return p;
}
struct Key {
  uint32_t k0, k1;
};
__device__ __forceinline__ Key key_of(uint64_t key, int tensor, int64_t at) {
  const uint64_t k = mix(key + static_cast<uint64_t>(tensor));
  return {static_cast<uint32_t>(k), static_cast<uint32_t>(k >> 32) ^ (static_cast<uint32_t>(at >> 32) * 0xBB67AE85u)};
}

// The work of one block: U times V elements a lane of every buffer, each time
// next to its neighbour's; FULL: all of them are there.  Bound by memory, which
// moves what the formulas need and up to 4% more (whole lines for a block's few
// scales): 308M elements in fp32 in 1309 us (6.59 TB/s), in bf16 with fp32 states in
// 1040 (6.52); with e4m3 states fp32 in 787 (6.29), bf16 rounded stochastically in 502
// (6.18), where the vector units are busy for 85% of the time too (43 instructions an
// element; two more took 2% more).
template <bool FULL, bool PB, bool GB, bool HELD, bool SR, int V, int U>
__device__ __forceinline__ void step_block(const AdamTensor& t, double decay_factor, int tensor, const AdamHyper& hyper,
                                           const AdamRecord& rec, int64_t begin) {
  if (rec.skip) return;  // here, so that the record is loaded beside the tensor's entry
  void* const pp = element_at<PB>(t.param, begin);
  const void* const gp = element_at<GB>(t.grad, begin);
  void* const mp = static_cast<char*>(t.m) + begin * (HELD ? 1 : 4);
  void* const vp = static_cast<char*>(t.v) + begin * (HELD ? 1 : 4);
  float* const ms = HELD ? t.m_scale + begin / EDIT_ADAMW_BLOCK : nullptr;
  float* const vs = HELD ? t.v_scale + begin / EDIT_ADAMW_BLOCK : nullptr;
  const uint32_t left = static_cast<uint32_t>(min(t.numel - begin, static_cast<int64_t>(kAdamThreads * V * U)));
  uint32_t at[U];
  Raw<PB, V> p_raw[U];
  Raw<GB, V> g_raw[U];
  Raw<false, 4> m_raw[U], v_raw[U];
  Codes<V> m_codes[U], v_codes[U];
  float m_scale[U], v_scale[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    at[u] = u * kAdamThreads * V + threadIdx.x * V;
    p_raw[u] = load_raw<FULL, PB, V>(pp, at[u], left);
    g_raw[u] = load_raw<FULL, GB, V>(gp, at[u], left);
    if constexpr (HELD) {
      m_scale[u] = ms[scale_index<FULL>(at[u], left)];
      v_scale[u] = vs[scale_index<FULL>(at[u], left)];
      m_codes[u] = load_codes<FULL, V>(mp, at[u], left);
      v_codes[u] = load_codes<FULL, V>(vp, at[u], left);
    } else {
      m_raw[u] = load_raw<FULL, false, V>(mp, at[u], left);
      v_raw[u] = load_raw<FULL, false, V>(vp, at[u], left);
    }
  }
  const float clip = rec.clip, root = rec.root, eps = rec.eps;
  const float decay = static_cast<float>(rec.lr_decay * decay_factor);
  const double b1 = hyper.beta1, b2 = hyper.beta2, a1 = 1.0 - b1, a2 = 1.0 - b2;
  const Key key = key_of(rec.key, tensor, begin);  // 2^32 is a multiple of what a block takes
#pragma unroll
  for (int u = 0; u < U; ++u) {
    float m[V], v[V], p[V];
    double keep1 = b1, keep2 = b2;
    if constexpr (HELD) {  // the scale, a power of two, goes with the factor
      decode<V>(m_codes[u], m);
      decode<V>(v_codes[u], v);
      keep1 *= m_scale[u];
      keep2 *= v_scale[u];
    }
#pragma unroll
    for (int e = 0; e < V; ++e) {
      if constexpr (!HELD) {
        m[e] = element<false, V>(m_raw[u], e);
        v[e] = element<false, V>(v_raw[u], e);
      }
      p[e] = element<PB, V>(p_raw[u], e);
      const double g = clip * element<GB, V>(g_raw[u], e);
      m[e] = static_cast<float>(__builtin_fma(keep1, static_cast<double>(m[e]), a1 * g));
      v[e] = static_cast<float>(__builtin_fma(keep2, static_cast<double>(v[e]), a2 * g * g));
    }
    // The hardware's square root is off by one place and takes values below 2^-126
    // as zero.
    auto update = [&](auto tiny) {
#pragma unroll
      for (int e = 0; e < V; ++e) {
        const bool up = tiny && v[e] < 0x1p-126f;
        const float s = __builtin_amdgcn_sqrtf(up ? v[e] * 0x1p64f : v[e]);
        const float d = __builtin_fmaf(up ? s * 0x1p-32f : s, root, eps);
        p[e] -= __builtin_fmaf(decay, p[e], m[e] * __builtin_amdgcn_rcpf(d));
      }
    };
    if (__builtin_expect(rec.tiny, 0))  // all lanes alike
      update(std::true_type{});
    else
      update(std::false_type{});
    uint32_t word[V], second[V];
    if constexpr (HELD || SR) {
      const uint32_t base = (static_cast<uint32_t>(begin) + at[u]) ^ key.k0;  // both are multiples of V: + e is ^ e
#pragma unroll
      for (int e = 0; e < V; ++e) {
        word[e] = random_word(base ^ e, key.k1);
        if constexpr (SR) second[e] = second_word(word[e], key.k0);
      }
    }
    store_raw<FULL, PB, V>(pp, at[u], left, rounded<PB, SR, V>(p, second));
    if constexpr (HELD) {
      const uint32_t em = block_exponent<true>(m), ev = block_exponent<false>(v);
      store_codes<FULL, V>(vp, at[u], left, encode<true>(v, ev, word));
      store_codes<FULL, V>(mp, at[u], left, encode<false>(m, em, word));
      if (at[u] % EDIT_ADAMW_BLOCK == 0 && (FULL || at[u] < left)) {
        ms[at[u] / EDIT_ADAMW_BLOCK] = scale_of(em);
        vs[at[u] / EDIT_ADAMW_BLOCK] = scale_of(ev);
      }
    } else {
      store_raw<FULL, false, V>(mp, at[u], left, rounded<false, false, V>(m, word));
      store_raw<FULL, false, V>(vp, at[u], left, rounded<false, false, V>(v, word));
    }
  }
}

template <bool PB, bool GB, bool HELD, bool SR, int V, int U>
__device__ __forceinline__ void step_tensor(const AdamTable& tab, const Place& place, const AdamHyper& hyper,
                                            const AdamRecord& r) {
  const AdamTensor t = tab.tensor[place.k];
  const double decay = tab.decay[place.k];
  if (place.at + kAdamThreads * V * U <= t.numel) {
    step_block<true, PB, GB, HELD, SR, V, U>(t, decay, tab.base + place.k, hyper, r, place.at);
  } else {
#pragma unroll 1
    for (int64_t at = place.at; at < t.numel; at += kAdamThreads * V)
      step_block<false, PB, GB, HELD, SR, V, 1>(t, decay, tab.base + place.k, hyper, r, at);
  }
}

// PB, GB: bf16 parameters, gradients; HELD: states in 8 bits; SR: bf16 parameters
// rounded stochastically.
template <bool PB, bool GB, bool HELD, bool SR, int V, int U>
__global__ __launch_bounds__(kAdamThreads, 4) void adamw_step_kernel(const AdamTable tab, const AdamHyper hyper,
                                                                     const AdamRecord* __restrict__ rec) {
  const AdamRecord r = *rec;
  step_tensor<PB, GB, HELD, SR, V, U>(tab, place_of(tab, kAdamThreads * V * U), hyper, r);
}

__device__ __forceinline__ float same(float x) {
  return __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(x)));
}
__device__ __forceinline__ uint64_t same(uint64_t x) {
  return static_cast<uint64_t>(static_cast<uint32_t>(__builtin_amdgcn_readfirstlane(static_cast<uint32_t>(x >> 32)))) << 32 |
         static_cast<uint32_t>(__builtin_amdgcn_readfirstlane(static_cast<uint32_t>(x)));
}
__device__ __forceinline__ double same(double x) {
  return __longlong_as_double(static_cast<int64_t>(same(static_cast<uint64_t>(__double_as_longlong(x)))));
}

// The same with the decision, which comes out alike in every block: S is summed in
// the same order, and t is the block's own.
template <bool PB, bool GB, bool HELD, bool SR, int V, int U>
__global__ __launch_bounds__(kAdamThreads, 4) void adamw_fused_kernel(const AdamTable tab, const AdamHyper hyper,
                                                                      const AdamCall call, const AdamState state, int before) {
  const Place place = place_of(tab, kAdamThreads * V * U);
  const int slot = before + gridDim.x - 1 - blockIdx.x;
  const int64_t t = state.steps[slot];
  double s = 0.0;
  for (int i = threadIdx.x; i < call.count; i += kAdamThreads) s += call.sums[i];
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) s += __shfl_xor(s, d);
  AdamRecord r = {};
  decide(s, t, call, hyper, r);
  if (threadIdx.x == 0) {
    if (!r.skip) state.steps[slot] = r.step;
    if (slot == 0) {  // no other block looks at the record
      AdamRecord out = *state.rec;
      out.skipped += r.skipped;
      if (call.count > 0) out.norm = r.norm;
      out.clip = r.clip;
      if (!r.skip) out.step = r.step;
      *state.rec = out;
    }
  }
  r.skip = __builtin_amdgcn_readfirstlane(r.skip);
  r.tiny = __builtin_amdgcn_readfirstlane(r.tiny);
  r.clip = same(r.clip), r.root = same(r.root), r.eps = same(r.eps);
  r.lr_decay = same(r.lr_decay), r.key = same(r.key);
  step_tensor<PB, GB, HELD, SR, V, U>(tab, place, hyper, r);
}

template <bool FULL, bool PACK, int V, int U>
__device__ __forceinline__ void convert_block(const AdamTensor& t, int tensor, uint64_t key64, int64_t begin) {
  void* const m32 = element_at<false>(t.param, begin);
  void* const v32 = element_at<false>(const_cast<void*>(t.grad), begin);
  void* const mp = static_cast<char*>(t.m) + begin;
  void* const vp = static_cast<char*>(t.v) + begin;
  float* const ms = t.m_scale + begin / EDIT_ADAMW_BLOCK;
  float* const vs = t.v_scale + begin / EDIT_ADAMW_BLOCK;
  const uint32_t left = static_cast<uint32_t>(min(t.numel - begin, static_cast<int64_t>(kAdamThreads * V * U)));
  uint32_t at[U];
  Raw<false, V> m_raw[U], v_raw[U];
  Codes<V> m_codes[U], v_codes[U];
  float m_scale[U], v_scale[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    at[u] = u * kAdamThreads * V + threadIdx.x * V;
    if constexpr (PACK) {
      m_raw[u] = load_raw<FULL, false, V>(m32, at[u], left);
      v_raw[u] = load_raw<FULL, false, V>(v32, at[u], left);
    } else {
      m_scale[u] = ms[scale_index<FULL>(at[u], left)];
      v_scale[u] = vs[scale_index<FULL>(at[u], left)];
      m_codes[u] = load_codes<FULL, V>(mp, at[u], left);
      v_codes[u] = load_codes<FULL, V>(vp, at[u], left);
    }
  }
  const Key key = key_of(key64, tensor, begin);
#pragma unroll
  for (int u = 0; u < U; ++u) {
    float m[V], v[V];
    uint32_t word[V];
    if constexpr (PACK) {
      const uint32_t base = (static_cast<uint32_t>(begin) + at[u]) ^ key.k0;
#pragma unroll
      for (int e = 0; e < V; ++e) {
        m[e] = element<false, V>(m_raw[u], e);
        // -0 and a negative v, which no step makes, are taken by their size
        v[e] = fabsf(element<false, V>(v_raw[u], e));
        word[e] = random_word(base ^ e, key.k1);
      }
      const uint32_t em = block_exponent<true>(m), ev = block_exponent<false>(v);
      store_codes<FULL, V>(vp, at[u], left, encode<true>(v, ev, word));
      store_codes<FULL, V>(mp, at[u], left, encode<false>(m, em, word));
      if (at[u] % EDIT_ADAMW_BLOCK == 0 && (FULL || at[u] < left)) {
        ms[at[u] / EDIT_ADAMW_BLOCK] = scale_of(em);
        vs[at[u] / EDIT_ADAMW_BLOCK] = scale_of(ev);
      }
    } else {
      decode<V>(m_codes[u], m);
      decode<V>(v_codes[u], v);
#pragma unroll
      for (int e = 0; e < V; ++e) m[e] *= m_scale[u], v[e] *= v_scale[u];
      store_raw<FULL, false, V>(m32, at[u], left, rounded<false, false, V>(m, word));
      store_raw<FULL, false, V>(v32, at[u], left, rounded<false, false, V>(v, word));
    }
  }
}

template <bool PACK, int V, int U>
__global__ __launch_bounds__(kAdamThreads) void adamw_convert_kernel(const AdamTable tab, uint64_t key) {
  constexpr int chunk = kAdamThreads * V * U;
  static_assert(chunk == adamw_convert_chunk(PACK), "as the tables count blocks");
  const Place place = place_of(tab, chunk);
  const AdamTensor t = tab.tensor[place.k];
  if (place.at + chunk <= t.numel) {
    convert_block<true, PACK, V, U>(t, tab.base + place.k, key, place.at);
  } else {
#pragma unroll 1
    for (int64_t at = place.at; at < t.numel; at += kAdamThreads * V)
      convert_block<false, PACK, V, 1>(t, tab.base + place.k, key, at);
  }
}

// The launch's own status: hipGetLastError() would also give what an earlier call of the program left.
template <typename... A>
hipError_t launch(void (*kernel)(A...), int blocks, int threads, int lds, hipStream_t stream, A... args) {
  void* at[] = {const_cast<void*>(static_cast<const void*>(&args))...};
  return hipLaunchKernel(reinterpret_cast<const void*>(kernel), dim3(blocks), dim3(threads), at, lds, stream);
}

template <bool PB, bool GB, bool HELD, bool SR>
hipError_t step(int blocks, const AdamTable& table, const AdamHyper& hyper, const AdamState& state, const AdamCall* call,
                int before, hipStream_t stream) {
  constexpr int V = adamw_vec(PB, GB, HELD), U = adamw_times(HELD), resident = adamw_resident(PB, GB, HELD);
  constexpr int lds = resident == 32 ? 0 : lds_for_blocks(resident, 0, kLdsPerCu);
  static_assert(resident == 32 || lds_blocks(lds, kLdsPerCu) == resident, "a number that LDS can leave room for");
  if (call)
    return launch<AdamTable, AdamHyper, AdamCall, AdamState, int>(adamw_fused_kernel<PB, GB, HELD, SR, V, U>, blocks, kAdamThreads,
                                                                  lds, stream, table, hyper, *call, state, before);
  return launch<AdamTable, AdamHyper, const AdamRecord*>(adamw_step_kernel<PB, GB, HELD, SR, V, U>, blocks, kAdamThreads, lds,
                                                         stream, table, hyper, state.rec);
}

}  // namespace

uint64_t adamw_key(uint64_t seed, uint64_t t) { return mix(mix(seed) + t); }

hipError_t launch_adamw_norm(bool bf16, int blocks, const AdamNormTable& table, double* partials, hipStream_t stream) {
  return launch<AdamNormTable, double*>(bf16 ? adamw_norm_kernel<true> : adamw_norm_kernel<false>, blocks,
                                        kAdamNormThreads, 0, stream, table, partials);
}

hipError_t launch_adamw_small(bool bf16, const AdamNormTable& table, double* out, hipStream_t stream) {
  return launch<AdamNormTable, double*>(bf16 ? adamw_small_kernel<true> : adamw_small_kernel<false>, 1, kAdamSmallThreads, 0,
                                        stream, table, out);
}

hipError_t launch_adamw_sum(const double* partials, int count, double* out, hipStream_t stream) {
  return launch<const double*, int, double*>(adamw_sum_kernel, 1, kAdamDecideThreads, 0, stream, partials, count, out);
}

hipError_t launch_adamw_decide(const AdamCall& call, const AdamHyper& hyper, const AdamState& state, hipStream_t stream) {
  return launch<AdamCall, AdamHyper, AdamState>(adamw_decide_kernel, 1, kAdamDecideThreads, 0, stream, call, hyper, state);
}

hipError_t launch_adamw_step(const AdamKind& kind, int blocks, const AdamTable& table, const AdamHyper& hyper,
                             const AdamState& state, const AdamCall* call, int before, hipStream_t stream) {
#define EDIT_ADAMW_KIND(PB, GB, HELD, SR)                                                                        \
  if (kind.param_bf16 == PB && kind.grad_bf16 == GB && kind.held == HELD && kind.stochastic == SR)               \
    return step<PB, GB, HELD, SR>(blocks, table, hyper, state, call, before, stream);
  EDIT_ADAMW_KIND(true, true, true, true)
  EDIT_ADAMW_KIND(true, true, false, true)
  EDIT_ADAMW_KIND(true, false, true, true)
  EDIT_ADAMW_KIND(true, false, false, true)
  EDIT_ADAMW_KIND(true, true, true, false)
  EDIT_ADAMW_KIND(true, true, false, false)
  EDIT_ADAMW_KIND(true, false, true, false)
  EDIT_ADAMW_KIND(true, false, false, false)
  EDIT_ADAMW_KIND(false, true, true, false)
  EDIT_ADAMW_KIND(false, true, false, false)
  EDIT_ADAMW_KIND(false, false, true, false)
  EDIT_ADAMW_KIND(false, false, false, false)
#undef EDIT_ADAMW_KIND
  return hipErrorInvalidValue;
}

hipError_t launch_adamw_convert(bool pack, int blocks, const AdamTable& table, uint64_t key, hipStream_t stream) {
  constexpr int lds = lds_for_blocks(kAdamUnpackResident, 0, kLdsPerCu);
  static_assert(lds_blocks(lds, kLdsPerCu) == kAdamUnpackResident, "a number that LDS can leave room for");
  return launch<AdamTable, uint64_t>(pack ? adamw_convert_kernel<true, 4, adamw_convert_times(true)>
                                          : adamw_convert_kernel<false, 4, adamw_convert_times(false)>,
                                     blocks, kAdamThreads, pack ? 0 : lds, stream, table, key);
}

}  // namespace edit
