// Device kernels of the AdamW step over many tensors (include/edit_outer.h,
// "AdamW"):
//
//   adamw_norm     streams the gradients once: partial sums of g^2 in fp64;
//   adamw_sum      their sum, in a fixed order;
//   adamw_decide   the same sum, the clip, whether the call is left out, the
//                  step count and the factors that the update goes by;
//   adamw_step     streams parameters, gradients and states once;
//   adamw_convert  fp32 states to 8-bit ones and back.
//
// All of them are bound by memory.  m and v are taken in fp64 and rounded once
// to fp32, so that what is rounded to 8 bits afterwards does not depend on the
// order of operations; fp64 multiply-adds run at the rate of fp32 ones here.
#include "edit_adamw_internal.h"

namespace edit {
namespace {

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
typedef unsigned int u32x1 __attribute__((ext_vector_type(1)));
typedef u32x4 u32x4_any __attribute__((aligned(4)));  // parameters and gradients begin at any element
typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

// The first 64 bits behind the point of sqrt(2) and of sqrt(3).
constexpr uint64_t kMixA = 0x6A09E667F3BCC909ull, kMixB = 0xBB67AE8584CAA73Bull;

__host__ __device__ __forceinline__ uint64_t mix(uint64_t z) {
  z = (z ^ (z >> 32)) * kMixA;
  z = (z ^ (z >> 29)) * kMixB;
  return z ^ (z >> 32);
}

// 32 random bits of the element whose low word is `element`; key: of its
// tensor, its high word mixed with the element's.
__device__ __forceinline__ uint32_t random_word(uint32_t element, uint32_t k0, uint32_t k1) {
  uint32_t x = (element ^ k0) * 0xBB67AE85u;
  x = (x ^ (x >> 17) ^ k1) * 0x6A09E667u;
  return x ^ (x >> 15);
}
__device__ __forceinline__ uint32_t second_word(uint32_t w, uint32_t k0) {
  const uint32_t y = (w + k0) * 0x9E3779B1u;
  return y ^ (y >> 15);
}

__device__ __forceinline__ uint32_t pack2(float a, float b) {
  const f32x2 f = {a, b};
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(f, bf16x2_t));  // RNE
}

// V elements of 16 bits or of 8, packed.
template <int V>
struct Packed;
template <>
struct Packed<8> {
  typedef u32x4 Half;
  typedef u32x2 Byte;
};
template <>
struct Packed<4> {
  typedef u32x2 Half;
  typedef u32x1 Byte;
};

// Elements [at, at + n) of a buffer, n <= V; zeros behind them.
template <bool BF16, int V>
__device__ __forceinline__ void load_vec(const void* base, int64_t at, int n, float (&x)[V]) {
  if constexpr (BF16) {
    typedef typename Packed<V>::Half Half;
    typedef Half Half_any __attribute__((aligned(2)));
    const uint16_t* p = static_cast<const uint16_t*>(base) + at;
    if (n == V) {
      const Half raw = __builtin_nontemporal_load(reinterpret_cast<const Half_any*>(p));
#pragma unroll
      for (int e = 0; e < V; ++e) {
        const uint32_t w = raw[e >> 1];
        x[e] = __uint_as_float((e & 1) ? (w & 0xffff0000u) : (w << 16));
      }
    } else {
#pragma unroll
      for (int e = 0; e < V; ++e) x[e] = e < n ? __uint_as_float(static_cast<uint32_t>(p[e]) << 16) : 0.f;
    }
  } else {
    const float* p = static_cast<const float*>(base) + at;
    if (n == V) {
#pragma unroll
      for (int h = 0; h < V / 4; ++h) {
        const u32x4 raw = __builtin_nontemporal_load(reinterpret_cast<const u32x4_any*>(p) + h);
#pragma unroll
        for (int e = 0; e < 4; ++e) x[4 * h + e] = __uint_as_float(raw[e]);
      }
    } else {
#pragma unroll
      for (int e = 0; e < V; ++e) x[e] = e < n ? p[e] : 0.f;
    }
  }
}

template <bool BF16, int V>
__device__ __forceinline__ void store_vec(void* base, int64_t at, int n, const float (&x)[V]) {
  if constexpr (BF16) {
    typedef typename Packed<V>::Half Half;
    typedef Half Half_any __attribute__((aligned(2)));
    uint16_t* p = static_cast<uint16_t*>(base) + at;
    Half raw;
#pragma unroll
    for (int e = 0; e < V / 2; ++e) raw[e] = pack2(x[2 * e], x[2 * e + 1]);
    if (n == V) {
      __builtin_nontemporal_store(raw, reinterpret_cast<Half_any*>(p));
    } else {
#pragma unroll
      for (int e = 0; e < V; ++e)
        if (e < n) p[e] = static_cast<uint16_t>(raw[e >> 1] >> (16 * (e & 1)));
    }
  } else {
    float* p = static_cast<float*>(base) + at;
    if (n == V) {
#pragma unroll
      for (int h = 0; h < V / 4; ++h) {
        u32x4 raw;
#pragma unroll
        for (int e = 0; e < 4; ++e) raw[e] = __float_as_uint(x[4 * h + e]);
        __builtin_nontemporal_store(raw, reinterpret_cast<u32x4_any*>(p) + h);
      }
    } else {
#pragma unroll
      for (int e = 0; e < V; ++e)
        if (e < n) p[e] = x[e];
    }
  }
}

// V codes.
template <int V, typename Byte = typename Packed<V>::Byte>
__device__ __forceinline__ Byte load_codes(const void* base, int64_t at, int n) {
  const uint8_t* p = static_cast<const uint8_t*>(base) + at;
  if (n == V) return __builtin_nontemporal_load(reinterpret_cast<const Byte*>(p));
  Byte raw = {};
#pragma unroll
  for (int e = 0; e < V; ++e)
    if (e < n) raw[e >> 2] |= static_cast<uint32_t>(p[e]) << (8 * (e & 3));
  return raw;
}
template <int V, typename Byte = typename Packed<V>::Byte>
__device__ __forceinline__ void store_codes(void* base, int64_t at, int n, Byte raw) {
  uint8_t* p = static_cast<uint8_t*>(base) + at;
  if (n == V) {
    __builtin_nontemporal_store(raw, reinterpret_cast<Byte*>(p));
  } else {
#pragma unroll
    for (int e = 0; e < V; ++e)
      if (e < n) p[e] = static_cast<uint8_t>(raw[e >> 2] >> (8 * (e & 3)));
  }
}
template <int V, typename Byte = typename Packed<V>::Byte>
__device__ __forceinline__ void decode(Byte raw, float scale, float (&x)[V]) {
#pragma unroll
  for (int h = 0; h < V / 4; ++h) {
    const f32x2 a = __builtin_amdgcn_cvt_pk_f32_fp8(raw[h], false), b = __builtin_amdgcn_cvt_pk_f32_fp8(raw[h], true);
    x[4 * h] = a[0] * scale, x[4 * h + 1] = a[1] * scale;
    x[4 * h + 2] = b[0] * scale, x[4 * h + 3] = b[1] * scale;
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
// scale and 1 / scale are normal numbers).
template <int V>
__device__ __forceinline__ uint32_t block_exponent(const float (&x)[V]) {
  uint32_t top = 0;
#pragma unroll
  for (int e = 0; e < V; ++e) top = max(top, __float_as_uint(x[e]) & 0x7fffffffu);
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

// x to 8 bits and their scale.  The conversion adds the top 20 bits of its
// random operand below the last place kept and cuts: q floor(|y| / q + u).
template <bool SECOND, int V>
__device__ __forceinline__ typename Packed<V>::Byte encode(const float (&x)[V], uint32_t exponent,
                                                           const uint32_t (&word)[V]) {
  const float inv = __uint_as_float((261 - exponent) << 23);  // 2^(134 - exponent), exact
  typename Packed<V>::Byte raw = {};
#pragma unroll
  for (int h = 0; h < V / 4; ++h) {
    uint32_t w = 0;
#define EDIT_ADAMW_CODE(I)                                                                            \
  {                                                                                                   \
    float y = x[4 * h + I] * inv;                                                                     \
    uint32_t r = word[4 * h + I];                                                                     \
    if constexpr (SECOND) {                                                                           \
      y = __uint_as_float(max(__float_as_uint(y), 0x3b000000u)); /* v: 2^-9 at least; keeps a NaN */  \
      r = __builtin_amdgcn_alignbit(r, r, 16);                                                        \
    }                                                                                                 \
    w = __builtin_amdgcn_cvt_sr_fp8_f32(y, r, w, I);                                                  \
  }
    EDIT_ADAMW_CODE(0) EDIT_ADAMW_CODE(1) EDIT_ADAMW_CODE(2) EDIT_ADAMW_CODE(3)
#undef EDIT_ADAMW_CODE
    raw[h] = w;
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

// 16 bytes from element `at` of n on; zeros behind them.
template <bool BF16>
__device__ __forceinline__ u32x4 load_raw(const void* base, int64_t at, int64_t n) {
  constexpr int V = BF16 ? 8 : 4;
  if constexpr (BF16) {
    typedef u32x4 u32x4_half __attribute__((aligned(2)));
    const uint16_t* p = static_cast<const uint16_t*>(base) + at;
    if (n - at >= V) return __builtin_nontemporal_load(reinterpret_cast<const u32x4_half*>(p));
    u32x4 raw = {0, 0, 0, 0};
#pragma unroll
    for (int e = 0; e < V; ++e)
      if (at + e < n) raw[e >> 1] |= static_cast<uint32_t>(p[e]) << (16 * (e & 1));
    return raw;
  } else {
    const uint32_t* p = static_cast<const uint32_t*>(base) + at;
    if (n - at >= V) return __builtin_nontemporal_load(reinterpret_cast<const u32x4_any*>(p));
    u32x4 raw = {0, 0, 0, 0};
#pragma unroll
    for (int e = 0; e < V; ++e)
      if (at + e < n) raw[e] = p[e];
    return raw;
  }
}

// Reads 2 or 4 bytes an element: 1.23G bf16 ones in 352 us (7.0 TB/s; where a
// chunk's tensor was looked up and its loads waited for before the next one's,
// 439).  Squares are exact in fp64.
template <bool BF16>
__global__ __launch_bounds__(kAdamNormThreads) void adamw_norm_kernel(const AdamNormTable tab, double* partials) {
  const int lane = threadIdx.x & 63;
  int first[kAdamNormTensors / 64];
#pragma unroll
  for (int h = 0; h < kAdamNormTensors / 64; ++h) first[h] = tab.first[64 * h + lane];
  auto load = [&](int c, u32x4 (&raw)[kAdamNormVecs]) {
    int k = -1;
#pragma unroll
    for (int h = 0; h < kAdamNormTensors / 64; ++h) k += __popcll(__ballot(first[h] <= c));
    const int64_t at = static_cast<int64_t>(c - tab.first[k]) * adamw_norm_chunk(BF16) + threadIdx.x * (BF16 ? 8 : 4);
#pragma unroll
    for (int u = 0; u < kAdamNormVecs; ++u)
      raw[u] = load_raw<BF16>(tab.grad[k], at + u * (adamw_norm_chunk(BF16) / kAdamNormVecs), tab.numel[k]);
  };
  double sum[2] = {0.0, 0.0};
  u32x4 raw[kAdamNormVecs];
  load(blockIdx.x, raw);  // the grid has at most a block a chunk
  for (int c = blockIdx.x; c < tab.chunks; c += gridDim.x) {
    u32x4 next[kAdamNormVecs] = {};
    if (c + static_cast<int>(gridDim.x) < tab.chunks) load(c + gridDim.x, next);
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

__global__ __launch_bounds__(kAdamDecideThreads) void adamw_decide_kernel(const double* partials, int count,
                                                                          const double* sumsq, const AdamCall call,
                                                                          const AdamHyper hyper, AdamRecord* rec) {
  double s = 0.0;
  if (sumsq)
    s = *sumsq;
  else if (count > 0)
    s = sum_partials(partials, count);
  if (threadIdx.x != 0) return;
  AdamRecord r = *rec;
  float clip = 1.f;
  r.skip = 0;
  if (call.check) {
    r.norm = sqrt(s);
    r.skip = !(r.norm <= 1.7976931348623157e308);
    if (!r.skip) clip = static_cast<float>(fmin(call.max_norm / (r.norm + EDIT_ADAMW_CLIP_EPS), 1.0));
  }
  if (r.skip) {
    r.skipped += 1;
    r.clip = 0.f;
  } else {
    const double lr = call.lr_device ? *call.lr_device : call.lr;
    r.step += 1;
    r.clip = clip;
    r.lr_decay = lr * call.weight_decay;
    r.rate = static_cast<float>(lr / (1.0 - power(hyper.beta1, r.step)));
    r.root = static_cast<float>(1.0 / sqrt(1.0 - power(hyper.beta2, r.step)));
    r.key = mix(mix(call.seed) + static_cast<uint64_t>(r.step));
  }
  *rec = r;
}

// Which tensor, and where in it, a block works.  Blocks are taken from the
// table's end: the norm pass has just read it, and the Infinity Cache still holds
// its gradients.
struct Place {
  int k;       // index of the tensor in the table
  int64_t at;  // first element of the block
};
__device__ __forceinline__ Place place_of(const AdamTable& tab, int chunk) {
  const int b = gridDim.x - 1 - blockIdx.x;
  Place p;
  p.k = __popcll(__ballot(tab.first[threadIdx.x] <= b)) - 1;
  p.at = static_cast<int64_t>(b - tab.first[p.k]) * chunk;
  return p;
}
// How many of the V elements from `at` on there are.
template <int V>
__device__ __forceinline__ int here(int64_t numel, int64_t at) {
  const int64_t left = numel - at;
  return left >= V ? V : left > 0 ? static_cast<int>(left) : 0;
}
struct Key {
  uint32_t k0, k1;
};
__device__ __forceinline__ Key key_of(uint64_t key, int tensor, int64_t at) {
  const uint64_t k = mix(key + static_cast<uint64_t>(tensor));
  return {static_cast<uint32_t>(k), static_cast<uint32_t>(k >> 32) ^ (static_cast<uint32_t>(at >> 32) * 0xBB67AE85u)};
}

// One lane: U times V elements of every buffer, each time next to its
// neighbour's.  PB, GB: bf16 parameters, gradients; HELD: states in 8 bits; SR:
// bf16 parameters rounded stochastically.
template <bool PB, bool GB, bool HELD, bool SR, int V, int U>
__global__ __launch_bounds__(kAdamThreads) void adamw_step_kernel(const AdamTable tab, const AdamHyper hyper,
                                                                  const AdamRecord* __restrict__ rec) {
  if (rec->skip) return;
  const Place place = place_of(tab, kAdamThreads * V * U);
  const AdamTensor& t = tab.tensor[place.k];
  int n[U];
  int64_t at[U];
  float p[U][V], g[U][V], m[U][V], v[U][V];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    at[u] = place.at + u * 64 * V + threadIdx.x * V;
    n[u] = here<V>(t.numel, at[u]);
    load_vec<PB>(t.param, at[u], n[u], p[u]);
    load_vec<GB>(t.grad, at[u], n[u], g[u]);
    if constexpr (HELD) {
      const int64_t block = at[u] / EDIT_ADAMW_BLOCK;
      const auto mc = load_codes<V>(t.m, at[u], n[u]), vc = load_codes<V>(t.v, at[u], n[u]);
      const float ms = n[u] ? t.m_scale[block] : 0.f, vs = n[u] ? t.v_scale[block] : 0.f;
      decode<V>(mc, ms, m[u]);
      decode<V>(vc, vs, v[u]);
    } else {
      load_vec<false>(t.m, at[u], n[u], m[u]);
      load_vec<false>(t.v, at[u], n[u], v[u]);
    }
  }
  const float clip = rec->clip, rate = rec->rate, root = rec->root, eps = static_cast<float>(hyper.eps);
  const float decay = static_cast<float>(rec->lr_decay * tab.decay[place.k]);
  const double b1 = hyper.beta1, b2 = hyper.beta2, a1 = 1.0 - b1, a2 = 1.0 - b2;
  const Key key = key_of(rec->key, tab.base + place.k, place.at);  // 2^32 is a multiple of what a block takes
#pragma unroll
  for (int u = 0; u < U; ++u) {
#pragma unroll
    for (int e = 0; e < V; ++e) {
      const double gd = clip * g[u][e];
      m[u][e] = static_cast<float>(__builtin_fma(b1, static_cast<double>(m[u][e]), a1 * gd));
      v[u][e] = static_cast<float>(__builtin_fma(b2, static_cast<double>(v[u][e]), a2 * gd * gd));
      // The hardware's square root is off by one place and takes values below
      // 2^-126 as zero; beside an eps of 1e-12 at least neither is seen in p.
      const float d = __builtin_fmaf(__builtin_amdgcn_sqrtf(v[u][e]), root, eps);
      p[u][e] -= __builtin_fmaf(decay, p[u][e], rate * m[u][e] * __builtin_amdgcn_rcpf(d));
    }
    if constexpr (HELD || SR) {
      uint32_t word[V];
#pragma unroll
      for (int e = 0; e < V; ++e) word[e] = random_word(static_cast<uint32_t>(at[u]) + e, key.k0, key.k1);
      if constexpr (SR) {
#pragma unroll
        for (int e = 0; e < V; ++e) {  // what cuts the low half afterwards is exact
          const uint32_t x = __float_as_uint(p[u][e]);
          const uint32_t up = (x + (second_word(word[e], key.k0) >> 16)) & 0xffff0000u;
          p[u][e] = (x & 0x7fffffffu) < 0x7f800000u ? __uint_as_float(up) : p[u][e];
        }
      }
      if constexpr (HELD) {
        const uint32_t em = block_exponent(m[u]), ev = block_exponent(v[u]);
        store_codes<V>(t.m, at[u], n[u], encode<false>(m[u], em, word));
        store_codes<V>(t.v, at[u], n[u], encode<true>(v[u], ev, word));
        if (at[u] % EDIT_ADAMW_BLOCK == 0 && n[u]) {
          t.m_scale[at[u] / EDIT_ADAMW_BLOCK] = scale_of(em);
          t.v_scale[at[u] / EDIT_ADAMW_BLOCK] = scale_of(ev);
        }
      }
    }
    if constexpr (!HELD) {
      store_vec<false>(t.m, at[u], n[u], m[u]);
      store_vec<false>(t.v, at[u], n[u], v[u]);
    }
    store_vec<PB>(t.param, at[u], n[u], p[u]);
  }
}

template <bool PACK, int V, int U>
__global__ __launch_bounds__(kAdamThreads) void adamw_convert_kernel(const AdamTable tab, uint64_t key64) {
  const Place place = place_of(tab, kAdamThreads * V * U);
  const AdamTensor& t = tab.tensor[place.k];
  int n[U];
  int64_t at[U];
  float m[U][V], v[U][V];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    at[u] = place.at + u * 64 * V + threadIdx.x * V;
    n[u] = here<V>(t.numel, at[u]);
    if constexpr (PACK) {
      load_vec<false>(t.param, at[u], n[u], m[u]);
      load_vec<false>(t.grad, at[u], n[u], v[u]);
    } else {
      const int64_t block = at[u] / EDIT_ADAMW_BLOCK;
      const auto mc = load_codes<V>(t.m, at[u], n[u]), vc = load_codes<V>(t.v, at[u], n[u]);
      const float ms = n[u] ? t.m_scale[block] : 0.f, vs = n[u] ? t.v_scale[block] : 0.f;
      decode<V>(mc, ms, m[u]);
      decode<V>(vc, vs, v[u]);
    }
  }
  const Key key = key_of(key64, tab.base + place.k, place.at);
#pragma unroll
  for (int u = 0; u < U; ++u) {
    if constexpr (PACK) {
      uint32_t word[V];
#pragma unroll
      for (int e = 0; e < V; ++e) word[e] = random_word(static_cast<uint32_t>(at[u]) + e, key.k0, key.k1);
      const uint32_t em = block_exponent(m[u]), ev = block_exponent(v[u]);
      store_codes<V>(t.m, at[u], n[u], encode<false>(m[u], em, word));
      store_codes<V>(t.v, at[u], n[u], encode<true>(v[u], ev, word));
      if (at[u] % EDIT_ADAMW_BLOCK == 0 && n[u]) {
        t.m_scale[at[u] / EDIT_ADAMW_BLOCK] = scale_of(em);
        t.v_scale[at[u] / EDIT_ADAMW_BLOCK] = scale_of(ev);
      }
    } else {
      store_vec<false>(t.param, at[u], n[u], m[u]);
      store_vec<false>(const_cast<void*>(t.grad), at[u], n[u], v[u]);
    }
  }
}

// The launch's own status: hipGetLastError() would also give what an earlier call of the program left.
template <typename... A>
hipError_t launch(void (*kernel)(A...), int blocks, int threads, int lds, hipStream_t stream, A... args) {
  void* at[] = {const_cast<void*>(static_cast<const void*>(&args))...};
  return hipLaunchKernel(reinterpret_cast<const void*>(kernel), dim3(blocks), dim3(threads), at, lds, stream);
}

template <bool PB, bool GB, bool HELD, bool SR>
hipError_t step(int blocks, const AdamTable& table, const AdamHyper& hyper, const AdamRecord* rec, hipStream_t stream) {
  constexpr int V = adamw_vec(PB, GB, HELD), U = adamw_times(PB, GB, HELD), resident = adamw_resident(PB, GB, HELD);
  constexpr int lds = resident == 32 ? 0 : lds_for_blocks(resident, 0, kLdsPerCu);
  return launch<AdamTable, AdamHyper, const AdamRecord*>(adamw_step_kernel<PB, GB, HELD, SR, V, U>, blocks, kAdamThreads, lds,
                                                         stream, table, hyper, rec);
}

}  // namespace

uint64_t adamw_key(uint64_t seed, uint64_t t) { return mix(mix(seed) + t); }

hipError_t launch_adamw_norm(bool bf16, int blocks, const AdamNormTable& table, double* partials, hipStream_t stream) {
  return launch<AdamNormTable, double*>(bf16 ? adamw_norm_kernel<true> : adamw_norm_kernel<false>, blocks,
                                        kAdamNormThreads, 0, stream, table, partials);
}

hipError_t launch_adamw_sum(const double* partials, int count, double* out, hipStream_t stream) {
  return launch<const double*, int, double*>(adamw_sum_kernel, 1, kAdamDecideThreads, 0, stream, partials, count, out);
}

hipError_t launch_adamw_decide(const double* partials, int count, const double* sumsq, const AdamCall& call,
                               const AdamHyper& hyper, AdamRecord* rec, hipStream_t stream) {
  return launch<const double*, int, const double*, AdamCall, AdamHyper, AdamRecord*>(
      adamw_decide_kernel, 1, count ? kAdamDecideThreads : 64, 0, stream, partials, count, sumsq, call, hyper, rec);
}

hipError_t launch_adamw_step(bool param_bf16, bool grad_bf16, bool held, bool stochastic, int blocks, const AdamTable& table,
                             const AdamHyper& hyper, const AdamRecord* rec, hipStream_t stream) {
  if (param_bf16) {
    if (stochastic) {
      if (grad_bf16) return held ? step<true, true, true, true>(blocks, table, hyper, rec, stream)
                                 : step<true, true, false, true>(blocks, table, hyper, rec, stream);
      return held ? step<true, false, true, true>(blocks, table, hyper, rec, stream)
                  : step<true, false, false, true>(blocks, table, hyper, rec, stream);
    }
    if (grad_bf16) return held ? step<true, true, true, false>(blocks, table, hyper, rec, stream)
                               : step<true, true, false, false>(blocks, table, hyper, rec, stream);
    return held ? step<true, false, true, false>(blocks, table, hyper, rec, stream)
                : step<true, false, false, false>(blocks, table, hyper, rec, stream);
  }
  if (grad_bf16) return held ? step<false, true, true, false>(blocks, table, hyper, rec, stream)
                             : step<false, true, false, false>(blocks, table, hyper, rec, stream);
  return held ? step<false, false, true, false>(blocks, table, hyper, rec, stream)
              : step<false, false, false, false>(blocks, table, hyper, rec, stream);
}

hipError_t launch_adamw_convert(bool pack, int blocks, const AdamTable& table, uint64_t key, hipStream_t stream) {
  return launch<AdamTable, uint64_t>(pack ? adamw_convert_kernel<true, 4, 2> : adamw_convert_kernel<false, 4, 2>, blocks, kAdamThreads,
                                     0, stream, table, key);
}

}  // namespace edit
