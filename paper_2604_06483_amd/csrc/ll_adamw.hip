// A training step over many tensors at once: the norm of all their gradients, and AdamW with states in 32 or in 8 bits.
//
//   g' = g min(1, max_norm / norm),   m' = b1 m + (1 - b1) g',   v' = b2 v + (1 - b2) g'^2
//   p' = p (1 - rate decay) - rate / (1 - b1^t) m' / ( sqrt(v') / sqrt(1 - b2^t) + eps )
//
// Bound by memory: an element is read once and written once, 28 bytes of it with everything in fp32 (30 with a bf16 working copy), 14 with
// bf16 gradients and states in 8 bits (16 with the copy).
//
// States in 8 bits.  m is e4m3, v e5m2, each relative to a power of two for 256 elements.  b2 = 0.999 moves v by a thousandth a step, and a
// step of e5m2 is an eighth to a quarter of the value: rounded to the nearest, v would never move.  So both are rounded stochastically, up
// with the probability of the distance from the value below, by a hash of (seed, step, tensor, element): the mean is kept, and the same
// call gives the same bits.  It is v that is rounded without bias and not its root, whose square would gain the rounding's variance at every
// step.  Scales are powers of two so that a block whose largest value grows or falls stays on one grid: with any other scale every value
// would be rounded again, by half a step, at every step.  A positive v never becomes 0, as the update is divided by its root.
#include "ll_common.h"

#include <math.h>

namespace {

using namespace ll;

constexpr int BLOCK = LL_STATE_BLOCK;          // of 8-bit states: four elements for each lane of a wavefront
constexpr int THREADS = 256;
constexpr int UNIT = THREADS * 4;              // elements of a workgroup at a time: four blocks
constexpr int STEP_TENSORS = 48;               // of one launch: their list is the kernel's argument (4 KB at most)
constexpr int NORM_TENSORS = 160;
constexpr int NORM_GROUPS = 1024;              // workgroups of a launch, and their partial sums
constexpr int NORM_UNIT = 8192;

// ---- numbers ------------------------------------------------------------------------------------
// A permutation of 32-bit words: PCG's RXS-M-XS output function over its own multiplier and increment (M. O'Neill, 2014), used as a hash
// of a counter.
__host__ __device__ __forceinline__ uint32_t scramble(uint32_t x) {
  const uint32_t s = x * 747796405u + 2891336453u;
  const uint32_t w = ((s >> ((s >> 28) + 4)) ^ s) * 277803737u;
  return (w >> 22) ^ w;
}

// What all tensors of a step share.
struct StepTerms {
  float keep, rate, root;     // 1 - rate decay;  rate / (1 - b1^t);  1 / sqrt(1 - b2^t)
  uint32_t key;               // of (seed, step)
};
__host__ __device__ __forceinline__ StepTerms step_terms(double rate, double beta1, double beta2, double decay, int64_t step, uint32_t seed) {
  const double t = (double)step;
  StepTerms s;
  s.keep = (float)(1.0 - rate * decay);
  s.rate = (float)(rate / (1.0 - pow(beta1, t)));
  s.root = (float)(1.0 / sqrt(1.0 - pow(beta2, t)));
  s.key = scramble(seed + scramble((uint32_t)step));
  return s;
}

// The smallest power of two, at least 2^-126, that brings `most` to at most 1.75 2^TOP.
template <int TOP>
__device__ __forceinline__ int scale_exponent(float most) {
  const uint32_t bits = __float_as_uint(most);
  const int e = (int)(bits >> 23) - 127 - TOP + ((bits & 0x7FFFFF) > 0x600000 ? 1 : 0);
  return e < -126 ? -126 : e;
}
__device__ __forceinline__ float power_of_two(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }

// x >= 0 as the code of an 8-bit float with MANTISSA bits, rounded up with the probability of its distance from the code below; r: 16 random bits.
template <int MANTISSA, int BIAS>
__device__ __forceinline__ uint32_t stochastic(float x, uint32_t r) {
  constexpr int STEP = 23 - MANTISSA;
  if (x >= __builtin_ldexpf(1.f, 1 - BIAS)) return ((__float_as_uint(x) + (r << (STEP - 16))) >> STEP) - ((127 - BIAS) << MANTISSA);
  return (uint32_t)floorf(fmaf(x, __builtin_ldexpf(1.f, BIAS - 1 + MANTISSA), (float)r * (1.f / 65536.f)));   // (both products exact)
}

// m' and v' of an element.  No product is contracted into a sum: what the 8-bit codes are made of is then the same number wherever the
// definition is computed.
__device__ __forceinline__ void moments(float g, float& m, float& v, float beta1, float less1, float beta2, float less2) {
#pragma clang fp contract(off)
  m = m * beta1 + g * less1;
  v = v * beta2 + (g * g) * less2;
}

// ---- the step -----------------------------------------------------------------------------------
struct StepTensor {
  void* param;
  const void* grad;
  void* m;
  void* v;
  float* m_scale;
  float* v_scale;
  uint16_t* copy;
  int64_t n;
  uint32_t ordinal;           // in the caller's list
};

struct StepArgs {
  StepTensor tensors[STEP_TENSORS];
  uint32_t first[STEP_TENSORS + 1];     // units before each tensor
  int count;
  StepTerms terms;
  const StepTerms* clock_terms;         // or nullptr: `terms`
  const float* norm;                    // or nullptr: no clipping
  float beta1, beta2, less1, less2, eps, max_norm;
};
static_assert(sizeof(StepArgs) <= 4096, "a kernel's arguments");

// Four elements, those that there are.
template <bool BF16>
__device__ __forceinline__ void load4(const void* from, int64_t at, int there, float (&x)[4]) {
  if constexpr (BF16) {
    const uint16_t* p = static_cast<const uint16_t*>(from) + at;
    if (there == 4) {
      const uint2 q = *reinterpret_cast<const uint2*>(p);
      x[0] = bf16_lo(q.x), x[1] = bf16_hi(q.x), x[2] = bf16_lo(q.y), x[3] = bf16_hi(q.y);
      return;
    }
    for (int i = 0; i < 4; ++i) x[i] = i < there ? __uint_as_float((uint32_t)p[i] << 16) : 0.f;
  } else {
    const float* p = static_cast<const float*>(from) + at;
    if (there == 4) {
      const float4 q = *reinterpret_cast<const float4*>(p);
      x[0] = q.x, x[1] = q.y, x[2] = q.z, x[3] = q.w;
      return;
    }
    for (int i = 0; i < 4; ++i) x[i] = i < there ? p[i] : 0.f;
  }
}
__device__ __forceinline__ void store4(float* to, int64_t at, int there, const float (&x)[4]) {
  to += at;
  if (there == 4) {
    *reinterpret_cast<float4*>(to) = make_float4(x[0], x[1], x[2], x[3]);
    return;
  }
  for (int i = 0; i < there; ++i) to[i] = x[i];
}
__device__ __forceinline__ void store4(uint16_t* to, int64_t at, int there, uint2 q) {
  to += at;
  if (there == 4) {
    *reinterpret_cast<uint2*>(to) = q;
    return;
  }
  for (int i = 0; i < there; ++i) to[i] = (uint16_t)((i < 2 ? q.x : q.y) >> (16 * (i & 1)));
}
__device__ __forceinline__ void store4(uint8_t* to, int64_t at, int there, uint32_t q) {
  to += at;
  if (there == 4) {
    *reinterpret_cast<uint32_t*>(to) = q;
    return;
  }
  for (int i = 0; i < there; ++i) to[i] = (uint8_t)(q >> (8 * i));
}
__device__ __forceinline__ uint32_t load_codes(const uint8_t* from, int64_t at, int there) {
  from += at;
  if (there == 4) return *reinterpret_cast<const uint32_t*>(from);
  uint32_t q = 0;
  for (int i = 0; i < there; ++i) q |= (uint32_t)from[i] << (8 * i);
  return q;
}

template <bool PARAM_BF16, bool GRAD_BF16, bool STATE_8>
__global__ __launch_bounds__(THREADS) void ll_adamw_kernel(const StepArgs p) {
  float clip = 1.f;
  if (p.norm != nullptr) {
    const float norm = *p.norm;
    if (!(norm < INFINITY)) return;                       // gradients that overflowed, or NaN: no step
    clip = norm > p.max_norm ? p.max_norm / norm : 1.f;
  }
  const StepTerms terms = p.clock_terms != nullptr ? *p.clock_terms : p.terms;
  int lo = 0, hi = p.count - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (blockIdx.x >= p.first[mid]) lo = mid;
    else hi = mid - 1;
  }
  const StepTensor& t = p.tensors[lo];
  const int64_t n = t.n, at = (int64_t)(blockIdx.x - p.first[lo]) * UNIT + 4 * (int)threadIdx.x;
  const int64_t block = (int64_t)__builtin_amdgcn_readfirstlane((int)(at / BLOCK));
  if (block * BLOCK >= n) return;                         // (a whole wavefront)
  const int there = n - at >= 4 ? 4 : n > at ? (int)(n - at) : 0;
  float g[4], w[4], m[4], v[4];
  load4<PARAM_BF16>(t.param, at, there, w);
  load4<GRAD_BF16>(t.grad, at, there, g);
  if constexpr (STATE_8) {
    const float m_by = t.m_scale[block], v_by = t.v_scale[block];
    const uint32_t mq = load_codes(static_cast<const uint8_t*>(t.m), at, there), vq = load_codes(static_cast<const uint8_t*>(t.v), at, there);
    const auto m0 = __builtin_amdgcn_cvt_pk_f32_fp8((int)mq, false), m1 = __builtin_amdgcn_cvt_pk_f32_fp8((int)mq, true);
    const auto v0 = __builtin_amdgcn_cvt_pk_f32_bf8((int)vq, false), v1 = __builtin_amdgcn_cvt_pk_f32_bf8((int)vq, true);
    m[0] = m0[0] * m_by, m[1] = m0[1] * m_by, m[2] = m1[0] * m_by, m[3] = m1[1] * m_by;
    v[0] = v0[0] * v_by, v[1] = v0[1] * v_by, v[2] = v1[0] * v_by, v[3] = v1[1] * v_by;
  } else {
    load4<false>(t.m, at, there, m);
    load4<false>(t.v, at, there, v);
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    moments(g[i] * clip, m[i], v[i], p.beta1, p.less1, p.beta2, p.less2);
    // (the quotient's last bits are far below the parameter's: the hardware's own root and reciprocal, each within one)
    const float by = __builtin_amdgcn_rcpf(fmaf(__builtin_amdgcn_sqrtf(v[i]), terms.root, p.eps));
    w[i] = fmaf(-terms.rate * m[i], by, w[i] * terms.keep);
  }
  uint32_t words[4];
  if (STATE_8 || PARAM_BF16) {
    uint32_t key = scramble(terms.key + t.ordinal);
    if ((at >> 32) != 0) key ^= scramble((uint32_t)(at >> 32));
#pragma unroll
    for (int i = 0; i < 4; ++i) words[i] = scramble((uint32_t)(at + i) ^ key);
  }
  if constexpr (STATE_8) {
    float most_m = 0.f, most_v = 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      most_m = fmaxf(most_m, i < there && fabsf(m[i]) < INFINITY ? fabsf(m[i]) : 0.f);
      most_v = fmaxf(most_v, i < there && v[i] < INFINITY ? v[i] : 0.f);
    }
    const int em = scale_exponent<8>(wave_max(most_m)), ev = scale_exponent<15>(wave_max(most_v));
    const float to_m = power_of_two(-em), to_v = power_of_two(-ev);
    uint32_t mq = 0, vq = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float x = m[i] * to_m, y = v[i] * to_v;
      uint32_t a = min(stochastic<3, 7>(fabsf(x), words[i] >> 16), 0x7Eu), b = min(stochastic<2, 15>(y, words[i] & 0xFFFF), 0x7Bu);
      if (!(fabsf(x) < INFINITY)) a = 0x7F;               // NaN, of its own element alone
      if (!(y < INFINITY)) b = 0x7F;
      b = max(b, y > 0.f ? 1u : 0u);
      a |= __float_as_uint(x) >> 31 << 7;
      mq |= a << (8 * i);
      vq |= b << (8 * i);
    }
    store4(static_cast<uint8_t*>(t.m), at, there, mq);
    store4(static_cast<uint8_t*>(t.v), at, there, vq);
    if ((threadIdx.x & 63) == 0) {
      t.m_scale[block] = power_of_two(em);
      t.v_scale[block] = power_of_two(ev);
    }
  } else {
    store4(static_cast<float*>(t.m), at, there, m);
    store4(static_cast<float*>(t.v), at, there, v);
  }
  if constexpr (PARAM_BF16) {
    // A step is a thousandth of the parameter, a last bit of bf16 a 256th: stochastically here too.
    uint32_t h[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t bits = __float_as_uint(w[i]);
      h[i] = fabsf(w[i]) < INFINITY ? (bits + (scramble(words[i]) & 0xFFFF)) >> 16 : pack_bf16(w[i], 0.f) & 0xFFFF;
    }
    store4(static_cast<uint16_t*>(t.param), at, there, make_uint2(h[0] | h[1] << 16, h[2] | h[3] << 16));
  } else {
    store4(static_cast<float*>(t.param), at, there, w);
    if (t.copy != nullptr) store4(t.copy, at, there, make_uint2(pack_bf16(w[0], w[1]), pack_bf16(w[2], w[3])));
  }
}

// A step that the GPU counts: clock[0] steps have been done; clock[1] and [2] take this one's terms.
__global__ void ll_adamw_clock_kernel(int64_t* clock, const float* device_rate, double rate, double beta1, double beta2, double decay, uint32_t seed,
                                      const float* norm) {
  if (threadIdx.x != 0 || (norm != nullptr && !(*norm < INFINITY))) return;
  const int64_t step = clock[0] + 1;
  clock[0] = step;
  *reinterpret_cast<StepTerms*>(clock + 1) = step_terms(device_rate != nullptr ? (double)*device_rate : rate, beta1, beta2, decay, step, seed);
}

// ---- the norm -----------------------------------------------------------------------------------
struct NormTensor {
  const void* grad;
  int64_t n;
};
struct NormArgs {
  NormTensor tensors[NORM_TENSORS];      // n below 0: -n values of bf16
  uint32_t first[NORM_TENSORS + 1];      // units before each tensor
  int count;
  double* partial;                       // [workgroups]
};
static_assert(sizeof(NormArgs) <= 4096, "a kernel's arguments");

// The sum over the workgroup, in one order; thread 0 has it.
__device__ __forceinline__ double sum_of_group(double x, double* red) {
  for (int off = 32; off > 0; off >>= 1) x += __shfl_xor(x, off);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = x;
  __syncthreads();
  return (red[0] + red[1]) + (red[2] + red[3]);
}

// Sums of squares in 64 bits: the norm is then exact to its last bit whatever the order, and so is what a step is clipped by.
__global__ __launch_bounds__(THREADS) void ll_grad_norm_kernel(const NormArgs p) {
  __shared__ double red[THREADS / 64];
  double sum = 0.;
  for (uint32_t unit = blockIdx.x; unit < p.first[p.count]; unit += gridDim.x) {
    int lo = 0, hi = p.count - 1;
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (unit >= p.first[mid]) lo = mid;
      else hi = mid - 1;
    }
    const NormTensor t = p.tensors[lo];
    const bool bf16 = t.n < 0;
    const int64_t n = bf16 ? -t.n : t.n, from = (int64_t)(unit - p.first[lo]) * NORM_UNIT;
    const int64_t end = from + NORM_UNIT < n ? from + NORM_UNIT : n;
    for (int64_t at = from + 4 * (int)threadIdx.x; at < end; at += 4 * THREADS) {
      float g[4];
      const int there = end - at >= 4 ? 4 : (int)(end - at);
      if (bf16) load4<true>(t.grad, at, there, g);
      else load4<false>(t.grad, at, there, g);
#pragma unroll
      for (int i = 0; i < 4; ++i) sum = fma((double)g[i], (double)g[i], sum);
    }
  }
  sum = sum_of_group(sum, red);
  if (threadIdx.x == 0) p.partial[blockIdx.x] = sum;
}

__global__ __launch_bounds__(THREADS) void ll_grad_norm_join_kernel(const double* __restrict__ partial, int parts, float* __restrict__ norm) {
  __shared__ double red[THREADS / 64];
  double sum = 0.;
  for (int i = threadIdx.x; i < parts; i += THREADS) sum += partial[i];
  sum = sum_of_group(sum, red);
  if (threadIdx.x == 0) *norm = (float)sqrt(sum);
}

// ---------------------------------------------------------------------------------------
// Host
// ---------------------------------------------------------------------------------------
bool misaligned(const void* p, size_t to) { return ((uintptr_t)p & (to - 1)) != 0; }

constexpr uint32_t ALL_FLAGS = LL_TENSOR_PARAM_BF16 | LL_TENSOR_GRAD_BF16 | LL_TENSOR_STATE_8BIT;
constexpr int64_t MOST_ELEMENTS = LL_TENSOR_MAX;

bool valid_list(const ll_tensor* tensors, int32_t count) {
  if (count < 0 || (count > 0 && tensors == nullptr)) return false;
  for (int32_t i = 0; i < count; ++i) {
    const ll_tensor& t = tensors[i];
    if (t.n < 0 || t.n > MOST_ELEMENTS || (t.flags & ~ALL_FLAGS) != 0) return false;
    if (t.n > 0 && (t.grad == nullptr || misaligned(t.grad, 16))) return false;
  }
  return true;
}

bool is_finite(double x) { return x - x == 0.; }

using StepKernel = void (*)(const StepArgs);
StepKernel step_kernel(uint32_t flags) {
  static const StepKernel kernels[8] = {ll_adamw_kernel<false, false, false>, ll_adamw_kernel<true, false, false>, ll_adamw_kernel<false, true, false>,
                                        ll_adamw_kernel<true, true, false>,   ll_adamw_kernel<false, false, true>, ll_adamw_kernel<true, false, true>,
                                        ll_adamw_kernel<false, true, true>,   ll_adamw_kernel<true, true, true>};
  return kernels[flags];
}
static_assert(LL_TENSOR_PARAM_BF16 == 1 && LL_TENSOR_GRAD_BF16 == 2 && LL_TENSOR_STATE_8BIT == 4, "as step_kernel has them");

// Units of one launch of a step: a grid has fewer than 2^32 threads.
constexpr int64_t MOST_UNITS = ((int64_t)1 << 24) - 1;
static_assert(MOST_ELEMENTS / UNIT <= MOST_UNITS && MOST_ELEMENTS / NORM_UNIT * NORM_TENSORS < (int64_t)1 << 31, "a tensor fits one, and units 32 bits");

}  // namespace

extern "C" {

size_t ll_grad_norm_workspace_bytes(int32_t n_tensors) {
  if (n_tensors < 0) return 0;
  const int64_t launches = n_tensors > 0 ? ((int64_t)n_tensors + NORM_TENSORS - 1) / NORM_TENSORS : 1;
  return align_up((size_t)launches * NORM_GROUPS * sizeof(double), 256);
}

int ll_grad_norm(const ll_tensor* tensors, int32_t n_tensors, void* workspace, size_t workspace_bytes, float* out_norm, void* stream) {
  if (!valid_list(tensors, n_tensors) || out_norm == nullptr || misaligned(out_norm, 4)) return LL_EINVAL;
  if (workspace == nullptr || workspace_bytes < ll_grad_norm_workspace_bytes(n_tensors) || misaligned(workspace, 256)) return LL_EWORKSPACE;
  double* const partial = static_cast<double*>(workspace);
  int parts = 0;
  for (int32_t i = 0; i < n_tensors;) {
    NormArgs a = {};
    int64_t units = 0;
    for (; i < n_tensors && a.count < NORM_TENSORS; ++i) {
      const ll_tensor& t = tensors[i];
      if (t.n == 0) continue;
      a.tensors[a.count] = {t.grad, (t.flags & LL_TENSOR_GRAD_BF16) != 0 ? -t.n : t.n};
      a.first[a.count++] = (uint32_t)units;
      units += (t.n + NORM_UNIT - 1) / NORM_UNIT;
      a.first[a.count] = (uint32_t)units;
    }
    if (a.count == 0) continue;
    const int groups = (int)(units < NORM_GROUPS ? units : NORM_GROUPS);
    a.partial = partial + parts;
    hipLaunchKernelGGL(ll_grad_norm_kernel, dim3(groups), dim3(THREADS), 0, (hipStream_t)stream, a);
    LL_HIP_CHECK(hipGetLastError());
    parts += groups;
  }
  hipLaunchKernelGGL(ll_grad_norm_join_kernel, dim3(1), dim3(THREADS), 0, (hipStream_t)stream, partial, parts, out_norm);
  LL_HIP_CHECK(hipGetLastError());
  return LL_OK;
}

int ll_adamw(const ll_tensor* tensors, int32_t n_tensors, const ll_adamw_options* options, const float* norm, int64_t* clock,
             const float* device_rate, void* stream) {
  if (!valid_list(tensors, n_tensors) || options == nullptr) return LL_EINVAL;
  const ll_adamw_options& o = *options;
  if (!(o.rate >= 0.) || !is_finite(o.rate) || !(o.beta1 >= 0. && o.beta1 < 1.) || !(o.beta2 >= 0. && o.beta2 < 1.) || !((float)o.eps > 0.f) || !is_finite(o.eps) ||
      !(o.decay >= 0.) || !is_finite(o.decay))
    return LL_EINVAL;
  if (clock == nullptr ? (o.step < 1 || device_rate != nullptr) : misaligned(clock, 8)) return LL_EINVAL;
  if ((norm != nullptr && !(o.max_norm > 0.)) || misaligned(norm, 4) || misaligned(device_rate, 4)) return LL_EINVAL;
  for (int32_t i = 0; i < n_tensors; ++i) {
    const ll_tensor& t = tensors[i];
    if (t.n == 0) continue;
    if (t.param == nullptr || t.m == nullptr || t.v == nullptr) return LL_EINVAL;
    if (misaligned(t.param, 16) || misaligned(t.m, 16) || misaligned(t.v, 16) || misaligned(t.copy, 16)) return LL_EINVAL;
    const bool eight = (t.flags & LL_TENSOR_STATE_8BIT) != 0;
    if (eight != (t.m_scale != nullptr) || eight != (t.v_scale != nullptr) || misaligned(t.m_scale, 4) || misaligned(t.v_scale, 4)) return LL_EINVAL;
    if (t.copy != nullptr && (t.flags & LL_TENSOR_PARAM_BF16) != 0) return LL_EINVAL;
  }
  StepArgs a = {};
  if (clock != nullptr) {
    hipLaunchKernelGGL(ll_adamw_clock_kernel, dim3(1), dim3(64), 0, (hipStream_t)stream, clock, device_rate, o.rate, o.beta1, o.beta2, o.decay, o.seed, norm);
    LL_HIP_CHECK(hipGetLastError());
    a.clock_terms = reinterpret_cast<const StepTerms*>(clock + 1);
  } else {
    a.terms = step_terms(o.rate, o.beta1, o.beta2, o.decay, o.step, o.seed);
  }
  a.norm = norm;
  a.beta1 = (float)o.beta1;
  a.beta2 = (float)o.beta2;
  a.less1 = (float)(1. - o.beta1);
  a.less2 = (float)(1. - o.beta2);
  a.eps = (float)o.eps;
  a.max_norm = (float)o.max_norm;
  for (uint32_t flags = 0; flags <= ALL_FLAGS; ++flags) {   // a launch for every kind of tensor that there is, and as many tensors as its arguments hold
    for (int32_t i = 0; i < n_tensors;) {
      a.count = 0;
      int64_t units = 0;
      for (; i < n_tensors && a.count < STEP_TENSORS; ++i) {
        const ll_tensor& t = tensors[i];
        if (t.n == 0 || t.flags != flags) continue;
        const int64_t more = (t.n + UNIT - 1) / UNIT;
        if (units + more > MOST_UNITS) break;
        a.tensors[a.count] = {t.param, t.grad, t.m, t.v, t.m_scale, t.v_scale, static_cast<uint16_t*>(t.copy), t.n, (uint32_t)i};
        a.first[a.count++] = (uint32_t)units;
        units += more;
        a.first[a.count] = (uint32_t)units;
      }
      if (a.count == 0) continue;
      hipLaunchKernelGGL(step_kernel(flags), dim3((unsigned)units), dim3(THREADS), 0, (hipStream_t)stream, a);
      LL_HIP_CHECK(hipGetLastError());
    }
  }
  return LL_OK;
}

}  // extern "C"
