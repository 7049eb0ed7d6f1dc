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
constexpr int UNIT_BLOCKS = THREADS / 64, UNIT = UNIT_BLOCKS * BLOCK;   // of a workgroup, a block a wavefront (two or four: 3 to 7 % slower)
constexpr int STEP_TENSORS = 48;               // of one launch: their list is the kernel's argument (4 KB at most)
constexpr int NORM_TENSORS = 160;
constexpr int NORM_GROUPS = 2048;              // workgroups of a launch, and their partial sums
constexpr int NORM_UNIT = 1024;                // elements, by a wavefront; four of them in flight
constexpr int NORM_ALONE = 128;                // units that one workgroup takes by itself (66: 6.2 us, two launches 10.1; 132: 9.0 | 8.7 to 9.9; 264: 11.9 | 8.8 to 9.9)

// ---- numbers ------------------------------------------------------------------------------------
// A permutation of 32-bit words: PCG's RXS-M-XS output function over its own multiplier and increment (M. O'Neill, 2014), used as a hash
// of a counter.
constexpr uint32_t SCRAMBLE = 747796405u, SCRAMBLE_MORE = 2891336453u;
__host__ __device__ __forceinline__ uint32_t scramble_state(uint32_t s) {
  const uint32_t w = ((s >> ((s >> 28) + 4)) ^ s) * 277803737u;
  return (w >> 22) ^ w;
}
__host__ __device__ __forceinline__ uint32_t scramble(uint32_t x) { return scramble_state(x * SCRAMBLE + SCRAMBLE_MORE); }

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

// The smallest power of two, at least 2^-126, that brings `most` to at most 1.75 2^TOP, as fp32's own exponent.  (It grows with `most`: the largest
// of several numbers' is the largest number's.)
template <int TOP>
__device__ __forceinline__ uint32_t scale_exponent(float most) {
  const int e = (int)((__float_as_uint(most) + 0x1FFFFF) >> 23) - TOP;   // (one more above 1.75)
  return e < 1 ? 1 : e;
}
__device__ __forceinline__ float power_of_two(uint32_t e) { return __uint_as_float(e << 23); }

// The hardware's own stochastic rounding is the one that the states are defined by: it adds the upper 20 (e4m3; 21, e5m2) bits of a word to
// those that a number loses, a subnormal code's as well.  Sixteen of them are random here.
template <int AT>
__device__ __forceinline__ uint32_t put_e4m3(uint32_t codes, float x, uint32_t word) {
  return (uint32_t)__builtin_amdgcn_cvt_sr_fp8_f32(x, (int)(word & 0xFFFF0000u), (int)codes, AT);
}
template <int AT>
__device__ __forceinline__ uint32_t put_e5m2(uint32_t codes, float x, uint32_t word) {
  return (uint32_t)__builtin_amdgcn_cvt_sr_bf8_f32(x, (int)(word << 16), (int)codes, AT);
}

// The larger of each half of two words.
__device__ __forceinline__ uint32_t most_of_halves(uint32_t a, uint32_t b) {
  typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, a), __builtin_bit_cast(u16x2, b)));
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
  uint32_t first[64];                   // units before each tensor; more than any unit behind the last
  int count;
  StepTerms terms;
  const StepTerms* clock_terms;         // or nullptr: `terms`
  const float* norm;                    // or nullptr: no clipping
  float beta1, beta2, less1, less2, eps, max_norm;
};
static_assert(sizeof(StepArgs) <= 4096, "a kernel's arguments");

// Past the caches: a step's tensors are read once and written once, and what is read between two steps is far more than the caches hold.  Both
// ways or not at all (us, loads and stores through the caches | loads past them | stores | both: eight d = 2560 layers in fp32 292 | 294 | 291 |
// 267; twelve of d = 4096, 8 bits 576 | 580 | 559 | 515; lists that the caches would hold see no difference).
template <int BYTES>
struct Word {
  typedef uint32_t type __attribute__((ext_vector_type(BYTES / 4)));
};
template <>
struct Word<4> {
  typedef uint32_t type;
};
template <class V>
__device__ __forceinline__ V load_past(const void* from) {
  typedef typename Word<sizeof(V)>::type T;
  return __builtin_bit_cast(V, __builtin_nontemporal_load(static_cast<const T*>(from)));
}
template <class V>
__device__ __forceinline__ void store_past(void* to, V x) {
  typedef typename Word<sizeof(V)>::type T;
  __builtin_nontemporal_store(__builtin_bit_cast(T, x), static_cast<T*>(to));
}

// A lane's four elements of those from `from` on, as many as there are.
template <bool BF16>
__device__ __forceinline__ void load4(const void* from, uint32_t at, int there, float (&x)[4]) {
  if constexpr (BF16) {
    const uint16_t* p = static_cast<const uint16_t*>(from) + at;
    if (there == 4) {
      const uint2 q = load_past<uint2>(p);
      x[0] = bf16_lo(q.x), x[1] = bf16_hi(q.x), x[2] = bf16_lo(q.y), x[3] = bf16_hi(q.y);
      return;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = i < there ? __uint_as_float((uint32_t)p[i] << 16) : 0.f;
  } else {
    const float* p = static_cast<const float*>(from) + at;
    if (there == 4) {
      const float4 q = load_past<float4>(p);
      x[0] = q.x, x[1] = q.y, x[2] = q.z, x[3] = q.w;
      return;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = i < there ? p[i] : 0.f;
  }
}
__device__ __forceinline__ void store4(float* to, int there, const float (&x)[4]) {
  if (there == 4) {
    store_past(to, make_float4(x[0], x[1], x[2], x[3]));
    return;
  }
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (i < there) to[i] = x[i];
}
__device__ __forceinline__ void store4(uint16_t* to, int there, uint2 q) {
  if (there == 4) {
    store_past(to, q);
    return;
  }
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (i < there) to[i] = (uint16_t)((i < 2 ? q.x : q.y) >> (16 * (i & 1)));
}
__device__ __forceinline__ void store4(uint8_t* to, int there, uint32_t q) {
  if (there == 4) {
    store_past(to, q);
    return;
  }
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (i < there) to[i] = (uint8_t)(q >> (8 * i));
}
__device__ __forceinline__ uint32_t load_codes(const uint8_t* from, int there) {
  if (there == 4) return load_past<uint32_t>(from);
  uint32_t q = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) q |= i < there ? (uint32_t)from[i] << (8 * i) : 0u;
  return q;
}

// Four elements of a lane, a block of a wavefront; in 8 bits the states' codes, a byte an element.
template <bool PARAM_BF16, bool GRAD_BF16, bool STATE_8>
struct StepFour {
  float g[4], w[4], m[4], v[4];
  uint32_t mq, vq;
  float m_by, v_by;

  // block, and all that is made of it, is the wavefront's: the lane adds a constant to its addresses
  static constexpr int PARAM = PARAM_BF16 ? 2 : 4, GRAD = GRAD_BF16 ? 2 : 4, STATE = STATE_8 ? 1 : 4;
  static __device__ __forceinline__ char* of_block(const void* p, int64_t block, int bytes) { return (char*)p + block * (BLOCK * bytes); }

  __device__ __forceinline__ void load(const StepTensor& t, int64_t block, uint32_t at, int there) {
    load4<PARAM_BF16>(of_block(t.param, block, PARAM), at, there, w);
    load4<GRAD_BF16>(of_block(t.grad, block, GRAD), at, there, g);
    if constexpr (STATE_8) {
      mq = load_codes((const uint8_t*)of_block(t.m, block, STATE) + at, there);
      vq = load_codes((const uint8_t*)of_block(t.v, block, STATE) + at, there);
      m_by = t.m_scale[block];
      v_by = t.v_scale[block];
    } else {
      load4<false>(of_block(t.m, block, STATE), at, there, m);
      load4<false>(of_block(t.v, block, STATE), at, there, v);
    }
  }

  __device__ __forceinline__ void step(const StepArgs& p, const StepTerms& terms, const StepTensor& t, float clip, int64_t block, uint32_t at, int there) {
    if constexpr (STATE_8) {
      const auto m0 = __builtin_amdgcn_cvt_pk_f32_fp8((int)mq, false), m1 = __builtin_amdgcn_cvt_pk_f32_fp8((int)mq, true);
      const auto v0 = __builtin_amdgcn_cvt_pk_f32_bf8((int)vq, false), v1 = __builtin_amdgcn_cvt_pk_f32_bf8((int)vq, true);
      m[0] = m0[0] * m_by, m[1] = m0[1] * m_by, m[2] = m1[0] * m_by, m[3] = m1[1] * m_by;
      v[0] = v0[0] * v_by, v[1] = v0[1] * v_by, v[2] = v1[0] * v_by, v[3] = v1[1] * v_by;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) moments(g[i] * clip, m[i], v[i], p.beta1, p.less1, p.beta2, p.less2);
    // The quotient's last bits are far below the parameter's: the hardware's own root and reciprocal, each within one.  They take subnormal numbers
    // for 0, which is nothing beside an eps that is large beside their roots.  (1 / eps may be more than 32 bits hold, and an element without a gradient
    // would be 0 times infinity.)
    if (p.eps >= 1e-10f) {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        w[i] = fmaf(-terms.rate * m[i], __builtin_amdgcn_rcpf(fmaf(__builtin_amdgcn_sqrtf(v[i]), terms.root, p.eps)), w[i] * terms.keep);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float under = fmaf(sqrtf(v[i]), terms.root, p.eps), by = 1.f / under, up = -terms.rate * m[i];
        w[i] = by < INFINITY ? fmaf(up, by, w[i] * terms.keep) : fmaf(w[i], terms.keep, up / under);
      }
    }
    uint32_t words[4];
    if (STATE_8 || PARAM_BF16) {
      uint32_t key = scramble(terms.key + t.ordinal);
      if ((block >> 24) != 0) key ^= scramble((uint32_t)(block >> 24));
      // words[i] = scramble(element ^ key), the four elements' products formed from one
      uint32_t product = (((uint32_t)block * BLOCK + at) ^ (key & ~3u)) * SCRAMBLE;
      asm("" : "+v"(product));                              // (the compiler would have four products again)
#pragma unroll
      for (int i = 0; i < 4; ++i) words[i] = scramble_state(product + (((key & 3) ^ i) * SCRAMBLE + SCRAMBLE_MORE));
    }
    if constexpr (STATE_8) {
      // (the largest of numbers passes NaN by; an infinite one, which says nothing of the others, is looked for apart)
      float most_m = fmaxf(fmaxf(fabsf(m[0]), fabsf(m[1])), fmaxf(fabsf(m[2]), fabsf(m[3]))), most_v = fmaxf(fmaxf(v[0], v[1]), fmaxf(v[2], v[3]));
      if (__builtin_amdgcn_ballot_w64(!(fmaxf(most_m, most_v) < INFINITY)) != 0) {
        asm volatile("; not worth doing ahead");
        most_m = most_v = 0.f;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          most_m = fmaxf(most_m, fabsf(m[i]) < INFINITY ? fabsf(m[i]) : 0.f);
          most_v = fmaxf(most_v, v[i] < INFINITY ? v[i] : 0.f);
        }
      }
      const uint32_t e = wave_combine(scale_exponent<8>(most_m) | scale_exponent<15>(most_v) << 16, most_of_halves);
      const uint32_t em = e & 0xFFFF, ev = e >> 16;
      const float to_m = power_of_two(254 - em), to_v = power_of_two(254 - ev);
      float y[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) y[i] = v[i] > 0.f ? fmaxf(v[i] * to_v, 0x1p-16f) : v[i];      // (at least the smallest code: rounded to it at least)
      uint32_t a = 0, b = 0;
      a = put_e4m3<0>(a, m[0] * to_m, words[0]);
      a = put_e4m3<1>(a, m[1] * to_m, words[1]);
      a = put_e4m3<2>(a, m[2] * to_m, words[2]);
      a = put_e4m3<3>(a, m[3] * to_m, words[3]);
      b = put_e5m2<0>(b, y[0], words[0]);
      b = put_e5m2<1>(b, y[1], words[1]);
      b = put_e5m2<2>(b, y[2], words[2]);
      b = put_e5m2<3>(b, y[3], words[3]);
      store4((uint8_t*)of_block(t.m, block, STATE) + at, there, a);
      store4((uint8_t*)of_block(t.v, block, STATE) + at, there, b);
      if ((threadIdx.x & 63) == 0) {
        t.m_scale[block] = power_of_two(em);
        t.v_scale[block] = power_of_two(ev);
      }
    } else {
      store4((float*)of_block(t.m, block, STATE) + at, there, m);
      store4((float*)of_block(t.v, block, STATE) + at, there, v);
    }
    if constexpr (PARAM_BF16) {
      // A step is a thousandth of the parameter, a last bit of bf16 a 256th: stochastically here too.
      uint32_t h[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t bits = __float_as_uint(w[i]);
        h[i] = fabsf(w[i]) < INFINITY ? (bits + (scramble(words[i]) & 0xFFFF)) >> 16 : pack_bf16(w[i], 0.f) & 0xFFFF;
      }
      store4((uint16_t*)of_block(t.param, block, PARAM) + at, there, make_uint2(h[0] | h[1] << 16, h[2] | h[3] << 16));
    } else {
      store4((float*)of_block(t.param, block, PARAM) + at, there, w);
      if (t.copy != nullptr) store4((uint16_t*)of_block(t.copy, block, 2) + at, there, make_uint2(pack_bf16(w[0], w[1]), pack_bf16(w[2], w[3])));
    }
  }
};

template <bool PARAM_BF16, bool GRAD_BF16, bool STATE_8>
__global__ __launch_bounds__(THREADS) void ll_adamw_kernel(const StepArgs p) {
  const int lane = threadIdx.x & 63;
  const uint32_t unit = blockIdx.x;
  const int which = __popcll(__builtin_amdgcn_ballot_w64(unit >= p.first[lane])) - 1;
  const StepTensor& t = p.tensors[which];
  const int64_t n = t.n;
  const int64_t block = (int64_t)(unit - p.first[which]) * UNIT_BLOCKS + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t left = n - block * BLOCK;
  if (left <= 0) return;
  StepFour<PARAM_BF16, GRAD_BF16, STATE_8> four;
  const int there = left >= BLOCK ? 4 : max(0, min(4, (int)left - 4 * lane));
  if (left >= BLOCK) four.load(t, block, 4 * lane, 4);
  else four.load(t, block, 4 * lane, there);
  float clip = 1.f;
  if (p.norm != nullptr) {
    const float norm = *p.norm;
    if (!(norm < INFINITY)) return;                       // gradients that overflowed, or NaN: no step
    if (norm > p.max_norm) clip = p.max_norm / norm;
  }
  StepTerms terms = p.terms;
  if (p.clock_terms != nullptr) terms = *p.clock_terms;
  if (left >= BLOCK) four.step(p, terms, t, clip, block, 4 * lane, 4);
  else four.step(p, terms, t, clip, block, 4 * lane, there);
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
  uint32_t first[192];                   // units before each tensor; more than any unit behind the last
  uint32_t units;
  double* partial;                       // [workgroups]
  float* norm;                           // or nullptr: of the one workgroup that there is
};
static_assert(sizeof(NormArgs) <= 4096 && NORM_TENSORS < 192, "a kernel's arguments");

// The sum over the workgroup, in one order; thread 0 has it.
template <int T>
__device__ __forceinline__ double sum_of_group(double x) {
  __shared__ double red[T / 64];
  for (int off = 32; off > 0; off >>= 1) x += __shfl_xor(x, off);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = x;
  __syncthreads();
  double sum = 0.;
#pragma unroll
  for (int i = 0; i < T / 64; ++i) sum += red[i];
  return sum;
}

__device__ __forceinline__ void add_square(double& sum, float x) { sum = fma((double)x, (double)x, sum); }
__device__ __forceinline__ void add_squares(double (&sum)[4], const float4 q) {
  add_square(sum[0], q.x);
  add_square(sum[1], q.y);
  add_square(sum[2], q.z);
  add_square(sum[3], q.w);
}
__device__ __forceinline__ void add_squares(double (&sum)[4], const uint4 q) {
  add_squares(sum, make_float4(bf16_lo(q.x), bf16_hi(q.x), bf16_lo(q.y), bf16_hi(q.y)));
  add_squares(sum, make_float4(bf16_lo(q.z), bf16_hi(q.z), bf16_lo(q.w), bf16_hi(q.w)));
}

// Sums of squares in 64 bits: the norm is then exact to its last bit whatever the order, and so is what a step is clipped by.  A wavefront
// takes four units, 8 or 16 KB in flight, one after the other where they are not all whole and of one tensor.
template <int T>
__global__ __launch_bounds__(T) void ll_grad_norm_kernel(const NormArgs p) {
  const int lane = threadIdx.x & 63;
  const uint32_t wave = blockIdx.x * (T / 64) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = gridDim.x * (T / 64);
  double sum[4] = {0., 0., 0., 0.};
  uint32_t begin = 1, end = 0;
  const void* grad = nullptr;
  int64_t n = 0;
  bool bf16 = false;
  const auto locate = [&](uint32_t unit) {
    if (unit >= begin && unit < end) return;
    int which = -1;
#pragma unroll
    for (int i = 0; i < 3; ++i) which += __popcll(__builtin_amdgcn_ballot_w64(unit >= p.first[64 * i + lane]));
    begin = p.first[which];
    end = p.first[which + 1];
    grad = p.tensors[which].grad;
    n = p.tensors[which].n;
    bf16 = n < 0;
    n = bf16 ? -n : n;
  };
  for (uint32_t unit = 4 * wave; unit < p.units; unit += 4 * waves) {
    locate(unit);
    const int64_t at = (int64_t)(unit - begin) * NORM_UNIT;
    if (at + 4 * NORM_UNIT <= n) {
      if (bf16) {
        const uint4* from = reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(grad) + at) + lane;
        uint4 q[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) q[i] = from[64 * i];
#pragma unroll
        for (int i = 0; i < 8; ++i) add_squares(sum, q[i]);
      } else {
        const float4* from = reinterpret_cast<const float4*>(static_cast<const float*>(grad) + at) + lane;
        float4 q[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) q[i] = from[64 * i];
#pragma unroll
        for (int i = 0; i < 16; ++i) add_squares(sum, q[i]);
      }
      continue;
    }
#pragma unroll 1
    for (uint32_t u = unit; u < unit + 4 && u < p.units; ++u) {
      locate(u);
      const int64_t from = (int64_t)(u - begin) * NORM_UNIT + 4 * lane;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int64_t e = from + 256 * i;
        const int there = n - e >= 4 ? 4 : n > e ? (int)(n - e) : 0;
        float g[4];
        if (bf16) load4<true>(static_cast<const uint16_t*>(grad) + e, 0, there, g);
        else load4<false>(static_cast<const float*>(grad) + e, 0, there, g);
        add_squares(sum, make_float4(g[0], g[1], g[2], g[3]));
      }
    }
  }
  const double all = sum_of_group<T>((sum[0] + sum[1]) + (sum[2] + sum[3]));
  if (threadIdx.x != 0) return;
  if (p.norm != nullptr) *p.norm = (float)sqrt(all);
  else p.partial[blockIdx.x] = all;
}

__global__ __launch_bounds__(THREADS) void ll_grad_norm_join_kernel(const double* __restrict__ partial, int parts, float* __restrict__ norm) {
  double sum = 0.;
#pragma unroll 8
  for (int i = threadIdx.x; i < parts; i += THREADS) sum += partial[i];
  sum = sum_of_group<THREADS>(sum);
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
static_assert(MOST_ELEMENTS / UNIT <= MOST_UNITS, "a tensor fits one");
static_assert(MOST_ELEMENTS / NORM_UNIT * NORM_TENSORS < (int64_t)1 << 31, "units, and a stride of the grid beyond them, in 32 bits");

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
    NormArgs a;
    for (uint32_t& first : a.first) first = UINT32_MAX;
    int count = 0;
    int64_t units = 0;
    const bool first_launch = i == 0;
    for (; i < n_tensors && count < NORM_TENSORS; ++i) {
      const ll_tensor& t = tensors[i];
      if (t.n == 0) continue;
      a.tensors[count] = {t.grad, (t.flags & LL_TENSOR_GRAD_BF16) != 0 ? -t.n : t.n};
      a.first[count++] = (uint32_t)units;
      units += (t.n + NORM_UNIT - 1) / NORM_UNIT;
    }
    if (count == 0) continue;
    a.units = (uint32_t)units;
    a.partial = partial + parts;
    a.norm = nullptr;
    if (first_launch && i == n_tensors && units <= NORM_ALONE) {
      a.norm = out_norm;
      hipLaunchKernelGGL(ll_grad_norm_kernel<1024>, dim3(1), dim3(1024), 0, (hipStream_t)stream, a);
      LL_HIP_CHECK(hipGetLastError());
      return LL_OK;
    }
    const int64_t wanted = (units + 15) / 16;             // four units for each of a workgroup's four wavefronts
    const int groups = (int)(wanted < NORM_GROUPS ? wanted : NORM_GROUPS);
    hipLaunchKernelGGL(ll_grad_norm_kernel<THREADS>, dim3(groups), dim3(THREADS), 0, (hipStream_t)stream, a);
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
      for (uint32_t& first : a.first) first = UINT32_MAX;
      int64_t units = 0;
      for (; i < n_tensors && a.count < STEP_TENSORS; ++i) {
        const ll_tensor& t = tensors[i];
        if (t.n == 0 || t.flags != flags) continue;
        const int64_t more = (t.n + UNIT - 1) / UNIT;
        if (units + more > MOST_UNITS) break;
        a.tensors[a.count] = {t.param, t.grad, t.m, t.v, t.m_scale, t.v_scale, static_cast<uint16_t*>(t.copy), t.n, (uint32_t)i};
        a.first[a.count++] = (uint32_t)units;
        units += more;
      }
      if (a.count == 0) continue;
      hipLaunchKernelGGL(step_kernel(flags), dim3((unsigned)units), dim3(THREADS), 0, (hipStream_t)stream, a);
      LL_HIP_CHECK(hipGetLastError());
    }
  }
  return LL_OK;
}

}  // extern "C"
