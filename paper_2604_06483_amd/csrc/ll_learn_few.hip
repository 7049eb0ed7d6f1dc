// Up to four rows that learn through the lens (eight, for the statistics alone): one read of W_U for the loss and the gradient together.
//
// With so few rows the gradient's sums, rows times d, fit the registers of every workgroup, and each of W_U's rows is used twice while it is
// there: for its logits, and then, times their exponentials, in the sums.  Exponents are relative to a running reference, as in a softmax over
// a stream; the workgroups' sums are joined by a second kernel, which adds the listed tokens' rows in fp32.
//
// A thread has NC chunks of eight columns.  Below d = 2056 several groups of threads take rows of W_U side by side, GROUPS of them in 512
// threads; else a row has the workgroup, of just the wavefronts that it needs.  A group takes R rows at a time and has the next 2 R
// there or in flight, up to 128 KB a compute unit.  The R x N products are summed over a wavefront by halving (each step adds two values' halves
// across lanes, so that 32 values take some 80 instructions and not 32 sums of six steps), over a group's wavefronts through LDS, one
// barrier for R rows, and go back to all lanes as scalars.  That is a long chain of waits for the two wavefronts of a SIMD, so from three
// rows on the R rows before are added to the sums behind the barrier, while the next R rows' logits come out of LDS (d = 2560, V = 151936, 4
// rows 209 | 192 us, 5120 360 | 330; for one or two rows the third buffer costs 2 to 4 %: d = 8192 341 | 355).
// Bound by the read of W_U up to four rows, by the fused multiply-adds above: 8 N + 8 instructions for a chunk's part of the sums, and
// half of 8 N for its logits (v_dot2_f32_bf16: two products a lane, fp32 sums, as exact as two fused multiply-adds).
#include "ll_learn.h"

namespace {

constexpr int log2_of(int x) { return x <= 1 ? 0 : 1 + log2_of(x / 2); }

// v[0 .. M): values of every lane.  Returns one sum over the wavefront a lane, of value (lane >> (6 - log2 M)).
template <int M, int OFF = 32>
__device__ __forceinline__ float sum_across(float (&v)[M > 0 ? M : 1]) {
  if constexpr (OFF == 0) {
    return v[0];
  } else if constexpr (M == 1) {
    float one[1] = {__uint_as_float(with_lane_xor<OFF>(__float_as_uint(v[0]), [](uint32_t a, uint32_t b) {
      return __float_as_uint(__uint_as_float(a) + __uint_as_float(b));
    }))};
    return sum_across<1, OFF / 2>(one);
  } else {
    float half[M / 2];
#pragma unroll
    for (int i = 0; i < M / 2; ++i) {
      const uint32_t x = __float_as_uint(v[i]), y = __float_as_uint(v[i + M / 2]);
      if constexpr (OFF == 32) {   // lanes 0 .. 31 get x's two halves, the others y's
        const auto p = __builtin_amdgcn_permlane32_swap(x, y, false, false);
        half[i] = __uint_as_float(p[0]) + __uint_as_float(p[1]);
      } else if constexpr (OFF == 16) {
        const auto p = __builtin_amdgcn_permlane16_swap(x, y, false, false);
        half[i] = __uint_as_float(p[0]) + __uint_as_float(p[1]);
      } else {
        const bool upper = (threadIdx.x & OFF) != 0;
        uint32_t send = upper ? x : y;
        if constexpr (OFF == 8) send = dpp<0x128>(send);
        else if constexpr (OFF == 4) send = dpp<0x1B>(dpp<0x141>(send));
        else send = dpp<OFF == 2 ? 0x4E : 0xB1>(send);
        half[i] = __uint_as_float(upper ? y : x) + __uint_as_float(send);
      }
    }
    return sum_across<M / 2, OFF / 2>(half);
  }
}

// x combined with the lanes that differ in the COUNT bits from lane bit FROM up.
template <int FROM, int COUNT, class F>
__device__ __forceinline__ uint32_t over_bits(uint32_t x, F f) {
  if constexpr (COUNT == 0) return x;
  else return over_bits<FROM + 1, COUNT - 1>(with_lane_xor<(1 << FROM)>(x, f), f);
}

__device__ __forceinline__ float from_lane(float x, int lane) { return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(x), lane)); }

__device__ __forceinline__ float dot2(uint32_t a, uint32_t b, float c) {
  return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2_t, a), __builtin_bit_cast(bf16x2_t, b), c, false);
}

template <int WHAT, int N, int NC, int GROUPS>
__device__ __forceinline__ void few_rows(const FewLearnArgs& p) {
  constexpr int R = few_learn_rows(N, NC), M = R * N, STEP = GROUPS * R;
  const int tpr = GROUPS > 1 ? FEW_LEARN_THREADS / GROUPS : blockDim.x;      // threads to a row of W
  constexpr int WAVES = GROUPS > 1 ? FEW_LEARN_THREADS / GROUPS / 64 : FEW_LEARN_THREADS / 64;   // of a group, at most
  constexpr int VALUE_BIT = 6 - log2_of(M);        // value i is lane i << VALUE_BIT's
  constexpr float MOST = 0x1p24f;                  // (see LearnEpilogue)
  __shared__ float partial[2][FEW_LEARN_THREADS / 64][M];
  __shared__ float z[LIST_MAX];
  __shared__ GradTerms shared_terms[WHAT == GRAD ? N : 1];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const ListArgs& l = p.list;
  if ((int)blockIdx.x >= p.streams) {              // the listed tokens of one row
    const int row = blockIdx.x - p.streams;
    list_logits(l, row, z);
    if (tid < l.k) p.z[row * l.k + tid] = z[tid];
    return;
  }
  const int group = GROUPS > 1 ? tid / tpr : 0, in_group = GROUPS > 1 ? tid % tpr : tid, n8 = l.d >> 3;
  if (WHAT == GRAD) {
    for (int n = wave; n < N; n += (int)(blockDim.x >> 6)) {
      const int row = min(n, p.n - 1);
      const int e = row * l.k + lane, id = lane < l.k ? l.ids[e] : -1;
      const GradTerms t = grad_terms(id >= 0 && id < l.V ? p.g_logp[e] : 0.f, p.lse[row], p.g_entropy != nullptr ? p.g_entropy[row] : 0.f,
                                     p.entropy != nullptr ? p.entropy[row] : 0.f, 1.f / p.temperature);
      if (lane == 0) shared_terms[n] = t;
    }
    __syncthreads();
  }
  uint4 a[N][NC];
#pragma unroll
  for (int n = 0; n < N; ++n)
#pragma unroll
    for (int i = 0; i < NC; ++i) {
      const int c = in_group + tpr * i;
      a[n][i] = make_uint4(0, 0, 0, 0);
      if (n < p.n && c < n8) a[n][i] = reinterpret_cast<const uint4*>(l.rows + (int64_t)n * l.d)[c];
    }
  const int value = lane >> VALUE_BIT, my_n = value / R, my_r = value % R;
  const int own = WHAT == OTHERS && my_n < p.n ? l.ids[my_n] : -1;     // OTHERS: one token a row, as in ll_learn_gemm.hip
  float ref = NEG_BIG, s = 0.f, t = 0.f, term_a = 0.f, term_b = 0.f;   // of the lane's own value
  if (WHAT == GRAD) {
    ref = shared_terms[my_n].lse2;
    term_a = shared_terms[my_n].a;
    term_b = shared_terms[my_n].b;
  }
  float acc[N][NC][8];
#pragma unroll
  for (int n = 0; n < N; ++n)
#pragma unroll
    for (int i = 0; i < NC; ++i)
#pragma unroll
      for (int e = 0; e < 8; ++e) acc[n][i][e] = 0.f;

  const int steps = (l.V + STEP - 1) / STEP;
  const int step0 = (int)((int64_t)blockIdx.x * steps / p.streams), step1 = (int)((int64_t)(blockIdx.x + 1) * steps / p.streams);
  const auto load = [&](int step, uint4 (&w)[R][NC]) {
    typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
    const u32x4* at[R][NC];
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
      for (int i = 0; i < NC; ++i)
        at[r][i] = reinterpret_cast<const u32x4*>(l.W + (int64_t)min(step * STEP + group * R + r, l.V - 1) * l.d) + min(in_group + tpr * i, n8 - 1);
    if (p.past_caches) {
#pragma unroll
      for (int r = 0; r < R; ++r)
#pragma unroll
        for (int i = 0; i < NC; ++i) {
          const u32x4 x = __builtin_nontemporal_load(at[r][i]);
          w[r][i] = make_uint4(x[0], x[1], x[2], x[3]);
        }
    } else {
#pragma unroll
      for (int r = 0; r < R; ++r)
#pragma unroll
        for (int i = 0; i < NC; ++i) {
          const u32x4 x = *at[r][i];
          w[r][i] = make_uint4(x[0], x[1], x[2], x[3]);
        }
    }
  };
  if (WAVES > 1 && GROUPS == 1) {   // (wavefronts that this d does without add nothing)
    for (int i = tid; i < 2 * WAVES * M; i += (int)blockDim.x) (&partial[0][0][0])[i] = 0.f;
    __syncthreads();
  }
  // The products of R rows, as far as the wavefront goes, and behind a barrier those of the group's wavefronts.
  const auto dots_of = [&](const uint4 (&w)[R][NC], int step, float (&sums)[WAVES]) {
    float dots[M];
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
      for (int n = 0; n < N; ++n) {
        float to = 0.f;
#pragma unroll
        for (int i = 0; i < NC; ++i) {
          to = dot2(w[r][i].x, a[n][i].x, to);
          to = dot2(w[r][i].y, a[n][i].y, to);
          to = dot2(w[r][i].z, a[n][i].z, to);
          to = dot2(w[r][i].w, a[n][i].w, to);
        }
        dots[n * R + r] = to;
      }
    const float x = sum_across<M>(dots);
    if constexpr (WAVES == 1) {
      sums[0] = x;
    } else {
      const int turn = (step - step0) & 1;   // (written again two steps on, behind a barrier that follows every read)
      if ((lane & ((1 << VALUE_BIT) - 1)) == 0) partial[turn][wave][value] = x;
      __syncthreads();
#pragma unroll
      for (int o = 0; o < WAVES; ++o) sums[o] = partial[turn][group * WAVES + o][value];
    }
  };
  const auto add_rows = [&](const uint4 (&w)[R][NC], float prob) {
#pragma unroll
    for (int r = 0; r < R; ++r) {
      float by[N];
#pragma unroll
      for (int n = 0; n < N; ++n) by[n] = from_lane(prob, (n * R + r) << VALUE_BIT);
#pragma unroll
      for (int i = 0; i < NC; ++i) {
        const uint32_t ws[4] = {w[r][i].x, w[r][i].y, w[r][i].z, w[r][i].w};
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const float lo = bf16_lo(ws[q]), hi = bf16_hi(ws[q]);
#pragma unroll
          for (int n = 0; n < N; ++n) {
            acc[n][i][2 * q] = fmaf(by[n], lo, acc[n][i][2 * q]);
            acc[n][i][2 * q + 1] = fmaf(by[n], hi, acc[n][i][2 * q + 1]);
          }
        }
      }
    }
  };
  // The lane's own value: its logit's exponential, or dz.
  const auto weigh = [&](const float (&sums)[WAVES], int step) {
    float x = sums[0];
#pragma unroll
    for (int o = 1; o < WAVES; ++o) x += sums[o];
    const bool inside = step * STEP + group * R + my_r < l.V;
    x *= l.to_log2;
    float e = inside ? x - ref : MASKED;
    float prob = __builtin_amdgcn_exp2f(e);
    if (WHAT != GRAD && __builtin_amdgcn_ballot_w64(prob > MOST) != 0) {
      const auto most = [](uint32_t u, uint32_t v) { return __float_as_uint(fmaxf(__uint_as_float(u), __uint_as_float(v))); };
      const float m = __uint_as_float(over_bits<VALUE_BIT, log2_of(R)>(__float_as_uint(inside ? x : NEG_BIG), most));
      const float to_ref = m - ref > 24.f ? m : ref, before = ref - to_ref, keep = __builtin_amdgcn_exp2f(before);
      t = keep * (WHAT == OTHERS ? t : fmaf(before, s, t));
      s *= keep;
      ref = to_ref;
#pragma unroll
      for (int n = 0; n < N; ++n) {
        const float by = from_lane(keep, (n * R) << VALUE_BIT);
#pragma unroll
        for (int i = 0; i < NC; ++i)
#pragma unroll
          for (int q = 0; q < 8; ++q) acc[n][i][q] *= by;
      }
      e = inside ? x - ref : MASKED;
      prob = __builtin_amdgcn_exp2f(e);
    }
    s += prob;
    if (WHAT == STATS) t = fmaf(prob, e, t);
    if (WHAT == OTHERS) {
      prob = step * STEP + group * R + my_r == own ? 0.f : prob;
      t += prob;
    }
    return WHAT == GRAD ? prob * fmaf(term_b, e, term_a) : prob;
  };
  if constexpr (N <= 2) {   // few instructions beside the read: one step after the other
    const auto take = [&](int step, const uint4 (&w)[R][NC], uint4 (&next)[R][NC]) {
      load(min(step + 1, step1 - 1), next);
      float sums[WAVES];
      dots_of(w, step, sums);
      const float prob = weigh(sums, step);
      if (WHAT != STATS) add_rows(w, prob);
    };
    uint4 w0[R][NC], w1[R][NC];
    if (step0 < step1) load(step0, w0);
    for (int step = step0; step < step1; step += 2) {
      take(step, w0, w1);
      if (step + 1 < step1) take(step + 1, w1, w0);
    }
  } else {
    // Rows of step, step + 1 (both there) and step + 2 (loaded): the first into the sums, the second's weights.
    float prob = 0.f;
    const auto advance = [&](int step, const uint4 (&w)[R][NC], const uint4 (&next)[R][NC], uint4 (&far)[R][NC]) {
      const bool more = step + 1 < step1;
      load(min(step + 2, step1 - 1), far);
      float sums[WAVES];
      if (more) dots_of(next, step + 1, sums);
      if (WHAT != STATS) add_rows(w, prob);
      if (more) prob = weigh(sums, step + 1);
    };
    uint4 w0[R][NC], w1[R][NC], w2[R][NC];
    if (step0 < step1) {
      load(step0, w0);
      load(min(step0 + 1, step1 - 1), w1);
      float sums[WAVES];
      dots_of(w0, step0, sums);
      prob = weigh(sums, step0);
    }
    for (int step = step0; step < step1; step += 3) {
      advance(step, w0, w1, w2);
      if (step + 1 < step1) advance(step + 1, w1, w2, w0);
      if (step + 2 < step1) advance(step + 2, w2, w0, w1);
    }
  }
  const bool speaks = wave % WAVES == 0 && my_r == 0 && (lane & ((1 << VALUE_BIT) - 1)) == 0;   // for a lens row of its group
  if (WHAT != GRAD) {
    const auto add = [](uint32_t u, uint32_t v) { return __float_as_uint(__uint_as_float(u) + __uint_as_float(v)); };
    s = __uint_as_float(over_bits<VALUE_BIT, log2_of(R)>(__float_as_uint(s), add));
    t = __uint_as_float(over_bits<VALUE_BIT, log2_of(R)>(__float_as_uint(t), add));
  }
  const int64_t part = blockIdx.x;
  if constexpr (GROUPS == 1) {
    if (WHAT != GRAD && speaks) p.stats[part * N + my_n] = make_float4(ref, s, t, 0.f);
    if (WHAT != STATS) {
#pragma unroll
      for (int n = 0; n < N; ++n)
#pragma unroll
        for (int i = 0; i < NC; ++i) {
          const int c = in_group + tpr * i;
          if (c >= n8 || n >= p.n) continue;
          float4* to = reinterpret_cast<float4*>(p.sums + (part * N + n) * l.d + 8 * c);
          to[0] = make_float4(acc[n][i][0], acc[n][i][1], acc[n][i][2], acc[n][i][3]);
          to[1] = make_float4(acc[n][i][4], acc[n][i][5], acc[n][i][6], acc[n][i][7]);
        }
    }
  } else {   // the groups' sums first joined here (one chunk a thread: NC is 1)
    __shared__ float4 of_group[WHAT != GRAD ? GROUPS : 1][N];
    __shared__ float columns[WHAT != STATS ? FEW_LEARN_THREADS * 8 : 1];
    if (WHAT != GRAD) {
      if (speaks) of_group[group][my_n] = make_float4(ref, s, t, 0.f);
      __syncthreads();
    }
#pragma unroll
    for (int n = 0; n < N; ++n) {
      float by = 1.f;
      if (WHAT != GRAD) {
        float m = NEG_BIG;
        for (int g = 0; g < GROUPS; ++g) m = fmaxf(m, of_group[g][n].y > 0.f ? of_group[g][n].x : NEG_BIG);
        by = of_group[group][n].y == 0.f ? 0.f : __builtin_amdgcn_exp2f(of_group[group][n].x - m);
        if (tid == n) {
          float sum_s = 0.f, sum_t = 0.f;
          for (int g = 0; g < GROUPS; ++g) {
            const float4 q = of_group[g][n];
            const float before = q.x - m, keep = __builtin_amdgcn_exp2f(before);
            if (q.y == 0.f) continue;
            sum_s = fmaf(keep, q.y, sum_s);
            sum_t += keep * (WHAT == OTHERS ? q.z : fmaf(before, q.y, q.z));
          }
          p.stats[part * N + n] = make_float4(m, sum_s, sum_t, 0.f);
        }
      }
      if (WHAT == STATS || n >= p.n) continue;
#pragma unroll
      for (int q = 0; q < 8; ++q) columns[tid * 8 + q] = by == 0.f ? 0.f : by * acc[n][0][q];
      __syncthreads();
      for (int c = tid; c < l.d; c += FEW_LEARN_THREADS) {
        float sum = 0.f;
        for (int g = 0; g < GROUPS; ++g) sum += columns[g * tpr * 8 + c];
        p.sums[(part * N + n) * l.d + c] = sum;
      }
      __syncthreads();
    }
  }
}

template <int WHAT, int N, int NC, int GROUPS>
__global__ __launch_bounds__(FEW_LEARN_THREADS) void ll_learn_few_kernel(const FewLearnArgs p) {
  few_rows<WHAT, N, NC, GROUPS>(p);
}

template <int N, int NC, int GROUPS>
__global__ __launch_bounds__(FEW_LEARN_THREADS) void ll_learn_few_others_kernel(const FewLearnArgs p) {
  few_rows<OTHERS, N, NC, GROUPS>(p);
}

template <int WHAT, int N, int NC, int GROUPS>
constexpr FewLearnKernel few_kernel() {
  if constexpr (WHAT == OTHERS) return ll_learn_few_others_kernel<N, NC, GROUPS>;
  else return ll_learn_few_kernel<WHAT, N, NC, GROUPS>;
}

}  // namespace

namespace ll {

FewLearnKernel few_learn_kernel(LearnWhat what, int rows, int chunks, int groups) {
  const auto pick = [&](auto w, auto n) -> FewLearnKernel {
    constexpr int WHAT = w(), N = n();
    if constexpr (N <= 4) {
      if (groups == 8) return few_kernel<WHAT, N, 1, 8>();
      if (groups == 4) return few_kernel<WHAT, N, 1, 4>();
      if (groups == 2) return few_kernel<WHAT, N, 1, 2>();
    }
    if (chunks == 1) return few_kernel<WHAT, N, 1, 1>();
    if (chunks == 2) return few_kernel<WHAT, N, 2, 1>();
    if constexpr (N <= 2) return few_kernel<WHAT, N, 4, 1>();
    return nullptr;
  };
  const auto of = [&](auto w) -> FewLearnKernel {
    using std::integral_constant;
    if (rows == 1) return pick(w, integral_constant<int, 1>{});
    if (rows == 2) return pick(w, integral_constant<int, 2>{});
    if (rows == 4) return pick(w, integral_constant<int, 4>{});
    if constexpr (w() == STATS) return pick(w, integral_constant<int, 8>{});
    return nullptr;
  };
  if (what == STATS) return of(std::integral_constant<int, STATS>{});
  if (what == OTHERS) return of(std::integral_constant<int, OTHERS>{});
  if (what == EXPS) return of(std::integral_constant<int, EXPS>{});
  return of(std::integral_constant<int, GRAD>{});
}

}  // namespace ll
