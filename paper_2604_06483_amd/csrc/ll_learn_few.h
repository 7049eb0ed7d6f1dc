// Up to eight rows that learn through the lens: one read of W_U for the loss and the gradient together.
//
// With so few rows the gradient's sums, rows times d, fit the registers of every workgroup, and each of W_U's rows is used twice while it is
// there: for its logits, and then, times their exponentials, in the sums.  Exponents are relative to a running reference, as in a softmax over
// a stream; the workgroups' sums are joined by a second kernel, which adds the listed tokens' rows in fp32.
//
// A thread has NC chunks of eight columns, TPR threads a row of W_U, 512 / TPR groups side by side (d below 4096); a group takes R = 8 / NC
// rows at a time (eight rows: 4, for the registers) and has the next R in flight: 64 KB a compute unit.  The R x N products are summed over a wavefront by halving (each
// step adds two values' halves across lanes, so that 32 values take some 80 instructions and not 32 sums of six steps), over a group's
// wavefronts through LDS, one barrier for R rows, and go back to all lanes as scalars.
// Bound by the read of W_U up to four rows, by the fused multiply-adds above (N + 1 for each product of the two).
#pragma once

namespace {

constexpr int FEW_LEARN_THREADS = 512;
constexpr int FEW_LEARN_STREAMS = 256;      // workgroups that read W_U: one a compute unit
constexpr int FEW_LEARN_MAX_D = 16384;

struct FewLearnArgs {
  ListArgs list;            // rows, W, ids, k, d, V, to_log2
  int n, streams;           // rows; workgroups that read W_U (those behind them: the listed tokens' logits)
  int past_caches;          // W's loads go past the caches
  float* z;                 // [n, k]: the listed tokens' logits (nullptr: not asked for)
  float4* stats;            // [streams x groups, N]: (ref, S, T)
  float* sums;              // [streams x groups, N, d]
  // GRAD: what the row's dz is made of
  const float* lse;
  const float* entropy;
  const float* g_logp;
  const float* g_entropy;
  float temperature;
};

constexpr int log2_of(int x) { return x <= 1 ? 0 : 1 + log2_of(x / 2); }

template <int OFF>
__device__ __forceinline__ float lane_xor(float x) {
  return __uint_as_float(with_lane_xor<OFF>(__float_as_uint(x), [](uint32_t, uint32_t b) { return b; }));
}

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

template <int WHAT, int N, int NC, int TPR>
__global__ __launch_bounds__(FEW_LEARN_THREADS) void ll_learn_few_kernel(const FewLearnArgs p) {
  constexpr int R = (N == 8 ? 4 : 8) / NC, M = R * N, GROUPS = FEW_LEARN_THREADS / TPR, WAVES = TPR / 64, STEP = GROUPS * R;
  constexpr int VALUE_BIT = 6 - log2_of(M);        // value i is lane i << VALUE_BIT's
  constexpr float MOST = 0x1p24f;                  // (see LearnEpilogue)
  __shared__ float partial[2][FEW_LEARN_THREADS / 64][M];
  __shared__ float z[LIST_MAX];
  __shared__ GradTerms shared_terms[WHAT == GRAD ? N : 1];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const ListArgs& l = p.list;
  if ((int)blockIdx.x >= p.streams) {              // the listed tokens of one row
    const int row = blockIdx.x - p.streams;
    list_logits(l.rows + (int64_t)row * l.d, l.W, l.ids + (int64_t)row * l.k, l.k, l.d, l.V, z);
    if (tid < l.k) p.z[row * l.k + tid] = z[tid];
    return;
  }
  const int group = tid / TPR, in_group = tid % TPR, n8 = l.d >> 3;
  if (WHAT == GRAD) {
    for (int n = wave; n < N; n += FEW_LEARN_THREADS / 64) {
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
      const int c = in_group + TPR * i;
      a[n][i] = make_uint4(0, 0, 0, 0);
      if (n < p.n && c < n8) a[n][i] = reinterpret_cast<const uint4*>(l.rows + (int64_t)n * l.d)[c];
    }
  const int value = lane >> VALUE_BIT, my_n = value / R, my_r = value % R;
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
        at[r][i] = reinterpret_cast<const u32x4*>(l.W + (int64_t)min(step * STEP + group * R + r, l.V - 1) * l.d) + min(in_group + TPR * i, n8 - 1);
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
  uint4 w[R][NC], next[R][NC];
  if (step0 < step1) load(step0, w);
  for (int step = step0; step < step1; ++step) {
    load(min(step + 1, step1 - 1), next);
    float dots[M];
#pragma unroll
    for (int r = 0; r < R; ++r) {
#pragma unroll
      for (int n = 0; n < N; ++n) dots[n * R + r] = 0.f;
#pragma unroll
      for (int i = 0; i < NC; ++i) {
        const uint32_t ws[4] = {w[r][i].x, w[r][i].y, w[r][i].z, w[r][i].w};
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const float lo = bf16_lo(ws[q]), hi = bf16_hi(ws[q]);
#pragma unroll
          for (int n = 0; n < N; ++n) {
            const uint32_t as = q == 0 ? a[n][i].x : q == 1 ? a[n][i].y : q == 2 ? a[n][i].z : a[n][i].w;
            dots[n * R + r] = fmaf(lo, bf16_lo(as), dots[n * R + r]);
            dots[n * R + r] = fmaf(hi, bf16_hi(as), dots[n * R + r]);
          }
        }
      }
    }
    float x = sum_across<M>(dots);
    if (WAVES > 1) {
      const int turn = (step - step0) & 1;   // (written again two steps on, behind a barrier that follows every read)
      if ((lane & ((1 << VALUE_BIT) - 1)) == 0) partial[turn][wave][value] = x;
      __syncthreads();
      x = 0.f;
#pragma unroll
      for (int o = 0; o < WAVES; ++o) x += partial[turn][group * WAVES + o][value];
    }
    const bool inside = step * STEP + group * R + my_r < l.V;
    x *= l.to_log2;
    float e = inside ? x - ref : MASKED;
    float prob = __builtin_amdgcn_exp2f(e);
    if (WHAT != GRAD && __builtin_amdgcn_ballot_w64(prob > MOST) != 0) {
      const auto most = [](uint32_t u, uint32_t v) { return __float_as_uint(fmaxf(__uint_as_float(u), __uint_as_float(v))); };
      const float m = __uint_as_float(over_bits<VALUE_BIT, log2_of(R)>(__float_as_uint(inside ? x : NEG_BIG), most));
      const float to_ref = m - ref > 24.f ? m : ref, before = ref - to_ref, keep = __builtin_amdgcn_exp2f(before);
      t = keep * fmaf(before, s, t);
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
    if (WHAT == GRAD) prob *= fmaf(term_b, e, term_a);
    if (WHAT != STATS) {
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
    }
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
      for (int i = 0; i < NC; ++i) w[r][i] = next[r][i];
  }
  const int part = blockIdx.x * GROUPS + group;
  if (WHAT != GRAD) {
    const auto add = [](uint32_t u, uint32_t v) { return __float_as_uint(__uint_as_float(u) + __uint_as_float(v)); };
    s = __uint_as_float(over_bits<VALUE_BIT, log2_of(R)>(__float_as_uint(s), add));
    t = __uint_as_float(over_bits<VALUE_BIT, log2_of(R)>(__float_as_uint(t), add));
    if (wave % WAVES == 0 && my_r == 0 && (lane & ((1 << VALUE_BIT) - 1)) == 0) p.stats[(int64_t)part * N + my_n] = make_float4(ref, s, t, 0.f);
  }
  if (WHAT != STATS) {
#pragma unroll
    for (int n = 0; n < N; ++n)
#pragma unroll
      for (int i = 0; i < NC; ++i) {
        const int c = in_group + TPR * i;
        if (c >= n8 || n >= p.n) continue;
        float4* to = reinterpret_cast<float4*>(p.sums + ((int64_t)part * N + n) * l.d + 8 * c);
        to[0] = make_float4(acc[n][i][0], acc[n][i][1], acc[n][i][2], acc[n][i][3]);
        to[1] = make_float4(acc[n][i][4], acc[n][i][5], acc[n][i][6], acc[n][i][7]);
      }
  }
}

// ll_logp of few rows: statistics from the parts, a row a workgroup.
__global__ __launch_bounds__(64) void ll_logp_few_finish_kernel(const ListArgs p, const float* __restrict__ z, const float4* __restrict__ stats,
                                                                int parts, int stride, float* __restrict__ logp, float* __restrict__ lse,
                                                                float* __restrict__ entropy) {
  const int row = blockIdx.x, lane = threadIdx.x;
  const RowStats r = join_stats(stats + row, parts, lane, stride);
  if (lane == 0) {
    lse[row] = r.lse2 * LN2;
    entropy[row] = -r.t * LN2;
  }
  if (lane < p.k) {
    const int e = row * p.k + lane;
    logp[e] = p.ids[e] >= 0 && p.ids[e] < p.V ? fmaf(z[e], p.to_log2, -r.lse2) * LN2 : NAN;
  }
}

// The parts' sums joined, and the listed tokens' rows of W: block (64 columns, row), sixteen runs of the parts and of the list side by side.
// DISTILL: parts relative to their references, dA = a (sum p W - sum t W_id), and the loss; else sums of dz W, and g / T W_id.
struct FewJoinArgs {
  FewLearnArgs f;
  int parts, stride;        // stride: rows of a part's sums and statistics
  const float* scores;
  const float* weight;
  float* loss;
  uint16_t* out;
};
constexpr int FEW_LEARN_MAX_PARTS = FEW_LEARN_STREAMS * (FEW_LEARN_THREADS / 64);
template <bool DISTILL>
__global__ __launch_bounds__(256) void ll_learn_few_join_kernel(const FewJoinArgs p) {
  __shared__ float scale[DISTILL ? FEW_LEARN_MAX_PARTS : 1];
  __shared__ float4 red[16][16];
  __shared__ float share[LIST_MAX];
  __shared__ int id_of[LIST_MAX];
  __shared__ float shared_factor, shared_ref;
  const ListArgs& l = p.f.list;
  const int row = blockIdx.y, k = l.k, lane = threadIdx.x & 63;
  const float temperature = p.f.temperature;
  if (threadIdx.x < 64) {
    const int e = row * k + lane;
    const int id = lane < k ? l.ids[e] : -1;
    if (DISTILL) {
      const RowStats r = join_stats(p.f.stats + row, p.parts, lane, p.stride);
      const Teacher teacher = teacher_of(id, lane < k ? p.scores[e] : -INFINITY, l.V, temperature);
      const float q = fmaf(lane < k ? p.f.z[e] : 0.f, l.to_log2, -r.lse2);
      const float loss = distill_loss(teacher, q * LN2, temperature);
      const float a = temperature * (p.weight != nullptr ? p.weight[row] : 1.f);
      if (lane == 0) {
        if (blockIdx.x == 0) p.loss[row] = loss;
        shared_factor = teacher.some ? a : 0.f;
        shared_ref = r.lse2;
      }
      share[lane] = -teacher.t;
      id_of[lane] = teacher.valid ? id : -1;
    } else {
      const bool valid = id >= 0 && id < l.V;
      const float g = valid ? p.f.g_logp[e] : 0.f;
      const bool live = __builtin_amdgcn_ballot_w64(g != 0.f) != 0 || (p.f.g_entropy != nullptr && p.f.g_entropy[row] != 0.f);
      if (lane == 0) shared_factor = live ? 1.f : 0.f;
      share[lane] = g / temperature;
      id_of[lane] = valid ? id : -1;
    }
  }
  __syncthreads();
  if (DISTILL) {
    for (int i = threadIdx.x; i < p.parts; i += 256) {
      const float4 q = p.f.stats[(int64_t)i * p.stride + row];
      scale[i] = q.y > 0.f || q.y != q.y ? __builtin_amdgcn_exp2f(q.x - shared_ref) : 0.f;
    }
    __syncthreads();
  }
  const int col = threadIdx.x & 15, run = threadIdx.x >> 4, c = blockIdx.x * 64 + col * 4;
  const float factor = shared_factor;
  float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
  if (c < l.d && factor != 0.f) {
    const float* from = p.f.sums + (int64_t)row * l.d + c;
    const int64_t stride = (int64_t)p.stride * l.d;
#pragma unroll 8
    for (int i = run; i < p.parts; i += 16) {
      const float4 x = *reinterpret_cast<const float4*>(from + i * stride);
      const float by = DISTILL ? scale[i] : 1.f;
      s.x = fmaf(by, x.x, s.x);
      s.y = fmaf(by, x.y, s.y);
      s.z = fmaf(by, x.z, s.z);
      s.w = fmaf(by, x.w, s.w);
    }
    for (int i = run; i < k; i += 16) {
      if (id_of[i] < 0) continue;
      const uint2 w = *reinterpret_cast<const uint2*>(l.W + (int64_t)id_of[i] * l.d + c);
      const float by = share[i];
      s.x = fmaf(by, bf16_lo(w.x), s.x);
      s.y = fmaf(by, bf16_hi(w.x), s.y);
      s.z = fmaf(by, bf16_lo(w.y), s.z);
      s.w = fmaf(by, bf16_hi(w.y), s.w);
    }
  }
  red[run][col] = s;
  __syncthreads();
  if (run != 0 || c >= l.d) return;
#pragma unroll
  for (int i = 1; i < 16; ++i) {
    const float4 x = red[i][col];
    s.x += x.x;
    s.y += x.y;
    s.z += x.z;
    s.w += x.w;
  }
  *reinterpret_cast<uint2*>(p.out + (int64_t)row * l.d + c) = make_uint2(pack_bf16(factor * s.x, factor * s.y), pack_bf16(factor * s.z, factor * s.w));
}

}  // namespace
