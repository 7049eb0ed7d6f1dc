// Learning from answers through the lens: a clipped policy loss with a KL term over sampled tokens, and a preference loss over pairs of
// answers, each with its gradient to the (normalised) rows.
//
//   l = log softmax(a W^T / T)[id],   dA = c / T (W_id - sum_v p_v W_v),   c = d loss / d l
//
// Both products are those of distillation (ll_learn.hip): the first leaves P = 2^(x - base) behind it in bf16, the second multiplies P by W_U.
// The row's own token is left out of P and its whole part, p - 1, which outweighs all others', joins the sums in fp32: rounded into P it would
// be most of the gradient's error (rms, of the gradient: 0.0026 with it in P, 0.0017 without, which is the result's own rounding).  p - 1 is the
// others' sum over the whole, negated, and the first product keeps that sum by itself: with p next to 1 the difference is rounding.
// What is new is c.  Nothing of it is needed before the second product's sums are rounded, where it is a factor of the row, so that the logits
// are formed once: with the log-probabilities and their gradient as two calls there is a third product.  Whole calls, us, ll_policy | ll_logp, the loss in torch, ll_logp_grad: 1 row, d = 4096, V = 128256 175 | 364; 111,
// 1608, 50257 104 | 161; 1500, 4096, 128256 2229 | 3190 (1.41 PFLOP/s; the vendor's bare product of that shape 1.28); 6000, 2560, 151936 6666 | 9510.
//
// A policy's c is the row's own.  A preference's is known when every row of its pair has been through W_U.  Up to one pass of rows the
// pairs are joined between the two products; beyond, every pass's sums stay in fp32 (4 d bytes a row and slice of the vocabulary, beside
// 4 d V flops) and are joined, scaled and rounded once behind the last pass: no product is formed again, however long the answers are.
#include "ll_learn_host.h"

namespace {

// What a row's gradient is made of: factor (P's product with W_U + own W_id).
struct AnswerTerms {
  float rest;               // what 32 bits leave of the log-probability
  float unit;               // the factor without c
  float own;                // the own token's part, (p - 1) 2^(lse2 - base)
  float factor;             // unit c; 0: the row takes no part
};

struct PolicyArgs {
  const float* advantage;
  const float* old_logp;    // or nullptr: the log-probability itself
  const float* ref_logp;    // or nullptr: no KL term
  const float* weight;      // or nullptr: 1
  float* loss;
  float low, high, kl;
};

struct AnswerArgs {
  const int32_t* ids;
  const float* z;             // the tokens' logits
  const float4* stats;
  int parts, stride;          // parts of a row, and rows between them (1: a row's are side by side)
  int V;
  float to_log2, inv_t;
  float* logp;
  AnswerTerms* terms;         // or nullptr: no gradient
  uint16_t* P;                // the products', where there are terms; else nullptr
  int64_t ldp;
  const float* ref;           // [rows], or nullptr: 0
  const float* moved;         // [rows, tiles]: what the exponents of a tile of `width` ids are relative to
  int tiles, width;
  PolicyArgs policy;
};

// Loss of a sampled token and what it gains by the token's log-probability.  A ratio on the border of the clipping counts as inside; an advantage of 0
// has no loss, whatever the ratio, but that of a row that holds no number.
struct PolicyTerm {
  float loss, c;
};
__device__ __forceinline__ PolicyTerm policy_term(const PolicyArgs& p, int64_t row, float logp) {
  const float A = p.advantage[row];
  const float ratio = p.old_logp != nullptr ? expf(logp - p.old_logp[row]) : 1.f;
  const float most = 1.f + p.high, least = 1.f - p.low;
  const bool clipped = A > 0.f ? ratio > most : ratio < least;
  PolicyTerm r;
  r.loss = A == 0.f ? 0.f : -A * (clipped ? (A > 0.f ? most : least) : ratio);
  r.c = A == 0.f || clipped ? 0.f : -A * ratio;
  if (logp != logp) r.loss = r.c = logp;
  if (p.ref_logp != nullptr) {
    const float q = p.ref_logp[row] - logp, e = expm1f(q);     // e^q - 1 keeps its digits where the two policies are near
    r.loss = fmaf(p.kl, e - q, r.loss);
    r.c = fmaf(-p.kl, e, r.c);
  }
  r.c *= p.weight != nullptr ? p.weight[row] : 1.f;
  if (p.weight != nullptr && p.weight[row] == 0.f) r.c = 0.f;  // (whatever the row holds)
  return r;
}

// A token's log-probability in powers of two, in 64 bits: a score's small log-ratios are differences of these, and the last bit of 32 at their
// size would be most of a short answer's error.  The reference and the sum's exponent come off before a logarithm is taken, at the size of 1.
__device__ __forceinline__ double log2_p(float z, float to_log2, const RowStats& r) {
  const float rest = __builtin_amdgcn_logf(__builtin_amdgcn_frexp_mantf(r.sum));          // of [1/2, 1)
  return (((double)z * (double)to_log2 - (double)r.ref) - (double)__builtin_amdgcn_frexp_expf(r.sum)) - (double)rest;
}
constexpr double LN2_64 = 0.69314718055994530942;
// The log-probability itself, beside a gradient: above a half from the others' part, of which it has every digit.
__device__ __forceinline__ double log_p(float z, float to_log2, const RowStats& r) {
  return r.t < 0.5f * r.sum ? (double)log1pf(-r.t / r.sum) : log2_p(z, to_log2, r) * LN2_64;
}

// Before the first product: the rows padded, the tokens' logits (before the temperature; 0 without a token; with a gradient the product's own take
// their place), and what P starts from, as in ll_distill_lists_kernel.  One token a row, so a workgroup shares a row, and has all of it in flight at once.
__global__ __launch_bounds__(256) void ll_answers_tokens_kernel(const ListArgs p, float* __restrict__ z, float* __restrict__ ref, uint16_t* __restrict__ panel,
                                                                int64_t lda) {
  __shared__ float part[4];
  const int64_t row = blockIdx.x;
  const int id = p.ids[row];
  const bool valid = id >= 0 && id < p.V;
  const uint4* const a = reinterpret_cast<const uint4*>(p.rows + row * p.d);
  const uint4* const w = reinterpret_cast<const uint4*>(p.W + (valid ? (int64_t)id * p.d : 0));
  float s[2] = {0.f, 0.f};
#pragma unroll 4
  for (int c = threadIdx.x; c < p.d / 8; c += 256) {
    const uint4 x = a[c], y = w[c];
    const uint32_t xs[4] = {x.x, x.y, x.z, x.w}, ys[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      s[0] = fmaf(bf16_lo(xs[q]), bf16_lo(ys[q]), s[0]);
      s[1] = fmaf(bf16_hi(xs[q]), bf16_hi(ys[q]), s[1]);
    }
    if (panel != nullptr) reinterpret_cast<uint4*>(panel + row * lda)[c] = x;
  }
  if (panel != nullptr && (int)threadIdx.x < lda / 8 - p.d / 8) reinterpret_cast<uint4*>(panel + row * lda)[p.d / 8 + threadIdx.x] = make_uint4(0, 0, 0, 0);
  const float sum = wave_sum(s[0] + s[1]);
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = sum;
  __syncthreads();
  if (threadIdx.x != 0) return;
  const float logit = valid ? (part[0] + part[1]) + (part[2] + part[3]) : 0.f, most = logit * p.to_log2;
  z[row] = logit;
  ref[row] = fabsf(most) < 1e30f ? rintf(most) : 0.f;
}

// The first product where the vocabulary is too short for the direct-to-LDS kernel (ll_learn_gemm.hip): its tiles of 256 ids leave compute units
// without one, and each that has one waits for a stage of 64 columns after the other (9 x 3024 x 19314: 76 workgroups, 56 us for 117 MB).
// Here a workgroup has 16 VT ids and 16 RT rows, and its four wavefronts a quarter of the columns each, so that there are several times as
// many workgroups and every wavefront has 4 (VT + RT) loads of 16 bytes a lane in flight, with nothing to wait for but its own.  W's and the rows'
// fragments come straight from memory (a load is 16 rows' 64 bytes, the next the other half of their lines); the rows are read where they are,
// whatever d.  The quarters are joined through LDS, in one order, and wavefront j makes statistics and exponentials of row tile j.  They are relative
// to 0, which is as good as any reference within 60 powers of two of the largest logit; a workgroup whose ids are further off takes its own largest, a
// whole number (see LearnEpilogue).  The row's token is met on the way: its logit goes to z, its place in P is 0, and the sum without it is kept.
struct ShortArgs {
  const uint16_t* rows;
  const uint16_t* W;
  const int32_t* ids;
  float* z;
  float4* stats;            // [n, tiles]
  float* moved;             // [n, tiles]
  uint16_t* P;
  int64_t ldp;
  int n, d, V, tiles;
  float to_log2;
};

template <int VT, int RT>
__global__ __launch_bounds__(256) void ll_answers_logits_kernel(const ShortArgs p) {
  constexpr int STEPS = 4;                     // of 32 columns, in flight together
  constexpr float MOST = 60.f;
  __shared__ f32x4 quarter[4][VT][RT][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), m = lane & 15, g = lane >> 4;
  const int tile = blockIdx.x, v0 = tile * 16 * VT, r0 = blockIdx.y * 16 * RT;
  const uint16_t* w_at[VT];
  const uint16_t* a_at[RT];
#pragma unroll
  for (int t = 0; t < VT; ++t) w_at[t] = p.W + (int64_t)min(v0 + 16 * t + m, p.V - 1) * p.d + 8 * g;
#pragma unroll
  for (int j = 0; j < RT; ++j) a_at[j] = p.rows + (int64_t)min(r0 + 16 * j + m, p.n - 1) * p.d + 8 * g;
  f32x4 acc[VT][RT];
#pragma unroll
  for (int t = 0; t < VT; ++t)
#pragma unroll
    for (int j = 0; j < RT; ++j) acc[t][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  const auto take = [&](const bf16x8 (&w)[VT], const bf16x8 (&a)[RT]) {
#pragma unroll
    for (int t = 0; t < VT; ++t)
#pragma unroll
      for (int j = 0; j < RT; ++j) acc[t][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w[t], a[j], acc[t][j], 0, 0, 0);
  };
  const int steps = (p.d + 31) / 32, each = (steps + 3) / 4, end = min((wave + 1) * each, steps), whole = min(end, p.d / 32);
  int s = wave * each;
  for (; s + STEPS <= whole; s += STEPS) {
    bf16x8 w[STEPS][VT], a[STEPS][RT];
#pragma unroll
    for (int u = 0; u < STEPS; ++u) {
#pragma unroll
      for (int t = 0; t < VT; ++t) w[u][t] = *reinterpret_cast<const bf16x8*>(w_at[t] + 32 * (s + u));
#pragma unroll
      for (int j = 0; j < RT; ++j) a[u][j] = *reinterpret_cast<const bf16x8*>(a_at[j] + 32 * (s + u));
    }
#pragma unroll
    for (int u = 0; u < STEPS; ++u) take(w[u], a[u]);
  }
  for (; s < end; ++s) {                       // columns past the row's end: 0 on both sides (0 times an infinity would not do)
    const bool in = 32 * s + 8 * g < p.d;
    bf16x8 w[VT], a[RT];
#pragma unroll
    for (int t = 0; t < VT; ++t) w[t] = in ? *reinterpret_cast<const bf16x8*>(w_at[t] + 32 * s) : bf16x8{};
#pragma unroll
    for (int j = 0; j < RT; ++j) a[j] = in ? *reinterpret_cast<const bf16x8*>(a_at[j] + 32 * s) : bf16x8{};
    take(w, a);
  }
#pragma unroll
  for (int t = 0; t < VT; ++t)
#pragma unroll
    for (int j = 0; j < RT; ++j) quarter[wave][t][j][lane] = acc[t][j];
  __syncthreads();
  if (wave >= RT) return;
  // ids v0 + 16 t + 4 g + i of row r0 + 16 wave + m
  const int row = r0 + 16 * wave + m, last = p.V - 1 - v0 - 4 * g, id = p.ids[min(row, p.n - 1)];
  const int own = (id >= 0 ? id : -1) - v0 - 4 * g;                // (no token: below 0 or past the vocabulary's last, whatever the id)
  float x[VT][4], most = NEG_BIG;
#pragma unroll
  for (int t = 0; t < VT; ++t) {
    const f32x4 z = (quarter[0][t][wave][lane] + quarter[1][t][wave][lane]) + (quarter[2][t][wave][lane] + quarter[3][t][wave][lane]);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[t][i] = z[i];
      most = 16 * t + i <= last ? fmaxf(most, z[i] * p.to_log2) : most;
      if (16 * t + i == own && own <= last && row < p.n) p.z[row] = z[i];
    }
  }
  const auto larger = [](uint32_t a, uint32_t b) { return __float_as_uint(fmaxf(__uint_as_float(a), __uint_as_float(b))); };
  const auto add = [](uint32_t a, uint32_t b) { return __float_as_uint(__uint_as_float(a) + __uint_as_float(b)); };
  most = __uint_as_float(with_lane_xor<32>(with_lane_xor<16>(__float_as_uint(most), larger), larger));      // the row's four lanes
  const float base = fabsf(most) > MOST && most > NEG_BIG ? ceilf(most) : 0.f;     // (NEG_BIG: no id, or no number)
  float sum = 0.f, others = 0.f;
#pragma unroll
  for (int t = 0; t < VT; ++t)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[t][i] = 16 * t + i <= last ? __builtin_amdgcn_exp2f(fmaf(x[t][i], p.to_log2, -base)) : 0.f;
      sum += x[t][i];
      if (16 * t + i == own) x[t][i] = 0.f;
      others += x[t][i];
    }
  sum = __uint_as_float(with_lane_xor<32>(with_lane_xor<16>(__float_as_uint(sum), add), add));
  others = __uint_as_float(with_lane_xor<32>(with_lane_xor<16>(__float_as_uint(others), add), add));
  if (row >= p.n) return;
  if (g == 0) {
    p.stats[(int64_t)row * p.tiles + tile] = make_float4(base, sum, others, 0.f);
    p.moved[(int64_t)row * p.tiles + tile] = base;
  }
  uint16_t* const to = p.P + row * p.ldp + (v0 & ~31) + 8 * g;      // (see place_in_p)
  if constexpr (VT == 1) {
    *reinterpret_cast<uint2*>(to + 4 * ((v0 >> 4) & 1)) = make_uint2(pack_bf16(x[0][0], x[0][1]), pack_bf16(x[0][2], x[0][3]));
  } else {
#pragma unroll
    for (int t = 0; t < VT; t += 2)
      *reinterpret_cast<uint4*>(to + 16 * t) = make_uint4(pack_bf16(x[t][0], x[t][1]), pack_bf16(x[t][2], x[t][3]), pack_bf16(x[t + 1][0], x[t + 1][1]),
                                                         pack_bf16(x[t + 1][2], x[t + 1][3]));
  }
}

// A row a workgroup: its log-probability and its terms (a preference's factor comes later: ll_preference_pairs_kernel).  Tiles of P are brought to
// one base as in ll_distill_rows_kernel.
template <bool POLICY>
__global__ __launch_bounds__(256) void ll_answers_rows_kernel(const AnswerArgs p) {
  __shared__ float shared_base;
  __shared__ int shared_moved;
  const int64_t row = blockIdx.x;
  const int lane = threadIdx.x & 63;
  if (threadIdx.x < 64) {
    const RowStats r = join_stats<true>(p.stride == 1 ? p.stats + row * p.parts : p.stats + row, p.parts, lane, p.stride);
    const int id = p.ids[row];
    const bool valid = id >= 0 && id < p.V;
    const double logp = p.P != nullptr ? log_p(p.z[row], p.to_log2, r) : log2_p(p.z[row], p.to_log2, r) * LN2_64;
    const float ref = p.ref != nullptr ? p.ref[row] : 0.f;
    bool other = false;
    if (p.P != nullptr)
      for (int i = lane; i < p.parts; i += 64) other |= p.stats[row * p.parts + i].x != ref;
    other = __builtin_amdgcn_ballot_w64(other) != 0;
    const float base = other ? rintf(r.lse2) : ref;
    PolicyTerm t = {0.f, 0.f};
    if (POLICY && valid) t = policy_term(p.policy, row, (float)logp);
    const bool live = valid && (!POLICY || t.c != 0.f);
    if (lane == 0) {
      p.logp[row] = valid ? (float)logp : NAN;
      if (POLICY) p.policy.loss[row] = t.loss;
      if (p.terms != nullptr) {
        const float unit = -p.inv_t * __builtin_amdgcn_exp2f(base - r.lse2);
        const float own = -r.t * __builtin_amdgcn_exp2f(r.ref - base);
        p.terms[row] = {(float)(logp - (double)(float)logp), unit, own, POLICY && live ? unit * t.c : 0.f};
      }
      shared_moved = live && other;
      shared_base = base;
    }
  }
  if (p.P == nullptr) return;
  __syncthreads();
  if (shared_moved) tiles_to_base(p.P + row * p.ldp, p.ldp, p.moved + row * p.tiles, shared_base, p.width);
}

struct PairArgs {
  const int32_t* ids;
  const int32_t* offsets;   // [2 pairs + 1]
  const float* logp;
  const float* ref_logp;    // or nullptr: 0
  const float* weight;      // or nullptr: 1
  int64_t N, pairs;
  int V, form, mean;
  float beta, smoothing;
  float* loss;
  float* score;             // [pairs, 2]
  AnswerTerms* terms;       // or nullptr: no gradient
};

// Rows of a sequence: [begin, end), brought into [0, N) whatever the offsets say.
struct Sequence {
  int64_t begin, end;
};
__device__ __forceinline__ Sequence sequence_of(const PairArgs& p, int64_t i) {
  const int64_t b = p.offsets[i], e = p.offsets[i + 1];
  Sequence s;
  s.begin = b < 0 ? 0 : b > p.N ? p.N : b;
  s.end = e < s.begin ? s.begin : e > p.N ? p.N : e;
  return s;
}

// A pair's loss and d loss / d h from its scores.
struct PairTerm {
  float loss, slope;
};
__device__ __forceinline__ PairTerm pair_term(const PairArgs& p, const double (&score)[2]) {
  const float h = (float)((double)p.beta * (score[0] - score[1]));
  PairTerm t;
  if (p.form == LL_PREFERENCE_LOGISTIC) {
    const float e = expf(-fabsf(h)), soft = log1pf(e);
    const float to = 1.f / (1.f + e), from = e / (1.f + e);        // sigmoids of |h| and of -|h|
    const float up = h > 0.f ? to : from, down = h > 0.f ? from : to;
    t.loss = (1.f - p.smoothing) * (soft + fmaxf(-h, 0.f));
    if (p.smoothing != 0.f) t.loss = fmaf(p.smoothing, soft + fmaxf(h, 0.f), t.loss);       // (0 times an infinite h is no 0)
    t.slope = p.smoothing * up - (1.f - p.smoothing) * down;
    if (h != h) t.loss = t.slope = h;
  } else if (p.form == LL_PREFERENCE_HINGE) {
    t.loss = h < 1.f ? 1.f - h : h > 1.f ? 0.f : h - h;            // (h - h: 0, or NaN of NaN)
    t.slope = h < 1.f ? -1.f : h > 1.f ? 0.f : h - h;
  } else {
    const float off = (float)((score[0] - score[1]) - 0.5 / (double)p.beta);
    t.loss = off * off;
    t.slope = 2.f * off / p.beta;
  }
  return t;
}
// What the loss gains by the log-probability of a row of the pair's first (side 0) or second sequence.
__device__ __forceinline__ float pair_c(const PairArgs& p, int64_t pair, float slope, double length, int side) {
  const float w = p.weight != nullptr ? p.weight[pair] : 1.f;
  return w == 0.f ? 0.f : w * slope * p.beta / (side == 0 ? (float)length : -(float)length);
}

__device__ __forceinline__ double group_total(double x, double* red) {
  for (int off = 32; off > 0; off >>= 1) x += __shfl_xor(x, off);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = x;
  __syncthreads();
  const double sum = (red[0] + red[1]) + (red[2] + red[3]);
  __syncthreads();                             // (`red` is free again)
  return sum;
}

// A pair a workgroup: the two answers' scores, summed in 64 bits (a long answer's log-ratios cancel) in one order, the loss, and every
// row's c.  Offsets that are out of order or out of range are brought into it: no row outside [0, N) is touched.
__global__ __launch_bounds__(256) void ll_preference_pairs_kernel(const PairArgs p) {
  __shared__ double red[4];
  for (int64_t pair = blockIdx.x; pair < p.pairs; pair += gridDim.x) {
    Sequence rows[2];
    double score[2], length[2];
#pragma unroll
    for (int side = 0; side < 2; ++side) {
      rows[side] = sequence_of(p, 2 * pair + side);
      double sum = 0., count = 0.;
      for (int64_t r = rows[side].begin + (int)threadIdx.x; r < rows[side].end; r += 256) {
        if (p.ids[r] < 0 || p.ids[r] >= p.V) continue;
        sum += (double)p.logp[r] + (p.terms != nullptr ? (double)p.terms[r].rest : 0.) - (p.ref_logp != nullptr ? (double)p.ref_logp[r] : 0.);
        count += 1.;
      }
      sum = group_total(sum, red);
      count = group_total(count, red);
      length[side] = p.mean && count > 1. ? count : 1.;
      score[side] = sum / length[side];
    }
    const PairTerm t = pair_term(p, score);
    if (threadIdx.x == 0) {
      p.loss[pair] = t.loss;
      p.score[2 * pair] = (float)score[0];
      p.score[2 * pair + 1] = (float)score[1];
    }
    if (p.terms == nullptr) continue;
#pragma unroll
    for (int side = 0; side < 2; ++side) {
      const float c = pair_c(p, pair, t.slope, length[side], side);
      for (int64_t r = rows[side].begin + (int)threadIdx.x; r < rows[side].end; r += 256)
        if (p.ids[r] >= 0 && p.ids[r] < p.V) p.terms[r].factor = c != 0.f ? p.terms[r].unit * c : 0.f;
    }
  }
}

// The slices' sums joined, in order, and the own token's part; a row that takes no part gets zeros whatever W holds.
__global__ __launch_bounds__(256) void ll_answers_join_kernel(const float* __restrict__ part, int splits, int rows, int d, const int32_t* __restrict__ ids,
                                                              const uint16_t* __restrict__ W, const AnswerTerms* __restrict__ terms,
                                                              uint16_t* __restrict__ out) {
  const int64_t row = blockIdx.y;
  const int c = (blockIdx.x * 256 + threadIdx.x) * 4;
  if (c >= d) return;
  const AnswerTerms t = terms[row];
  float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
  if (t.factor != 0.f) {                       // (so the row has a token)
    const uint2 w = *reinterpret_cast<const uint2*>(W + (int64_t)ids[row] * d + c);
#pragma unroll 8
    for (int q = 0; q < splits; ++q) {
      const float4 x = *reinterpret_cast<const float4*>(part + ((int64_t)q * rows + row) * d + c);
      s.x += x.x;
      s.y += x.y;
      s.z += x.z;
      s.w += x.w;
    }
    s = make_float4(t.factor * fmaf(t.own, bf16_lo(w.x), s.x), t.factor * fmaf(t.own, bf16_hi(w.x), s.y), t.factor * fmaf(t.own, bf16_lo(w.y), s.z),
                    t.factor * fmaf(t.own, bf16_hi(w.y), s.w));
  }
  *reinterpret_cast<uint2*>(out + row * d + c) = make_uint2(pack_bf16(s.x, s.y), pack_bf16(s.z, s.w));
}

// Few rows: block (64 columns, row) forms the row's terms itself (a preference's from all rows', which are no more than its wavefronts), in
// place of a launch or two of some 5 us each, then joins the parts' sums and the row's token.
constexpr int FEW_MOST = 4;
template <bool POLICY>
__global__ __launch_bounds__(256) void ll_answers_few_join_kernel(const FewJoinArgs p, const AnswerArgs r, const PairArgs q) {
  static_assert(FEW_MOST * 64 == 256, "a wavefront a row");
  __shared__ float scale[FEW_LEARN_STREAMS];
  __shared__ float share[1];
  __shared__ int id_of[1];
  __shared__ double logp[FEW_MOST];
  __shared__ float shared_ref, shared_c;
  const int row = blockIdx.y, rows = gridDim.y, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int of_wave = POLICY ? row : wave;
  FewColumns columns;
  columns.load(p, row);
  if (POLICY ? wave == 0 : wave < rows) {
    const RowStats stats = join_stats<true>(r.stats + of_wave, r.parts, lane, r.stride);
    const int id = r.ids[of_wave];
    if (lane == 0) {
      logp[POLICY ? 0 : wave] = id >= 0 && id < r.V ? log_p(r.z[of_wave], r.to_log2, stats) : (double)NAN;
      if (of_wave == row) {
        shared_ref = stats.lse2;
        shared_c = 0.f;
        share[0] = -stats.t * __builtin_amdgcn_exp2f(stats.ref - stats.lse2);
        id_of[0] = id < r.V ? id : -1;
      }
    }
  }
  __syncthreads();
  const bool valid = id_of[0] >= 0, writes = blockIdx.x == 0;
  if (POLICY) {
    if (threadIdx.x == 0) {
      PolicyTerm t = {0.f, 0.f};
      if (valid) t = policy_term(r.policy, row, (float)logp[0]);
      shared_c = t.c;
      if (writes) {
        r.logp[row] = (float)logp[0];
        r.policy.loss[row] = t.loss;
      }
    }
  } else {
    if (threadIdx.x == 0 && writes) r.logp[row] = (float)logp[row];
    for (int64_t pair = threadIdx.x; pair < q.pairs; pair += 256) {
      Sequence of[2];
      double score[2], length[2];
#pragma unroll
      for (int side = 0; side < 2; ++side) {
        of[side] = sequence_of(q, 2 * pair + side);
        double sum = 0., count = 0.;
        for (int64_t i = of[side].begin; i < of[side].end; ++i) {
          if (q.ids[i] < 0 || q.ids[i] >= q.V) continue;
          sum += logp[i] - (q.ref_logp != nullptr ? (double)q.ref_logp[i] : 0.);
          count += 1.;
        }
        length[side] = q.mean && count > 1. ? count : 1.;
        score[side] = sum / length[side];
      }
      const PairTerm t = pair_term(q, score);
      if (writes && row == 0) {
        q.loss[pair] = t.loss;
        q.score[2 * pair] = (float)score[0];
        q.score[2 * pair + 1] = (float)score[1];
      }
#pragma unroll
      for (int side = 0; side < 2; ++side)
        if (valid && row >= of[side].begin && row < of[side].end) shared_c = pair_c(q, pair, t.slope, length[side], side);
    }
  }
  for (int i = threadIdx.x; i < p.parts; i += 256) {
    const float4 part = p.f.stats[(int64_t)i * p.stride + row];
    scale[i] = part.y == 0.f ? 0.f : __builtin_amdgcn_exp2f(part.x - shared_ref);
  }
  __syncthreads();
  columns.join(p, row, shared_c != 0.f ? -r.inv_t * shared_c : 0.f, scale, share, id_of);
}

// ---------------------------------------------------------------------------------------
// Host
// ---------------------------------------------------------------------------------------
// What distillation from one token has, every row's terms, and where pairs take more rows than a pass every pass's sums.
struct AnswerPlan {
  LearnPlan l;
  bool keep;                // the sums of all passes are joined behind the last
  int id_tiles, row_tiles;  // of 16, a workgroup of ll_answers_logits_kernel; id_tiles 0: the direct-to-LDS kernel
  int parts;                // of a row's statistics
  size_t stats, moved, terms, total;
};

// Whether ll_answers_logits_kernel is the faster one, by the tiles of 256 ids that the direct-to-LDS kernel would have.  Whole calls, us, through that
// kernel | this one: d = 4096, V = 4000 (16 tiles), 16 rows 48 | 27, 64 53 | 42, 200 102 | 64, 400 110 | 97, 800 105 | 157; V = 8000 (32), 16 rows 53 | 36, 64
// 59 | 51, 200 109 | 96, 400 119 | 162; V = 16 000 (63), 16 rows 83 | 61, 64 93 | 88, 100 101 | 100, 200 126 | 172; V = 32 000 (125), 16 rows 114 | 111, 64
// 125 | 129; V = 50 257 (197), 16 rows 164 | 186; d = 8192, V = 4000, 16 rows 80 | 39, 400 180 | 160; d = 512, V = 4000, 16 rows 27 | 23, 400 47 | 39, 800
// 46 | 46.  (It reads the rows again for every 64 ids, which is what bounds it with many of both.)
bool few_ids(int rows, int tiles) { return tiles <= 100 && rows * tiles <= 6400; }

AnswerPlan answer_plan(const ll_shape* s, bool pairs, Needs needs) {
  AnswerPlan a = {};
  a.l = plan_for(s, 1, needs, 1);
  const int64_t N = s->N > 0 ? s->N : 1, passes = (N + a.l.pass_rows - 1) / a.l.pass_rows;
  a.keep = pairs && needs == BACKWARD && passes > 1;
  if (a.keep) a.l = plan_for(s, 1, needs, passes);
  a.parts = a.l.splits;
  a.stats = a.l.stats;
  a.moved = a.l.moved;
  a.total = a.l.total;
  const auto take = [&](size_t bytes) {
    const size_t at = a.total;
    a.total = align_up(a.total + bytes, 256);
    return at;
  };
  // (the losses alone have ll_logp's workspace, and its kernel)
  if (needs == BACKWARD && !a.l.few && few_ids(a.l.pass_rows, a.l.tiles)) {
    const int blocks = (a.l.pass_rows + 63) / 64, ids = (int)a.l.ldp / 16;
    a.row_tiles = ((a.l.pass_rows + blocks - 1) / blocks + 15) / 16;
    a.id_tiles = ids / 4 * blocks >= NUM_CU ? 4 : ids / 2 * blocks >= NUM_CU ? 2 : 1;
    a.parts = ids / a.id_tiles;
    a.stats = take((size_t)a.l.pass_rows * a.parts * sizeof(float4));
    a.moved = take((size_t)a.l.pass_rows * a.parts * sizeof(float));
  }
  if (needs == BACKWARD) a.terms = take((size_t)N * sizeof(AnswerTerms));
  return a;
}

using ShortKernel = void (*)(const ShortArgs);
ShortKernel short_kernel(int id_tiles, int row_tiles) {
  return with_row_tiles(row_tiles, [&](auto rt) -> ShortKernel {
    return id_tiles == 4 ? ll_answers_logits_kernel<4, rt()> : id_tiles == 2 ? ll_answers_logits_kernel<2, rt()> : ll_answers_logits_kernel<1, rt()>;
  });
}

// The first product of a pass and its rows' terms; POLICY: and losses.  Of few rows with a gradient, all there is.
template <bool POLICY>
int answer_rows(const Pass& p, const AnswerPlan& a, void* ws, const int32_t* ids, float temperature, float* logp, AnswerTerms* terms,
                const PolicyArgs& policy, const PairArgs& pairs, void* out) {
  const LearnPlan& l = a.l;
  AnswerArgs r = {};
  r.ids = ids;
  r.z = at<float>(ws, l.z);
  r.stats = at<float4>(ws, l.stats);
  r.V = p.shape->V;
  r.to_log2 = p.to_log2;
  r.inv_t = 1.f / temperature;
  r.logp = logp;
  r.terms = terms;
  r.policy = policy;
  if (l.few) {
    FewJoinArgs j = {};
    LL_TRY(terms != nullptr ? p.few<OTHERS>(ids, j.f) : p.few<STATS>(ids, j.f));
    j.parts = r.parts = l.few_parts;
    j.stride = r.stride = l.few_rows;
    j.out = (uint16_t*)out;
    if (terms != nullptr) {
      hipLaunchKernelGGL(ll_answers_few_join_kernel<POLICY>, dim3((p.shape->d + 63) / 64, p.n), dim3(256), 0, p.stream, j, r, pairs);
      LL_HIP_CHECK(hipGetLastError());
      return LL_OK;
    }
  } else {
    r.stats = at<float4>(ws, a.stats);
    r.parts = a.parts;
    r.stride = 1;
    if (terms != nullptr) {
      r.P = at<uint16_t>(ws, l.P);
      r.ldp = l.ldp;
      r.moved = at<float>(ws, a.moved);
      r.tiles = a.id_tiles != 0 ? a.parts : l.tiles;
      r.width = a.id_tiles != 0 ? 16 * a.id_tiles : BM;
    }
    if (a.id_tiles != 0) {
      const ShortArgs q = {p.rows, p.W, ids, at<float>(ws, l.z), at<float4>(ws, a.stats), at<float>(ws, a.moved), r.P, l.ldp, p.n, p.shape->d, p.shape->V,
                           a.parts, p.to_log2};
      hipLaunchKernelGGL(short_kernel(a.id_tiles, a.row_tiles), dim3(a.parts, (p.n + 16 * a.row_tiles - 1) / (16 * a.row_tiles)), dim3(256), 0, p.stream, q);
      LL_HIP_CHECK(hipGetLastError());
    } else {
      r.ref = at<float>(ws, l.ref);
      hipLaunchKernelGGL(ll_answers_tokens_kernel, dim3(p.n), dim3(256), 0, p.stream, p.list(ids), at<float>(ws, l.z), at<float>(ws, l.ref), p.panel(), l.lda);
      LL_HIP_CHECK(hipGetLastError());
      LL_TRY(terms != nullptr ? p.logits<OTHERS>(ids) : p.logits<STATS>());
    }
  }
  hipLaunchKernelGGL(ll_answers_rows_kernel<POLICY>, dim3(p.n), dim3(r.P != nullptr ? 256 : 64), 0, p.stream, r);
  LL_HIP_CHECK(hipGetLastError());
  return LL_OK;
}

// The gradient of a pass from its sums.
int answer_join(const Pass& p, const AnswerPlan& a, const float* sums, const int32_t* ids, const AnswerTerms* terms, uint16_t* out) {
  hipLaunchKernelGGL(ll_answers_join_kernel, dim3((p.shape->d + 1023) / 1024, p.n), dim3(256), 0, p.stream, sums, a.l.back_splits, p.n, p.shape->d, ids,
                     p.W, terms, out);
  LL_HIP_CHECK(hipGetLastError());
  return LL_OK;
}

constexpr int MOST_PAIRS = 1 << 16;   // workgroups that take pairs in turn

bool finite(float x) { return x - x == 0.f; }

}  // namespace

extern "C" {

size_t ll_policy_workspace_bytes(const ll_shape* shape) { return valid(shape, 1) ? answer_plan(shape, false, BACKWARD).total : 0; }

int ll_policy(const ll_shape* shape, void* workspace, size_t workspace_bytes, const void* rows, const void* W_U, float temperature,
              const int32_t* ids, const float* advantage, const float* old_logp, const float* ref_logp, const float* weight, float clip_low,
              float clip_high, float kl, float* out_loss, float* out_logp, void* out_grad, void* stream) {
  if (!valid(shape, 1)) return LL_EINVAL;
  if (!(clip_low >= 0.f && clip_low <= 1.f) || !(clip_high >= 0.f) || !(kl >= 0.f) || !finite(kl) || (kl != 0.f && ref_logp == nullptr))
    return LL_EINVAL;
  if (shape->N == 0) return LL_OK;
  if (advantage == nullptr || out_loss == nullptr || out_logp == nullptr) return LL_EINVAL;
  if (misaligned(advantage, 4) || misaligned(old_logp, 4) || misaligned(ref_logp, 4) || misaligned(weight, 4) || misaligned(out_loss, 4) ||
      misaligned(out_logp, 4) || misaligned(out_grad, 16))
    return LL_EINVAL;
  const bool grad = out_grad != nullptr;
  const AnswerPlan a = answer_plan(shape, false, grad ? BACKWARD : FORWARD);
  LL_TRY(check(shape, workspace, workspace_bytes, a.total, rows, W_U, temperature, ids));
  return for_passes(shape, a.l, workspace, rows, W_U, temperature, 1, stream, [&](const Pass& p, int64_t r0) -> int {
    const auto from = [&](const float* x) { return x != nullptr ? x + r0 : nullptr; };
    const PolicyArgs policy = {advantage + r0, from(old_logp), kl != 0.f ? from(ref_logp) : nullptr, from(weight), out_loss + r0, clip_low, clip_high, kl};
    AnswerTerms* const terms = grad ? at<AnswerTerms>(workspace, a.terms) + r0 : nullptr;
    LL_TRY(answer_rows<true>(p, a, workspace, ids + r0, temperature, out_logp + r0, terms, policy, PairArgs{}, out_grad));
    if (!grad || a.l.few) return LL_OK;
    float* const sums = at<float>(workspace, a.l.part);
    LL_TRY(p.back(nullptr, sums));
    return answer_join(p, a, sums, ids + r0, terms, (uint16_t*)out_grad + r0 * shape->d);
  });
}

size_t ll_preference_workspace_bytes(const ll_shape* shape, int32_t n_pairs) {
  return valid(shape, 1) && n_pairs >= 0 ? answer_plan(shape, true, BACKWARD).total : 0;
}

int ll_preference(const ll_shape* shape, void* workspace, size_t workspace_bytes, const void* rows, const void* W_U, float temperature,
                  const int32_t* ids, const int32_t* offsets, int32_t n_pairs, const float* ref_logp, const float* weight, int form, int mean,
                  float beta, float smoothing, float* out_loss, float* out_score, float* out_logp, void* out_grad, void* stream) {
  if (!valid(shape, 1) || n_pairs < 0) return LL_EINVAL;
  if (form != LL_PREFERENCE_LOGISTIC && form != LL_PREFERENCE_HINGE && form != LL_PREFERENCE_SQUARE) return LL_EINVAL;
  if ((mean != 0 && mean != 1) || !(beta > 0.f) || !finite(beta) || !(smoothing >= 0.f && smoothing <= 0.5f)) return LL_EINVAL;
  if (form != LL_PREFERENCE_LOGISTIC && smoothing != 0.f) return LL_EINVAL;
  if (n_pairs > 0 && (offsets == nullptr || out_loss == nullptr || out_score == nullptr)) return LL_EINVAL;
  if (misaligned(offsets, 4) || misaligned(ref_logp, 4) || misaligned(weight, 4) || misaligned(out_loss, 4) || misaligned(out_score, 4) ||
      misaligned(out_logp, 4) || misaligned(out_grad, 16))
    return LL_EINVAL;
  const bool grad = out_grad != nullptr;
  const AnswerPlan a = answer_plan(shape, true, grad ? BACKWARD : FORWARD);
  if (shape->N > 0) {
    if (out_logp == nullptr) return LL_EINVAL;
    LL_TRY(check(shape, workspace, workspace_bytes, a.total, rows, W_U, temperature, ids));
  }
  AnswerTerms* const terms = grad && shape->N > 0 ? at<AnswerTerms>(workspace, a.terms) : nullptr;
  const PairArgs q = {ids, offsets, out_logp, ref_logp, weight, shape->N, n_pairs, shape->V, form, mean, beta, smoothing, out_loss, out_score, terms};
  const auto pairs = [&]() -> int {
    if (n_pairs == 0) return LL_OK;
    hipLaunchKernelGGL(ll_preference_pairs_kernel, dim3(n_pairs < MOST_PAIRS ? n_pairs : MOST_PAIRS), dim3(256), 0, (hipStream_t)stream, q);
    LL_HIP_CHECK(hipGetLastError());
    return LL_OK;
  };
  const auto sums_of = [&](int64_t r0) { return at<float>(workspace, a.l.part) + (a.keep ? r0 * a.l.back_splits * shape->d : 0); };
  const bool between = grad && shape->N > 0 && !a.keep;      // one pass: the pairs come between the products
  LL_TRY(for_passes(shape, a.l, workspace, rows, W_U, temperature, 1, stream, [&](const Pass& p, int64_t r0) -> int {
    LL_TRY(answer_rows<false>(p, a, workspace, ids + r0, temperature, out_logp + r0, grad ? terms + r0 : nullptr, PolicyArgs{}, q, out_grad));
    if (!grad || a.l.few) return LL_OK;
    if (!a.keep) LL_TRY(pairs());
    LL_TRY(p.back(nullptr, sums_of(r0)));
    return a.keep ? LL_OK : answer_join(p, a, sums_of(r0), ids, terms, (uint16_t*)out_grad);
  }));
  if (between) return LL_OK;
  LL_TRY(pairs());
  if (!a.keep) return LL_OK;
  return for_passes(shape, a.l, workspace, rows, W_U, temperature, 1, stream,
                    [&](const Pass& p, int64_t r0) -> int { return answer_join(p, a, sums_of(r0), ids + r0, terms + r0, (uint16_t*)out_grad + r0 * shape->d); });
}

}  // extern "C"
