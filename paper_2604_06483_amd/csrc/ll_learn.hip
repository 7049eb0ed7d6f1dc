// What learns through the lens: log-probabilities of listed tokens, distillation from a teacher's top tokens, and the gradient of
// either to the (normalised) rows.
//
//   z = A W^T / T,  p = softmax(z) over the whole vocabulary,  dA = dz W
//
// Forward, the logits stay in MFMA accumulators as in ll_project: the direct-to-LDS kernel (ll_gemm_lds.h) with an epilogue of its
// own.  A gradient needs every logit a second time, as the left factor of a product over the vocabulary.  Forming them again would be a
// third product; instead the first one's epilogue leaves P, e^z relative to a reference, as bf16 behind it (2 bytes a logit, beside 4 d
// flops), whose relative error is that of any bf16 number however small it is, and the second product reads that.
#include "ll_learn.h"

namespace {

// A row of a hidden size that is not a multiple of 64, zero padded to one, by a workgroup; no panel: the rows are read where they are.
__device__ __forceinline__ void pad_row(const uint16_t* __restrict__ rows, int64_t row, int d, uint16_t* __restrict__ panel, int64_t lda) {
  if (panel == nullptr) return;
  for (int c = threadIdx.x; c < lda / 8; c += (int)blockDim.x)
    reinterpret_cast<uint4*>(panel + row * lda)[c] =
        8 * c < d ? reinterpret_cast<const uint4*>(rows + row * d)[c] : make_uint4(0, 0, 0, 0);
}
__global__ __launch_bounds__(256) void ll_learn_pad_kernel(const uint16_t* __restrict__ rows, uint16_t* __restrict__ panel, int d, int64_t lda) {
  pad_row(rows, blockIdx.x, d, panel, lda);
}

struct RowStats {
  float lse2, t;   // log2 of the sum of 2^x; sum of p (x - lse2), x = z log2 e: minus the entropy, in powers of two
};
// A row's parts, `stride` apart, joined by a wavefront.
__device__ __forceinline__ RowStats join_stats(const float4* __restrict__ stats, int parts, int lane, int stride = 1) {
  float m = NEG_BIG;
  bool nan = false;
  for (int i = lane; i < parts; i += 64) {
    const float4 q = stats[(int64_t)i * stride];
    m = fmaxf(m, q.y > 0.f ? q.x : NEG_BIG);
    nan |= q.y != q.y;
  }
  m = wave_max(m);
  float s = 0.f, t = 0.f;
  for (int i = lane; i < parts; i += 64) {
    const float4 q = stats[(int64_t)i * stride];
    const float by = q.x - m, e = __builtin_amdgcn_exp2f(by);
    s += q.y > 0.f ? e * q.y : 0.f;
    t += q.y > 0.f ? e * fmaf(by, q.y, q.z) : 0.f;
  }
  s = wave_sum(s);
  t = wave_sum(t);
  const float log_s = __builtin_amdgcn_logf(s);
  RowStats r = {m + log_s, t / s - log_s};
  if (wave_sum(nan ? 1.f : 0.f) > 0.f) r.lse2 = r.t = NAN;
  return r;
}

// A row's listed tokens' logits, by the workgroup, then its statistics from their parts and the log-probabilities, by the first wavefront, one
// lane an entry.
__global__ __launch_bounds__(1024) void ll_logp_finish_kernel(const ListArgs p, const float4* __restrict__ stats, int parts,
                                                              float* __restrict__ logp, float* __restrict__ lse, float* __restrict__ entropy) {
  __shared__ float z[LIST_MAX];
  list_logits(p, blockIdx.x, z);
  const int64_t row = blockIdx.x;
  const int lane = threadIdx.x;
  if (lane >= 64) return;
  const RowStats r = join_stats(stats + row * parts, parts, lane);
  if (lane == 0) {
    lse[row] = r.lse2 * LN2;
    entropy[row] = -r.t * LN2;
  }
  if (lane < p.k) {
    const int64_t e = row * p.k + lane;
    logp[e] = p.ids[e] >= 0 && p.ids[e] < p.V ? fmaf(z[lane], p.to_log2, -r.lse2) * LN2 : NAN;
  }
}

// What the listed entries of a row add to dz: `g` of every lane whose id is this lane's.  Of entries with one id the first has the
// sum; returns whether the lane is one that has.
__device__ __forceinline__ bool gather_same(int id, bool valid, int k, int lane, float& g) {
  float sum = 0.f;
  bool first = valid;
  for (int j = 0; j < k; ++j) {
    const int other = __builtin_amdgcn_readlane(valid ? id : -1, j);
    const float share = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(g), j));
    if (valid && other == id) {
      sum += share;
      if (j < lane) first = false;
    }
  }
  g = sum;
  return first;
}

// Before the first product: the rows padded, the listed tokens' logits, and the largest in powers of two, to the nearest whole one (of a row
// without any: 0).  What P is relative to is always whole: to change it then changes exponents only, and rounds nothing again.
__global__ __launch_bounds__(1024) void ll_distill_lists_kernel(const ListArgs p, float* __restrict__ z_out, float* __restrict__ ref,
                                                                uint16_t* __restrict__ panel, int64_t lda) {
  __shared__ float z[LIST_MAX];
  pad_row(p.rows, blockIdx.x, p.d, panel, lda);
  list_logits(p, blockIdx.x, z);
  const int lane = threadIdx.x;
  if (lane >= 64) return;
  const int64_t row = blockIdx.x, e = row * p.k + lane;
  float most = NEG_BIG;
  if (lane < p.k) {
    z_out[e] = z[lane];
    if (p.ids[e] >= 0 && p.ids[e] < p.V) most = z[lane] * p.to_log2;
  }
  most = wave_max(most);
  if (lane == 0) ref[row] = fabsf(most) < 1e30f ? rintf(most) : 0.f;
}

// A row's teacher, by a wavefront, one lane an entry: t = softmax of the scores / temperature over the entries that there are.
struct Teacher {
  bool valid, some;     // the lane's entry is one; the row has one
  float t, log_t;
};
__device__ __forceinline__ Teacher teacher_of(int id, float score, int V, float temperature) {
  Teacher r;
  r.valid = id >= 0 && id < V && score != -INFINITY;
  r.some = __builtin_amdgcn_ballot_w64(r.valid) != 0;
  const float most = wave_max(r.valid ? score : -INFINITY);
  const float q = r.valid ? (score - most) / temperature : 0.f;
  const float share = r.valid ? expf(q) : 0.f;
  const float total = wave_sum(share);
  r.t = r.some ? share / total : 0.f;
  r.log_t = q - logf(total);
  return r;
}
// logp: the student's log-probability of the lane's entry.  (A share that underflows adds nothing.)
__device__ __forceinline__ float distill_loss(const Teacher& teacher, float logp, float temperature) {
  const float sum = wave_sum(teacher.valid && teacher.t != 0.f ? teacher.t * (teacher.log_t - logp) : 0.f);
  return teacher.some ? temperature * temperature * sum : 0.f;
}

// Teacher, loss, and what the gradient is made of: a row a workgroup, the first wavefront one lane an entry.  With P = 2^(x - base) over the
// whole row, dz = a (p - t) is a 2^(base - lse2) (P - t 2^(lse2 - base)): the listed tokens' entries are put into P, from their fp32 logits
// and rounded once, and the rest is the row's factor of the gradient.  A row whose reference has moved in some tile first has its tiles
// brought to one base here, the whole number next to lse2: by whole powers of two, so that nothing is rounded again.  Of a row without a
// teacher (or of weight 0, as far as the gradient goes) nothing that the row holds matters.
__global__ __launch_bounds__(256) void ll_distill_rows_kernel(const int32_t* __restrict__ ids, const float* __restrict__ z, int k, int V,
                                                              float to_log2, const float4* __restrict__ stats, int parts, int stride,
                                                              const float* __restrict__ scores, const float* __restrict__ weight,
                                                              float temperature, float* __restrict__ loss, RowTerms* __restrict__ terms,
                                                              const float* __restrict__ ref, const float* __restrict__ moved, int tiles,
                                                              uint16_t* __restrict__ P, int64_t ldp) {
  __shared__ float shared_base;
  __shared__ int shared_moved;
  const int64_t row = blockIdx.x;
  const int lane = threadIdx.x & 63;
  const bool first_wave = threadIdx.x < 64;
  int id = -1;
  bool first = false, live = false;
  float l = 0.f, t = 0.f;
  if (first_wave) {
    const RowStats r = join_stats(stride == 1 ? stats + row * parts : stats + row, parts, lane, stride);
    const int64_t e = row * k + lane;
    id = lane < k ? ids[e] : -1;
    const Teacher teacher = teacher_of(id, lane < k ? scores[e] : -INFINITY, V, temperature);
    t = teacher.t;
    l = fmaf(lane < k ? z[e] : 0.f, to_log2, -r.lse2);
    const float sum = distill_loss(teacher, l * LN2, temperature);
    if (lane == 0) loss[row] = sum;
    if (terms != nullptr) {
      const float a = temperature * (weight != nullptr ? weight[row] : 1.f);
      live = teacher.some && a != 0.f;
      first = gather_same(id, teacher.valid, k, lane, t);
      bool other = false;
      for (int i = lane; i < parts; i += 64) other |= stats[row * parts + i].x != ref[row];
      other = __builtin_amdgcn_ballot_w64(other) != 0;
      const float base = other ? rintf(r.lse2) : ref[row];
      if (lane == 0) {
        terms[row] = {r.lse2, 0.f, 0.f, live ? a * __builtin_amdgcn_exp2f(base - r.lse2) : 0.f};
        shared_moved = live && other;
        shared_base = base;
      }
      t *= __builtin_amdgcn_exp2f(r.lse2 - base);
      l += r.lse2 - base;
    }
  }
  if (terms == nullptr) return;
  __syncthreads();
  uint16_t* const at = P + row * ldp;
  if (shared_moved) {
    for (int64_t c = 8 * (int)threadIdx.x; c < ldp; c += 8 * 256) {
      const uint4 q = *reinterpret_cast<const uint4*>(at + c);
      const float by = __builtin_amdgcn_exp2f(moved[row * tiles + c / BM] - shared_base);
      *reinterpret_cast<uint4*>(at + c) = make_uint4(pack_bf16(bf16_lo(q.x) * by, bf16_hi(q.x) * by), pack_bf16(bf16_lo(q.y) * by, bf16_hi(q.y) * by),
                                                     pack_bf16(bf16_lo(q.z) * by, bf16_hi(q.z) * by), pack_bf16(bf16_lo(q.w) * by, bf16_hi(q.w) * by));
    }
    __syncthreads();
  }
  if (first_wave && live && first) at[place_in_p(id)] = (uint16_t)pack_bf16(__builtin_amdgcn_exp2f(l) - t, 0.f);
}

// ll_logp_grad, before the first product: the rows padded, what a row's dz is made of, -p (G + gH (log p + H)) / T and g / T for a listed token,
// and the listed tokens' whole dz.  Those are added up here, in fp32, and rounded once: of a likely token the two parts cancel, and the rounding
// of p alone would be large beside their sum.
__global__ __launch_bounds__(1024) void ll_logp_terms_kernel(const ListArgs p, const float* __restrict__ lse, const float* __restrict__ entropy,
                                                             const float* __restrict__ g_logp, const float* __restrict__ g_entropy,
                                                             float temperature, RowTerms* __restrict__ terms, float2* __restrict__ list,
                                                             uint16_t* __restrict__ panel, int64_t lda) {
  __shared__ float z[LIST_MAX];
  pad_row(p.rows, blockIdx.x, p.d, panel, lda);
  list_logits(p, blockIdx.x, z);
  const int row = blockIdx.x, lane = threadIdx.x, k = p.k;
  if (lane >= 64) return;
  const int64_t e = (int64_t)row * k + lane;
  const int id = lane < k ? p.ids[e] : -1;
  const bool valid = id >= 0 && id < p.V;
  float g = valid ? g_logp[e] : 0.f;
  const float inv_t = 1.f / temperature;
  const GradTerms r = grad_terms(g, lse[row], g_entropy != nullptr ? g_entropy[row] : 0.f, entropy != nullptr ? entropy[row] : 0.f, inv_t);
  const float l = fmaf(lane < k ? z[lane] : 0.f, p.to_log2, -r.lse2);
  const bool first = gather_same(id, valid, k, lane, g);
  if (lane == 0) terms[row] = {r.lse2, r.a, r.b, r.live ? 1.f : 0.f};
  if (lane < k) list[e] = make_float2(fmaf(g, inv_t, __builtin_amdgcn_exp2f(l) * fmaf(r.b, l, r.a)), __int_as_float(r.live && first ? id : -1));
}
// And behind it: the listed tokens' dz to their places.
__global__ __launch_bounds__(256) void ll_learn_put_list_kernel(const float2* __restrict__ list, int64_t entries, int k, uint16_t* __restrict__ P,
                                                                int64_t ldp) {
  const int64_t e = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (e >= entries) return;
  const float2 entry = list[e];
  const int id = __float_as_int(entry.y);
  if (id >= 0) P[e / k * ldp + place_in_p(id)] = (uint16_t)pack_bf16(entry.x, 0.f);
}

// The slices joined, in order; a row that takes no part gets zeros whatever W holds.  (Eight slices' loads in flight at a time.)
__global__ __launch_bounds__(256) void ll_learn_join_kernel(const float* __restrict__ part, int splits, int rows, int d,
                                                            const RowTerms* __restrict__ terms, uint16_t* __restrict__ out) {
  const int64_t row = blockIdx.y;
  const int c = (blockIdx.x * 256 + threadIdx.x) * 4;
  if (c >= d) return;
  const float f = terms[row].factor;
  float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
  if (f != 0.f) {
#pragma unroll 8
    for (int q = 0; q < splits; ++q) {
      const float4 x = *reinterpret_cast<const float4*>(part + ((int64_t)q * rows + row) * d + c);
      s.x += x.x;
      s.y += x.y;
      s.z += x.z;
      s.w += x.w;
    }
    s = make_float4(f * s.x, f * s.y, f * s.z, f * s.w);
  }
  *reinterpret_cast<uint2*>(out + row * d + c) = make_uint2(pack_bf16(s.x, s.y), pack_bf16(s.z, s.w));
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
template <bool DISTILL>
__global__ __launch_bounds__(256) void ll_learn_few_join_kernel(const FewJoinArgs p) {
  __shared__ float scale[DISTILL ? FEW_LEARN_STREAMS : 1];
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
      scale[i] = q.y == 0.f ? 0.f : __builtin_amdgcn_exp2f(q.x - shared_ref);
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

// ---------------------------------------------------------------------------------------
// Host
// ---------------------------------------------------------------------------------------
constexpr int64_t INFINITY_CACHE_BYTES = (int64_t)256 << 20;
constexpr int LEARN_MAX_D = 65536, LEARN_MAX_V = 1 << 22;   // (a lane's offsets within 256 rows of P, or of W, fit 32 bits)

bool valid(const ll_shape* s, int k) {
  return s != nullptr && s->N >= 0 && s->N <= INT32_MAX && s->d > 0 && s->d % 8 == 0 && s->d <= LEARN_MAX_D && s->V > 0 &&
         s->V <= LEARN_MAX_V && k >= 1 && k <= LL_LIST_MAX;
}

enum Needs { FORWARD, BACKWARD };

struct LearnPlan {
  bool few;                            // up to eight rows: one read of W (ll_learn_few.hip)
  int few_rows, few_parts;
  int pass_rows, tiles, splits, row_tiles, block_rows, row_blocks;   // row_tiles: of 16 rows a wavefront
  int col_blocks, back_splits;
  int64_t lda, ldp;
  size_t stats, z, ref, panel, terms, list, moved, P, part, total;
};

// Tiles of 16 rows a wavefront (64 rows a workgroup each): the fewest that hold all rows, else what costs least.  A row block costs 0.47,
// 0.6, 0.79 and 1 of one of 256 rows (1500 rows in 24, 12, 8 and 6: d = 4096, V = 128256, ll_logp 2057, 1320, 1168, 1098 us).  Whole
// calls, us, with 1 | 2 | 3 | 4, ll_logp and ll_distill: d = 2560, V = 151936, 37 rows 161 | 181 | 202 | 228 and 325 | 344 | 367 | 400, 111 rows
// 203 | 175 | 185 | 198 and 454 | 368 | 374 | 393, 192 rows 256 | 223 | 193 | 201 and 565 | 490 | 414 | 427, 348 rows 453 | 301 | 270 | 301 and
// 967 | 682 | 586 | 661, 500 rows 567 | 406 | 355 | 313 and 1225 | 888 | 777 | 688; d = 1608, V = 50257, 777 rows 228 | 164 | 143 | 162 and 513 | 350
// | 328 | 343; d = 8192, V = 128256, 37 rows 427 | 428 | 411 | 456 and 776 | 772 | 759 | 868, 777 rows 2204 | 1513 | 1446 | 1428 and 4545 |
// 3247 | 2990 | 2900.  (The rule takes no account of d: at 8192 it gives away 4 and 2 % of 37 rows' calls and 1 and 3 % of 777's.)
constexpr double BLOCK_COST[4] = {0.47, 0.6, 0.79, 1.0};
int row_tiles(int rows) {
  if (rows <= BN) return (rows + 63) / 64;
  int best = 4;
  double least = 1e30;
  for (int rt = 4; rt >= 1; --rt) {
    const double c = (rows + 64 * rt - 1) / (64 * rt) * BLOCK_COST[rt - 1];
    if (c < least) {
      least = c;
      best = rt;
    }
  }
  return best;
}

// Calls of so few rows that one read of W does (rows 0: not so): rows as the kernel has them, chunks a thread, groups and threads of a
// workgroup, workgroups that read W.
struct FewShape {
  int rows, nc, groups, threads, streams;
};
// A gradient: up to four rows (two above d = 8192, what the registers hold).  Whole calls, us, so | in two products, ll_distill: d = 256, V =
// 150 000, 1 row 24 | 56, 4 rows 39 | 56; 1608, 50257: 35 | 76, 49 | 77; 2560, 151936: 136 | 275, 192 | 279; 4096, 128256: 176 | 372, 186 | 374;
// 8192, 128256: 341 | 760, 363 | 761; 16384, 60000, 1 row 336 | 706.  (Eight rows: 60 | 56, 79 | 79, 360 | 284, 319 | 375 and, in too many registers,
// 851 | 755.  One limit for every d: eight rows gain at 4096 alone.)  Statistics alone: up to eight where a row of W fills the workgroup.  ll_logp, 4 rows and 8: d = 256 23 | 27, 34 | 27; 2560 137 | 145,
// 185 | 147; 4096 176 | 202, 178 | 205; 8192 342 | 436, 346 | 431.
FewShape few_shape(const ll_shape* s, Needs needs) {
  const int n8 = s->d >> 3;
  FewShape f = {};
  if (s->d > FEW_LEARN_MAX_D) return f;
  f.nc = n8 <= 512 ? 1 : n8 <= 1024 ? 2 : 4;
  f.groups = n8 <= 64 ? 8 : n8 <= 128 ? 4 : n8 <= 256 ? 2 : 1;
  f.threads = f.groups > 1 ? FEW_LEARN_THREADS : ((n8 + f.nc - 1) / f.nc + kWave - 1) / kWave * kWave;
  const int most = f.nc == 4 ? 2 : needs == FORWARD && (f.nc == 2 || f.threads == FEW_LEARN_THREADS) && f.groups == 1 ? 8 : 4;
  if (s->N > most) return f;
  f.rows = s->N <= 2 ? (s->N < 2 ? 1 : 2) : s->N <= 4 ? 4 : 8;
  const int step = f.groups * few_learn_rows(f.rows, f.nc), steps = (s->V + step - 1) / step;
  f.streams = NUM_CU - (int)s->N;   // (the listed tokens' logits have a compute unit each at first)
  if (f.streams > steps) f.streams = steps;
  return f;
}

// Slices of the vocabulary for the product backwards: one workgroup a compute unit at a time, so that `tiles` of it take whole rounds,
// of a stage's time each (and three to fill and empty the ring); a slice more is written and read, at some 4 TB/s, by a launch of some 5 us.
int slices(int64_t tiles, int stages, int rows, int d, double stage_us) {
  int best = 1;
  double least = 1e30;
  for (int s = 1; s <= 64 && s <= stages; ++s) {
    const double rounds = (double)((tiles * s + NUM_CU - 1) / NUM_CU);
    const double us = rounds * ((stages + s - 1) / s + 3) * stage_us + (s > 1 ? s * (double)rows * d * 8 / 4e6 + 5 : 0);
    if (us < least) {
      least = us;
      best = s;
    }
  }
  return best;
}

LearnPlan plan_for(const ll_shape* s, int k, Needs needs) {
  LearnPlan l = {};
  const int64_t N = s->N > 0 ? s->N : 1;
  const int64_t passes = (N + PASS_ROWS - 1) / PASS_ROWS, each = (N + passes - 1) / passes;
  l.pass_rows = (int)(passes == 1 ? N : (each + BN - 1) / BN * BN);
  l.tiles = (s->V + BM - 1) / BM;
  l.row_tiles = row_tiles(l.pass_rows);
  l.block_rows = 64 * l.row_tiles;
  l.row_blocks = (l.pass_rows + l.block_rows - 1) / l.block_rows;
  const int most = NUM_CU / l.row_blocks < l.tiles ? NUM_CU / l.row_blocks : l.tiles;
  const int per = (l.tiles + most - 1) / most;
  l.splits = (l.tiles + per - 1) / per;
  l.lda = (s->d + STAGE_K - 1) / STAGE_K * STAGE_K;
  l.ldp = (int64_t)l.tiles * BM;
  l.col_blocks = (s->d + BM - 1) / BM;
  l.back_splits = slices(l.row_blocks * l.col_blocks, (s->V + STAGE_K - 1) / STAGE_K, l.pass_rows, s->d, l.row_blocks == 1 ? 1.5 : 1.5 * BLOCK_COST[l.row_tiles - 1]);
  size_t off = 0;
  auto take = [&](size_t bytes) {
    const size_t at = off;
    off = align_up(off + bytes, 256);
    return at;
  };
  const size_t rows = (size_t)l.pass_rows;
  const FewShape few = few_shape(s, needs);
  l.few = few.rows > 0;
  if (l.few) {
    l.few_rows = few.rows;
    l.few_parts = few.streams;
    l.stats = take((size_t)l.few_parts * few.rows * sizeof(float4));
    l.z = take(rows * k * sizeof(float));
    if (needs == BACKWARD) l.part = take((size_t)l.few_parts * few.rows * s->d * sizeof(float));
    l.total = off;
    return l;
  }
  l.stats = take(rows * l.splits * sizeof(float4));
  l.z = take(rows * k * sizeof(float));
  l.ref = take(rows * sizeof(float));
  l.panel = take(l.lda != s->d ? rows * l.lda * 2 : 0);
  if (needs == BACKWARD) {
    l.terms = take(rows * sizeof(RowTerms));
    l.moved = take(rows * l.tiles * sizeof(float));
    l.P = take(rows * l.ldp * 2);
    l.part = take(l.back_splits > 1 ? rows * l.back_splits * s->d * sizeof(float) : 0);
    l.list = take(rows * k * sizeof(float2));
  }
  l.total = off;
  return l;
}

template <class T>
T* at(void* workspace, size_t offset) {
  return reinterpret_cast<T*>(static_cast<unsigned char*>(workspace) + offset);
}

bool misaligned(const void* p, size_t to) { return ((uintptr_t)p & (to - 1)) != 0; }

int check(const ll_shape* shape, void* workspace, size_t workspace_bytes, size_t need, const void* rows, const void* W_U, float temperature,
          const int32_t* ids) {
  if (rows == nullptr || W_U == nullptr || ids == nullptr || !(temperature > 0.f) || isinf(temperature)) return LL_EINVAL;
  if (!(LOG2E / temperature > 0.f) || isinf(LOG2E / temperature)) return LL_EINVAL;
  if (misaligned(rows, 16) || misaligned(W_U, 16) || misaligned(ids, 4)) return LL_EINVAL;
  if (workspace == nullptr || workspace_bytes < need || misaligned(workspace, 256)) return LL_EWORKSPACE;
  return LL_OK;
}

struct Pass {
  const ll_shape* shape;
  const LearnPlan& l;
  void* ws;
  const uint16_t* rows;
  const uint16_t* W;
  float to_log2;
  int n, k;
  hipStream_t stream;

  int64_t w_bytes() const { return (int64_t)shape->V * shape->d * 2; }
  bool whole_lines() const { return ((uintptr_t)W | (uintptr_t)shape->d * 2) % 128 == 0; }   // (else W's rows share lines, which the caches keep between two loads)
  // The products read W past the caches where it is read once, by one row block, and is more than the Infinity Cache holds.  Whole calls
  // past the caches over through them, ll_logp and ll_distill: d = 2560, V = 151936, 37 rows 0.92 and 0.96, 100 rows 0.95 and 1.01; 4096, 128256:
  // 0.89 and 0.92, 0.90 and 0.95; 8192, 128256: 0.91 and 0.94, 0.89 and 0.96; two row blocks (348 rows) 0.98 to 1.0; 103 MB of W 1.1 and 1.13.
  bool past_caches() const { return l.row_blocks == 1 && whole_lines() && w_bytes() > INFINITY_CACHE_BYTES; }
  ListArgs list(const int32_t* ids) const { return {rows, W, ids, k, shape->d, shape->V, to_log2}; }
  dim3 list_threads() const { return dim3(64 * (k < 16 ? k : 16)); }   // a wavefront an entry

  // Few rows: the one read of W, as it goes into ll_learn_few_join_kernel and its like.
  template <LearnWhat WHAT>
  int few(const int32_t* ids, FewLearnArgs& p) const {
    p.list = list(ids);
    p.n = n;
    p.streams = l.few_parts;
    // (as in ll_project: more of W than stays in the Infinity Cache beside other weights)
    p.past_caches = whole_lines() && w_bytes() > INFINITY_CACHE_BYTES / 3;
    p.z = at<float>(ws, l.z);
    p.stats = at<float4>(ws, l.stats);
    p.sums = at<float>(ws, l.part);
    const int lists = WHAT == GRAD ? 0 : n;
    const FewShape f = few_shape(shape, WHAT == STATS ? FORWARD : BACKWARD);
    hipLaunchKernelGGL(few_learn_kernel(WHAT, f.rows, f.nc, f.groups), dim3(p.streams + lists), dim3(f.threads), 0, stream, p);
    LL_HIP_CHECK(hipGetLastError());
    return LL_OK;
  }
  template <bool DISTILL>
  int few_join(const FewJoinArgs& p) const {
    hipLaunchKernelGGL(ll_learn_few_join_kernel<DISTILL>, dim3((shape->d + 63) / 64, n), dim3(256), 0, stream, p);
    LL_HIP_CHECK(hipGetLastError());
    return LL_OK;
  }

  // where the rows are padded to, by a kernel before the first product
  uint16_t* panel() const { return l.lda != shape->d ? at<uint16_t>(ws, l.panel) : nullptr; }

  template <LearnWhat WHAT>
  int logits() const {
    LearnArgs p = {};
    p.A = panel() != nullptr ? panel() : rows;
    p.W = W;
    p.stats = at<float4>(ws, l.stats);
    p.lda = l.lda;
    p.rows = n;
    p.d = shape->d;
    p.V = shape->V;
    p.splits = l.splits;
    p.tiles = l.tiles;
    p.row_blocks = (n + l.block_rows - 1) / l.block_rows;
    p.last_row = n - 1;
    p.group_rows = group_rows(p.row_blocks, p.splits);
    p.to_log2 = to_log2;
    if (WHAT != STATS) {
      p.P = at<uint16_t>(ws, l.P);
      p.ldp = l.ldp;
      p.moved = at<float>(ws, l.moved);
      p.ref = at<float>(ws, l.ref);
      p.terms = at<RowTerms>(ws, l.terms);
    }
    const LearnKernel kernel = learn_kernel(WHAT, l.lda != shape->d, past_caches(), l.row_tiles);
    const size_t lds = LEARN_LDS;
    if (const int rc = allow_dynamic_lds(reinterpret_cast<const void*>(kernel), lds); rc != LL_OK) return rc;
    const unsigned groups = (unsigned)((p.row_blocks * p.splits + NUM_XCD - 1) / NUM_XCD * NUM_XCD);
    hipLaunchKernelGGL(kernel, dim3(groups), dim3(NTHREADS), lds, stream, p);
    LL_HIP_CHECK(hipGetLastError());
    return LL_OK;
  }

  // P to the gradient of the rows
  int back(uint16_t* out) const {
    LearnBackArgs p = {};
    p.A = at<uint16_t>(ws, l.P);
    p.W = W;
    p.part = at<float>(ws, l.part);
    p.lda = l.ldp;
    p.rows = n;
    p.last_row = n - 1;
    p.d = shape->d;
    p.V = shape->V;
    p.splits = l.back_splits;
    p.row_blocks = (n + l.block_rows - 1) / l.block_rows;
    p.col_blocks = l.col_blocks;
    p.out = p.splits == 1 ? out : nullptr;
    p.terms = at<RowTerms>(ws, l.terms);
    const size_t lds = LEARN_LDS;
    const LearnBackKernel kernel = learn_back_kernel(past_caches(), l.row_tiles);
    if (const int rc = allow_dynamic_lds(reinterpret_cast<const void*>(kernel), lds); rc != LL_OK) return rc;
    const unsigned groups = (unsigned)((p.row_blocks * p.col_blocks * p.splits + NUM_XCD - 1) / NUM_XCD * NUM_XCD);
    hipLaunchKernelGGL(kernel, dim3(groups), dim3(NTHREADS), lds, stream, p);
    LL_HIP_CHECK(hipGetLastError());
    if (p.out != nullptr) return LL_OK;
    hipLaunchKernelGGL(ll_learn_join_kernel, dim3((shape->d + 1023) / 1024, n), dim3(256), 0, stream, p.part, p.splits, n, shape->d,
                       at<RowTerms>(ws, l.terms), out);
    LL_HIP_CHECK(hipGetLastError());
    return LL_OK;
  }
};

template <class F>
int for_passes(const ll_shape* shape, const LearnPlan& l, void* ws, const void* rows, const void* W, float temperature, int k, void* stream, F f) {
  for (int64_t r0 = 0; r0 < shape->N; r0 += l.pass_rows) {
    const int n = (int)(shape->N - r0 < l.pass_rows ? shape->N - r0 : l.pass_rows);
    const Pass pass = {shape, l, ws, (const uint16_t*)rows + r0 * shape->d, (const uint16_t*)W, LOG2E / temperature, n, k, (hipStream_t)stream};
    if (const int rc = f(pass, r0); rc != LL_OK) return rc;
  }
  return LL_OK;
}

#define LL_TRY(expr) \
  if (const int rc__ = (expr); rc__ != LL_OK) return rc__

}  // namespace

extern "C" {

size_t ll_logp_workspace_bytes(const ll_shape* shape, int k) { return valid(shape, k) ? plan_for(shape, k, FORWARD).total : 0; }

int ll_logp(const ll_shape* shape, void* workspace, size_t workspace_bytes, const void* rows, const void* W_U, float temperature, int k,
            const int32_t* ids, float* out_logp, float* out_lse, float* out_entropy, void* stream) {
  if (!valid(shape, k)) return LL_EINVAL;
  if (shape->N == 0) return LL_OK;
  if (out_logp == nullptr || out_lse == nullptr || out_entropy == nullptr) return LL_EINVAL;
  if (misaligned(out_logp, 4) || misaligned(out_lse, 4) || misaligned(out_entropy, 4)) return LL_EINVAL;
  const LearnPlan l = plan_for(shape, k, FORWARD);
  LL_TRY(check(shape, workspace, workspace_bytes, l.total, rows, W_U, temperature, ids));
  return for_passes(shape, l, workspace, rows, W_U, temperature, k, stream, [&](const Pass& p, int64_t r0) -> int {
    if (l.few) {
      FewLearnArgs f = {};
      LL_TRY(p.few<STATS>(ids, f));
      hipLaunchKernelGGL(ll_logp_few_finish_kernel, dim3(p.n), dim3(64), 0, p.stream, f.list, f.z, f.stats, l.few_parts, l.few_rows, out_logp, out_lse,
                         out_entropy);
      LL_HIP_CHECK(hipGetLastError());
      return LL_OK;
    }
    if (p.panel() != nullptr) {
      hipLaunchKernelGGL(ll_learn_pad_kernel, dim3(p.n), dim3(256), 0, p.stream, p.rows, p.panel(), shape->d, l.lda);
      LL_HIP_CHECK(hipGetLastError());
    }
    LL_TRY(p.logits<STATS>());
    hipLaunchKernelGGL(ll_logp_finish_kernel, dim3(p.n), p.list_threads(), 0, p.stream, p.list(ids + r0 * k), at<float4>(workspace, l.stats),
                       l.splits, out_logp + r0 * k, out_lse + r0, out_entropy + r0);
    LL_HIP_CHECK(hipGetLastError());
    return LL_OK;
  });
}

size_t ll_logp_grad_workspace_bytes(const ll_shape* shape, int k) { return valid(shape, k) ? plan_for(shape, k, BACKWARD).total : 0; }

int ll_logp_grad(const ll_shape* shape, void* workspace, size_t workspace_bytes, const void* rows, const void* W_U, float temperature, int k,
                 const int32_t* ids, const float* lse, const float* entropy, const float* g_logp, const float* g_entropy, void* out_grad,
                 void* stream) {
  if (!valid(shape, k)) return LL_EINVAL;
  if (shape->N == 0) return LL_OK;
  if (lse == nullptr || g_logp == nullptr || out_grad == nullptr || (g_entropy != nullptr && entropy == nullptr)) return LL_EINVAL;
  if (misaligned(lse, 4) || misaligned(entropy, 4) || misaligned(g_logp, 4) || misaligned(g_entropy, 4) || misaligned(out_grad, 16)) return LL_EINVAL;
  const LearnPlan l = plan_for(shape, k, BACKWARD);
  LL_TRY(check(shape, workspace, workspace_bytes, l.total, rows, W_U, temperature, ids));
  return for_passes(shape, l, workspace, rows, W_U, temperature, k, stream, [&](const Pass& p, int64_t r0) -> int {
    if (l.few) {
      FewJoinArgs j = {};
      j.f.lse = lse;
      j.f.entropy = entropy;
      j.f.g_logp = g_logp;
      j.f.g_entropy = g_entropy;
      j.f.temperature = temperature;
      LL_TRY(p.few<GRAD>(ids, j.f));
      j.parts = l.few_parts;
      j.stride = l.few_rows;
      j.out = (uint16_t*)out_grad;
      return p.few_join<false>(j);
    }
    hipLaunchKernelGGL(ll_logp_terms_kernel, dim3(p.n), p.list_threads(), 0, p.stream, p.list(ids + r0 * k), lse + r0,
                       entropy != nullptr ? entropy + r0 : nullptr, g_logp + r0 * k, g_entropy != nullptr ? g_entropy + r0 : nullptr, temperature,
                       at<RowTerms>(workspace, l.terms), at<float2>(workspace, l.list), p.panel(), l.lda);
    LL_HIP_CHECK(hipGetLastError());
    LL_TRY(p.logits<GRAD>());
    const int64_t entries = (int64_t)p.n * k;
    hipLaunchKernelGGL(ll_learn_put_list_kernel, dim3((unsigned)((entries + 255) / 256)), dim3(256), 0, p.stream, at<float2>(workspace, l.list),
                       entries, k, at<uint16_t>(workspace, l.P), l.ldp);
    LL_HIP_CHECK(hipGetLastError());
    return p.back((uint16_t*)out_grad + r0 * shape->d);
  });
}

size_t ll_distill_workspace_bytes(const ll_shape* shape, int k) { return ll_logp_grad_workspace_bytes(shape, k); }

int ll_distill(const ll_shape* shape, void* workspace, size_t workspace_bytes, const void* rows, const void* W_U, float temperature, int k,
               const int32_t* teacher_ids, const float* teacher_scores, const float* weight, float* out_loss, void* out_grad, void* stream) {
  if (!valid(shape, k)) return LL_EINVAL;
  if (shape->N == 0) return LL_OK;
  if (teacher_scores == nullptr || out_loss == nullptr) return LL_EINVAL;
  if (misaligned(teacher_scores, 4) || misaligned(weight, 4) || misaligned(out_loss, 4) || misaligned(out_grad, 16)) return LL_EINVAL;
  const LearnPlan l = plan_for(shape, k, out_grad != nullptr ? BACKWARD : FORWARD);
  LL_TRY(check(shape, workspace, workspace_bytes, l.total, rows, W_U, temperature, teacher_ids));
  return for_passes(shape, l, workspace, rows, W_U, temperature, k, stream, [&](const Pass& p, int64_t r0) -> int {
    const bool grad = out_grad != nullptr;
    if (l.few && grad) {
      FewJoinArgs j = {};
      j.f.temperature = temperature;
      LL_TRY(p.few<EXPS>(teacher_ids, j.f));
      j.parts = l.few_parts;
      j.stride = l.few_rows;
      j.scores = teacher_scores;
      j.weight = weight;
      j.loss = out_loss;
      j.out = (uint16_t*)out_grad;
      return p.few_join<true>(j);
    }
    if (l.few) {
      FewLearnArgs f = {};
      LL_TRY(p.few<STATS>(teacher_ids, f));
      hipLaunchKernelGGL(ll_distill_rows_kernel, dim3(p.n), dim3(64), 0, p.stream, teacher_ids, f.z, k, shape->V, p.to_log2, f.stats, l.few_parts,
                         l.few_rows, teacher_scores, weight, temperature, out_loss, nullptr, nullptr, nullptr, 0, nullptr, 0);
      LL_HIP_CHECK(hipGetLastError());
      return LL_OK;
    }
    hipLaunchKernelGGL(ll_distill_lists_kernel, dim3(p.n), p.list_threads(), 0, p.stream, p.list(teacher_ids + r0 * k), at<float>(workspace, l.z),
                       at<float>(workspace, l.ref), p.panel(), l.lda);
    LL_HIP_CHECK(hipGetLastError());
    LL_TRY(grad ? p.logits<EXPS>() : p.logits<STATS>());
    hipLaunchKernelGGL(ll_distill_rows_kernel, dim3(p.n), dim3(grad ? 256 : 64), 0, p.stream, teacher_ids + r0 * k, at<float>(workspace, l.z), k,
                       shape->V, p.to_log2, at<float4>(workspace, l.stats), l.splits, 1, teacher_scores + r0 * k,
                       weight != nullptr ? weight + r0 : nullptr, temperature, out_loss + r0, grad ? at<RowTerms>(workspace, l.terms) : nullptr,
                       at<float>(workspace, l.ref), grad ? at<float>(workspace, l.moved) : nullptr, l.tiles,
                       grad ? at<uint16_t>(workspace, l.P) : nullptr, l.ldp);
    LL_HIP_CHECK(hipGetLastError());
    if (!grad) return LL_OK;
    return p.back((uint16_t*)out_grad + r0 * shape->d);
  });
}

}  // extern "C"
