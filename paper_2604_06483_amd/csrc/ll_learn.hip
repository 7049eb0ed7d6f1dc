// What learns through the lens: log-probabilities of listed tokens, distillation from a teacher's top tokens, and the gradient of
// either to the (normalised) rows.
//
//   z = A W^T / T,  p = softmax(z) over the whole vocabulary,  dA = dz W
//
// Forward, the logits stay in MFMA accumulators as in ll_project: the direct-to-LDS kernel (ll_gemm_lds.h) with an epilogue of its
// own.  A gradient needs every logit a second time, as the left factor of a product over the vocabulary.  Forming them again would be a
// third product; instead the first one's epilogue leaves P, e^z relative to a reference, as bf16 behind it (2 bytes a logit, beside 4 d
// flops), whose relative error is that of any bf16 number however small it is, and the second product reads that.
#include "ll_learn_host.h"

namespace {

__global__ __launch_bounds__(256) void ll_learn_pad_kernel(const uint16_t* __restrict__ rows, uint16_t* __restrict__ panel, int d, int64_t lda) {
  pad_row(rows, blockIdx.x, d, panel, lda);
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
    tiles_to_base(at, ldp, moved + row * tiles, shared_base);
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

// DISTILL: parts relative to their references, dA = a (sum p W - sum t W_id), and the loss; else sums of dz W, and g / T W_id.
template <bool DISTILL>
__global__ __launch_bounds__(256) void ll_learn_few_join_kernel(const FewJoinArgs p) {
  __shared__ float scale[DISTILL ? FEW_LEARN_STREAMS : 1];
  __shared__ float share[LIST_MAX];
  __shared__ int id_of[LIST_MAX];
  __shared__ float shared_factor, shared_ref;
  const ListArgs& l = p.f.list;
  const int row = blockIdx.y, k = l.k, lane = threadIdx.x & 63;
  const float temperature = p.f.temperature;
  FewColumns columns;
  columns.load(p, row);
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
  columns.join(p, row, shared_factor, DISTILL ? scale : nullptr, share, id_of);
}

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
      return p.few_join(ll_learn_few_join_kernel<false>, j);
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
      return p.few_join(ll_learn_few_join_kernel<true>, j);
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
