// What the kernels that learn through the lens share: their arguments, the layout of P, a row's statistics and its list.
#pragma once

#include "ll_epilogue.h"

#include <math.h>

namespace ll {

constexpr int LIST_MAX = LL_LIST_MAX;      // one lane of a wavefront each
constexpr int PASS_ROWS = 2048;            // rows of a pass: what the workspace holds of P, 0.6 GB at V = 152 000
constexpr int STAGE_K = 64;                // columns (backwards: ids) of a stage of the products
constexpr size_t LEARN_LDS = 160 << 10;    // what they take of LDS
constexpr float LN2 = 0.6931471805599453f;

// Statistics only; and the exponentials; dz where the statistics are known.
enum LearnWhat { STATS, EXPS, GRAD };
constexpr float MASKED = -1024.f;  // an exponent that stands for a column past the vocabulary: 2^l is 0, and l times whatever a gradient is no infinity

struct RowTerms {   // of a row's dz: with l = z log2 e - lse2, dz = 2^l (a + b l); its gradient is `factor` times P's product, zeros where that is 0
  float lse2, a, b, factor;
};

struct LearnArgs : GemmArgs {
  uint16_t* P;          // [rows, ldp] bf16
  float* moved;         // [rows, tiles]: what the exponents of a tile are relative to, in powers of two
  const float* ref;     // [rows]: what they start from
  const RowTerms* terms;   // [rows]
  int64_t ldp;
  float to_log2;        // log2(e) / T
};

struct LearnBackArgs : BackArgs {
  uint16_t* out;           // one slice: the gradient itself, [rows, d] bf16; else nullptr
  const RowTerms* terms;
};

struct ListArgs {
  const uint16_t* rows;
  const uint16_t* W;
  const int32_t* ids;
  int k, d, V;
  float to_log2;
};

constexpr int FEW_LEARN_THREADS = 512;
constexpr int FEW_LEARN_STREAMS = 256;      // most workgroups that read W_U: one a compute unit
constexpr int FEW_LEARN_MAX_D = 16384;

struct FewLearnArgs {
  ListArgs list;            // rows, W, ids, k, d, V, to_log2
  int n, streams;           // rows; workgroups that read W_U (behind them one a row for the listed tokens' logits, but for GRAD)
  int past_caches;          // W's loads go past the caches
  float* z;                 // [n, k]: the listed tokens' logits (not GRAD)
  float4* stats;            // [streams, N]: (ref, S, T)
  float* sums;              // [streams, N, d]
  // GRAD: what the row's dz is made of
  const float* lse;
  const float* entropy;
  const float* g_logp;
  const float* g_entropy;
  float temperature;
};

// Rows of W that a group takes at a time.
constexpr int few_learn_rows(int n, int nc) { return (n == 8 ? 4 : 8) / nc; }

using LearnKernel = void (*)(const LearnArgs);
using LearnBackKernel = void (*)(const LearnBackArgs);
using FewLearnKernel = void (*)(const FewLearnArgs);

// The product with W_U, and backwards (ll_learn_gemm.hip).  ragged: d is not a multiple of 64; past_caches: W's loads go past the caches;
// row_tiles: of 16 rows a wavefront, 1 to 4.
LearnKernel learn_kernel(LearnWhat what, bool ragged, bool past_caches, int row_tiles);
LearnBackKernel learn_back_kernel(bool past_caches, int row_tiles);
// Up to eight rows in one read of W_U (ll_learn_few.hip); nullptr where there is none.
FewLearnKernel few_learn_kernel(LearnWhat what, int rows, int chunks, int groups);

template <class F>
auto with_row_tiles(int rt, F f) {
  using std::integral_constant;
  return rt == 1 ? f(integral_constant<int, 1>{}) : rt == 2 ? f(integral_constant<int, 2>{}) : rt == 3 ? f(integral_constant<int, 3>{}) : f(integral_constant<int, 4>{});
}

}  // namespace ll

namespace {

// Within 64 columns of P the vocabulary is permuted: a lane of the first product holds ids 16 t + 4 g .. + 3 of tiles t, and puts two
// tiles' side by side, 16 bytes at a time; the second product takes W's rows in the same order.
__device__ __forceinline__ int64_t place_in_p(int v) {
  return (v & ~31) + 8 * ((v >> 2) & 3) + 4 * ((v >> 4) & 1) + (v & 3);
}

// Logits of a row's listed tokens (before the temperature), a wavefront an entry at a time; 0 for an id outside the vocabulary.  The
// whole workgroup comes here.  Bound by the gathered rows of W: 1500 x 20 of 16 KB in 103 us, 4.8 TB/s.
__device__ __forceinline__ void list_logits(const ListArgs& p, int row, float* z) {
  const uint16_t* const W = p.W;
  const int32_t* const ids = p.ids + (int64_t)row * p.k;
  const int k = p.k, d = p.d, V = p.V;
  const int lane = threadIdx.x & 63, waves = blockDim.x >> 6;
  const uint4* a = reinterpret_cast<const uint4*>(p.rows + (int64_t)row * d);
  for (int i = threadIdx.x >> 6; i < k; i += waves) {
    const int id = ids[i];
    float s = 0.f;
    if (id >= 0 && id < V) {
      const uint4* w = reinterpret_cast<const uint4*>(W + (int64_t)id * d);
      float part[2] = {0.f, 0.f};
#pragma unroll 4
      for (int c = lane; c < d / 8; c += 64) {
        const uint4 x = a[c], y = w[c];
        const uint32_t xs[4] = {x.x, x.y, x.z, x.w}, ys[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          part[0] = fmaf(bf16_lo(xs[q]), bf16_lo(ys[q]), part[0]);
          part[1] = fmaf(bf16_hi(xs[q]), bf16_hi(ys[q]), part[1]);
        }
      }
      s = wave_sum(part[0] + part[1]);
    }
    if (lane == 0) z[i] = s;
  }
  __syncthreads();
}

// ll_logp_grad: a and b of a row's dz (see RowTerms), by a wavefront; g: the gradient of the lane's entry, 0 where there is none; gh and h
// the entropy's gradient and the entropy.
struct GradTerms {
  float lse2, a, b;
  bool live;              // some gradient is not zero
};
__device__ __forceinline__ GradTerms grad_terms(float g, float lse, float gh, float h, float inv_t) {
  const bool live = __builtin_amdgcn_ballot_w64(g != 0.f) != 0 || gh != 0.f;
  return {lse / LN2, -(wave_sum(g) + (gh != 0.f ? gh * h : 0.f)) * inv_t, -gh * LN2 * inv_t, live};
}

}  // namespace
