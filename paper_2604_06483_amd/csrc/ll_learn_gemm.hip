// The products of what learns through the lens, on the direct-to-LDS kernel (ll_gemm_lds.h): rows times W_U, with an epilogue that makes
// statistics, exponentials or the gradient of the logits of it, and backwards.
#include "ll_learn.h"

#include "ll_gemm_lds.h"

namespace {

static_assert(DK == STAGE_K && (size_t)SLOTS * SLOT_BYTES == LEARN_LDS, "as the host takes them");

// STATS: statistics only; EXPS: and the exponentials; GRAD: dz where the statistics are known; OTHERS: as EXPS, with the row's own token left
// out of P and out of the sum, and its exponential beside that: what a gradient needs is p - 1 of that token, and where p is next to 1 a
// difference of sums that are rounded by themselves holds nothing of it (1 - p = 1e-4 at d = 4096: 19 % off).  A row tile has two forms, with and
// without a token of one of its 16 rows in it, and the first looks for it 32 columns at a time.  ll_policy and ll_preference, us, without any of this |
// with | with the first form alone: 1500 x 4096 x 128256 2224 | 2229 | 2247; 6000 x 2560 x 151936 6653 | 6666 | 6739; 348 x 1608 x 50257 161 | 162 | 167.
//
// Exponents are relative to a reference that is no maximum: with fp32's range a sum of 2^(x - ref) does as well for any ref that is
// not far from it, and so does bf16 for the exponentials, so that a tile takes one look at its accumulators and not two.  The reference
// moves, to the tile's maximum, where the lane's sum over a tile leaves `MOST` behind (or has overflowed), and the tile is taken again.
// STATS starts from below everything, so that the first tile sets it, and moves it early, for the sake of T, whose terms are 2^l l.
// EXPS starts from the largest listed logit, one for all splits of a row, and so near the row's maximum that hardly any row ever moves:
// then all of P's row is relative to one number, which the product backwards need not know (see ll_distill_rows_kernel).
template <int WHAT, int RT, bool PAST>
struct LearnEpilogue {
  struct State {   // of the lane's rows, 16 j + lane % 16 of the wavefront's; s and t over the vocabulary that the lane has seen
    float ref[RT], s[RT], t[RT];
    RowTerms terms[WHAT == GRAD ? RT : 1];
    int own[WHAT == OTHERS ? RT : 1];
  };
  static constexpr bool TO_P = WHAT == EXPS || WHAT == OTHERS;
  static constexpr bool RELOAD_FRAGMENTS = WHAT == STATS && RT == 4, OWN_U = false, BACK = false, PAST_CACHES = PAST, HALVES_APART = true;
  static constexpr int ROWS = 64 * RT, ROW_TILES = RT;
  static constexpr float MOST = TO_P ? 0x1p60f : 0x1p16f;
  static __device__ __forceinline__ bool skip(const GemmArgs&) { return false; }
  static __device__ __forceinline__ int row_of(int my_row, int j) { return my_row - (threadIdx.x & 63) + 16 * j + (threadIdx.x & 15); }
  static __device__ __forceinline__ void init(State& st, const GemmArgs& args, int my_row, int) {
    const LearnArgs& p = static_cast<const LearnArgs&>(args);
#pragma unroll
    for (int j = 0; j < RT; ++j) {
      const int row = min(row_of(my_row, j), p.rows - 1);
      st.ref[j] = TO_P ? p.ref[row] : NEG_BIG;
      st.s[j] = st.t[j] = 0.f;
      if (WHAT == GRAD) st.terms[j] = p.terms[row];
      if (WHAT == OTHERS) st.own[j] = (uint32_t)p.target[row] < (uint32_t)p.V ? p.target[row] : -1;
    }
  }
  template <class ACC>
  static __device__ __forceinline__ void tile(const ACC& acc, State& st, int v0, const GemmArgs& args, int my_row) {
    const LearnArgs& p = static_cast<const LearnArgs&>(args);
    asm volatile("s_nop 15\n\ts_nop 15\n\ts_nop 15" ::: "memory");   // the last MFMA's result is in its registers
    if (v0 + BM <= p.V) rows_of_tile<true>(acc, st, v0, p, my_row);
    else rows_of_tile<false>(acc, st, v0, p, my_row);
  }
  // Whether column q of the lane's eight of columns 32 u .. is in the vocabulary.
  static __device__ __forceinline__ bool inside(int u, int q, int last) { return 16 * (2 * u + (q >> 2)) + (q & 3) <= last; }
  // One row tile, eight values at a time: what they add to the sums, and what goes to P.  WHOLE: all columns are in the vocabulary.  MEETS: own is the
  // lane's column of its row's token, or none.
  template <bool WHOLE, bool MEETS, class ACC>
  static __device__ __forceinline__ float2 sums_of_tile(const ACC& acc, const State& st, int j, int last, float c, uint4* to, bool present, int own, float& logit) {
    float s = 0.f, t = 0.f;
    const float ref = WHAT == GRAD ? st.terms[j].lse2 : st.ref[j];
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      float x[8], z[8];
      const float before = s;
#pragma unroll
      for (int q = 0; q < 8; ++q) {
        z[q] = acc_read(acc[2 * u + (q >> 2)][j][q & 3]);
        float l = fmaf(z[q], c, -ref);
        if (!WHOLE) l = inside(u, q, last) ? l : MASKED;
        x[q] = __builtin_amdgcn_exp2f(l);
        if (WHAT == GRAD) x[q] *= fmaf(st.terms[j].b, l, st.terms[j].a);
        else s += x[q];
        if (WHAT == STATS) t = fmaf(x[q], l, t);
      }
      if (MEETS && __builtin_amdgcn_ballot_w64((own >> 5) == u) != 0) {
        s = before;
#pragma unroll
        for (int q = 0; q < 8; ++q) {
          const bool mine = 16 * (2 * u + (q >> 2)) + (q & 3) == own;
          t = mine ? x[q] : t;
          logit = mine ? z[q] : logit;
          x[q] = mine ? 0.f : x[q];
          s += x[q];
        }
      }
      if (WHAT != STATS && present)
        to[4 * u] = make_uint4(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(x[4], x[5]), pack_bf16(x[6], x[7]));
      LL_SCHED_FENCE();
    }
    return make_float2(s, t);
  }
  template <bool WHOLE, class ACC>
  static __device__ __forceinline__ void rows_of_tile(const ACC& acc, State& st, int v0, const LearnArgs& p, int my_row) {
    const int g = (threadIdx.x & 63) >> 4;
    const float c = p.to_log2;
    const int last = p.V - 1 - v0 - 4 * g;   // of the lane's 16 t + i, the last in the vocabulary
#pragma unroll
    for (int j = 0; j < RT; ++j) {
      const int row = row_of(my_row, j);
      const bool present = row < p.rows;
      uint4* const to = reinterpret_cast<uint4*>(p.P + row * p.ldp + v0 + 8 * g);
      int own = -1;
      if (WHAT == OTHERS) {
        own = st.own[j] - v0 - 4 * g;             // (no token: -1, and so below 0)
        if ((own & 15) >= 4) own = -1;            // (another lane's)
      }
      const bool meets = WHAT == OTHERS && __builtin_amdgcn_ballot_w64(own >= 0 && own < BM) != 0;
      float logit = 0.f;
      float2 add;
      if (meets) add = sums_of_tile<WHOLE, WHAT == OTHERS>(acc, st, j, last, c, to, present, own, logit);
      else add = sums_of_tile<WHOLE, false>(acc, st, j, last, c, to, present, own, logit);
      if (WHAT == GRAD) continue;
      const auto large = [&] { return add.x > MOST || (WHAT == OTHERS && add.y > MOST); };
      if (__builtin_amdgcn_ballot_w64(large()) != 0) {
        float m = NEG_BIG;
#pragma unroll
        for (int u = 0; u < 8; ++u) {
#pragma unroll
          for (int q = 0; q < 8; ++q) {
            const float z = acc_read(acc[2 * u + (q >> 2)][j][q & 3]);
            m = WHOLE || inside(u, q, last) ? fmaxf(m, z) : m;
          }
          LL_SCHED_FENCE();
        }
        const auto most = [](uint32_t a, uint32_t b) { return __float_as_uint(fmaxf(__uint_as_float(a), __uint_as_float(b))); };
        const auto any = [](uint32_t a, uint32_t b) { return a | b; };
        // the four lanes of a row together
        m = __uint_as_float(with_lane_xor<32>(with_lane_xor<16>(__float_as_uint(m), most), most)) * c;
        const bool move = with_lane_xor<32>(with_lane_xor<16>(large() ? 1u : 0u, any), any) != 0;
        if (TO_P) m = ceilf(m);   // (whole, as it was)
        const float to_ref = move ? fmaxf(m, st.ref[j]) : st.ref[j], before = st.ref[j] - to_ref, keep = __builtin_amdgcn_exp2f(before);
        st.t[j] = keep * (WHAT == OTHERS ? st.t[j] : fmaf(before, st.s[j], st.t[j]));
        st.s[j] *= keep;
        st.ref[j] = to_ref;
        add = sums_of_tile<WHOLE, WHAT == OTHERS>(acc, st, j, last, c, to, present, own, logit);
      }
      if (WHAT == OTHERS && own >= 0 && own < BM && present) p.z[row] = logit;
      st.s[j] += add.x;
      st.t[j] += add.y;
      if (TO_P && g == 0 && present) p.moved[(int64_t)row * p.tiles + v0 / BM] = st.ref[j];
    }
  }
  // The four lanes of a row have one reference.
  static __device__ __forceinline__ void store(const GemmArgs& p, const State& st, int my_row, int split) {
    if (WHAT == GRAD) return;
    const auto add = [](uint32_t a, uint32_t b) { return __float_as_uint(__uint_as_float(a) + __uint_as_float(b)); };
    const auto four = [&](float x) { return __uint_as_float(with_lane_xor<32>(with_lane_xor<16>(__float_as_uint(x), add), add)); };
#pragma unroll
    for (int j = 0; j < RT; ++j) {
      const int row = row_of(my_row, j);
      const float s = four(st.s[j]), t = four(st.t[j]);
      if (row < p.rows && (threadIdx.x & 63) < 16)
        p.stats[(int64_t)row * p.splits + split] = WHAT == OTHERS ? make_float4(st.ref[j], s + t, s, 0.f) : make_float4(st.ref[j], s, t, 0.f);
    }
  }
};

template <int WHAT, bool TAIL, int RT, bool PAST>
__global__ __launch_bounds__(NTHREADS) __attribute__((amdgpu_waves_per_eu(1, 1)))
void ll_learn_logits_kernel(const LearnArgs p) {
  extern __shared__ __align__(16) unsigned char smem[];
  lens_gemm_dma<LearnEpilogue<WHAT, RT, PAST>, TAIL>(p, smem);
}

template <bool TAIL, int RT, bool PAST>
__global__ __launch_bounds__(NTHREADS) __attribute__((amdgpu_waves_per_eu(1, 1)))
void ll_learn_others_kernel(const LearnArgs p) {
  extern __shared__ __align__(16) unsigned char smem[];
  lens_gemm_dma<LearnEpilogue<OTHERS, RT, PAST>, TAIL>(p, smem);
}

// dA = dz W over one slice of the vocabulary: the tile as it is, for ll_learn_join_kernel, or rounded where the slice is the whole.  A
// lane has four columns of a row in each 16.
template <int RT, bool PAST>
struct BackEpilogue {
  struct State {
    int split;
  };
  static constexpr bool RELOAD_FRAGMENTS = false, OWN_U = false, BACK = true, PAST_CACHES = PAST, HALVES_APART = true;
  static constexpr int ROWS = 64 * RT, ROW_TILES = RT;
  static __device__ __forceinline__ bool skip(const GemmArgs&) { return false; }
  static __device__ __forceinline__ void init(State& st, const GemmArgs&, int, int split) { st.split = split; }
  template <class ACC>
  static __device__ __forceinline__ void tile(const ACC& acc, State& st, int c0, const GemmArgs& args, int my_row) {
    const LearnBackArgs& p = static_cast<const LearnBackArgs&>(args);
    asm volatile("s_nop 15\n\ts_nop 15\n\ts_nop 15" ::: "memory");   // the last MFMA's result is in its registers
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int j = 0; j < RT; ++j) {
      const int row = my_row - lane + 16 * j + (lane & 15);
      if (row >= p.rows) continue;
      const int c = c0 + 4 * (lane >> 4);
      if (p.out != nullptr) {
        const float f = p.terms[row].factor;
        uint16_t* const to = p.out + (int64_t)row * p.d + c;
#pragma unroll
        for (int t = 0; t < 16; ++t) {
          if (c + 16 * t < p.d)
            *reinterpret_cast<uint2*>(to + 16 * t) = f != 0.f ? make_uint2(pack_bf16(f * acc_read(acc[t][j][0]), f * acc_read(acc[t][j][1])),
                                                                           pack_bf16(f * acc_read(acc[t][j][2]), f * acc_read(acc[t][j][3])))
                                                              : make_uint2(0, 0);
        }
        continue;
      }
      float* const to = p.part + ((int64_t)st.split * p.rows + row) * p.d + c;
#pragma unroll
      for (int t = 0; t < 16; ++t) {
        if (c + 16 * t < p.d)
          *reinterpret_cast<float4*>(to + 16 * t) = make_float4(acc_read(acc[t][j][0]), acc_read(acc[t][j][1]), acc_read(acc[t][j][2]), acc_read(acc[t][j][3]));
      }
    }
  }
  static __device__ __forceinline__ void store(const GemmArgs&, const State&, int, int) {}
};

template <int RT, bool PAST>
__global__ __launch_bounds__(NTHREADS) __attribute__((amdgpu_waves_per_eu(1, 1)))
void ll_learn_back_kernel(const LearnBackArgs p) {
  extern __shared__ __align__(16) unsigned char smem[];
  lens_gemm_dma<BackEpilogue<RT, PAST>, false>(p, smem);
}

}  // namespace

namespace ll {

LearnKernel learn_kernel(LearnWhat what, bool ragged, bool past_caches, int row_tiles) {
  return with_row_tiles(row_tiles, [&](auto rt) -> LearnKernel {
    const auto form = [&](auto w) -> LearnKernel {
      return ragged        ? ll_learn_logits_kernel<w(), true, rt(), false>
             : past_caches ? ll_learn_logits_kernel<w(), false, rt(), true>
                           : ll_learn_logits_kernel<w(), false, rt(), false>;
    };
    if (what == OTHERS) return ragged ? ll_learn_others_kernel<true, rt(), false> : past_caches ? ll_learn_others_kernel<false, rt(), true>
                                                                                                : ll_learn_others_kernel<false, rt(), false>;
    if (what == STATS) return form(std::integral_constant<int, STATS>{});
    if (what == EXPS) return form(std::integral_constant<int, EXPS>{});
    return form(std::integral_constant<int, GRAD>{});
  });
}

LearnBackKernel learn_back_kernel(bool past_caches, int row_tiles) {
  return with_row_tiles(row_tiles, [&](auto rt) -> LearnBackKernel {
    return past_caches ? ll_learn_back_kernel<rt(), true> : ll_learn_back_kernel<rt(), false>;
  });
}

}  // namespace ll
