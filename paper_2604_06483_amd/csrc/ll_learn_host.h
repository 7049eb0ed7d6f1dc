// What the calls that learn through the lens share (ll_learn.hip, ll_answers.hip): the small kernels around the products, the plan of a call
// and its launches.
#pragma once

#include "ll_learn.h"

namespace {

// A row of a hidden size that is not a multiple of 64, zero padded to one, by a workgroup; no panel: the rows are read where they are.
__device__ __forceinline__ void pad_row(const uint16_t* __restrict__ rows, int64_t row, int d, uint16_t* __restrict__ panel, int64_t lda) {
  if (panel == nullptr) return;
  for (int c = threadIdx.x; c < lda / 8; c += (int)blockDim.x)
    reinterpret_cast<uint4*>(panel + row * lda)[c] =
        8 * c < d ? reinterpret_cast<const uint4*>(rows + row * d)[c] : make_uint4(0, 0, 0, 0);
}
struct RowStats {
  float lse2, t;     // log2 of the sum of 2^x; sum of p (x - lse2), x = z log2 e: minus the entropy, in powers of two
  float ref, sum;    // that sum is 2^ref sum
};
// A row's parts, `stride` apart, joined by a wavefront.  OTHERS: they hold sums without the row's token, and so does t, relative to 2^ref.
template <bool OTHERS = false>
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
    t += q.y > 0.f ? e * (OTHERS ? q.z : fmaf(by, q.y, q.z)) : 0.f;
  }
  s = wave_sum(s);
  t = wave_sum(t);
  const float log_s = __builtin_amdgcn_logf(s);
  RowStats r = {m + log_s, OTHERS ? t : t / s - log_s, m, s};
  if (wave_sum(nan ? 1.f : 0.f) > 0.f) r.lse2 = r.t = r.sum = NAN;
  return r;
}

// What brings a tile of P, relative to `moved`, to the row's base.  A tile that adds to the row's sum has a reference at most 60 powers of two above the
// sum; one past the vocabulary, or of ids that have no probability, holds zeros relative to anything, and 0 times infinity is none.  (NaN passes.)
__device__ __forceinline__ float tile_to_base(float moved, float base) {
  const float up = moved - base;
  return __builtin_amdgcn_exp2f(up > 127.f ? 127.f : up);
}

// A row of P brought to one base, by a workgroup of 256 threads (see ll_distill_rows_kernel).  width: of a tile that has a reference of its own, 16 ids
// or a multiple; eight places hold four ids of each half of 32 (see place_in_p).
__device__ __forceinline__ void tiles_to_base(uint16_t* at, int64_t ldp, const float* __restrict__ moved, float base, int width = BM) {
  for (int64_t c = 8 * (int)threadIdx.x; c < ldp; c += 8 * 256) {
    const uint4 q = *reinterpret_cast<const uint4*>(at + c);
    const int64_t id = c & ~(int64_t)31;
    const float by = tile_to_base(moved[id / width], base), and_by = tile_to_base(moved[(id + 16) / width], base);
    *reinterpret_cast<uint4*>(at + c) = make_uint4(pack_bf16(bf16_lo(q.x) * by, bf16_hi(q.x) * by), pack_bf16(bf16_lo(q.y) * by, bf16_hi(q.y) * by),
                                                   pack_bf16(bf16_lo(q.z) * and_by, bf16_hi(q.z) * and_by), pack_bf16(bf16_lo(q.w) * and_by, bf16_hi(q.w) * and_by));
  }
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

struct FewJoinArgs {
  FewLearnArgs f;
  int parts, stride;        // stride: rows of a part's sums and statistics
  const float* scores;      // ll_distill's
  const float* weight;
  float* loss;
  uint16_t* out;
};
// The parts' sums joined, and the listed tokens' rows of W: block (64 columns, row), sixteen runs of the parts and of the list side by side.  What
// a thread adds is asked for first and waits in registers for what it is multiplied by.
struct FewColumns {
  static constexpr int RUNS = 16, MOST = FEW_LEARN_STREAMS / RUNS;
  float4 x[MOST];
  static __device__ __forceinline__ int column() { return blockIdx.x * 64 + (threadIdx.x & 15) * 4; }

  __device__ __forceinline__ void load(const FewJoinArgs& p, int row) {
    const int run = threadIdx.x >> 4, c = column(), d = p.f.list.d;
    const float* from = p.f.sums + (int64_t)row * d + (c < d ? c : 0);
    const int64_t stride = (int64_t)p.stride * d;
#pragma unroll
    for (int j = 0; j < MOST; ++j) {
      const int i = run + RUNS * j;
      x[j] = *reinterpret_cast<const float4*>(from + (i < p.parts ? i : 0) * stride);
    }
  }
  // scale: what each part is multiplied by, or nullptr (1); share and id_of: the list's entries (id below 0: none); all three in LDS.
  __device__ __forceinline__ void join(const FewJoinArgs& p, int row, float factor, const float* scale, const float* share, const int* id_of) {
    __shared__ float4 red[RUNS][16];
    const ListArgs& l = p.f.list;
    const int col = threadIdx.x & 15, run = threadIdx.x >> 4, c = column();
    float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
    if (c < l.d && factor != 0.f) {
#pragma unroll
      for (int j = 0; j < MOST; ++j) {
        const int i = run + RUNS * j;
        if (i >= p.parts) continue;
        const float by = scale != nullptr ? scale[i] : 1.f;
        s.x = fmaf(by, x[j].x, s.x);
        s.y = fmaf(by, x[j].y, s.y);
        s.z = fmaf(by, x[j].z, s.z);
        s.w = fmaf(by, x[j].w, s.w);
      }
      for (int i = run; i < l.k; i += RUNS) {
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
    for (int i = 1; i < RUNS; ++i) {
      const float4 y = red[i][col];
      s.x += y.x;
      s.y += y.y;
      s.z += y.z;
      s.w += y.w;
    }
    *reinterpret_cast<uint2*>(p.out + (int64_t)row * l.d + c) = make_uint2(pack_bf16(factor * s.x, factor * s.y), pack_bf16(factor * s.z, factor * s.w));
  }
};

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

// sums_of: the passes whose sums of the product backwards are kept, or 0: as many as the call itself needs.
LearnPlan plan_for(const ll_shape* s, int k, Needs needs, int64_t sums_of = 0) {
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
    l.part = take((l.back_splits > 1 || sums_of > 0 ? rows * l.back_splits * s->d * sizeof(float) : 0) * (size_t)(sums_of > 1 ? sums_of : 1));
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
  int few_join(void (*kernel)(const FewJoinArgs), const FewJoinArgs& p) const {
    hipLaunchKernelGGL(kernel, dim3((shape->d + 63) / 64, n), dim3(256), 0, stream, p);
    LL_HIP_CHECK(hipGetLastError());
    return LL_OK;
  }

  // where the rows are padded to, by a kernel before the first product
  uint16_t* panel() const { return l.lda != shape->d ? at<uint16_t>(ws, l.panel) : nullptr; }

  template <LearnWhat WHAT>
  int logits(const int32_t* ids = nullptr) const {   // ids: OTHERS'
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
      p.target = ids;
      p.z = at<float>(ws, l.z);
    }
    const LearnKernel kernel = learn_kernel(WHAT, l.lda != shape->d, past_caches(), l.row_tiles);
    const size_t lds = LEARN_LDS;
    if (const int rc = allow_dynamic_lds(reinterpret_cast<const void*>(kernel), lds); rc != LL_OK) return rc;
    const unsigned groups = (unsigned)((p.row_blocks * p.splits + NUM_XCD - 1) / NUM_XCD * NUM_XCD);
    hipLaunchKernelGGL(kernel, dim3(groups), dim3(NTHREADS), lds, stream, p);
    LL_HIP_CHECK(hipGetLastError());
    return LL_OK;
  }

  // P to the gradient of the rows; or, without `out`, its product alone to `part`, a slice of the vocabulary after the other.
  int back(uint16_t* out, float* part) const {
    LearnBackArgs p = {};
    p.A = at<uint16_t>(ws, l.P);
    p.W = W;
    p.part = part;
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
    return LL_OK;
  }
  int back(uint16_t* out) const {
    float* const part = at<float>(ws, l.part);
    if (const int rc = back(out, part); rc != LL_OK || l.back_splits == 1) return rc;
    hipLaunchKernelGGL(ll_learn_join_kernel, dim3((shape->d + 1023) / 1024, n), dim3(256), 0, stream, part, l.back_splits, n, shape->d,
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
