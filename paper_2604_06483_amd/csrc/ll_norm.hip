// The norms around a block (a lens translator, a wrapped layer) with its gate and residual scale, and their gradient.
//
//   u = gamma_y * y / rms(y), or y;   x = h + scale * gate * u;   n = gamma * x / rms(x);   rms(x) = sqrt(mean x^2 + eps)
//
// and backwards, with xh = x / rms(x), e = g_n * gamma:
//
//   dx = g_h + (e - xh mean(e xh)) / rms(x);   du = scale * gate * dx;   d_gate = scale * u * dx;   d_gamma = sum_rows g_n * xh
//   with gamma_y: yh = y / rms(y), f = du * gamma_y, dy = (f - yh mean(f yh)) / rms(y), d_gamma_y = sum_rows du * yh;   else dy = du
//
// Bound by memory: a row is read once, kept in registers (as it came, 16 bits a value) from the statistics to the last output and
// never written in between; the backward pass forms x again from h and y, so that nothing but the inputs need be kept for it.
// All sums are fp32; each output is rounded once.
#include "ll_common.h"

#include <math.h>

#include <type_traits>

namespace {

using namespace ll;

constexpr int NORM_MAX_D = 16384;        // two chunks of eight values for each of 1024 threads

struct NormArgs {
  const uint16_t* hidden;     // [rows, d]
  const uint16_t* y;          // [rows, d]
  const uint16_t* gate;       // [d] (gate_stride 0), [rows, d] (gate_stride d) or nullptr
  const uint16_t* gamma_y;    // [d] or nullptr
  const uint16_t* gamma;      // [d]
  int64_t gate_stride;
  int64_t rows;
  int d;
  float scale, eps;
  uint16_t* out_hidden;       // forward
  uint16_t* out_normed;
  const uint16_t* g_hidden;   // backward: [rows, d] or nullptr
  const uint16_t* g_normed;
  uint16_t* d_hidden;
  uint16_t* d_y;
  uint16_t* d_gate_rows;      // [rows, d], where the gate is
  float* partial;             // [3][workgroups][d]: sums for gate (shared), gamma_y, gamma
};

struct Eight {
  float v[8];
};
__device__ __forceinline__ Eight widen(const uint4 q) {
  return {{bf16_lo(q.x), bf16_hi(q.x), bf16_lo(q.y), bf16_hi(q.y), bf16_lo(q.z), bf16_hi(q.z), bf16_lo(q.w), bf16_hi(q.w)}};
}
__device__ __forceinline__ uint4 narrow(const Eight& e) {
  return make_uint4(pack_bf16(e.v[0], e.v[1]), pack_bf16(e.v[2], e.v[3]), pack_bf16(e.v[4], e.v[5]), pack_bf16(e.v[6], e.v[7]));
}
__device__ __forceinline__ uint4 load8(const uint16_t* p) { return *reinterpret_cast<const uint4*>(p); }
__device__ __forceinline__ void store8(uint16_t* p, const Eight& e) { *reinterpret_cast<uint4*>(p) = narrow(e); }

// Two sums over the workgroup's threads at once; `red` is this reduction's own place (see the kernels for when it is free again).  A lane
// reads one wavefront's pair and the sixteen are summed across lanes: one trip to LDS, not one for every wavefront.
__device__ __forceinline__ float2 group_sum(float a, float b, float2* red) {
  a = wave_sum(a);
  b = wave_sum(b);
  const int lane = threadIdx.x & 63, waves = blockDim.x >> 6;
  if (waves == 1) return make_float2(a, b);
  if (lane == 0) red[threadIdx.x >> 6] = make_float2(a, b);
  __syncthreads();
  const float2 q = (lane & 15) < waves ? red[lane & 15] : make_float2(0.f, 0.f);
  const auto add = [](uint32_t u, uint32_t v) { return __float_as_uint(__uint_as_float(u) + __uint_as_float(v)); };
  const auto sixteen = [&](float x) {
    return __uint_as_float(with_lane_xor<1>(with_lane_xor<2>(with_lane_xor<4>(with_lane_xor<8>(__float_as_uint(x), add), add), add), add));
  };
  return make_float2(sixteen(q.x), sixteen(q.y));
}

// One workgroup a row, NIT chunks of eight values a thread.
template <int NIT, int THREADS, bool POST>
__global__ __launch_bounds__(THREADS) void ll_block_norm_kernel(const NormArgs p) {
  __shared__ float2 red[2][THREADS / 64];
  const int n8 = p.d >> 3, threads = blockDim.x;
  const int64_t row = blockIdx.x, at = row * (int64_t)p.d;
  uint4 h[NIT], y[NIT], k[NIT];
#pragma unroll
  for (int it = 0; it < NIT; ++it) {
    const int c = threadIdx.x + threads * it;
    h[it] = y[it] = k[it] = make_uint4(0, 0, 0, 0);
    if (c < n8) {
      h[it] = load8(p.hidden + at + 8 * c);
      y[it] = load8(p.y + at + 8 * c);
      if (p.gate != nullptr) k[it] = load8(p.gate + row * p.gate_stride + 8 * c);
    }
  }
  float inv_y = 1.f;
  if (POST) {
    float s0 = 0.f, s1 = 0.f;
#pragma unroll
    for (int it = 0; it < NIT; ++it) accum_sq(y[it], s0, s1);
    inv_y = inv_rms_from_sumsq(group_sum(s0 + s1, 0.f, red[0]).x, p.d, p.eps);
  }
  Eight x[NIT];
  float ss = 0.f;
#pragma unroll
  for (int it = 0; it < NIT; ++it) {
    const int c = threadIdx.x + threads * it;
    const Eight hv = widen(h[it]), yv = widen(y[it]), kv = widen(k[it]);
    Eight gy = {{1.f, 1.f, 1.f, 1.f, 1.f, 1.f, 1.f, 1.f}};
    if (POST && c < n8) gy = widen(load8(p.gamma_y + 8 * c));
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float u = POST ? yv.v[i] * inv_y * gy.v[i] : yv.v[i];
      x[it].v[i] = fmaf(p.gate != nullptr ? p.scale * kv.v[i] : p.scale, u, hv.v[i]);
      ss = fmaf(x[it].v[i], x[it].v[i], ss);
    }
  }
  const float inv = inv_rms_from_sumsq(group_sum(ss, 0.f, red[1]).x, p.d, p.eps);
#pragma unroll
  for (int it = 0; it < NIT; ++it) {
    const int c = threadIdx.x + threads * it;
    if (c >= n8) continue;
    const Eight g = widen(load8(p.gamma + 8 * c));
    Eight n;
#pragma unroll
    for (int i = 0; i < 8; ++i) n.v[i] = x[it].v[i] * inv * g.v[i];
    store8(p.out_hidden + at + 8 * c, x[it]);
    store8(p.out_normed + at + 8 * c, n);
  }
}

// A workgroup takes rows blockIdx.x, + gridDim.x, ... and keeps its sums for the parameters in registers over all of them (one column
// belongs to one thread), which are written once, for ll_block_norm_sums_kernel: no atomics, the same bits every time.
// Places of the reductions alternate between rows: a place is written again two rows on, behind a barrier that every thread reaches
// only after it has read it.
// The next row's loads go out before this row's sums (AHEAD) and x is kept from its sum on, where the registers hold them: one chunk a
// thread, d up to 8192; so does what all rows share.  More chunks form x twice and load the shared parameters, and g_hidden, where they
// are used.  The sums for gate and gamma_y are in LDS (IN_LDS: more chunks; or both of them, which leaves 128 registers and no spill:
// d = 2560, 55 500 rows 424 us with both in registers).  More chunks, of 1024 threads, have no more than 128 registers in any case, and all
// but the form without gate and gamma_y spill: 9 to 70 of them, 8000 x 16384 with both norms 970 us, 1.6 TB/s.
enum { NO_GATE, SHARED_GATE, ROWS_GATE };
constexpr bool sums_in_lds(int nit, bool post, int gate) { return nit > 1 || (post && gate == SHARED_GATE); }
template <int NIT, int THREADS, bool POST, int GATE>
__global__ __launch_bounds__(THREADS) void ll_block_norm_grad_kernel(const NormArgs p) {
  constexpr bool AHEAD = NIT == 1, GATED = GATE != NO_GATE, IN_LDS = sums_in_lds(NIT, POST, GATE);
  __shared__ float2 red[2][3][THREADS / 64];
  const int n8 = p.d >> 3, threads = blockDim.x;
  const float inv_d = 1.f / (float)p.d;
  struct Row {
    uint4 h[NIT], y[NIT], k[NIT], gh[NIT], gn[NIT];
  };
  const auto load = [&](int64_t row, Row& q) {
    const int64_t at = row * (int64_t)p.d;
#pragma unroll
    for (int it = 0; it < NIT; ++it) {
      const int c = threadIdx.x + threads * it;
      q.h[it] = q.y[it] = q.gh[it] = q.gn[it] = q.k[it] = make_uint4(0, 0, 0, 0);
      if (c < n8) {
        q.h[it] = load8(p.hidden + at + 8 * c);
        q.y[it] = load8(p.y + at + 8 * c);
        q.gn[it] = load8(p.g_normed + at + 8 * c);
        if (AHEAD && p.g_hidden != nullptr) q.gh[it] = load8(p.g_hidden + at + 8 * c);
        if (GATE == ROWS_GATE) q.k[it] = load8(p.gate + at + 8 * c);
      }
    }
  };
  uint4 gammas[AHEAD ? NIT : 1], gammas_y[POST && AHEAD ? NIT : 1], gates[GATE == SHARED_GATE && AHEAD ? NIT : 1];
  const auto shared = [&](const uint4* kept, const uint16_t* from, int it) {
    const int c = threadIdx.x + threads * it;
    return AHEAD ? kept[it] : c < n8 ? load8(from + 8 * c) : make_uint4(0, 0, 0, 0);
  };
  extern __shared__ __align__(16) float lds_sums[];      // [2][d]: a thread's own columns
  Eight sum_gate[GATE == SHARED_GATE && !IN_LDS ? NIT : 1], sum_y[POST && !IN_LDS ? NIT : 1], sum[NIT];
  const auto lds_sum = [&](int which, int it) { return reinterpret_cast<float4*>(lds_sums + which * p.d + 8 * (threadIdx.x + threads * it)); };
  const auto add = [&](Eight* sums, int which, int it, const Eight& v) {
    if constexpr (!IN_LDS) {
#pragma unroll
      for (int i = 0; i < 8; ++i) sums[it].v[i] += v.v[i];
    } else if ((int)threadIdx.x + threads * it < n8) {
      float4* at = lds_sum(which, it);
#pragma unroll
      for (int q = 0; q < 2; ++q) {
        const float4 x = at[q];
        at[q] = make_float4(x.x + v.v[4 * q], x.y + v.v[4 * q + 1], x.z + v.v[4 * q + 2], x.w + v.v[4 * q + 3]);
      }
    }
  };
#pragma unroll
  for (int it = 0; it < NIT; ++it) {
    const int c = threadIdx.x + threads * it;
    if (AHEAD) {
      gammas[it] = c < n8 ? load8(p.gamma + 8 * c) : make_uint4(0, 0, 0, 0);
      if (POST) gammas_y[it] = c < n8 ? load8(p.gamma_y + 8 * c) : make_uint4(0, 0, 0, 0);
      if (GATE == SHARED_GATE) gates[it] = c < n8 ? load8(p.gate + 8 * c) : make_uint4(0, 0, 0, 0);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      sum[it].v[i] = 0.f;
      if (GATE == SHARED_GATE && !IN_LDS) sum_gate[it].v[i] = 0.f;
      if (POST && !IN_LDS) sum_y[it].v[i] = 0.f;
    }
    if (IN_LDS && c < n8)
      for (int which = 0; which < 2; ++which) lds_sum(which, it)[0] = lds_sum(which, it)[1] = make_float4(0.f, 0.f, 0.f, 0.f);
  }
  int turn = 0;
  Row now, next;
  if (AHEAD) load(blockIdx.x, next);
  for (int64_t row = blockIdx.x; row < p.rows; row += gridDim.x, turn ^= 1) {
    const int64_t at = row * (int64_t)p.d;
    if (AHEAD) {
      now = next;
      if (row + gridDim.x < p.rows) load(row + gridDim.x, next);
    } else {
      load(row, now);
    }
    float inv_y = 1.f;
    if (POST) {
      float s0 = 0.f, s1 = 0.f;
#pragma unroll
      for (int it = 0; it < NIT; ++it) accum_sq(now.y[it], s0, s1);
      inv_y = inv_rms_from_sumsq(group_sum(s0 + s1, 0.f, red[turn][0]).x, p.d, p.eps);
    }
    // x, and at once the sums of x^2 and of e x
    const auto stream = [&](int it) {
      const Eight hv = widen(now.h[it]), yv = widen(now.y[it]);
      Eight gy, kv;
      if (POST) gy = widen(shared(gammas_y, p.gamma_y, it));
      if (GATED) kv = widen(GATE == SHARED_GATE ? shared(gates, p.gate, it) : now.k[it]);
      Eight v;
#pragma unroll
      for (int i = 0; i < 8; ++i) v.v[i] = fmaf(GATED ? p.scale * kv.v[i] : p.scale, POST ? yv.v[i] * inv_y * gy.v[i] : yv.v[i], hv.v[i]);
      return v;
    };
    Eight x[AHEAD ? NIT : 1];
    float ss = 0.f, ex = 0.f;
#pragma unroll
    for (int it = 0; it < NIT; ++it) {
      const Eight v = stream(it), gv = widen(now.gn[it]), gamma = widen(shared(gammas, p.gamma, it));
      if (AHEAD) x[it] = v;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        ss = fmaf(v.v[i], v.v[i], ss);
        ex = fmaf(gv.v[i] * gamma.v[i], v.v[i], ex);
      }
    }
    const float2 both = group_sum(ss, ex, red[turn][1]);
    const float inv = inv_rms_from_sumsq(both.x, p.d, p.eps);
    const float mean_exh = both.y * inv * inv_d;
    Eight du[NIT];
    float fy = 0.f;
#pragma unroll
    for (int it = 0; it < NIT; ++it) {
      const int c = threadIdx.x + threads * it;
      if (!AHEAD && p.g_hidden != nullptr && c < n8) now.gh[it] = load8(p.g_hidden + at + 8 * c);
      const Eight yv = widen(now.y[it]), gv = widen(now.gn[it]), ghv = widen(now.gh[it]), gamma = widen(shared(gammas, p.gamma, it));
      Eight gy, kv;
      if (POST) gy = widen(shared(gammas_y, p.gamma_y, it));
      if (GATED) kv = widen(GATE == SHARED_GATE ? shared(gates, p.gate, it) : now.k[it]);
      const Eight xv = AHEAD ? x[AHEAD ? it : 0] : stream(it);
      Eight dx, dk, dgy;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float yh = yv.v[i] * inv_y, u = POST ? yh * gy.v[i] : yv.v[i];
        const float factor = GATED ? p.scale * kv.v[i] : p.scale;
        const float xh = xv.v[i] * inv;
        dx.v[i] = fmaf(gv.v[i] * gamma.v[i] - xh * mean_exh, inv, ghv.v[i]);
        du[it].v[i] = factor * dx.v[i];
        sum[it].v[i] = fmaf(gv.v[i], xh, sum[it].v[i]);
        if (GATED) dk.v[i] = p.scale * u * dx.v[i];
        if (POST) {
          dgy.v[i] = du[it].v[i] * yh;
          du[it].v[i] *= gy.v[i];
          fy = fmaf(du[it].v[i], yh, fy);
        }
      }
      if (GATE == SHARED_GATE) add(sum_gate, 0, it, dk);
      if (POST) add(sum_y, 1, it, dgy);
      if (c < n8) {
        store8(p.d_hidden + at + 8 * c, dx);
        if (GATE == ROWS_GATE) store8(p.d_gate_rows + at + 8 * c, dk);
        if (!POST) store8(p.d_y + at + 8 * c, du[it]);
      }
    }
    if (POST) {
      const float mean_fyh = group_sum(fy, 0.f, red[turn][2]).x * inv_d;
#pragma unroll
      for (int it = 0; it < NIT; ++it) {
        const int c = threadIdx.x + threads * it;
        if (c >= n8) continue;
        const Eight yv = widen(now.y[it]);
        Eight dy;
#pragma unroll
        for (int i = 0; i < 8; ++i) dy.v[i] = (du[it].v[i] - yv.v[i] * inv_y * mean_fyh) * inv_y;
        store8(p.d_y + at + 8 * c, dy);
      }
    }
  }
  const auto put = [&](int which, auto&& of) {
    float* to = p.partial + ((int64_t)which * gridDim.x + blockIdx.x) * p.d;
#pragma unroll
    for (int it = 0; it < NIT; ++it) {
      const int c = threadIdx.x + threads * it;
      if (c >= n8) continue;
      const Eight s = of(it);
      *reinterpret_cast<float4*>(to + 8 * c) = make_float4(s.v[0], s.v[1], s.v[2], s.v[3]);
      *reinterpret_cast<float4*>(to + 8 * c + 4) = make_float4(s.v[4], s.v[5], s.v[6], s.v[7]);
    }
  };
  const auto kept = [&](const Eight* sums, int which, int it) {
    if (!IN_LDS) return sums[it];
    const float4 lo = lds_sum(which, it)[0], hi = lds_sum(which, it)[1];
    return Eight{{lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w}};
  };
  if (GATE == SHARED_GATE) put(0, [&](int it) { return kept(sum_gate, 0, it); });
  if (POST) put(1, [&](int it) { return kept(sum_y, 1, it); });
  put(2, [&](int it) { return sum[it]; });
}

// The workgroups' sums joined: block (32 columns, parameter); 32 runs of the workgroups side by side, then the runs in order.
__global__ __launch_bounds__(256) void ll_block_norm_sums_kernel(const float* __restrict__ partial, int groups, int d,
                                                                 float* __restrict__ d_gate, float* __restrict__ d_gamma_y,
                                                                 float* __restrict__ d_gamma) {
  constexpr int LANES = 8, RUNS = 32;
  __shared__ float4 red[RUNS][LANES];
  float* out = blockIdx.y == 0 ? d_gate : blockIdx.y == 1 ? d_gamma_y : d_gamma;
  if (out == nullptr) return;
  const int col = threadIdx.x % LANES, run = threadIdx.x / LANES, c = (blockIdx.x * LANES + col) * 4;
  float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
  if (c < d) {
    const float* from = partial + (int64_t)blockIdx.y * groups * d + c;
#pragma unroll 8
    for (int g = run; g < groups; g += RUNS) {
      const float4 x = *reinterpret_cast<const float4*>(from + (int64_t)g * d);
      s.x += x.x;
      s.y += x.y;
      s.z += x.z;
      s.w += x.w;
    }
  }
  red[run][col] = s;
  __syncthreads();
  if (run != 0 || c >= d) return;
#pragma unroll
  for (int r = 1; r < RUNS; ++r) {
    const float4 x = red[r][col];
    s.x += x.x;
    s.y += x.y;
    s.z += x.z;
    s.w += x.w;
  }
  *reinterpret_cast<float4*>(out + c) = s;
}

// Chunks of eight values a thread and most threads of a workgroup: the fewest chunks that 512 threads hold a row with, up to two, then
// 1024 threads; of the gradient, whose registers are short, 1024 threads before a second chunk.
template <class F>
void with_chunks(int d, bool grad, F f) {
  using std::integral_constant;
  const int n8 = d >> 3;
  if (n8 <= 512) f(integral_constant<int, 1>{}, integral_constant<int, 512>{});
  else if (n8 <= 1024 && grad) f(integral_constant<int, 1>{}, integral_constant<int, 1024>{});
  else if (n8 <= 1024) f(integral_constant<int, 2>{}, integral_constant<int, 512>{});
  else f(integral_constant<int, 2>{}, integral_constant<int, 1024>{});
}
unsigned threads_for(int d, int nit) { return (unsigned)(((d >> 3) + nit - 1) / nit + kWave - 1) / kWave * kWave; }

// Workgroups of the gradient: as many as are on the chip at once (some 16 wavefronts a compute unit), each with its own sums of the
// parameters' gradients; once every compute unit has one, at least four rows each, or the sums (twelve bytes a column, written and
// read) are more than the rows: 777 x 1608 with all inputs 14.8 -> 13.1 us, 3000 x 1024 21.7 -> 19.6, 400 x 4096 19.9 -> 17.0 (a row each -> four).
int grad_groups(int64_t rows, int d) {
  int waves = 0;
  with_chunks(d, true, [&](auto nit, auto) { waves = (int)threads_for(d, nit()) / kWave; });
  const int most = 256 * (waves >= 16 ? 1 : 16 / waves);
  const int64_t groups = rows <= 256 ? rows : rows <= 1024 ? 256 : (rows + 3) / 4;
  return (int)(groups < most ? groups : most);
}

template <class F>
void with_gate(int gate, F f) {
  if (gate == NO_GATE) f(std::integral_constant<int, NO_GATE>{});
  else if (gate == SHARED_GATE) f(std::integral_constant<int, SHARED_GATE>{});
  else f(std::integral_constant<int, ROWS_GATE>{});
}
template <class F>
void with_bool(bool b, F f) {
  if (b) f(std::true_type{});
  else f(std::false_type{});
}

bool misaligned(const void* p) { return ((uintptr_t)p & 15) != 0; }

bool valid_shape(const ll_shape* s) {
  return s != nullptr && s->N >= 0 && s->N <= INT32_MAX && s->d > 0 && s->d % 8 == 0 && s->d <= NORM_MAX_D;
}

int check_block(const ll_shape* s, const void* hidden, const void* y, const void* gate, int gate_rows, float scale, const void* gamma_y,
                const void* gamma, float eps) {
  if (hidden == nullptr || y == nullptr || gamma == nullptr || !(eps >= 0.f) || isinf(eps) || !isfinite(scale)) return LL_EINVAL;
  if (gate_rows != 0 && gate_rows != 1) return LL_EINVAL;
  if (gate == nullptr && gate_rows != 0) return LL_EINVAL;
  if (misaligned(hidden) || misaligned(y) || misaligned(gate) || misaligned(gamma_y) || misaligned(gamma)) return LL_EINVAL;
  return LL_OK;
}

}  // namespace

extern "C" {

int ll_block_norm(const ll_shape* shape, const void* hidden, const void* y, const void* gate, int gate_rows, float scale,
                  const void* gamma_y, const void* gamma, float eps, void* out_hidden, void* out_normed, void* stream) {
  if (!valid_shape(shape)) return LL_EINVAL;
  if (shape->N == 0) return LL_OK;
  const int rc = check_block(shape, hidden, y, gate, gate_rows, scale, gamma_y, gamma, eps);
  if (rc != LL_OK) return rc;
  if (out_hidden == nullptr || out_normed == nullptr || misaligned(out_hidden) || misaligned(out_normed)) return LL_EINVAL;
  NormArgs p = {};
  p.hidden = (const uint16_t*)hidden;
  p.y = (const uint16_t*)y;
  p.gate = (const uint16_t*)gate;
  p.gamma_y = (const uint16_t*)gamma_y;
  p.gamma = (const uint16_t*)gamma;
  p.gate_stride = gate_rows ? shape->d : 0;
  p.rows = shape->N;
  p.d = shape->d;
  p.scale = scale;
  p.eps = eps;
  p.out_hidden = (uint16_t*)out_hidden;
  p.out_normed = (uint16_t*)out_normed;
  // (a launch has at most 2^32 threads)
  constexpr int64_t MOST = (int64_t)1 << 21;
  for (int64_t left = shape->N; left > 0; left -= MOST) {
    p.rows = left < MOST ? left : MOST;
    with_chunks(p.d, false, [&](auto nit, auto threads) {
      with_bool(gamma_y != nullptr, [&](auto post) {
        if constexpr (nit() > 1 || threads() == 512)
          hipLaunchKernelGGL((ll_block_norm_kernel<nit(), threads(), post()>), dim3((unsigned)p.rows), dim3(threads_for(p.d, nit())), 0,
                             (hipStream_t)stream, p);
      });
    });
    LL_HIP_CHECK(hipGetLastError());
    const int64_t step = MOST * p.d;
    p.hidden += step;
    p.y += step;
    if (gate_rows) p.gate += step;
    p.out_hidden += step;
    p.out_normed += step;
  }
  return LL_OK;
}

size_t ll_block_norm_grad_workspace_bytes(const ll_shape* shape) {
  if (!valid_shape(shape)) return 0;
  return align_up((size_t)3 * grad_groups(shape->N > 0 ? shape->N : 1, shape->d) * shape->d * sizeof(float), 256);
}

int ll_block_norm_grad(const ll_shape* shape, void* workspace, size_t workspace_bytes, const void* hidden, const void* y,
                       const void* gate, int gate_rows, float scale, const void* gamma_y, const void* gamma, float eps,
                       const void* g_hidden, const void* g_normed, void* d_hidden, void* d_y, void* d_gate, float* d_gamma_y,
                       float* d_gamma, void* stream) {
  if (!valid_shape(shape)) return LL_EINVAL;
  if (shape->N > 0) {
    const int rc = check_block(shape, hidden, y, gate, gate_rows, scale, gamma_y, gamma, eps);
    if (rc != LL_OK) return rc;
    if (g_normed == nullptr || d_hidden == nullptr || d_y == nullptr) return LL_EINVAL;
    if (misaligned(g_hidden) || misaligned(g_normed) || misaligned(d_hidden) || misaligned(d_y)) return LL_EINVAL;
  }
  if (d_gamma == nullptr || (gate != nullptr) != (d_gate != nullptr) || (gamma_y != nullptr) != (d_gamma_y != nullptr)) return LL_EINVAL;
  if (misaligned(d_gate) || misaligned(d_gamma_y) || misaligned(d_gamma)) return LL_EINVAL;
  const size_t need = ll_block_norm_grad_workspace_bytes(shape);
  if (workspace == nullptr || workspace_bytes < need || ((uintptr_t)workspace & 255) != 0) return LL_EWORKSPACE;
  NormArgs p = {};
  p.hidden = (const uint16_t*)hidden;
  p.y = (const uint16_t*)y;
  p.gate = (const uint16_t*)gate;
  p.gamma_y = (const uint16_t*)gamma_y;
  p.gamma = (const uint16_t*)gamma;
  p.gate_stride = gate_rows ? shape->d : 0;
  p.rows = shape->N;
  p.d = shape->d;
  p.scale = scale;
  p.eps = eps;
  p.g_hidden = (const uint16_t*)g_hidden;
  p.g_normed = (const uint16_t*)g_normed;
  p.d_hidden = (uint16_t*)d_hidden;
  p.d_y = (uint16_t*)d_y;
  p.d_gate_rows = gate_rows ? (uint16_t*)d_gate : nullptr;
  p.partial = (float*)workspace;
  const int groups = grad_groups(p.rows, p.d);
  int rc = LL_OK;
  if (groups > 0) {
    with_chunks(p.d, true, [&](auto nit, auto threads) {
      with_bool(gamma_y != nullptr, [&](auto post) {
        with_gate(gate == nullptr ? NO_GATE : gate_rows ? ROWS_GATE : SHARED_GATE, [&](auto gated) {
          if constexpr (nit() == 1 || threads() == 1024) {
            const auto kernel = ll_block_norm_grad_kernel<nit(), threads(), post(), gated()>;
            const size_t lds = sums_in_lds(nit(), post(), gated()) ? (size_t)2 * p.d * sizeof(float) : 0;
            if (lds > 0) rc = allow_dynamic_lds(reinterpret_cast<const void*>(kernel), (size_t)2 * NORM_MAX_D * sizeof(float));
            if (rc == LL_OK) hipLaunchKernelGGL(kernel, dim3(groups), dim3(threads_for(p.d, nit())), lds, (hipStream_t)stream, p);
          }
        });
      });
    });
    if (rc != LL_OK) return rc;
    LL_HIP_CHECK(hipGetLastError());
  }
  // (no rows: the sums over none are zeros)
  hipLaunchKernelGGL(ll_block_norm_sums_kernel, dim3((unsigned)((p.d + 31) / 32), 3), dim3(256), 0, (hipStream_t)stream, p.partial, groups,
                     p.d, gate != nullptr && !gate_rows ? (float*)d_gate : nullptr, d_gamma_y, d_gamma);
  LL_HIP_CHECK(hipGetLastError());
  return LL_OK;
}

}  // extern "C"
