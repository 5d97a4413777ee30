// residual_norm_back.hip -- the step between two blocks on the residual stream, its
// gradients (residual_norm.h has the formulas).
//
// Bound: memory, r, y and the gradients of r and h in, those of x and y out: 32,760 rows of
// 1,536 columns in bf16 132 us (4.6 TB/s) and 7 for the sums, of 5,120 columns with a stream
// in 32 bits 612 and 15 (4.8 TB/s in all).  Rows are held in registers as forward, norms taken
// again from them (nothing is saved for the backward pass); eight columns a thread, as the
// sums of three more rows stay there too (32 columns a thread took 300 registers, one wave a
// SIMD: 315 us), the next row's loads going out before a row is worked (170 us without).
// The sums over a frame's rows stay in registers over a unit's rows, are joined in LDS over
// the teams of a workgroup, and (unless they are the whole frame's) go as one row of partial
// sums a workgroup to the second kernel, which adds a frame's in a fixed order; weights, which
// belong to all frames, take another, and long sums a step between.
#include <algorithm>

#include "residual_norm.h"

namespace lvsa {
namespace {

// Sums over rows (sum_rows): SLICES threads share the rows of four columns, a workgroup works
// LANES fours of columns.
constexpr int SLICES = 32, LANES = 16;
constexpr int MIN_SHARED = 192;   // partial sums of a frame from which on they are shared out
                                  // (share_kernel; 191 of them 13.8 us, 256 shared out 14.0)
constexpr int MAX_SHARES = 512;
constexpr int ENOUGH = 512;       // workgroups that need no shares

template <typename S, typename Y, int TEAM, int V, int MODE>
__global__ __launch_bounds__(norm_bound(TEAM)) void backward_kernel(const NormArgs a) {
  __shared__ StatsLds lds;
  __shared__ float join[whole_group(TEAM) ? 1 : kNormGroup * 8];
  int turn = 0;
  constexpr bool GROUP = whole_group(TEAM);
  const int team = GROUP ? (int)blockDim.x : TEAM, teams = GROUP ? 1 : kNormGroup / TEAM;
  const int t = GROUP ? threadIdx.x : threadIdx.x % TEAM;
  const int64_t id = (int64_t)blockIdx.x * teams + (GROUP ? 0 : threadIdx.x / TEAM);
  const bool there = id < (int64_t)a.frames * a.units;   // all of a workgroup where joined
  NormUnit u = {0, 0, 0};
  if (there) u = norm_unit(a, id);
  const float inv_dim = 1.f / (float)a.dim;

  bool ok[V];
  float g[V][8], m[V][8], sa[V][8], sb[V][8], sc[V][8];
#pragma unroll
  for (int v = 0; v < V; ++v) {
    const int32_t col = 8 * (t + team * v);
    ok[v] = there && col < a.dim;
#pragma unroll
    for (int k = 0; k < 8; ++k) sa[v][k] = sb[v][k] = sc[v][k] = g[v][k] = m[v][k] = 0.f;
    if (!ok[v]) continue;
    float p[8];
    load_param(a.gate, a.param_type, (int64_t)u.f * a.gate_st + col, 1.f, g[v]);
    load_param(a.post_weight, a.param_type, col, 1.f, p);
#pragma unroll
    for (int k = 0; k < 8; ++k) g[v][k] *= p[k];
    load_param(a.weight, a.param_type, col, 1.f, m[v]);
    load_param(a.scale, a.param_type, (int64_t)u.f * a.scale_st + col, 0.f, p);
#pragma unroll
    for (int k = 0; k < 8; ++k) m[v][k] *= 1.f + p[k];
  }

  Raw8<S> rx[V], re[V];
  Raw8<Y> rd[V], ry[V];
#pragma unroll
  for (int v = 0; v < V; ++v) rx[v].v = 0, re[v].v = 0, rd[v].v = 0, ry[v].v = 0;
  auto load_row = [&](int64_t i) {
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const int64_t col = 8 * (t + team * v);
      if (!ok[v]) continue;
      if (a.norm != LVSA_NORM_NONE) {
        rx[v].load((const S*)a.x + i * a.x_st + col);
        rd[v].load((const Y*)a.gh + i * a.gh_st + col);
      }
      if (a.gr) re[v].load((const S*)a.gr + i * a.gr_st + col);
      if (MODE != NORM_OF_X) ry[v].load((const Y*)a.y + i * a.y_st + col);
    }
  };
  if (u.lo < u.hi) load_row(u.lo);
  for (int64_t i = u.lo; i < u.hi; ++i) {
    float e[V][8], x[V][8], y[V][8], d[V][8];
#pragma unroll
    for (int v = 0; v < V; ++v) {
      re[v].get(e[v]);
      rx[v].get(x[v]);
      ry[v].get(y[v]);
      rd[v].get(d[v]);
    }
    if (i + 1 < u.hi) load_row(i + 1);
    if (a.norm != LVSA_NORM_NONE) {
      float dm[V][8];
#pragma unroll
      for (int v = 0; v < V; ++v)
#pragma unroll
        for (int k = 0; k < 8; ++k) dm[v][k] = d[v][k] * m[v][k];
      const RowStats r =
          row_stats<TEAM, V, true>(x, dm, ok, a.norm, inv_dim, a.dim, a.eps, &lds, turn);
#pragma unroll
      for (int v = 0; v < V; ++v)
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          const float unit = (x[v][k] - r.mean) * r.factor;
          sa[v][k] = __builtin_fmaf(d[v][k], unit, sa[v][k]);
          sb[v][k] += d[v][k];
          const float back =
              r.factor * (d[v][k] * m[v][k] - r.g_mean - unit * r.gu_mean);
          e[v][k] = ok[v] ? e[v][k] + back : 0.f;
        }
    }
    if (a.r) {
#pragma unroll
      for (int v = 0; v < V; ++v) {
        if (!ok[v]) continue;
        float w[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) w[k] = a.a * e[v][k];
        store8((S*)a.r + i * a.r_st + 8 * (t + team * v), w);
      }
    }
    if constexpr (MODE == NORM_OF_X) continue;
    if constexpr (MODE == NORM_POST) {
      float eg[V][8];
#pragma unroll
      for (int v = 0; v < V; ++v)
#pragma unroll
        for (int k = 0; k < 8; ++k) eg[v][k] = e[v][k] * g[v][k];
      const RowStats r =
          row_stats<TEAM, V, true>(y, eg, ok, a.post, inv_dim, a.dim, a.eps, &lds, turn);
#pragma unroll
      for (int v = 0; v < V; ++v)
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          const float unit = (y[v][k] - r.mean) * r.factor;
          sc[v][k] = __builtin_fmaf(e[v][k], unit, sc[v][k]);
          y[v][k] = r.factor * (e[v][k] * g[v][k] - r.g_mean - unit * r.gu_mean);
        }
    } else {
#pragma unroll
      for (int v = 0; v < V; ++v)
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          sc[v][k] = __builtin_fmaf(e[v][k], y[v][k], sc[v][k]);
          y[v][k] = e[v][k] * g[v][k];
        }
    }
    if (a.h) {
#pragma unroll
      for (int v = 0; v < V; ++v)
        if (ok[v]) store8((Y*)a.h + i * a.h_st + 8 * (t + team * v), y[v]);
    }
  }

  if (a.direct) {   // the team has had all of the frame's rows
#pragma unroll
    for (int v = 0; v < V; ++v) {
      if (!ok[v]) continue;
      const int32_t col = 8 * (t + team * v);
      const int64_t at = (int64_t)u.f * a.dim + col;
      float w[8], b[8];
      load_param(a.weight, a.param_type, col, 1.f, w);
      load_param(a.bias, a.param_type, col, 0.f, b);
#pragma unroll
      for (int k = 0; k < 8; ++k) w[k] = w[k] * sa[v][k] + b[k] * sb[v][k];
      if (a.d_scale) store_param(a.d_scale, a.param_type, at, w);
      if (a.d_shift) store_param(a.d_shift, a.param_type, at, sb[v]);
      load_param(a.post_weight, a.param_type, col, 1.f, w);
#pragma unroll
      for (int k = 0; k < 8; ++k) w[k] *= sc[v][k];
      if (a.d_gate) store_param(a.d_gate, a.param_type, at, w);
      if (!a.weights) continue;
      load_param(a.scale, a.param_type, (int64_t)u.f * a.scale_st + col, 0.f, w);
      load_param(a.gate, a.param_type, (int64_t)u.f * a.gate_st + col, 1.f, b);
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        sa[v][k] *= 1.f + w[k];
        sb[v][k] *= 1.f + w[k];
        sc[v][k] *= b[k];
      }
      if (a.frame_sums) {
        float* const to = a.frame_sums + 3 * (int64_t)u.f * a.dim + col;
        store8(to, sa[v]);
        store8(to + a.dim, sb[v]);
        store8(to + 2 * (int64_t)a.dim, sc[v]);
      } else {   // the only frame
        if (a.d_weight) store_param(a.d_weight, a.param_type, col, sa[v]);
        if (a.d_bias) store_param(a.d_bias, a.param_type, col, sb[v]);
        if (a.d_post_weight) store_param(a.d_post_weight, a.param_type, col, sc[v]);
      }
    }
    return;
  }
  if (!a.partial) return;
  if (!GROUP && a.joined) {
    // V is 1: a team's columns are 8 t .. 8 t + 7.
    const int64_t row = (int64_t)blockIdx.x * 3;
#pragma unroll
    for (int which = 0; which < 3; ++which) {
      __syncthreads();
      store8(join + threadIdx.x * 8, which == 0 ? sa[0] : which == 1 ? sb[0] : sc[0]);
      __syncthreads();
      for (int c = threadIdx.x; c < a.dim; c += kNormGroup) {
        float s = 0.f;
        for (int w = 0; w < teams; ++w) s += join[w * team * 8 + c];
        a.partial[(row + which) * a.dim + c] = s;
      }
    }
  } else {
#pragma unroll
    for (int v = 0; v < V; ++v) {
      if (!ok[v]) continue;
      float* const at = a.partial + id * 3 * a.dim + 8 * (t + team * v);
      store8(at, sa[v]);
      store8(at + a.dim, sb[v]);
      store8(at + 2 * (int64_t)a.dim, sc[v]);
    }
  }
}

// Adds rows of three sums, in the order of the slices; the results are in every thread.
__device__ __forceinline__ void sum_rows(const float* rows, int64_t n, int32_t dim, int32_t col,
                                         f32x4v (&s)[3], f32x4v (&lds)[3][SLICES][LANES]) {
  const int lane = threadIdx.x % LANES, slice = threadIdx.x / LANES;
#pragma unroll
  for (int w = 0; w < 3; ++w) s[w] = f32x4v{};
  if (col < dim) {
#pragma unroll 4
    for (int64_t i = slice; i < n; i += SLICES)
#pragma unroll
      for (int w = 0; w < 3; ++w) s[w] += *(const f32x4v*)(rows + (i * 3 + w) * dim + col);
  }
#pragma unroll
  for (int w = 0; w < 3; ++w) lds[w][slice][lane] = s[w];
  __syncthreads();
  f32x4v sum = f32x4v{};
  if (slice < 3)
    for (int k = 0; k < SLICES; ++k) sum += lds[slice][k][lane];
  __syncthreads();
  if (slice < 3) lds[slice][0][lane] = sum;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < 3; ++w) s[w] = lds[w][0][lane];
}

__device__ __forceinline__ f32x4v param4(const void* p, int32_t type, int64_t i, float none) {
  if (!p) return f32x4v{none, none, none, none};
  if (type == LVSA_F32) return *(const f32x4v*)((const float*)p + i);
  f32x4v x;
#pragma unroll
  for (int k = 0; k < 4; ++k)
    x[k] = type == LVSA_BF16 ? (float)((const __bf16*)p)[i + k] : (float)((const _Float16*)p)[i + k];
  return x;
}
__device__ __forceinline__ void put4(void* p, int32_t type, int64_t i, f32x4v x) {
  if (!p) return;
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    if (type == LVSA_F32)
      ((float*)p)[i + k] = x[k];
    else if (type == LVSA_BF16)
      ((__bf16*)p)[i + k] = (__bf16)x[k];
    else
      ((_Float16*)p)[i + k] = (_Float16)x[k];
  }
}

// A frame's sums: the gradients of its gate, scale and shift, and what it adds to those
// of the weights (to frame_sums; a single frame's are the gradients, which saves a launch:
// 64 rows of 1,536 columns with five parameters 11.8 -> 9.4 us).
__global__ __launch_bounds__(SLICES* LANES) void frame_kernel(const NormArgs a, const float* rows,
                                                              int32_t per_frame) {
  __shared__ f32x4v lds[3][SLICES][LANES];
  const int32_t f = blockIdx.x;
  const int32_t col = 4 * (int32_t)(blockIdx.y * LANES + threadIdx.x % LANES);
  f32x4v s[3];
  sum_rows(rows + (int64_t)f * per_frame * 3 * a.dim, per_frame, a.dim, col, s, lds);
  if (threadIdx.x < LANES && col < a.dim) {
    const int64_t at = (int64_t)f * a.dim + col;
    const f32x4v w = param4(a.weight, a.param_type, col, 1.f);
    const f32x4v b = param4(a.bias, a.param_type, col, 0.f);
    put4(a.d_scale, a.param_type, at, w * s[0] + b * s[1]);
    put4(a.d_shift, a.param_type, at, s[1]);
    put4(a.d_gate, a.param_type, at, param4(a.post_weight, a.param_type, col, 1.f) * s[2]);
    const f32x4v k = param4(a.scale, a.param_type, (int64_t)f * a.scale_st + col, 0.f) + 1.f;
    const f32x4v g = param4(a.gate, a.param_type, (int64_t)f * a.gate_st + col, 1.f);
    if (a.frame_sums) {
      float* const to = a.frame_sums + (int64_t)f * 3 * a.dim + col;
      *(f32x4v*)to = k * s[0];
      *(f32x4v*)(to + a.dim) = k * s[1];
      *(f32x4v*)(to + 2 * (int64_t)a.dim) = g * s[2];
    } else if (a.frames == 1) {
      put4(a.d_weight, a.param_type, col, k * s[0]);
      put4(a.d_bias, a.param_type, col, k * s[1]);
      put4(a.d_post_weight, a.param_type, col, g * s[2]);
    }
  }
}

// Few frames of many partial sums: of each frame's `per_frame` rows `shares` equal stretches'
// sums, [frame][share][3][dim], for the frame kernel.  (One frame of 1,000 rows of 1,536
// columns 45 -> 24 us, of 32,760 rows 159 -> 140; of 256 rows 18.9 -> 14.0.)  And of many
// frames' sums for the weights (4,000 rows of 1,536 columns, each a frame, 422 -> 77 us, with
// the frames' gradients from the first kernel).
__global__ __launch_bounds__(SLICES* LANES) void share_kernel(const NormArgs a, const float* rows,
                                                              float* to, int32_t per_frame,
                                                              int32_t shares) {
  __shared__ f32x4v lds[3][SLICES][LANES];
  const int32_t f = blockIdx.x / shares, share = blockIdx.x % shares;
  const int32_t col = 4 * (int32_t)(blockIdx.y * LANES + threadIdx.x % LANES);
  const int32_t len = (per_frame + shares - 1) / shares, first = min(share * len, per_frame);
  f32x4v s[3];
  sum_rows(rows + ((int64_t)f * per_frame + first) * 3 * a.dim, min(len, per_frame - first),
           a.dim, col, s, lds);
  if (threadIdx.x >= LANES || col >= a.dim) return;
#pragma unroll
  for (int w = 0; w < 3; ++w) *(f32x4v*)(to + ((int64_t)blockIdx.x * 3 + w) * a.dim + col) = s[w];
}

// Those of the weights, over the frames.  (The frame kernel's last workgroup of each group of
// columns doing it instead takes a release of every workgroup's sums: 68 us against 16 for
// both kernels at 21 frames of 5,120 columns.)
__global__ __launch_bounds__(SLICES* LANES) void weight_kernel(const NormArgs a, const float* rows,
                                                               int32_t n) {
  __shared__ f32x4v lds[3][SLICES][LANES];
  const int32_t col = 4 * (int32_t)(blockIdx.x * LANES + threadIdx.x % LANES);
  f32x4v s[3];
  sum_rows(rows, n, a.dim, col, s, lds);
  if (threadIdx.x >= LANES || col >= a.dim) return;
  put4(a.d_weight, a.param_type, col, s[0]);
  put4(a.d_bias, a.param_type, col, s[1]);
  put4(a.d_post_weight, a.param_type, col, s[2]);
}

int64_t partial_rows(const NormArgs& a) {
  const NormTeam t = norm_team(a.dim);
  const int64_t teams = whole_group(t.team) ? 1 : kNormGroup / t.team;
  return (int64_t)a.frames * (a.joined ? a.units / teams : a.units);
}

// Workgroups along the columns of a sum, and the shares of `n` rows, 1: added in one go.
uint32_t wide_of(const NormArgs& a) { return (uint32_t)((a.dim / 4 + LANES - 1) / LANES); }
int32_t shares_of(int64_t n) {
  return n < MIN_SHARED ? 1 : (int32_t)std::min<int64_t>(MAX_SHARES, (n + SLICES - 1) / SLICES);
}

struct Backward {
  const NormArgs& a;
  hipStream_t stream;
  template <typename S, typename Y, int TEAM, int V>
  hipError_t run() {
    constexpr int TEAMS = whole_group(TEAM) ? 1 : kNormGroup / TEAM;
    const int64_t units = (int64_t)a.frames * a.units;
    const dim3 grid((uint32_t)((units + TEAMS - 1) / TEAMS));
    const dim3 block(whole_group(TEAM) ? norm_team(a.dim).threads : kNormGroup);
    if (norm_mode(a) == NORM_OF_X)
      backward_kernel<S, Y, TEAM, V, NORM_OF_X><<<grid, block, 0, stream>>>(a);
    else if (norm_mode(a) == NORM_STEP)
      backward_kernel<S, Y, TEAM, V, NORM_STEP><<<grid, block, 0, stream>>>(a);
    else
      backward_kernel<S, Y, TEAM, V, NORM_POST><<<grid, block, 0, stream>>>(a);
    return hipGetLastError();
  }
};

// Where the sums lie, in rows of three: a workgroup's or team's, the shares of each frame's,
// the frames' weighted for the weights, and shares of those.
struct Sums {
  bool direct, any, weights;
  int32_t per_frame, shares, weight_shares;
  int64_t shared, frames, weight_shared, rows;
};
Sums sums_of(const NormArgs& a) {
  Sums s = {};
  s.weights = a.d_weight || a.d_bias || a.d_post_weight;
  s.any = s.weights || a.d_gate || a.d_scale || a.d_shift;
  s.direct = a.units == 1;
  if (!s.any) return s;
  s.per_frame = (int32_t)(partial_rows(a) / a.frames);
  s.shares = s.direct || a.frames * (int64_t)wide_of(a) >= ENOUGH ? 1 : shares_of(s.per_frame);
  s.weight_shares = wide_of(a) >= ENOUGH ? 1 : shares_of(a.frames);
  s.shared = s.direct ? 0 : partial_rows(a);
  s.frames = s.shared + (s.shares > 1 ? (int64_t)s.shares * a.frames : 0);
  s.weight_shared = s.frames + (s.weights && a.frames > 1 ? a.frames : 0);
  s.rows = s.weight_shared + (s.weights && s.weight_shares > 1 ? s.weight_shares : 0);
  return s;
}

}  // namespace

int64_t norm_workspace(const NormArgs& a) { return sums_of(a).rows * 3 * a.dim * 4; }

hipError_t launch_norm_backward(const NormArgs& args, int32_t stream_type, int32_t block_type,
                                hipStream_t stream) {
  NormArgs a = args;
  const Sums s = sums_of(a);
  auto at = [&](int64_t row) { return args.partial + row * 3 * a.dim; };
  // Frames of few rows, one team each: their sums are whole in its registers.
  a.direct = s.direct && s.any;
  a.weights = s.weights;
  a.frame_sums = s.weights && a.frames > 1 ? at(s.frames) : nullptr;
  if (s.direct || !s.any) a.partial = nullptr;
  hipError_t e = norm_dispatch(stream_type, block_type, norm_team(a.dim), Backward{a, stream});
  const uint32_t wide = wide_of(a);
  const dim3 block(SLICES * LANES);
  if (e == hipSuccess && s.any && !s.direct) {
    if (s.shares > 1) {
      share_kernel<<<dim3((uint32_t)(a.frames * s.shares), wide), block, 0, stream>>>(
          a, a.partial, at(s.shared), s.per_frame, s.shares);
      if ((e = hipGetLastError()) != hipSuccess) return e;
    }
    frame_kernel<<<dim3((uint32_t)a.frames, wide), block, 0, stream>>>(
        a, s.shares > 1 ? at(s.shared) : a.partial, s.shares > 1 ? s.shares : s.per_frame);
    e = hipGetLastError();
  }
  if (e != hipSuccess || !a.frame_sums) return e;
  if (s.weight_shares > 1) {
    share_kernel<<<dim3((uint32_t)s.weight_shares, wide), block, 0, stream>>>(
        a, a.frame_sums, at(s.weight_shared), a.frames, s.weight_shares);
    if ((e = hipGetLastError()) != hipSuccess) return e;
  }
  weight_kernel<<<dim3(wide), block, 0, stream>>>(
      a, s.weight_shares > 1 ? at(s.weight_shared) : a.frame_sums,
      s.weight_shares > 1 ? s.weight_shares : a.frames);
  return hipGetLastError();
}

}  // namespace lvsa
