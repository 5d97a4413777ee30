// residual_norm.hip -- the step between two blocks on the residual stream, forward
// (residual_norm.h has the formulas).
//
// Bound: memory, x and y in, r and h out: 32,760 rows of 1,536 columns in bf16 79 us, 5.1 TB/s
// (a 1 GiB copy reaches 5.0).  A team of threads holds a row in registers, eight columns a
// thread, so every element is read once and written once whatever norms are taken, and the
// next row is loaded meanwhile.  (32 columns a thread, fewer threads a row: 90 us.)
// Parameters stay in registers over a unit's rows, which are of one frame.
#include <algorithm>

#include "residual_norm.h"

namespace lvsa {
namespace {

template <typename S, typename Y, int TEAM, int V, int MODE>
__global__ __launch_bounds__(norm_bound(TEAM)) void forward_kernel(const NormArgs a) {
  __shared__ StatsLds lds;
  int turn = 0;
  constexpr bool GROUP = whole_group(TEAM);
  const int team = GROUP ? (int)blockDim.x : TEAM, teams = GROUP ? 1 : kNormGroup / TEAM;
  const int t = GROUP ? threadIdx.x : threadIdx.x % TEAM;
  const int64_t id = (int64_t)blockIdx.x * teams + (GROUP ? 0 : threadIdx.x / TEAM);
  if (id >= (int64_t)a.frames * a.units) return;
  const NormUnit u = norm_unit(a, id);
  if (u.lo >= u.hi) return;
  const float inv_dim = 1.f / (float)a.dim;

  bool ok[V];
  float g[V][8], m[V][8], c[V][8];
#pragma unroll
  for (int v = 0; v < V; ++v) {
    const int32_t col = 8 * (t + team * v);
    ok[v] = col < a.dim;
    if (!ok[v]) continue;
    float p[8], s[8];
    load_param(a.gate, a.param_type, (int64_t)u.f * a.gate_st + col, 1.f, g[v]);
    load_param(a.post_weight, a.param_type, col, 1.f, p);
    load_param(a.weight, a.param_type, col, 1.f, m[v]);
    load_param(a.bias, a.param_type, col, 0.f, c[v]);
#pragma unroll
    for (int k = 0; k < 8; ++k) g[v][k] *= p[k];
    load_param(a.scale, a.param_type, (int64_t)u.f * a.scale_st + col, 0.f, s);
    load_param(a.shift, a.param_type, (int64_t)u.f * a.shift_st + col, 0.f, p);
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      m[v][k] *= 1.f + s[k];
      c[v][k] = __builtin_fmaf(c[v][k], 1.f + s[k], p[k]);
    }
  }

  Raw8<S> rx[V];
  Raw8<Y> ry[V];
#pragma unroll
  for (int v = 0; v < V; ++v) rx[v].v = 0, ry[v].v = 0;
  auto load_row = [&](int64_t i) {
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const int64_t col = 8 * (t + team * v);
      if (!ok[v]) continue;
      rx[v].load((const S*)a.x + i * a.x_st + col);
      if (MODE != NORM_OF_X) ry[v].load((const Y*)a.y + i * a.y_st + col);
    }
  };
  load_row(u.lo);
  for (int64_t i = u.lo; i < u.hi; ++i) {
    float x[V][8], y[V][8];
#pragma unroll
    for (int v = 0; v < V; ++v) {
      rx[v].get(x[v]);
      ry[v].get(y[v]);
    }
    if (i + 1 < u.hi) load_row(i + 1);
    if constexpr (MODE != NORM_OF_X) {
      if constexpr (MODE == NORM_POST) {
        const RowStats r =
            row_stats<TEAM, V, false>(y, y, ok, a.post, inv_dim, a.dim, a.eps, &lds, turn);
#pragma unroll
        for (int v = 0; v < V; ++v)
#pragma unroll
          for (int k = 0; k < 8; ++k) y[v][k] = (y[v][k] - r.mean) * r.factor;
      }
#pragma unroll
      for (int v = 0; v < V; ++v) {
        if (!ok[v]) continue;
#pragma unroll
        for (int k = 0; k < 8; ++k) x[v][k] = __builtin_fmaf(g[v][k], y[v][k], a.a * x[v][k]);
        store8((S*)a.r + i * a.r_st + 8 * (t + team * v), x[v]);
      }
    }
    if (a.norm == LVSA_NORM_NONE) continue;
    const RowStats r =
        row_stats<TEAM, V, false>(x, x, ok, a.norm, inv_dim, a.dim, a.eps, &lds, turn);
#pragma unroll
    for (int v = 0; v < V; ++v) {
      if (!ok[v]) continue;
#pragma unroll
      for (int k = 0; k < 8; ++k)
        x[v][k] = __builtin_fmaf((x[v][k] - r.mean) * r.factor, m[v][k], c[v][k]);
      store8((Y*)a.h + i * a.h_st + 8 * (t + team * v), x[v]);
    }
  }
}

struct Forward {
  const NormArgs& a;
  hipStream_t stream;
  template <typename S, typename Y, int TEAM, int V>
  hipError_t run() {
    constexpr int TEAMS = whole_group(TEAM) ? 1 : kNormGroup / TEAM;
    const int64_t units = (int64_t)a.frames * a.units;
    const dim3 grid((uint32_t)((units + TEAMS - 1) / TEAMS));
    const dim3 block(whole_group(TEAM) ? norm_team(a.dim).threads : kNormGroup);
    if (norm_mode(a) == NORM_OF_X)
      forward_kernel<S, Y, TEAM, V, NORM_OF_X><<<grid, block, 0, stream>>>(a);
    else if (norm_mode(a) == NORM_STEP)
      forward_kernel<S, Y, TEAM, V, NORM_STEP><<<grid, block, 0, stream>>>(a);
    else
      forward_kernel<S, Y, TEAM, V, NORM_POST><<<grid, block, 0, stream>>>(a);
    return hipGetLastError();
  }
};

}  // namespace

hipError_t launch_norm_forward(const NormArgs& a, int32_t stream_type, int32_t block_type,
                               hipStream_t stream) {
  return norm_dispatch(stream_type, block_type, norm_team(a.dim), Forward{a, stream});
}

// Forward a team takes ROWS_FORWARD rows (fewer where that leaves compute units idle), so
// what is worked at one time lies together in memory: 32,760 rows of 1,536 columns 79 us, with
// 8 rows 84, 12 rows 87, all rows shared out evenly to what fits at once 86, and dealt out to
// it in turn 94.  Back, where a team leaves a row of three sums, there are as many as fit at
// once: 12 waves on each of 256 compute units, on any device, as the sums' order follows from
// it (these rows 140 us; 24 waves 145; in turn 146).
constexpr int64_t ROWS_FORWARD = 4;
void norm_units(NormArgs& a, bool backward) {
  const NormTeam t = norm_team(a.dim);
  const int64_t teams = whole_group(t.team) ? 1 : kNormGroup / t.team;
  const int64_t waves = whole_group(t.team) ? t.threads / 64 : kNormGroup / 64;
  const int64_t target = 256 * std::max<int64_t>(1, 12 / waves) * teams;
  // Frames are alike but for the last, which may be shorter.
  const int64_t rows =
      std::min(ROWS_FORWARD, std::max<int64_t>(1, a.n / (256 * teams)));
  int64_t units = backward ? target * a.frame / a.n : (a.frame + rows - 1) / rows;
  units = std::min<int64_t>(std::max<int64_t>(1, units), a.frame);
  a.joined = backward && teams > 1 && a.frame >= 4 * teams;
  if (a.joined) units = (units + teams - 1) / teams * teams;
  a.per = (int32_t)((a.frame + units - 1) / units);
  if (!a.joined) units = (a.frame + a.per - 1) / a.per;
  a.units = (int32_t)units;
}

}  // namespace lvsa
