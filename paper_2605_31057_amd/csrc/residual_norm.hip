// residual_norm.hip -- the step between two blocks on the residual stream, forward
// (residual_norm.h has the formulas).
//
// Bound: memory, x and y in, r and h out.  A team of 16, 64, 256 or 1024 threads holds a
// row in registers (at most 32 columns a thread), so every element is read once and
// written once whatever norms are taken; mean and variance are two passes over the
// registers, in fp32.  Parameters stay in registers over a unit's rows, which are of one
// frame.
#include "residual_norm.h"

namespace lvsa {
namespace {

template <typename S, typename Y, int TEAM, int V, int MODE>
__global__ __launch_bounds__(kNormThreads<TEAM>) void forward_kernel(const NormArgs a) {
  constexpr int TEAMS = kNormThreads<TEAM> / TEAM;
  __shared__ float lds[kNormSumLds<TEAM>];
  int turn = 0;
  const int t = threadIdx.x % TEAM;
  const int64_t id = (int64_t)blockIdx.x * TEAMS + threadIdx.x / TEAM;
  if (id >= (int64_t)a.frames * a.units) return;
  const NormUnit u = norm_unit(a, id);
  if (u.lo >= u.hi) return;
  const float inv_dim = 1.f / (float)a.dim;

  bool ok[V];
  float g[V][8], m[V][8], c[V][8];
#pragma unroll
  for (int v = 0; v < V; ++v) {
    const int32_t col = 8 * (t + TEAM * v);
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

  for (int64_t i = u.lo; i < u.hi; ++i) {
    float x[V][8], y[V][8];
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const int64_t col = 8 * (t + TEAM * v);
#pragma unroll
      for (int k = 0; k < 8; ++k) x[v][k] = y[v][k] = 0.f;
      if (!ok[v]) continue;
      load8((const S*)a.x + i * a.x_st + col, x[v]);
      if (MODE != NORM_OF_X) load8((const Y*)a.y + i * a.y_st + col, y[v]);
    }
    if constexpr (MODE != NORM_OF_X) {
      if constexpr (MODE == NORM_POST)
        normalise<TEAM, V>(y, ok, a.post, inv_dim, a.eps, lds, turn);
#pragma unroll
      for (int v = 0; v < V; ++v) {
        if (!ok[v]) continue;
#pragma unroll
        for (int k = 0; k < 8; ++k) x[v][k] = __builtin_fmaf(g[v][k], y[v][k], a.a * x[v][k]);
        store8((S*)a.r + i * a.r_st + 8 * (t + TEAM * v), x[v]);
      }
    }
    if (a.norm == LVSA_NORM_NONE) continue;
    normalise<TEAM, V>(x, ok, a.norm, inv_dim, a.eps, lds, turn);
#pragma unroll
    for (int v = 0; v < V; ++v) {
      if (!ok[v]) continue;
#pragma unroll
      for (int k = 0; k < 8; ++k) x[v][k] = __builtin_fmaf(x[v][k], m[v][k], c[v][k]);
      store8((Y*)a.h + i * a.h_st + 8 * (t + TEAM * v), x[v]);
    }
  }
}

struct Forward {
  const NormArgs& a;
  hipStream_t stream;
  template <typename S, typename Y, int TEAM, int V>
  hipError_t run() {
    constexpr int TEAMS = kNormThreads<TEAM> / TEAM;
    const int64_t units = (int64_t)a.frames * a.units;
    const dim3 grid((uint32_t)((units + TEAMS - 1) / TEAMS)), block(kNormThreads<TEAM>);
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

// Forward: workgroups for every compute unit several times over.  Backward: fewer, as
// each leaves partial sums.
void norm_units(NormArgs& a, bool backward) {
  const NormTeam t = norm_team(a.dim);
  const int64_t teams = t.threads < 256 ? 256 / t.threads : 1;
  const int64_t target = (backward ? 1024 : 2048) * teams;
  int64_t units = target * a.frame / a.n;
  units = units < 1 ? 1 : units > a.frame ? a.frame : units;
  a.joined = backward && teams > 1 && a.frame >= 4 * teams;
  if (a.joined) units = (units + teams - 1) / teams * teams;
  a.per = (int32_t)((a.frame + units - 1) / units);
  if (!a.joined) units = (a.frame + a.per - 1) / a.per;
  a.units = (int32_t)units;
}

}  // namespace lvsa
