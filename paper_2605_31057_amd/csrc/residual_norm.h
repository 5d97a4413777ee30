// residual_norm.h -- what the kernels of the residual step and their launches share.
//
//   u = y^ * post_weight,  y^ = P(y)            (P: layer norm, RMS norm or nothing)
//   r = a x + gate * u
//   h = (r^ * weight + bias) * (1 + scale) + shift,  r^ = N(r)
//
// gate, scale and shift have a row for every `frame` tokens.  A thread works the same
// eight columns of every row it takes, so what it needs of the parameters it holds in
// registers as long as the frame stays: G = gate * post_weight, and h = r^ * M + C with
// M = weight * (1 + scale), C = bias * (1 + scale) + shift.
//
// Backward, from dr (of r, by the residual path) and dh:
//   A_f = sum dh * r^,  B_f = sum dh            over a frame's rows
//   dscale_f = weight A_f + bias B_f,  dshift_f = B_f
//   dweight = sum_f (1 + scale_f) A_f,  dbias = sum_f (1 + scale_f) B_f
//   e = dr + rstd (dh M - mean(dh M) - r^ mean(dh M r^))      (RMS: without the mean)
//   dx = a e,  C_f = sum e * y^,  dgate_f = post_weight C_f,
//   dpost_weight = sum_f gate_f C_f,  dy = the same of P with e G in dh M's place
// so three sums a frame give the six gradients of parameters.
#pragma once

#include "values.h"

namespace lvsa {

struct NormArgs {
  int32_t n, dim, frame, frames;   // rows, columns, rows of a frame
  int32_t norm, post, param_type;
  float eps, a;
  const void* gate;
  const void* scale;
  const void* shift;
  int64_t gate_st, scale_st, shift_st;
  const void* weight;
  const void* bias;
  const void* post_weight;
  // forward: x, y -> r, h.  backward: r, y, gh, gr -> gx, gy.
  const void* x;
  const void* y;
  const void* gh;
  const void* gr;
  void* r;
  void* h;
  int64_t x_st, y_st, gh_st, gr_st, r_st, h_st;
  // Rows are shared out in units: `units` of a frame, `per` rows each.
  int32_t units, per;
  // backward: partial sums [unit or joined units][3][dim], and where they go.
  float* partial;
  float* frame_sums;               // [frames][3][dim], weighted for the weights' gradients
  int32_t joined;                  // the teams of a workgroup share a partial sum
  void* d_gate;
  void* d_scale;
  void* d_shift;
  void* d_weight;
  void* d_bias;
  void* d_post_weight;
};

hipError_t launch_norm_forward(const NormArgs& a, int32_t stream_type, int32_t block_type,
                               hipStream_t stream);
hipError_t launch_norm_backward(const NormArgs& a, int32_t stream_type, int32_t block_type,
                                hipStream_t stream);
// Sets a's units for a pass over its rows (backward: with sums of columns).
void norm_units(NormArgs& a, bool backward);
int64_t norm_workspace(const NormArgs& a);

// Threads that work a row, and eights of columns of each.
struct NormTeam {
  int32_t threads, eights;
};
inline NormTeam norm_team(int32_t dim) {
  const int32_t c8 = dim / 8;
  if (c8 <= 16) return {16, 1};
  if (c8 <= 256) return {64, (c8 + 63) / 64};
  if (c8 <= 1024) return {256, c8 <= 512 ? 2 : (c8 + 255) / 256};
  return {1024, 4};
}
constexpr int32_t kMaxNormDim = 1024 * 4 * 8;

// Eight parameters from element i on, as floats (`none` without them).
__device__ __forceinline__ void load_param(const void* p, int32_t type, int64_t i, float none,
                                           float (&x)[8]) {
  if (!p) {
#pragma unroll
    for (int k = 0; k < 8; ++k) x[k] = none;
  } else if (type == LVSA_F32) {
    load8((const float*)p + i, x);
  } else if (type == LVSA_BF16) {
    load8((const __bf16*)p + i, x);
  } else {
    load8((const _Float16*)p + i, x);
  }
}
__device__ __forceinline__ void store_param(void* p, int32_t type, int64_t i,
                                            const float (&x)[8]) {
  if (type == LVSA_F32)
    store8((float*)p + i, x);
  else if (type == LVSA_BF16)
    store8((__bf16*)p + i, x);
  else
    store8((_Float16*)p + i, x);
}

// Sums of K values over a team of TEAM threads (consecutive ones of the workgroup),
// the same in each of them; teams of more than a wave are the whole workgroup.
// `turn` alternates from call to call, so one barrier a call is enough: a wave writes
// a buffer again only past the barrier of the call between.
template <int TEAM, int K>
__device__ __forceinline__ void team_sum(float (&v)[K], float* lds, int& turn) {
#pragma unroll
  for (int k = 0; k < K; ++k)
#pragma unroll
    for (int d = (TEAM < 64 ? TEAM : 64) / 2; d; d /= 2) v[k] += __shfl_xor(v[k], d);
  if constexpr (TEAM > 64) {
    constexpr int WAVES = TEAM / 64;
    float* const at = lds + turn * (WAVES * 4);
    turn ^= 1;
    if (threadIdx.x % 64 == 0) {
#pragma unroll
      for (int k = 0; k < K; ++k) at[threadIdx.x / 64 * 4 + k] = v[k];
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < K; ++k) {
      v[k] = 0.f;
      for (int w = 0; w < WAVES; ++w) v[k] += at[w * 4 + k];
    }
  }
}

template <int TEAM>
constexpr int kNormThreads = TEAM > 256 ? TEAM : 256;
template <int TEAM>
constexpr int kNormSumLds = TEAM > 64 ? 2 * 4 * TEAM / 64 : 1;

// The rows of unit `id`: frame f, rows lo .. hi - 1 (none where the frame has fewer).
struct NormUnit {
  int32_t f, lo, hi;
};
__device__ __forceinline__ NormUnit norm_unit(const NormArgs& a, int64_t id) {
  NormUnit u;
  u.f = (int32_t)(id / a.units);
  const int64_t first = (int64_t)u.f * a.frame;
  const int64_t end = first + a.frame < a.n ? first + a.frame : a.n;
  const int64_t lo = first + (id - (int64_t)u.f * a.units) * a.per;
  u.lo = (int32_t)(lo < end ? lo : end);
  u.hi = (int32_t)(lo + a.per < end ? lo + a.per : end);
  return u;
}

// x becomes normalised over the row's `dim` columns, of which this thread has those
// of `ok`; returns the factor 1 / sqrt(var + eps).  The RMS norm takes the mean too and
// multiplies it by 0: with a branch around it the compiler (clang 20, ROCm 7.2) lost the
// columns of the thread's second eight on one side of it, and a sum over a team costs little
// beside the row's way from memory.
template <int TEAM, int V>
__device__ __forceinline__ float normalise(float (&x)[V][8], const bool (&ok)[V], int32_t kind,
                                           float inv_dim, float eps, float* lds, int& turn) {
  float s[1] = {0.f};
#pragma unroll
  for (int v = 0; v < V; ++v)
#pragma unroll
    for (int k = 0; k < 8; ++k) s[0] += x[v][k];   // columns it does not have hold 0
  team_sum<TEAM>(s, lds, turn);
  const float mean = kind == LVSA_NORM_LAYER ? s[0] * inv_dim : 0.f;
#pragma unroll
  for (int v = 0; v < V; ++v)
#pragma unroll
    for (int k = 0; k < 8; ++k) x[v][k] = ok[v] ? x[v][k] - mean : 0.f;
  s[0] = 0.f;
#pragma unroll
  for (int v = 0; v < V; ++v)
#pragma unroll
    for (int k = 0; k < 8; ++k) s[0] = __builtin_fmaf(x[v][k], x[v][k], s[0]);
  team_sum<TEAM>(s, lds, turn);
  const float factor = 1.f / __builtin_sqrtf(__builtin_fmaf(s[0], inv_dim, eps));
#pragma unroll
  for (int v = 0; v < V; ++v)
#pragma unroll
    for (int k = 0; k < 8; ++k) x[v][k] *= factor;
  return factor;
}

// Gradient of what normalise() took, in place of that of what it gave: `unit` is that,
// `factor` what it returned.
template <int TEAM, int V>
__device__ __forceinline__ void normalise_back(float (&g)[V][8], const float (&unit)[V][8],
                                               const bool (&ok)[V], int32_t kind, float factor,
                                               float inv_dim, float* lds, int& turn) {
  float s[2] = {0.f, 0.f};
#pragma unroll
  for (int v = 0; v < V; ++v)
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      s[0] = __builtin_fmaf(g[v][k], unit[v][k], s[0]);
      s[1] += g[v][k];
    }
  team_sum<TEAM>(s, lds, turn);
  const float along = s[0] * inv_dim, mean = kind == LVSA_NORM_LAYER ? s[1] * inv_dim : 0.f;
#pragma unroll
  for (int v = 0; v < V; ++v)
#pragma unroll
    for (int k = 0; k < 8; ++k)
      g[v][k] = ok[v] ? factor * (g[v][k] - mean - unit[v][k] * along) : 0.f;
}

// What a launch has of a block's output: nothing, y, or y and a norm of it.
enum NormMode { NORM_OF_X = 0, NORM_STEP = 1, NORM_POST = 2 };
inline NormMode norm_mode(const NormArgs& a) {
  return !a.y ? NORM_OF_X : a.post == LVSA_NORM_NONE ? NORM_STEP : NORM_POST;
}

// Calls fn.run<S, Y, TEAM, V>() for a launch's types and team.
template <typename S, typename Y, typename F>
hipError_t norm_dispatch_team(const NormTeam& t, F&& fn) {
  if (t.threads == 16) return fn.template run<S, Y, 16, 1>();
  if (t.threads == 64) {
    if (t.eights == 1) return fn.template run<S, Y, 64, 1>();
    if (t.eights == 2) return fn.template run<S, Y, 64, 2>();
    if (t.eights == 3) return fn.template run<S, Y, 64, 3>();
    return fn.template run<S, Y, 64, 4>();
  }
  if (t.threads == 256) {
    if (t.eights == 2) return fn.template run<S, Y, 256, 2>();
    if (t.eights == 3) return fn.template run<S, Y, 256, 3>();
    return fn.template run<S, Y, 256, 4>();
  }
  return fn.template run<S, Y, 1024, 4>();
}
template <typename F>
hipError_t norm_dispatch(int32_t stream_type, int32_t block_type, const NormTeam& t, F&& fn) {
  if (stream_type == LVSA_BF16) return norm_dispatch_team<__bf16, __bf16>(t, fn);
  if (stream_type == LVSA_F16) return norm_dispatch_team<_Float16, _Float16>(t, fn);
  if (block_type == LVSA_BF16) return norm_dispatch_team<float, __bf16>(t, fn);
  if (block_type == LVSA_F16) return norm_dispatch_team<float, _Float16>(t, fn);
  return norm_dispatch_team<float, float>(t, fn);
}

}  // namespace lvsa
