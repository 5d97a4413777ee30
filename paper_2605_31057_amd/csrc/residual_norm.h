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
  int32_t direct;                  // a frame is one unit, its gradients need no partial sums
  int32_t weights;                 // gradients of weight, bias or post_weight are wanted
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

// Threads that work a row: 16, 32 or 64 of a workgroup of 256, or the whole workgroup of at most
// 768 or 1024 (`team`), eight columns each, past 8192 columns sixteen.  The bound is also one
// on registers, 168 or 128 a thread; the gradients of a stream in 32 bits take 148 (with 128
// they spill: 32,760 rows of 5,120 columns 692 us against 654).
struct NormTeam {
  int32_t team, threads, eights;
};
inline NormTeam norm_team(int32_t dim) {
  const int32_t c8 = dim / 8, threads = (c8 + 63) / 64 * 64;
  if (c8 <= 16) return {16, 16, 1};
  if (c8 <= 32) return {32, 32, 1};
  if (c8 <= 64) return {64, 64, 1};
  if (threads <= 768) return {768, threads, 1};
  if (c8 <= 1024) return {1024, threads, 1};
  return {1024, 1024, 2};
}
inline __host__ __device__ constexpr bool whole_group(int team) { return team > 64; }
inline __host__ __device__ constexpr int norm_bound(int team) { return team > 64 ? team : 256; }
constexpr int kNormGroup = 256;   // threads of a workgroup of several teams

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

// Eight elements as they are in memory: a row's are loaded while the row before is worked.
template <typename T>
struct Raw8 {
  typedef T t8 __attribute__((ext_vector_type(8)));
  t8 v;
  __device__ __forceinline__ void load(const T* p) {
    if constexpr (sizeof(T) == 4) {
      const f32x4v a = *(const f32x4v*)p, b = *(const f32x4v*)(p + 4);
      v = __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
    } else {
      v = *(const t8*)p;
    }
  }
  __device__ __forceinline__ void get(float (&x)[8]) const {
#pragma unroll
    for (int k = 0; k < 8; ++k) x[k] = (float)v[k];
  }
};

// x plus its value in another lane of the same 16: CTRL a DPP control.
template <int CTRL>
__device__ __forceinline__ float add_dpp(float x) {
  return x + __uint_as_float(
                 __builtin_amdgcn_update_dpp(0, __float_as_uint(x), CTRL, 0xF, 0xF, true));
}
// Sum over 16 consecutive lanes, the same in each: pairs and quads by quad_perm, then
// mirrored halves and rows.
__device__ __forceinline__ float sum16(float x) {
  x = add_dpp<0xB1>(x);    // quad_perm [1 0 3 2]
  x = add_dpp<0x4E>(x);    // quad_perm [2 3 0 1]
  x = add_dpp<0x141>(x);   // row_half_mirror
  return add_dpp<0x140>(x);   // row_mirror
}
// Over 32, and over the wave: rows of 16 by swaps, [x0 x0 x2 x2] + [x1 x1 x3 x3], then halves.
__device__ __forceinline__ float sum32(float x) {
  x = sum16(x);
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false,
                                                  false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
__device__ __forceinline__ float sum64(float x) {
  x = sum32(x);
  const auto s = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false,
                                                  false);
  return __uint_as_float(s[0]) + __uint_as_float(s[1]);
}
template <int TEAM>
__device__ __forceinline__ float sum_team_wave(float x) {
  return TEAM == 16 ? sum16(x) : TEAM == 32 ? sum32(x) : sum64(x);
}

// What a row's norm and its gradient need of the whole row: mean (0 for the RMS norm),
// factor = 1 / sqrt(mean square of the deviations + eps), and of a gradient g of the
// normalised row u its mean and the mean of g u.
struct RowStats {
  float mean, factor, g_mean, gu_mean;
};
// LDS of a workgroup that is one team: five sums a wave, in two buffers that alternate, so
// one barrier a call is enough (a wave writes a buffer again only past the barrier of the
// call between).
struct StatsLds {
  float v[2][16][8];
};

// RowStats of x (and g, BACK).  Columns a thread does not have hold 0 in both; `count`:
// columns it has.  Deviations are taken from the wave's own mean before they are squared or
// multiplied, and the waves' results put together about the row's mean,
//   sum (x - m)^2 = sum_w [sum (x - m_w)^2 + n_w (m_w - m)^2],
//   sum g (x - m) = sum_w [sum g (x - m_w) + (m_w - m) sum g],
// so a mean far larger than the deviations costs nothing, and waves meet once.
template <int TEAM, int V, bool BACK>
__device__ __forceinline__ RowStats row_stats(const float (&x)[V][8], const float (&g)[V][8],
                                              const bool (&ok)[V], int32_t kind, float inv_dim,
                                              int32_t dim, float eps, StatsLds* lds, int& turn) {
  constexpr int WAVE = whole_group(TEAM) ? 64 : TEAM;
  const bool layer = kind == LVSA_NORM_LAYER;
  float n = (float)dim;
  if constexpr (whole_group(TEAM)) {
    // Columns of this wave: eights 64 w .. 64 w + 63 of each of the V stretches.
    n = 0.f;
    for (int v = 0; v < V; ++v) {
      const int at = 8 * ((int)(threadIdx.x & ~63u) + (int)blockDim.x * v);
      n += (float)max(0, min(512, dim - at));
    }
  }
  float s = 0.f;
#pragma unroll
  for (int v = 0; v < V; ++v)
#pragma unroll
    for (int k = 0; k < 8; ++k) s += x[v][k];
  s = sum_team_wave<WAVE>(s);
  const float mean = layer ? s / fmaxf(n, 1.f) : 0.f;
  float m2 = 0.f, gs = 0.f, gx = 0.f;
#pragma unroll
  for (int v = 0; v < V; ++v)
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const float d = ok[v] ? x[v][k] - mean : 0.f;
      m2 = __builtin_fmaf(d, d, m2);
      if (BACK) {
        gx = __builtin_fmaf(g[v][k], d, gx);
        gs += g[v][k];
      }
    }
  m2 = sum_team_wave<WAVE>(m2);
  if (BACK) {
    gx = sum_team_wave<WAVE>(gx);
    gs = sum_team_wave<WAVE>(gs);
  }
  RowStats r = {mean, 0.f, 0.f, 0.f};
  if constexpr (whole_group(TEAM)) {
    const int wave = threadIdx.x / 64, waves = blockDim.x / 64, lane = threadIdx.x % 16;
    float(*const at)[8] = lds->v[turn];
    turn ^= 1;
    if (threadIdx.x % 64 == 0) {
      *(f32x4v*)at[wave] = f32x4v{n, mean, m2, gx};
      at[wave][4] = gs;
    }
    __syncthreads();
    // Lane w of every 16 takes wave w's.
    const f32x4v o = lane < waves ? *(const f32x4v*)at[lane] : f32x4v{};
    r.mean = sum16(o[0] * o[1]) * inv_dim;
    const float off = o[1] - r.mean;
    m2 = sum16(__builtin_fmaf(o[0] * off, off, o[2]));
    if (BACK) {
      const float og = lane < waves ? at[lane][4] : 0.f;
      gx = sum16(__builtin_fmaf(off, og, o[3]));
      gs = sum16(og);
    }
  }
  r.factor = 1.f / __builtin_sqrtf(__builtin_fmaf(m2, inv_dim, eps));
  if (BACK) {
    r.g_mean = layer ? gs * inv_dim : 0.f;
    r.gu_mean = gx * r.factor * inv_dim;
  }
  return r;
}

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

// What a launch has of a block's output: nothing, y, or y and a norm of it.
enum NormMode { NORM_OF_X = 0, NORM_STEP = 1, NORM_POST = 2 };
inline NormMode norm_mode(const NormArgs& a) {
  return !a.y ? NORM_OF_X : a.post == LVSA_NORM_NONE ? NORM_STEP : NORM_POST;
}

// Calls fn.run<S, Y, TEAM, V>() for a launch's types and team.
template <typename S, typename Y, typename F>
hipError_t norm_dispatch_team(const NormTeam& t, F&& fn) {
  if (t.team == 16) return fn.template run<S, Y, 16, 1>();
  if (t.team == 32) return fn.template run<S, Y, 32, 1>();
  if (t.team == 64) return fn.template run<S, Y, 64, 1>();
  if (t.team == 768) return fn.template run<S, Y, 768, 1>();
  if (t.eights == 1) return fn.template run<S, Y, 1024, 1>();
  return fn.template run<S, Y, 1024, 2>();
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
