// values.h -- element types, e4m3 conversions and rotary positions shared by the
// rotary, cache and cache-attention kernels.
#pragma once

#include "internal.h"

namespace lvsa {

typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4v __attribute__((ext_vector_type(4)));

// Eight elements of a row, as floats; 16 or 32 bytes, aligned to 16.
template <typename T>
__device__ __forceinline__ void load8(const T* p, float (&x)[8]) {
  if constexpr (sizeof(T) == 4) {
    const f32x4v a = *(const f32x4v*)p, b = *(const f32x4v*)(p + 4);
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = a[i], x[4 + i] = b[i];
  } else {
    typedef T t8 __attribute__((ext_vector_type(8)));
    const t8 a = *(const t8*)p;
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = (float)a[i];
  }
}

// Stores eight floats, rounded to nearest even.
template <typename T>
__device__ __forceinline__ void store8(T* p, const float (&x)[8]) {
  if constexpr (sizeof(T) == 4) {
    *(f32x4v*)p = f32x4v{x[0], x[1], x[2], x[3]};
    *(f32x4v*)(p + 4) = f32x4v{x[4], x[5], x[6], x[7]};
  } else {
    typedef T t8 __attribute__((ext_vector_type(8)));
    t8 a;
#pragma unroll
    for (int i = 0; i < 8; ++i) a[i] = (T)x[i];
    *(t8*)p = a;
  }
}

// What the rotation of a token needs: its position on the grid, and where the
// table's three parts begin.
struct RopeArgs {
  const float* table;        // (cos, sin) entries; null: no rotation
  int32_t grid;              // tokens of the grid
  int32_t plane, width;      // tokens of a frame, of a row
  int32_t p0, p01, p012;     // pairs of the frame axis, of it and the rows, of all three
  int32_t at_row, at_col;    // first entries of the row and column parts
  int32_t halves;
};

// The table rows of one token: the entry of pair j is at base[axis of j] + j.
struct TokenTurn {
  int32_t t, y, x;
  bool turns;
};
__device__ __forceinline__ TokenTurn token_turn(const RopeArgs& r, int32_t token) {
  TokenTurn k;
  k.turns = token < r.grid;
  const int32_t t = token / r.plane, in = token - t * r.plane;
  const int32_t y = in / r.width, x = in - y * r.width;
  k.t = t * r.p0;
  k.y = r.at_row + y * (r.p01 - r.p0) - r.p0;
  k.x = r.at_col + x * (r.p012 - r.p01) - r.p01;
  return k;
}
// Whether pair j of the token turns.
__device__ __forceinline__ bool pair_turns(const RopeArgs& r, const TokenTurn& k, int j) {
  return k.turns && j < r.p012;
}
// (cos, sin) of a pair j that turns.
__device__ __forceinline__ f32x2 turn_of(const RopeArgs& r, const TokenTurn& k, int j) {
  const int32_t e = j + (j < r.p0 ? k.t : j < r.p01 ? k.y : k.x);
  return *(const f32x2*)(r.table + 2 * (int64_t)e);
}

// A row is worked by eight threads: thread c holds elements 8c .. 8c+7 (lo) and
// 64+8c .. 64+8c+7 (hi), which is whole pairs in either layout.  The (cos, sin) of
// its eight pairs, and which of them turn: the others keep their values as they are (times
// (1, 0) an infinity would make its partner NaN).
struct Turns {
  f32x2 cs[8];
  bool on[8];
};
__device__ __forceinline__ void load_turns(const RopeArgs& r, int32_t token, int c, Turns& turns) {
  const TokenTurn k = token_turn(r, token);
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int j = r.halves ? 8 * c + i : i < 4 ? 4 * c + i : 32 + 4 * c + i - 4;
    turns.on[i] = pair_turns(r, k, j);
    turns.cs[i] = turns.on[i] ? turn_of(r, k, j) : f32x2{1.f, 0.f};
  }
}
// F: the type of the arithmetic (float or double).  sign -1: the opposite angles.
template <typename F>
__device__ __forceinline__ void turn_pair(float& a, float& b, f32x2 cs, bool on, float sign) {
  if (!on) return;
  const F x = a, y = b, c = cs[0], s = sign * cs[1];
  if constexpr (sizeof(F) == 8) {
    a = (float)(x * c - y * s);
    b = (float)(x * s + y * c);
  } else {
    a = __builtin_fmaf(x, c, -(y * s));
    b = __builtin_fmaf(x, s, y * c);
  }
}
template <typename F>
__device__ __forceinline__ void rotate16(float (&lo)[8], float (&hi)[8], const Turns& t,
                                         bool halves, float sign) {
  if (halves) {
#pragma unroll
    for (int i = 0; i < 8; ++i) turn_pair<F>(lo[i], hi[i], t.cs[i], t.on[i], sign);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      turn_pair<F>(lo[2 * i], lo[2 * i + 1], t.cs[i], t.on[i], sign);
      turn_pair<F>(hi[2 * i], hi[2 * i + 1], t.cs[4 + i], t.on[4 + i], sign);
    }
  }
}

// e4m3 bytes of four floats within +-448 (or NaN).
__device__ __forceinline__ uint32_t to_e4m3(float a, float b, float c, float d) {
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
}
// The four floats of a word of e4m3 bytes.
__device__ __forceinline__ void from_e4m3(uint32_t w, float (&x)[4]) {
  const f32x2 a = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false);
  const f32x2 b = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
  x[0] = a[0], x[1] = a[1], x[2] = b[0], x[3] = b[1];
}

// Exponent e of a block's scale 2^e: the least e >= -117 with most <= 448 * 2^e, at
// most 119 (448 * 2^119 is the largest such product that fp32 and bf16 hold).
// With most = m * 2^E, 1 <= m < 2, and 448 = 1.75 * 2^8 this is E - 8, one more
// where m > 1.75: adding 2^23 - 1 - (mantissa of 1.75) to the bits carries into
// the exponent exactly then.
__device__ __forceinline__ int scale_exponent(float most) {
  const uint32_t carried = __float_as_uint(most) + (0x7FFFFFu - 0x600000u);
  return min(max((int)(carried >> 23) - 127 - 8, -117), 119);
}
__device__ __forceinline__ float pow2(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }

// Place of a token in its 64-token V tile (lvsa.h).
__host__ __device__ __forceinline__ int v_place(int token) {
  return ((token >> 2) & 3) * 16 + ((token >> 4) & 3) * 4 + (token & 3);
}

// 4x4 byte transpose: byte i of w[j] becomes byte j of w[i].
__device__ __forceinline__ void transpose4(uint32_t (&w)[4]) {
  const uint32_t a = __builtin_amdgcn_perm(w[1], w[0], 0x05010400u);   // w0.0 w1.0 w0.1 w1.1
  const uint32_t b = __builtin_amdgcn_perm(w[1], w[0], 0x07030602u);   // w0.2 w1.2 w0.3 w1.3
  const uint32_t c = __builtin_amdgcn_perm(w[3], w[2], 0x05010400u);
  const uint32_t d = __builtin_amdgcn_perm(w[3], w[2], 0x07030602u);
  w[0] = __builtin_amdgcn_perm(c, a, 0x05040100u);
  w[1] = __builtin_amdgcn_perm(c, a, 0x07060302u);
  w[2] = __builtin_amdgcn_perm(d, b, 0x05040100u);
  w[3] = __builtin_amdgcn_perm(d, b, 0x07060302u);
}

}  // namespace lvsa
