// kv_cache.hip -- writing keys and values into the 8-bit cache, and reading them back.
//
// A block of B tokens of a head holds x as e4m3(x / 2^e) with one e (lvsa.h).
// Dividing by a power of two is exact, so the only rounding is the one to e4m3, a
// held value is exact in bf16, and raising e rounds again only what falls below
// e4m3's normal range.  V is held transposed in tiles of 64 tokens: the attention
// product P V then takes 16 bytes of consecutive k-slots a lane (lvsa.h's order of
// places is that of the accumulator registers that hold P).
//
// Bound: memory, sizeof(T) bytes read and one written an element: 40 heads of 32,760
// tokens, keys rotated, 209 us (4.8 TB/s); 16 heads of 103,862 tokens back in bf16 233 us
// (5.5 TB/s).  One workgroup a block, head and tensor (K or V): the block's values stay
// in registers between the maximum and the rounding, so they are read once.
#include "values.h"

namespace lvsa {
namespace {

constexpr int LDS_ROW = 136;        // bytes of a token's row in LDS, 8 more than its 128

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

struct WriteArgs {
  lvsa_kv_cache c;                  // n_tokens: held before
  const void* k;
  const void* v;
  int64_t k_sh, k_st, v_sh, v_st;
  int32_t start, n, first_block;
};

__device__ __forceinline__ float finite_abs(float x) {
  const float a = fabsf(x);
  return a < __builtin_inff() ? a : 0.f;   // NaN compares false
}

// The V tiles of a block (64 tokens each, at `tiles`) from or to token rows in LDS, four
// elements and 16 tokens a thread, transposed four bytes by four.
template <int B, int THREADS>
__device__ __forceinline__ void tiles_to_rows(const uint8_t* tiles, uint8_t* rows) {
#pragma unroll
  for (int at = threadIdx.x; at < B / 64 * 128; at += THREADS) {
    const int tile = at / 128, dq = at % 128 / 4, g = at % 4;
    u32x4 in[4];
#pragma unroll
    for (int j = 0; j < 4; ++j)
      in[j] = *(const u32x4*)(tiles + tile * 8192 + (4 * dq + j) * 64 + 16 * g);
#pragma unroll
    for (int kt = 0; kt < 4; ++kt) {
      uint32_t w[4] = {in[0][kt], in[1][kt], in[2][kt], in[3][kt]};
      transpose4(w);
#pragma unroll
      for (int j = 0; j < 4; ++j)
        *(uint32_t*)(rows + (tile * 64 + 16 * kt + 4 * g + j) * LDS_ROW + 4 * dq) = w[j];
    }
  }
}
template <int B, int THREADS>
__device__ __forceinline__ void rows_to_tiles(const uint8_t* rows, uint8_t* tiles) {
#pragma unroll
  for (int at = threadIdx.x; at < B / 64 * 128; at += THREADS) {
    const int tile = at / 128, dq = at % 128 / 4, g = at % 4;
    u32x4 out[4];
#pragma unroll
    for (int kt = 0; kt < 4; ++kt) {
      uint32_t w[4];
#pragma unroll
      for (int j = 0; j < 4; ++j)
        w[j] = *(const uint32_t*)(rows + (tile * 64 + 16 * kt + 4 * g + j) * LDS_ROW + 4 * dq);
      transpose4(w);
#pragma unroll
      for (int j = 0; j < 4; ++j) out[j][kt] = w[j];
    }
#pragma unroll
    for (int j = 0; j < 4; ++j)
      *(u32x4*)(tiles + tile * 8192 + (4 * dq + j) * 64 + 16 * g) = out[j];
  }
}

// Eight threads a row (values.h), two rows a thread.  Every load is issued before the
// first value is used and none depends on a lane's token: rows of the source are
// clamped to those that exist and chosen afterwards, so a block of a few new tokens
// waits for memory once: 7 us for one token into a held block of 12 heads, 8.8 us for
// 1,560 tokens (a branch a row and four rows a thread took 2 us longer in both).
template <typename T, int B>
__global__ __launch_bounds__(4 * B) void write_kernel(WriteArgs a, RopeArgs r) {
  constexpr int THREADS = 4 * B, ROWS = B / 2;
  __shared__ float most_lds[THREADS / 64];
  __shared__ __attribute__((aligned(16))) uint8_t bytes[B * LDS_ROW];
  const int block = a.first_block + blockIdx.x;
  const int64_t head = blockIdx.y;
  const bool is_v = blockIdx.z != 0;
  const int row = threadIdx.x / 8, c = threadIdx.x % 8;
  const lvsa_kv_cache& m = a.c;
  const int64_t base = head * m.capacity;              // the head's first place
  const int32_t token0 = block * B, end = a.start + a.n;
  float* const scale = (is_v ? m.v_scale : m.k_scale) + base / B + block;
  uint8_t* const k_rows = (uint8_t*)m.k + (base + token0) * 128;
  uint8_t* const v_tiles = (uint8_t*)m.v + (base + token0) / 64 * 8192;
  const T* const src = is_v ? (const T*)a.v + head * a.v_sh : (const T*)a.k + head * a.k_sh;
  const int64_t st = is_v ? a.v_st : a.k_st;
  const bool turn = !is_v && r.table;
  // Whether the block holds tokens that stay.
  const bool stays = token0 < min(a.start, m.n_tokens) || end < min(token0 + B, m.n_tokens);

  float lo[2][8], hi[2][8];
  Turns turns[2];
#pragma unroll
  for (int p = 0; p < 2; ++p) {
    const int32_t token = token0 + p * ROWS + row;
    const int32_t i = min(max(token - a.start, 0), a.n - 1);
    load8(src + i * st + 8 * c, lo[p]);
    load8(src + i * st + 64 + 8 * c, hi[p]);
    if (turn) load_turns(r, token, c, turns[p]);
  }
  u32x2 old[2][2];
  float old_scale = 0.f;
  if (stays) {
    old_scale = *scale;
    if (is_v) {
      tiles_to_rows<B, THREADS>(v_tiles, bytes);
      __syncthreads();
    }
#pragma unroll
    for (int p = 0; p < 2; ++p)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int at = p * ROWS + row, d = 64 * h + 8 * c;
        if (is_v)
          old[p][h] = *(const u32x2*)(bytes + at * LDS_ROW + d);
        else
          old[p][h] = *(const u32x2*)(k_rows + at * 128 + d);
      }
  }
  // The block's values: new tokens, held ones, zeros behind the last.
  float most = 0.f;
#pragma unroll
  for (int p = 0; p < 2; ++p) {
    const int32_t token = token0 + p * ROWS + row;
    const bool fresh = token >= a.start && token < end;
    if (turn) rotate16<double>(lo[p], hi[p], turns[p], r.halves, 1.f);
    if (stays) {
      const bool held = token < m.n_tokens;
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int q = 0; q < 2; ++q) {
          float x[4];
          from_e4m3(old[p][h][q], x);
#pragma unroll
          for (int b = 0; b < 4; ++b) {
            float& y = (h ? hi : lo)[p][4 * q + b];
            y = fresh ? y : held ? x[b] * old_scale : 0.f;
          }
        }
    } else {
#pragma unroll
      for (int b = 0; b < 8; ++b) {
        lo[p][b] = fresh ? lo[p][b] : 0.f;
        hi[p][b] = fresh ? hi[p][b] : 0.f;
      }
    }
#pragma unroll
    for (int b = 0; b < 8; ++b)
      most = fmaxf(most, fmaxf(finite_abs(lo[p][b]), finite_abs(hi[p][b])));
  }
#pragma unroll
  for (int off = 32; off > 0; off /= 2) most = fmaxf(most, __shfl_xor(most, off));
  if (threadIdx.x % 64 == 0) most_lds[threadIdx.x / 64] = most;
  // Every held value has been read when the first one is overwritten.
  __syncthreads();
#pragma unroll
  for (int w = 0; w < THREADS / 64; ++w) most = fmaxf(most, most_lds[w]);
  const int e = scale_exponent(most);
  const float inv = pow2(-e);
  if (threadIdx.x == 0) *scale = pow2(e);
  auto word = [&](const float (&x)[8], int j) {
    float y[4];
#pragma unroll
    for (int b = 0; b < 4; ++b) {
      const float z = x[4 * j + b];
      const float in = __builtin_amdgcn_fmed3f(z * inv, -448.f, 448.f);   // e = 119 only
      y[b] = fabsf(z) < __builtin_inff() ? in : __builtin_nanf("");
    }
    return to_e4m3(y[0], y[1], y[2], y[3]);
  };
#pragma unroll
  for (int p = 0; p < 2; ++p) {
    const u32x2 wl = {word(lo[p], 0), word(lo[p], 1)}, wh = {word(hi[p], 0), word(hi[p], 1)};
    const int at = p * ROWS + row;
    if (is_v) {
      *(u32x2*)(bytes + at * LDS_ROW + 8 * c) = wl;
      *(u32x2*)(bytes + at * LDS_ROW + 64 + 8 * c) = wh;
    } else {
      *(u32x2*)(k_rows + at * 128 + 8 * c) = wl;
      *(u32x2*)(k_rows + at * 128 + 64 + 8 * c) = wh;
    }
  }
  if (!is_v) return;
  __syncthreads();
  rows_to_tiles<B, THREADS>(bytes, v_tiles);
}

constexpr int THREADS = 256;        // of a read

struct ReadArgs {
  lvsa_kv_cache c;
  void* k;
  void* v;
  int64_t k_sh, k_st, v_sh, v_st;
  int32_t start, n, first_tile;
};

template <typename T>
__device__ __forceinline__ void store4(T* p, const float (&x)[4]) {
  typedef T t4 __attribute__((ext_vector_type(4)));
  t4 a;
#pragma unroll
  for (int i = 0; i < 4; ++i) a[i] = (T)x[i];
  *(t4*)p = a;
}

// One workgroup a tile of 64 tokens, head and tensor.
template <typename T>
__global__ __launch_bounds__(THREADS) void read_kernel(ReadArgs a) {
  const int tile = a.first_tile + blockIdx.x;
  const int64_t head = blockIdx.y;
  const lvsa_kv_cache& m = a.c;
  const int64_t base = head * m.capacity;
  const bool is_v = a.k == nullptr || blockIdx.z != 0;
  const float scale =
      (is_v ? m.v_scale : m.k_scale)[base / m.block + (int64_t)tile * 64 / m.block];
  if (!is_v) {
    T* const out = (T*)a.k + head * a.k_sh;
    for (int at = threadIdx.x; at < 64 * 32; at += THREADS) {
      const int token = tile * 64 + at / 32, i = token - a.start;
      if (i < 0 || i >= a.n) continue;
      float x[4];
      from_e4m3(*(const uint32_t*)((const uint8_t*)m.k + (base + token) * 128 + at % 32 * 4), x);
#pragma unroll
      for (int b = 0; b < 4; ++b) x[b] *= scale;
      store4(out + i * a.k_st + at % 32 * 4, x);
    }
    return;
  }
  // V: four elements d and 16 tokens a thread.
  T* const out = (T*)a.v + head * a.v_sh;
  if (threadIdx.x >= 128) return;
  const int dq = threadIdx.x % 32, g = threadIdx.x / 32;
  const uint8_t* const from =
      (const uint8_t*)m.v + (base / 64 + tile) * 8192 + 4 * dq * 64 + 16 * g;
  u32x4 in[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) in[j] = *(const u32x4*)(from + 64 * j);
#pragma unroll
  for (int kt = 0; kt < 4; ++kt) {
    uint32_t w[4] = {in[0][kt], in[1][kt], in[2][kt], in[3][kt]};
    transpose4(w);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int i = tile * 64 + 16 * kt + 4 * g + j - a.start;
      if (i < 0 || i >= a.n) continue;
      float x[4];
      from_e4m3(w[j], x);
#pragma unroll
      for (int b = 0; b < 4; ++b) x[b] *= scale;
      store4(out + i * a.v_st + 4 * dq, x);
    }
  }
}

template <typename T>
void start_write(const WriteArgs& a, const RopeArgs& r, dim3 grid, hipStream_t s) {
  if (a.c.block == 64)
    write_kernel<T, 64><<<grid, 256, 0, s>>>(a, r);
  else
    write_kernel<T, 128><<<grid, 512, 0, s>>>(a, r);
}

}  // namespace

hipError_t launch_kv_write(const lvsa_kv_cache& c, int32_t held, const lvsa_tensor& k,
                           const lvsa_tensor& v, int32_t dtype, int32_t start,
                           const RopeArgs& rope, hipStream_t stream) {
  WriteArgs a;
  a.c = c;
  a.c.n_tokens = held;
  a.k = k.data, a.v = v.data;
  a.k_sh = k.stride_head, a.k_st = k.stride_token;
  a.v_sh = v.stride_head, a.v_st = v.stride_token;
  a.start = start, a.n = k.n_tokens;
  a.first_block = start / c.block;
  const int32_t last = (start + k.n_tokens - 1) / c.block;
  const dim3 grid((uint32_t)(last - a.first_block + 1), (uint32_t)c.heads, 2);
  if (dtype == LVSA_BF16)
    start_write<__bf16>(a, rope, grid, stream);
  else if (dtype == LVSA_F16)
    start_write<_Float16>(a, rope, grid, stream);
  else
    start_write<float>(a, rope, grid, stream);
  return hipGetLastError();
}

hipError_t launch_kv_read(const lvsa_kv_cache& c, int32_t start, const lvsa_tensor* k,
                          const lvsa_tensor* v, int32_t n, int32_t dtype, hipStream_t stream) {
  ReadArgs a = {};
  a.c = c;
  if (k) a.k = k->data, a.k_sh = k->stride_head, a.k_st = k->stride_token;
  if (v) a.v = v->data, a.v_sh = v->stride_head, a.v_st = v->stride_token;
  a.start = start, a.n = n;
  a.first_tile = start / 64;
  const int32_t last = (start + n - 1) / 64;
  const dim3 grid((uint32_t)(last - a.first_tile + 1), (uint32_t)c.heads, k && v ? 2 : 1);
  if (dtype == LVSA_BF16)
    read_kernel<__bf16><<<grid, THREADS, 0, stream>>>(a);
  else if (dtype == LVSA_F16)
    read_kernel<_Float16><<<grid, THREADS, 0, stream>>>(a);
  else
    read_kernel<float><<<grid, THREADS, 0, stream>>>(a);
  return hipGetLastError();
}

}  // namespace lvsa
