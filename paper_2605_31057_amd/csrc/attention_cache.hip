// attention_cache.hip -- attention over the 8-bit K/V cache.
//
//   out = softmax(q K^T / sqrt(128)) V, K and V from e4m3 bytes times a power of two.
//
// e4m3 * 2^e is exact in bf16, so K and V fragments are converted on their way to
// the bf16 matrix instructions (cvt_scalef32, the scale at no cost) and the only
// roundings are those of P to bf16 and of the output.
//
// Work: an item is up to ROWS query rows that share a key head and, with a mask, a
// query block (row = query head of the group times the block's tokens + token, so
// shared key heads are read once for the whole group).  Its keys, units of 64
// tokens, are split over `splits` workgroups, and a workgroup's over its four
// waves.  A wave takes K and V fragments from memory straight into registers, one
// unit ahead: nothing is shared between waves but the final combination.  With
// splits > 1 partial results (fp32 O, reference m and row sum l) go to the
// workspace and a second kernel combines them in the order of the splits.
#include "values.h"

namespace lvsa {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int D = 128;
constexpr int UNIT = 64;              // keys of a unit
constexpr int WAVES = 4;
constexpr int THREADS = 64 * WAVES;

// How a launch is cut (the same for workspace and kernels).
struct Plan {
  int32_t rt;          // 16-row tiles of an item
  int32_t blocks;      // query blocks (1 without a mask)
  int32_t tiles;       // items of a key head and query block
  int32_t splits;
};

struct KernelArgs {
  CacheAttnArgs a;
  Plan p;
  float scale_log2;
};

// The query rows of an item.
struct Item {
  int32_t kvh;         // key head
  int32_t first, len;  // query tokens of its query block: first .. first + len - 1
  int32_t row0;        // first row
  int32_t walk, units; // CSR entry of its first unit, units
};

__device__ __forceinline__ Item item_of(const KernelArgs& k, int32_t id) {
  const CacheAttnArgs& a = k.a;
  Item it;
  const int32_t tile = id % k.p.tiles, rest = id / k.p.tiles;
  const int32_t qb = rest % k.p.blocks;
  it.kvh = rest / k.p.blocks;
  it.row0 = tile * k.p.rt * 16;
  if (!a.row_ptr) {
    it.first = 0;
    it.len = a.n;
    it.walk = 0;
    it.units = (a.n_tokens + UNIT - 1) / UNIT;
  } else {
    const int32_t block = a.q_start / a.mask_block + qb;
    const int32_t lo = max(block * a.mask_block, a.q_start) - a.q_start;
    it.first = lo;
    it.len = min((block + 1) * a.mask_block - a.q_start, a.n) - lo;
    it.walk = a.row_ptr[block];
    it.units = min(max(a.row_ptr[block + 1] - it.walk, 0), a.mask_blocks) * (a.mask_block / UNIT);
  }
  return it;
}

__device__ __forceinline__ bf16x8 to_bf16(uint32_t w0, uint32_t w1, float scale) {
  const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w0, scale, false);
  const bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w0, scale, true);
  const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w1, scale, false);
  const bf16x2 d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w1, scale, true);
  return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

__device__ __forceinline__ float row_max(float x) {
  x = fmaxf(x, __shfl_xor(x, 16));
  return fmaxf(x, __shfl_xor(x, 32));
}

// One unit's K and V bytes of a lane (group g = lane/16, i = lane%16).  K: rows
// 16kt + i, elements 16g .. +15 and 64 + 16g .. +15.  V: columns d = 16dt + i,
// places 16g .. +15, tokens 16kt + 4g + r of the unit in the order (kt, r).
struct UnitData {
  u32x4 k[4][2];
  u32x4 v[8];
  float k_scale, v_scale;
  int32_t key0;        // first token; at or past n_tokens: nothing to do
};

template <int RT>
__global__ __launch_bounds__(THREADS, RT <= 2 ? 2 : 1) void rows_kernel(KernelArgs ka) {
  constexpr int ROWS = 16 * RT;
  const CacheAttnArgs& a = ka.a;
  __shared__ __attribute__((aligned(16))) float lds_o[WAVES][ROWS][D + 4];
  __shared__ float lds_m[WAVES][ROWS], lds_l[WAVES][ROWS];
  const int wave = threadIdx.x / 64, lane = threadIdx.x % 64;
  const int g = lane / 16, i = lane % 16;
  const int32_t split = blockIdx.x % ka.p.splits, id = blockIdx.x / ka.p.splits;
  const Item it = item_of(ka, id);
  const int32_t rows = it.len * a.group;
  if (it.row0 >= rows) return;
  const int32_t u0 = (int32_t)((int64_t)it.units * split / ka.p.splits);
  const int32_t u1 = (int32_t)((int64_t)it.units * (split + 1) / ka.p.splits);

  // Q fragments: row 16rt + i, elements in the order of K's.
  bf16x8 qf[RT][4];
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    const int32_t row = it.row0 + 16 * rt + i;
    const bool ok = row < rows;
    const int32_t h = ok ? row / it.len : 0, t = ok ? row - h * it.len : 0;
    const __bf16* q = (const __bf16*)a.q + (int64_t)(it.kvh * a.group + h) * a.q_sh +
                      (int64_t)(it.first + t) * a.q_st + 16 * g;
#pragma unroll
    for (int s = 0; s < 4; ++s)
      qf[rt][s] = ok ? *(const bf16x8*)(q + (s / 2) * 64 + (s % 2) * 8) : bf16x8{};
  }

  const int64_t base = (int64_t)it.kvh * a.capacity;
  const uint8_t* const kb = a.k + (base + i) * D + 16 * g;
  const uint8_t* const vb = a.v + base * D + i * UNIT + 16 * g;
  const float* const ks = a.k_scale + (base >> a.scale_shift);
  const float* const vs = a.v_scale + (base >> a.scale_shift);
  const int32_t per = a.row_ptr ? a.mask_block / UNIT : 1;
  auto load = [&](int32_t u, UnitData& d) {
    d.key0 = a.n_tokens;
    if (u >= u1) return;
    int32_t unit = u;
    if (a.row_ptr) {
      const int32_t kblock = a.col_idx[it.walk + u / per];
      if ((uint32_t)kblock >= (uint32_t)a.mask_blocks) return;
      unit = kblock * per + u % per;
    }
    const int32_t key0 = __builtin_amdgcn_readfirstlane(unit * UNIT);
    d.key0 = key0;
    if (key0 >= a.n_tokens) return;
#pragma unroll
    for (int kt = 0; kt < 4; ++kt)
#pragma unroll
      for (int half = 0; half < 2; ++half)
        d.k[kt][half] = *(const u32x4*)(kb + (int64_t)(key0 + 16 * kt) * D + 64 * half);
#pragma unroll
    for (int dt = 0; dt < 8; ++dt)
      d.v[dt] = *(const u32x4*)(vb + (int64_t)key0 * D + dt * 16 * UNIT);
    d.k_scale = ks[key0 >> a.scale_shift];
    d.v_scale = vs[key0 >> a.scale_shift];
  };

  f32x4 o[8][RT];
  float m[RT], l[RT];
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    m[rt] = -__builtin_inff();
    l[rt] = 0.f;
#pragma unroll
    for (int dt = 0; dt < 8; ++dt) o[dt][rt] = f32x4{};
  }
  auto work = [&](UnitData& d) {
    if (d.key0 >= a.n_tokens) return;
    f32x4 s[4][RT];
#pragma unroll
    for (int kt = 0; kt < 4; ++kt) {
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) s[kt][rt] = f32x4{};
#pragma unroll
      for (int st = 0; st < 4; ++st) {
        const u32x4 w = d.k[kt][st / 2];
        const bf16x8 f = to_bf16(w[(st % 2) * 2], w[(st % 2) * 2 + 1], d.k_scale);
#pragma unroll
        for (int rt = 0; rt < RT; ++rt)
          s[kt][rt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f, qf[rt][st], s[kt][rt], 0, 0, 0);
      }
    }
    // Keys at or past n_tokens: no weight, and V bytes of zero whatever they hold.
    const int32_t left = a.n_tokens - d.key0;
    if (left < UNIT) {
#pragma unroll
      for (int kt = 0; kt < 4; ++kt) {
        uint32_t keep = 0u;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const bool ok = 16 * kt + 4 * g + r < left;
          keep |= ok ? 0xFFu << (8 * r) : 0u;
#pragma unroll
          for (int rt = 0; rt < RT; ++rt) s[kt][rt][r] = ok ? s[kt][rt][r] : -__builtin_inff();
        }
#pragma unroll
        for (int dt = 0; dt < 8; ++dt) d.v[dt][kt] &= keep;
      }
    }
    bf16x8 p[RT][2];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      float top = -__builtin_inff();
#pragma unroll
      for (int kt = 0; kt < 4; ++kt)
#pragma unroll
        for (int r = 0; r < 4; ++r) top = fmaxf(top, s[kt][rt][r]);
      top = row_max(top) * ka.scale_log2;
      if (__builtin_amdgcn_ballot_w64(top > m[rt])) {
        const float now = fmaxf(m[rt], top);
        const float f = now == m[rt] ? 1.f : __builtin_amdgcn_exp2f(m[rt] - now);
        m[rt] = now;
        l[rt] *= f;
#pragma unroll
        for (int dt = 0; dt < 8; ++dt) o[dt][rt] *= f;
      }
      const float ref = m[rt] == -__builtin_inff() ? 0.f : m[rt];
#pragma unroll
      for (int kt = 0; kt < 4; ++kt)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const float x =
              __builtin_amdgcn_exp2f(__builtin_fmaf(s[kt][rt][r], ka.scale_log2, -ref));
          const __bf16 b = (__bf16)x;
          p[rt][kt / 2][kt % 2 * 4 + r] = b;
          l[rt] += (float)b;    // of the rounded P: the weights of a row add up to 1
        }
    }
#pragma unroll
    for (int dt = 0; dt < 8; ++dt)
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        const bf16x8 f = to_bf16(d.v[dt][2 * half], d.v[dt][2 * half + 1], d.v_scale);
#pragma unroll
        for (int rt = 0; rt < RT; ++rt)
          o[dt][rt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f, p[rt][half], o[dt][rt], 0, 0, 0);
      }
  };

  UnitData d0, d1;
  load(u0 + wave, d0);
  for (int32_t u = u0 + wave; u < u1; u += 2 * WAVES) {
    load(u + WAVES, d1);
    work(d0);
    load(u + 2 * WAVES, d0);
    work(d1);
  }

  // The waves' parts, combined in LDS in the waves' order.
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    float sum = l[rt];
    sum += __shfl_xor(sum, 16);
    sum += __shfl_xor(sum, 32);
    if (g == 0) {
      lds_m[wave][16 * rt + i] = m[rt];
      lds_l[wave][16 * rt + i] = sum;
    }
#pragma unroll
    for (int dt = 0; dt < 8; ++dt) *(f32x4*)&lds_o[wave][16 * rt + i][16 * dt + 4 * g] = o[dt][rt];
  }
  __syncthreads();
  for (int at = threadIdx.x; at < ROWS * (D / 4); at += THREADS) {
    const int r = at / (D / 4), c = at % (D / 4) * 4;
    const int32_t row = it.row0 + r;
    if (row >= rows) break;
    float top = -__builtin_inff(), sum = 0.f;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) top = fmaxf(top, lds_m[w][r]);
    f32x4 acc = {};
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
      const float mw = lds_m[w][r];
      const float f = mw == -__builtin_inff() ? 0.f : __builtin_amdgcn_exp2f(mw - top);
      sum += f * lds_l[w][r];
      acc += f * *(const f32x4*)&lds_o[w][r][c];
    }
    if (ka.p.splits == 1) {
      const int32_t h = row / it.len, t = row - h * it.len;
      __bf16* out = (__bf16*)a.o + (int64_t)(it.kvh * a.group + h) * a.o_sh +
                    (int64_t)(it.first + t) * a.o_st + c;
      const float inv = sum > 0.f || sum != sum ? 1.f / sum : 0.f;
      bf16x4 b;
#pragma unroll
      for (int e = 0; e < 4; ++e) b[e] = (__bf16)(acc[e] * inv);
      *(bf16x4*)out = b;
    } else {
      const int64_t slot = ((int64_t)id * ka.p.splits + split) * ROWS + r;
      const int64_t slots = (int64_t)gridDim.x * ROWS;
      *(f32x4*)(a.workspace + slot * D + c) = acc;
      if (c == 0) {
        a.workspace[slots * D + 2 * slot] = top;
        a.workspace[slots * D + 2 * slot + 1] = sum;
      }
    }
  }
}

// Combines the splits of a row, in their order: 32 threads a row.
__global__ __launch_bounds__(THREADS) void combine_kernel(KernelArgs ka, int32_t rows_item) {
  const CacheAttnArgs& a = ka.a;
  const int32_t id = blockIdx.x / (rows_item / 8);
  const int r = blockIdx.x % (rows_item / 8) * 8 + threadIdx.x / 32, c = threadIdx.x % 32 * 4;
  const Item it = item_of(ka, id);
  const int32_t row = it.row0 + r;
  if (row >= it.len * a.group) return;
  const int64_t items = gridDim.x / (rows_item / 8);
  const int64_t slots = items * ka.p.splits * rows_item;
  const int64_t slot0 = (int64_t)id * ka.p.splits * rows_item + r;
  const float* ml = a.workspace + slots * D;
  float top = -__builtin_inff(), sum = 0.f;
  for (int s = 0; s < ka.p.splits; ++s)
    top = fmaxf(top, ml[2 * (slot0 + (int64_t)s * rows_item)]);
  f32x4 acc = {};
  for (int s = 0; s < ka.p.splits; ++s) {
    const int64_t slot = slot0 + (int64_t)s * rows_item;
    const float ms = ml[2 * slot];
    const float f = ms == -__builtin_inff() ? 0.f : __builtin_amdgcn_exp2f(ms - top);
    sum += f * ml[2 * slot + 1];
    acc += f * *(const f32x4*)(a.workspace + slot * D + c);
  }
  const float inv = sum > 0.f || sum != sum ? 1.f / sum : 0.f;
  const int32_t h = row / it.len, t = row - h * it.len;
  bf16x4 b;
#pragma unroll
  for (int e = 0; e < 4; ++e) b[e] = (__bf16)(acc[e] * inv);
  *(bf16x4*)((__bf16*)a.o + (int64_t)(it.kvh * a.group + h) * a.o_sh +
             (int64_t)(it.first + t) * a.o_st + c) = b;
}

Plan plan_of(const CacheAttnArgs& a, int32_t cus) {
  Plan p;
  p.blocks = 1;
  int64_t rows = (int64_t)a.n * a.group;
  int64_t units = (a.n_tokens + UNIT - 1) / UNIT;
  if (a.row_ptr) {
    p.blocks = (a.q_start + a.n - 1) / a.mask_block - a.q_start / a.mask_block + 1;
    rows = (int64_t)(a.n < a.mask_block ? a.n : a.mask_block) * a.group;
  }
  p.rt = rows > 16 ? 2 : 1;
  p.tiles = (int32_t)((rows + 16 * p.rt - 1) / (16 * p.rt));
  // Two workgroups a compute unit; a wave's share is at least two units.
  const int64_t items = (int64_t)a.heads * p.blocks * p.tiles;
  int64_t splits = 2 * cus / items;
  if (splits > units / (2 * WAVES)) splits = units / (2 * WAVES);
  p.splits = splits < 1 ? 1 : (int32_t)splits;
  return p;
}

}  // namespace

int64_t cache_attention_workspace(const CacheAttnArgs& a, int32_t cus) {
  const Plan p = plan_of(a, cus);
  if (p.splits == 1) return 0;
  return (int64_t)a.heads * p.blocks * p.tiles * p.splits * 16 * p.rt * (D + 2) * 4;
}

hipError_t launch_cache_attention(const CacheAttnArgs& a, int32_t cus, hipStream_t stream) {
  KernelArgs k;
  k.a = a;
  k.p = plan_of(a, cus);
  k.scale_log2 = 1.4426950408889634f / 11.313708498984761f;   // log2(e) / sqrt(128)
  const int64_t items = (int64_t)a.heads * k.p.blocks * k.p.tiles;
  const dim3 grid((uint32_t)(items * k.p.splits));
  if (k.p.rt == 1)
    rows_kernel<1><<<grid, THREADS, 0, stream>>>(k);
  else
    rows_kernel<2><<<grid, THREADS, 0, stream>>>(k);
  if (hipError_t e = hipGetLastError(); e != hipSuccess || k.p.splits == 1) return e;
  combine_kernel<<<dim3((uint32_t)(items * (k.p.rt * 2))), THREADS, 0, stream>>>(k, 16 * k.p.rt);
  return hipGetLastError();
}

}  // namespace lvsa
