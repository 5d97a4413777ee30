// attention_cache.hip -- attention over the 8-bit K/V cache.
//
//   out = softmax(q K^T / sqrt(128)) V, K and V from e4m3 bytes times a power of two.
//
// e4m3 * 2^e is exact in bf16: bytes become bf16 matrix operands by one conversion
// (cvt_scalef32, the scale at no cost), and the only roundings are those of P to bf16
// and of the output, besides fp32 sums.
//
// Work: an item is some query rows of one key head; its keys, units of 64 tokens, are
// split over `splits` workgroups.  With splits > 1 partial results (fp32 O, reference
// m and row sum l) go to the workspace and combine_kernel adds them in the order of
// the splits.  Two forms (plan_of): up to 64 rows the keys' bytes bound the call and
// rows_kernel streams them, from there on the products do and tile_kernel works 256 rows
// at a time.
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
constexpr int TILE_ROWS = 256;

// How a launch is cut (the same for workspace and kernels).  Rows form: an item's rows
// share a key head and, with a mask, a query block.  Tile form: 256 rows; with a
// mask of one query head and 256 / mask_block query blocks, else of a key head's
// queries.
struct Plan {
  bool tile;
  int32_t item_rows;   // rows of an item
  int32_t blocks;      // rows form: query blocks (1 without a mask)
  int32_t tiles;       // items of a key head and query block (of a head, tile form)
  int32_t heads;       // tile form with a mask: query heads; else key heads
  int32_t splits;
};

struct KernelArgs {
  CacheAttnArgs a;
  Plan p;
  float scale_log2;
};

// The rows of an item.  Row r is row row0 + r of `rows`, which are the tokens first ..
// first + len - 1 of the query heads head0, head0 + 1, .. one head after the other.
struct Item {
  int32_t kvh, head0;
  int32_t first, len, rows, row0;
  int32_t block0, blocks;   // query blocks of the mask
};

__device__ __forceinline__ Item item_of(const KernelArgs& k, int32_t tile, int32_t rest) {
  const CacheAttnArgs& a = k.a;
  Item it;
  it.row0 = tile * k.p.item_rows;
  it.block0 = 0;
  it.blocks = 0;
  it.first = 0;
  it.len = a.n;
  if (k.p.tile && a.row_ptr) {
    const int32_t per = TILE_ROWS / a.mask_block, from = a.q_start / a.mask_block;
    it.kvh = rest / a.group;
    it.head0 = rest;
    it.block0 = from + tile * per;
    it.blocks = min(per, (a.q_start + a.n - 1) / a.mask_block + 1 - it.block0);
    it.first = it.block0 * a.mask_block - a.q_start;
    it.len = it.rows = TILE_ROWS;
    it.row0 = 0;
    return it;
  }
  const int32_t qb = rest % k.p.blocks;
  it.kvh = rest / k.p.blocks;
  it.head0 = it.kvh * a.group;
  if (a.row_ptr) {
    it.block0 = a.q_start / a.mask_block + qb;
    it.blocks = 1;
    it.first = max(it.block0 * a.mask_block - a.q_start, 0);
    it.len = min((it.block0 + 1) * a.mask_block - a.q_start, a.n) - it.first;
  }
  it.rows = it.len * a.group;
  return it;
}

// Query head and token of row r of an item; false (and 0, 0) where there is none.
__device__ __forceinline__ bool row_of(const Item& it, const CacheAttnArgs& a, int32_t r,
                                       int32_t& head, int32_t& token) {
  const int32_t row = it.row0 + r, h = row / it.len, t = it.first + row - h * it.len;
  const bool ok = row < it.rows && (uint32_t)t < (uint32_t)a.n;
  head = ok ? it.head0 + h : 0;
  token = ok ? t : 0;
  return ok;
}

__device__ __forceinline__ bf16x8 to_bf16(uint32_t w0, uint32_t w1, float scale) {
  const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w0, scale, false);
  const bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w0, scale, true);
  const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w1, scale, false);
  const bf16x2 d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w1, scale, true);
  return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// Whether a lane's part of a query row holds an element that is not finite: adding 2^7
// to a half's magnitude carries into its sign bit from the exponent of infinity on.
// Such a row becomes NaN whatever signs its keys have (scores of -inf alone would look
// like a row without keys).
__device__ __forceinline__ bool not_finite(const bf16x8 (&q)[4]) {
  uint32_t over = 0u;
#pragma unroll
  for (int s = 0; s < 4; ++s) {
    const u32x4 w = __builtin_bit_cast(u32x4, q[s]);
#pragma unroll
    for (int e = 0; e < 4; ++e) over |= (w[e] & 0x7FFF7FFFu) + 0x00800080u;
  }
  return (over & 0x80008000u) != 0u;
}

// A value that the launch only reads, at an index that is the same in the whole wave:
// by a scalar load, which no wait for the wave's vector loads holds up (they are
// counted in order, so a vector load behind K's and V's would wait for those).
template <typename T>
__device__ __forceinline__ T uniform_load(const T* p, int32_t at) {
  typedef const __attribute__((address_space(4))) T* constant;
  return *((constant)(uintptr_t)p + __builtin_amdgcn_readfirstlane(at));
}

__device__ __forceinline__ float row_max(float x) {
  x = fmaxf(x, __shfl_xor(x, 16));
  return fmaxf(x, __shfl_xor(x, 32));
}

// Few query rows: an item is up to 16 RT rows that share a key head and, with a mask, a
// query block (row = query head of the group times the block's tokens + token, so
// shared key heads are read once for the whole group).  Four waves take every fourth
// unit and share nothing until their results are combined in LDS.  One query of 12
// heads over 32,760 tokens: 19 us, 5.3 TB/s of keys and values; 40 rows of 8 key heads
// over 131,071 tokens 59 us, 4.6 TB/s (and the combining launch, 4 to 5 us).
//
// RT: 16-row tiles of the item, each K and V fragment is used for all of them.  A wave
// holds one unit's bytes: K's of the next unit are loaded when this one's scores are
// done, V's when its products are, so both are on their way for most of a unit, and
// with two waves a SIMD (one from 33 rows on, for the registers) a compute unit has
// some 64 KB in flight.
//
// A lane (group g = lane/16, i = lane%16) takes K rows 16kt + i, elements 16g .. +15 and
// 64 + 16g .. +15, and V columns d = 16dt + i, places 16g .. +15, which are tokens 16kt + 4g
// + r of the unit in the order (kt, r): what its score registers hold.
template <int RT>
__global__ __launch_bounds__(THREADS, RT <= 2 ? 2 : 1) void rows_kernel(KernelArgs ka) {
  constexpr int ROWS = 16 * RT;
  const CacheAttnArgs& a = ka.a;
  __shared__ __attribute__((aligned(16))) float lds_o[WAVES][ROWS][D + 4];
  __shared__ float lds_m[WAVES][ROWS], lds_l[WAVES][ROWS];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), lane = threadIdx.x % 64;
  const int g = lane / 16, i = lane % 16;
  const int32_t split = blockIdx.x % ka.p.splits, id = blockIdx.x / ka.p.splits;
  const Item it = item_of(ka, id % ka.p.tiles, id / ka.p.tiles);
  if (it.row0 >= it.rows) return;
  // Its units: the first `units` of the walk, or with a mask of the row's entries.
  const int32_t per = a.row_ptr ? a.mask_block / UNIT : 1;
  int32_t walk = 0, units = (a.n_tokens + UNIT - 1) / UNIT;
  if (a.row_ptr) {
    walk = a.row_ptr[it.block0];
    units = min(max(a.row_ptr[it.block0 + 1] - walk, 0), a.mask_blocks) * per;
  }
  const int32_t u0 = (int32_t)((int64_t)units * split / ka.p.splits);
  const int32_t u1 = (int32_t)((int64_t)units * (split + 1) / ka.p.splits);

  // Q fragments: row 16rt + i, elements in the order of K's.
  bf16x8 qf[RT][4];
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    int32_t h, t;
    const bool ok = row_of(it, a, 16 * rt + i, h, t);
    const __bf16* q =
        (const __bf16*)a.q + (int64_t)h * a.q_sh + (int64_t)t * a.q_st + 16 * g;
#pragma unroll
    for (int s = 0; s < 4; ++s)
      qf[rt][s] = ok ? *(const bf16x8*)(q + (s / 2) * 64 + (s % 2) * 8) : bf16x8{};
  }

  const int64_t base = (int64_t)it.kvh * a.capacity;
  const uint8_t* const kb = a.k + base * D;
  const uint8_t* const vb = a.v + base * D;
  const uint32_t k_lane = i * D + 16 * g, v_lane = i * UNIT + 16 * g;
  const float* const ks = a.k_scale + (base >> a.scale_shift);
  const float* const vs = a.v_scale + (base >> a.scale_shift);
  // First token of the walk's unit u; n_tokens where there is none.
  auto key_of = [&](int32_t u) -> int32_t {
    if (u >= u1) return a.n_tokens;
    if (!a.row_ptr) return u * UNIT;
    const int32_t block = uniform_load(a.col_idx, walk + u / per);
    if ((uint32_t)block >= (uint32_t)a.mask_blocks) return a.n_tokens;
    return min((block * per + u % per) * UNIT, a.n_tokens);
  };
  u32x4 k[4][2], v[8];
  auto load_k = [&](int32_t key0) {
    const uint8_t* const at = kb + (int64_t)key0 * D;
#pragma unroll
    for (int kt = 0; kt < 4; ++kt)
#pragma unroll
      for (int half = 0; half < 2; ++half)
        k[kt][half] = *(const u32x4*)(at + k_lane + kt * 16 * D + 64 * half);
  };
  auto load_v = [&](int32_t key0) {
    const uint8_t* const at = vb + (int64_t)key0 * D;
#pragma unroll
    for (int dt = 0; dt < 8; ++dt) v[dt] = *(const u32x4*)(at + v_lane + dt * 16 * UNIT);
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
  // Units of the wave: u0 + wave, then every fourth.  Columns outside the mask are
  // passed over (their place holds no tokens).
  int32_t u = u0 + wave;
  auto next_unit = [&]() -> int32_t {
    int32_t key = a.n_tokens;
    while (u < u1 && key >= a.n_tokens) {
      key = key_of(u);
      u += WAVES;
    }
    return key;
  };
  int32_t key0 = next_unit();
  float k_scale = 1.f, v_scale = 1.f;
  if (key0 < a.n_tokens) {
    load_k(key0);
    load_v(key0);
    k_scale = uniform_load(ks, key0 >> a.scale_shift);
    v_scale = uniform_load(vs, key0 >> a.scale_shift);
  }
  const bool worked = key0 < a.n_tokens;
  while (key0 < a.n_tokens) {
    const int32_t key1 = next_unit();
    const int32_t scale1 = min(key1, a.n_tokens - 1) >> a.scale_shift;
    const float k_scale1 = uniform_load(ks, scale1), v_scale1 = uniform_load(vs, scale1);
    f32x4 s[4][RT];
#pragma unroll
    for (int kt = 0; kt < 4; ++kt) {
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) s[kt][rt] = f32x4{};
#pragma unroll
      for (int st = 0; st < 4; ++st) {
        const u32x4 w = k[kt][st / 2];
        const bf16x8 f = to_bf16(w[(st % 2) * 2], w[(st % 2) * 2 + 1], k_scale);
#pragma unroll
        for (int rt = 0; rt < RT; ++rt)
          s[kt][rt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f, qf[rt][st], s[kt][rt], 0, 0, 0);
      }
    }
    __builtin_amdgcn_sched_barrier(0);
    if (key1 < a.n_tokens) load_k(key1);
    __builtin_amdgcn_sched_barrier(0);
    // Keys at or past n_tokens: no weight, and V bytes of zero whatever they hold.
    const int32_t left = a.n_tokens - key0;
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
        for (int dt = 0; dt < 8; ++dt) v[dt][kt] &= keep;
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
        const bf16x8 f = to_bf16(v[dt][2 * half], v[dt][2 * half + 1], v_scale);
#pragma unroll
        for (int rt = 0; rt < RT; ++rt)
          o[dt][rt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f, p[rt][half], o[dt][rt], 0, 0, 0);
      }
    __builtin_amdgcn_sched_barrier(0);
    if (key1 < a.n_tokens) load_v(key1);
    key0 = key1;
    k_scale = k_scale1;
    v_scale = v_scale1;
  }

  // The waves' parts, combined in LDS in the waves' order.
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    float sum = worked && not_finite(qf[rt]) ? __builtin_nanf("") : l[rt];
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
    int32_t h, t;
    if (!row_of(it, a, r, h, t)) break;
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
      __bf16* out = (__bf16*)a.o + (int64_t)h * a.o_sh + (int64_t)t * a.o_st + c;
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

// ------------------------------------------------------------------- tiles
//
// Many query rows: an item is 256 rows, eight waves of 32, which walk the union of its
// query blocks' key lists 128 keys (two units) a step, sharing every K and V byte
// through LDS.
//
//   S^T = K Q^T     bf16 MFMA 16x16x32, K as bytes in LDS, converted in registers
//   O^T += V^T P^T  bf16 MFMA 16x16x32, V converted to bf16 on its way into LDS
//
// Scores take bf16 products and fp32 sums, as the other form's do.  The fp8 matrix
// instructions would take K's bytes as they are (Q as the sum of two e4m3 numbers), but
// add 128 products with an error of up to 2^-13 of sum |q k|: where one channel of q
// and k is 32 (128) and the others N(0, 1), the result was off by 1.4e-2 (0.15) of its
// norm, and is by 2.2e-3 now, as without such a channel (2 heads, 128 queries, 4,096
// tokens).  They were 8 to 11% faster (40 heads of 4,680 queries over 63,960 tokens 4.40
// and 4.88 ms, one frame of 12 heads over the 121-frame mask 211 and 233 us).  V is
// converted once a workgroup, 32 elements a thread and step; K by every wave, 128
// conversions of two elements.  K converted once a workgroup, in place of its bytes in
// LDS, takes twice the LDS reads and some spills: 4.90 ms, and 217 us with a mask.
//
// What bounds it: the matrix phase, its issue slots shared with the other wave's softmax.
// 4,680 queries of 40 heads over 63,960 tokens take 4.88 ms (1.26 PFLOP/s; a large bf16
// matrix product 1.6), the matrix cores busy 55% of the cycles.
//
// Schedule: waves w and w + 4 share a SIMD and run half a step apart, one in its
// matrix phase while the other is in its softmax phase; a barrier ends each half
// step.  Half steps 2j and 2j + 1: the leaders (waves 0-3) are in matrix phase j, then
// softmax j + 1; the others in softmax j, then matrix phase j.  K(j+1) and V(j) stay
// in LDS through both; K(j+2) and V(j+1) go into the other two stages, by every wave
// in its softmax phase: K's loads before the weights; after them V's bytes, loaded a step
// ago into a place of the wave's own, are converted and written into the stage, and
// the next step's loaded (held in registers meanwhile, 8 of them, they made the compiler
// spill).  All loads go from memory into LDS.

typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) void lds_void;

constexpr int TILE_THREADS = 512;
constexpr int K_STAGE = 2 * UNIT * D;        // 128 rows of 128 bytes
constexpr int V_STAGE = 2 * UNIT * D * 2;    // 128 rows (d) of 256 bytes (keys)
constexpr int V_AT = 2 * K_STAGE;
constexpr int RAW_AT = V_AT + 2 * V_STAGE;   // V's bytes of a step
constexpr int ZERO_AT = RAW_AT + K_STAGE;    // with a mask: two slabs of zeros, the list
constexpr int LIST_AT = ZERO_AT + V_STAGE / 2;
constexpr int LIST_WORDS = kMaxSparseBlocks;
constexpr int BITMAP_WORDS = 256;
static_assert(BITMAP_WORDS * 32 >= LIST_WORDS, "a bit a block");
constexpr int TILE_LDS = LIST_AT + LIST_WORDS * 4 + 64;

// Distance (log2) of a row's reference above the largest score it was set from.
constexpr float HEADROOM = 7.f;
constexpr float WIDE_HEADROOM = 39.f;

// LDS layout: slabs of rows of 64 bytes (four chunks of 16), chunk c of row r at place
// c ^ x(r), x(r) = -(r/4) mod 4.  The 64 lanes of a fragment read 16 rows whole, chunk g
// of row i for lane (g, i); a read is served 16 lanes at a time, four rows' worth of
// banks, and x puts the four lanes that share a row's banks at four chunks.
//   K stage: slab h (elements 64h .. 64h+63), row = key, 128 rows
//   V stage: slab u (keys of the 32-key group u), row = d, 128 rows; chunk g holds the
//   keys that lane group g's P registers hold: tokens 32u + 4g + r, 32u + 16 + 4g + r
constexpr int SLAB = 128 * 64;
__device__ __forceinline__ int xsw(int row) { return -(row >> 2) & 3; }

// One wave load (1 KiB) from memory into LDS.  Inline assembly, so that the compiler
// puts no wait for it between here and the half step's end, where tile_sync waits.
// The nop is the wait state between a write of M0 and the load.
__device__ __forceinline__ void load_to_lds(uint32_t dst, const u32x4& rsrc, uint32_t voff,
                                            uint32_t soff) {
  asm volatile(
      "s_mov_b32 m0, %0\n\t"
      "s_nop 0\n\t"
      "buffer_load_dwordx4 %1, %2, %3 offen lds"
      :
      : "s"(__builtin_amdgcn_readfirstlane(dst)), "v"(voff), "s"(rsrc),
        "s"(__builtin_amdgcn_readfirstlane(soff))
      : "memory", "m0");
}
__device__ __forceinline__ void tile_barrier() {
  asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
}
// The same, with the wave's loads into LDS done but for the last LEFT (other loads
// among them only make the wait longer).
template <int LEFT>
__device__ __forceinline__ void tile_sync() {
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"i"(LEFT) : "memory");
}

// Buffer resource of `bytes` bytes from p on, in scalar registers.
__device__ __forceinline__ u32x4 rsrc_of(const void* p, uint32_t bytes) {
  const uint64_t at = (uint64_t)p;
  return u32x4{(uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)at),
               (uint32_t)__builtin_amdgcn_readfirstlane((int)(at >> 32) & 0xFFFF),
               (uint32_t)__builtin_amdgcn_readfirstlane((int)bytes), 0x00020000u};
}

// The scale of exponent byte `at` of a step's.
__device__ __forceinline__ float scale_of(int32_t scales, int at) {
  return __uint_as_float((((uint32_t)scales >> (8 * at)) & 0xFFu) << 23);
}

// The lane's index, made anew where a rare branch needs it: what is derived from it
// there is not kept in registers through the loop.
__device__ __forceinline__ int fresh_lane() {
  int lane = (int)__builtin_amdgcn_mbcnt_hi(~0u, __builtin_amdgcn_mbcnt_lo(~0u, 0u));
  asm volatile("" : "+v"(lane));
  return lane;
}

// One step's units.
struct Step {
  int32_t unit[2];
  int32_t left[2];   // held tokens from the unit's first on, at most 0: none
  int32_t keep;      // bit u: this wave's query block keeps unit u
  int32_t scales;    // exponent bytes: K of unit 0, of unit 1, V of unit 0, of unit 1
};
// One of two by value: a reference to either would put both into memory.
__device__ __forceinline__ Step pick(bool first, const Step& a, const Step& b) {
  Step s;
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    s.unit[u] = first ? a.unit[u] : b.unit[u];
    s.left[u] = first ? a.left[u] : b.left[u];
  }
  s.keep = first ? a.keep : b.keep;
  s.scales = first ? a.scales : b.scales;
  return s;
}

// Q of a wave: two 16-row tiles, elements in the order of K's fragments.
struct QTiles {
  bf16x8 f[2][4];
};

struct TileState {
  f32x4 o[8][2];   // O^T [d tile][query tile]
  f32x4 l[2];      // row sums, in register 0 (the others add the same products, but are not
                   // rescaled; an accumulator each: a row that is NaN would spoil the other
                   // tile's row of the same lane)
  float m[2];      // references (log2)
  int flags;       // READY: every row has a finite m; WIDE: a step was redone
};
constexpr int READY = 1, WIDE = 2;

struct Scores {
  f32x4 s[8][2];   // [16-key tile][query tile]
};
struct Probs {
  bf16x8 p[4][2];  // [32-key group][query tile]
};

// Fragments: `at` is the lane's offset in a slab's first 16 rows.
__device__ __forceinline__ i32x8 k_frag(const char* k, uint32_t at, int kt) {
  const i32x4 a = *(const i32x4*)(k + at + kt * 1024);
  const i32x4 b = *(const i32x4*)(k + at + kt * 1024 + SLAB);
  return i32x8{a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
}
// Scores of keys that do not exist or that the wave's query block does not keep: -inf.
__device__ __forceinline__ void mask_scores(Scores& sc, const Step& st) {
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    if (st.keep == 0) break;   // its weights are zeros (weigh)
    const int left = (st.keep >> u) & 1 ? st.left[u] : 0;
    if (left >= UNIT) continue;
    const int lim = left - 4 * (fresh_lane() / 16);
#pragma unroll
    for (int kt = 0; kt < 4; ++kt)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        if (r % 2 == 0) __builtin_amdgcn_sched_barrier(0);
        const bool ok = 16 * kt + r < lim;
#pragma unroll
        for (int qt = 0; qt < 2; ++qt)
          sc.s[4 * u + kt][qt][r] = ok ? sc.s[4 * u + kt][qt][r] : -__builtin_inff();
      }
  }
}

// Raises the reference of rows whose largest score lies above it to `head` above that
// score, the others by `lift`, and rescales O and l.
__device__ __forceinline__ void raise(const Scores& sc, TileState& st, float scale, float head,
                                      float lift) {
#pragma unroll
  for (int qt = 0; qt < 2; ++qt) {
    float top = -__builtin_inff();
#pragma unroll
    for (int kt = 0; kt < 8; ++kt)
#pragma unroll
      for (int r = 0; r < 4; ++r) top = fmaxf(top, sc.s[kt][qt][r]);
    top = row_max(top) * scale;
    const float m = top > st.m[qt] ? top + head : st.m[qt] + lift;
    const float f = m == st.m[qt] ? 1.f : __builtin_amdgcn_exp2f(st.m[qt] - m);
    st.m[qt] = m;
    st.l[qt][0] *= f;
#pragma unroll
    for (int dt = 0; dt < 8; ++dt) st.o[dt][qt] *= f;
  }
  const bool ready = __builtin_amdgcn_ballot_w64(st.m[0] == -__builtin_inff() ||
                                                 st.m[1] == -__builtin_inff()) == 0;
  st.flags = (st.flags & ~READY) | (ready ? READY : 0);
}

// P = 2^(s * scale - m); returns the bits of all probabilities or-ed together.
__device__ __forceinline__ uint32_t weights(const Scores& sc, Probs& pr, const float (&m)[2],
                                            float scale) {
  uint32_t bits = 0u;
#pragma unroll
  for (int u = 0; u < 4; ++u)
#pragma unroll
    for (int qt = 0; qt < 2; ++qt) {
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int r = 0; r < 4; r += 2) {
          const float a =
              __builtin_amdgcn_exp2f(__builtin_fmaf(sc.s[2 * u + t][qt][r], scale, -m[qt]));
          const float b =
              __builtin_amdgcn_exp2f(__builtin_fmaf(sc.s[2 * u + t][qt][r + 1], scale, -m[qt]));
          const bf16x2 pk = {(__bf16)a, (__bf16)b};
          bits |= __builtin_bit_cast(uint32_t, pk);
          pr.p[u][qt][4 * t + r] = pk[0];
          pr.p[u][qt][4 * t + r + 1] = pk[1];
        }
    }
  return bits;
}

// Scores to weights against the rows' references as they stand, HEADROOM above the
// score they were set from: a step takes a row maximum only when some weight reaches 2
// (the top exponent bit of its bf16), and is then done again with the reference
// raised.  Exact either way: O and l always use the same reference.  The sums l are
// taken of the rounded weights, so a row's weights add up to 1.
__device__ __forceinline__ void softmax_phase(const Scores& sc, TileState& st, Probs& pr,
                                              float scale) {
  const int flags = __builtin_amdgcn_readfirstlane(st.flags);
  const bool first = !(flags & READY);
  if (first) raise(sc, st, scale, (flags & WIDE) ? WIDE_HEADROOM : HEADROOM, 0.f);
  float m[2];
#pragma unroll
  for (int qt = 0; qt < 2; ++qt) m[qt] = st.m[qt] == -__builtin_inff() ? 0.f : st.m[qt];
  const uint32_t bits = weights(sc, pr, m, scale);
  if (__builtin_amdgcn_ballot_w64((bits & 0x40004000u) != 0u) && !first) {
    st.flags |= WIDE;
    raise(sc, st, scale, WIDE_HEADROOM, (flags & WIDE) ? 0.f : WIDE_HEADROOM - HEADROOM);
    weights(sc, pr, st.m, scale);
  }
}

// Weights of a step: zeros where the wave's query block keeps none of it (rows without a
// key have no reference, and would look for one every step).
template <bool MASKED>
__device__ __forceinline__ void weigh(const Scores& sc, TileState& st, Probs& pr, float scale,
                                      int keep) {
  if (MASKED && keep == 0) {
#pragma unroll
    for (int u = 0; u < 4; ++u)
#pragma unroll
      for (int qt = 0; qt < 2; ++qt) pr.p[u][qt] = bf16x8{};
    return;
  }
  softmax_phase(sc, st, pr, scale);
}

// Matrix phase: l += row sums of P, O += P V, S = K Q^T of the next step.  MASKED: the
// wave's query block may keep a unit or not (`keep`); V of one that it does not is read
// from slabs of zeros, so that what the unit holds (NaN) never reaches the block.  (A
// branch around the products made the compiler spill; its weights are zeros and the
// workgroup's other waves take the time anyway.)
template <bool MASKED>
__device__ __forceinline__ void matrix_phase(const char* lds, int k_at, int v_at, const QTiles& q,
                                             Scores& sc, const Probs& pr, TileState& st,
                                             uint32_t f, int keep, int k_scales) {
  // Fragments read ahead, 8, 10 and 12.  4,680 queries of 40 heads over 63,960 tokens:
  // 4.94, 4.83 and 4.80 ms; one frame of 12 heads over the 121-frame mask: 231, 237 and
  // 236 us, with 64-token blocks 231, 238 and 233.
  constexpr int AHEAD = MASKED ? 8 : 12;
  const char* const k = lds + k_at;
  uint32_t from[2];   // the slabs of V's units
#pragma unroll
  for (int u = 0; u < 2; ++u)
    from[u] = f + (uint32_t)(MASKED && !((keep >> u) & 1) ? ZERO_AT : v_at + u * 2 * SLAB);
  auto frag = [&](int i) {
    return *(const bf16x8*)(lds + from[i % 4 / 2] + i % 2 * SLAB + i / 4 * 1024);
  };
  // Made anew each time: kept, they would hold four registers.
  uint32_t one = 0x3F803F80u;
  asm volatile("" : "+v"(one));
  const bf16x8 ones = __builtin_bit_cast(bf16x8, u32x4{one, one, one, one});
  bf16x8 fr[32];
  i32x8 kf[8];
#pragma unroll
  for (int i = 0; i < AHEAD; ++i) fr[i] = frag(i);
  __builtin_amdgcn_sched_barrier(0);
#pragma unroll
  for (int qt = 0; qt < 2; ++qt)
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      st.l[qt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ones, pr.p[u][qt], st.l[qt], 0, 0, 0);
      __builtin_amdgcn_sched_barrier(0);
    }
  // Chains of four MFMAs into one accumulator; consecutive chains share an operand.
#pragma unroll
  for (int dt = 0; dt < 8; ++dt)
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int at = 8 * dt + 4 * t + i;
        const int u = t ? 3 - i : i, qt = t ^ (dt & 1);
        if (at % 2 == 0) {
          const int n = at / 2 + AHEAD;
          if (n < 32) fr[n] = frag(n);
          else if ((n - 32) % 4 == 0) kf[(n - 32) / 4] = k_frag(k, f, (n - 32) / 4);
        }
        st.o[dt][qt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fr[4 * dt + u], pr.p[u][qt],
                                                               st.o[dt][qt], 0, 0, 0);
        __builtin_amdgcn_sched_barrier(0);
      }
  // Scores, in such chains too: 16 keys' fragments are converted among the MFMAs of the
  // 16 before, one behind every other.
  const float scale[2] = {scale_of(k_scales, 0), scale_of(k_scales, 1)};
  auto convert = [&](int kt, int c) {
    return to_bf16(kf[kt][2 * c], kf[kt][2 * c + 1], scale[kt / 4]);
  };
  bf16x8 fk[2][4];
#pragma unroll
  for (int c = 0; c < 4; ++c) fk[0][c] = convert(0, c);
#pragma unroll
  for (int kt = 0; kt < 8; ++kt) {
    if (kt + 2 < 8) kf[kt + 2] = k_frag(k, f, kt + 2);
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int c = t ? 3 - i : i, qt = t ^ (kt & 1);
        sc.s[kt][qt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
            fk[kt % 2][c], q.f[qt][c], i ? sc.s[kt][qt] : f32x4{}, 0, 0, 0);
        if (i % 2 && kt < 7) fk[(kt + 1) % 2][2 * t + i / 2] = convert(kt + 1, 2 * t + i / 2);
        __builtin_amdgcn_sched_barrier(0);
      }
  }
}

// The union of the CSR rows block0 .. block0 + count - 1 (at most four) as words in
// `list`, ascending: key block in bits 0..27, bit 28 + r set when row r keeps it.
// `bm`: LDS for four bitmaps.  Columns outside [0, nb) are skipped and at most nb entries
// of a row are read.  Returns the number of words.
__device__ __forceinline__ int32_t union_list(uint32_t* list, uint32_t* bm, int32_t* sums,
                                              const int32_t* __restrict__ row_ptr,
                                              const int32_t* __restrict__ col_idx, int block0,
                                              int count, int nb) {
  const int tid = threadIdx.x, lane = tid % 64, wave = tid / 64;
  for (int t = tid; t < 4 * BITMAP_WORDS; t += TILE_THREADS) bm[t] = 0u;
  __syncthreads();
  for (int r = 0; r < count; ++r) {
    const int32_t lo = row_ptr[block0 + r], hi = min(row_ptr[block0 + r + 1], lo + nb);
    for (int t = lo + tid; t < hi; t += TILE_THREADS) {
      const uint32_t kb = (uint32_t)col_idx[t];
      if (kb < (uint32_t)nb) atomicOr(&bm[r * BITMAP_WORDS + kb / 32], 1u << (kb % 32));
    }
  }
  __syncthreads();
  uint32_t row[4] = {}, all = 0u;
  int32_t incl = 0;
  if (tid < BITMAP_WORDS) {
#pragma unroll
    for (int r = 0; r < 4; ++r) all |= row[r] = bm[r * BITMAP_WORDS + tid];
    incl = __popc(all);
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
      const int32_t y = __shfl_up(incl, off);
      if (lane >= off) incl += y;
    }
    if (lane == 63) sums[wave] = incl;
  }
  __syncthreads();
  int32_t total = 0, before = 0;
#pragma unroll
  for (int w = 0; w < BITMAP_WORDS / 64; ++w) {
    if (w < wave) before += sums[w];
    total += sums[w];
  }
  int32_t at = before + incl - __popc(all);
  for (uint32_t rest = all; rest; rest &= rest - 1u) {
    const int b = __ffs(rest) - 1;
    uint32_t word = (uint32_t)(32 * tid + b);
#pragma unroll
    for (int r = 0; r < 4; ++r) word |= ((row[r] >> b) & 1u) << (28 + r);
    list[at++] = word;
  }
  __syncthreads();
  return __builtin_amdgcn_readfirstlane(total);
}

// MB: the mask's block, 0 without a mask.
template <int MB>
__global__ __launch_bounds__(TILE_THREADS, 2) void tile_kernel(KernelArgs ka) {
  __shared__ __attribute__((aligned(1024))) char lds[MB ? TILE_LDS : ZERO_AT];
  const CacheAttnArgs& a = ka.a;
  const int tid = threadIdx.x, lane = tid % 64;
  const int wave = __builtin_amdgcn_readfirstlane(tid / 64);
  const int g = lane / 16, i = lane % 16;
  // Workgroups go round the eight XCDs; each takes a run of consecutive items, tiles
  // of one head first, which share keys in its L2.
  const uint32_t total = gridDim.x;
  const uint32_t xcd = blockIdx.x % 8, nth = blockIdx.x / 8;
  const uint32_t id = xcd * (total / 8) + min(xcd, total % 8) + nth;
  const int32_t tile = id % ka.p.tiles;
  const int32_t split = id / ka.p.tiles % ka.p.splits;
  const Item it = item_of(ka, tile, id / ka.p.tiles / ka.p.splits);

  // Steps of the split.
  const uint32_t* const list = (const uint32_t*)(lds + LIST_AT);
  int32_t words, n, s0 = 0;
  if constexpr (MB == 0) {
    words = (a.n_tokens + UNIT - 1) / UNIT;
    n = (words + 1) / 2;
  } else {
    words = union_list((uint32_t*)(lds + LIST_AT), (uint32_t*)(lds + V_AT),
                       (int32_t*)(lds + TILE_LDS - 64), a.row_ptr, a.col_idx, it.block0,
                       it.blocks, a.mask_blocks);
    n = MB == 128 ? words : (words + 1) / 2;
    for (int at = tid * 16; at < V_STAGE / 2; at += TILE_THREADS * 16)
      *(u32x4*)(lds + ZERO_AT + at) = u32x4{};   // read after the next barriers
  }
  s0 = (int32_t)((int64_t)n * split / ka.p.splits);
  n = (int32_t)((int64_t)n * (split + 1) / ka.p.splits) - s0;
  const int my_block = MB ? 32 * wave / (MB ? MB : 1) : 0;   // of the item's query blocks
  // Units and scales of 64 steps, a step a lane, from which a step's are read by lane:
  // memory or LDS reads in the loop would be counted together with the fragments' reads
  // (scalar loads come back in any order, so the next wait is for all of them).
  const int64_t base = (int64_t)it.kvh * a.capacity;
  const float* const ks = a.k_scale + (base >> a.scale_shift);
  const float* const vs = a.v_scale + (base >> a.scale_shift);
  uint32_t win_w[2] = {}, win_s = 0;   // words (two with 64-token blocks), scales
  auto fill_window = [&](int first) {
    const int j = s0 + min(first + fresh_lane(), n - 1);
    int32_t unit[2] = {2 * j, 2 * j + 1};
    if constexpr (MB == 128) {
      win_w[0] = list[j];
      unit[0] = 2 * (int)(win_w[0] & 0x0FFFFFFFu);
      unit[1] = unit[0] + 1;
    } else if constexpr (MB == 64) {
      win_w[0] = list[2 * j];
      win_w[1] = 2 * j + 1 < words ? list[2 * j + 1] : 0u;   // no row keeps it
      unit[0] = (int)(win_w[0] & 0x0FFFFFFFu);
      unit[1] = (int)(win_w[1] & 0x0FFFFFFFu);
    }
    win_s = 0u;
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int32_t at = (unit[u] * UNIT) >> a.scale_shift;
      const bool held = unit[u] * UNIT < a.n_tokens;   // else no write may have set them
      const uint32_t k = held ? __float_as_uint(ks[at]) >> 23 & 0xFFu : 127u;
      const uint32_t v = held ? __float_as_uint(vs[at]) >> 23 & 0xFFu : 127u;
      win_s |= k << (8 * u) | v << (16 + 8 * u);
    }
  };
  auto step_at = [&](int j) {
    Step st;
    const int in = j % 64;
    st.scales = __builtin_amdgcn_readlane((int)win_s, in);
    if constexpr (MB == 0) {
      st.unit[0] = 2 * (s0 + j);
      st.unit[1] = 2 * (s0 + j) + 1;
      st.keep = 3;
    } else if constexpr (MB == 128) {
      const uint32_t w = (uint32_t)__builtin_amdgcn_readlane((int)win_w[0], in);
      st.unit[0] = 2 * (int)(w & 0x0FFFFFFFu);
      st.unit[1] = st.unit[0] + 1;
      st.keep = ((w >> (28 + my_block)) & 1u) * 3;
    } else {
      const uint32_t w0 = (uint32_t)__builtin_amdgcn_readlane((int)win_w[0], in);
      const uint32_t w1 = (uint32_t)__builtin_amdgcn_readlane((int)win_w[1], in);
      st.unit[0] = (int)(w0 & 0x0FFFFFFFu);
      st.unit[1] = (int)(w1 & 0x0FFFFFFFu);
      st.keep = ((w0 >> (28 + my_block)) & 1u) | ((w1 >> (28 + my_block)) & 1u) << 1;
    }
#pragma unroll
    for (int u = 0; u < 2; ++u) st.left[u] = a.n_tokens - st.unit[u] * UNIT;
    return st;
  };

  // The wave's rows.
  QTiles q;
#pragma unroll
  for (int qt = 0; qt < 2; ++qt) {
    int32_t head, token;
    const bool ok = row_of(it, a, 32 * wave + 16 * qt + i, head, token);
    const __bf16* row =
        (const __bf16*)a.q + (int64_t)head * a.q_sh + (int64_t)token * a.q_st + 16 * g;
#pragma unroll
    for (int s = 0; s < 4; ++s)
      q.f[qt][s] = ok ? *(const bf16x8*)(row + (s / 2) * 64 + (s % 2) * 8) : bf16x8{};
    if (not_finite(q.f[qt])) q.f[qt][0][0] = (__bf16)__builtin_nanf("");
  }
  TileState ts;
#pragma unroll
  for (int qt = 0; qt < 2; ++qt) {
#pragma unroll
    for (int dt = 0; dt < 8; ++dt) ts.o[dt][qt] = f32x4{};
    ts.m[qt] = -__builtin_inff();
  }
  ts.l[0] = ts.l[1] = f32x4{};
  ts.flags = 0;

  if (n > 0) {
    const uint32_t lds_base = (uint32_t)(uintptr_t)(lds_void*)lds;
    const uint32_t bytes = (uint32_t)a.capacity * D;
    const uint8_t* const k_head = a.k + base * D;
    const uint8_t* const v_head = a.v + base * D;
    // Loads into LDS, 1 KiB each.  K: a wave brings in 16 keys, both slabs, of unit
    // wave / 4.  V: 16 columns d of each unit, as they lie.
    const uint32_t k_off = (uint32_t)((16 * (wave % 4) + lane / 4) * D +
                                      ((lane % 4) ^ xsw(lane / 4)) * 16);
    const uint32_t dst0 = lds_base + (uint32_t)wave * 1024u;
    auto load_k = [&](const Step& st, int stage) {
      const uint32_t so = (uint32_t)(wave / 4 ? st.unit[1] : st.unit[0]) * (UNIT * D);
      const uint32_t dst = dst0 + (uint32_t)stage * K_STAGE;
      const u32x4 rk = rsrc_of(k_head, bytes);
      load_to_lds(dst, rk, k_off, so);
      load_to_lds(dst + SLAB, rk, k_off, so + 64u);
    };
    auto load_v = [&](const Step& st) {
      const uint32_t so = (uint32_t)wave * 1024u;
      const u32x4 rv = rsrc_of(v_head, bytes);
#pragma unroll
      for (int u = 0; u < 2; ++u)
        load_to_lds(dst0 + RAW_AT + u * SLAB, rv, (uint32_t)lane * 16u,
                    (uint32_t)st.unit[u] * (UNIT * D) + so);
    };
    // The thread's 16 places (16 (tid % 4) .. of d = tid / 4) of each unit, taken from the
    // wave's raw bytes, and converted into the stage.
    const char* const raw = lds + RAW_AT + tid * 16;
    char* const v_to = lds + V_AT + (tid / 4) * 64 + ((tid % 4) ^ xsw(tid / 4)) * 16;
    auto take_v = [&](u32x4 (&w)[2]) {
      asm volatile("s_waitcnt vmcnt(2)" ::: "memory");   // all but K's loads, later ones
      w[0] = *(const u32x4*)raw;
      w[1] = *(const u32x4*)(raw + SLAB);
      // Read before the next loads into the same place are issued.
      asm volatile("s_waitcnt lgkmcnt(0)" : "+v"(w[0]), "+v"(w[1]) : : "memory");
    };
    auto store_v = [&](const Step& st, u32x4 (&w)[2], int stage) {
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const float scale = scale_of(st.scales, 2 + u);
        if (st.left[u] < UNIT) {   // bytes of tokens that are not held: zeros
          const int from = 4 * (fresh_lane() % 4);
#pragma unroll
          for (int kt = 0; kt < 4; ++kt) {
            uint32_t keep = 0u;
#pragma unroll
            for (int r = 0; r < 4; ++r)
              keep |= 16 * kt + from + r < st.left[u] ? 0xFFu << (8 * r) : 0u;
            w[u][kt] &= keep;
          }
        }
        *(bf16x8*)(v_to + stage * V_STAGE + (2 * u) * SLAB) = to_bf16(w[u][0], w[u][1], scale);
        *(bf16x8*)(v_to + stage * V_STAGE + (2 * u + 1) * SLAB) =
            to_bf16(w[u][2], w[u][3], scale);
      }
    };
    const uint32_t f = (uint32_t)(i * 64 + (g ^ xsw(i)) * 16);

    const bool lead = wave < 4;
    const float scale = ka.scale_log2;
    // V of step a is converted into stage 1 - stage, the bytes of step b are loaded.
    auto bring_v = [&](const Step& sa, const Step& sb, int stage) {
      u32x4 w[2];
      take_v(w);
      load_v(sb);
      store_v(sa, w, stage ^ 1);
    };
    // The loop begins with matrix phase -1, which has no weights and zeros for V and gives
    // the scores of step 0.  With code of its own for these scores and their softmax, 4,680
    // queries of 40 heads over 63,960 tokens took 4.48 ms instead of 4.43, 256 queries of
    // 256 heads over 32,768 tokens 910 us instead of 903; one frame over a mask the same.
    fill_window(0);
    Step s1 = step_at(0), s2 = step_at(min(1, n - 1)), s3 = step_at(min(2, n - 1));   // j + 1 ..
    load_v(s1);
    load_k(s1, 0);
    if (MB == 0)
      for (int at = tid * 16; at < V_STAGE; at += TILE_THREADS * 16)
        *(u32x4*)(lds + V_AT + V_STAGE + at) = u32x4{};
    Scores sc;
    Probs pr;
#pragma unroll
    for (int u = 0; u < 4; ++u)
#pragma unroll
      for (int qt = 0; qt < 2; ++qt) pr.p[u][qt] = bf16x8{};
    int keep = 0;   // of the step whose weights are at hand
    tile_sync<0>();
    // The others begin half a step later, with their share of V(0) and K(1).
    if (!lead) {
      load_k(s2, 1);
      bring_v(s1, s2, 1);
      tile_barrier();
    }
    // Steps j + 1, j + 2 and j + 3 become j + 2, j + 3 and j + 4.
    auto advance = [&](int j) {
      if ((j + 4) % 64 == 0 && j + 4 < n) fill_window(j + 4);
      s1 = s2;
      s2 = s3;
      s3 = step_at(min(j + 4, n - 1));
    };
    // A wave without a row only brings its share of the bytes in.
    int32_t head, token;
    if (!__builtin_amdgcn_ballot_w64(row_of(it, a, 32 * wave + lane % 32, head, token))) {
      for (int j = -1; j < n; ++j) {
        tile_sync<2>();
        if (j + 1 < n) {
          const int stage = (j & 1) ^ (lead ? 0 : 1);
          load_k(pick(lead, s2, s3), stage);
          bring_v(pick(lead, s1, s2), pick(lead, s2, s3), stage);
        }
        if (lead || j + 1 < n) tile_sync<2>();
        advance(j);
      }
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
      return;
    }
    // Both sides run the same loop: matrix phase j, then a softmax phase, the leaders'
    // of the same step (loads of j + 2), the others' of the next one (loads of j + 3).
    for (int j = -1; j < n; ++j) {
      const int even = j & 1;
      matrix_phase<MB != 0>(lds, (even ^ 1) * K_STAGE, V_AT + even * V_STAGE, q, sc, pr, ts, f,
                            keep, s1.scales);
      keep = s1.keep;
      mask_scores(sc, s1);
      tile_sync<2>();   // K's loads; V's have until the bytes are taken
      if (j + 1 < n) {
        const int stage = lead ? even : even ^ 1;
        load_k(pick(lead, s2, s3), stage);
        weigh<MB != 0>(sc, ts, pr, scale, keep);
        bring_v(pick(lead, s1, s2), pick(lead, s2, s3), stage);
      }
      if (lead)
        tile_sync<2>();
      else if (j + 1 < n)
        tile_barrier();
      advance(j);
    }
    // No load may land in LDS that is another workgroup's by then.
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  }

  // Every wave holds whole rows.  (The lane anew: rows and addresses are not kept from
  // the start.)
  const int lane2 = fresh_lane(), g2 = lane2 / 16, i2 = lane2 % 16;
  if (ka.p.splits == 1) {
#pragma unroll
    for (int qt = 0; qt < 2; ++qt) {
      int32_t head, token;
      if (!row_of(it, a, 32 * wave + 16 * qt + i2, head, token)) continue;
      const float l = ts.l[qt][0];
      const float inv = l > 0.f || l != l ? 1.f / l : 0.f;
      __bf16* const out =
          (__bf16*)a.o + (int64_t)head * a.o_sh + (int64_t)token * a.o_st + 4 * g2;
#pragma unroll
      for (int dt = 0; dt < 8; ++dt) {
        bf16x4 b;
#pragma unroll
        for (int e = 0; e < 4; ++e) b[e] = (__bf16)(ts.o[dt][qt][e] * inv);
        *(bf16x4*)(out + 16 * dt) = b;
      }
    }
    return;
  }
  const int64_t item = (int64_t)(id / ka.p.tiles / ka.p.splits) * ka.p.tiles + tile;
  const int64_t slots = (int64_t)total * TILE_ROWS;
#pragma unroll
  for (int qt = 0; qt < 2; ++qt) {
    int32_t head, token;
    if (!row_of(it, a, 32 * wave + 16 * qt + i2, head, token)) continue;
    const int64_t slot = (item * ka.p.splits + split) * TILE_ROWS + 32 * wave + 16 * qt + i2;
#pragma unroll
    for (int dt = 0; dt < 8; ++dt)
      *(f32x4*)(a.workspace + slot * D + 16 * dt + 4 * g2) = ts.o[dt][qt];
    if (g2 == 0) {
      a.workspace[slots * D + 2 * slot] = ts.m[qt];
      a.workspace[slots * D + 2 * slot + 1] = ts.l[qt][0];
    }
  }
}

// Combines the splits of the rows.  GROUPS * 32 threads a row, each taking every
// GROUPS-th split of four elements, then the groups in their order: with many splits
// their loads are on their way together (42 splits of 12 rows: 25 us one split after the
// other, 4 so).
template <int GROUPS>
__global__ __launch_bounds__(THREADS) void combine_kernel(KernelArgs ka) {
  constexpr int BLOCK_ROWS = 8 / GROUPS;
  __shared__ f32x4 part[GROUPS > 1 ? GROUPS : 1][32];
  __shared__ float part_l[GROUPS > 1 ? GROUPS : 1];
  const CacheAttnArgs& a = ka.a;
  const int32_t rows_item = ka.p.item_rows, splits = ka.p.splits;
  const int32_t blocks = rows_item / BLOCK_ROWS;      // of an item
  const int32_t id = blockIdx.x / blocks;
  const int grp = GROUPS > 1 ? threadIdx.x / 32 : 0, c = threadIdx.x % 32 * 4;
  const int r = blockIdx.x % blocks * BLOCK_ROWS + (GROUPS > 1 ? 0 : threadIdx.x / 32);
  const Item it = item_of(ka, id % ka.p.tiles, id / ka.p.tiles);
  int32_t h, t;
  if (!row_of(it, a, r, h, t)) return;
  const int64_t slots = (int64_t)(gridDim.x / blocks) * splits * rows_item;
  const int64_t slot0 = (int64_t)id * splits * rows_item + r;
  const float* const ml = a.workspace + slots * D;
  float top = -__builtin_inff();
  if (GROUPS > 1) {
    for (int s = threadIdx.x % 64; s < splits; s += 64)
      top = fmaxf(top, ml[2 * (slot0 + (int64_t)s * rows_item)]);
#pragma unroll
    for (int off = 32; off > 0; off /= 2) top = fmaxf(top, __shfl_xor(top, off));
  } else {
    for (int s = 0; s < splits; ++s)
      top = fmaxf(top, ml[2 * (slot0 + (int64_t)s * rows_item)]);
  }
  f32x4 acc = {};
  float sum = 0.f;
#pragma unroll 4
  for (int s = grp; s < splits; s += GROUPS) {
    const int64_t slot = slot0 + (int64_t)s * rows_item;
    const float ms = ml[2 * slot], ls = ml[2 * slot + 1];
    const f32x4 os = *(const f32x4*)(a.workspace + slot * D + c);
    const float f = ms == -__builtin_inff() ? 0.f : __builtin_amdgcn_exp2f(ms - top);
    sum += f * ls;
    acc += f * os;
  }
  if (GROUPS > 1) {
    part[grp][threadIdx.x % 32] = acc;
    if (c == 0) part_l[grp] = sum;
    __syncthreads();
    if (grp > 0) return;
    sum = part_l[0];
#pragma unroll
    for (int p = 1; p < GROUPS; ++p) {
      acc += part[p][threadIdx.x];
      sum += part_l[p];
    }
  }
  const float inv = sum > 0.f || sum != sum ? 1.f / sum : 0.f;
  bf16x4 b;
#pragma unroll
  for (int e = 0; e < 4; ++e) b[e] = (__bf16)(acc[e] * inv);
  *(bf16x4*)((__bf16*)a.o + (int64_t)h * a.o_sh + (int64_t)t * a.o_st + c) = b;
}

// Items of a launch, without the splits.
int64_t items_of(const Plan& p) { return (int64_t)p.heads * p.blocks * p.tiles; }

// Tiles from this many rows a key head (with a mask, which keeps a tile within one
// query head, from this many queries) on.  Rows form and tiles, us, at 32, 64, 80, 128 and
// 200 rows: 12 heads over 32,768 tokens 27/41, 36/43, 53/44, 53/47 and 91/61; 8 key
// heads of 8 query heads 27/32 (64 rows), 37/33 (72) and 62/50 (256).  Under a mask of
// 121 frames (18% of 188,760 tokens), at 32, 64, 65, 100 and 200 queries: 12 heads 25/40,
// 31/42, 45/42, 73/51 and 75/58, with 64-token blocks 33/39, 44/41, 44/41, 59/49 and 75/56;
// 8 key heads of 8 query heads 52/124, 86/128, 108/129, 276/160 and 278/176.
constexpr int64_t TILE_FROM = 65;

Plan plan_of(const CacheAttnArgs& a, int32_t cus) {
  Plan p;
  p.blocks = 1;
  p.heads = a.heads;
  int64_t rows = (int64_t)a.n * a.group;
  const int64_t units = (a.n_tokens + UNIT - 1) / UNIT;
  int32_t blocks = 1;
  if (a.row_ptr) {
    blocks = (a.q_start + a.n - 1) / a.mask_block - a.q_start / a.mask_block + 1;
    rows = (int64_t)(a.n < a.mask_block ? a.n : a.mask_block) * a.group;
  }
  p.tile = (a.row_ptr ? a.n : rows) >= TILE_FROM;
  if (p.tile) {
    p.item_rows = TILE_ROWS;
    if (a.row_ptr) {
      const int32_t per = TILE_ROWS / a.mask_block;
      p.heads = a.heads * a.group;
      p.tiles = (blocks + per - 1) / per;
    } else {
      p.tiles = (int32_t)((rows + TILE_ROWS - 1) / TILE_ROWS);
    }
    // One workgroup a compute unit: the number of splits that ends first, in steps (a
    // round of the grid takes its splits' steps and about TILE_FIXED more: 84 workgroups of
    // 2, 4 and 8 steps take 19.4, 25.6 and 38 us, with a mask 4 and 8 steps 27.8 and 41 us,
    // which is 3.1 to 3.4 us a step and 13 to 14 us; combining takes 8 to 9 us).  With a
    // mask the steps are those of every block: what its rows keep is on the device.
    constexpr int64_t TILE_FIXED = 6;
    const int64_t steps = (units + 1) / 2, items = items_of(p);
    int64_t best = 0;
    p.splits = 1;
    for (int64_t s = 1; s <= 64 && (s == 1 || s <= steps / 2); ++s) {
      const int64_t time = (items * s + cus - 1) / cus * ((steps + s - 1) / s + TILE_FIXED) +
                           (s > 1 ? TILE_FIXED : 0);
      if (s == 1 || time < best) {
        best = time;
        p.splits = (int32_t)s;
      }
    }
    return p;
  }
  p.blocks = blocks;
  p.item_rows = rows > 32 ? 64 : rows > 16 ? 32 : 16;
  p.tiles = (int32_t)((rows + p.item_rows - 1) / p.item_rows);
  // Two workgroups a compute unit; a wave's share is at least two units.
  int64_t splits = (p.item_rows > 32 ? 1 : 2) * (int64_t)cus / items_of(p);
  if (splits > units / (2 * WAVES)) splits = units / (2 * WAVES);
  p.splits = splits < 1 ? 1 : (int32_t)splits;
  return p;
}

}  // namespace

int64_t cache_attention_workspace(const CacheAttnArgs& a, int32_t cus) {
  const Plan p = plan_of(a, cus);
  return p.splits == 1 ? 0 : items_of(p) * p.splits * p.item_rows * (D + 2) * 4;
}

hipError_t launch_cache_attention(const CacheAttnArgs& a, int32_t cus, hipStream_t stream) {
  KernelArgs k;
  k.a = a;
  k.p = plan_of(a, cus);
  k.scale_log2 = 1.4426950408889634f / 11.313708498984761f;   // log2(e) / sqrt(128)
  const int64_t items = items_of(k.p);
  const dim3 grid((uint32_t)(items * k.p.splits));
  if (k.p.tile) {
    if (!a.row_ptr)
      tile_kernel<0><<<grid, TILE_THREADS, 0, stream>>>(k);
    else if (a.mask_block == 64)
      tile_kernel<64><<<grid, TILE_THREADS, 0, stream>>>(k);
    else
      tile_kernel<128><<<grid, TILE_THREADS, 0, stream>>>(k);
  } else if (k.p.item_rows == 16) {
    rows_kernel<1><<<grid, THREADS, 0, stream>>>(k);
  } else if (k.p.item_rows == 32) {
    rows_kernel<2><<<grid, THREADS, 0, stream>>>(k);
  } else {
    rows_kernel<4><<<grid, THREADS, 0, stream>>>(k);
  }
  if (hipError_t e = hipGetLastError(); e != hipSuccess || k.p.splits == 1) return e;
  if (k.p.splits > 4)
    combine_kernel<8><<<dim3((uint32_t)(items * k.p.item_rows)), THREADS, 0, stream>>>(k);
  else
    combine_kernel<1><<<dim3((uint32_t)(items * (k.p.item_rows / 8))), THREADS, 0, stream>>>(k);
  return hipGetLastError();
}

}  // namespace lvsa
