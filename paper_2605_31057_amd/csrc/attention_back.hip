// attention_back.hip -- gradients of block-sparse and dense attention for gfx950.
//
//   s = q k' / sqrt(d),  p = exp(s - lse),  e = p (do v' - delta),  delta = rowsum(do o)
//   dv = p' do,  dk = e' q / sqrt(d),  dq = e k / sqrt(d)
//
// The probabilities are taken again from the scores and the rows' log-sum-exps: storing
// them would move 2 bytes a pair, 150 GB for the Wan-1.3B layer at 6x.
//
// Work decomposition
//   An item is 128 rows of two tensors ("resident": R0, R1), kept in the registers of four
//   waves, 32 rows each, and a stretch of the rows they meet, streamed in tiles of 64 rows
//   of two other tensors (X0, X1) through LDS:
//     queries  R0 = q, R1 = do, X0 = k, X1 = v: dq of 128 queries over their kept keys
//     keys     R0 = k, R1 = v,  X0 = q, X1 = do: dk and dv of 128 keys over the queries
//              that keep them
//   Both take  S = X0 R0',  T = X1 R1'  (scores and do v', [streamed][resident]), keys
//   then  dv' += X1' P  and both  (dq or dk)' += X0' E.  Scores are computed in both, 7
//   products in all for the 5 that the gradients need; adding up dq over workgroups instead
//   would take atomics (an order that changes) or all of dq's parts in memory.
//   One launch works both, the longest items first, two workgroups a compute unit.  Items
//   longer than their share of the launch are split along the streamed rows, their parts
//   left in memory in fp32 and added by combine_kernel in their order: where a few key
//   blocks are kept by every query and the others by few, and where there are few rows.
//
// Before it, prep_kernel takes what S and T begin with, -lse sqrt(d) and -delta of every
// query (so that an element takes a product, an exponential and a product), and the mask
// as bitmaps, of every query block's key blocks and, transposed, of every key block's
// query blocks; plan_kernel (for few blocks prep_kernel itself) makes the items from them.
//
// Contractions (bf16 MFMA 16x16x32, fp32 accumulate), as in attention.hip: a lane (group
// g = lane/16, i = lane%16) holds resident row i of a 16-row tile in its columns, so P and
// E go from the accumulators of S and T to the B operand of the next products without
// leaving registers, and X0 and X1 are read from LDS twice, by rows (ds_read_b128) and
// transposed (ds_read_b64_tr_b16).  P and E are rounded to bf16 there, the price of the bf16
// instruction (the rest of a number in a second product would take 7 products to 10), and
// delta is of the output as it was rounded: the unrounded one is 2 bytes an element more to
// write and to read, and would mend half of delta's part of the error (the forward pass rounds
// its probabilities too).  2.4e-3 to 2.7e-3 of the 2-norm in all, 1.7e-3 of it the results' own
// rounding.
#include <algorithm>

#include "attention_lds.h"

namespace lvsa {
namespace {

constexpr int D = 128;
constexpr int ROWS = 128;             // resident rows of a workgroup
constexpr int STEP = 64;              // streamed rows of a step
constexpr int WAVES = 4;
// Fragments read ahead of their products: as many as registers allow.
template <bool KEYS>
constexpr int AHEAD_OF = KEYS ? 3 : 4;
constexpr int SLAB = STEP * SLAB_ROW; // bytes of a slab
constexpr int TILE = 4 * SLAB;        // bytes of a streamed tile
constexpr int MAX_WORDS = (kMaxSparseBlocks + 31) / 32;   // of a bitmap
constexpr int UNIT = ROWS * D;        // floats of a part's sums: one for dq, two for dk and dv

// Costs of a step of 64 streamed rows, in products.  An item of cost c is split into c / T
// parts.  Fewer items than workgroup slots: T is the least (of FITS, each 2% above the one
// before, from a slot's share of the launch on) that leaves no more parts than slots.  A
// compute unit with one workgroup runs it nearly twice as fast as one of two, so slots left
// over cost little and a second round of few much: 8 heads of 4,096 tokens 191 us in 512
// whole items, 214 in 1,024 parts; 1 of 16,384 380 in 512 parts, 398 in 768, 449 in 640.
// More items than slots: T = (0.8 + 0.7 / rounds) shares, so that long ones end with the
// rest, but 0.6 without a mask for up to a quarter more of LONG tiles, which whole would take a
// round of their own (6 heads of 5,723 tokens, 1.05 rounds, 361 us whole, 328 so; 14 of 3,200,
// 1.37 rounds, 223 and 244; 19 of 2,000, 16 tiles, 143 and 159; under masks, whose items end
// at different times, 4 of 8,200 in 64-token blocks 199 and 211).  Never below MIN_COST
// (4 heads of 1,024 tokens 27.6 us, with 8 33, with 16 28.8).
constexpr int COST[2] = {3, 4};       // queries, keys
constexpr int MIN_COST = 12;
constexpr double SHARE = 0.8, SHARE_ROUND = 0.7, SHARE_FEW_MORE = 0.6, FEW_MORE = 1.25;
constexpr int LONG = 24;
constexpr int SLOTS = 2;              // workgroups a compute unit
constexpr int HERE = 2;               // words of a bitmap that one workgroup of prep_kernel works
constexpr int FITS = 64, FIT_ITEMS = 512;   // items of a head for which T is sought
__host__ __device__ inline int fit_at(int T, int j) { return (int)(T * exp2f(j * (1.f / 35.f))); }

enum { Q = 0, GO = 1, K = 2, V = 3, O = 4 };   // tensors read

struct Item {
  int32_t tile;      // bit 31: keys
  int32_t first;     // its stretch: blocks of its walk, from the first'th on
  int32_t count;
  int32_t unit;      // where its part goes, -1: it is the whole walk
};
struct Split {       // an item in parts
  int32_t tile, unit, parts, pad;
};
struct Plan {        // of one head, the same for all
  int32_t items, splits;
  int32_t done;      // workgroups of plan_kernel that are through
};

struct BArgs {
  const __bf16* t[5];
  int64_t sh[5], st[5];
  __bf16* g[3];              // dq, dk, dv
  int64_t g_sh[3], g_st[3];
  const float* lse;          // natural log
  // Of every query, what S and T begin with: -lse sqrt(d) (-inf for rows without keys: p
  // is 0 then) and -delta.
  float* row_lse;
  float* row_delta;
  const int32_t* row_ptr;
  const int32_t* col_idx;
  uint32_t* by_row;          // [nb][words], null without a mask
  uint32_t* by_col;          // [words][nb]
  Plan* plan;
  int32_t* counts;           // blocks of the walks, queries' tiles and then keys'
  Item* list;
  Split* splits;
  float* units;
  int32_t N, nb, block, heads, tiles, words;
  int32_t list_here;         // prep_kernel makes the list (up to 32 HERE blocks)
  int32_t stat_groups;       // prep: workgroups of 64 rows
  int32_t max_units;         // of a head
  int32_t parts[2], len[2];  // without a mask: parts of every item, blocks of each
  int32_t unit0[2];          // and where their units begin
  int32_t room;              // parts of a head that fit at once, 0: not sought
  double share;              // T: parts of a head's costs
};

__device__ __forceinline__ bf16x8 row_frag(const char* tile, uint32_t at, int row0, int stp) {
  return *(const bf16x8*)(tile + at + stp * SLAB + row0 * SLAB_ROW);
}
// (A fragment of the transposed tile, columns 16*dt .. +15 of 32 rows, is two transposing
// reads of 16 rows: k-slot e < 4 of lane group g is row 4g + e, e >= 4 row 16 + 4g + e - 4.)

// Walks `left` set bits of a bitmap (or blocks) from the first'th on, ascending.
template <bool SPARSE>
struct Walk {
  const uint32_t* words;   // LDS
  int n, word, left;
  uint32_t bits;
  __device__ __forceinline__ uint32_t at(int w) const {
    return (uint32_t)__builtin_amdgcn_readfirstlane((int)words[w]);
  }
  __device__ __forceinline__ void begin(int first) {
    if constexpr (SPARSE) {
      word = 0;
      bits = at(0);
      int c;
      while ((c = __builtin_popcount(bits)) <= first && word + 1 < n) {
        first -= c;
        bits = at(++word);
      }
      for (; first > 0; --first) bits &= bits - 1u;
    } else {
      word = first - 1;
    }
  }
  // The next block, -1 past the last.
  __device__ __forceinline__ int next() {
    if (--left < 0) return -1;
    if constexpr (!SPARSE) return ++word;
    while (bits == 0u) {
      if (++word >= n) return -1;
      bits = at(word);
    }
    const int b = __builtin_ctz(bits);
    bits &= bits - 1u;
    return 32 * word + b;
  }
};

// Four columns of a gradient's row (0: dq, 1: dk, 2: dv) from their sums.
template <int WHICH>
__device__ __forceinline__ void store_sums(const BArgs& a, int head, int row, int col, f32x4 sum) {
  bf16x4 w;
#pragma unroll
  for (int r = 0; r < 4; ++r)
    w[r] = (__bf16)(WHICH == 2 ? sum[r] : sum[r] * 0.08838834764831845f);   // 1 / sqrt(128)
  *(bf16x4*)(a.g[WHICH] + head * a.g_sh[WHICH] + row * a.g_st[WHICH] + col) = w;
}

// LDS of a workgroup.
template <bool SPARSE, int PER>
struct Lds {
  char tile[2][2][TILE];                       // [stage][X0, X1]
  float stat[2][2][STEP];                      // [stage][lse, delta] of streamed queries
  uint32_t own[SPARSE ? PER : 1][SPARSE ? MAX_WORDS : 1];   // bitmaps of the resident blocks
  uint32_t any[SPARSE && PER > 1 ? MAX_WORDS : 1];
};

template <int BLOCK, bool KEYS, bool SPARSE>
__device__ __forceinline__ void work_item(const BArgs& a, Lds<SPARSE, ROWS / BLOCK>& L, int head,
                                          int tile, int first, int count, int unit) {
  constexpr int PER = ROWS / BLOCK;      // resident blocks
  constexpr int R0 = KEYS ? K : Q, R1 = KEYS ? V : GO, X0 = KEYS ? Q : K, X1 = KEYS ? GO : V;
  const int tid = threadIdx.x, lane = tid % 64;
  const int wave = __builtin_amdgcn_readfirstlane(tid / 64);
  const int g = lane / 16, li = lane % 16;
  const int row0 = tile * ROWS;
  const int N = a.N;
  constexpr float SCALE = 0.08838834764831845f;        // 1 / sqrt(128)
  constexpr float SCALE_LOG2 = SCALE * 1.4426950408889634f;
  auto& lds = L.tile;
  auto& stat = L.stat;

  // Resident rows: columns of the products.
  const int wrow = row0 + 32 * wave;
  bf16x8 r0[4][2], r1[4][2];
  float lse[2], delta[2];
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    const int row = wrow + 16 * t + li;
#pragma unroll
    for (int stp = 0; stp < 4; ++stp) {
      const int64_t c = 32 * stp + 8 * g;
      r0[stp][t] = row < N ? *(const bf16x8*)(a.t[R0] + head * a.sh[R0] + row * a.st[R0] + c)
                           : bf16x8{};
      r1[stp][t] = row < N ? *(const bf16x8*)(a.t[R1] + head * a.sh[R1] + row * a.st[R1] + c)
                           : bf16x8{};
    }
    if constexpr (!KEYS) {
      lse[t] = row < N ? a.row_lse[(int64_t)head * N + row] : -__builtin_inff();
      delta[t] = row < N ? a.row_delta[(int64_t)head * N + row] : 0.f;
    }
  }

  // Bitmaps of the resident blocks.
  const int block0 = row0 / BLOCK;
  if constexpr (SPARSE) {
    for (int i = tid; i < a.words; i += 64 * WAVES) {
      uint32_t all = 0u;
#pragma unroll
      for (int b = 0; b < PER; ++b) {
        const uint32_t w = block0 + b >= a.nb ? 0u
                           : KEYS             ? a.by_col[(int64_t)i * a.nb + block0 + b]
                                              : a.by_row[(int64_t)(block0 + b) * a.words + i];
        L.own[b][i] = w;
        all |= w;
      }
      if (PER > 1) L.any[i] = all;
    }
    __syncthreads();
  }

  const __bf16* const x0 = a.t[X0] + head * a.sh[X0];
  const __bf16* const x1 = a.t[X1] + head * a.sh[X1];
  const float* const sl = a.row_lse + (int64_t)head * N;
  const float* const sd = a.row_delta + (int64_t)head * N;
  const uint32_t lds_base = (uint32_t)(uintptr_t)(lds_void*)&lds[0][0][0];
  const uint32_t stat_base = (uint32_t)(uintptr_t)(lds_void*)&stat[0][0][0];
  // Wave w's load j of a tile: slab j, rows 16 w + lane / 4, chunk lane % 4.
  const int lrow = 16 * wave + lane / 4;
  const uint32_t chunk = 16u * (uint32_t)((lane % 4) ^ xsw(lrow));
  const uint32_t off0 = (uint32_t)lrow * (uint32_t)(a.st[X0] * 2) + chunk;
  const uint32_t off1 = (uint32_t)lrow * (uint32_t)(a.st[X1] * 2) + chunk;
  auto bytes_at = [&](int64_t st, int row) {
    return (uint32_t)(((int64_t)(N - 1 - row) * st + D) * 2);
  };
  // Streamed rows row .. row + 63 (row < N) into stage s; rows past N come as zeros: their
  // offsets lie past the buffer's end, also where rows are less than D apart and the next
  // ones would begin before it.
  auto load_step = [&](int row, int s) {
    const uint32_t n0 = bytes_at(a.st[X0], row), n1 = bytes_at(a.st[X1], row);
    const auto q0 = make_rsrc(x0 + (int64_t)row * a.st[X0], n0);
    const auto q1 = make_rsrc(x1 + (int64_t)row * a.st[X1], n1);
    const bool there = row + lrow < N;
    const uint32_t v0 = there ? off0 : n0, v1 = there ? off1 : n1;
    const uint32_t to =
        (uint32_t)__builtin_amdgcn_readfirstlane(lds_base + 2 * TILE * s + 1024 * wave);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      issue_load(to + 4096u * j, q0, v0, 64u * j);
      issue_load(to + TILE + 4096u * j, q1, v1, 64u * j);
    }
    if (KEYS && wave < 2) {
      const float* const from = wave ? sd : sl;
      const auto q = make_rsrc(from + row, (uint32_t)(N - row) * 4u);
      issue_load_dword(
          (uint32_t)__builtin_amdgcn_readfirstlane(stat_base + 512 * s + 256 * wave), q, 4u * lane);
    }
  };

  const uint32_t at_row = li * SLAB_ROW + ((g ^ xsw(li)) * 16);
  const int vrow = 4 * g + li / 4;
  const uint32_t at_even = vrow * SLAB_ROW + ((((li % 4) / 2) ^ xsw(vrow)) * 16) + (li % 2) * 8;
  const uint32_t at_odd = at_even ^ 32u;

  f32x4 acc0[8][2], acc1[KEYS ? 8 : 1][2];
#pragma unroll
  for (int dt = 0; dt < 8; ++dt)
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      acc0[dt][t] = f32x4{};
      if (KEYS) acc1[dt][t] = f32x4{};
    }

  Walk<SPARSE> walk{SPARSE ? (PER > 1 ? L.any : L.own[0]) : nullptr, a.words, 0, count, 0u};
  walk.begin(first);
  // Steps: a block of 128 streamed rows is two of them.
  int block = walk.next(), half = 0;
  auto step_row = [&]() { return block * BLOCK + half * STEP; };
  auto advance = [&]() {
    if (BLOCK == 128 && half == 0 && block >= 0 && block * BLOCK + STEP < N) {
      half = 1;
    } else {
      half = 0;
      block = walk.next();
    }
  };
  if (block >= 0) load_step(step_row(), 0);
  for (int s = 0; block >= 0; s ^= 1) {
    const int now = block, row = step_row();
    advance();
    wait_loads_and_sync();     // this step's tiles are there, the other stage is free
    if (block >= 0) load_step(step_row(), s ^ 1);
    if (PER > 1 && SPARSE) {
      const uint32_t w = L.own[PER > 1 ? wave / 2 : 0][now / 32];
      if (!((__builtin_amdgcn_readfirstlane((int)w) >> (now % 32)) & 1)) continue;
    }
    const char* const t0 = lds[s][0];
    const char* const t1 = lds[s][1];
    // Fragments of the step, in the order of their use: for each 32 rows u the row fragments
    // of S and of T (16 rows x, 32 columns stp), then the column fragments of the gradients
    // (16 columns dt; for keys of one tensor and then of the other).  Each is read AHEAD of
    // its two products, which take the resident tiles in turn to and fro, so that products
    // that follow each other share an operand or an accumulator: the launch runs at the
    // board's power limit, and this takes 1% off it.
    constexpr int NA = 16, NB = KEYS ? 16 : 8, NF = NA + NB, AHEAD = AHEAD_OF<KEYS>;
    bf16x8 fr[2 * NF];
    i16x4 lo = i16x4{};
    auto row_of = [&](int i) {
      const int u = i / NF, f = i % NF;
      return row_frag(f / 4 % 2 ? t1 : t0, at_row, 32 * u + 16 * (f / 8), f % 4);
    };
    auto col_half = [&](int i, int half) {
      const int u = i / NF, f = i % NF - NA, dt = f % 8;
      const char* const tile = KEYS && f / 8 ? t1 : t0;
      return __builtin_amdgcn_ds_read_tr16_b64_v4i16(
          (lds_i16x4*)(tile + ((dt & 1) ? at_odd : at_even) + (dt / 2) * SLAB +
                       (32 * u + 16 * half) * SLAB_ROW));
    };
    // What goes along with product `m` of fragment i: the read of fragment i + AHEAD.
    auto carry = [&](int i, int m) {
      const int n = i + AHEAD;
      if (n >= 2 * NF) return;
      if (n % NF < NA) {
        if (m == 0) fr[n] = row_of(n);
      } else if (m == 0) {
        lo = col_half(n, 0);
      } else {
        fr[n] = join(lo, col_half(n, 1));
      }
    };
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) fr[i] = row_of(i);
    // Products go before the other workgroup's element work on the same SIMD: 1.5% of the
    // launch (12 heads of 32,760 tokens 22.40 -> 22.06 ms, interleaved on one board).
    __builtin_amdgcn_s_setprio(1);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      bf16x8 pb[2], eb[2];
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        // S and T begin with -lse / scale and -delta of their queries.
        f32x4 sc[2], tp[2];
        if constexpr (KEYS) {
          sc[0] = sc[1] = *(const f32x4*)&stat[s][0][32 * u + 16 * x + 4 * g];
          tp[0] = tp[1] = *(const f32x4*)&stat[s][1][32 * u + 16 * x + 4 * g];
        } else {
#pragma unroll
          for (int t = 0; t < 2; ++t) {
            sc[t] = f32x4{lse[t], lse[t], lse[t], lse[t]};
            tp[t] = f32x4{delta[t], delta[t], delta[t], delta[t]};
          }
        }
#pragma unroll
        for (int w = 0; w < 2; ++w)
#pragma unroll
          for (int stp = 0; stp < 4; ++stp) {
            const int i = u * NF + 8 * x + 4 * w + stp;
#pragma unroll
            for (int m = 0; m < 2; ++m) {
              const int t = m ^ (stp & 1);
              carry(i, m);
              if (w == 0)
                sc[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fr[i], r0[stp][t], sc[t], 0, 0, 0);
              else
                tp[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fr[i], r1[stp][t], tp[t], 0, 0, 0);
              __builtin_amdgcn_sched_barrier(0);
            }
          }
        __builtin_amdgcn_s_setprio(0);
        // Keys past the last: their elements are zeros, their scores would be 0.
        if (!KEYS && row + STEP > N) {
#pragma unroll
          for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int r = 0; r < 4; ++r)
              if (row + 32 * u + 16 * x + 4 * g + r >= N) sc[t][r] = -__builtin_inff();
        }
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const float p = __builtin_amdgcn_exp2f(sc[t][r] * SCALE_LOG2);
            const float e = p * tp[t][r];
            if (KEYS) pb[t][4 * x + r] = (__bf16)p;
            eb[t][4 * x + r] = (__bf16)e;
          }
        __builtin_amdgcn_s_setprio(1);
      }
#pragma unroll
      for (int f = 0; f < NB; ++f) {
        const int i = u * NF + NA + f, dt = f % 8;
#pragma unroll
        for (int m = 0; m < 2; ++m) {
          const int t = m ^ (f & 1);
          carry(i, m);
          if (KEYS && f / 8)
            acc1[dt][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fr[i], pb[t], acc1[dt][t], 0, 0, 0);
          else
            acc0[dt][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fr[i], eb[t], acc0[dt][t], 0, 0, 0);
          __builtin_amdgcn_sched_barrier(0);
        }
      }
    }
  }

  if (unit >= 0) {
    // A part: its sums as the lanes hold them.
    float* const to = a.units + ((int64_t)head * a.max_units + unit) * UNIT + 4 * lane;
#pragma unroll
    for (int dt = 0; dt < 8; ++dt)
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const int at = (wave * 16 + 2 * dt + t) * 256;
        *(f32x4*)(to + at) = acc0[dt][t];
        if constexpr (KEYS) *(f32x4*)(to + UNIT + at) = acc1[dt][t];
      }
    return;
  }
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    const int row = wrow + 16 * t + li;
    if (row >= N) continue;
#pragma unroll
    for (int dt = 0; dt < 8; ++dt) {
      store_sums<KEYS ? 1 : 0>(a, head, row, 16 * dt + 4 * g, acc0[dt][t]);
      if constexpr (KEYS) store_sums<2>(a, head, row, 16 * dt + 4 * g, acc1[dt][t]);
    }
  }
}

template <int BLOCK, bool SPARSE>
__global__ __launch_bounds__(64 * WAVES, 2) void back_kernel(const BArgs a) {
  __shared__ __attribute__((aligned(1024))) Lds<SPARSE, ROWS / BLOCK> L;
  const int head = (int)(blockIdx.x % a.heads), rank = (int)(blockIdx.x / a.heads);
  Item it;
  if constexpr (SPARSE) {
    if (rank >= a.plan->items) return;
    it = a.list[rank];
  } else {
    // Keys first: parts[1] of each tile, then queries.
    const int keys = rank < a.tiles * a.parts[1];
    const int i = keys ? rank : rank - a.tiles * a.parts[1];
    const int tile = i / a.parts[keys], part = i % a.parts[keys];
    it.tile = tile | (keys << 31);
    it.first = part * a.len[keys];
    it.count = min(a.len[keys], a.nb - it.first);
    it.unit = a.parts[keys] > 1 ? a.unit0[keys] + i * (keys + 1) : -1;
  }
  const int tile = __builtin_amdgcn_readfirstlane(it.tile) & 0x7FFFFFFF;
  const int first = __builtin_amdgcn_readfirstlane(it.first);
  const int count = __builtin_amdgcn_readfirstlane(it.count);
  const int unit = __builtin_amdgcn_readfirstlane(it.unit);
  if (__builtin_amdgcn_readfirstlane(it.tile) < 0)
    work_item<BLOCK, true, SPARSE>(a, L, head, tile, first, count, unit);
  else
    work_item<BLOCK, false, SPARSE>(a, L, head, tile, first, count, unit);
}

// Adds the parts of split items, in their order: a quarter of one gradient's tile a
// workgroup (blockIdx.y).
__global__ __launch_bounds__(64 * WAVES) void combine_kernel(const BArgs a) {
  const int head = (int)(blockIdx.x % a.heads), i = (int)(blockIdx.x / a.heads);
  const int second = blockIdx.y / 4, j0 = 4 * (blockIdx.y % 4);   // second: dv
  int tile, keys, unit, parts;
  if (a.plan) {
    if (i >= a.plan->splits) return;
    const Split s = a.splits[i];
    keys = s.tile < 0, tile = s.tile & 0x7FFFFFFF, unit = s.unit, parts = s.parts;
  } else {
    // The tiles of the kind, or kinds, that are in parts.
    keys = a.parts[1] > 1 && i < a.tiles;
    tile = i % a.tiles;
    parts = a.parts[keys];
    unit = a.unit0[keys] + tile * parts * (keys + 1);
  }
  if (second > keys) return;
  const int wave = threadIdx.x / 64, lane = threadIdx.x % 64;
  const float* from = a.units + ((int64_t)head * a.max_units + unit + second) * UNIT +
                      (wave * 16 + j0) * 256 + 4 * lane;
  f32x4 sum[4] = {f32x4{}, f32x4{}, f32x4{}, f32x4{}};
#pragma unroll 4
  for (int p = 0; p < parts; ++p, from += (keys + 1) * UNIT)
#pragma unroll
    for (int j = 0; j < 4; ++j) sum[j] += *(const f32x4*)(from + 256 * j);
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int row = tile * ROWS + 32 * wave + 16 * (j % 2) + lane % 16;
    if (row >= a.N) continue;
    const int c = 16 * ((j0 + j) / 2) + 4 * (lane / 16);
    if (!keys)
      store_sums<0>(a, head, row, c, sum[j]);
    else if (!second)
      store_sums<1>(a, head, row, c, sum[j]);
    else
      store_sums<2>(a, head, row, c, sum[j]);
  }
}

// The items of one head from the blocks of its walks, count_of(i) for item i < 2 tiles
// (queries' tiles, then keys'), the longest first, by one workgroup.  An item of cost c
// (steps times products) is split where c > T >= max(MIN_COST, share * C), C the sum of all
// costs, into at most ceil(c / T) <= 2 floor(c / T) parts.  So there are at most C / T parts more
// than items, no more split ones and at most 4 C / T units (two for a part of keys), which the
// host bounds by T's two bounds.  Order among items of like cost, and where parts lie, follow atomics; results
// do not depend on either.
struct PlanLds {
  unsigned long long total;
  int last, units, splits, fit, hist[64];
  int cost[FIT_ITEMS];
};
template <int THREADS, typename F>
__device__ __forceinline__ void make_list(const BArgs& a, PlanLds& L, F&& count_of) {
  const int tid = threadIdx.x, lane = tid % 64;
  const int steps = a.block / STEP;
  if (tid < 64) L.hist[tid] = 0;
  if (tid == 0) L.total = 0ull, L.units = 0, L.splits = 0, L.fit = FITS;
  __syncthreads();
  auto cost_of = [&](int i, int n) { return n * steps * COST[i >= a.tiles]; };
  unsigned long long sum = 0ull;
  for (int i = tid; i < 2 * a.tiles; i += THREADS) {
    const int c = cost_of(i, count_of(i));
    sum += (unsigned long long)c;
    if (a.room) L.cost[i] = c;
  }
  for (int d = 32; d; d /= 2) sum += __shfl_xor(sum, d);
  if (lane == 0) atomicAdd(&L.total, sum);
  __syncthreads();
  int T = max(MIN_COST, (int)min(a.share * (double)L.total, 1e9) + 1);
  if (a.room) {   // each wave up to the least of its T
    bool fits = false;
    for (int j = tid / 64; j < FITS && !fits; j += THREADS / 64) {
      const int t = fit_at(T, j);
      int parts = 0;
      for (int i = lane; i < 2 * a.tiles; i += 64) parts += max(1, (L.cost[i] + t - 1) / t);
      for (int d = 32; d; d /= 2) parts += __shfl_xor(parts, d);
      fits = parts <= a.room;
      if (lane == 0 && fits) atomicMin(&L.fit, j);
    }
    __syncthreads();
    if (L.fit < FITS) T = fit_at(T, L.fit);
  }
  // Parts of an item, and blocks of each.
  auto parts_of = [&](int i, int n, int& len) {
    const int c = cost_of(i, n), want = c > T ? min((c + T - 1) / T, n) : 1;
    len = (n + want - 1) / want;
    return n ? (n + len - 1) / len : 1;
  };
  // Buckets of like cost: no part costs more than T.
  const float scale = 63.f / (float)T;
  auto bucket_of = [&](int i, int len) {
    return 63 - min(63, (int)((float)cost_of(i, len) * scale));
  };
  for (int i = tid; i < 2 * a.tiles; i += THREADS) {
    int len;
    const int parts = parts_of(i, count_of(i), len);
    atomicAdd(&L.hist[bucket_of(i, len)], parts);
  }
  __syncthreads();
  if (tid < 64) {   // the buckets' first places
    const int own = L.hist[tid];
    int upto = own;
    for (int d = 1; d < 64; d *= 2) {
      const int below = __shfl_up(upto, d);
      if (tid >= d) upto += below;
    }
    L.hist[tid] = upto - own;
    if (tid == 63) a.plan->items = upto;
  }
  __syncthreads();
  for (int i = tid; i < 2 * a.tiles; i += THREADS) {
    int len;
    const int n = count_of(i), parts = parts_of(i, n, len), keys = i >= a.tiles;
    const int tile = (i - keys * a.tiles) | (keys << 31);
    int unit = -1;
    if (parts > 1) {
      unit = atomicAdd(&L.units, parts * (keys + 1));
      a.splits[atomicAdd(&L.splits, 1)] = Split{tile, unit, parts, 0};
    }
    int at = atomicAdd(&L.hist[bucket_of(i, len)], parts);
    for (int p = 0; p < parts; ++p, ++at)
      a.list[at] = Item{tile, p * len, min(len, n - p * len),
                        parts > 1 ? unit + p * (keys + 1) : -1};
  }
  __syncthreads();
  if (tid == 0) a.plan->splits = L.splits;
}

// Blocks in word w of the walk of item i.
__device__ __forceinline__ int walk_word(const BArgs& a, int i, int w) {
  const int per = ROWS / a.block, keys = i >= a.tiles, b0 = (i - keys * a.tiles) * per;
  uint32_t bits = 0u;
  for (int b = b0; b < min(b0 + per, a.nb); ++b)
    bits |= keys ? a.by_col[(int64_t)w * a.nb + b] : a.by_row[(int64_t)b * a.words + w];
  return __popc(bits);
}

// Whether this workgroup is the last of `groups` to come here.  Its thread 0's ticket
// releases what its wave has written, and acquires what the others' first waves have.
__device__ __forceinline__ bool last_group(const BArgs& a, PlanLds& L, int groups) {
  __syncthreads();
  if (threadIdx.x == 0)
    L.last = __hip_atomic_fetch_add(&a.plan->done, 1, __ATOMIC_ACQ_REL,
                                    __HIP_MEMORY_SCOPE_AGENT) == groups - 1;
  __syncthreads();
  return L.last;
}

// The first `stat_groups` workgroups: -lse sqrt(d) and -delta of 64 rows each, 16 threads a
// row.  The others: bitmaps of a block CSR, a workgroup for every 32 rows: bit kb % 32 of
// by_row[row][kb / 32], bit qb % 32 of by_col[qb / 32][col].  Entries outside [0, nb) are
// skipped, as in the forward pass.
__global__ __launch_bounds__(256) void prep_kernel(const BArgs a) {
  extern __shared__ uint32_t bits[];
  __shared__ PlanLds plan;
  __shared__ int counts[2 * 32 * HERE];
  if ((int)blockIdx.x < a.stat_groups) {
    const int c = 8 * (threadIdx.x % 16);
    bf16x8 x[4], o[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int64_t i = (int64_t)blockIdx.x * 64 + 16 * k + threadIdx.x / 16;
      const bool there = i < (int64_t)a.heads * a.N;
      const int head = there ? (int)(i / a.N) : 0, row = there ? (int)(i % a.N) : 0;
      x[k] = *(const bf16x8*)(a.t[GO] + head * a.sh[GO] + row * a.st[GO] + c);
      o[k] = *(const bf16x8*)(a.t[O] + head * a.sh[O] + row * a.st[O] + c);
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int64_t i = (int64_t)blockIdx.x * 64 + 16 * k + threadIdx.x / 16;
      float d = 0.f;
#pragma unroll
      for (int e = 0; e < 8; ++e) d = __builtin_fmaf((float)x[k][e], (float)o[k][e], d);
#pragma unroll
      for (int w = 8; w; w /= 2) d += __shfl_xor(d, w);
      if (c == 0 && i < (int64_t)a.heads * a.N) {
        const float l = a.lse[i];
        a.row_lse[i] = l == -__builtin_inff() ? l : l * -11.313708498984761f;
        a.row_delta[i] = -d;
      }
    }
    return;
  }
  if (!a.list_here && (int)blockIdx.x == a.stat_groups && threadIdx.x == 0) a.plan->done = 0;
  const int nb = a.nb, words = a.words;
  uint32_t* const rows = bits;               // [32][words]
  uint32_t* const cols = bits + 32 * words;  // [nb]
  const int own = (int)blockIdx.x - a.stat_groups;
  for (int group = own; group < (a.list_here ? words : own + 1); ++group) {
    __syncthreads();
    for (int i = threadIdx.x; i < 32 * words + nb; i += 256) bits[i] = 0u;
    __syncthreads();
    // Eight threads a row.
    const int r = threadIdx.x / 8, row = 32 * group + r;
    if (row < nb) {
      const int32_t hi = a.row_ptr[row + 1];
      for (int32_t i = a.row_ptr[row] + (int)threadIdx.x % 8; i < hi; i += 8) {
        const uint32_t kb = (uint32_t)a.col_idx[i];
        if (kb >= (uint32_t)nb) continue;
        atomicOr(&rows[r * words + kb / 32], 1u << (kb % 32));
        atomicOr(&cols[kb], 1u << r);
      }
    }
    __syncthreads();
    const int mine = min(32, nb - 32 * group) * words;
    for (int i = threadIdx.x; i < mine; i += 256)
      a.by_row[(int64_t)32 * group * words + i] = rows[i];
    for (int i = threadIdx.x; i < nb; i += 256) a.by_col[(int64_t)group * nb + i] = cols[i];
  }
  // One workgroup has all bitmaps: it makes the list too, which saves a launch (5 us of the
  // 42 of one head of 1,024 tokens; two of 4,200 in blocks of 128 47.3 -> 43.3 us; with 94
  // blocks 63.5 -> 62.3 where they are few a row and 103 -> 105 where they are many).
  if (!a.list_here) return;
  __syncthreads();
  for (int i = threadIdx.x; i < 2 * a.tiles; i += 256) {
    int n = 0;
    for (int w = 0; w < words; ++w) n += walk_word(a, i, w);
    counts[i] = n;
  }
  __syncthreads();
  make_list<256>(a, plan, [&](int i) { return counts[i]; });
}

// The list where there are many blocks: a wave counts each walk's, the workgroup that is
// through last makes the list.
constexpr int PLAN_WAVES = 16;
__global__ __launch_bounds__(64 * PLAN_WAVES) void plan_kernel(const BArgs a) {
  __shared__ PlanLds L;
  __shared__ int own[PLAN_WAVES];
  const int first = (int)blockIdx.x * PLAN_WAVES;
  const int tid = threadIdx.x, wave = tid / 64, lane = tid % 64;
  int n = 0;
  if (first + wave < 2 * a.tiles)
    for (int w = lane; w < a.words; w += 64) n += walk_word(a, first + wave, w);
  for (int d = 32; d; d /= 2) n += __shfl_xor(n, d);
  if (lane == 0) own[wave] = n;
  __syncthreads();
  // The first wave stores them all: the ticket's release waits for its wave's stores alone.
  if (tid < PLAN_WAVES && first + tid < 2 * a.tiles)
    __hip_atomic_store(&a.counts[first + tid], own[tid], __ATOMIC_RELAXED,
                       __HIP_MEMORY_SCOPE_AGENT);
  if (!last_group(a, L, (int)gridDim.x)) return;
  make_list<64 * PLAN_WAVES>(a, L, [&](int i) {
    return __hip_atomic_load(&a.counts[i], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  });
}

int64_t round_up(int64_t bytes) { return (bytes + 255) / 256 * 256; }

// How a call's work is laid out, and where in its workspace what lies.
struct Layout {
  int32_t tiles, words, slots;
  int32_t room;
  double share;
  int32_t parts[2] = {1, 1}, len[2], unit0[2] = {0, 0};
  int64_t max_items, max_splits, max_units;     // of a head
  int64_t delta, by_row, by_col, plan, counts, list, splits, units, bytes;
};

Layout layout_of(int32_t heads, int32_t n, int32_t nb, bool sparse) {
  Layout l;
  l.tiles = (int32_t)(((int64_t)n + ROWS - 1) / ROWS);
  l.words = (nb + 31) / 32;
  l.slots = SLOTS * cu_count();
  const int64_t steps = 2 * (int64_t)l.tiles;
  const int64_t cost = l.tiles * steps * (COST[0] + COST[1]);   // of a head, at most
  const double rounds = 2. * l.tiles * heads / l.slots;
  l.room = rounds <= 1. && 2 * l.tiles <= FIT_ITEMS ? l.slots / heads : 0;
  const bool few_more = !sparse && rounds < FEW_MORE && l.tiles >= LONG;
  l.share = (l.room     ? 1.
             : few_more ? SHARE_FEW_MORE
                        : SHARE + SHARE_ROUND / rounds) * heads / l.slots;
  if (sparse) {
    // C / T by make_list's two bounds of T (the first against the rounding of the division),
    // and none where no item can cost more than either: a head of 64 tokens would else take
    // 256 KB, 17 GB for 65,536 of them.
    int64_t more = std::min((int64_t)(1. / l.share * (1. + 1e-9)), cost / MIN_COST);
    if (l.share >= 1. || steps * COST[1] <= MIN_COST) more = 0;
    l.max_items = 2 * l.tiles + more;
    l.max_splits = std::min<int64_t>(2 * l.tiles, more);
    l.max_units = 4 * more;
  } else {
    int T = std::max(MIN_COST, (int)std::min(l.share * (double)cost, 1e9) + 1);
    auto parts_of = [&](int k, int t) { return (steps * COST[k] + t - 1) / t; };
    for (int j = 0; l.room && j < FITS; ++j) {
      const int t = fit_at(T, j);
      if (l.tiles * (parts_of(0, t) + parts_of(1, t)) <= l.room) {
        T = t;
        break;
      }
    }
    l.max_items = l.max_splits = l.max_units = 0;
    for (int k = 1; k >= 0; --k) {
      const int64_t want = std::min(parts_of(k, T), (int64_t)nb);
      l.len[k] = (int32_t)((nb + want - 1) / want);
      l.parts[k] = (nb + l.len[k] - 1) / l.len[k];
      l.unit0[k] = (int32_t)l.max_units;
      l.max_items += (int64_t)l.tiles * l.parts[k];
      if (l.parts[k] > 1) {
        l.max_splits += l.tiles;
        l.max_units += (int64_t)l.tiles * l.parts[k] * (k + 1);
      }
    }
  }
  const int64_t stats = round_up((int64_t)heads * n * 4);
  int64_t at = l.delta = stats;
  at += stats;
  l.by_row = at;
  if (sparse) {
    l.by_col = l.by_row + round_up((int64_t)l.words * nb * 4);
    l.plan = l.by_col + round_up((int64_t)l.words * nb * 4);
    l.counts = l.plan + round_up(sizeof(Plan));
    l.list = l.counts + round_up(2 * (int64_t)l.tiles * 4);
    l.splits = l.list + round_up(l.max_items * (int64_t)sizeof(Item));
    at = l.splits + round_up(l.max_splits * (int64_t)sizeof(Split));
  }
  l.units = at;
  l.bytes = at + heads * l.max_units * UNIT * (int64_t)sizeof(float);
  return l;
}

template <int BLOCK, bool SPARSE>
hipError_t launch_t(const BArgs& b, const Layout& l, hipStream_t stream) {
  back_kernel<BLOCK, SPARSE><<<dim3((uint32_t)(l.max_items * b.heads)), dim3(64 * WAVES), 0,
                               stream>>>(b);
  return hipGetLastError();
}

}  // namespace

int64_t attention_backward_workspace(int32_t heads, int32_t n_tokens, int32_t n_blocks,
                                     bool sparse) {
  const Layout l = layout_of(heads, n_tokens, n_blocks, sparse);
  // A launch holds less than 2^32 work-items (and there are no more split items than items).
  return l.max_items * heads >= ((int64_t)1 << 32) / (64 * WAVES) ? -1 : l.bytes;
}

hipError_t launch_attention_backward(const AttnBackArgs& a, hipStream_t stream) {
  const AttnArgs& f = a.f;
  const bool sparse = f.row_ptr != nullptr;
  const Layout l = layout_of(f.heads, f.n_tokens, f.n_blocks, sparse);
  const void* const t[5] = {f.q, a.go, f.k, f.v, f.o};
  const int64_t sh[5] = {f.q_sh, a.go_sh, f.k_sh, f.v_sh, f.o_sh};
  const int64_t st[5] = {f.q_st, a.go_st, f.k_st, f.v_st, f.o_st};
  BArgs b = {};
  for (int i = 0; i < 5; ++i) b.t[i] = (const __bf16*)t[i], b.sh[i] = sh[i], b.st[i] = st[i];
  b.g[0] = (__bf16*)a.gq, b.g_sh[0] = a.gq_sh, b.g_st[0] = a.gq_st;
  b.g[1] = (__bf16*)a.gk, b.g_sh[1] = a.gk_sh, b.g_st[1] = a.gk_st;
  b.g[2] = (__bf16*)a.gv, b.g_sh[2] = a.gv_sh, b.g_st[2] = a.gv_st;
  b.lse = f.lse;
  b.row_lse = (float*)a.workspace;
  b.row_delta = (float*)(a.workspace + l.delta);
  b.N = f.n_tokens, b.nb = f.n_blocks, b.heads = f.heads, b.tiles = l.tiles, b.words = l.words;
  b.block = a.block;
  b.list_here = l.words <= HERE;
  b.units = (float*)(a.workspace + l.units);
  b.max_units = (int32_t)l.max_units;
  b.room = l.room;
  b.share = l.share;
  for (int k = 0; k < 2; ++k)
    b.parts[k] = l.parts[k], b.len[k] = l.len[k], b.unit0[k] = l.unit0[k];
  if (sparse) {
    b.row_ptr = f.row_ptr, b.col_idx = (const int32_t*)f.rows;
    b.by_row = (uint32_t*)(a.workspace + l.by_row);
    b.by_col = (uint32_t*)(a.workspace + l.by_col);
    b.plan = (Plan*)(a.workspace + l.plan);
    b.counts = (int32_t*)(a.workspace + l.counts);
    b.list = (Item*)(a.workspace + l.list);
    b.splits = (Split*)(a.workspace + l.splits);
  }
  b.stat_groups = (int32_t)(((int64_t)f.heads * f.n_tokens + 63) / 64);
  const uint32_t lds = sparse ? (32u * l.words + f.n_blocks) * 4u : 0u;
  const int32_t mask_groups = !sparse ? 0 : b.list_here ? 1 : l.words;
  prep_kernel<<<dim3((uint32_t)(b.stat_groups + mask_groups)), dim3(256), lds, stream>>>(b);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  if (sparse) {
    if (!b.list_here) {
      plan_kernel<<<dim3((uint32_t)((2 * l.tiles + PLAN_WAVES - 1) / PLAN_WAVES)),
                    dim3(64 * PLAN_WAVES), 0, stream>>>(b);
      if ((e = hipGetLastError()) != hipSuccess) return e;
    }
    e = a.block == 64 ? launch_t<64, true>(b, l, stream) : launch_t<128, true>(b, l, stream);
  } else {
    e = launch_t<128, false>(b, l, stream);
  }
  if (e != hipSuccess || l.max_splits == 0) return e;
  combine_kernel<<<dim3((uint32_t)(l.max_splits * f.heads), 8), dim3(64 * WAVES), 0, stream>>>(b);
  return hipGetLastError();
}

}  // namespace lvsa
