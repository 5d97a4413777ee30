// attention_back.hip -- gradients of block-sparse and dense attention for gfx950.
//
//   s = q k' / sqrt(d),  p = exp(s - lse),  e = p (do v' - delta),  delta = rowsum(do o)
//   dv = p' do,  dk = e' q / sqrt(d),  dq = e k / sqrt(d)
//
// The probabilities are taken again from the scores and the rows' log-sum-exps: storing
// them would move 2 bytes a pair, 150 GB for the Wan-1.3B layer at 6x.
//
// Work decomposition
//   Two kernels of one design.  A workgroup of four waves keeps 128 rows of two tensors
//   ("resident": R0, R1) in registers, 32 a wave, and streams 64-row tiles of two others
//   (X0, X1) through LDS:
//     queries  R0 = q, R1 = do, X0 = k, X1 = v: dq of 128 queries over their kept keys
//     keys     R0 = k, R1 = v,  X0 = q, X1 = do: dk and dv of 128 keys over the queries
//              that keep them
//   Both take  S = X0 R0',  T = X1 R1'  (scores and do v', [streamed][resident]), the keys
//   kernel then  dv' += X1' P  and both  (dq or dk)' += X0' E.  Scores are computed in
//   both, 7 products in all for the 5 that the gradients need; one kernel would have to add
//   up dq over workgroups, by atomics (an order that changes) or through memory.
//   The queries kernel runs first and leaves (lse, delta) of its rows for the keys
//   kernel; S and T begin with them (negated, lse times sqrt(d)) instead of zeros, so an
//   element takes a product, an exponential and a product.
//
// The mask is taken as bitmaps (mask_bits_kernel): of every query block's key blocks and,
// transposed, of every key block's query blocks; a workgroup walks the set bits of its
// rows' bitmaps.
//
// Contractions (bf16 MFMA 16x16x32, fp32 accumulate), as in attention.hip: a lane (group
// g = lane/16, i = lane%16) holds resident row i of a 16-row tile in its columns, so P and
// E go from the accumulators of S and T to the B operand of the next products without
// leaving registers, and X0 and X1 are read from LDS twice, by rows (ds_read_b128) and
// transposed (ds_read_b64_tr_b16).
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

// Of every query, from the queries kernel to the keys kernel: what S and T begin with, so
// that they end as (s - lse) sqrt(d) and do v' - delta.
struct Stats {
  float* lse;       // [heads][N] -lse sqrt(d), -inf for rows without keys (p = 0 then)
  float* delta;     // [heads][N] -delta
};

struct BArgs {
  const __bf16* r0;
  const __bf16* r1;
  const __bf16* x0;
  const __bf16* x1;
  const __bf16* o;           // queries kernel: the forward output
  const float* lse;          // queries kernel: natural log
  __bf16* g0;                // dq or dk
  __bf16* g1;                // dv
  int64_t r0_sh, r0_st, r1_sh, r1_st, x0_sh, x0_st, x1_sh, x1_st, o_sh, o_st;
  int64_t g0_sh, g0_st, g1_sh, g1_st;
  Stats stats;
  const uint32_t* bits;      // bitmaps of the resident blocks, null: every block
  int64_t bits_word, bits_block;   // strides of a word and of a block's bitmap
  int32_t N, nb, heads, tiles;
};

__device__ __forceinline__ bf16x8 row_frag(const char* tile, uint32_t at, int row0, int stp) {
  return *(const bf16x8*)(tile + at + stp * SLAB + row0 * SLAB_ROW);
}
// (A fragment of the transposed tile, columns 16*dt .. +15 of 32 rows, is two transposing
// reads of 16 rows: k-slot e < 4 of lane group g is row 4g + e, e >= 4 row 16 + 4g + e - 4.)

// Walks the set bits of a bitmap (or all blocks), ascending.
template <bool SPARSE>
struct Walk {
  const uint32_t* words;   // LDS
  int n;                   // blocks
  int word;
  uint32_t left;
  __device__ __forceinline__ void begin() {
    word = SPARSE ? 0 : -1;
    left = SPARSE ? (uint32_t)__builtin_amdgcn_readfirstlane((int)words[0]) : 0u;
  }
  // The next block, -1 past the last.
  __device__ __forceinline__ int next() {
    if constexpr (!SPARSE) {
      ++word;
      return word < n ? word : -1;
    } else {
      while (left == 0u) {
        if (++word >= (n + 31) / 32) return -1;
        left = (uint32_t)__builtin_amdgcn_readfirstlane((int)words[word]);
      }
      const int b = __builtin_ctz(left);
      left &= left - 1u;
      return 32 * word + b;
    }
  }
};

template <int BLOCK, bool KEYS, bool SPARSE>
__global__ __launch_bounds__(64 * WAVES, 2) void back_kernel(const BArgs a) {
  constexpr int PER = ROWS / BLOCK;      // resident blocks
  __shared__ __attribute__((aligned(1024))) char lds[2][2][TILE];
  __shared__ __attribute__((aligned(256))) float stat[2][2][STEP];
  __shared__ uint32_t own[SPARSE ? PER : 1][SPARSE ? MAX_WORDS : 1];
  __shared__ uint32_t any[SPARSE && PER > 1 ? MAX_WORDS : 1];
  const int tid = threadIdx.x, lane = tid % 64;
  const int wave = __builtin_amdgcn_readfirstlane(tid / 64);
  const int g = lane / 16, li = lane % 16;
  const int head = blockIdx.x % a.heads;
  const int row0 = (int)(blockIdx.x / a.heads) * ROWS;
  const int N = a.N;
  constexpr float SCALE = 0.08838834764831845f;        // 1 / sqrt(128)
  constexpr float SCALE_LOG2 = SCALE * 1.4426950408889634f;

  // Resident rows: columns of the products.
  const int wrow = row0 + 32 * wave;
  bf16x8 r0[4][2], r1[4][2];
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    const int row = wrow + 16 * t + li;
#pragma unroll
    for (int stp = 0; stp < 4; ++stp) {
      const int64_t c = 32 * stp + 8 * g;
      r0[stp][t] = row < N ? *(const bf16x8*)(a.r0 + head * a.r0_sh + row * a.r0_st + c) : bf16x8{};
      r1[stp][t] = row < N ? *(const bf16x8*)(a.r1 + head * a.r1_sh + row * a.r1_st + c) : bf16x8{};
    }
  }
  float lse[2], delta[2];   // -lse / scale and -delta
  if constexpr (!KEYS) {
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const int row = wrow + 16 * t + li;
      lse[t] = -__builtin_inff();
      delta[t] = 0.f;
      if (row < N) {
#pragma unroll
        for (int stp = 0; stp < 4; ++stp) {
          const bf16x8 o =
              *(const bf16x8*)(a.o + head * a.o_sh + row * a.o_st + 32 * stp + 8 * g);
#pragma unroll
          for (int k = 0; k < 8; ++k)
            delta[t] = __builtin_fmaf(-(float)o[k], (float)r1[stp][t][k], delta[t]);
        }
        const float l = a.lse[(int64_t)head * N + row];
        lse[t] = l == -__builtin_inff() ? -__builtin_inff() : l * (-1.f / SCALE);
      }
      delta[t] += __shfl_xor(delta[t], 16);
      delta[t] += __shfl_xor(delta[t], 32);
      if (row < N && g == 0) {
        a.stats.lse[(int64_t)head * N + row] = lse[t];
        a.stats.delta[(int64_t)head * N + row] = delta[t];
      }
    }
  }

  // Bitmaps of the resident blocks.
  const int words = (a.nb + 31) / 32;
  const int block0 = row0 / BLOCK;
  if constexpr (SPARSE) {
    for (int i = tid; i < words; i += 64 * WAVES) {
      uint32_t all = 0u;
#pragma unroll
      for (int b = 0; b < PER; ++b) {
        const uint32_t w = block0 + b < a.nb
                               ? a.bits[(int64_t)(block0 + b) * a.bits_block + i * a.bits_word]
                               : 0u;
        own[b][i] = w;
        all |= w;
      }
      if (PER > 1) any[i] = all;
    }
    __syncthreads();
  }

  const __bf16* const x0 = a.x0 + head * a.x0_sh;
  const __bf16* const x1 = a.x1 + head * a.x1_sh;
  const float* const sl = a.stats.lse + (int64_t)head * N;
  const float* const sd = a.stats.delta + (int64_t)head * N;
  const uint32_t lds_base = (uint32_t)(uintptr_t)(lds_void*)&lds[0][0][0];
  const uint32_t stat_base = (uint32_t)(uintptr_t)(lds_void*)&stat[0][0][0];
  // Wave w's load j of a tile: slab j, rows 16 w + lane / 4, chunk lane % 4.
  const int lrow = 16 * wave + lane / 4;
  const uint32_t chunk = 16u * (uint32_t)((lane % 4) ^ xsw(lrow));
  const uint32_t off0 = (uint32_t)lrow * (uint32_t)(a.x0_st * 2) + chunk;
  const uint32_t off1 = (uint32_t)lrow * (uint32_t)(a.x1_st * 2) + chunk;
  auto rsrc_at = [&](const __bf16* base, int64_t st, int row) {
    return make_rsrc(base + (int64_t)row * st, (uint32_t)(((int64_t)(N - 1 - row) * st + D) * 2));
  };
  // Streamed rows row .. row + 63 (row < N) into stage s.
  auto load_step = [&](int row, int s) {
    const auto q0 = rsrc_at(x0, a.x0_st, row), q1 = rsrc_at(x1, a.x1_st, row);
    const uint32_t to = (uint32_t)__builtin_amdgcn_readfirstlane(lds_base + 2 * TILE * s + 1024 * wave);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      issue_load(to + 4096u * j, q0, off0, 64u * j);
      issue_load(to + TILE + 4096u * j, q1, off1, 64u * j);
    }
    if (KEYS && wave < 2) {
      const float* const from = wave ? sd : sl;
      const auto q = make_rsrc(from + row, (uint32_t)(N - row) * 4u);
      issue_load_dword((uint32_t)__builtin_amdgcn_readfirstlane(stat_base + 512 * s + 256 * wave), q,
                       4u * lane);
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

  Walk<SPARSE> walk{SPARSE ? (PER > 1 ? any : own[0]) : nullptr, a.nb, 0, 0u};
  walk.begin();
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
      const uint32_t w = own[PER > 1 ? wave / 2 : 0][now / 32];
      if (!((__builtin_amdgcn_readfirstlane((int)w) >> (now % 32)) & 1)) continue;
    }
    const char* const t0 = lds[s][0];
    const char* const t1 = lds[s][1];
    // Fragments of the step, in the order of their use: for each 32 rows u the row fragments
    // of S and T (16 rows x, 32 columns stp, both tensors), then the column fragments of the
    // gradients (16 columns dt; both tensors in the keys kernel).  Each is read AHEAD of its
    // two products.
    constexpr int NA = 16, NB = KEYS ? 16 : 8, NF = NA + NB, AHEAD = AHEAD_OF<KEYS>;
    bf16x8 fr[2 * NF];
    i16x4 lo = i16x4{};
    auto row_of = [&](int i) {
      const int u = i / NF, f = i % NF;
      return row_frag(f % 2 ? t1 : t0, at_row, 32 * u + 16 * (f / 8), f / 2 % 4);
    };
    auto col_half = [&](int i, int half) {
      const int u = i / NF, f = i % NF - NA, dt = KEYS ? f / 2 : f;
      const char* const tile = KEYS && f % 2 ? t1 : t0;
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
        for (int stp = 0; stp < 4; ++stp)
#pragma unroll
          for (int w = 0; w < 2; ++w) {
            const int i = u * NF + 8 * x + 2 * stp + w;
#pragma unroll
            for (int t = 0; t < 2; ++t) {
              carry(i, t);
              if (w == 0)
                sc[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fr[i], r0[stp][t], sc[t], 0, 0, 0);
              else
                tp[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fr[i], r1[stp][t], tp[t], 0, 0, 0);
              __builtin_amdgcn_sched_barrier(0);
            }
          }
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
      }
#pragma unroll
      for (int f = 0; f < NB; ++f) {
        const int i = u * NF + NA + f, dt = KEYS ? f / 2 : f;
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          carry(i, t);
          if (KEYS && f % 2)
            acc1[dt][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fr[i], pb[t], acc1[dt][t], 0, 0, 0);
          else
            acc0[dt][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fr[i], eb[t], acc0[dt][t], 0, 0, 0);
          __builtin_amdgcn_sched_barrier(0);
        }
      }
    }
  }

#pragma unroll
  for (int t = 0; t < 2; ++t) {
    const int row = wrow + 16 * t + li;
    if (row >= N) continue;
    __bf16* const o0 = a.g0 + head * a.g0_sh + row * a.g0_st + 4 * g;
    __bf16* const o1 = KEYS ? a.g1 + head * a.g1_sh + row * a.g1_st + 4 * g : nullptr;
#pragma unroll
    for (int dt = 0; dt < 8; ++dt) {
      bf16x4 w;
#pragma unroll
      for (int r = 0; r < 4; ++r) w[r] = (__bf16)(acc0[dt][t][r] * SCALE);
      *(bf16x4*)(o0 + 16 * dt) = w;
      if constexpr (KEYS) {
#pragma unroll
        for (int r = 0; r < 4; ++r) w[r] = (__bf16)acc1[dt][t][r];
        *(bf16x4*)(o1 + 16 * dt) = w;
      }
    }
  }
}

// Bitmaps of a block CSR, a workgroup for every 32 rows: by_row [nb][words], bit kb % 32
// of word kb / 32; by_col [words][nb], bit qb % 32 of word qb / 32.  Entries outside
// [0, nb) are skipped, as in the forward pass.
__global__ __launch_bounds__(256) void mask_bits_kernel(const int32_t* __restrict__ row_ptr,
                                                        const int32_t* __restrict__ col_idx,
                                                        int32_t nb, uint32_t* __restrict__ by_row,
                                                        uint32_t* __restrict__ by_col) {
  __shared__ uint32_t rows[32][MAX_WORDS];
  __shared__ uint32_t cols[kMaxSparseBlocks];
  const int words = (nb + 31) / 32, first = 32 * (int)blockIdx.x;
  for (int i = threadIdx.x; i < 32 * words; i += 256) rows[i / words][i % words] = 0u;
  for (int i = threadIdx.x; i < nb; i += 256) cols[i] = 0u;
  __syncthreads();
  // Eight threads a row.
  const int r = threadIdx.x / 8, row = first + r;
  if (row < nb) {
    const int32_t lo = row_ptr[row], hi = row_ptr[row + 1];
    for (int32_t i = lo + (int)threadIdx.x % 8; i < hi; i += 8) {
      const uint32_t kb = (uint32_t)col_idx[i];
      if (kb >= (uint32_t)nb) continue;
      atomicOr(&rows[r][kb / 32], 1u << (kb % 32));
      atomicOr(&cols[kb], 1u << r);
    }
  }
  __syncthreads();
  for (int i = threadIdx.x; i < 32 * words; i += 256)
    if (first + i / words < nb) by_row[(int64_t)(first + i / words) * words + i % words] = rows[i / words][i % words];
  for (int i = threadIdx.x; i < nb; i += 256) by_col[(int64_t)blockIdx.x * nb + i] = cols[i];
}

int64_t round_up(int64_t bytes) { return (bytes + 255) / 256 * 256; }

template <int BLOCK, bool SPARSE>
hipError_t launch_t(const AttnBackArgs& a, const uint32_t* by_row, const uint32_t* by_col,
                    Stats stats, hipStream_t stream) {
  const AttnArgs& f = a.f;
  const int32_t words = (f.n_blocks + 31) / 32;
  BArgs b;
  b.N = f.n_tokens, b.nb = f.n_blocks, b.heads = f.heads;
  b.tiles = (f.n_tokens + ROWS - 1) / ROWS;
  b.stats = stats;
  b.o = (const __bf16*)f.o, b.o_sh = f.o_sh, b.o_st = f.o_st;
  b.lse = f.lse;
  const dim3 grid((uint32_t)b.tiles * (uint32_t)f.heads);
  b.r0 = (const __bf16*)f.q, b.r0_sh = f.q_sh, b.r0_st = f.q_st;
  b.r1 = (const __bf16*)a.go, b.r1_sh = a.go_sh, b.r1_st = a.go_st;
  b.x0 = (const __bf16*)f.k, b.x0_sh = f.k_sh, b.x0_st = f.k_st;
  b.x1 = (const __bf16*)f.v, b.x1_sh = f.v_sh, b.x1_st = f.v_st;
  b.g0 = (__bf16*)a.gq, b.g0_sh = a.gq_sh, b.g0_st = a.gq_st;
  b.g1 = nullptr, b.g1_sh = b.g1_st = 0;
  b.bits = by_row, b.bits_word = 1, b.bits_block = words;
  back_kernel<BLOCK, false, SPARSE><<<grid, dim3(64 * WAVES), 0, stream>>>(b);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  b.r0 = (const __bf16*)f.k, b.r0_sh = f.k_sh, b.r0_st = f.k_st;
  b.r1 = (const __bf16*)f.v, b.r1_sh = f.v_sh, b.r1_st = f.v_st;
  b.x0 = (const __bf16*)f.q, b.x0_sh = f.q_sh, b.x0_st = f.q_st;
  b.x1 = (const __bf16*)a.go, b.x1_sh = a.go_sh, b.x1_st = a.go_st;
  b.g0 = (__bf16*)a.gk, b.g0_sh = a.gk_sh, b.g0_st = a.gk_st;
  b.g1 = (__bf16*)a.gv, b.g1_sh = a.gv_sh, b.g1_st = a.gv_st;
  b.bits = by_col, b.bits_word = f.n_blocks, b.bits_block = 1;
  back_kernel<BLOCK, true, SPARSE><<<grid, dim3(64 * WAVES), 0, stream>>>(b);
  return hipGetLastError();
}

}  // namespace

int64_t attention_backward_workspace(int32_t heads, int32_t n_tokens, int32_t n_blocks,
                                     bool sparse) {
  const int64_t words = (n_blocks + 31) / 32;
  return 2 * round_up((int64_t)heads * n_tokens * 4) +
         (sparse ? 2 * round_up(words * n_blocks * 4) : 0);
}

hipError_t launch_attention_backward(const AttnBackArgs& a, hipStream_t stream) {
  const int32_t nb = a.f.n_blocks;
  const int64_t words = (nb + 31) / 32, part = round_up((int64_t)a.f.heads * a.f.n_tokens * 4);
  const Stats stats = {(float*)a.workspace, (float*)(a.workspace + part)};
  if (!a.f.row_ptr) return launch_t<128, false>(a, nullptr, nullptr, stats, stream);
  uint32_t* const by_row = (uint32_t*)(a.workspace + 2 * part);
  uint32_t* const by_col = (uint32_t*)(a.workspace + 2 * part + round_up(words * nb * 4));
  mask_bits_kernel<<<dim3((uint32_t)words), dim3(256), 0, stream>>>(
      a.f.row_ptr, (const int32_t*)a.f.rows, nb, by_row, by_col);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  return a.block == 64 ? launch_t<64, true>(a, by_row, by_col, stats, stream)
                       : launch_t<128, true>(a, by_row, by_col, stats, stream);
}

}  // namespace lvsa
