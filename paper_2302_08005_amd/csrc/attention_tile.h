// What the attention kernels on 16-bit types share: tiles in LDS and their MFMA operands, direct loads of tiles, the walk over tiles.
#pragma once
#include "common.h"

namespace slapo {

constexpr float LOG2E = 1.4426950408889634f;

// ---- LDS tile [64 rows][D] of bf16, unpadded, 16-byte chunks permuted inside each row ---------------
// The LDS serves 256 B per clock (64 banks of 4 B): 16 lanes of a 16-byte read, 32 lanes of a transposing 8-byte read.
// The same tile is read both ways: 16 consecutive rows x one chunk (operand with the contraction along D), and 4
// consecutive rows x 4 chunks with the transposing read (operand with the contraction along the rows). Position p of
// row r holds chunk p ^ f(r); f is a bijection of the rows that share a chunk position (16 rows at D = 128; 8 pairs of
// rows at D = 64, whose rows are half as long as the banks), so the first kind of read meets every bank group once,
// and the bits of f that choose a group of four chunks come from the lowest bits of r, so the four rows of the second
// kind lie in different groups. (Rows padded by 16 bytes, the layout before, are conflict-free for the first kind
// only: the four rows of a transposing read overlapped in 12 of 16 banks at D = 128, and the LDS spent 50-59 % of its
// cycles on conflicts there.) A fragment address is a per-lane base with a compile-time XOR and a compile-time offset.
template <int D>
struct Tile {
  static constexpr int P = D;              // row pitch in elements
  static constexpr int ELEMS = 64 * P;     // one 64-row tile
  static __device__ __forceinline__ int f(int row) {   // of rows that are equal modulo 16 the same
    return D == 128 ? ((row & 3) << 2) | ((row >> 2) & 3) : (((row >> 1) & 1) << 2) | ((row >> 2) & 3);
  }
};
// per-lane bases, computed once per kernel
template <int D>
__device__ __forceinline__ int rows_base(int lane) {
  const int row = lane & 31;
  return row * Tile<D>::P + ((Tile<D>::f(row) ^ (lane >> 5)) << 3);
}
template <int D>
__device__ __forceinline__ int tr_base(int lane) {
  const int j = lane & 15, g = lane >> 4, row = 4 * (g >> 1) + (j >> 2);
  return row * Tile<D>::P + ((Tile<D>::f(row) ^ (2 * (g & 1) + ((j >> 1) & 1))) << 3) + 4 * (j & 1);
}
// MFMA operand whose 32 rows are tile rows r0.. (a multiple of 16) and whose contraction runs along D (step s of 16)
template <int D>
__device__ __forceinline__ bf16x8_t frag_rows(const bf16_t* tile, int base, int r0, int s) {
  return *reinterpret_cast<const bf16x8_t*>(tile + (base ^ (16 * s)) + r0 * Tile<D>::P);
}
// MFMA operand whose 32 rows are tile COLUMNS t*32.. and whose contraction runs over tile rows
// c0 + {4kc..4kc+3, 8+4kc..8+4kc+3} (kc = lane/32; c0 a multiple of 16): the order in which a 32x32 accumulator holds
// them. Eight rows further f differs in bit 1.
template <int D>
__device__ __forceinline__ bf16x8_t frag_tr(const bf16_t* tile, int base, int c0, int t) {
  const bf16_t* p0 = tile + (base ^ (32 * t)) + c0 * Tile<D>::P;
  const bf16_t* p1 = tile + (base ^ (32 * t + 16)) + (c0 + 8) * Tile<D>::P;
  s16x4_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((s16x4_t __attribute__((address_space(3)))*)p0);
  s16x4_t hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((s16x4_t __attribute__((address_space(3)))*)p1);
  typedef short s16x8_t __attribute__((ext_vector_type(8)));
  s16x8_t v = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
  return __builtin_bit_cast(bf16x8_t, v);
}
// eight accumulator registers 8h..8h+7 as a bf16 operand
template <bool F16>
__device__ __forceinline__ bf16x8_t pack8(const f32x16_t& v, int h) {
  uint4 w;
  w.x = pack2<F16>(v[8 * h + 0], v[8 * h + 1]); w.y = pack2<F16>(v[8 * h + 2], v[8 * h + 3]);
  w.z = pack2<F16>(v[8 * h + 4], v[8 * h + 5]); w.w = pack2<F16>(v[8 * h + 6], v[8 * h + 7]);
  return __builtin_bit_cast(bf16x8_t, w);
}
// (mfma16_agpr, common.h: the dK/dV kernel of 128-wide heads needs 128 registers for its two output accumulators
// alone; as ordinary registers they leave so few for operands that fragments and the K/V operands are shuttled in
// and out of spill registers inside the loop. The operands of these accumulations are packed by vector
// instructions right before, hence the default two wait states in front.)
// The value exists in ordinary registers at this point of the program: an ordering anchor for operations that
// have no side effects of their own (nothing is emitted).
__device__ __forceinline__ void pin_here(f32x16_t& v) { asm volatile("" : "+v"(v)); }
// row index inside a 32x32 accumulator tile of register r
__device__ __forceinline__ int acc_row(int r, int lane) { return (r >> 2) * 8 + 4 * (lane >> 5) + (r & 3); }

typedef unsigned int u32x4_t __attribute__((ext_vector_type(4)));

// A 64 x D tile is brought in by direct global -> LDS loads (no staging registers, no ds_write). One
// wave-level load fills 1 KB of consecutive LDS, lane l at byte 16 l: the lane fetches the chunk that the permutation
// puts there. The D/8 loads of a tile are dealt out to the four wavefronts. Rows past the end of the sequence are whatever
// follows in memory (the next sample's rows, zero past the end of the tensor: the buffer bounds): finite
// values that only ever meet masked scores.
template <int D>
struct TileDirect {
  static constexpr int SPR = D / 8;                // 16-byte chunks per row = wave-level loads per tile
  static constexpr int MINE = SPR / 4;             // loads per tile of one wavefront
  unsigned voff[MINE];
  int wave;                                        // wave-uniform
  __device__ __forceinline__ void init(int lane, int wave_uniform, unsigned row_stride_bytes) {
    wave = wave_uniform;
#pragma unroll
    for (int k = 0; k < MINE; ++k) {
      const int slot = (wave + 4 * k) * 64 + lane, row = slot / SPR, pos = slot % SPR;
      voff[k] = (unsigned)row * row_stride_bytes + (unsigned)(pos ^ Tile<D>::f(row)) * 16u;
    }
  }
  // tile rows row0.. of the operand that starts at `base` (`bytes` long from there) -> LDS tile
  __device__ __forceinline__ void issue(const bf16_t* base, unsigned bytes, bf16_t* tile, unsigned row0_bytes) const {
#pragma unroll
    for (int k = 0; k < MINE; ++k) {
      buffer_load_lds_16_untracked(base, bytes, tile + (wave + 4 * k) * 512, voff[k], row0_bytes);
    }
  }
};

// The tile loop of the forward kernel: a ring of NSTG LDS stages, tiles t+1 .. t+NSTG-1 on their way while
// tile t is computed, one barrier per tile. LPT = loads every wavefront issues per tile step:
// waiting until at most (NSTG-2)*LPT loads are outstanding leaves only younger tiles in flight (loads
// complete in issue order). On the last steps nothing is issued any more and the wait is for everything.
template <int NSTG, int LPT, typename Issue, typename Compute>
__device__ __forceinline__ void tile_ring(int n_tiles, Issue&& issue_tile, Compute&& compute) {
  static_assert(NSTG >= 2, "ring");
  if (n_tiles <= 0) return;
#pragma unroll
  for (int t = 0; t < NSTG - 1; ++t)
    if (t < n_tiles) issue_tile(t, t);
  if (n_tiles >= NSTG - 1) wait_loads_and_lds<(NSTG - 2) * LPT>();
  else wait_loads_and_lds<0>();
  block_barrier();
  for (int it0 = 0; it0 < n_tiles; it0 += NSTG) {
#pragma unroll
    for (int s = 0; s < NSTG; ++s) {   // (stages at compile time: a fragment address is a per-lane base plus an offset in the instruction)
      const int it = it0 + s;
      if (it >= n_tiles) break;        // uniform
      const bool more = it + NSTG - 1 < n_tiles;
      if (more) issue_tile((s + NSTG - 1) % NSTG, it + NSTG - 1);   // that stage was last read before the barrier that ended step it - 1
      compute(s, it);
      if (more) wait_loads_and_lds<(NSTG - 2) * LPT>();
      else wait_loads_and_lds<0>();
      block_barrier();
    }
  }
}

// Small grids (few heads, few rows) leave most of the chip idle while each block walks its tiles one after the other. Their
// blocks own 128 / G rows instead of 128 and their wavefronts form G groups that take every G-th tile of the walk (a step
// brings in G tiles); the groups' results meet in LDS. G = 2: twice the blocks, half the steps.
// Per-lane values of groups 1.. -> LDS, and back in group 0: slot [group - 1][row wavefront][register][lane].
template <int G, int REGS>
__device__ __forceinline__ float* group_slot(void* smem, int grp, int row_wave, int lane) {
  return reinterpret_cast<float*>(smem) + ((grp - 1) * (4 / G) + row_wave) * (REGS * 64) + lane;
}

// dK and dV of 32 keys, one step: a tile of 64 queries without a mask boundary, 128-wide heads. qtile, dtile: Q and dO; stats: 64 lse (in powers
// of two), 64 deltas; kf, vf: the keys and values; dk, dv: the sums, in the accumulation registers.
// One wavefront per SIMD (128-wide heads): nothing else runs while this wavefront does the softmax
// arithmetic of a sub-tile, so for tiles without a mask boundary the two sub-tiles are software-
// pipelined by hand: every MFMA is followed by the vector work of one score element of the OTHER
// sub-tile, which issues while the matrix core is busy.
//   scores(0);  scores(1) || softmax(0);  dV,dK(0) || softmax(1);  dV,dK(1)
template <bool F16>
__device__ __forceinline__ void dkdv_interior(const bf16_t* qtile, const bf16_t* dtile, const float* stats, const bf16x8_t (&kf)[8], const bf16x8_t (&vf)[8],
                                              f32x16_t (&dk)[4], f32x16_t (&dv)[4], int fr_base, int ft_base, int kc, float sl2) {
  constexpr int D = 128, NS = 8, NT = 4;
  constexpr int FB = 4;                 // k-steps of fragment prefetch
  f32x16_t sc0, dp0, sc1, dp1;
#pragma unroll
  for (int r = 0; r < 16; ++r) sc0[r] = dp0[r] = sc1[r] = dp1[r] = 0.f;
  // scores of sub-tile 0
#pragma unroll
  for (int s0 = 0; s0 < NS; s0 += FB) {
    bf16x8_t fq[FB], fd[FB];
#pragma unroll
    for (int s = 0; s < FB; ++s) {
      fq[s] = frag_rows<D>(qtile, fr_base, 0, s0 + s);
      fd[s] = frag_rows<D>(dtile, fr_base, 0, s0 + s);
    }
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int s = 0; s < FB; ++s) {
      sc0 = mfma16<F16>(fq[s], kf[s0 + s], sc0);
      dp0 = mfma16<F16>(fd[s], vf[s0 + s], dp0);
    }
    __builtin_amdgcn_sched_barrier(0);
  }
  // The 16 score elements of a sub-tile go through three steps each - a = sc * scale - lse; p = exp2(a);
  // sc = p, dp = p * (dp - delta) - and run as a pipeline beside 16 MFMAs of the OTHER sub-tile: the slot of
  // MFMA s holds step 1 of element s + 1, step 2 of element s and step 3 of element s - 1, so no vector
  // instruction waits for the result of the one in front of it (one element's steps back to back are a
  // dependent chain whose latencies nothing hides with a single wavefront per SIMD). The row statistics of
  // four elements (one float4 each of lse and delta) are read from LDS three slots ahead of their first use.
  auto pick = [](const float4& v, int e) { return e == 0 ? v.x : e == 1 ? v.y : e == 2 ? v.z : v.w; };
  auto soft_slots = [&](f32x16_t& sc, f32x16_t& dp, const float* srow, auto&& mfma_slot) {
    float4 l[2], d[2];
    l[0] = *reinterpret_cast<const float4*>(srow + 4 * kc);
    d[0] = *reinterpret_cast<const float4*>(srow + 64 + 4 * kc);
    float a_next = fmaf(sc[0], sl2, -l[0].x), p_prev = 0.f;
#pragma unroll
    for (int s = 0; s < 16; ++s) {
      const int g = s >> 2, e = s & 3;
      if (e == 1 && g + 1 < 4) {
        l[(g + 1) & 1] = *reinterpret_cast<const float4*>(srow + (g + 1) * 8 + 4 * kc);
        d[(g + 1) & 1] = *reinterpret_cast<const float4*>(srow + 64 + (g + 1) * 8 + 4 * kc);
      }
      mfma_slot(s);
      const float a_cur = a_next;
      if (s + 1 < 16) a_next = fmaf(sc[s + 1], sl2, -pick(l[((s + 1) >> 2) & 1], (s + 1) & 3));
      const float p_cur = __builtin_amdgcn_exp2f(a_cur);
      if (s > 0) {
        sc[s - 1] = p_prev;
        dp[s - 1] = p_prev * (dp[s - 1] - pick(d[((s - 1) >> 2) & 1], (s - 1) & 3));
      }
      p_prev = p_cur;
      __builtin_amdgcn_sched_barrier(0);
    }
    sc[15] = p_prev;
    dp[15] = p_prev * (dp[15] - d[1].w);
  };
  // scores of sub-tile 1 (two k-steps = four MFMAs per round) || softmax of sub-tile 0
  {
    bf16x8_t fq[2][2], fd[2][2];
#pragma unroll
    for (int k = 0; k < 2; ++k) { fq[0][k] = frag_rows<D>(qtile, fr_base, 32, k); fd[0][k] = frag_rows<D>(dtile, fr_base, 32, k); }
    soft_slots(sc0, dp0, stats, [&](int s) {
      const int g = s >> 2, e = s & 3, cur = g & 1;
      if (e == 0 && g + 1 < NS / 2) {
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          fq[cur ^ 1][k] = frag_rows<D>(qtile, fr_base, 32, 2 * g + 2 + k);
          fd[cur ^ 1][k] = frag_rows<D>(dtile, fr_base, 32, 2 * g + 2 + k);
        }
      }
      // (a compiler-visible MFMA is a pure operation that the instruction selector may move past scheduling
      // barriers - all sixteen ended up behind the softmax; the empty statement pins its result to this slot)
      if (e == 0) { sc1 = mfma16<F16>(fq[cur][0], kf[2 * g], sc1); pin_here(sc1); }
      else if (e == 1) { dp1 = mfma16<F16>(fd[cur][0], vf[2 * g], dp1); pin_here(dp1); }
      else if (e == 2) { sc1 = mfma16<F16>(fq[cur][1], kf[2 * g + 1], sc1); pin_here(sc1); }
      else { dp1 = mfma16<F16>(fd[cur][1], vf[2 * g + 1], dp1); pin_here(dp1); }
    });
  }
  // dV, dK of sub-tile 0 (four MFMAs per round) || softmax of sub-tile 1
  {
    const bf16x8_t pf[2] = {pack8<F16>(sc0, 0), pack8<F16>(sc0, 1)}, dsf[2] = {pack8<F16>(dp0, 0), pack8<F16>(dp0, 1)};
    bf16x8_t td[2][2], tq[2][2];   // [round parity][column block of the round]
#pragma unroll
    for (int k = 0; k < 2; ++k) { td[0][k] = frag_tr<D>(dtile, ft_base, 0, k); tq[0][k] = frag_tr<D>(qtile, ft_base, 0, k); }
    soft_slots(sc1, dp1, stats + 32, [&](int s) {   // round g: half h = g / 2, column blocks t = 2 (g % 2), 2 (g % 2) + 1
      const int g = s >> 2, e = s & 3, cur = g & 1, h = g >> 1, t0 = 2 * (g & 1);
      if (e == 0 && g + 1 < 4) {
        const int hn = (g + 1) >> 1, tn = 2 * ((g + 1) & 1);
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          td[cur ^ 1][k] = frag_tr<D>(dtile, ft_base, 16 * hn, tn + k);
          tq[cur ^ 1][k] = frag_tr<D>(qtile, ft_base, 16 * hn, tn + k);
        }
      }
      if (e == 0) mfma16_agpr<F16>(dv[t0], td[cur][0], pf[h]);
      else if (e == 1) mfma16_agpr<F16>(dk[t0], tq[cur][0], dsf[h]);
      else if (e == 2) mfma16_agpr<F16>(dv[t0 + 1], td[cur][1], pf[h]);
      else mfma16_agpr<F16>(dk[t0 + 1], tq[cur][1], dsf[h]);
    });
  }
  // dV, dK of sub-tile 1
  {
    const bf16x8_t pf[2] = {pack8<F16>(sc1, 0), pack8<F16>(sc1, 1)}, dsf[2] = {pack8<F16>(dp1, 0), pack8<F16>(dp1, 1)};
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      bf16x8_t td[NT], tq[NT];
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        td[t] = frag_tr<D>(dtile, ft_base, 32 + 16 * h, t);
        tq[t] = frag_tr<D>(qtile, ft_base, 32 + 16 * h, t);
      }
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int t = 0; t < NT; ++t) { mfma16_agpr<F16>(dv[t], td[t], pf[h]); mfma16_agpr<F16>(dk[t], tq[t], dsf[h]); }
      __builtin_amdgcn_sched_barrier(0);
    }
  }
}

}  // namespace slapo
