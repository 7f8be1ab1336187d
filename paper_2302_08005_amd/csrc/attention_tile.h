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

}  // namespace slapo
