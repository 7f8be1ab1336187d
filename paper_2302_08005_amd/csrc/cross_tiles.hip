// Cross attention on 16-bit types. The arrangement of the self-attention kernels: all products on v_mfma_f32_32x32x16, "transposed"
// (S^T = K Q^T, O^T = V^T P^T, ...), so that the accumulators of the scores are the operand of the next product as they are, and the softmax
// state of a row is one scalar per lane. Sums, softmax statistics and scores are 32-bit; the probabilities, and the gradients of the scores, are
// rounded to the storage type where a matrix product takes them.
//
// A block of four wavefronts owns 128 / G rows of a (sample, key head): queries of all the heads that share the key head (CrossRows), or
// states for dK/dV. Each wavefront owns 32 rows; G groups of wavefronts own the same rows and take every G-th 64-row tile of the other
// sequence. Tiles come into two LDS stages by direct loads; what lies behind the visible states is out of the loads' bounds and arrives as zeros.
#include <algorithm>
#include <type_traits>

#include "attention_tile.h"
#include "cross_attention.h"

namespace slapo {

namespace {

// head: of all samples' key heads, sample after sample
struct CrossBlock { int x, b, h, head, split; bool none; };
// The sample with the `rank`-th most visible states (any order among equals, the same in every block).
__device__ __forceinline__ int sample_by_length(const int32_t* lens, int batch, int rank) {
  const int lane = threadIdx.x & 63, mine = lane < batch ? lens[lane] : 0;
  int longer = 0;
  for (int j = 0; j < batch; ++j) {
    const int other = __builtin_amdgcn_readlane(mine, j);
    longer += other > mine || (other == mine && j < lane) ? 1 : 0;
  }
  return __builtin_ctzll(__ballot(lane < batch && longer == rank));
}
// Which block of the work a workgroup is. Workgroups are handed to the 8 XCDs round-robin in launch order, so (sample, head, split) `unit`s are dealt out
// to the XCDs in turn, and the nx blocks of a unit sit on one XCD next to each other in time and share the tiles through its L2. Samples of
// different lengths come longest first; an XCD deals its list out to its 32 CUs, every other time backwards, so that a CU that has begun with a long
// block gets a short one beside it. Grid: cross_grid.
template <bool ORDER>
__device__ __forceinline__ CrossBlock cross_block(int nx, int splits, const CrossShape& sh, const int32_t* lens) {
  const unsigned units = (unsigned)sh.batch * sh.kv_heads * splits, count = gridDim.x >> 3;   // count: of an XCD
  unsigned i = blockIdx.x >> 3;
  const bool order = ORDER && lens && sh.batch > 1 && sh.batch <= 64;
  if (order && (i & 32) && (i | 31) < count) i ^= 31;
  unsigned u = i / nx * 8 + (blockIdx.x & 7);
  CrossBlock id;
  id.none = u >= units;
  if (id.none) return id;
  id.x = i % nx;
  id.split = u % splits;
  u /= splits;
  id.h = u % sh.kv_heads;
  id.b = u / sh.kv_heads;
  if (order) id.b = sample_by_length(lens, sh.batch, id.b);
  id.head = id.b * sh.kv_heads + id.h;
  return id;
}
int64_t cross_grid(const CrossShape& s, int nx, int splits) { return ((int64_t)s.batch * s.kv_heads * splits + 7) / 8 * 8 * nx; }
// tiles of a split: the walk cut evenly
__device__ __forceinline__ int split_begin(int n_tiles, int split, int splits) { return (int)((int64_t)n_tiles * split / splits); }

// 64-row tiles of an operand whose rows are an even stride apart (states).
template <int D>
struct StateTiles {
  static constexpr int SPR = D / 8, MINE = SPR / 4;
  unsigned voff[MINE], bytes, step;
  const bf16_t* base;
  int wave;
  // `rows` rows exist from base on
  __device__ __forceinline__ StateTiles(const bf16_t* base, int64_t stride, int rows, int lane, int wave) : base(base), wave(wave) {
    bytes = rows > 0 ? (unsigned)(((int64_t)(rows - 1) * stride + D) * 2) : 0u;
    step = (unsigned)(64 * stride * 2);
#pragma unroll
    for (int k = 0; k < MINE; ++k) {
      const int slot = (wave + 4 * k) * 64 + lane, row = slot / SPR, pos = slot % SPR;
      voff[k] = (unsigned)(row * stride * 2) + (unsigned)(pos ^ Tile<D>::f(row)) * 16u;
    }
  }
  __device__ __forceinline__ void issue(bf16_t* tile, int t) const {
#pragma unroll
    for (int k = 0; k < MINE; ++k) buffer_load_lds_16_untracked(base, bytes, tile + (wave + 4 * k) * 512, voff[k] + (unsigned)t * step, 0);
  }
};
// 64-row tiles of two operands whose rows are CrossRows (queries and the gradients of their outputs), one tile after the other.
template <int D>
struct QueryTiles {
  static constexpr int SPR = D / 8, MINE = SPR / 4;
  unsigned qoff[MINE], ooff[MINE], qbytes, obytes, qstep, ostep, qcarry, ocarry;
  int head[MINE], group, hstep, wave;
  const bf16_t *q, *o;
  __device__ __forceinline__ QueryTiles(const CrossRows& rows, const bf16_t* q, int64_t q_stride, const bf16_t* o, int64_t o_stride, int row0, int lane, int wave)
      : group(rows.group), wave(wave), q(q), o(o) {
    const int w = rows.group * D, tokens = 64 / rows.group;
    hstep = 64 - tokens * rows.group;
    qbytes = (unsigned)(((int64_t)(rows.q_len - 1) * q_stride + w) * 2);
    obytes = (unsigned)(((int64_t)(rows.q_len - 1) * o_stride + w) * 2);
    qstep = (unsigned)((tokens * q_stride + hstep * D) * 2);
    ostep = (unsigned)((tokens * o_stride + hstep * D) * 2);
    qcarry = (unsigned)((q_stride - w) * 2);   // from the last head of a token to the first of the next
    ocarry = (unsigned)((o_stride - w) * 2);
#pragma unroll
    for (int k = 0; k < MINE; ++k) {
      const int slot = (wave + 4 * k) * 64 + lane, row = slot / SPR, pos = slot % SPR, t = rows.token(row0 + row);
      const unsigned chunk = (unsigned)(pos ^ Tile<D>::f(row)) * 16u;
      head[k] = row0 + row - t * rows.group;
      qoff[k] = (unsigned)((t * q_stride + head[k] * D) * 2) + chunk;
      ooff[k] = (unsigned)((t * o_stride + head[k] * D) * 2) + chunk;
    }
  }
  __device__ __forceinline__ void issue(bf16_t* qtile, bf16_t* otile) {
#pragma unroll
    for (int k = 0; k < MINE; ++k) {
      buffer_load_lds_16_untracked(q, qbytes, qtile + (wave + 4 * k) * 512, qoff[k], 0);
      buffer_load_lds_16_untracked(o, obytes, otile + (wave + 4 * k) * 512, ooff[k], 0);
    }
#pragma unroll
    for (int k = 0; k < MINE; ++k) {   // 64 rows on
      head[k] += hstep;
      const bool carry = head[k] >= group;
      head[k] -= carry ? group : 0;
      qoff[k] += qstep + (carry ? qcarry : 0u);
      ooff[k] += ostep + (carry ? ocarry : 0u);
    }
  }
};

// A wavefront's 32 rows of output, [32][D] in its accumulators, on their way out through LDS, so that whole rows are stored (8 bytes of a lane at a
// time join those of its neighbours). value(t, e): column 32 t + 8 (e / 4) + 4 (lane / 32) + e % 4 of row lane % 32; address(r): where row r
// of the 32 starts; `rows` of them exist.
template <int D, bool F16>
struct RowStage {
  static constexpr int P = D + 4, ELEMS = 32 * P;
  static __device__ __forceinline__ void meet() {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
  }
  // the same in the room of 16 rows
  template <class Value, class Address>
  static __device__ __forceinline__ void store_halves(bf16_t* stage, int lane, int rows, Value&& value, Address&& address) {
    const int row = lane & 31, col = 4 * (lane >> 5);
    constexpr int CPR = D / 8, RPI = 64 / CPR;
    const int c = (lane % CPR) * 8;
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      meet();
      if (row >> 4 == half) {
#pragma unroll
        for (int t = 0; t < D / 32; ++t)
#pragma unroll
          for (int g = 0; g < 4; ++g)
            *reinterpret_cast<uint2*>(stage + (row & 15) * P + t * 32 + g * 8 + col) =
                make_uint2(pack2<F16>(value(t, 4 * g), value(t, 4 * g + 1)), pack2<F16>(value(t, 4 * g + 2), value(t, 4 * g + 3)));
      }
      meet();
#pragma unroll
      for (int k = 0; k < 16 / RPI; ++k) {
        const int r = k * RPI + lane / CPR;
        const uint2* p = reinterpret_cast<const uint2*>(stage + r * P + c);
        const uint2 w0 = p[0], w1 = p[1];
        if (16 * half + r < rows) *reinterpret_cast<uint4*>(address(16 * half + r) + c) = make_uint4(w0.x, w0.y, w1.x, w1.y);
      }
    }
  }
  template <class Value, class Address>
  static __device__ __forceinline__ void store(bf16_t* stage, int lane, int rows, Value&& value, Address&& address) {
    const int row = lane & 31, col = 4 * (lane >> 5);
    meet();
#pragma unroll
    for (int t = 0; t < D / 32; ++t)
#pragma unroll
      for (int g = 0; g < 4; ++g)
        *reinterpret_cast<uint2*>(stage + row * P + t * 32 + g * 8 + col) =
            make_uint2(pack2<F16>(value(t, 4 * g), value(t, 4 * g + 1)), pack2<F16>(value(t, 4 * g + 2), value(t, 4 * g + 3)));
    meet();
    constexpr int CPR = D / 8, RPI = 64 / CPR;   // 16-byte chunks per row, rows per access
    const int c = (lane % CPR) * 8;
#pragma unroll 1
    for (int r = lane / CPR; r < rows; r += RPI) {
      const uint2* p = reinterpret_cast<const uint2*>(stage + r * P + c);
      const uint2 w0 = p[0], w1 = p[1];
      *reinterpret_cast<uint4*>(address(r) + c) = make_uint4(w0.x, w0.y, w1.x, w1.y);
    }
  }
};
// The same rows as 32-bit values, packed [row][D] from `out` on.
template <int D, class Value>
__device__ __forceinline__ void store_part(float* out, int lane, int rows, Value&& value) {
  const int row = lane & 31;
  if (row >= rows) return;
  float* p = out + row * D + 4 * (lane >> 5);
#pragma unroll
  for (int t = 0; t < D / 32; ++t)
#pragma unroll
    for (int g = 0; g < 4; ++g)
      *reinterpret_cast<float4*>(p + t * 32 + g * 8) = make_float4(value(t, 4 * g), value(t, 4 * g + 1), value(t, 4 * g + 2), value(t, 4 * g + 3));
}

template <int N>
__device__ __forceinline__ void zero(f32x16_t (&v)[N]) {
#pragma unroll
  for (int t = 0; t < N; ++t)
#pragma unroll
    for (int r = 0; r < 16; ++r) v[t][r] = 0.f;
}

// Running softmax of a row (a lane holds half of it) and the output accumulated under it. Probabilities are taken against m, which follows the
// row's maximum from below: it moves when the maximum has grown by more than 2^GROWN since (and all that was accumulated is then scaled down), not
// with every tile whose maximum is a little larger (of 32 rows, one has such a tile nearly always). They are at most 2^GROWN, which every type holds.
template <int D>
struct Softmax {
  static constexpr int NT = D / 32, GROWN = 8;
  f32x16_t o[NT];
  float m = -INFINITY, l = 0.f;   // what probabilities are relative to (raw scores), sum of this lane's half
  __device__ __forceinline__ Softmax() { zero(o); }
  // GROWN in raw scores; finite, so that the first tile always moves m from -infinity
  static __device__ __forceinline__ float grown(float sl2) { return fminf(GROWN / sl2, 3e38f); }
  // 32-row sub-tiles of scores -> probabilities
  template <int SUBS>
  __device__ __forceinline__ void add(f32x16_t (&sc)[SUBS], float sl2, float grown) {
    float mx = -INFINITY;
#pragma unroll
    for (int i = 0; i < SUBS; ++i)
#pragma unroll
      for (int r = 0; r < 16; ++r) mx = fmaxf(mx, sc[i][r]);
    mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
    if (__any(mx > m + grown)) {
      const float m_new = fmaxf(m, mx), al = m_new == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((m - m_new) * sl2);
      l *= al;
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[t][r] *= al;
      m = m_new;
    }
    const float mb = m == -INFINITY ? 0.f : m * sl2;
#pragma unroll
    for (int i = 0; i < SUBS; ++i)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const float p = __builtin_amdgcn_exp2f(fmaf(sc[i][r], sl2, -mb));
        sc[i][r] = p;
        l += p;
      }
  }
  // what another wavefront has for the same rows and other states
  template <class Other>
  __device__ __forceinline__ void join(float m2, float l2, float sl2, Other&& o2) {
    const float m_new = fmaxf(m, m2);
    const float mine = m_new == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((m - m_new) * sl2);
    const float theirs = m_new == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((m2 - m_new) * sl2);
    l = l * mine + l2 * theirs;
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int r = 0; r < 16; ++r) o[t][r] = o[t][r] * mine + o2(t, r) * theirs;
    m = m_new;
  }
};

// (a sum of 0: no state was seen; one that is no number stays so)
__device__ __forceinline__ float inverse(float l) { return l != 0.f ? 1.f / l : 0.f; }
__device__ __forceinline__ float log_sum(float m, float l, float scale) { return l != 0.f ? m * scale + __logf(l) : -INFINITY; }

// Where forward's splits leave their outputs (32 bits, normalised over their own states) and logsumexps: [head][split][row][D], [head][split][row].
struct FwdParts {
  float *o, *lse;
  int splits;
  template <int D>
  __device__ __forceinline__ float* rows(int head, int split, int64_t n_rows, int64_t r) const { return o + (((int64_t)head * splits + split) * n_rows + r) * D; }
  __device__ __forceinline__ float* stat(int head, int split, int64_t n_rows, int64_t r) const { return lse + ((int64_t)head * splits + split) * n_rows + r; }
};

// =================================== forward: 128 / G rows per block ===================================
template <int D, bool F16, int G>
__global__ __launch_bounds__(256) void cross_fwd_kernel(CrossShape sh, CrossOperands p, int nx, FwdParts parts) {
  constexpr int NS = D / 16, NT = D / 32, TE = Tile<D>::ELEMS, RB = 128 / G;
  extern __shared__ __attribute__((aligned(16))) bf16_t smem[];   // [2][G][K tile | V tile]
  const CrossBlock blk = cross_block<true>(nx, parts.splits, sh, p.lens);
  if (blk.none) return;
  const int b = blk.b, h = blk.h;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), kc = lane >> 5;
  const int row_wave = wave % (4 / G), grp = G == 1 ? 0 : wave / (4 / G);
  const int fr_base = rows_base<D>(lane), ft_base = tr_base<D>(lane);
  const CrossRows rows(sh);
  const int n_rows = rows.count(), n_keys = visible(sh, p.lens, b), all_tiles = (n_keys + 63) / 64;
  const int first = split_begin(all_tiles, blk.split, parts.splits), n_tiles = split_begin(all_tiles, blk.split + 1, parts.splits) - first;
  const int wave_row = blk.x * RB + 32 * row_wave, my_row = wave_row + (lane & 31);
  const int64_t head0 = (int64_t)h * sh.group * D;
  const float sl2 = LOG2E * sh.scale, grown = Softmax<D>::grown(sl2);

  const bf16_t* q = (const bf16_t*)p.q + (int64_t)b * sh.q_len * sh.q_stride + head0 + rows.at(min(my_row, n_rows - 1), sh.q_stride, D);
  bf16x8_t qf[NS];
#pragma unroll
  for (int s = 0; s < NS; ++s) qf[s] = *reinterpret_cast<const bf16x8_t*>(q + 16 * s + 8 * kc);
  Softmax<D> sm;

  const int64_t kv0 = (int64_t)b * sh.kv_len * sh.kv_stride + h * D;
  const StateTiles<D> kt((const bf16_t*)p.k + kv0, sh.kv_stride, n_keys, lane, wave), vt((const bf16_t*)p.v + kv0, sh.kv_stride, n_keys, lane, wave);
  auto issue_step = [&](int stage, int step) {
#pragma unroll
    for (int g = 0; g < G; ++g) {
      const int t = step * G + g;
      if (t >= n_tiles) break;   // uniform
      kt.issue(smem + (stage * G + g) * 2 * TE, first + t);
      vt.issue(smem + (stage * G + g) * 2 * TE + TE, first + t);
    }
  };
  auto compute = [&](int stage, int step) {
    const int t = step * G + grp, kv0 = (first + t) * 64;
    if (G > 1 && t >= n_tiles) return;
    const bf16_t* ktile = smem + (stage * G + grp) * 2 * TE;
    const bf16_t* vtile = ktile + TE;
    f32x16_t sc[2];
    zero(sc);
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int s = 0; s < NS; ++s) sc[i] = mfma16<F16>(frag_rows<D>(ktile, fr_base, i * 32, s), qf[s], sc[i]);
    if (kv0 + 64 > n_keys) {
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r) sc[i][r] = kv0 + i * 32 + acc_row(r, lane) >= n_keys ? -INFINITY : sc[i][r];
    }
    sm.add(sc, sl2, grown);
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        const bf16x8_t pf = pack8<F16>(sc[i], half);
#pragma unroll
        for (int t = 0; t < NT; ++t) sm.o[t] = mfma16<F16>(frag_tr<D>(vtile, ft_base, i * 32 + 16 * half, t), pf, sm.o[t]);
      }
  };
  tile_ring<2, G * 2 * StateTiles<D>::MINE>((n_tiles + G - 1) / G, issue_step, compute);
  if constexpr (G > 1) {   // (the ring ends behind a barrier: the stages are free)
    constexpr int REGS = NT * 16 + 2;
    if (grp > 0) {
      float* s = group_slot<G, REGS>(smem, grp, row_wave, lane);
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int r = 0; r < 16; ++r) s[(t * 16 + r) * 64] = sm.o[t][r];
      s[NT * 16 * 64] = sm.m;
      s[(NT * 16 + 1) * 64] = sm.l;
    }
    __syncthreads();
    if (grp > 0) return;
    for (int g = 1; g < G; ++g) {
      const float* s = group_slot<G, REGS>(smem, g, row_wave, lane);
      sm.join(s[NT * 16 * 64], s[(NT * 16 + 1) * 64], sl2, [&](int t, int r) { return s[(t * 16 + r) * 64]; });
    }
  }
  const float l = sm.l + __shfl_xor(sm.l, 32, 64), inv = inverse(l);
  if (wave_row >= n_rows) return;
  const auto value = [&](int t, int e) { return sm.o[t][e] * inv; };
  const float my_lse = log_sum(sm.m, l, sh.scale);
  if (parts.splits > 1) {
    store_part<D>(parts.rows<D>(blk.head, blk.split, n_rows, wave_row), lane, n_rows - wave_row, value);
    if (kc == 0 && my_row < n_rows) *parts.stat(blk.head, blk.split, n_rows, my_row) = my_lse;
    return;
  }
  bf16_t* out = (bf16_t*)p.o + (int64_t)b * sh.q_len * sh.out_stride + head0;
  // (a group's wavefront writes over its own slot of what the groups handed it)
  bf16_t* stage = smem + row_wave * (G > 1 ? (NT * 16 + 2) * 128 : RowStage<D, F16>::ELEMS);
  RowStage<D, F16>::store(stage, lane, min(32, n_rows - wave_row), value, [&](int r) { return out + rows.at(wave_row + r, sh.out_stride, D); });
  if (p.lse && kc == 0 && my_row < n_rows) p.lse[((int64_t)b * sh.heads + h * sh.group) * sh.q_len + rows.stat(my_row)] = my_lse;
}

// ================================ forward: at most 32 rows of a head ====================================
// A token or a few that are being generated: one wavefront has all rows, and the walk over the states is all there is to share. Bound by
// reading them, so every wavefront walks tiles of 32 states of its own and waits for nobody: while one computes, the others' tiles are on
// their way. Their results meet in LDS, those of several blocks in a second kernel.
template <int D> constexpr int FEW_WAVES = D == 64 ? 16 : 8;   // (K and V tiles of all of them: 128 KB of LDS)
template <int D, bool F16>
__global__ __launch_bounds__(64 * FEW_WAVES<D>) void cross_few_kernel(CrossShape sh, CrossOperands p, FwdParts parts) {
  constexpr int NS = D / 16, NT = D / 32, TE = 32 * D, WAVES = FEW_WAVES<D>, SPR = D / 8, LOADS = SPR / 2;   // LOADS: wave-level, of 32 rows
  extern __shared__ __attribute__((aligned(16))) bf16_t smem[];   // per wavefront [K tile | V tile]
  const CrossBlock blk = cross_block<true>(1, parts.splits, sh, p.lens);
  if (blk.none) return;
  const int b = blk.b, h = blk.h;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), kc = lane >> 5;
  const int fr_base = rows_base<D>(lane), ft_base = tr_base<D>(lane);
  const CrossRows rows(sh);
  const int n_rows = rows.count(), n_keys = visible(sh, p.lens, b), all_tiles = (n_keys + 31) / 32;
  const int first = split_begin(all_tiles, blk.split, parts.splits) + wave, end = split_begin(all_tiles, blk.split + 1, parts.splits);
  const int my_row = lane & 31;
  const int64_t head0 = (int64_t)h * sh.group * D;
  const float sl2 = LOG2E * sh.scale, grown = Softmax<D>::grown(sl2);

  bf16_t *ktile = smem + wave * 2 * TE, *vtile = ktile + TE;
  const int64_t kv0 = (int64_t)b * sh.kv_len * sh.kv_stride + h * D;
  const bf16_t *k = (const bf16_t*)p.k + kv0, *v = (const bf16_t*)p.v + kv0;
  const unsigned bytes = n_keys > 0 ? (unsigned)(((int64_t)(n_keys - 1) * sh.kv_stride + D) * 2) : 0u, step = (unsigned)(32 * sh.kv_stride * 2);
  unsigned voff[LOADS];
#pragma unroll
  for (int i = 0; i < LOADS; ++i) {
    const int slot = i * 64 + lane, row = slot / SPR, pos = slot % SPR;
    voff[i] = (unsigned)(row * sh.kv_stride * 2) + (unsigned)(pos ^ Tile<D>::f(row)) * 16u;
  }
  // the room of K is free again behind the scores, that of V behind the outputs, and either is asked for the next tile at once
  auto issue = [&](const bf16_t* x, bf16_t* tile, int t) {
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // what this wavefront has read of the tile in front has arrived
    const unsigned at = (unsigned)t * step;
#pragma unroll
    for (int n = 0; n < LOADS; ++n) buffer_load_lds_16_untracked(x, bytes, tile + n * 512, voff[n] + at, 0);
  };
  if (first < end) {
    issue(k, ktile, first);
    issue(v, vtile, first);
  }
  const bf16_t* q = (const bf16_t*)p.q + (int64_t)b * sh.q_len * sh.q_stride + head0 + rows.at(min(my_row, n_rows - 1), sh.q_stride, D);
  bf16x8_t qf[NS];
#pragma unroll
  for (int s = 0; s < NS; ++s) qf[s] = *reinterpret_cast<const bf16x8_t*>(q + 16 * s + 8 * kc);
  Softmax<D> sm;
  for (int t = first; t < end; t += WAVES) {
    const bool more = t + WAVES < end;
    wait_loads_and_lds<LOADS>();   // all but V's (and, of the first tile, those of the queries, which the compiler waits for)
    asm volatile("" ::: "memory");
    f32x16_t sc[1];
    zero(sc);
#pragma unroll
    for (int s = 0; s < NS; ++s) sc[0] = mfma16<F16>(frag_rows<D>(ktile, fr_base, 0, s), qf[s], sc[0]);
    if (more) issue(k, ktile, t + WAVES);
    if (32 * t + 32 > n_keys) {
#pragma unroll
      for (int r = 0; r < 16; ++r) sc[0][r] = 32 * t + acc_row(r, lane) >= n_keys ? -INFINITY : sc[0][r];
    }
    sm.add(sc, sl2, grown);
    if (more) wait_loads_and_lds<LOADS>();   // all but the next tile's K
    else wait_loads_and_lds<0>();
    asm volatile("" ::: "memory");
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      const bf16x8_t pf = pack8<F16>(sc[0], half);
#pragma unroll
      for (int c = 0; c < NT; ++c) sm.o[c] = mfma16<F16>(frag_tr<D>(vtile, ft_base, 16 * half, c), pf, sm.o[c]);
    }
    if (more) issue(v, vtile, t + WAVES);
  }
  // every wavefront puts some of the accumulators of all together: registers REGS w .. of the 16 NT
  __syncthreads();
  constexpr int REGS = 16 * NT / WAVES, SLOT = 16 * NT + 2;
  static_assert(REGS % 2 == 0 && 16 % REGS == 0, "whole pairs of columns, of one 32-column block");
  float* slots = reinterpret_cast<float*>(smem) + lane;
  {
    float* s = slots + wave * SLOT * 64;
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int r = 0; r < 16; ++r) s[(t * 16 + r) * 64] = sm.o[t][r];
    s[16 * NT * 64] = sm.m;
    s[(16 * NT + 1) * 64] = sm.l + __shfl_xor(sm.l, 32, 64);
  }
  __syncthreads();
  if (my_row >= n_rows) return;
  float m = -INFINITY, l = 0.f, o[REGS];
#pragma unroll
  for (int w = 0; w < WAVES; ++w) m = fmaxf(m, slots[(w * SLOT + 16 * NT) * 64]);
  const float base = m == -INFINITY ? 0.f : m * sl2;
#pragma unroll
  for (int r = 0; r < REGS; ++r) o[r] = 0.f;
#pragma unroll
  for (int w = 0; w < WAVES; ++w) {
    const float weight = __builtin_amdgcn_exp2f(fmaf(slots[(w * SLOT + 16 * NT) * 64], sl2, -base));
    l = fmaf(weight, slots[(w * SLOT + 16 * NT + 1) * 64], l);
#pragma unroll
    for (int r = 0; r < REGS; ++r) o[r] = fmaf(weight, slots[(w * SLOT + wave * REGS + r) * 64], o[r]);
  }
  const float inv = inverse(l), my_lse = log_sum(m, l, sh.scale);
  const int reg = wave * REGS % 16, col = wave * REGS / 16 * 32 + 8 * (reg / 4) + 4 * kc + reg % 4;   // of o[0]
  bf16_t* out = (bf16_t*)p.o + (int64_t)b * sh.q_len * sh.out_stride + head0 + rows.at(my_row, sh.out_stride, D) + col;
  float* part = parts.splits > 1 ? parts.rows<D>(blk.head, blk.split, n_rows, my_row) + col : nullptr;
#pragma unroll
  for (int r = 0; r < REGS; r += 2) {   // (registers 4 g .. 4 g + 3: consecutive columns; the next four eight columns on)
    const int c = r / 4 * 8 + r % 4;
    if (part) *reinterpret_cast<float2*>(part + c) = make_float2(o[r] * inv, o[r + 1] * inv);
    else *reinterpret_cast<uint32_t*>(out + c) = pack2<F16>(o[r] * inv, o[r + 1] * inv);
  }
  if (wave == 0 && kc == 0) {
    if (part) *parts.stat(blk.head, blk.split, n_rows, my_row) = my_lse;
    else if (p.lse) p.lse[((int64_t)b * sh.heads + h * sh.group) * sh.q_len + rows.stat(my_row)] = my_lse;
  }
}

// Puts the splits of a row together, by their logsumexps: eight columns per thread; `groups` threads share the splits of a row, one or two each as far as
// a block's threads go, and put theirs together through LDS.
constexpr int MAX_SPLITS = 64;
template <int D> constexpr int JOIN_GROUPS = 256 / (D / 8);   // at most
template <int D, bool F16>
__global__ __launch_bounds__(256) void cross_join_kernel(CrossShape sh, CrossOperands p, FwdParts parts, int groups) {
  constexpr int C = D / 8;
  __shared__ float4 sums[2 * 256];
  __shared__ float2 stats[256];
  const CrossRows rows(sh);
  const int n_rows = rows.count(), tid = threadIdx.x, c = 8 * (tid % C), g = tid / C % groups;
  const int64_t all = (int64_t)sh.batch * sh.kv_heads * n_rows, row = (int64_t)blockIdx.x * (256 / (C * groups)) + tid / (C * groups);
  const int64_t my_row = row < all ? row : all - 1;
  const int head = (int)(my_row / n_rows), r = (int)(my_row - (int64_t)head * n_rows), b = head / sh.kv_heads, h = head - b * sh.kv_heads;
  const float* lse = parts.stat(head, 0, n_rows, r);
  const float* src = parts.rows<D>(head, 0, n_rows, r) + c;
  float m = -INFINITY, total = 0.f, o[8] = {};
  for (int s = g; s < parts.splits; s += groups) m = fmaxf(m, lse[(int64_t)s * n_rows]);
  const float base = m == -INFINITY ? 0.f : m;
#pragma unroll 2
  for (int s = g; s < parts.splits; s += groups) {
    const float weight = __expf(lse[(int64_t)s * n_rows] - base);
    float v[8];
    load8(src + (int64_t)s * n_rows * D, v);
    total += weight;
#pragma unroll
    for (int e = 0; e < 8; ++e) o[e] = fmaf(weight, v[e], o[e]);
  }
  for (int half = groups >> 1; half > 0; half >>= 1) {
    if (g >= half && g < 2 * half) {
      stats[tid] = make_float2(m, total);
      sums[tid] = make_float4(o[0], o[1], o[2], o[3]);
      sums[256 + tid] = make_float4(o[4], o[5], o[6], o[7]);
    }
    __syncthreads();
    if (g < half) {
      const int other = tid + half * C;
      const float2 st = stats[other];
      const float4 x = sums[other], y = sums[256 + other];
      const float theirs[8] = {x.x, x.y, x.z, x.w, y.x, y.y, y.z, y.w};
      const float top = fmaxf(m, st.x), from = top == -INFINITY ? 0.f : top, wm = __expf(m - from), wt = __expf(st.x - from);
      total = total * wm + st.y * wt;
#pragma unroll
      for (int e = 0; e < 8; ++e) o[e] = o[e] * wm + theirs[e] * wt;
      m = top;
    }
    __syncthreads();
  }
  if (g != 0 || row >= all) return;
  const float inv = inverse(total);
#pragma unroll
  for (int e = 0; e < 8; ++e) o[e] *= inv;
  store8h<F16>((bf16_t*)p.o + (int64_t)b * sh.q_len * sh.out_stride + (int64_t)h * sh.group * D + rows.at(r, sh.out_stride, D) + c, o);
  if (p.lse && c == 0) p.lse[((int64_t)b * sh.heads + h * sh.group) * sh.q_len + rows.stat(r)] = log_sum(m, total, 1.f);
}

// ======================================== backward ======================================================
// 32-bit parts of gradients that several blocks share: [part][head][array][row][D].
struct BwdParts {
  float* o;
  int splits;
  float* off;   // of dq: [split][head][row] sums of the scores' gradients
  template <int D>
  __device__ __forceinline__ float* rows(int head, int heads, int split, int arrays, int array, int64_t n_rows, int64_t r) const {
    return o + ((((int64_t)split * heads + head) * arrays + array) * n_rows + r) * D;
  }
};

// dQ of 128 / G rows. Also leaves delta of its rows, laid out as lse, for the kernel of dK and dV.
// delta = rowsum(dO * O), of the stored O, whose rounding is a third of what the scores' gradients as the matrix instructions' operands (16 bits) put
// into dQ. Where a lane has registers for it (not 128-wide heads at two wavefronts per SIMD) it is taken out again: the gradients of a row's scores add
// up to 0, so what they do add up to is what delta lacks, and dQ gets as much of sum p K, a fourth product, less. Error of dQ, in units of what rounding
// the result costs, and us, without / with: 8 x 512 rows, 1024 states, 16 heads of 64 1.495 / 1.444, 28.9 / 33.3; 5 x 1143, 777, 4 in IEEE half 1.504 /
// 1.436, 14.0 / 15.5.
template <int D, bool F16, int G>
__global__ __launch_bounds__(256, D == 128 && G == 1 ? 2 : 1) void cross_dq_kernel(CrossShape sh, CrossOperands p, int nx, float* __restrict__ delta, BwdParts parts) {
  constexpr int NS = D / 16, NT = D / 32, TE = Tile<D>::ELEMS, RB = 128 / G;
  extern __shared__ __attribute__((aligned(16))) bf16_t smem[];   // [2][G][K tile | V tile]
  const CrossBlock blk = cross_block<true>(nx, parts.splits, sh, p.lens);
  if (blk.none) return;
  const int b = blk.b, h = blk.h;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), kc = lane >> 5;
  const int row_wave = wave % (4 / G), grp = G == 1 ? 0 : wave / (4 / G);
  const int fr_base = rows_base<D>(lane), ft_base = tr_base<D>(lane);
  const CrossRows rows(sh);
  const int n_rows = rows.count(), n_keys = visible(sh, p.lens, b), all_tiles = (n_keys + 63) / 64;
  const int first = split_begin(all_tiles, blk.split, parts.splits), n_tiles = split_begin(all_tiles, blk.split + 1, parts.splits) - first;
  const int wave_row = blk.x * RB + 32 * row_wave, my_row = wave_row + (lane & 31), ld_row = min(my_row, n_rows - 1);
  const int64_t head0 = (int64_t)h * sh.group * D, stat = ((int64_t)b * sh.heads + h * sh.group) * sh.q_len + rows.stat(ld_row);
  const float sl2 = LOG2E * sh.scale;

  const bf16_t* q = (const bf16_t*)p.q + (int64_t)b * sh.q_len * sh.q_stride + head0 + rows.at(ld_row, sh.q_stride, D);
  const int64_t out0 = (int64_t)b * sh.q_len * sh.out_stride + head0 + rows.at(ld_row, sh.out_stride, D);
  bf16x8_t qf[NS], df[NS];
#pragma unroll
  for (int s = 0; s < NS; ++s) {
    qf[s] = *reinterpret_cast<const bf16x8_t*>(q + 16 * s + 8 * kc);
    df[s] = *reinterpret_cast<const bf16x8_t*>((const bf16_t*)p.dout + out0 + 16 * s + 8 * kc);
  }
  const float my_lse2 = p.lse[stat] * LOG2E;
  // the lane holds half of the row's dO, lane ^ 32 the other half
  float my_delta = 0.f;
#pragma unroll
  for (int s = 0; s < NS; ++s) {
    const bf16x8_t of = *reinterpret_cast<const bf16x8_t*>((const bf16_t*)p.out + out0 + 16 * s + 8 * kc);
    const u32x4_t ow = __builtin_bit_cast(u32x4_t, of), dw = __builtin_bit_cast(u32x4_t, df[s]);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      my_delta = fmaf(unpack_lo<F16>(ow[e]), unpack_lo<F16>(dw[e]), my_delta);
      my_delta = fmaf(unpack_hi<F16>(ow[e]), unpack_hi<F16>(dw[e]), my_delta);
    }
  }
  my_delta += __shfl_xor(my_delta, 32, 64);
  constexpr bool EXACT = D == 64 || G == 2;
  f32x16_t dq[NT], pk[EXACT ? NT : 1];
  zero(dq);
  zero(pk);
  float off = 0.f;

  const int64_t kv0 = (int64_t)b * sh.kv_len * sh.kv_stride + h * D;
  const StateTiles<D> kt((const bf16_t*)p.k + kv0, sh.kv_stride, n_keys, lane, wave), vt((const bf16_t*)p.v + kv0, sh.kv_stride, n_keys, lane, wave);
  auto issue_step = [&](int stage, int step) {
#pragma unroll
    for (int g = 0; g < G; ++g) {
      const int t = step * G + g;
      if (t >= n_tiles) break;   // uniform
      kt.issue(smem + (stage * G + g) * 2 * TE, first + t);
      vt.issue(smem + (stage * G + g) * 2 * TE + TE, first + t);
    }
  };
  // probabilities and their gradients of 32 states
  auto scores = [&](const bf16_t* ktile, const bf16_t* vtile, int i, int kv0, f32x16_t& sc, f32x16_t& dp) {
#pragma unroll
    for (int r = 0; r < 16; ++r) sc[r] = dp[r] = 0.f;
#pragma unroll
    for (int s = 0; s < NS; ++s) {
      sc = mfma16<F16>(frag_rows<D>(ktile, fr_base, i * 32, s), qf[s], sc);
      dp = mfma16<F16>(frag_rows<D>(vtile, fr_base, i * 32, s), df[s], dp);
    }
    auto elements = [&](auto edge) {   // (two instances: interior tiles carry no mask code)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        sc[r] = __builtin_amdgcn_exp2f(fmaf(sc[r], sl2, -my_lse2));
        if (decltype(edge)::value) sc[r] = kv0 + i * 32 + acc_row(r, lane) >= n_keys ? 0.f : sc[r];
      }
    };
    if (kv0 + 64 > n_keys) elements(std::true_type{});
    else elements(std::false_type{});
  };
  auto compute = [&](int stage, int step) {
    const int t = step * G + grp, kv0 = (first + t) * 64;
    if (G > 1 && t >= n_tiles) return;
    const bf16_t* ktile = smem + (stage * G + grp) * 2 * TE;
    const bf16_t* vtile = ktile + TE;
    if (all_tiles == 1) {
      // All states of the sample are here: delta as sum p dP, without the rounding of O. With few states the gradient of a score is a
      // small difference (none at all with one), where that rounding would show.
      my_delta = 0.f;
      float only;
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        f32x16_t sc, dp;
        scores(ktile, vtile, i, kv0, sc, dp);
#pragma unroll
        for (int r = 0; r < 16; ++r) my_delta = fmaf(sc[r], dp[r], my_delta);
        if (i == 0) only = dp[0];
      }
      my_delta += __shfl_xor(my_delta, 32, 64);
      if (n_keys == 1) my_delta = __shfl(only, lane & 31, 64);   // p is 1, and the gradient of its score 0, exactly
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      f32x16_t sc, dp;
      scores(ktile, vtile, i, kv0, sc, dp);
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        dp[r] = sc[r] * (dp[r] - my_delta);
        if (EXACT) off += dp[r];
      }
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        const bf16x8_t dsf = pack8<F16>(dp, half);
        if constexpr (EXACT) {
          const bf16x8_t pf = pack8<F16>(sc, half);   // (a correction's factor: its rounding is of no account)
#pragma unroll
          for (int t = 0; t < NT; ++t) {
            const bf16x8_t kt = frag_tr<D>(ktile, ft_base, i * 32 + 16 * half, t);
            dq[t] = mfma16<F16>(kt, dsf, dq[t]);
            pk[t] = mfma16<F16>(kt, pf, pk[t]);
          }
        } else {
#pragma unroll
          for (int t = 0; t < NT; ++t) dq[t] = mfma16<F16>(frag_tr<D>(ktile, ft_base, i * 32 + 16 * half, t), dsf, dq[t]);
        }
      }
    }
  };
  tile_ring<2, G * 2 * StateTiles<D>::MINE>((n_tiles + G - 1) / G, issue_step, compute);
  if constexpr (EXACT) off += __shfl_xor(off, 32, 64);
  constexpr int REGS = 2 * NT * 16 + 1;
  if constexpr (G == 2) {
    if (grp > 0) {
      float* s = group_slot<G, REGS>(smem, grp, row_wave, lane);
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int r = 0; r < 16; ++r) { s[(t * 16 + r) * 64] = dq[t][r]; s[((NT + t) * 16 + r) * 64] = pk[t][r]; }
      s[2 * NT * 16 * 64] = off;
    }
    __syncthreads();
    if (grp > 0) return;
    const float* s = group_slot<G, REGS>(smem, 1, row_wave, lane);
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int r = 0; r < 16; ++r) { dq[t][r] += s[(t * 16 + r) * 64]; pk[t][r] += s[((NT + t) * 16 + r) * 64]; }
    off += s[2 * NT * 16 * 64];
  }
  if (wave_row >= n_rows) return;
  if constexpr (G == 2) {
    if (parts.splits > 1) {   // (the kernel that adds them up does the rest; a walk of one tile is the last split's)
      const int heads = sh.batch * sh.kv_heads;
      store_part<D>(parts.rows<D>(blk.head, heads, blk.split, 2, 0, n_rows, wave_row), lane, n_rows - wave_row, [&](int t, int e) { return dq[t][e]; });
      store_part<D>(parts.rows<D>(blk.head, heads, blk.split, 2, 1, n_rows, wave_row), lane, n_rows - wave_row, [&](int t, int e) { return pk[t][e]; });
      if (kc == 0 && my_row < n_rows) {
        parts.off[((int64_t)blk.split * heads + blk.head) * n_rows + my_row] = off;
        if (blk.split == parts.splits - 1) delta[stat] = my_delta;
      }
      return;
    }
  }
  if constexpr (EXACT) {
    my_delta += off;
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int r = 0; r < 16; ++r) dq[t][r] = fmaf(-off, pk[t][r], dq[t][r]);
  }
  if (kc == 0 && my_row < n_rows) delta[stat] = my_delta;
  const auto value = [&](int t, int e) { return dq[t][e] * sh.scale; };
  bf16_t* out = (bf16_t*)p.dq + (int64_t)b * sh.q_len * sh.q_stride + head0;
  bf16_t* stage = smem + row_wave * (G == 2 ? REGS * 128 : RowStage<D, F16>::ELEMS);   // (a wavefront writes over its own slot of what the groups handed it)
  RowStage<D, F16>::store(stage, lane, min(32, n_rows - wave_row), value, [&](int r) { return out + rows.at(wave_row + r, sh.q_stride, D); });
}

// The end of a step's products into the accumulation registers. The compiler does not know them for matrix instructions (see mfma16_agpr) and waits for
// none; where an accumulator has another register on the next path it moves it, and a move right behind the product reads a sum that is not there yet.
// What is moved behind this statement is its results, and it waits longer than any product takes.
template <int NT>
__device__ __forceinline__ void settle(f32x16_t (&dk)[NT], f32x16_t (&dv)[NT]) {
  if constexpr (NT == 4) {
    asm volatile("s_nop 15\n\ts_nop 15" : "+a"(dk[0]), "+a"(dk[1]), "+a"(dk[2]), "+a"(dk[3]), "+a"(dv[0]), "+a"(dv[1]), "+a"(dv[2]), "+a"(dv[3]));
  }
}
// dK and dV of 128 / G states; those of hidden states are zeros.
template <int D, bool F16, int G>
__global__ __launch_bounds__(256, D == 64 && G == 1 ? 2 : 1) void cross_dkdv_kernel(CrossShape sh, CrossOperands p, int nx, const float* __restrict__ delta, BwdParts parts) {
  constexpr int NS = D / 16, NT = D / 32, TE = Tile<D>::ELEMS, RB = 128 / G;
  constexpr int TILE = 2 * TE + 256;    // 16-bit units: Q tile, dO tile, 64 lse + 64 delta floats
  constexpr int STAGE = G * TILE;
  constexpr int FB = 4;                 // k-steps of fragment prefetch
  constexpr bool ACC_A = D == 128;      // dK/dV accumulators in AGPRs (see mfma16_agpr)
  extern __shared__ __attribute__((aligned(16))) bf16_t smem[];
  const CrossBlock blk = cross_block<true>(nx, parts.splits, sh, p.lens);
  if (blk.none) return;
  const int b = blk.b, h = blk.h;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), kc = lane >> 5;
  const int row_wave = wave % (4 / G), grp = G == 1 ? 0 : wave / (4 / G);
  const int fr_base = rows_base<D>(lane), ft_base = tr_base<D>(lane);
  const CrossRows rows(sh);
  const int kv_base = blk.x * RB, n_keys = visible(sh, p.lens, b), n_rows = rows.count();
  const int all_tiles = kv_base < n_keys ? (n_rows + 63) / 64 : 0;   // nothing to do for hidden states
  const int first = split_begin(all_tiles, blk.split, parts.splits), n_tiles = split_begin(all_tiles, blk.split + 1, parts.splits) - first;
  const int wave_key = kv_base + 32 * row_wave, my_key = wave_key + (lane & 31);
  const bool seen = my_key < n_keys;
  const int64_t head0 = (int64_t)h * sh.group * D, stats0 = ((int64_t)b * sh.heads + h * sh.group) * sh.q_len;
  const int64_t kv0 = (int64_t)b * sh.kv_len * sh.kv_stride + h * D;
  const float sl2 = LOG2E * sh.scale;

  bf16x8_t kf[NS], vf[NS];
  {
    const int64_t at = kv0 + (int64_t)min(my_key, sh.kv_len - 1) * sh.kv_stride + 8 * kc;
    const bf16x8_t none = {};
#pragma unroll
    for (int s = 0; s < NS; ++s) {
      kf[s] = seen ? *reinterpret_cast<const bf16x8_t*>((const bf16_t*)p.k + at + 16 * s) : none;
      vf[s] = seen ? *reinterpret_cast<const bf16x8_t*>((const bf16_t*)p.v + at + 16 * s) : none;
    }
  }
  f32x16_t dk[NT], dv[NT];
  zero(dk);
  zero(dv);

  // threads 0..63 carry lse, threads 64..127 delta, threads 128..255 duplicate them or bring the second tile of a step
  const float* stat_src = ((tid & 127) < 64 ? p.lse : delta) + stats0;
  const float stat_mul = (tid & 127) < 64 ? LOG2E : 1.0f;
  const int stat_tile = (tid >> 7) % G;
  // Nothing in the loop is masked. Rows behind the last one arrive as zeros and get an lse of infinity, which makes their p zero; a hidden state's
  // column is its lane's own in every product, and is not stored.
  auto load_stats = [&](int step) {
    const int row = (first + step * G + stat_tile) * 64 + (tid & 63);
    const float v = stat_src[rows.stat(min(row, n_rows - 1))];
    return row >= n_rows && (tid & 127) < 64 ? INFINITY : v;
  };
  auto store_stats = [&](int stage, float v) { reinterpret_cast<float*>(smem + stage * STAGE + stat_tile * TILE + 2 * TE)[tid & 127] = v * stat_mul; };
  QueryTiles<D> tiles(rows, (const bf16_t*)p.q + (int64_t)b * sh.q_len * sh.q_stride + head0, sh.q_stride,
                      (const bf16_t*)p.dout + (int64_t)b * sh.q_len * sh.out_stride + head0, sh.out_stride, first * 64, lane, wave);
  auto issue_step = [&](int stage, int step) {
#pragma unroll
    for (int g = 0; g < G; ++g) {
      if (step * G + g >= n_tiles) break;   // uniform
      tiles.issue(smem + stage * STAGE + g * TILE, smem + stage * STAGE + g * TILE + TE);
    }
  };
  auto compute = [&](int stage, int step, auto last) {
    if constexpr (G > 1 && decltype(last)::value) {
      if (step * G + grp >= n_tiles) return;
    }
    const bf16_t* qtile = smem + stage * STAGE + grp * TILE;
    const bf16_t* dtile = qtile + TE;
    const float* stat = reinterpret_cast<const float*>(qtile + 2 * TE);
    if constexpr (D == 128 && G == 1) {   // (two groups' tiles leave no registers for it)
      dkdv_interior<F16>(qtile, dtile, stat, kf, vf, dk, dv, fr_base, ft_base, kc, sl2);
      settle(dk, dv);
      return;
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      f32x16_t sc, dp;
#pragma unroll
      for (int r = 0; r < 16; ++r) sc[r] = dp[r] = 0.f;
      // Fragments are requested FB k-steps ahead of the MFMAs that use them and the order is pinned: left to itself the scheduler
      // reuses one register set for all fragments, and every MFMA then waits out the LDS latency of its own read.
#pragma unroll
      for (int s0 = 0; s0 < NS; s0 += FB) {
        bf16x8_t fq[FB], fd[FB];
#pragma unroll
        for (int s = 0; s < FB; ++s) {
          fq[s] = frag_rows<D>(qtile, fr_base, i * 32, s0 + s);
          fd[s] = frag_rows<D>(dtile, fr_base, i * 32, s0 + s);
        }
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int s = 0; s < FB; ++s) {
          sc = mfma16<F16>(fq[s], kf[s0 + s], sc);
          dp = mfma16<F16>(fd[s], vf[s0 + s], dp);
        }
        __builtin_amdgcn_sched_barrier(0);
      }
      // the first operands of the dV / dK products do not depend on the softmax: on their way during it
      bf16x8_t td0[NT], tq0[NT];
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        td0[t] = frag_tr<D>(dtile, ft_base, i * 32, t);
        tq0[t] = frag_tr<D>(qtile, ft_base, i * 32, t);
      }
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const float4 l4 = *reinterpret_cast<const float4*>(stat + i * 32 + g * 8 + 4 * kc);
        const float4 d4 = *reinterpret_cast<const float4*>(stat + 64 + i * 32 + g * 8 + 4 * kc);
        const float ls[4] = {l4.x, l4.y, l4.z, l4.w}, ds[4] = {d4.x, d4.y, d4.z, d4.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int r = 4 * g + e;
          sc[r] = __builtin_amdgcn_exp2f(fmaf(sc[r], sl2, -ls[e]));
          dp[r] = sc[r] * (dp[r] - ds[e]);
        }
      }
      const bf16x8_t pf0 = pack8<F16>(sc, 0), dsf0 = pack8<F16>(dp, 0), pf1 = pack8<F16>(sc, 1), dsf1 = pack8<F16>(dp, 1);
      __builtin_amdgcn_sched_barrier(0);
      bf16x8_t td1[NT], tq1[NT];   // second half's operands, requested in front of the first half's MFMAs
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        td1[t] = frag_tr<D>(dtile, ft_base, i * 32 + 16, t);
        tq1[t] = frag_tr<D>(qtile, ft_base, i * 32 + 16, t);
      }
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        if constexpr (ACC_A) { mfma16_agpr<F16>(dv[t], td0[t], pf0); mfma16_agpr<F16>(dk[t], tq0[t], dsf0); }
        else { dv[t] = mfma16<F16>(td0[t], pf0, dv[t]); dk[t] = mfma16<F16>(tq0[t], dsf0, dk[t]); }
      }
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        if constexpr (ACC_A) { mfma16_agpr<F16>(dv[t], td1[t], pf1); mfma16_agpr<F16>(dk[t], tq1[t], dsf1); }
        else { dv[t] = mfma16<F16>(td1[t], pf1, dv[t]); dk[t] = mfma16<F16>(tq1[t], dsf1, dk[t]); }
      }
      __builtin_amdgcn_sched_barrier(0);
    }
    if (ACC_A) settle(dk, dv);
  };
  // Two stages: step it + 1 is requested while step it is computed; its statistics travel through registers and are requested before its tile
  // loads, so that waiting for them leaves those in flight.
  const int n_steps = (n_tiles + G - 1) / G;
  if (n_steps > 0) {
    const float stat0 = load_stats(0);
    issue_step(0, 0);
    store_stats(0, stat0);
    wait_loads_and_lds<0>();
    block_barrier();
    int it = 0;
    for (; it + 1 < n_steps; ++it) {
      const int st = it & 1;
      const float next = load_stats(it + 1);
      issue_step(st ^ 1, it + 1);
      compute(st, it, std::false_type{});
      store_stats(st ^ 1, next);
      wait_loads_and_lds<0>();
      block_barrier();
    }
    compute(it & 1, it, std::true_type{});
    wait_loads_and_lds<0>();
    block_barrier();
  }
  if (ACC_A) agpr_results_ready();
  if constexpr (G > 1) {   // (behind the last barrier: the stages are free)
    constexpr int REGS = 2 * NT * 16;
    if (grp > 0) {
      float* s = group_slot<G, REGS>(smem, grp, row_wave, lane);
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int r = 0; r < 16; ++r) { s[(t * 16 + r) * 64] = dk[t][r]; s[((NT + t) * 16 + r) * 64] = dv[t][r]; }
    }
    __syncthreads();
    if (grp > 0) return;
    for (int g = 1; g < G; ++g) {
      const float* s = group_slot<G, REGS>(smem, g, row_wave, lane);
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int r = 0; r < 16; ++r) { dk[t][r] += s[(t * 16 + r) * 64]; dv[t][r] += s[((NT + t) * 16 + r) * 64]; }
    }
  }
  if (wave_key >= sh.kv_len) return;
  const auto dk_value = [&](int t, int e) { return seen ? dk[t][e] * sh.scale : 0.f; };   // (a row whose gradient is no number must not reach a hidden state)
  const auto dv_value = [&](int t, int e) { return seen ? dv[t][e] : 0.f; };
  const int there = sh.kv_len - wave_key;
  if (parts.splits > 1) {
    store_part<D>(parts.rows<D>(blk.head, sh.batch * sh.kv_heads, blk.split, 2, 0, sh.kv_len, wave_key), lane, there, dk_value);
    store_part<D>(parts.rows<D>(blk.head, sh.batch * sh.kv_heads, blk.split, 2, 1, sh.kv_len, wave_key), lane, there, dv_value);
    return;
  }
  bf16_t* stage = smem + row_wave * (G > 1 ? 2 * NT * 16 * 128 : RowStage<D, F16>::ELEMS);
  const int64_t at = kv0 + wave_key * sh.kv_stride;
  RowStage<D, F16>::store(stage, lane, min(32, there), dk_value, [&](int r) { return (bf16_t*)p.dk + at + r * sh.kv_stride; });
  RowStage<D, F16>::store(stage, lane, min(32, there), dv_value, [&](int r) { return (bf16_t*)p.dv + at + r * sh.kv_stride; });
}

// ===================================== at most 128 states ===============================================
// A prompt, the latents of a resampler, the patches of a small image: all states of a head fit into LDS and every wavefront sees all of them, so a
// wavefront needs nobody else: it takes tiles of 32 rows of its own, one after the other, the next one on its way, and softmax and delta are those
// of whole rows. (Tiles shared by the wavefronts of a block, with barriers between their steps, took 1.5 times as long for backward.)
constexpr int SHORT_KEYS = 128;
// 32-row tiles of an operand whose rows are CrossRows, for one wavefront.
template <int D>
struct RowTiles {
  static constexpr int SPR = D / 8, LOADS = SPR / 2;
  unsigned bytes;
  const bf16_t* base;
  const CrossRows& rows;
  int64_t stride;
  int lane;
  __device__ __forceinline__ RowTiles(const CrossRows& rows, const bf16_t* base, int64_t stride, int lane) : base(base), rows(rows), stride(stride), lane(lane) {
    bytes = (unsigned)(((int64_t)(rows.q_len - 1) * stride + rows.group * D) * 2);
  }
  __device__ __forceinline__ void issue(bf16_t* tile, int row0) const {
#pragma unroll
    for (int k = 0; k < LOADS; ++k) {
      const int slot = k * 64 + lane, row = slot / SPR, pos = slot % SPR, t = rows.token(row0 + row);
      const unsigned at = (unsigned)((t * (int)stride + (row0 + row - t * rows.group) * D) * 2) + (unsigned)(pos ^ Tile<D>::f(row)) * 16u;
      buffer_load_lds_16_untracked(base, bytes, tile + k * 512, at, 0);
    }
  }
};
// K and V of all visible states of a head, zeros behind them, as one or two 64-row tiles each.
template <int D, int KEYS>
__device__ __forceinline__ void load_states(const CrossShape& sh, const CrossOperands& p, int64_t kv0, int n_keys, bf16_t* ktile, bf16_t* vtile, int lane, int wave) {
  const StateTiles<D> kt((const bf16_t*)p.k + kv0, sh.kv_stride, n_keys, lane, wave), vt((const bf16_t*)p.v + kv0, sh.kv_stride, n_keys, lane, wave);
  kt.issue(ktile, 0);
  vt.issue(vtile, 0);
  if (KEYS == 128) {
    kt.issue(ktile + Tile<D>::ELEMS, 1);   // (out of bounds where there are at most 64: zeros)
    vt.issue(vtile + Tile<D>::ELEMS, 1);
  }
}

template <int D> constexpr size_t SHORT_FWD_LDS = (4 * Tile<D>::ELEMS + 4 * 2 * 32 * D) * sizeof(bf16_t);
template <int D, bool F16>
__global__ __launch_bounds__(256) void cross_fwd_short_kernel(CrossShape sh, CrossOperands p, int nx) {
  constexpr int NS = D / 16, NT = D / 32, TE = Tile<D>::ELEMS, KT = SHORT_KEYS / 32;
  extern __shared__ __attribute__((aligned(16))) bf16_t smem[];   // K, V, per wavefront two tiles of queries
  const CrossBlock blk = cross_block<true>(nx, 1, sh, p.lens);
  if (blk.none) return;
  const int b = blk.b, h = blk.h;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), kc = lane >> 5;
  const int fr_base = rows_base<D>(lane), ft_base = tr_base<D>(lane);
  const CrossRows rows(sh);
  const int n_keys = visible(sh, p.lens, b), n_sub = (n_keys + 31) / 32, n_rows = rows.count();
  const int64_t head0 = (int64_t)h * sh.group * D;
  const float sl2 = LOG2E * sh.scale;
  bf16_t *ktile = smem, *vtile = smem + 2 * TE, *mine = smem + 4 * TE + wave * 2 * 32 * D;
  load_states<D, SHORT_KEYS>(sh, p, (int64_t)b * sh.kv_len * sh.kv_stride + h * D, n_keys, ktile, vtile, lane, wave);
  const RowTiles<D> tiles(rows, (const bf16_t*)p.q + (int64_t)b * sh.q_len * sh.q_stride + head0, sh.q_stride, lane);
  bf16_t* out = (bf16_t*)p.o + (int64_t)b * sh.q_len * sh.out_stride + head0;
  const int step = nx * 128;
  int row0 = blk.x * 128 + wave * 32;
  if (row0 < n_rows) tiles.issue(mine, row0);
  wait_loads_and_lds<0>();
  __syncthreads();
  for (int stage = 0; row0 < n_rows; row0 += step, stage ^= 1) {
    bf16_t* qtile = mine + stage * 32 * D;
    bf16x8_t qf[NS];
    wait_loads_and_lds<D / 16>();   // (all but the stores of the tile in front, which had 32 rows)
    asm volatile("" ::: "memory");
#pragma unroll
    for (int s = 0; s < NS; ++s) qf[s] = frag_rows<D>(qtile, fr_base, 0, s);
    if (row0 + step < n_rows) tiles.issue(mine + (stage ^ 1) * 32 * D, row0 + step);
    f32x16_t sc[KT];
    float m = -INFINITY, l = 0.f;
#pragma unroll
    for (int i = 0; i < KT; ++i) {
      if (i < n_sub) {   // (uniform)
#pragma unroll
        for (int r = 0; r < 16; ++r) sc[i][r] = 0.f;
#pragma unroll
        for (int s = 0; s < NS; ++s) sc[i] = mfma16<F16>(frag_rows<D>(ktile, fr_base, i * 32, s), qf[s], sc[i]);
        if (32 * i + 32 > n_keys) {
#pragma unroll
          for (int r = 0; r < 16; ++r) sc[i][r] = 32 * i + acc_row(r, lane) >= n_keys ? -INFINITY : sc[i][r];
        }
#pragma unroll
        for (int r = 0; r < 16; ++r) m = fmaxf(m, sc[i][r]);
      }
    }
    m = fmaxf(m, __shfl_xor(m, 32, 64));
    const float mb = m == -INFINITY ? 0.f : m * sl2;
    f32x16_t o[NT];
    zero(o);
#pragma unroll
    for (int i = 0; i < KT; ++i) {
      if (i < n_sub) {
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          sc[i][r] = __builtin_amdgcn_exp2f(fmaf(sc[i][r], sl2, -mb));
          l += sc[i][r];
        }
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          const bf16x8_t pf = pack8<F16>(sc[i], half);
#pragma unroll
          for (int t = 0; t < NT; ++t) o[t] = mfma16<F16>(frag_tr<D>(vtile, ft_base, i * 32 + 16 * half, t), pf, o[t]);
        }
      }
    }
    l += __shfl_xor(l, 32, 64);
    const float inv = inverse(l);
    // (through the room of the queries of this tile, which are in registers)
    static_assert(32 * D >= 16 * RowStage<D, F16>::P, "half a tile of rows");
    const int my_row = row0 + (lane & 31);
    RowStage<D, F16>::store_halves(qtile, lane, min(32, n_rows - row0), [&](int t, int e) { return o[t][e] * inv; },
                                   [&](int r) { return out + rows.at(row0 + r, sh.out_stride, D); });
    if (p.lse && kc == 0 && my_row < n_rows) p.lse[((int64_t)b * sh.heads + h * sh.group) * sh.q_len + rows.stat(my_row)] = log_sum(m, l, sh.scale);
  }
}

// Backward: dQ, dK and dV of one pass over the queries, five products. Scores and gradients of probabilities have the queries along the lanes, so
// delta = sum p dP is a lane's own sum (O is not read, and the gradients of scores do not inherit its rounding: with few states they are small
// differences). dQ^T = K^T dS^T takes them as they are; for dV^T = dO^T P and dK^T = Q^T dS, whose sums run along the queries, P and dS go through
// a [query][state] tile in LDS, 64 states at a time. dK and dV of the four wavefronts meet in LDS, those of several blocks in cross_sum_kernel.
// 64-wide heads have two stages of rows and request the next one's at the beginning of a tile, 128-wide ones one, which is free in the middle of it.
template <int D> constexpr int SHORT_BWD_STAGES = D == 64 ? 2 : 1;
template <int D> constexpr int SHORT_BWD_KEYS = D == 64 ? 128 : 64;   // as many as leave a wavefront's dK and dV in its registers
template <int D> constexpr size_t SHORT_BWD_LDS = (2 * SHORT_BWD_KEYS<D> * D + 4 * (2 * SHORT_BWD_STAGES<D> * 32 * D + 2 * 32 * 64)) * sizeof(bf16_t);
template <int D, bool F16, int KT>
__global__ __launch_bounds__(256, 1) void cross_bwd_short_kernel(CrossShape sh, CrossOperands p, BwdParts parts) {
  constexpr int NS = D / 16, NT = D / 32, KEYS = SHORT_BWD_KEYS<D>, NSTG = SHORT_BWD_STAGES<D>, QT = 32 * D, XT = 32 * 64;
  extern __shared__ __attribute__((aligned(16))) bf16_t smem[];   // K, V; per wavefront two stages of queries and dO, and P, dS
  const CrossBlock blk = cross_block<true>(1, parts.splits, sh, p.lens);
  if (blk.none) return;
  const int b = blk.b, h = blk.h;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), kc = lane >> 5;
  const int fr_base = rows_base<D>(lane), ft_base = tr_base<D>(lane), ft_x = tr_base<64>(lane);
  const CrossRows rows(sh);
  const int n_keys = visible(sh, p.lens, b), n_rows = rows.count();
  const int64_t head0 = (int64_t)h * sh.group * D, stats0 = ((int64_t)b * sh.heads + h * sh.group) * sh.q_len;
  const int64_t kv0 = (int64_t)b * sh.kv_len * sh.kv_stride + h * D;
  const float sl2 = LOG2E * sh.scale;
  bf16_t *ktile = smem, *vtile = smem + KEYS * D, *mine = smem + 2 * KEYS * D + wave * (2 * NSTG * QT + 2 * XT), *pt = mine + 2 * NSTG * QT, *dst = pt + XT;
  load_states<D, KEYS>(sh, p, kv0, n_keys, ktile, vtile, lane, wave);
  const RowTiles<D> qtiles(rows, (const bf16_t*)p.q + (int64_t)b * sh.q_len * sh.q_stride + head0, sh.q_stride, lane);
  const RowTiles<D> dtiles(rows, (const bf16_t*)p.dout + (int64_t)b * sh.q_len * sh.out_stride + head0, sh.out_stride, lane);
  bf16_t* dq_out = (bf16_t*)p.dq + (int64_t)b * sh.q_len * sh.q_stride + head0;
  f32x16_t dk[KT][NT], dv[KT][NT];
#pragma unroll
  for (int i = 0; i < KT; ++i) { zero(dk[i]); zero(dv[i]); }
  const int step = parts.splits * 128;
  int row0 = blk.split * 128 + wave * 32;
  float next_lse = 0.f;
  auto issue = [&](int stage, int row0) {
    next_lse = p.lse[stats0 + rows.stat(min(row0 + (lane & 31), n_rows - 1))];
    qtiles.issue(mine + stage * 2 * QT, row0);
    dtiles.issue(mine + stage * 2 * QT + QT, row0);
  };
  if (row0 < n_rows) issue(0, row0);
  wait_loads_and_lds<0>();
  __syncthreads();
  for (int stage = 0; row0 < n_rows; row0 += step, stage = NSTG - 1 - stage) {
    bf16_t *qtile = mine + stage * 2 * QT, *dtile = qtile + QT;
    wait_loads_and_lds<D / 16>();   // (all but the stores of the tile in front, which had 32 rows)
    asm volatile("" ::: "memory");
    const float lse2 = next_lse * LOG2E;
    const bool row_there = row0 + (lane & 31) < n_rows;
    if (NSTG == 2 && row0 + step < n_rows) issue(stage ^ 1, row0 + step);
    f32x16_t pr[KT], dp[KT];
    float delta = 0.f;
    {
      bf16x8_t qf[NS], df[NS];
#pragma unroll
      for (int s = 0; s < NS; ++s) { qf[s] = frag_rows<D>(qtile, fr_base, 0, s); df[s] = frag_rows<D>(dtile, fr_base, 0, s); }
#pragma unroll
      for (int i = 0; i < KT; ++i) {
#pragma unroll
        for (int r = 0; r < 16; ++r) pr[i][r] = dp[i][r] = 0.f;
#pragma unroll
        for (int s = 0; s < NS; ++s) {
          pr[i] = mfma16<F16>(frag_rows<D>(ktile, fr_base, i * 32, s), qf[s], pr[i]);
          dp[i] = mfma16<F16>(frag_rows<D>(vtile, fr_base, i * 32, s), df[s], dp[i]);
        }
        const bool edge = 32 * i + 32 > n_keys || row0 + 32 > n_rows;
#pragma unroll
        for (int r = 0; r < 16; ++r) pr[i][r] = __builtin_amdgcn_exp2f(fmaf(pr[i][r], sl2, -lse2));
        if (edge) {
#pragma unroll
          for (int r = 0; r < 16; ++r) pr[i][r] = row_there && 32 * i + acc_row(r, lane) < n_keys ? pr[i][r] : 0.f;
        }
#pragma unroll
        for (int r = 0; r < 16; ++r) delta = fmaf(pr[i][r], dp[i][r], delta);
        __builtin_amdgcn_sched_barrier(0);   // (left to itself the scheduler requests the operands of all states at once and spills)
      }
    }
    delta += __shfl_xor(delta, 32, 64);
    if (n_keys == 1) delta = __shfl(dp[0][0], lane & 31, 64);   // (see cross_dq_kernel)
    f32x16_t dq[NT];
    zero(dq);
    __builtin_amdgcn_sched_barrier(0);
    // operands whose sums run along the queries: of both halves of 16
    bf16x8_t tq[2][NT], td[2][NT];
#pragma unroll
    for (int half = 0; half < 2; ++half)
#pragma unroll
      for (int t = 0; t < NT; ++t) { tq[half][t] = frag_tr<D>(qtile, ft_base, 16 * half, t); td[half][t] = frag_tr<D>(dtile, ft_base, 16 * half, t); }
    if (NSTG == 1 && row0 + step < n_rows) {
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // what has been read of the stage has arrived
      issue(0, row0 + step);
    }
#pragma unroll
    for (int i = 0; i < KT; ++i) {
#pragma unroll
      for (int r = 0; r < 16; ++r) dp[i][r] = pr[i][r] * (dp[i][r] - delta);
      const bf16x8_t pf[2] = {pack8<F16>(pr[i], 0), pack8<F16>(pr[i], 1)}, dsf[2] = {pack8<F16>(dp[i], 0), pack8<F16>(dp[i], 1)};
#pragma unroll
      for (int half = 0; half < 2; ++half)
#pragma unroll
        for (int t = 0; t < NT; ++t) dq[t] = mfma16<F16>(frag_tr<D>(ktile, ft_base, i * 32 + 16 * half, t), dsf[half], dq[t]);
      // four states at a time, 8 bytes, into row `lane % 32`: states 32 (i % 2) + 8 c + 4 kc ..
      const int row = lane & 31, f = Tile<64>::f(row);
      RowStage<D, F16>::meet();
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        const int at = row * 64 + (((4 * (i & 1) + c) ^ f) << 3) + 4 * kc;
        const u32x4_t pw = __builtin_bit_cast(u32x4_t, pf[c >> 1]), dw = __builtin_bit_cast(u32x4_t, dsf[c >> 1]);
        *reinterpret_cast<uint2*>(pt + at) = make_uint2(pw[2 * (c & 1)], pw[2 * (c & 1) + 1]);
        *reinterpret_cast<uint2*>(dst + at) = make_uint2(dw[2 * (c & 1)], dw[2 * (c & 1) + 1]);
      }
      RowStage<D, F16>::meet();
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        const bf16x8_t xp = frag_tr<64>(pt, ft_x, 16 * half, i & 1), xd = frag_tr<64>(dst, ft_x, 16 * half, i & 1);
#pragma unroll
        for (int t = 0; t < NT; ++t) { mfma16_agpr<F16>(dv[i][t], td[half][t], xp); mfma16_agpr<F16>(dk[i][t], tq[half][t], xd); }
      }
      __builtin_amdgcn_sched_barrier(0);
    }
    static_assert(2 * XT >= 16 * RowStage<D, F16>::P, "half a tile of rows");
    RowStage<D, F16>::store_halves(pt, lane, min(32, n_rows - row0), [&](int t, int e) { return dq[t][e] * sh.scale; },
                                   [&](int r) { return dq_out + rows.at(row0 + r, sh.q_stride, D); });
  }
  agpr_results_ready();
  // 32 states at a time: the sums of every wavefront that had rows, and each wavefront adds up a quarter of the registers of all
  constexpr int QUADS = 2 * NT * 4;   // four registers: four columns
  float4* slots = reinterpret_cast<float4*>(smem) + lane;
  const int n_store = (sh.kv_len + 31) / 32, busy = min(4, (n_rows - blk.split * 128 + 31) / 32);
#pragma unroll
  for (int i = 0; i < KT; ++i) {
    if (i >= n_store) break;   // (uniform)
    __syncthreads();
    if (wave < busy) {
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          slots[(wave * QUADS + t * 4 + g) * 64] = make_float4(dk[i][t][4 * g], dk[i][t][4 * g + 1], dk[i][t][4 * g + 2], dk[i][t][4 * g + 3]);
          slots[(wave * QUADS + (NT + t) * 4 + g) * 64] = make_float4(dv[i][t][4 * g], dv[i][t][4 * g + 1], dv[i][t][4 * g + 2], dv[i][t][4 * g + 3]);
        }
    }
    __syncthreads();
    const int key = 32 * i + (lane & 31);
#pragma unroll
    for (int k = 0; k < QUADS / 4; ++k) {
      const int quad = wave * (QUADS / 4) + k, array = quad / (4 * NT), col = quad % (4 * NT) * 8 + 4 * kc;
      float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
      for (int w = 0; w < busy; ++w) {
        const float4 x = slots[(w * QUADS + quad) * 64];
        v.x += x.x; v.y += x.y; v.z += x.z; v.w += x.w;
      }
      const float factor = array ? 1.f : sh.scale;
      v = key < n_keys ? make_float4(v.x * factor, v.y * factor, v.z * factor, v.w * factor)
                       : make_float4(0.f, 0.f, 0.f, 0.f);   // (a row whose gradient is no number must not reach a hidden state)
      if (key >= sh.kv_len) continue;
      if (parts.splits > 1) *reinterpret_cast<float4*>(parts.rows<D>(blk.head, sh.batch * sh.kv_heads, blk.split, 2, array, sh.kv_len, key) + col) = v;
      else *reinterpret_cast<uint2*>((bf16_t*)(array ? p.dv : p.dk) + kv0 + key * sh.kv_stride + col) = make_uint2(pack2<F16>(v.x, v.y), pack2<F16>(v.z, v.w));
    }
  }
}

// ================================ backward: at most 32 rows of a head ===================================
// As in forward, every wavefront walks tiles of 32 states of its own. All rows are in one tile, so dK and dV of a tile's states are complete at once,
// and only dQ is a sum over the walk: K and V are read once, for all gradients. The products want the scores either way round, S^T = K Q^T for dQ and
// S = Q K^T for dK and dV, and both are computed (seven products), which spares a way through LDS. delta as in cross_dq_kernel: of the stored O, and
// corrected in dQ. Bound by memory where the walk is long. us, against two kernels on tiles: 16 x 4 rows, 16384 states, 8 key heads of 128 432 / 828
// (2.15 GB, 5.0 TB/s); 16 x 8, 4096, 16 of 64 128 / 198; 32 x 32, 500, 16 of 128 75.6 / 119, of 64 43.2 / 54.7; 7 x 2, 242, 2 of 64 9.1 / 11.8.
template <int D> constexpr int FEW_BWD_WAVES = D == 64 ? 8 : 4;
template <int D> constexpr size_t FEW_BWD_LDS = (2 + 2 * FEW_BWD_WAVES<D>) * 32 * D * sizeof(bf16_t) + (64 + 32 * FEW_BWD_WAVES<D>) * sizeof(float);
template <int D, bool F16>
__global__ __launch_bounds__(64 * FEW_BWD_WAVES<D>) void cross_bwd_few_kernel(CrossShape sh, CrossOperands p, BwdParts parts) {
  constexpr int NS = D / 16, NT = D / 32, TE = 32 * D, WAVES = FEW_BWD_WAVES<D>, SPR = D / 8, LOADS = SPR / 2;
  extern __shared__ __attribute__((aligned(16))) bf16_t smem[];   // Q, dO; per wavefront K and V, then what goes out; lse and delta; sums of scores' gradients
  const CrossBlock blk = cross_block<true>(1, parts.splits, sh, p.lens);
  if (blk.none) return;
  const int b = blk.b, h = blk.h;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), kc = lane >> 5;
  const int fr_base = rows_base<D>(lane), ft_base = tr_base<D>(lane);
  const CrossRows rows(sh);
  const int n_rows = rows.count(), n_keys = visible(sh, p.lens, b), all_tiles = (sh.kv_len + 31) / 32;
  const int first = split_begin(all_tiles, blk.split, parts.splits) + wave, end = split_begin(all_tiles, blk.split + 1, parts.splits);
  const int my_row = lane & 31, ld_row = min(my_row, n_rows - 1);
  const int64_t head0 = (int64_t)h * sh.group * D, stat = ((int64_t)b * sh.heads + h * sh.group) * sh.q_len + rows.stat(ld_row);
  const float sl2 = LOG2E * sh.scale;

  bf16_t *qtile = smem, *dtile = smem + TE, *ktile = smem + (2 + 2 * wave) * TE, *vtile = ktile + TE;
  float *stats = reinterpret_cast<float*>(smem + (2 + 2 * WAVES) * TE), *offs = stats + 64;
  const int64_t kv0 = (int64_t)b * sh.kv_len * sh.kv_stride + h * D;
  const bf16_t *k = (const bf16_t*)p.k + kv0, *v = (const bf16_t*)p.v + kv0;
  const unsigned bytes = n_keys > 0 ? (unsigned)(((int64_t)(n_keys - 1) * sh.kv_stride + D) * 2) : 0u, step = (unsigned)(32 * sh.kv_stride * 2);
  unsigned voff[LOADS];
#pragma unroll
  for (int i = 0; i < LOADS; ++i) {
    const int slot = i * 64 + lane, row = slot / SPR, pos = slot % SPR;
    voff[i] = (unsigned)(row * sh.kv_stride * 2) + (unsigned)(pos ^ Tile<D>::f(row)) * 16u;
  }
  auto issue = [&](int t) {   // (hidden tiles: nothing is read)
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // what this wavefront has read of its room has arrived
    const unsigned at = (unsigned)t * step;
#pragma unroll
    for (int n = 0; n < LOADS; ++n) {
      buffer_load_lds_16_untracked(k, bytes, ktile + n * 512, voff[n] + at, 0);
      buffer_load_lds_16_untracked(v, bytes, vtile + n * 512, voff[n] + at, 0);
    }
  };
  const bool whole = n_keys <= 64, mine = first < end && 32 * first < n_keys;
  if (!whole && mine) issue(first);
  const bf16_t *q = (const bf16_t*)p.q + (int64_t)b * sh.q_len * sh.q_stride + head0, *dout = (const bf16_t*)p.dout + (int64_t)b * sh.q_len * sh.out_stride + head0;
  if (wave == 0) RowTiles<D>(rows, q, sh.q_stride, lane).issue(qtile, 0);
  if (wave == 1) RowTiles<D>(rows, dout, sh.out_stride, lane).issue(dtile, 0);
  const float lse2 = p.lse[stat] * LOG2E;
  float delta = 0.f;
  {
    const bf16_t *o = (const bf16_t*)p.out + (int64_t)b * sh.q_len * sh.out_stride + head0;
    const int64_t at = rows.at(ld_row, sh.out_stride, D) + 8 * kc;
#pragma unroll
    for (int s = 0; s < NS; ++s) {
      float ov[8], dv[8];
      load8h<F16>(o + at + 16 * s, ov);
      load8h<F16>(dout + at + 16 * s, dv);
#pragma unroll
      for (int e = 0; e < 8; ++e) delta = fmaf(ov[e], dv[e], delta);
    }
    delta += __shfl_xor(delta, 32, 64);
  }
  // probabilities and their gradients, S^T
  f32x16_t pr, dp;
  auto scores = [&](int t) {
#pragma unroll
    for (int r = 0; r < 16; ++r) pr[r] = dp[r] = 0.f;
#pragma unroll
    for (int s = 0; s < NS; ++s) {
      pr = mfma16<F16>(frag_rows<D>(ktile, fr_base, 0, s), frag_rows<D>(qtile, fr_base, 0, s), pr);
      dp = mfma16<F16>(frag_rows<D>(vtile, fr_base, 0, s), frag_rows<D>(dtile, fr_base, 0, s), dp);
    }
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      pr[r] = __builtin_amdgcn_exp2f(fmaf(pr[r], sl2, -lse2));
      pr[r] = 32 * t + acc_row(r, lane) < n_keys ? pr[r] : 0.f;
    }
  };
  wait_loads_and_lds<0>();
  __syncthreads();
  if (whole) {   // delta as sum p dP, which every wavefront takes: with few states that shows in dk too (see cross_dq_kernel)
    delta = 0.f;
#pragma unroll 1
    for (int t = 0; 32 * t < n_keys; ++t) {
      issue(t);
      wait_loads_and_lds<0>();
      asm volatile("" ::: "memory");
      scores(t);
#pragma unroll
      for (int r = 0; r < 16; ++r) delta = fmaf(pr[r], dp[r], delta);
    }
    delta += __shfl_xor(delta, 32, 64);
    if (n_keys == 1) delta = __shfl(dp[0], lane & 31, 64);   // (see cross_dq_kernel)
    if (mine) issue(first);
  }
  if (wave == 0 && kc == 0) {   // (rows that are not there: zeros, and a p of 0)
    stats[my_row] = my_row < n_rows ? lse2 : INFINITY;
    stats[32 + my_row] = delta;
  }
  __syncthreads();

  f32x16_t dq[NT], pk[NT];
  zero(dq);
  zero(pk);
  float off = 0.f;
  for (int t = first; t < end; t += WAVES) {
    const int left = sh.kv_len - 32 * t;
    const bool seen = 32 * t + my_row < n_keys;
    const int64_t at = kv0 + (int64_t)32 * t * sh.kv_stride;
    f32x16_t acc[NT];
    const auto put = [&](void* out, float scale) {
      RowStage<D, F16>::store(ktile, lane, min(32, left), [&](int c, int e) { return seen ? acc[c][e] * scale : 0.f; },
                              [&](int r) { return (bf16_t*)out + at + r * sh.kv_stride; });
    };
    if (32 * t >= n_keys) {
      zero(acc);
      put(p.dk, 0.f);
      put(p.dv, 0.f);
      continue;
    }
    wait_loads_and_lds<0>();
    asm volatile("" ::: "memory");
    scores(t);
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      dp[r] = pr[r] * (dp[r] - delta);
      off += dp[r];
    }
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      const bf16x8_t pf = pack8<F16>(pr, half), dsf = pack8<F16>(dp, half);
#pragma unroll
      for (int c = 0; c < NT; ++c) {
        const bf16x8_t kt = frag_tr<D>(ktile, ft_base, 16 * half, c);
        dq[c] = mfma16<F16>(kt, dsf, dq[c]);
        pk[c] = mfma16<F16>(kt, pf, pk[c]);
      }
    }
#pragma unroll
    for (int r = 0; r < 16; ++r) pr[r] = dp[r] = 0.f;
#pragma unroll
    for (int s = 0; s < NS; ++s) {
      pr = mfma16<F16>(frag_rows<D>(qtile, fr_base, 0, s), frag_rows<D>(ktile, fr_base, 0, s), pr);
      dp = mfma16<F16>(frag_rows<D>(dtile, fr_base, 0, s), frag_rows<D>(vtile, fr_base, 0, s), dp);
    }
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const float4 l4 = *reinterpret_cast<const float4*>(stats + g * 8 + 4 * kc), d4 = *reinterpret_cast<const float4*>(stats + 32 + g * 8 + 4 * kc);
      const float ls[4] = {l4.x, l4.y, l4.z, l4.w}, ds[4] = {d4.x, d4.y, d4.z, d4.w};
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int r = 4 * g + e;
        pr[r] = __builtin_amdgcn_exp2f(fmaf(pr[r], sl2, -ls[e]));
        dp[r] = pr[r] * (dp[r] - ds[e]);
      }
    }
    const bf16x8_t pf[2] = {pack8<F16>(pr, 0), pack8<F16>(pr, 1)}, dsf[2] = {pack8<F16>(dp, 0), pack8<F16>(dp, 1)};
    zero(acc);
#pragma unroll
    for (int half = 0; half < 2; ++half)
#pragma unroll
      for (int c = 0; c < NT; ++c) acc[c] = mfma16<F16>(frag_tr<D>(dtile, ft_base, 16 * half, c), pf[half], acc[c]);
    put(p.dv, 1.f);
    zero(acc);
#pragma unroll
    for (int half = 0; half < 2; ++half)
#pragma unroll
      for (int c = 0; c < NT; ++c) acc[c] = mfma16<F16>(frag_tr<D>(qtile, ft_base, 16 * half, c), dsf[half], acc[c]);
    put(p.dk, sh.scale);
    if (t + WAVES < end && 32 * (t + WAVES) < n_keys) issue(t + WAVES);
  }
  // every wavefront puts some of the accumulators of all together: registers REGS w .. of the 16 NT, dq's, then those of sum p K
  constexpr int REGS = 16 * NT / WAVES;
  static_assert(REGS % 2 == 0 && 16 % REGS == 0, "whole pairs of columns, of one 32-column block");
  float* slots = reinterpret_cast<float*>(smem + 2 * TE) + lane;
  off += __shfl_xor(off, 32, 64);
  if (kc == 0) offs[wave * 32 + my_row] = off;
  float sum[2][REGS];
#pragma unroll
  for (int a = 0; a < 2; ++a) {
    __syncthreads();
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int r = 0; r < 16; ++r) slots[((wave * NT + t) * 16 + r) * 64] = a ? pk[t][r] : dq[t][r];
    __syncthreads();
#pragma unroll
    for (int r = 0; r < REGS; ++r) sum[a][r] = 0.f;
#pragma unroll
    for (int w = 0; w < WAVES; ++w)
#pragma unroll
      for (int r = 0; r < REGS; ++r) sum[a][r] += slots[(w * NT * 16 + wave * REGS + r) * 64];
  }
  if (my_row >= n_rows) return;
  off = 0.f;
#pragma unroll
  for (int w = 0; w < WAVES; ++w) off += offs[w * 32 + my_row];
  const int reg = wave * REGS % 16, col = wave * REGS / 16 * 32 + 8 * (reg / 4) + 4 * kc + reg % 4;   // of the first of them
  bf16_t* out = (bf16_t*)p.dq + (int64_t)b * sh.q_len * sh.q_stride + head0 + rows.at(my_row, sh.q_stride, D) + col;
  const int heads = sh.batch * sh.kv_heads;
#pragma unroll
  for (int r = 0; r < REGS; r += 2) {   // (registers 4 g .. 4 g + 3: consecutive columns; the next four eight columns on)
    const int c = r / 4 * 8 + r % 4;
    if (parts.splits > 1) {
#pragma unroll
      for (int a = 0; a < 2; ++a)
        *reinterpret_cast<float2*>(parts.rows<D>(blk.head, heads, blk.split, 2, a, n_rows, my_row) + col + c) = make_float2(sum[a][r], sum[a][r + 1]);
    } else {
      *reinterpret_cast<uint32_t*>(out + c) = pack2<F16>(fmaf(-off, sum[1][r], sum[0][r]) * sh.scale, fmaf(-off, sum[1][r + 1], sum[0][r + 1]) * sh.scale);
    }
  }
  if (parts.splits > 1 && wave == 0 && kc == 0) parts.off[((int64_t)blk.split * heads + blk.head) * n_rows + my_row] = off;
}

// Adds up the parts of dk and dv, in their order, eight columns per thread.
template <int D, bool F16>
__global__ __launch_bounds__(256) void cross_sum_kernel(CrossShape sh, CrossOperands p, BwdParts parts) {
  constexpr int C = D / 8;
  const int64_t heads = (int64_t)sh.batch * sh.kv_heads, items = heads * 2 * sh.kv_len * C;
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= items) return;
  float v[8], w[8];
  load8(parts.o + 8 * i, v);
#pragma unroll 4
  for (int s = 1; s < parts.splits; ++s) {
    load8(parts.o + 8 * (i + s * items), w);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] += w[e];
  }
  const int c = (int)(i % C) * 8;
  const int64_t row = i / C, r = row % sh.kv_len, plane = row / sh.kv_len, head = plane / 2, b = head / sh.kv_heads, h = head - b * sh.kv_heads;
  store8h<F16>((bf16_t*)(plane % 2 ? p.dv : p.dk) + (b * sh.kv_len + r) * sh.kv_stride + h * D + c, v);
}
// The same of dq, whose rows are CrossRows: dq, sum p K and what delta lacks, of which it makes the one of all splits (delta may be NULL: nobody wants it).
// A wavefront takes a row, its lanes eight columns each and the splits between them: a thread alone took 13 us for 30 splits, not 4.2.
template <int D, bool F16>
__global__ __launch_bounds__(256) void cross_sum_rows_kernel(CrossShape sh, CrossOperands p, BwdParts parts, float* __restrict__ delta) {
  constexpr int C = D / 8, GROUPS = 64 / C;
  const CrossRows rows(sh);
  const int64_t n_rows = rows.count(), heads = (int64_t)sh.batch * sh.kv_heads;
  const int64_t row = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (row >= heads * n_rows) return;
  const int lane = threadIdx.x & 63, c = lane % C * 8, g = lane / C;
  const int64_t r = row % n_rows, head = row / n_rows, b = head / sh.kv_heads, h = head - b * sh.kv_heads;
  float dq[8] = {}, pk[8] = {}, w[8], off = 0.f;
#pragma unroll 2
  for (int s = g; s < parts.splits; s += GROUPS) {
    load8(parts.rows<D>((int)head, (int)heads, s, 2, 0, n_rows, r) + c, w);
#pragma unroll
    for (int e = 0; e < 8; ++e) dq[e] += w[e];
    load8(parts.rows<D>((int)head, (int)heads, s, 2, 1, n_rows, r) + c, w);
#pragma unroll
    for (int e = 0; e < 8; ++e) pk[e] += w[e];
    off += parts.off[(s * heads + head) * n_rows + r];
  }
#pragma unroll
  for (int o = C; o < 64; o *= 2) {
#pragma unroll
    for (int e = 0; e < 8; ++e) { dq[e] += __shfl_xor(dq[e], o, 64); pk[e] += __shfl_xor(pk[e], o, 64); }
    off += __shfl_xor(off, o, 64);
  }
  if (g != 0) return;
#pragma unroll
  for (int e = 0; e < 8; ++e) dq[e] = fmaf(-off, pk[e], dq[e]) * sh.scale;
  if (delta && c == 0) delta[(b * sh.heads + h * sh.group) * sh.q_len + rows.stat((int)r)] += off;
  store8h<F16>((bf16_t*)p.dq + b * sh.q_len * sh.q_stride + h * sh.group * D + rows.at((int)r, sh.q_stride, D) + c, dq);
}

// ======================================== launches ======================================================
// What a launch looks like: groups of wavefronts per block, blocks along the rows, splits of the walk.
struct Form { int groups, nx, splits; };

// `rows` own rows of each of `heads` heads, a walk of `walk` others.
// Two groups, i.e. blocks of 64 rows that take two tiles at a time: 64-wide heads while blocks of 128 rows are at most one per CU (two of those with two
// groups fit one), 128-wide ones, whose two groups fill the LDS of a CU, while those of 64 rows are. us, one group / two: 64-wide, forward 2 x 512
// rows, 1024 states, 16 heads (128 blocks of 128) 19.8 / 13.1; 5 x 1143, 777, 4 (180) 14.1 / 11.6; 8 x 512, 1024, 16 (512) 24.1 / 28.9; dQ and dK/dV of
// the second 51.1 / 46.3, of the third 75.6 / 84.0; 128-wide, forward 1 x 1024, 1024, 20 heads (320 blocks of 64) 26.2 / 34.7, dQ and dK/dV 68 / 108.
// Splits of the walk, which a second kernel adds up (5 to 10 us): while the blocks, then of two groups, are far fewer than the CUs and the walk is long.
// 1 x 128 rows, 8192 states, 16 heads of 128 in 2 / 4 / 8 splits 58.9 / 37.4 / 29.7; 1 x 512, 4096, 16 of 64 (128 blocks) in 1 / 2 / 4 26.3 / 26.2 / 25.6.
Form form(int head_dim, int64_t rows, int64_t walk, int64_t heads) {
  Form f;
  const int64_t tiles = (walk + 63) / 64, wide = (rows + 127) / 128 * heads, narrow = (rows + 63) / 64 * heads;
  f.groups = (head_dim == 64 ? wide : narrow) <= 256 && tiles > 1 ? 2 : 1;
  f.nx = (int)((rows + 128 / f.groups - 1) / (128 / f.groups));
  const int64_t blocks = f.nx * heads;
  f.splits = 1;
  while (f.splits < MAX_SPLITS && blocks * f.splits <= 128 && tiles >= 4 * f.groups * f.splits) f.splits *= 2;
  return f;
}
constexpr int FEW_ROWS = 32;
// Blocks that share a walk over the states. Estimated in us, for what a block at a time on each CU takes: 3 for a block's beginning and end, for
// every step of its wavefronts over tiles (128 KB) what a CU's rate of reading (37 GB/s) or the memory's (5.9 TB/s) takes, 5 for the second kernel.
// Measured for 1 / 2 / 4 / 8: 16 samples x 16384 states, 8 key heads of 128 242 / 182 / 187 / 198 (estimate 227 / 189 / 193 / 198); 8 x 1024, 16 of 64
// 11.0 / 12.9 / 16.4.
int few_splits(int head_dim, int64_t walk, int64_t heads) {
  const int64_t tiles = (walk + 31) / 32, waves = head_dim == 64 ? 16 : 8;
  int best = 1;
  double least = 1e30;
  for (int s = 1; s <= MAX_SPLITS && (s == 1 || tiles >= waves * s); ++s) {
    const int64_t blocks = heads * s, rounds = (blocks + 255) / 256, steps = (tiles + waves * s - 1) / (waves * s);
    const double step = std::max(131072 / 37e3, (blocks < 256 ? blocks : 256) * (131072 / 5.9e6));
    const double t = rounds * (3.0 + steps * step) + (s > 1 ? 5.0 : 0.0);
    if (t < least) { least = t; best = s; }
  }
  return best;
}
// The same for backward, in us: 4 for a block's beginning and end, 3 for a tile.
int few_bwd_splits(int head_dim, int64_t walk, int64_t heads) {
  const int64_t tiles = (walk + 31) / 32, waves = head_dim == 64 ? 8 : 4;
  int best = 1;
  double least = 1e30;
  for (int s = 1; s <= MAX_SPLITS && (s == 1 || tiles >= waves * s); ++s) {
    const int64_t blocks = heads * s, rounds = (blocks + 255) / 256, steps = (tiles + waves * s - 1) / (waves * s);
    const double t = rounds * (4.0 + steps * 3.0) + (s > 1 ? 5.0 : 0.0);
    if (t < least) { least = t; best = s; }
  }
  return best;
}
// Blocks that share the rows of a head (cross_bwd_short_kernel), one at a time on each CU. Estimated in us: 5 for a block's beginning and end, 2.5
// for 128 rows, 5 for the kernel that adds up the blocks' parts.
int short_splits(int64_t rows, int64_t heads) {
  const int64_t tiles = (rows + 127) / 128;
  int best = 1;
  double least = 1e30;
  for (int s = 1; s <= MAX_SPLITS && s <= tiles; ++s) {
    const double t = (double)((heads * s + 255) / 256) * (5.0 + 2.5 * ((tiles + s - 1) / s)) + (s > 1 ? 5.0 : 0.0);
    if (t < least) { least = t; best = s; }
  }
  return best;
}
// The same for forward, where blocks leave nothing to add up: as many as the chip holds at a time.
int short_blocks(int head_dim, int64_t rows, int64_t heads) {
  const int64_t room = head_dim == 64 ? 512 : 256, tiles = (rows + 127) / 128, most = std::max<int64_t>(1, room / heads);
  return (int)(tiles < most ? tiles : most);
}
inline size_t up256(size_t v) { return (v + 255) & ~(size_t)255; }

struct FwdPlan { bool few, one; Form form; size_t o_bytes, total; };
FwdPlan fwd_plan(int head_dim, const CrossShape& s) {
  FwdPlan f;
  const int64_t rows = (int64_t)s.q_len * s.group, heads = (int64_t)s.batch * s.kv_heads;
  f.one = s.kv_len <= SHORT_KEYS;
  f.few = !f.one && rows <= FEW_ROWS;
  f.form = f.one ? Form{1, short_blocks(head_dim, rows, heads), 1} : f.few ? Form{1, 1, few_splits(head_dim, s.kv_len, heads)} : form(head_dim, rows, s.kv_len, heads);
  const size_t all = (size_t)(heads * rows * f.form.splits);
  f.o_bytes = f.form.splits > 1 ? up256(all * head_dim * 4) : 0;
  f.total = f.form.splits > 1 ? f.o_bytes + up256(all * 4) : 0;
  return f;
}
struct BwdPlan { bool one, few; Form q, kv; size_t delta_bytes, total; };   // the parts of dq and those of dk and dv share memory one after the other
BwdPlan bwd_plan(int head_dim, const CrossShape& s) {
  BwdPlan f;
  const int64_t rows = (int64_t)s.q_len * s.group, heads = (int64_t)s.batch * s.kv_heads;
  f.one = s.kv_len <= (head_dim == 64 ? SHORT_BWD_KEYS<64> : SHORT_BWD_KEYS<128>);
  if (f.one) {
    f.few = false;
    f.q = f.kv = Form{1, 1, short_splits(rows, heads)};
    f.delta_bytes = 0;
    f.total = f.kv.splits > 1 ? up256((size_t)(heads * s.kv_len * f.kv.splits) * 2 * head_dim * 4) : 256;   // (never 0: one is always passed)
    return f;
  }
  f.few = rows <= FEW_ROWS;
  if (f.few) {
    f.q = f.kv = Form{1, 1, few_bwd_splits(head_dim, s.kv_len, heads)};
    f.delta_bytes = 0;
    f.total = f.q.splits > 1 ? up256((size_t)(heads * rows * f.q.splits) * (2 * head_dim + 1) * 4) : 256;
    return f;
  }
  f.q = form(head_dim, rows, s.kv_len, heads);
  f.kv = form(head_dim, s.kv_len, rows, heads);
  f.delta_bytes = up256((size_t)(heads * rows) * 4);
  const size_t dq = f.q.splits > 1 ? (size_t)(heads * rows * f.q.splits) * (2 * head_dim + 1) * 4 : 0;
  const size_t dkv = f.kv.splits > 1 ? (size_t)(heads * s.kv_len * f.kv.splits) * 2 * head_dim * 4 : 0;
  f.total = f.delta_bytes + up256(dq > dkv ? dq : dkv);
  return f;
}

template <int THREADS = 256, class Kernel, class... Args>
void launch(Kernel kernel, int64_t blocks, size_t lds, hipStream_t st, Args... args) {
  if (lds > 65536) (void)hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
  hipLaunchKernelGGL(kernel, dim3((unsigned)blocks), dim3(THREADS), lds, st, args...);
}

template <int D, bool F16>
void fwd(const CrossShape& s, const CrossOperands& p, hipStream_t st) {
  const FwdPlan f = fwd_plan(D, s);
  const int64_t heads = (int64_t)s.batch * s.kv_heads, rows = (int64_t)s.q_len * s.group;
  const FwdParts parts = {p.ws, (float*)((char*)p.ws + f.o_bytes), f.form.splits};
  constexpr size_t tile = 2 * Tile<D>::ELEMS * sizeof(bf16_t);   // K and V
  const int64_t blocks = cross_grid(s, f.form.nx, f.form.splits);
  if (f.few) launch<64 * FEW_WAVES<D>>(cross_few_kernel<D, F16>, blocks, std::max(FEW_WAVES<D> * tile / 2, (size_t)FEW_WAVES<D> * (D / 2 + 2) * 64 * sizeof(float)), st, s, p, parts);
  else if (f.one) launch(cross_fwd_short_kernel<D, F16>, blocks, SHORT_FWD_LDS<D>, st, s, p, f.form.nx);
  else if (f.form.groups == 2) launch(cross_fwd_kernel<D, F16, 2>, blocks, 4 * tile, st, s, p, f.form.nx, parts);
  else launch(cross_fwd_kernel<D, F16, 1>, blocks, std::max(2 * tile, (size_t)4 * RowStage<D, F16>::ELEMS * 2), st, s, p, f.form.nx, parts);
  if (f.form.splits > 1) {
    int groups = 1;
    while (groups < JOIN_GROUPS<D> && 2 * groups < f.form.splits) groups *= 2;
    launch(cross_join_kernel<D, F16>, (heads * rows * (D / 8) * groups + 255) / 256, 0, st, s, p, parts, groups);
  }
}

template <int D, bool F16>
void bwd(const CrossShape& s, const CrossOperands& p, hipStream_t st) {
  const BwdPlan f = bwd_plan(D, s);
  const int64_t heads = (int64_t)s.batch * s.kv_heads, rows = (int64_t)s.q_len * s.group;
  float *delta = p.ws, *memory = (float*)((char*)p.ws + f.delta_bytes);
  constexpr size_t tile = 2 * Tile<D>::ELEMS * sizeof(bf16_t), rows_out = (size_t)4 * RowStage<D, F16>::ELEMS * 2;
  if (f.one) {
    const BwdParts parts = {p.ws, f.kv.splits, nullptr};
    static_assert(4 * 2 * D * 16 * 4 <= SHORT_BWD_LDS<D>, "dK and dV of 32 states of four wavefronts");
    const int64_t blocks = cross_grid(s, 1, f.kv.splits);
    if (s.kv_len <= 64) launch(cross_bwd_short_kernel<D, F16, 2>, blocks, SHORT_BWD_LDS<D>, st, s, p, parts);
    else if constexpr (D == 64) {
      if (s.kv_len <= 96) launch(cross_bwd_short_kernel<D, F16, 3>, blocks, SHORT_BWD_LDS<D>, st, s, p, parts);
      else launch(cross_bwd_short_kernel<D, F16, 4>, blocks, SHORT_BWD_LDS<D>, st, s, p, parts);
    }
    if (f.kv.splits > 1) launch(cross_sum_kernel<D, F16>, (heads * s.kv_len * 2 * (D / 8) + 255) / 256, 0, st, s, p, parts);
    return;
  }
  if (f.few) {
    const BwdParts parts = {p.ws, f.q.splits, p.ws + heads * rows * f.q.splits * 2 * D};
    static_assert(RowStage<D, F16>::ELEMS <= 2 * 32 * D, "32 rows on their way out in the room of K and V");
    launch<64 * FEW_BWD_WAVES<D>>(cross_bwd_few_kernel<D, F16>, cross_grid(s, 1, f.q.splits), FEW_BWD_LDS<D>, st, s, p, parts);
    if (f.q.splits > 1) launch(cross_sum_rows_kernel<D, F16>, (heads * rows + 3) / 4, 0, st, s, p, parts, (float*)nullptr);
    return;
  }
  {
    const BwdParts parts = {memory, f.q.splits, memory + heads * rows * f.q.splits * 2 * D};
    const int64_t blocks = cross_grid(s, f.q.nx, f.q.splits);
    if (f.q.groups == 2) launch(cross_dq_kernel<D, F16, 2>, blocks, 4 * tile, st, s, p, f.q.nx, delta, parts);
    else launch(cross_dq_kernel<D, F16, 1>, blocks, std::max(2 * tile, rows_out), st, s, p, f.q.nx, delta, parts);
    if (f.q.splits > 1) launch(cross_sum_rows_kernel<D, F16>, (heads * rows + 3) / 4, 0, st, s, p, parts, delta);
  }
  {
    const BwdParts parts = {memory, f.kv.splits, nullptr};
    const int64_t blocks = cross_grid(s, f.kv.nx, f.kv.splits);
    constexpr size_t stage = tile + 512, meet = (size_t)2 * D * 2 * 64 * sizeof(float);   // two wavefronts' dK and dV
    if (f.kv.groups == 2) launch(cross_dkdv_kernel<D, F16, 2>, blocks, std::max(4 * stage, meet), st, s, p, f.kv.nx, (const float*)delta, parts);
    else launch(cross_dkdv_kernel<D, F16, 1>, blocks, std::max(2 * stage, rows_out), st, s, p, f.kv.nx, (const float*)delta, parts);
    if (f.kv.splits > 1) launch(cross_sum_kernel<D, F16>, (heads * s.kv_len * 2 * (D / 8) + 255) / 256, 0, st, s, p, parts);
  }
}

}  // namespace

size_t cross_tiles_fwd_ws_bytes(int head_dim, const CrossShape& s) { return fwd_plan(head_dim, s).total; }
size_t cross_tiles_bwd_ws_bytes(int head_dim, const CrossShape& s) { return bwd_plan(head_dim, s).total; }
void launch_cross_tiles_fwd(bool f16, int head_dim, const CrossShape& s, const CrossOperands& p, hipStream_t st) {
  if (f16) head_dim == 64 ? fwd<64, true>(s, p, st) : fwd<128, true>(s, p, st);
  else head_dim == 64 ? fwd<64, false>(s, p, st) : fwd<128, false>(s, p, st);
}
void launch_cross_tiles_bwd(bool f16, int head_dim, const CrossShape& s, const CrossOperands& p, hipStream_t st) {
  if (f16) head_dim == 64 ? bwd<64, true>(s, p, st) : bwd<128, true>(s, p, st);
  else head_dim == 64 ? bwd<64, false>(s, p, st) : bwd<128, false>(s, p, st);
}

}  // namespace slapo
