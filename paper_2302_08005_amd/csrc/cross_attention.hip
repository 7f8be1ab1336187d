// Cross attention: the query tokens of a sample attend to the states of another sequence (an encoder's, of another length, with a
// visible length per sample). o_i = sum_j p_ij v_j, p_ij = exp(s_ij - lse_i), s_ij = scale q_i . k_j over the visible j.
//
// 16-bit types: cross_tiles.hip. Here the fp32 mode, which checks others: a block of four wavefronts owns 16 rows (queries, or states for dK/dV) of one (sample, key
// head) and walks the other sequence in chunks of CHUNK. Products on v_mfma_f32_16x16x4_f32: inputs, products and sums in 32 bits. The four
// wavefronts share the chunk's score tiles of 16 x 16, whose softmax values stay in LDS, then, behind a barrier, the 16-wide column tiles of
// the outputs. States beyond the visible length are read as zeros, whatever lies there.
#include <algorithm>

#include "cross_attention.h"

namespace slapo {

namespace {

constexpr int CHUNK = 128, PITCH = CHUNK + 4;   // floats per LDS row: 16 rows x 16 bytes meet every bank once

__device__ __forceinline__ float4 load4(const float* p) { return *reinterpret_cast<const float4*>(p); }
__device__ __forceinline__ void store4(float* p, const float (&v)[4]) { *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]); }

// 16 rows x D, this lane's share: row lane % 16, columns 16 c + 4 (lane / 16) ..; a row that is not there: zeros
template <int D>
struct RowFrags {
  float4 v[D / 16];
  __device__ __forceinline__ void load(const float* row, int g, bool there) {
#pragma unroll
    for (int c = 0; c < D / 16; ++c) v[c] = there ? load4(row + 16 * c + 4 * g) : make_float4(0.f, 0.f, 0.f, 0.f);
  }
};
// element r: row 4 (lane / 16) + r of a, row lane % 16 of b
template <int D>
__device__ __forceinline__ f32x4_t rows_times_rows(const RowFrags<D>& a, const RowFrags<D>& b) {
  f32x4_t acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int c = 0; c < D / 16; ++c) {
    acc = __builtin_amdgcn_mfma_f32_16x16x4f32(a.v[c].x, b.v[c].x, acc, 0, 0, 0);
    acc = __builtin_amdgcn_mfma_f32_16x16x4f32(a.v[c].y, b.v[c].y, acc, 0, 0, 0);
    acc = __builtin_amdgcn_mfma_f32_16x16x4f32(a.v[c].z, b.v[c].z, acc, 0, 0, 0);
    acc = __builtin_amdgcn_mfma_f32_16x16x4f32(a.v[c].w, b.v[c].w, acc, 0, 0, 0);
  }
  return acc;
}
// acc + sum over rows 0 .. n - 1 of a chunk of w[lane % 16][row] * x(row)[column lane % 16 of 16]; element r: column 4 (lane / 16) + r, for
// row lane % 16 of w. x(row): element of this lane's column in that row; rows from n on (to the next multiple of 16) count as zeros.
template <class X>
__device__ __forceinline__ f32x4_t weighted_rows(f32x4_t acc, const float* w, int n, int g, X&& x) {
  constexpr int U = CHUNK / 16;   // tiles of 16 rows in flight, all of a chunk: the walk is a chain of load latencies
  for (int t0 = 0; t0 < n; t0 += 16 * U) {
    float v[U][4];
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int s = 0; s < 4; ++s) {
        const int row = t0 + 16 * u + 4 * g + s;
        v[u][s] = x(min(row, n - 1));
        v[u][s] = row < n ? v[u][s] : 0.f;
      }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (t0 + 16 * u >= n) break;   // (uniform)
      const float4 wv = *reinterpret_cast<const float4*>(w + t0 + 16 * u + 4 * g);
      acc = __builtin_amdgcn_mfma_f32_16x16x4f32(v[u][0], wv.x, acc, 0, 0, 0);
      acc = __builtin_amdgcn_mfma_f32_16x16x4f32(v[u][1], wv.y, acc, 0, 0, 0);
      acc = __builtin_amdgcn_mfma_f32_16x16x4f32(v[u][2], wv.z, acc, 0, 0, 0);
      acc = __builtin_amdgcn_mfma_f32_16x16x4f32(v[u][3], wv.w, acc, 0, 0, 0);
    }
  }
  return acc;
}
template <class Op>
__device__ __forceinline__ float over16(float v, Op&& op) {
#pragma unroll
  for (int o = 8; o > 0; o >>= 1) v = op(v, __shfl_xor(v, o, 16));
  return v;
}
__device__ __forceinline__ float sum2(float a, float b) { return a + b; }
__device__ __forceinline__ float max2(float a, float b) { return fmaxf(a, b); }

template <int D>
__global__ __launch_bounds__(256) void cross_fwd_f32_kernel(CrossShape sh, CrossOperands p) {
  __shared__ __attribute__((aligned(16))) float prob[16 * PITCH];
  __shared__ float top[16], total[16], shrink[16];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, i = lane & 15, g = lane >> 4;
  const int b = blockIdx.z, h = blockIdx.y, r0 = blockIdx.x * 16;
  const CrossRows rows(sh);
  const int n_rows = rows.count(), n_keys = visible(sh, p.lens, b), my_row = min(r0 + i, n_rows - 1);
  const int64_t head0 = (int64_t)h * sh.group * D;
  const float* q = (const float*)p.q + (int64_t)b * sh.q_len * sh.q_stride + head0;
  const float* k = (const float*)p.k + (int64_t)b * sh.kv_len * sh.kv_stride + h * D;
  const float* v = (const float*)p.v + (int64_t)b * sh.kv_len * sh.kv_stride + h * D;
  RowFrags<D> qf;
  qf.load(q + rows.at(my_row, sh.q_stride, D), g, true);
  constexpr int MINE = D / 64;
  f32x4_t acc[MINE];
#pragma unroll
  for (int m = 0; m < MINE; ++m) acc[m] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  if (threadIdx.x < 16) { top[threadIdx.x] = -INFINITY; total[threadIdx.x] = 0.f; }
  for (int j0 = 0; j0 < n_keys; j0 += CHUNK) {
    const int n = min(CHUNK, n_keys - j0), tiles = (n + 15) / 16;
    for (int t = wave; t < tiles; t += 4) {
      const int key = j0 + 16 * t + i;
      RowFrags<D> kf;
      kf.load(k + min(key, n_keys - 1) * sh.kv_stride, g, key < n_keys);
      f32x4_t s = rows_times_rows<D>(kf, qf);
#pragma unroll
      for (int r = 0; r < 4; ++r) s[r] = 16 * t + 4 * g + r < n ? s[r] * sh.scale : -INFINITY;
      *reinterpret_cast<f32x4_t*>(prob + i * PITCH + 16 * t + 4 * g) = s;
    }
    __syncthreads();
    {   // 16 threads per row
      const int row = threadIdx.x >> 4, c = threadIdx.x & 15;
      float* pr = prob + row * PITCH;
      float mx = top[row];
      for (int j = c; j < 16 * tiles; j += 16) mx = fmaxf(mx, pr[j]);
      mx = over16(mx, max2);
      const float base = mx == -INFINITY ? 0.f : mx;
      float sum = 0.f;
      for (int j = c; j < 16 * tiles; j += 16) {
        const float e = __expf(pr[j] - base);
        pr[j] = e;
        sum += e;
      }
      sum = over16(sum, sum2);
      if (c == 0) {
        const float less = __expf(top[row] - base);
        shrink[row] = less;
        total[row] = total[row] * less + sum;
        top[row] = mx;
      }
    }
    __syncthreads();
    const float less = shrink[i];
#pragma unroll
    for (int m = 0; m < MINE; ++m) {
#pragma unroll
      for (int r = 0; r < 4; ++r) acc[m][r] *= less;
      const float* col = v + j0 * sh.kv_stride + 16 * (wave + 4 * m) + i;
      acc[m] = weighted_rows(acc[m], prob + i * PITCH, n, g, [&](int row) { return col[row * sh.kv_stride]; });
    }
    __syncthreads();
  }
  __syncthreads();
  if (r0 + i < n_rows) {
    const float sum = total[i], inv = sum != 0.f ? 1.f / sum : 0.f;   // (a sum that is no number stays one)
    float* o = (float*)p.o + (int64_t)b * sh.q_len * sh.out_stride + head0 + rows.at(r0 + i, sh.out_stride, D);
#pragma unroll
    for (int m = 0; m < MINE; ++m) {
      const float out[4] = {acc[m][0] * inv, acc[m][1] * inv, acc[m][2] * inv, acc[m][3] * inv};
      store4(o + 16 * (wave + 4 * m) + 4 * g, out);
    }
    if (p.lse && wave == 0 && g == 0)
      p.lse[((int64_t)b * sh.heads + h * sh.group) * sh.q_len + rows.stat(r0 + i)] = sum != 0.f ? top[i] + __logf(sum) : -INFINITY;
  }
}

// delta = rowsum(dO * O) of the row lane % 16, in all lanes that hold a share of it
template <int D>
__device__ __forceinline__ float delta_of(const RowFrags<D>& dout, const RowFrags<D>& out) {
  float d = 0.f;
#pragma unroll
  for (int c = 0; c < D / 16; ++c) {
    d = fmaf(dout.v[c].x, out.v[c].x, d); d = fmaf(dout.v[c].y, out.v[c].y, d);
    d = fmaf(dout.v[c].z, out.v[c].z, d); d = fmaf(dout.v[c].w, out.v[c].w, d);
  }
  d += __shfl_xor(d, 16, 64);
  return d + __shfl_xor(d, 32, 64);
}

// dQ of the 16 rows of block x. LEAVE: also leaves their delta in p.ws, laid out as lse.
template <int D, bool LEAVE>
__device__ __forceinline__ void dq_f32(const CrossShape& sh, const CrossOperands& p, int x, float* grad) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, i = lane & 15, g = lane >> 4;
  const int b = blockIdx.z, h = blockIdx.y, r0 = x * 16;
  const CrossRows rows(sh);
  const int n_rows = rows.count(), n_keys = visible(sh, p.lens, b), my_row = min(r0 + i, n_rows - 1);
  const int64_t head0 = (int64_t)h * sh.group * D, stats = ((int64_t)b * sh.heads + h * sh.group) * sh.q_len;
  const float* q = (const float*)p.q + (int64_t)b * sh.q_len * sh.q_stride + head0;
  const float* k = (const float*)p.k + (int64_t)b * sh.kv_len * sh.kv_stride + h * D;
  const float* v = (const float*)p.v + (int64_t)b * sh.kv_len * sh.kv_stride + h * D;
  const int64_t out0 = (int64_t)b * sh.q_len * sh.out_stride + head0 + rows.at(my_row, sh.out_stride, D);
  RowFrags<D> qf, df, of;
  qf.load(q + rows.at(my_row, sh.q_stride, D), g, true);
  df.load((const float*)p.dout + out0, g, true);
  of.load((const float*)p.out + out0, g, true);
  const float lse = p.lse[stats + rows.stat(my_row)];
  const float my_delta = delta_of(df, of);
  if (LEAVE && wave == 0 && g == 0 && r0 + i < n_rows) p.ws[stats + rows.stat(my_row)] = my_delta;
  constexpr int MINE = D / 64;
  f32x4_t acc[MINE];
#pragma unroll
  for (int m = 0; m < MINE; ++m) acc[m] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  for (int j0 = 0; j0 < n_keys; j0 += CHUNK) {
    const int n = min(CHUNK, n_keys - j0), tiles = (n + 15) / 16;
    for (int t = wave; t < tiles; t += 4) {
      const int key = j0 + 16 * t + i;
      const int64_t at = min(key, n_keys - 1) * sh.kv_stride;
      RowFrags<D> kf, vf;
      kf.load(k + at, g, key < n_keys);
      vf.load(v + at, g, key < n_keys);
      const f32x4_t s = rows_times_rows<D>(kf, qf), dp = rows_times_rows<D>(vf, df);
      f32x4_t ds;
#pragma unroll
      for (int r = 0; r < 4; ++r) ds[r] = 16 * t + 4 * g + r < n ? __expf(s[r] * sh.scale - lse) * (dp[r] - (n_keys == 1 ? dp[r] : my_delta)) : 0.f;   // (a state alone: exactly 0)
      *reinterpret_cast<f32x4_t*>(grad + i * PITCH + 16 * t + 4 * g) = ds;
    }
    __syncthreads();
#pragma unroll
    for (int m = 0; m < MINE; ++m) {
      const float* col = k + j0 * sh.kv_stride + 16 * (wave + 4 * m) + i;
      acc[m] = weighted_rows(acc[m], grad + i * PITCH, n, g, [&](int row) { return col[row * sh.kv_stride]; });
    }
    __syncthreads();
  }
  if (r0 + i < n_rows) {
    float* o = (float*)p.dq + (int64_t)b * sh.q_len * sh.q_stride + head0 + rows.at(r0 + i, sh.q_stride, D);
#pragma unroll
    for (int m = 0; m < MINE; ++m) {
      const float out[4] = {acc[m][0] * sh.scale, acc[m][1] * sh.scale, acc[m][2] * sh.scale, acc[m][3] * sh.scale};
      store4(o + 16 * (wave + 4 * m) + 4 * g, out);
    }
  }
}

// dK and dV of the 16 states of block x; hidden ones get zeros. OWN: takes delta of its own, else finds it in p.ws.
template <int D, bool OWN>
__device__ __forceinline__ void dkdv_f32(const CrossShape& sh, const CrossOperands& p, int x, float* prob, float* grad) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, i = lane & 15, g = lane >> 4;
  const int b = blockIdx.z, h = blockIdx.y, k0 = x * 16;
  const CrossRows rows(sh);
  const int n_keys = visible(sh, p.lens, b), n_rows = k0 < n_keys ? rows.count() : 0;
  const int64_t head0 = (int64_t)h * sh.group * D, stats = ((int64_t)b * sh.heads + h * sh.group) * sh.q_len;
  const float* q = (const float*)p.q + (int64_t)b * sh.q_len * sh.q_stride + head0;
  const int64_t out0 = (int64_t)b * sh.q_len * sh.out_stride + head0;
  const float* dout = (const float*)p.dout + out0;
  const int64_t kv0 = (int64_t)b * sh.kv_len * sh.kv_stride + h * D;
  const bool seen = k0 + i < n_keys;
  RowFrags<D> kf, vf;
  kf.load((const float*)p.k + kv0 + min(k0 + i, sh.kv_len - 1) * sh.kv_stride, g, seen);
  vf.load((const float*)p.v + kv0 + min(k0 + i, sh.kv_len - 1) * sh.kv_stride, g, seen);
  constexpr int MINE = D / 64;
  f32x4_t dk[MINE], dv[MINE];
#pragma unroll
  for (int m = 0; m < MINE; ++m) dk[m] = dv[m] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  for (int r0 = 0; r0 < n_rows; r0 += CHUNK) {
    const int n = min(CHUNK, n_rows - r0), tiles = (n + 15) / 16;
    for (int t = wave; t < tiles; t += 4) {
      const int row = r0 + 16 * t + i, at = min(row, n_rows - 1);
      RowFrags<D> qf, df;
      qf.load(q + rows.at(at, sh.q_stride, D), g, row < n_rows);
      df.load(dout + rows.at(at, sh.out_stride, D), g, row < n_rows);
      float row_delta = 0.f;
      if constexpr (OWN) {
        RowFrags<D> of;
        of.load((const float*)p.out + out0 + rows.at(at, sh.out_stride, D), g, row < n_rows);
        row_delta = delta_of(df, of);
      }
      const f32x4_t s = rows_times_rows<D>(qf, kf), dp = rows_times_rows<D>(df, vf);
      f32x4_t pv, ds;
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int mine = 16 * t + 4 * g + r;
        const int64_t stat = stats + rows.stat(min(r0 + mine, n_rows - 1));
        const float e = seen && mine < n ? __expf(s[r] * sh.scale - p.lse[stat]) : 0.f;
        pv[r] = e;
        const float delta = n_keys == 1 ? dp[r] : OWN ? __shfl(row_delta, 4 * g + r, 64) : p.ws[stat];
        ds[r] = seen && mine < n ? e * (dp[r] - delta) : 0.f;
      }
      *reinterpret_cast<f32x4_t*>(prob + i * PITCH + 16 * t + 4 * g) = pv;
      *reinterpret_cast<f32x4_t*>(grad + i * PITCH + 16 * t + 4 * g) = ds;
    }
    __syncthreads();
#pragma unroll
    for (int m = 0; m < MINE; ++m) {
      const int col = 16 * (wave + 4 * m) + i;
      dv[m] = weighted_rows(dv[m], prob + i * PITCH, n, g, [&](int row) { return dout[rows.at(r0 + row, sh.out_stride, D) + col]; });
      dk[m] = weighted_rows(dk[m], grad + i * PITCH, n, g, [&](int row) { return q[rows.at(r0 + row, sh.q_stride, D) + col]; });
    }
    __syncthreads();
  }
  if (k0 + i < sh.kv_len) {
    const int64_t at = kv0 + (k0 + i) * sh.kv_stride;
#pragma unroll
    for (int m = 0; m < MINE; ++m) {
      const int col = 16 * (wave + 4 * m) + 4 * g;
      const float a[4] = {dk[m][0] * sh.scale, dk[m][1] * sh.scale, dk[m][2] * sh.scale, dk[m][3] * sh.scale};
      const float c[4] = {dv[m][0], dv[m][1], dv[m][2], dv[m][3]};
      store4((float*)p.dk + at + col, a);
      store4((float*)p.dv + at + col, c);
    }
  }
}

template <int D>
__global__ __launch_bounds__(256) void cross_dq_f32_kernel(CrossShape sh, CrossOperands p) {
  __shared__ __attribute__((aligned(16))) float grad[16 * PITCH];
  dq_f32<D, true>(sh, p, blockIdx.x, grad);
}
template <int D>
__global__ __launch_bounds__(256) void cross_dkdv_f32_kernel(CrossShape sh, CrossOperands p) {
  __shared__ __attribute__((aligned(16))) float prob[16 * PITCH], grad[16 * PITCH];
  dkdv_f32<D, false>(sh, p, blockIdx.x, prob, grad);
}
// Both in one launch: a third operand to read for the blocks of states, nothing to wait for.
template <int D>
__global__ __launch_bounds__(256, D == 64 ? 2 : 1) void cross_bwd_f32_kernel(CrossShape sh, CrossOperands p, int key_blocks) {
  __shared__ __attribute__((aligned(16))) float prob[16 * PITCH], grad[16 * PITCH];
  if ((int)blockIdx.x < key_blocks) dkdv_f32<D, true>(sh, p, blockIdx.x, prob, grad);   // (the longer ones first)
  else dq_f32<D, false>(sh, p, blockIdx.x - key_blocks, grad);
}

template <int D>
void fwd_f32(const CrossShape& s, const CrossOperands& p, hipStream_t st) {
  const unsigned blocks = (unsigned)(((int64_t)s.q_len * s.group + 15) / 16);
  hipLaunchKernelGGL((cross_fwd_f32_kernel<D>), dim3(blocks, s.kv_heads, s.batch), dim3(256), 0, st, s, p);
}
template <int D>
void bwd_f32(const CrossShape& s, const CrossOperands& p, hipStream_t st) {
  const unsigned blocks = (unsigned)(((int64_t)s.q_len * s.group + 15) / 16), key_blocks = (unsigned)(((int64_t)s.kv_len + 15) / 16);
  // One launch while every block has a CU: beyond that its registers, those of both, cost more blocks at a time than a launch does. us of backward, one
  // launch / two: 2 x 128 rows, 96 states, 4 heads of 64 (112 blocks) 12.0 / 18.9, of 128 24.1 / 34.3; 4 x 512, 512, 8 of 64 (2048) 200 / 178; 2 x 99,
  // 5, 20 of 128 (320) 44.8 / 28.4.
  if ((int64_t)(blocks + key_blocks) * s.kv_heads * s.batch <= 256) {
    hipLaunchKernelGGL((cross_bwd_f32_kernel<D>), dim3(key_blocks + blocks, s.kv_heads, s.batch), dim3(256), 0, st, s, p, (int)key_blocks);
    return;
  }
  hipLaunchKernelGGL((cross_dq_f32_kernel<D>), dim3(blocks, s.kv_heads, s.batch), dim3(256), 0, st, s, p);
  hipLaunchKernelGGL((cross_dkdv_f32_kernel<D>), dim3(key_blocks, s.kv_heads, s.batch), dim3(256), 0, st, s, p);
}

}  // namespace

size_t cross_attn_fwd_ws_bytes(int dtype, int head_dim, const CrossShape& s) { return dtype == DT_FP32 ? 0 : cross_tiles_fwd_ws_bytes(head_dim, s); }
size_t cross_attn_bwd_ws_bytes(int dtype, int head_dim, const CrossShape& s) {
  return dtype == DT_FP32 ? (size_t)s.batch * s.heads * s.q_len * sizeof(float) : cross_tiles_bwd_ws_bytes(head_dim, s);
}
void launch_cross_attn_fwd(int dtype, int head_dim, const CrossShape& s, const CrossOperands& p, hipStream_t st) {
  if (dtype != DT_FP32) launch_cross_tiles_fwd(dtype == DT_FP16, head_dim, s, p, st);
  else head_dim == 64 ? fwd_f32<64>(s, p, st) : fwd_f32<128>(s, p, st);
}
void launch_cross_attn_bwd(int dtype, int head_dim, const CrossShape& s, const CrossOperands& p, hipStream_t st) {
  if (dtype != DT_FP32) launch_cross_tiles_bwd(dtype == DT_FP16, head_dim, s, p, st);
  else head_dim == 64 ? bwd_f32<64>(s, p, st) : bwd_f32<128>(s, p, st);
}

}  // namespace slapo
