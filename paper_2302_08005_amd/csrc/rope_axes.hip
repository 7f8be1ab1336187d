// Rotary positions of several axes. Tokens of an image or a video have a position per axis (time, height, width), and every axis turns
// its own pairs of a head: pair j, of axis a, by positions[row][a] * base^(-step(j)).
//
// A pass reads and writes the turned heads once and is bound by memory; the angles of a row are common to all of its heads. A block
// computes those of the rows that it handles into LDS, as (cos, sin), and its threads then turn eight elements (four pairs, 16 bytes
// of a 16-bit type) at a time.
#include <algorithm>

#include "common.h"
#include "kernels.h"

namespace slapo {

namespace {

// (cos, sin) of `turns` full turns. The whole turns leave in 64 bits: 2^31 positions at one radian each are 3.4e8 turns, of which 64 bits
// leave 6e-8. What is left goes through the nearest quarter, so that the 32-bit functions see at most an eighth of a turn.
__device__ __forceinline__ float2 unit_at(double turns) {
  const double part = turns - rint(turns), quarter = rint(4.0 * part);
  const float half = (float)(0.5 * (4.0 * part - quarter));   // of half turns
  const float s = sinpif(half), c = cospif(half);
  switch ((int)quarter & 3) {
    case 0: return make_float2(c, s);
    case 1: return make_float2(-s, c);
    case 2: return make_float2(-c, -s);
    default: return make_float2(s, -c);
  }
}

template <typename T>
__global__ __launch_bounds__(256) void rope_axes_kernel(RopeAxes r, int group_rows, const int32_t* __restrict__ positions, const T* in, T* out) {
  extern __shared__ __attribute__((aligned(16))) float2 unit[];   // [group_rows][head_dim / 2]
  __shared__ double turns_per_step[ROPE_MAX_PAIRS];
  __shared__ int axis_of[ROPE_MAX_PAIRS];
  const int pairs = r.head_dim / 2, chunks = r.heads * (r.head_dim / 8);
  for (int j = threadIdx.x; j < r.turned; j += 256) {
    int a = 0;
    while (j >= r.first[a + 1]) ++a;
    const double step = r.own_ladders ? (double)(j - r.first[a]) / (r.first[a + 1] - r.first[a]) : 2.0 * j / r.head_dim;
    const double turns = exp2(-step * r.log2_base) * 0.15915494309189533577;   // 1 / (2 pi)
    turns_per_step[j] = r.inverse ? -turns : turns;
    axis_of[j] = a;
  }
  for (int64_t row0 = (int64_t)blockIdx.x * group_rows; row0 < r.rows; row0 += (int64_t)gridDim.x * group_rows) {
    const int n = r.rows - row0 < group_rows ? (int)(r.rows - row0) : group_rows;
    __syncthreads();
    for (int i = threadIdx.x; i < n * r.turned; i += 256) {
      const int row = i / r.turned, j = i - row * r.turned;
      unit[row * pairs + j] = unit_at((double)positions[(row0 + row) * r.axes + axis_of[j]] * turns_per_step[j]);
    }
    __syncthreads();
    for (int i = threadIdx.x; i < n * chunks; i += 256) {
      const int row = i / chunks, c = 8 * (i - row * chunks), j0 = (c % r.head_dim) / 2;
      float v[8];
      load8(in + (row0 + row) * r.in_stride + c, v);
#pragma unroll
      for (int p = 0; p < 4; ++p)
        if (j0 + p < r.turned) {
          const float2 u = unit[row * pairs + j0 + p];
          turn_pair(v[2 * p], v[2 * p + 1], u.x, u.y);
        }
      store8(out + (row0 + row) * r.out_stride + c, v);
    }
  }
}

template <typename T>
void rope_axes(const RopeAxes& r, const int32_t* positions, const void* in, void* out, hipStream_t st) {
  // Rows at a time: as many as give every thread something to turn (at most 8 KB of LDS), while four blocks of them are left for each CU. us, one row
  // / so many: 32768 rows of one head of 64 23.9 / 6.9, of 4 heads of 128 28.8 / 16.6; 8192 of 16 heads of 64 11.9 / 9.7; but 512 of one of 128 3.6 / 4.7.
  const int64_t chunks = (int64_t)r.heads * (r.head_dim / 8), some = std::min<int64_t>(256 / chunks, r.rows / 1024);
  const int group_rows = some > 1 ? (int)some : 1;
  const int64_t groups = (r.rows + group_rows - 1) / group_rows;
  const unsigned grid = (unsigned)(groups < 4096 ? groups : 4096);
  hipLaunchKernelGGL(rope_axes_kernel<T>, dim3(grid), dim3(256), (size_t)group_rows * (r.head_dim / 2) * sizeof(float2), st, r, group_rows, positions,
                     (const T*)in, (T*)out);
}

}  // namespace

void launch_rope_axes(int dtype, const RopeAxes& r, const int32_t* positions, const void* in, void* out, hipStream_t st) {
  if (dtype == DT_FP32) rope_axes<float>(r, positions, in, out, st);
  else if (dtype == DT_FP16) rope_axes<f16_t>(r, positions, in, out, st);
  else rope_axes<bf16_t>(r, positions, in, out, st);
}

}  // namespace slapo
