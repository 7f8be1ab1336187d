// The norm of many gradient arrays taken together, and their scaling by what a bound on it leaves (clipping). Both are bound by memory:
// one pass reads everything for the sum of squares, another reads it again and writes the scaled arrays.
//
// The arrays are cut into segments; a plan in device memory says which array each belongs to. A block takes every grid-th segment, so the
// order of the sums is fixed by the plan alone. Squares are taken and added in 64 bits: those of 16- and 32-bit values neither overflow
// nor vanish there, and the vector units have the room (an element costs a conversion and a multiply-add).
#include "common.h"
#include "kernels.h"

namespace slapo {

namespace {

constexpr int TABLE = 64;   // entries that one launch writes into a plan
struct GradTable { GradEntry e[TABLE]; };

__global__ __launch_bounds__(256) void grad_plan_kernel(GradTable table, int first_entry, int64_t segment, int64_t segments, GradEntry* entries,
                                                        int32_t* map, unsigned* counter) {
  const GradEntry e = table.e[blockIdx.x];
  const int64_t per = segment / (e.dtype == DT_FP32 ? 4 : 2), n = (e.count + per - 1) / per;
  if (threadIdx.x == 0) {
    entries[first_entry + blockIdx.x] = e;
    if (first_entry + blockIdx.x == 0) *counter = 0;
  }
  for (int64_t i = threadIdx.x; i < n && e.first + i < segments; i += 256) map[e.first + i] = first_entry + blockIdx.x;
}

constexpr int IN_FLIGHT = 4;   // loads of eight elements that a thread has on their way

// elements [from, to) of a segment's array, `from` a multiple of 8
template <typename T>
__device__ __forceinline__ double sum_squares(const T* x, int64_t from, int64_t to) {
  double s[IN_FLIGHT] = {};
  const auto add = [](double& s, const Raw8<T>& r) {
    float v[8];
    r.get(v);
#pragma unroll
    for (int k = 0; k < 8; ++k) s = fma((double)v[k], (double)v[k], s);
  };
  int64_t i = from + 8 * (int64_t)threadIdx.x;
  for (; i + 8 * 256 * (IN_FLIGHT - 1) + 8 <= to; i += 8 * 256 * IN_FLIGHT) {
    Raw8<T> r[IN_FLIGHT];
#pragma unroll
    for (int u = 0; u < IN_FLIGHT; ++u) r[u].load(x + i + 8 * 256 * u);
#pragma unroll
    for (int u = 0; u < IN_FLIGHT; ++u) add(s[u], r[u]);
  }
  for (; i + 8 <= to; i += 8 * 256) {
    Raw8<T> r;
    r.load(x + i);
    add(s[0], r);
  }
  for (; i < to; ++i) {   // (only the last thread's)
    const double v = (double)to_f32(x[i]);
    s[0] = fma(v, v, s[0]);
  }
  return (s[0] + s[1]) + (s[2] + s[3]);
}

// Sum over the block, in thread 0.
__device__ __forceinline__ double block_sum(double v, double* shared) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_down(v, o, 64);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) shared[threadIdx.x >> 6] = v;
  __syncthreads();
  return shared[0] + shared[1] + shared[2] + shared[3];
}

// The block that is done last adds up the blocks' sums, in their order. (The counter ends at the number of blocks' last value and wraps to 0.)
__global__ __launch_bounds__(256) void grad_sumsq_kernel(int64_t segments, int64_t segment, const GradEntry* __restrict__ entries,
                                                         const int32_t* __restrict__ map, double* partials, unsigned* counter, int accumulate,
                                                         double* sumsq) {
  __shared__ double shared[4];
  __shared__ bool last;
  double s = 0.0;
  for (int64_t g = blockIdx.x; g < segments; g += gridDim.x) {
    const GradEntry e = entries[map[g]];
    const int64_t per = segment / (e.dtype == DT_FP32 ? 4 : 2), from = (g - e.first) * per, to = from + per < e.count ? from + per : e.count;
    if (e.dtype == DT_FP32) s += sum_squares((const float*)e.in, from, to);
    else if (e.dtype == DT_FP16) s += sum_squares((const f16_t*)e.in, from, to);
    else s += sum_squares((const bf16_t*)e.in, from, to);
  }
  s = block_sum(s, shared);
  if (threadIdx.x == 0) {
    // Sums and counter are device-wide atomics, which go past the caches that blocks on other dies do not share, so order between the two is all
    // that is wanted, and no cache is written back.
    __hip_atomic_store(partials + blockIdx.x, s, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // the sum is there
    last = atomicInc(counter, gridDim.x - 1) == gridDim.x - 1;
  }
  __syncthreads();
  if (!last) return;
  double t = 0.0;
  for (unsigned i = threadIdx.x; i < gridDim.x; i += 256) t += __hip_atomic_load(partials + i, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  t = block_sum(t, shared);
  if (threadIdx.x == 0) *sumsq = (accumulate ? *sumsq : 0.0) + t;
}

template <typename T>
__device__ __forceinline__ void scale_segment(const T* in, T* out, int64_t from, int64_t to, float factor, float step) {
  const auto put = [&](int64_t i, const Raw8<T>& r) {
    float v[8];
    r.get(v);
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = v[k] * step * factor;
    store8(out + i, v);
  };
  int64_t i = from + 8 * (int64_t)threadIdx.x;
  for (; i + 8 * 256 * (IN_FLIGHT - 1) + 8 <= to; i += 8 * 256 * IN_FLIGHT) {
    Raw8<T> r[IN_FLIGHT];
#pragma unroll
    for (int u = 0; u < IN_FLIGHT; ++u) r[u].load(in + i + 8 * 256 * u);
#pragma unroll
    for (int u = 0; u < IN_FLIGHT; ++u) put(i + 8 * 256 * u, r[u]);
  }
  for (; i + 8 <= to; i += 8 * 256) {
    Raw8<T> r;
    r.load(in + i);
    put(i, r);
  }
  for (; i < to; ++i) from_f32(out[i], to_f32(in[i]) * step * factor);
}

// Segments are taken from the last to the first: the sums were taken the other way round, and what they read last the caches still hold.
__global__ __launch_bounds__(256) void grad_clip_kernel(int64_t segments, int64_t segment, const GradEntry* __restrict__ entries,
                                                        const int32_t* __restrict__ map, const double* __restrict__ sumsq, float max_norm,
                                                        float* __restrict__ norm_out) {
  const double norm = sqrt(*sumsq);
  if (norm_out && blockIdx.x == 0 && threadIdx.x == 0) *norm_out = (float)norm;
  const bool scaled = norm > (double)max_norm && norm < INFINITY;   // (a norm that is no number: the gradients stay as they are)
  // (in two factors, so that neither is below the normal 32-bit numbers where the norm is 2^100 times the bound)
  const double ratio = scaled ? (double)max_norm / norm : 1.0;
  const float step = ratio < 0x1p-100 ? 0x1p-64f : 1.f, factor = (float)(ratio / (double)step);
  for (int64_t g = segments - 1 - blockIdx.x; g >= 0; g -= gridDim.x) {
    const GradEntry e = entries[map[g]];
    if (!scaled && e.in == e.out) continue;
    const int64_t per = segment / (e.dtype == DT_FP32 ? 4 : 2), from = (g - e.first) * per, to = from + per < e.count ? from + per : e.count;
    if (e.dtype == DT_FP32) scale_segment((const float*)e.in, (float*)e.out, from, to, factor, step);
    else if (e.dtype == DT_FP16) scale_segment((const f16_t*)e.in, (f16_t*)e.out, from, to, factor, step);
    else scale_segment((const bf16_t*)e.in, (bf16_t*)e.out, from, to, factor, step);
  }
}

unsigned grad_grid(int64_t segments) { return (unsigned)(segments < 1 ? 1 : segments < GRAD_BLOCKS ? segments : GRAD_BLOCKS); }

}  // namespace

GradPlanLayout grad_plan_layout(int64_t n, int64_t segments) {
  GradPlanLayout L;
  const auto up = [](size_t v) { return (v + 255) & ~(size_t)255; };
  L.entries = 256;   // (behind the counter)
  L.map = up(L.entries + (size_t)n * sizeof(GradEntry));
  L.partials = up(L.map + (size_t)segments * sizeof(int32_t));
  L.total = L.partials + GRAD_BLOCKS * sizeof(double);
  return L;
}

void launch_grad_plan(int n, const GradEntry* entries, int64_t segments, int64_t segment, void* memory, hipStream_t st) {
  const GradPlanLayout L = grad_plan_layout(n, segments);
  char* m = (char*)memory;
  for (int at = 0; at < n || at == 0; at += TABLE) {
    GradTable table = {};
    const int some = n - at < TABLE ? n - at : TABLE;
    for (int i = 0; i < some; ++i) table.e[i] = entries[at + i];
    // (a plan without arrays has one entry of no elements, behind which nothing is looked up: its block clears the counter)
    hipLaunchKernelGGL(grad_plan_kernel, dim3(some > 0 ? some : 1), dim3(256), 0, st, table, at, segment, segments, (GradEntry*)(m + L.entries),
                       (int32_t*)(m + L.map), (unsigned*)m);
  }
}

void launch_grad_sumsq(int64_t n, int64_t segments, int64_t segment, void* memory, int accumulate, double* sumsq, hipStream_t st) {
  const GradPlanLayout L = grad_plan_layout(n, segments);
  char* m = (char*)memory;
  hipLaunchKernelGGL(grad_sumsq_kernel, dim3(grad_grid(segments)), dim3(256), 0, st, segments, segment, (const GradEntry*)(m + L.entries),
                     (const int32_t*)(m + L.map), (double*)(m + L.partials), (unsigned*)m, accumulate, sumsq);
}

void launch_grad_clip(int64_t n, int64_t segments, int64_t segment, void* memory, const double* sumsq, float max_norm, float* norm, hipStream_t st) {
  const GradPlanLayout L = grad_plan_layout(n, segments);
  char* m = (char*)memory;
  hipLaunchKernelGGL(grad_clip_kernel, dim3(grad_grid(segments)), dim3(256), 0, st, segments, segment, (const GradEntry*)(m + L.entries),
                     (const int32_t*)(m + L.map), sumsq, max_norm, norm);
}

}  // namespace slapo
