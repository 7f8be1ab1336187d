// The norm of many gradient arrays taken together, and their scaling by what a bound on it leaves (clipping). Both are bound by memory:
// one pass reads everything for the sum of squares, another reads it again and writes the scaled arrays.
//
// The arrays are cut into segments, which a plan in device memory lists. A block takes every grid-th segment, so the order of the sums is fixed by the
// plan alone. Squares are taken and added in 64 bits: those of 16- and 32-bit values neither overflow nor vanish there, and the vector units have the
// room (an element costs a conversion and a multiply-add). 302M bf16 values: sums 105 us (5.7 TB/s), clipping 211 us (5.7 TB/s read and written).
#include "common.h"
#include "kernels.h"

namespace slapo {

namespace {

typedef unsigned int u32x4_t __attribute__((ext_vector_type(4)));

constexpr int TABLE = 64;   // arrays that one launch cuts into a plan's segments
struct GradTable { GradArray a[TABLE]; };

__global__ __launch_bounds__(256) void grad_plan_kernel(GradTable table, GradSegment* segments, unsigned* counter, int clear) {
  const GradArray a = table.a[blockIdx.x];
  const int64_t eb = a.dtype == DT_FP32 ? 4 : 2, per = GRAD_SEGMENT / eb, n = (a.count + per - 1) / per;
  if (clear && blockIdx.x == 0 && threadIdx.x == 0) *counter = 0;
  for (int64_t i = threadIdx.x; i < n; i += 256) {
    const int64_t left = a.count - i * per;
    segments[a.first + i] = {(const char*)a.in + i * GRAD_SEGMENT, (char*)a.out + i * GRAD_SEGMENT, (int32_t)(left < per ? left : per), a.dtype};
  }
}

// Threads of a block and loads of eight elements that a thread has on their way: of the sums, whose blocks meet at one counter (12 ns each: 25 MB on 2048
// blocks of 256 threads 40 us, on 768 25), few large blocks.
constexpr int SUM_THREADS = 1024, SUM_BLOCKS = 512, SUM_IN_FLIGHT = 2, IN_FLIGHT = 4;

template <typename T>
__device__ __forceinline__ double sum_squares(const T* x, int n) {
  double s[SUM_IN_FLIGHT] = {};
  const auto add = [](double& s, const Raw8<T>& r) {
    float v[8];
    r.get(v);
#pragma unroll
    for (int k = 0; k < 8; ++k) s = fma((double)v[k], (double)v[k], s);
  };
  int i = 8 * threadIdx.x;
  for (; i + 8 * SUM_THREADS * (SUM_IN_FLIGHT - 1) + 8 <= n; i += 8 * SUM_THREADS * SUM_IN_FLIGHT) {
    Raw8<T> r[SUM_IN_FLIGHT];
#pragma unroll
    for (int u = 0; u < SUM_IN_FLIGHT; ++u) r[u].load(x + i + 8 * SUM_THREADS * u);
#pragma unroll
    for (int u = 0; u < SUM_IN_FLIGHT; ++u) add(s[u], r[u]);
  }
  for (; i + 8 <= n; i += 8 * SUM_THREADS) {
    Raw8<T> r;
    r.load(x + i);
    add(s[0], r);
  }
  for (; i < n; ++i) {   // (only the last thread's)
    const double v = (double)to_f32(x[i]);
    s[0] = fma(v, v, s[0]);
  }
  return s[0] + s[1];
}

// Sum over the block, in thread 0.
__device__ __forceinline__ double block_sum(double v, double* shared) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_down(v, o, 64);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) shared[threadIdx.x >> 6] = v;
  __syncthreads();
  double sum = 0.0;
  if (threadIdx.x == 0)
    for (int i = 0; i < SUM_THREADS / 64; ++i) sum += shared[i];
  return sum;
}

// The block that is done last adds up the blocks' sums, in their order. (The counter ends at the number of blocks' last value and wraps to 0.)
__global__ __launch_bounds__(SUM_THREADS) void grad_sumsq_kernel(int64_t n, const GradSegment* __restrict__ segments, double* partials, unsigned* counter,
                                                         int accumulate, double* sumsq) {
  __shared__ double shared[SUM_THREADS / 64];
  __shared__ bool last;
  double s = 0.0;
  for (int64_t i = blockIdx.x; i < n; i += gridDim.x) {
    const GradSegment g = segments[i];
    if (g.dtype == DT_FP32) s += sum_squares((const float*)g.in, g.count);
    else if (g.dtype == DT_FP16) s += sum_squares((const f16_t*)g.in, g.count);
    else s += sum_squares((const bf16_t*)g.in, g.count);
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
  for (unsigned i = threadIdx.x; i < gridDim.x; i += SUM_THREADS) t += __hip_atomic_load(partials + i, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  t = block_sum(t, shared);
  if (threadIdx.x == 0) *sumsq = (accumulate ? *sumsq : 0.0) + t;
}

// Eight elements past the caches.
__device__ __forceinline__ void store8_past(bf16_t* p, const float (&v)[8]) {
  const u32x4_t w = {pack2<false>(v[0], v[1]), pack2<false>(v[2], v[3]), pack2<false>(v[4], v[5]), pack2<false>(v[6], v[7])};
  __builtin_nontemporal_store(w, reinterpret_cast<u32x4_t*>(p));
}
__device__ __forceinline__ void store8_past(f16_t* p, const float (&v)[8]) {
  const u32x4_t w = {pack2<true>(v[0], v[1]), pack2<true>(v[2], v[3]), pack2<true>(v[4], v[5]), pack2<true>(v[6], v[7])};
  __builtin_nontemporal_store(w, reinterpret_cast<u32x4_t*>(p));
}
__device__ __forceinline__ void store8_past(float* p, const float (&v)[8]) {
  __builtin_nontemporal_store(f32x4_t{v[0], v[1], v[2], v[3]}, reinterpret_cast<f32x4_t*>(p));
  __builtin_nontemporal_store(f32x4_t{v[4], v[5], v[6], v[7]}, reinterpret_cast<f32x4_t*>(p + 4));
}

template <bool PAST, typename T>
__device__ __forceinline__ void scale_segment(const T* in, T* out, int n, float factor, float step) {
  const auto put = [&](int i, const Raw8<T>& r) {
    float v[8];
    r.get(v);
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = v[k] * step * factor;
    if constexpr (PAST) store8_past(out + i, v);
    else store8(out + i, v);
  };
  int i = 8 * threadIdx.x;
  for (; i + 8 * 256 * (IN_FLIGHT - 1) + 8 <= n; i += 8 * 256 * IN_FLIGHT) {
    Raw8<T> r[IN_FLIGHT];
#pragma unroll
    for (int u = 0; u < IN_FLIGHT; ++u) r[u].load(in + i + 8 * 256 * u);
#pragma unroll
    for (int u = 0; u < IN_FLIGHT; ++u) put(i + 8 * 256 * u, r[u]);
  }
  for (; i + 8 <= n; i += 8 * 256) {
    Raw8<T> r;
    r.load(in + i);
    put(i, r);
  }
  for (; i < n; ++i) from_f32(out[i], to_f32(in[i]) * step * factor);
}

// Segments are taken from the last to the first: the sums were taken the other way round, and what they read last the caches still hold. PAST: what is
// written goes past them, and does not drive out what is still to be read. From PAST_FROM segments (64 MB in, 64 MB out) on; below, whoever reads the
// clipped gradients next finds them there. Sums and clipping, bf16, cached / past: 302M values 350 / 321 us, 50M 61.5 / 52.5, 25M 31.8 / 31.8.
constexpr int64_t PAST_FROM = 2048;
template <bool PAST>
__global__ __launch_bounds__(256) void grad_clip_kernel(int64_t n, const GradSegment* __restrict__ segments, const double* __restrict__ sumsq, float max_norm,
                                                        float* __restrict__ norm_out) {
  const double norm = sqrt(*sumsq);
  if (norm_out && blockIdx.x == 0 && threadIdx.x == 0) *norm_out = (float)norm;
  const bool scaled = norm > (double)max_norm && norm < INFINITY;   // (a norm that is no number: the gradients stay as they are)
  // (in two factors, so that neither is below the normal 32-bit numbers where the norm is 2^100 times the bound)
  const double ratio = scaled ? (double)max_norm / norm : 1.0;
  const float step = ratio < 0x1p-100 ? 0x1p-64f : 1.f, factor = (float)(ratio / (double)step);
  for (int64_t i = n - 1 - blockIdx.x; i >= 0; i -= gridDim.x) {
    const GradSegment g = segments[i];
    if (!scaled && g.in == g.out) continue;
    if (g.dtype == DT_FP32) scale_segment<PAST>((const float*)g.in, (float*)g.out, g.count, factor, step);
    else if (g.dtype == DT_FP16) scale_segment<PAST>((const f16_t*)g.in, (f16_t*)g.out, g.count, factor, step);
    else scale_segment<PAST>((const bf16_t*)g.in, (bf16_t*)g.out, g.count, factor, step);
  }
}

unsigned grad_grid(int64_t segments, int most) { return (unsigned)(segments < 1 ? 1 : segments < most ? segments : most); }

}  // namespace

GradPlanLayout grad_plan_layout(int64_t segments) {
  GradPlanLayout L;
  L.segments = 256;   // (behind the counter)
  L.partials = (L.segments + (size_t)segments * sizeof(GradSegment) + 255) & ~(size_t)255;
  L.total = L.partials + SUM_BLOCKS * sizeof(double);
  return L;
}

void launch_grad_plan(int n, const GradArray* arrays, void* memory, hipStream_t st) {
  char* m = (char*)memory;
  for (int at = 0; at < n || at == 0; at += TABLE) {
    GradTable table = {};
    const int some = n - at < TABLE ? n - at : TABLE;
    for (int i = 0; i < some; ++i) table.a[i] = arrays[at + i];
    // (a plan without arrays: one block, which finds no elements and clears the counter)
    hipLaunchKernelGGL(grad_plan_kernel, dim3(some > 0 ? some : 1), dim3(256), 0, st, table, (GradSegment*)(m + grad_plan_layout(0).segments), (unsigned*)m, at == 0 ? 1 : 0);
  }
}

void launch_grad_sumsq(int64_t segments, void* memory, int accumulate, double* sumsq, hipStream_t st) {
  const GradPlanLayout L = grad_plan_layout(segments);
  char* m = (char*)memory;
  hipLaunchKernelGGL(grad_sumsq_kernel, dim3(grad_grid(segments, SUM_BLOCKS)), dim3(SUM_THREADS), 0, st, segments, (const GradSegment*)(m + L.segments),
                     (double*)(m + L.partials), (unsigned*)m, accumulate, sumsq);
}

void launch_grad_clip(int64_t segments, void* memory, const double* sumsq, float max_norm, float* norm, hipStream_t st) {
  const GradPlanLayout L = grad_plan_layout(segments);
  hipLaunchKernelGGL(segments >= PAST_FROM ? grad_clip_kernel<true> : grad_clip_kernel<false>, dim3(grad_grid(segments, 2048)), dim3(256), 0, st,
                     segments, (const GradSegment*)((char*)memory + L.segments), sumsq, max_norm, norm);
}

}  // namespace slapo
