// The global norm of many gradients, and their clipping.
//
// A launch takes up to kGradTensors tensors, whose addresses and sizes are its
// arguments: no table has to be brought to the device first.  The tensors are cut
// into segments; a block walks the segments in a stride of the grid and leaves one
// sum of squares.  Squares and sums are float64 (a float32 square is exact in it and
// cannot overflow), so neither the largest values nor the count cost accuracy; the
// blocks' sums are joined in a fixed order.  The clipping blocks join the sums
// themselves, each all of them, which saves a launch between the two passes.
//
// Bound by memory: the norm reads every value once, clipping reads it again and
// writes it.  871 million float32 values: 0.57 ms, 6.1 TB/s (reads alone pass the rate of a
// copy); 118 million bf16 and float32 ones clipped in 173 us, 4.1 TB/s of all three passes;
// 2 million: 4.0 + 6.8 us, of which a launch and its search are some 3 each.
#include "block.h"

namespace hapi {
namespace {

constexpr int kThreads = 256;

// Sum of v over the block, known to all its threads, in a fixed order.
__device__ __forceinline__ double block_sum(double v) {
  __shared__ double red[kThreads / 64];
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) v += __shfl_xor(v, o, 64);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  return (red[0] + red[1]) + (red[2] + red[3]);
}

__device__ __forceinline__ double sum_parts(const double *part, int64_t parts) {
  double s = 0.0;
  for (int64_t i = threadIdx.x; i < parts; i += kThreads) s += part[i];
  return block_sum(s);
}

template <typename T>
struct Vec;
template <>
struct Vec<uint16_t> {
  static constexpr int N = 8;
  static __device__ __forceinline__ float get(uint16_t v) { return __uint_as_float((uint32_t)v << 16); }
  static __device__ __forceinline__ uint16_t put(float v) { return f2bf(v); }
};
template <>
struct Vec<float> {
  static constexpr int N = 4;
  static __device__ __forceinline__ float get(float v) { return v; }
  static __device__ __forceinline__ float put(float v) { return v; }
};

// A tensor's segment [from, to), 4 x 16 bytes of each thread in flight; the tensors
// need only their elements' alignment (loads and stores of 16 bytes need no more here).
template <typename T, typename F>
__device__ __forceinline__ void walk(const T *in, int64_t from, int64_t to, F &&f) {
  constexpr int N = Vec<T>::N, U = 4;
  constexpr int STEP = kThreads * N;
  int64_t at = from + threadIdx.x * N;
  // whole steps of the block without a question
  for (const int64_t whole = to - U * STEP; at - threadIdx.x * N <= whole; at += U * STEP) {
    T v[U][N];
#pragma unroll
    for (int u = 0; u < U; ++u) __builtin_memcpy(v[u], in + at + u * STEP, 16);
#pragma unroll
    for (int u = 0; u < U; ++u) f(at + u * STEP, v[u]);
  }
  for (; at < to; at += STEP) {
    T v[N];
    if (at + N <= to) {
      __builtin_memcpy(v, in + at, 16);
    } else {
#pragma unroll
      for (int j = 0; j < N; ++j) v[j] = at + j < to ? in[at + j] : T{};
    }
    f(at, v);
  }
}

// Calls f(in, out, is float32, first value, end) for each of this block's segments.  The
// tensors' entries stay in the lanes of each wave (two to a lane), so that finding a
// segment's tensor is a comparison and a count, with no chain of loads.
template <bool OUT, typename F>
__device__ __forceinline__ void segments(const GradArgs &a, F &&f) {
  static_assert(kGradTensors <= 128, "two entries to a lane");
  const int lane = threadIdx.x & 63, total = a.seg[a.count];
  int first[2];
  uint64_t in[2], out[2], size[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int t = lane + 64 * i;
    const bool there = t < a.count;
    first[i] = there ? a.seg[t] : INT32_MAX;
    in[i] = there ? (uint64_t)(uintptr_t)a.in[t] : 0;
    out[i] = there && OUT ? (uint64_t)(uintptr_t)a.out[t] : 0;
    size[i] = there ? (uint64_t)a.size[t] : 0;
  }
  auto of = [](const uint64_t (&v)[2], int t) {
    const uint64_t x = t < 64 ? v[0] : v[1];
    const uint32_t lo = __builtin_amdgcn_readlane((uint32_t)x, t & 63), hi = __builtin_amdgcn_readlane((uint32_t)(x >> 32), t & 63);
    return (uint64_t)hi << 32 | lo;
  };
  for (int s = blockIdx.x; s < total; s += gridDim.x) {
    // the last tensor whose first segment is <= s
    const int t = __popcll(__ballot(first[0] <= s)) + __popcll(__ballot(first[1] <= s)) - 1;
    const int start = t < 64 ? __builtin_amdgcn_readlane(first[0], t & 63) : __builtin_amdgcn_readlane(first[1], t & 63);
    const int64_t n = (int64_t)of(size, t), from = (int64_t)(s - start) * a.seg_size;
    const int64_t to = from + a.seg_size < n ? from + a.seg_size : n;
    f((const void *)(uintptr_t)of(in, t), (void *)(uintptr_t)of(out, t), (bool)(a.f32[t >> 5] >> (t & 31) & 1), from, to);
  }
}

__global__ __launch_bounds__(kThreads) void grad_squares_kernel(GradArgs a) {
  double sum = 0.0;
  segments<false>(a, [&](const void *in, void *, bool f32, int64_t from, int64_t to) {
    auto add = [&](auto *p) {
      typedef std::remove_const_t<std::remove_pointer_t<decltype(p)>> T;
      walk(p, from, to, [&](int64_t, const T *v) {
#pragma unroll
        for (int j = 0; j < Vec<T>::N; ++j) {
          const double d = (double)Vec<T>::get(v[j]);
          sum = fma(d, d, sum);
        }
      });
    };
    if (f32) add(static_cast<const float *>(in));
    else add(static_cast<const uint16_t *>(in));
  });
  sum = block_sum(sum);
  if (threadIdx.x == 0) a.part[blockIdx.x] = sum;
}

__global__ __launch_bounds__(kThreads) void grad_clip_kernel(GradArgs a) {
  const double norm = sqrt(sum_parts(a.part, a.parts));
  if (a.norm && blockIdx.x == 0 && threadIdx.x == 0) *a.norm = (float)norm;
  // a norm that is not finite is the caller's to see: it changes no gradient
  const double factor = norm > a.max_norm && norm < INFINITY ? a.max_norm / norm : 1.0;
  segments<true>(a, [&](const void *in, void *out, bool f32, int64_t from, int64_t to) {
    if (factor == 1.0 && in == out) return;
    auto scale = [&](auto *p, auto *o) {
      typedef std::remove_pointer_t<decltype(o)> T;
      constexpr int N = Vec<T>::N;
      walk(p, from, to, [&](int64_t i, const T *v) {
        T r[N];
#pragma unroll
        for (int j = 0; j < N; ++j) r[j] = factor == 1.0 ? v[j] : Vec<T>::put((float)((double)Vec<T>::get(v[j]) * factor));
        if (i + N <= to) {
          __builtin_memcpy(o + i, r, 16);
        } else {
#pragma unroll
          for (int j = 0; j < N; ++j)
            if (i + j < to) o[i + j] = r[j];
        }
      });
    };
    if (f32) scale(static_cast<const float *>(in), static_cast<float *>(out));
    else scale(static_cast<const uint16_t *>(in), static_cast<uint16_t *>(out));
  });
}

// Block b sums part[b], part[b + blocks], ...
__global__ __launch_bounds__(kThreads) void grad_join_kernel(const double *part, int64_t parts, double *out) {
  double s = 0.0;
  for (int64_t i = blockIdx.x + (int64_t)threadIdx.x * gridDim.x; i < parts; i += (int64_t)kThreads * gridDim.x) s += part[i];
  s = block_sum(s);
  if (threadIdx.x == 0) out[blockIdx.x] = s;
}

__global__ __launch_bounds__(kThreads) void grad_norm_kernel(const double *part, int64_t parts, float *norm) {
  const double s = sum_parts(part, parts);
  if (threadIdx.x == 0) *norm = (float)sqrt(s);
}

}  // namespace

hipError_t launch_grad_squares(const GradArgs &a, int blocks, hipStream_t s) {
  hapi_launch(grad_squares_kernel, dim3(blocks), dim3(kThreads), 0, s, a);
  return hipGetLastError();
}
hipError_t launch_grad_clip(const GradArgs &a, int blocks, hipStream_t s) {
  hapi_launch(grad_clip_kernel, dim3(blocks), dim3(kThreads), 0, s, a);
  return hipGetLastError();
}
hipError_t launch_grad_join(const double *part, int64_t parts, double *out, hipStream_t s) {
  hapi_launch(grad_join_kernel, dim3((uint32_t)(parts < kGradBlocks ? parts : kGradBlocks)), dim3(kThreads), 0, s, part, parts, out);
  return hipGetLastError();
}
hipError_t launch_grad_norm(const double *part, int64_t parts, float *norm, hipStream_t s) {
  hapi_launch(grad_norm_kernel, dim3(1), dim3(kThreads), 0, s, part, parts, norm);
  return hipGetLastError();
}

}  // namespace hapi
