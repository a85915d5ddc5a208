// Layer norm with its statistics, and its backward pass.
//
// A row's values stay in the registers of TPR threads between the passes over
// them, so each is read once.  Rows are walked by a fixed grid: gamma and beta
// stay in registers, and the next row's loads are in flight during this one's
// sums.  The backward pass adds each thread's columns of gamma's and beta's
// gradients in registers over its rows, a block's rows in LDS, and a second
// kernel the blocks, all in a fixed order, so results do not vary.
// Statistics, sums and gradients are float32; y and dx are rounded once.
//
// Bound by memory: x read and y written, backward x and dy read and dx written.
// 25,216 x 768 bf16: forward 14.8 us (5.2 TB/s; a copy of as many bytes 11.6), backward
// with both launches 30.1 us (3.9 TB/s); 8191 x 1111 float32 backward, rows with no
// alignment, 34.7 us (3.1 TB/s; 2.3 requests to the L2 for each 128 bytes, where aligned
// bf16 rows have 1.4); 197 x 768 is one launch's 6 us.
#include "tail.h"

namespace hapi {
namespace {

// 16 bytes of a row from an address with the element's alignment only (global
// loads of several dwords need no more on this hardware).
template <typename T>
struct Pack;
template <>
struct Pack<uint16_t> {
  static constexpr int N = 8;
  static __device__ __forceinline__ void unpack(const uint4 &q, float *v) {
    const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      v[2 * j] = __uint_as_float(w[j] << 16);
      v[2 * j + 1] = __uint_as_float(w[j] & 0xffff0000u);
    }
  }
  static __device__ __forceinline__ uint4 pack(const float *v) {
    return make_uint4(f2bf2(v[0], v[1]), f2bf2(v[2], v[3]), f2bf2(v[4], v[5]), f2bf2(v[6], v[7]));
  }
};
template <>
struct Pack<float> {
  static constexpr int N = 4;
  static __device__ __forceinline__ void unpack(const uint4 &q, float *v) {
    v[0] = __uint_as_float(q.x); v[1] = __uint_as_float(q.y);
    v[2] = __uint_as_float(q.z); v[3] = __uint_as_float(q.w);
  }
  static __device__ __forceinline__ uint4 pack(const float *v) {
    return make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]));
  }
};

// n: values of the chunk inside the row (<= 0: none); the rest is zero.
template <typename T>
__device__ __forceinline__ uint4 load_chunk(const T *p, int n) {
  constexpr int N = Pack<T>::N;
  uint4 q = make_uint4(0, 0, 0, 0);
  if (n >= N) {
    __builtin_memcpy(&q, p, 16);
  } else if (n > 0) {
    T v[N] = {};
#pragma unroll
    for (int j = 0; j < N; ++j)
      if (j < n) v[j] = p[j];
    __builtin_memcpy(&q, v, 16);
  }
  return q;
}
template <typename T>
__device__ __forceinline__ void store_chunk(T *p, int n, const uint4 &q) {
  constexpr int N = Pack<T>::N;
  if (n >= N) {
    __builtin_memcpy(p, &q, 16);
  } else if (n > 0) {
    T v[N];
    __builtin_memcpy(v, &q, 16);
#pragma unroll
    for (int j = 0; j < N; ++j)
      if (j < n) p[j] = v[j];
  }
}

// Sums of K values over the TPR threads of a row, known to all of them.  red:
// two alternating buffers, so one barrier a call is enough.
template <int TPR, int K>
__device__ __forceinline__ void row_sum(float (&v)[K], float (*red)[8][2], int &flip) {
#pragma unroll
  for (int o = (TPR < 64 ? TPR : 64) / 2; o >= 1; o >>= 1)
#pragma unroll
    for (int k = 0; k < K; ++k) v[k] += __shfl_xor(v[k], o, 64);
  if constexpr (TPR > 64) {
    constexpr int W = TPR / 64;
    if ((threadIdx.x & 63) == 0)
#pragma unroll
      for (int k = 0; k < K; ++k) red[flip][threadIdx.x >> 6][k] = v[k];
    __syncthreads();
#pragma unroll
    for (int k = 0; k < K; ++k) {
      float t = 0.0f;
#pragma unroll
      for (int w = 0; w < W; ++w) t += red[flip][w][k];
      v[k] = t;
    }
    flip ^= 1;
  }
}

constexpr int block_of(int tpr) { return tpr < 256 ? 256 : tpr; }

// N float32 weights from d on, zero past dim.
template <int N>
__device__ __forceinline__ void load_weights(const float *p, int d, int dim, float (&v)[N]) {
  if (d + N <= dim) {
    __builtin_memcpy(v, p + d, 4 * N);
  } else {
#pragma unroll
    for (int j = 0; j < N; ++j) v[j] = d + j < dim ? p[d + j] : 0.0f;
  }
}

template <typename T, int TPR, int CH>
__global__ __launch_bounds__(block_of(TPR)) void norm_forward_kernel(NormArgs a) {
  constexpr int N = Pack<T>::N, RPB = block_of(TPR) / TPR;
  __shared__ float red[2][8][2];
  int flip = 0;
  const int tl = threadIdx.x % TPR, D = a.dim;
  const float inv_d = 1.0f / (float)D;
  const int64_t step = (int64_t)gridDim.x * RPB;
  int64_t row = (int64_t)blockIdx.x * RPB + threadIdx.x / TPR;
  const T *x = static_cast<const T *>(a.x);
  T *y = static_cast<T *>(a.y);
  uint4 nx[CH];
  auto load = [&](int64_t r) {
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      const int d = (tl + TPR * c) * N;
      nx[c] = load_chunk<T>(x + r * a.x_ld + d, r < a.rows ? D - d : 0);
    }
  };
  load(row);
  float g[CH][N], b[CH][N];
#pragma unroll
  for (int c = 0; c < CH; ++c) {
    load_weights<N>(a.gamma, (tl + TPR * c) * N, D, g[c]);
    load_weights<N>(a.beta, (tl + TPR * c) * N, D, b[c]);
  }
  // every thread of a block walks as many rows: the barriers in row_sum
  for (int64_t r0 = (int64_t)blockIdx.x * RPB; r0 < a.rows; r0 += step, row += step) {
    float v[CH][N];
    float s[1] = {0.0f};
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      Pack<T>::unpack(nx[c], v[c]);
#pragma unroll
      for (int j = 0; j < N; ++j) s[0] += v[c][j];
    }
    if (r0 + step < a.rows) load(row + step);
    row_sum<TPR>(s, red, flip);
    const float mean = s[0] * inv_d;
    float var[1] = {0.0f};
#pragma unroll
    for (int c = 0; c < CH; ++c)
#pragma unroll
      for (int j = 0; j < N; ++j) {
        v[c][j] -= mean;
        if ((tl + TPR * c) * N + j < D) var[0] = fmaf(v[c][j], v[c][j], var[0]);
      }
    row_sum<TPR>(var, red, flip);
    const float rstd = 1.0f / sqrtf(fmaf(var[0], inv_d, a.eps));
    if (row < a.rows) {
#pragma unroll
      for (int c = 0; c < CH; ++c) {
        const int d = (tl + TPR * c) * N;
        float o[N];
#pragma unroll
        for (int j = 0; j < N; ++j) o[j] = fmaf(v[c][j] * rstd, g[c][j], b[c][j]);
        store_chunk<T>(y + row * a.y_ld + d, D - d, Pack<T>::pack(o));
      }
      if (tl == 0) {
        a.mean[row] = mean;
        a.rstd[row] = rstd;
      }
    }
  }
}

template <typename T, int TPR, int CH>
__global__ __launch_bounds__(block_of(TPR)) void norm_backward_kernel(NormArgs a) {
  constexpr int N = Pack<T>::N, RPB = block_of(TPR) / TPR;
  __shared__ float red[2][8][2];
  __shared__ float acc_s[RPB > 1 ? 2 * TPR * CH * N : 1];
  int flip = 0;
  const int tl = threadIdx.x % TPR, D = a.dim;
  const float inv_d = 1.0f / (float)D;
  float g[CH][N], dg[CH][N], db[CH][N];
#pragma unroll
  for (int c = 0; c < CH; ++c) {
    load_weights<N>(a.gamma, (tl + TPR * c) * N, D, g[c]);
#pragma unroll
    for (int j = 0; j < N; ++j) dg[c][j] = db[c][j] = 0.0f;
  }
  const int64_t step = (int64_t)gridDim.x * RPB;
  int64_t row = (int64_t)blockIdx.x * RPB + threadIdx.x / TPR;
  const T *x = static_cast<const T *>(a.x), *dy = static_cast<const T *>(a.dy);
  T *dx = static_cast<T *>(a.dx);
  uint4 nx[CH], ny[CH];
  float mean = 0.0f, rstd = 0.0f;
  auto load = [&](int64_t r) {
    const bool live = r < a.rows;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      const int d = (tl + TPR * c) * N;
      nx[c] = load_chunk<T>(x + r * a.x_ld + d, live ? D - d : 0);
      ny[c] = load_chunk<T>(dy + r * a.y_ld + d, live ? D - d : 0);
    }
    mean = live ? a.mean[r] : 0.0f;
    rstd = live ? a.rstd[r] : 0.0f;
  };
  // the next row's loads in flight during this one's sums, where the registers hold both
  constexpr bool kAhead = TPR < 512;
  if (kAhead) load(row);
  for (int64_t r0 = (int64_t)blockIdx.x * RPB; r0 < a.rows; r0 += step, row += step) {
    if (!kAhead) load(row);
    // past the row's end x and dy are 0 and gamma is 0: h is -mean rstd there,
    // and every product with it is 0
    float h[CH][N], u[CH][N];
    float s[2] = {0.0f, 0.0f};
    const float rs = rstd;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      Pack<T>::unpack(nx[c], h[c]);
      Pack<T>::unpack(ny[c], u[c]);
#pragma unroll
      for (int j = 0; j < N; ++j) {
        h[c][j] = (h[c][j] - mean) * rs;
        dg[c][j] = fmaf(u[c][j], h[c][j], dg[c][j]);
        db[c][j] += u[c][j];
        u[c][j] *= g[c][j];
        s[0] += u[c][j];
        s[1] = fmaf(u[c][j], h[c][j], s[1]);
      }
    }
    if (kAhead) load(row + step);
    row_sum<TPR>(s, red, flip);
    const float m0 = s[0] * inv_d, m1 = s[1] * inv_d;
    if (row < a.rows) {
#pragma unroll
      for (int c = 0; c < CH; ++c) {
        const int d = (tl + TPR * c) * N;
        float o[N];
#pragma unroll
        for (int j = 0; j < N; ++j) o[j] = rs * (u[c][j] - fmaf(h[c][j], m1, m0));
        store_chunk<T>(dx + row * a.x_ld + d, D - d, Pack<T>::pack(o));
      }
    }
  }
  float *out = a.part + (int64_t)blockIdx.x * 2 * D;
  if constexpr (RPB > 1) {
    constexpr int W = TPR * CH * N;
    for (int r = 0; r < RPB; ++r) {
      if ((int)threadIdx.x / TPR == r) {
#pragma unroll
        for (int c = 0; c < CH; ++c)
#pragma unroll
          for (int j = 0; j < N; ++j) {
            const int d = (tl + TPR * c) * N + j;
            acc_s[d] = (r ? acc_s[d] : 0.0f) + dg[c][j];
            acc_s[W + d] = (r ? acc_s[W + d] : 0.0f) + db[c][j];
          }
      }
      __syncthreads();
    }
    for (int d = threadIdx.x; d < D; d += block_of(TPR)) {
      out[d] = acc_s[d];
      out[D + d] = acc_s[W + d];
    }
  } else {
#pragma unroll
    for (int c = 0; c < CH; ++c)
#pragma unroll
      for (int j = 0; j < N; ++j) {
        const int d = (tl + TPR * c) * N + j;
        if (d < D) {
          out[d] = dg[c][j];
          out[D + d] = db[c][j];
        }
      }
  }
}

// dgamma and dbeta: the sum of the blocks' partial sums, 16 columns a block and 64
// slices of the parts side by side, then the slices in order.
__global__ __launch_bounds__(1024) void norm_reduce_kernel(const float *__restrict__ part, int parts, int D,
                                                           float *__restrict__ dgamma, float *__restrict__ dbeta) {
  __shared__ float red[64][17];
  const int col = threadIdx.x & 15, slice = threadIdx.x >> 4;
  const int c = blockIdx.x * 16 + col;
  float t = 0.0f;
  if (c < 2 * D) {
#pragma unroll
    for (int i = 0; i < kNormParts / 64; ++i) {
      const int p = slice + 64 * i;
      t += p < parts ? part[(int64_t)p * 2 * D + c] : 0.0f;
    }
  }
  red[slice][col] = t;
  __syncthreads();
  if (slice == 0 && c < 2 * D) {
    t = 0.0f;
#pragma unroll
    for (int i = 0; i < 64; ++i) t += red[i][col];
    (c < D ? dgamma[c] : dbeta[c - D]) = t;
  }
}

template <typename T, int TPR, int CH, bool BACK>
hipError_t launch_one(const NormArgs &a, hipStream_t s) {
  constexpr int RPB = block_of(TPR) / TPR;
  const int64_t want = (a.rows + RPB - 1) / RPB;
  if constexpr (BACK) {
    // two blocks a CU, as many rows to each
    const int64_t iters = (want + kNormParts - 1) / kNormParts;
    const int blocks = want > 0 ? (int)((want + iters - 1) / iters) : 0;
    if (blocks > 0) hapi_launch((norm_backward_kernel<T, TPR, CH>), dim3(blocks), dim3(block_of(TPR)), 0, s, a);
    hapi_launch(norm_reduce_kernel, dim3((2 * a.dim + 15) / 16), dim3(1024), 0, s, (const float *)a.part, blocks, a.dim,
                a.dgamma, a.dbeta);
  } else {
    const int64_t blocks = norm_forward_blocks(want, block_of(TPR));
    if (blocks > 0) hapi_launch((norm_forward_kernel<T, TPR, CH>), dim3((uint32_t)blocks), dim3(block_of(TPR)), 0, s, a);
  }
  return hipGetLastError();
}

// The threads a row gets: as few as hold it in 32 values each (one pass over the
// registers), and of the shapes that hold it the one with the fewest idle lanes.
template <typename T, bool BACK>
hipError_t launch_dim(const NormArgs &a, hipStream_t s) {
  constexpr int N = Pack<T>::N;
  const int ch = (a.dim + N - 1) / N;  // 16-byte chunks of a row
  if (ch <= 16 * 1) return launch_one<T, 16, 1, BACK>(a, s);
  if (ch <= 32 * 1) return launch_one<T, 32, 1, BACK>(a, s);
  if (ch <= 32 * 2) return launch_one<T, 32, 2, BACK>(a, s);
  if (ch <= 32 * 3) return launch_one<T, 32, 3, BACK>(a, s);
  if (ch <= 32 * 4) return launch_one<T, 32, 4, BACK>(a, s);
  if (ch <= 64 * 3) return launch_one<T, 64, 3, BACK>(a, s);
  if (ch <= 64 * 4) return launch_one<T, 64, 4, BACK>(a, s);
  if constexpr (sizeof(T) == 4) {
    if (ch <= 64 * 5) return launch_one<T, 64, 5, BACK>(a, s);
    if (ch <= 64 * 6) return launch_one<T, 64, 6, BACK>(a, s);
    if (ch <= 64 * 8) return launch_one<T, 64, 8, BACK>(a, s);
  } else {
    if (ch <= 256 * 2) return launch_one<T, 256, 2, BACK>(a, s);
  }
  if (ch <= 256 * 3) return launch_one<T, 256, 3, BACK>(a, s);
  if (ch <= 256 * 4) return launch_one<T, 256, 4, BACK>(a, s);
  if constexpr (sizeof(T) == 4) {
    if (ch <= 256 * 6) return launch_one<T, 256, 6, BACK>(a, s);
  }
  if (ch <= 512 * 4) return launch_one<T, 512, 4, BACK>(a, s);
  if constexpr (sizeof(T) == 4) {
    if (ch <= 512 * 6) return launch_one<T, 512, 6, BACK>(a, s);
    if (ch <= 512 * 8) return launch_one<T, 512, 8, BACK>(a, s);
  }
  return hipErrorInvalidValue;
}

}  // namespace

hipError_t launch_norm_forward(bool bf16, const NormArgs &a, hipStream_t s) {
  return bf16 ? launch_dim<uint16_t, false>(a, s) : launch_dim<float, false>(a, s);
}
hipError_t launch_norm_backward(bool bf16, const NormArgs &a, hipStream_t s) {
  return bf16 ? launch_dim<uint16_t, true>(a, s) : launch_dim<float, true>(a, s);
}

}  // namespace hapi
