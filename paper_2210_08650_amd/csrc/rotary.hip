// Rotary positions on several axes, with the heads' RMS norm in the same pass,
// forward and backward.
//
// A vector (one head of one token) belongs to LV lanes of a wave, a lane to V pairs of
// it: V values of either side of the pairs, 16 bytes each where the widths divide into them
// and the call is large enough (strides and addresses need their elements' alignment only);
// what is not rotated goes as pairs that do not turn.  A lane keeps its pairs over the heads
// of a token, so that angles, sines and cosines are formed once for all of them; q and k go
// to blocks of their own, each with one gamma.
// The angle is position times frequency in float64, reduced to a part of a turn there:
// in float32 its rounding at position 1e6 would be 0.03 radians.  Norm, rotation and sums
// are float32, outputs are rounded once.
//
// Backward turns dy by the opposite angle and goes back through the norm, whose
// 1 / sqrt it forms again from x.  A lane sums its columns of the gammas' gradients
// over its vectors, a block its lanes in LDS and a second kernel the blocks, in a
// fixed order.
//
// Bound by memory: x read and y written, backward x and dy read and dx written.  128 x
// 197 tokens, 12 + 12 heads of 64 in bf16: forward 32.2 us, 4.8 TB/s; backward 50 us, 4.6
// TB/s, and 4.7 for the blocks' sums.  1 x 197 tokens: 4.4 us, a launch and one lane's
// angles.
#include "block.h"

namespace hapi {
namespace {

constexpr int kThreads = 256;

// V values of a row as they lie in memory; zeros where there are none.
template <typename T, int V>
struct Raw {
  T v[V];
  __device__ __forceinline__ void load(const T *p, bool there) {
    // one load of all of them, the element's alignment is enough for it on this hardware
#pragma unroll
    for (int j = 0; j < V; ++j) v[j] = T{};
    if (there) __builtin_memcpy(v, p, V * sizeof(T));
  }
  __device__ __forceinline__ void widen(float *f) const {
#pragma unroll
    for (int j = 0; j < V; ++j) {
      if constexpr (sizeof(T) == 2) f[j] = __uint_as_float((uint32_t)v[j] << 16);
      else f[j] = v[j];
    }
  }
};
template <typename T, int V>
__device__ __forceinline__ void store(T *p, bool there, const float *f) {
  if (!there) return;
  T v[V];
  if constexpr (sizeof(T) == 2) {
    if constexpr (V == 1) {
      v[0] = f2bf(f[0]);
    } else {
#pragma unroll
      for (int j = 0; j < V; j += 2) {
        const uint32_t w = f2bf2(f[j], f[j + 1]);
        __builtin_memcpy(v + j, &w, 4);
      }
    }
  } else {
#pragma unroll
    for (int j = 0; j < V; ++j) v[j] = f[j];
  }
  __builtin_memcpy(p, v, V * sizeof(T));
}

// LV lanes of a vector, NU units (V pairs each) of a lane.  blockIdx.y: q or k, where both
// are there.
template <typename T, int V, int LV, int NU, bool NEIGHBOURS, bool BACK>
__global__ __launch_bounds__(kThreads) void rotary_kernel(RotaryArgs a) {
  constexpr int GPB = kThreads / LV;
  __shared__ float acc_s[BACK ? kThreads * 2 * V * NU : 1];
  const int w = a.heads[0] > 0 ? blockIdx.y : 1;
  const int lane = threadIdx.x % LV;
  const int D = a.dim, P = a.pairs, heads = a.heads[w], groups = a.head_groups[w];
  // where this lane's units lie
  int ea[NU], eb[NU];
  uint32_t axis[NU];  // four bits for each pair; kRotaryAxes: not rotated
  float gamma[NU][2 * V];
#pragma unroll
  for (int n = 0; n < NU; ++n) {
    const int u = lane + n * LV;
    const bool halves = u * V < P && !NEIGHBOURS;
    ea[n] = halves ? u * V : 2 * u * V;
    eb[n] = halves ? P + u * V : 2 * u * V + V;
    axis[n] = 0;
#pragma unroll
    for (int j = 0; j < V; ++j) {
      const int i = u * V + j;
      uint32_t x = i < P ? 0 : kRotaryAxes;
#pragma unroll
      for (int k = 1; k < kRotaryAxes; ++k)
        if (i < P && k < a.axes && i >= a.first[k]) x = k;
      axis[n] |= x << (4 * j);
    }
#pragma unroll
    for (int j = 0; j < 2 * V; ++j) {
      const int e = j < V ? ea[n] + j : eb[n] + j - V;
      gamma[n][j] = a.norm && e < D ? a.gamma[w][e] : 1.0f;
    }
  }
  float dg[NU][2 * V];
#pragma unroll
  for (int n = 0; n < NU; ++n)
#pragma unroll
    for (int j = 0; j < 2 * V; ++j) dg[n][j] = 0.0f;

  const uint32_t total = (uint32_t)(a.tokens * groups);  // < 2^31
  for (uint32_t g = blockIdx.x * GPB + threadIdx.x / LV; g < total; g += gridDim.x * GPB) {
    const uint32_t token = g / (uint32_t)groups;
    const int first_head = (int)(g - token * groups);
    const uint32_t b = token / (uint32_t)a.len, l = token - b * a.len;
    const bool counts = !a.lens || (int64_t)l < a.lens[b];
    const int64_t x0 = (int64_t)b * a.x_st[w][0] + (int64_t)l * a.x_st[w][1];
    const int64_t y0 = (int64_t)b * a.y_st[w][0] + (int64_t)l * a.y_st[w][1];
    const T *xp = static_cast<const T *>(a.x[w]) + x0, *dyp = static_cast<const T *>(a.dy[w]) + y0;
    T *out = static_cast<T *>(a.y[w]) + (BACK ? x0 : y0);
    const int64_t x_step = a.x_st[w][2], y_step = a.y_st[w][2], out_step = BACK ? x_step : y_step;
    // a head's values as they lie in memory, the next one's on their way during this one's
    // arithmetic; backward: dy and x
    Raw<T, V> src[NU][2], xs[BACK ? NU : 1][2];
    auto fetch = [&](int h) {
#pragma unroll
      for (int n = 0; n < NU; ++n) {
        const bool there = counts && h < heads && ea[n] < D, second = there && eb[n] < D;
        const T *p = BACK ? dyp + h * y_step : xp + h * x_step;
        src[n][0].load(p + ea[n], there);
        src[n][1].load(p + eb[n], second);
        if constexpr (BACK) {
          const T *q = xp + h * x_step;
          xs[n][0].load(q + ea[n], there && a.norm);
          xs[n][1].load(q + eb[n], second && a.norm);
        }
      }
    };
    fetch(first_head);
    double pos[kRotaryAxes];
#pragma unroll
    for (int x = 0; x < kRotaryAxes; ++x) pos[x] = x < a.axes && counts ? (double)a.positions[x * a.tokens + token] : 0.0;
    float cs[NU][V], sn[NU][V];
#pragma unroll
    for (int n = 0; n < NU; ++n)
#pragma unroll
      for (int j = 0; j < V; ++j) {
        double p = 0.0;
#pragma unroll
        for (int x = 0; x < kRotaryAxes; ++x) p = ((axis[n] >> (4 * j)) & 15) == x ? pos[x] : p;
        const int i = (lane + n * LV) * V + j;
        const double freq = i < P ? a.freq[i] : 0.0;  // read again for each token: 16 registers fewer for the heads' values
        // part of a turn, in [-1/2, 1/2]
        double turn = p * freq * 0.15915494309189535;
        turn -= rint(turn);
        sincospif(2.0f * (float)turn, &sn[n][j], &cs[n][j]);
        if (BACK) sn[n][j] = -sn[n][j];
      }
    for (int h = first_head; h < heads; h += groups) {
      float v[NU][2 * V], x[BACK ? NU : 1][2 * V];
#pragma unroll
      for (int n = 0; n < NU; ++n) {
        src[n][0].widen(v[n]);
        src[n][1].widen(v[n] + V);
        if constexpr (BACK) {
          xs[n][0].widen(x[n]);
          xs[n][1].widen(x[n] + V);
        }
      }
      fetch(h + groups);
      auto rotate = [&](int n) {
#pragma unroll
        for (int j = 0; j < V; ++j) {
          float &p = NEIGHBOURS ? v[n][2 * j] : v[n][j];
          float &q = NEIGHBOURS ? v[n][2 * j + 1] : v[n][V + j];
          const float p0 = p, q0 = q;
          // what is not rotated stays as it is: 0 times its neighbour may be 0 times infinity
          const bool turns = (lane + n * LV) * V + j < P;
          p = turns ? p0 * cs[n][j] - q0 * sn[n][j] : p0;
          q = turns ? q0 * cs[n][j] + p0 * sn[n][j] : q0;
        }
      };
      if constexpr (!BACK) {
        if (a.norm) {
          float ss = 0.0f;
#pragma unroll
          for (int n = 0; n < NU; ++n)
#pragma unroll
            for (int j = 0; j < 2 * V; ++j) ss = fmaf(v[n][j], v[n][j], ss);
#pragma unroll
          for (int o = LV / 2; o >= 1; o >>= 1) ss += __shfl_xor(ss, o, 64);
          const float r = 1.0f / sqrtf(fmaf(ss, a.inv_dim, a.eps));
#pragma unroll
          for (int n = 0; n < NU; ++n)
#pragma unroll
            for (int j = 0; j < 2 * V; ++j) v[n][j] = counts ? v[n][j] * r * gamma[n][j] : 0.0f;
        }
#pragma unroll
        for (int n = 0; n < NU; ++n) rotate(n);
      } else {
#pragma unroll
        for (int n = 0; n < NU; ++n) rotate(n);
        if (a.norm) {
          float ss = 0.0f, ex = 0.0f;
#pragma unroll
          for (int n = 0; n < NU; ++n)
#pragma unroll
            for (int j = 0; j < 2 * V; ++j) {
              ss = fmaf(x[n][j], x[n][j], ss);
              ex = fmaf(v[n][j] * gamma[n][j], x[n][j], ex);
            }
#pragma unroll
          for (int o = LV / 2; o >= 1; o >>= 1) {
            ss += __shfl_xor(ss, o, 64);
            ex += __shfl_xor(ex, o, 64);
          }
          const float r = 1.0f / sqrtf(fmaf(ss, a.inv_dim, a.eps));
          const float c = ex * r * a.inv_dim;  // mean of e h
#pragma unroll
          for (int n = 0; n < NU; ++n)
#pragma unroll
            for (int j = 0; j < 2 * V; ++j) {
              const float hx = x[n][j] * r, u = v[n][j];
              if (counts) dg[n][j] = fmaf(u, hx, dg[n][j]);
              v[n][j] = counts ? r * (u * gamma[n][j] - hx * c) : 0.0f;
            }
        }
      }
      T *dst = out + h * out_step;
#pragma unroll
      for (int n = 0; n < NU; ++n) {
        store<T, V>(dst + ea[n], ea[n] < D, v[n]);
        store<T, V>(dst + eb[n], eb[n] < D, v[n] + V);
      }
    }
  }
  if constexpr (BACK) {
    if (!a.norm) return;
    // a column's sum over the block's groups of lanes
#pragma unroll
    for (int n = 0; n < NU; ++n)
#pragma unroll
      for (int j = 0; j < 2 * V; ++j) acc_s[(n * 2 * V + j) * kThreads + threadIdx.x] = dg[n][j];
    __syncthreads();
    for (int i = threadIdx.x; i < LV * NU * 2 * V; i += kThreads) {
      const int ln = i % LV, k = i / LV, n = k / (2 * V), j = k % (2 * V);
      const int u = ln + n * LV;
      const bool halves = u * V < P && !NEIGHBOURS;
      const int e = j < V ? (halves ? u * V : 2 * u * V) + j : (halves ? P + u * V : 2 * u * V + V) + j - V;
      if (e >= D) continue;
      float s = 0.0f;
      for (int q = 0; q < GPB; ++q) s += acc_s[k * kThreads + q * LV + ln];
      a.part[((int64_t)w * gridDim.x + blockIdx.x) * D + e] = s;
    }
  }
}

// dgamma of q and of k: 16 columns a block, the parts over 64 threads each.
__global__ __launch_bounds__(1024) void rotary_reduce_kernel(RotaryArgs a, int parts) {
  __shared__ double s[64][17];
  const int c = threadIdx.x & 15, slice = threadIdx.x >> 4;
  const int e = blockIdx.x * 16 + c, w = blockIdx.y;
  if (a.heads[w] == 0) return;
  double t = 0.0;
  if (e < a.dim) {
#pragma unroll 8
    for (int p = slice; p < parts; p += 64) t += (double)a.part[((int64_t)w * parts + p) * a.dim + e];
  }
  s[slice][c] = t;
  __syncthreads();
  if (slice == 0 && e < a.dim) {
    t = 0.0;
#pragma unroll
    for (int i = 0; i < 64; ++i) t += s[i][c];
    a.dgamma[w][e] = (float)t;
  }
}

template <typename T, int V, int LV, int NU>
hipError_t run(const RotaryArgs &a, bool back, hipStream_t s) {
  constexpr int gpb = kThreads / LV;
  const int64_t groups = a.head_groups[0] > a.head_groups[1] ? a.head_groups[0] : a.head_groups[1];
  const int64_t want = ceil_div(a.tokens * groups, gpb);
  const int64_t most = back && a.norm ? kRotaryParts : kMaxLaunchThreads / kThreads / 2;
  const dim3 grid((uint32_t)(want < most ? want : most), a.heads[0] > 0 && a.heads[1] > 0 ? 2 : 1), block(kThreads);
  const dim3 columns((a.dim + 15) / 16, 2);
  if (want == 0) {  // no tokens: the gammas' gradients are sums of nothing
    hapi_launch(rotary_reduce_kernel, columns, dim3(1024), 0, s, a, 0);
    return hipGetLastError();
  }
  if (a.neighbours) {
    if (back) hapi_launch(rotary_kernel<T, V, LV, NU, true, true>, grid, block, 0, s, a);
    else hapi_launch(rotary_kernel<T, V, LV, NU, true, false>, grid, block, 0, s, a);
  } else {
    if (back) hapi_launch(rotary_kernel<T, V, LV, NU, false, true>, grid, block, 0, s, a);
    else hapi_launch(rotary_kernel<T, V, LV, NU, false, false>, grid, block, 0, s, a);
  }
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || !back || !a.norm) return e;
  hapi_launch(rotary_reduce_kernel, columns, dim3(1024), 0, s, a, (int)grid.x);
  return hipGetLastError();
}

template <typename T, int V>
hipError_t pick(const RotaryArgs &a, bool back, hipStream_t s) {
  const int units = (a.dim + 2 * V - 1) / (2 * V);
  if (units <= 4) return run<T, V, 4, 1>(a, back, s);
  if (units <= 8) return run<T, V, 8, 1>(a, back, s);
  if constexpr (2 * V * 8 < kRotaryMaxDim) {
    if (units <= 16) return run<T, V, 16, 1>(a, back, s);
  }
  if constexpr (2 * V * 16 < kRotaryMaxDim) {
    if (units <= 32) return run<T, V, 32, 1>(a, back, s);
  }
  if constexpr (2 * V * 32 < kRotaryMaxDim) {
    if (units <= 64) return run<T, V, 64, 1>(a, back, s);
  }
  if constexpr (2 * V * 64 < kRotaryMaxDim) return run<T, V, 64, 2>(a, back, s);
  return hipErrorInvalidValue;
}

hipError_t launch(bool bf16, int v, const RotaryArgs &a, bool back, hipStream_t s) {
  if (bf16) {
    switch (v) {
      case 8: return pick<uint16_t, 8>(a, back, s);
      case 4: return pick<uint16_t, 4>(a, back, s);
      case 2: return pick<uint16_t, 2>(a, back, s);
      default: return pick<uint16_t, 1>(a, back, s);
    }
  }
  switch (v) {
    case 4: return pick<float, 4>(a, back, s);
    case 2: return pick<float, 2>(a, back, s);
    default: return pick<float, 1>(a, back, s);
  }
}

}  // namespace

hipError_t launch_rotary_forward(bool bf16, int v, const RotaryArgs &a, hipStream_t s) { return launch(bf16, v, a, false, s); }
hipError_t launch_rotary_backward(bool bf16, int v, const RotaryArgs &a, hipStream_t s) { return launch(bf16, v, a, true, s); }

}  // namespace hapi
