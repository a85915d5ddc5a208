// Rotary positions on several axes, with the heads' RMS norm in the same pass,
// forward and backward.
//
// A vector (one head of one token) belongs to LV lanes of a wave, a lane to V pairs of
// it: V values of either side of the pairs, 16 bytes each where widths, strides and
// addresses allow it; what is not rotated goes as pairs that turn by nothing.  A lane
// keeps its pairs over the heads of a token, so that angles, sines and cosines are
// formed once for all of them.  The angle is position times frequency in float64,
// reduced to a part of a turn there: in float32 its rounding at position 1e6 would be
// 0.03 radians.  Norm, rotation and sums are float32, outputs are rounded once.
//
// Backward turns dy by the opposite angle and goes back through the norm, whose
// 1 / sqrt it forms again from x.  A lane sums its columns of the gammas' gradients
// over its vectors, a block its lanes in LDS and a second kernel the blocks, in a
// fixed order.
//
// Bound by memory: x read and y written, backward x and dy read and dx written.
#include "block.h"

namespace hapi {
namespace {

constexpr int kThreads = 256;

template <typename T>
__device__ __forceinline__ float widen(T v) {
  if constexpr (sizeof(T) == 2) return __uint_as_float((uint32_t)v << 16);
  else return v;
}

// V values from p on; n: how many there are (V = 1: it may be none).
template <typename T, int V>
__device__ __forceinline__ void load(const T *p, bool there, float (&f)[V]) {
  if constexpr (V == 1) {
    f[0] = there ? widen(*p) : 0.0f;
  } else {
    T v[V];
    __builtin_memcpy(v, p, V * sizeof(T));
#pragma unroll
    for (int j = 0; j < V; ++j) f[j] = widen(v[j]);
  }
}
template <typename T, int V>
__device__ __forceinline__ void store(T *p, bool there, const float (&f)[V]) {
  if constexpr (V == 1) {
    if (there) {
      if constexpr (sizeof(T) == 2) *p = f2bf(f[0]);
      else *p = f[0];
    }
  } else {
    T v[V];
    if constexpr (sizeof(T) == 2) {
#pragma unroll
      for (int j = 0; j < V; j += 2) {
        const uint32_t w = f2bf2(f[j], f[j + 1]);
        __builtin_memcpy(v + j, &w, 4);
      }
    } else {
#pragma unroll
      for (int j = 0; j < V; ++j) v[j] = f[j];
    }
    __builtin_memcpy(p, v, V * sizeof(T));
  }
}

// LV lanes of a vector, NU units (V pairs each) of a lane.
template <typename T, int V, int LV, int NU, bool NEIGHBOURS, bool BACK>
__global__ __launch_bounds__(kThreads) void rotary_kernel(RotaryArgs a) {
  constexpr int GPB = kThreads / LV;
  __shared__ float acc_s[BACK ? kThreads * 2 * V * NU : 1];
  const int lane = threadIdx.x % LV;
  const int D = a.dim, P = a.pairs;
  // where this lane's units lie
  int ea[NU], eb[NU];
  bool there[NU], second[NU];
  double freq[NU][V];
  int axis[NU][V];  // kRotaryAxes: not rotated
  float gamma[2][NU][2 * V];
#pragma unroll
  for (int n = 0; n < NU; ++n) {
    const int u = lane + n * LV;
    const bool turns = u * V < P;
    ea[n] = turns && !NEIGHBOURS ? u * V : 2 * u * V;
    eb[n] = turns && !NEIGHBOURS ? P + u * V : 2 * u * V + V;
    there[n] = ea[n] < D;
    second[n] = eb[n] < D;
#pragma unroll
    for (int j = 0; j < V; ++j) {
      freq[n][j] = turns ? a.freq[u * V + j] : 0.0;
      axis[n][j] = kRotaryAxes;
      if (turns) {
#pragma unroll
        for (int x = 0; x < kRotaryAxes; ++x)
          if (x < a.axes && u * V + j >= a.first[x]) axis[n][j] = x;
      }
    }
#pragma unroll
    for (int w = 0; w < 2; ++w)
#pragma unroll
      for (int j = 0; j < 2 * V; ++j) {
        const int e = j < V ? ea[n] + j : eb[n] + j - V;
        gamma[w][n][j] = a.norm && a.heads[w] > 0 && there[n] && e < D ? a.gamma[w][e] : 1.0f;
      }
  }
  float dg[2][NU][2 * V];
#pragma unroll
  for (int w = 0; w < 2; ++w)
#pragma unroll
    for (int n = 0; n < NU; ++n)
#pragma unroll
      for (int j = 0; j < 2 * V; ++j) dg[w][n][j] = 0.0f;

  const int groups = a.head_groups, heads = a.heads[0] + a.heads[1];
  const uint32_t total = (uint32_t)(a.tokens * groups);  // < 2^31
  for (uint32_t g = blockIdx.x * GPB + threadIdx.x / LV; g < total; g += gridDim.x * GPB) {
    const uint32_t token = g / (uint32_t)groups;
    const int first_head = (int)(g - token * groups);
    const uint32_t b = token / (uint32_t)a.len, l = token - b * a.len;
    const bool counts = !a.lens || (int64_t)l < a.lens[b];
    double pos[kRotaryAxes + 1];
#pragma unroll
    for (int x = 0; x < kRotaryAxes; ++x) pos[x] = x < a.axes && counts ? (double)a.positions[x * a.tokens + token] : 0.0;
    float cs[NU][V], sn[NU][V];
#pragma unroll
    for (int n = 0; n < NU; ++n)
#pragma unroll
      for (int j = 0; j < V; ++j) {
        double p = 0.0;
#pragma unroll
        for (int x = 0; x < kRotaryAxes; ++x) p = axis[n][j] == x ? pos[x] : p;
        // part of a turn, in [-1/2, 1/2]
        double turn = p * freq[n][j] * 0.15915494309189535;
        turn -= rint(turn);
        sincospif(2.0f * (float)turn, &sn[n][j], &cs[n][j]);
        if (BACK) sn[n][j] = -sn[n][j];
      }
    for (int h = first_head; h < heads; h += groups) {
      const int w = h >= a.heads[0];
      const int64_t hh = w ? h - a.heads[0] : h;
      const int64_t xo = (int64_t)b * a.x_st[w][0] + (int64_t)l * a.x_st[w][1] + hh * a.x_st[w][2];
      const int64_t yo = (int64_t)b * a.y_st[w][0] + (int64_t)l * a.y_st[w][1] + hh * a.y_st[w][2];
      // forward: v = x; backward: v = dy, x = x
      float v[NU][2 * V], x[NU][2 * V];
      const T *src = static_cast<const T *>(BACK ? a.dy[w] : a.x[w]) + (BACK ? yo : xo);
      const T *xs = static_cast<const T *>(a.x[w]) + xo;
#pragma unroll
      for (int n = 0; n < NU; ++n) {
        float lo[V], hi[V];
#pragma unroll
        for (int j = 0; j < V; ++j) lo[j] = hi[j] = 0.0f;
        if (counts && there[n]) {
          load<T, V>(src + ea[n], true, lo);
          load<T, V>(src + eb[n], second[n], hi);
        }
#pragma unroll
        for (int j = 0; j < V; ++j) v[n][j] = lo[j], v[n][V + j] = hi[j];
        if (BACK) {
#pragma unroll
          for (int j = 0; j < V; ++j) lo[j] = hi[j] = 0.0f;
          if (counts && there[n] && a.norm) {
            load<T, V>(xs + ea[n], true, lo);
            load<T, V>(xs + eb[n], second[n], hi);
          }
#pragma unroll
          for (int j = 0; j < V; ++j) x[n][j] = lo[j], x[n][V + j] = hi[j];
        }
      }
      auto rotate = [&](int n) {
#pragma unroll
        for (int j = 0; j < V; ++j) {
          float &p = NEIGHBOURS ? v[n][2 * j] : v[n][j];
          float &q = NEIGHBOURS ? v[n][2 * j + 1] : v[n][V + j];
          const float p0 = p, q0 = q;
          p = p0 * cs[n][j] - q0 * sn[n][j];
          q = q0 * cs[n][j] + p0 * sn[n][j];
        }
      };
      if (!BACK) {
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
            for (int j = 0; j < 2 * V; ++j) v[n][j] = counts ? v[n][j] * r * (w ? gamma[1][n][j] : gamma[0][n][j]) : 0.0f;
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
              ex = fmaf(v[n][j] * (w ? gamma[1][n][j] : gamma[0][n][j]), x[n][j], ex);
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
              if (w) dg[1][n][j] = fmaf(u, hx, dg[1][n][j]);
              else dg[0][n][j] = fmaf(u, hx, dg[0][n][j]);
              v[n][j] = counts ? r * (u * (w ? gamma[1][n][j] : gamma[0][n][j]) - hx * c) : 0.0f;
            }
        }
      }
      T *dst = static_cast<T *>(a.y[w]) + (BACK ? xo : yo);
#pragma unroll
      for (int n = 0; n < NU; ++n)
        if (there[n]) {
          float lo[V], hi[V];
#pragma unroll
          for (int j = 0; j < V; ++j) lo[j] = v[n][j], hi[j] = v[n][V + j];
          store<T, V>(dst + ea[n], true, lo);
          store<T, V>(dst + eb[n], second[n], hi);
        }
    }
  }
  if constexpr (BACK) {
    if (!a.norm) return;
    // a column's sum over the block's groups of lanes
    for (int w = 0; w < 2; ++w) {
      if (a.heads[w] == 0) continue;
      __syncthreads();
#pragma unroll
      for (int n = 0; n < NU; ++n)
#pragma unroll
        for (int j = 0; j < 2 * V; ++j) acc_s[(n * 2 * V + j) * kThreads + threadIdx.x] = w ? dg[1][n][j] : dg[0][n][j];
      __syncthreads();
      for (int i = threadIdx.x; i < LV * NU * 2 * V; i += kThreads) {
        const int ln = i % LV, k = i / LV, n = k / (2 * V), j = k % (2 * V);
        const int u = ln + n * LV;
        const bool turns = u * V < P;
        const int e = j < V ? (turns && !NEIGHBOURS ? u * V : 2 * u * V) + j : (turns && !NEIGHBOURS ? P + u * V : 2 * u * V + V) + j - V;
        if ((turns && !NEIGHBOURS ? u * V : 2 * u * V) >= D || e >= D) continue;
        float s = 0.0f;
        for (int q = 0; q < GPB; ++q) s += acc_s[k * kThreads + q * LV + ln];
        a.part[((int64_t)blockIdx.x * 2 + w) * D + e] = s;
      }
    }
  }
}

// dgamma of q and k: 16 columns a block, 16 slices of the parts.
__global__ __launch_bounds__(256) void rotary_reduce_kernel(RotaryArgs a, int parts) {
  __shared__ double s[16][17];
  const int c = threadIdx.x & 15, slice = threadIdx.x >> 4;
  const int e = blockIdx.x * 16 + c, w = blockIdx.y;
  if (a.heads[w] == 0) return;
  double t = 0.0;
  if (e < a.dim)
    for (int p = slice; p < parts; p += 16) t += (double)a.part[((int64_t)p * 2 + w) * a.dim + e];
  s[slice][c] = t;
  __syncthreads();
  if (slice == 0 && e < a.dim) {
#pragma unroll
    for (int i = 1; i < 16; ++i) t += s[i][c];
    a.dgamma[w][e] = (float)t;
  }
}

template <typename T, int V, int LV, int NU>
hipError_t run(const RotaryArgs &a, bool back, hipStream_t s) {
  constexpr int gpb = kThreads / LV;
  const int64_t want = ceil_div(a.tokens * a.head_groups, gpb);
  const int64_t most = back && a.norm ? kRotaryParts : kMaxLaunchThreads / kThreads;
  const dim3 grid((uint32_t)(want < most ? want : most)), block(kThreads);
  if (want == 0) {  // no tokens: the gammas' gradients are sums of nothing
    hapi_launch(rotary_reduce_kernel, dim3((a.dim + 15) / 16, 2), dim3(256), 0, s, a, 0);
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
  hapi_launch(rotary_reduce_kernel, dim3((a.dim + 15) / 16, 2), dim3(256), 0, s, a, (int)grid.x);
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
