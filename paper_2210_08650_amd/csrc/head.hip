// Cross entropy and distillation of a linear classifier over many classes,
// with its gradients, the logits never in memory.
//
// Every product is one tiled kernel, out[b][a] = sum_k A(a, k) B(b, k), on
// 32 x 32 MFMAs whose lanes own b and whose registers own a, so that a lane
// holds runs of consecutive a of one output row.  An operand's k is contiguous
// (a row of the tile is 128 bytes of LDS) or its a / b is (a row of the tile is
// one k; 16-bit fragments are then read transposed, ds_read_b64_tr_b16).
//
//   forward    a = class, b = row:  epilogue = (max, sum of exp) of a row over the
//              tile's classes; a second kernel joins these and forms the loss.
//   dz^T       a = row, b = class:  the same product again, epilogue
//              g exp(z - m) / sum, stored transposed, one piece of the classes at a
//              time: a lane owns a class, so the bias's gradient is a sum of its
//              own registers.  The targets' entries are put in by a small kernel.
//   dx         a = feature, b = row, k = class: dz^T and the weights as they lie,
//              the piece's classes split over workgroups, float32 partial sums.
//   dW         a = feature, b = class, k = row: dz^T and x as they lie.
//
// float32 uses v_mfma_f32_32x32x2_f32 in the same tiles (128 bytes of k).
// dz is rounded to the operands' type before its two products (the matrix
// cores' bf16 operands; 2^-8 of each entry at most, against 2^-8 of the
// outputs' own rounding); sums, softmax statistics and the bias's gradient are
// float32 throughout.
#include "gemm_util.h"
#include "tail.h"

namespace hapi {
namespace {

typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef short s16x4_t __attribute__((ext_vector_type(4)));

constexpr float kLog2e = 1.4426950408889634f;

// One product's operands and extents.
struct Gemm {
  const void *a, *b;
  int64_t a_ld, b_ld;
  int a_ext, b_ext, k_ext;  // valid rows of A and B and valid k
  int tiles_a, tiles_b;
  int splits;               // of k, over workgroups: whole k-tiles
};

enum Epi { E_STATS, E_DLOGITS, E_DX, E_DW };

template <typename T>
struct Elem;
template <>
struct Elem<uint16_t> {
  typedef bf16x8_t Frag;
};
template <>
struct Elem<float> {
  typedef f32x4_t Frag;
};

__device__ __forceinline__ f32x16_t mma(bf16x8_t a, bf16x8_t b, f32x16_t c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ f32x16_t mma(f32x4_t a, f32x4_t b, f32x16_t c) {
#pragma unroll
  for (int j = 0; j < 4; ++j) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a[j], b[j], c, 0, 0, 0);
  return c;
}

// A tile's operand of R rows (of a or b) by 128 bytes of k.  KR: memory and LDS
// rows are k.  LDS slots of 16 bytes are permuted within a row so that the
// fragment reads spread over the banks; a DMA writes them in order, so the
// permutation is in the address each lane loads from.
template <typename T, int R, bool KR, int WAVES>
struct Side {
  static constexpr int V = 16 / (int)sizeof(T), KT = 128 / (int)sizeof(T);
  static constexpr int LOADS = R / 8 / WAVES;  // DMAs of 1 KB a wave issues per k-tile
  static constexpr int BYTES = R * 128;
  static_assert(LOADS * 8 * WAVES == R, "whole DMAs per wave");
  static constexpr int CPR = KR ? R / V : 8;      // 16-byte slots of an LDS row (a power of two)
  static constexpr int RPD = 64 / CPR;            // LDS rows of one DMA
  static_assert(CPR <= 64, "a DMA covers whole LDS rows");

  uint32_t off[LOADS];  // byte offset of this lane from the k-tile's base
  int lk[LOADS];        // this lane's k within the k-tile

  static __device__ __forceinline__ int swz(int row) {
    if constexpr (!KR) return (row >> 1) & 7;
    if constexpr (KR && sizeof(T) == 2) return (4 * (row & 3)) & (CPR - 1);
    return 0;
  }
  __device__ __forceinline__ void init(int r0, int ext, int64_t ld, int wave, int lane) {
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
      const int lr = (wave * LOADS + i) * RPD + lane / CPR;  // LDS row
      const int c = (lane % CPR) ^ swz(lr);                  // 16-byte slot of the memory row
      const int r = KR ? r0 + c * V : r0 + lr;
      lk[i] = KR ? lr : c * V;
      // r0's own offset is in the base
      const int64_t o = KR ? (int64_t)lr * ld + c * V : (int64_t)lr * ld + c * V;
      off[i] = r < ext ? (uint32_t)(o * (int64_t)sizeof(T)) : kOob;
    }
  }
  __device__ __forceinline__ void issue(const uint8_t *base, uint32_t lds, int k_left, int wave) const {
    const u32x4_t srd = make_srd(base);
#pragma unroll
    for (int i = 0; i < LOADS; ++i)
      lds_dma16(srd, lds + (wave * LOADS + i) * 1024, lk[i] < k_left ? off[i] : kOob, 0);
  }
  // Bytes from one k-tile to the next, and of the tile's first row.
  static __device__ __forceinline__ int64_t k_step(int64_t ld) { return KR ? KT * ld * (int64_t)sizeof(T) : 128; }
  static __device__ __forceinline__ int64_t row_base(int r0, int64_t ld) {
    return (KR ? (int64_t)r0 : (int64_t)r0 * ld) * (int64_t)sizeof(T);
  }
  // This lane's fragment of 32 rows from r on, k-step ks (16 values of 16 bits, 8 of 32).
  static __device__ __forceinline__ typename Elem<T>::Frag frag(const uint8_t *tile, int r, int ks, int lane) {
    typedef typename Elem<T>::Frag F;
    const int lh = lane >> 5;
    if constexpr (!KR) {
      const int row = r + (lane & 31);
      return *reinterpret_cast<const F *>(tile + row * 128 + (((2 * ks + lh) ^ swz(row)) * 16));
    } else if constexpr (sizeof(T) == 2) {
      // 16 lanes read 4 k of 16 rows, lane i getting row i's four
      const int i = lane & 15, col = r + (lane & 16) + 4 * (i & 3);
      union {
        s16x4_t h[2];
        F f;
      } u;
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int k = 16 * ks + 8 * lh + 4 * e + (i >> 2);
        const uint8_t *p = tile + k * (R * 2) + (((col >> 3) ^ swz(k)) * 16) + (col & 7) * 2;
        u.h[e] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
            (__attribute__((address_space(3))) s16x4_t *)(__attribute__((address_space(3))) void *)p);
      }
      return u.f;
    } else {
      F f;
#pragma unroll
      for (int j = 0; j < 4; ++j)
        f[j] = *reinterpret_cast<const float *>(tile + (8 * ks + 4 * lh + j) * (R * 4) + (r + (lane & 31)) * 4);
      return f;
    }
  }
};

// What the epilogue needs of the tile's reg side: the bias of its classes (-inf
// past the last one), or its rows' info.
template <int EPI, int BA, int THREADS>
__device__ __forceinline__ void load_side(const Gemm &g, const HeadArgs &h, float2 *side_s, int a0, int t) {
  if constexpr (EPI == E_STATS)
    for (int i = t; i < BA; i += THREADS)
      side_s[i].x = a0 + i < g.a_ext ? (h.bias ? h.bias[a0 + i] : 0.0f) : -INFINITY;
  if constexpr (EPI == E_DLOGITS)
    for (int i = t; i < BA; i += THREADS) side_s[i] = a0 + i < h.rows_pad ? h.info[a0 + i] : make_float2(INFINITY, 0.0f);
}

// Where a wave's blocks lie: block (i, j) is out[lane(j) + lane % 32][reg(i) + 8 q +
// 4 lh + e] = acc[i][j][4 q + e]; part: which of the reg side's parts the wave holds.
template <int REG_STEP, int LANE_A, int LANE_B>
struct Place {
  int a0, r0, l0, part;
  __device__ __forceinline__ int reg(int i) const { return r0 + REG_STEP * i; }
  __device__ __forceinline__ int lane(int j) const { return l0 + (j >> 1) * LANE_B + (j & 1) * LANE_A; }
};

template <typename T, int EPI, int TA, int TB, typename P>
__device__ __forceinline__ void epilogue(const Gemm &g, const HeadArgs &h, f32x16_t (&acc)[TA][TB], const P &at,
                                         const float2 *side_s, int split, int lane) {
  const int lh = lane >> 5;
  if constexpr (EPI == E_STATS) {
    const float c = kLog2e * h.inv_t;
#pragma unroll
    for (int j = 0; j < TB; ++j) {
      float m = -INFINITY;
#pragma unroll
      for (int i = 0; i < TA; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          acc[i][j][r] += side_s[at.reg(i) - at.a0 + 8 * (r >> 2) + 4 * lh + (r & 3)].x;
          m = fmaxf(m, acc[i][j][r]);
        }
      m = fmaxf(m, __shfl_xor(m, 32, 64));
      const float mm = m == -INFINITY ? 0.0f : m;  // no class with weight: the sum is 0, not NaN
      float s = 0.0f;
#pragma unroll
      for (int i = 0; i < TA; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r) s += __builtin_amdgcn_exp2f((acc[i][j][r] - mm) * c);
      s += __shfl_xor(s, 32, 64);
      const int row = at.lane(j) + (lane & 31);
      if (lh == 0 && row < g.b_ext) h.part[(int64_t)at.part * h.rows + row] = make_float2(m, s);
    }
  }
  if constexpr (EPI == E_DLOGITS) {
    T *gt = static_cast<T *>(h.gt);
    const float c = kLog2e * h.inv_t;
#pragma unroll
    for (int j = 0; j < TB; ++j) {
      const int cls = at.lane(j) + (lane & 31);  // in the piece
      const bool live = cls < g.b_ext;
      const float bias = live && h.bias ? h.bias[h.v0 + cls] : 0.0f;
      float sum = 0.0f;
#pragma unroll
      for (int i = 0; i < TA; ++i) {
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const float2 in = side_s[at.reg(i) - at.a0 + 8 * (r >> 2) + 4 * lh + (r & 3)];
          const float z = acc[i][j][r] + bias;
          const float v = __builtin_amdgcn_exp2f((z - in.x) * c) * in.y;
          acc[i][j][r] = v;
          sum += v;
        }
        const int a = at.reg(i);
        T *o = gt + (int64_t)cls * h.rows_pad + a;
        if constexpr (sizeof(T) == 2) {
#pragma unroll
          for (int p = 0; p < 2; ++p) {
            float v[8];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const auto s2 = __builtin_amdgcn_permlane32_swap(__float_as_uint(acc[i][j][8 * p + e]),
                                                               __float_as_uint(acc[i][j][8 * p + 4 + e]), false, false);
              v[e] = __uint_as_float(s2[0]);
              v[4 + e] = __uint_as_float(s2[1]);
            }
            const int n = 16 * p + 8 * lh;
            if (live && a + n < h.rows_pad)
              *reinterpret_cast<uint4 *>(o + n) =
                  make_uint4(f2bf2(v[0], v[1]), f2bf2(v[2], v[3]), f2bf2(v[4], v[5]), f2bf2(v[6], v[7]));
          }
        } else {
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            const int n = 8 * q + 4 * lh;
            if (live && a + n < h.rows_pad)
              *reinterpret_cast<float4 *>(o + n) =
                  make_float4(acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]);
          }
        }
      }
      if (h.db_part) {
        sum += __shfl_xor(sum, 32, 64);
        if (lh == 0 && live) h.db_part[(int64_t)at.part * h.classes + h.v0 + cls] = sum;
      }
    }
  }
  if constexpr (EPI == E_DX) {
    float *out = h.dx_part + (int64_t)split * h.rows * h.dx_pad;
#pragma unroll
    for (int j = 0; j < TB; ++j) {
      const int row = at.lane(j) + (lane & 31);
      if (row >= g.b_ext) continue;
#pragma unroll
      for (int i = 0; i < TA; ++i)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const int a = at.reg(i) + 8 * q + 4 * lh;
          if (a >= h.dx_pad) continue;
          float4 *p = reinterpret_cast<float4 *>(out + (int64_t)row * h.dx_pad + a);
          float4 v = make_float4(acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]);
          if (!h.first) {
            const float4 u = *p;
            v.x += u.x; v.y += u.y; v.z += u.z; v.w += u.w;
          }
          *p = v;
        }
    }
  }
  if constexpr (EPI == E_DW) {
    T *out = static_cast<T *>(h.dw);
    const bool vec = h.dw_ld % (16 / (int)sizeof(T)) == 0 && (uintptr_t)out % 16 == 0;
#pragma unroll
    for (int j = 0; j < TB; ++j) {
      const int cls = at.lane(j) + (lane & 31);
      const bool live = cls < g.b_ext;
      T *o = out + (h.v0 + cls) * h.dw_ld;
#pragma unroll
      for (int i = 0; i < TA; ++i) {
        const int a = at.reg(i);
        if constexpr (sizeof(T) == 2) {
#pragma unroll
          for (int p = 0; p < 2; ++p) {
            float v[8];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const auto s2 = __builtin_amdgcn_permlane32_swap(__float_as_uint(acc[i][j][8 * p + e]),
                                                               __float_as_uint(acc[i][j][8 * p + 4 + e]), false, false);
              v[e] = __uint_as_float(s2[0]);
              v[4 + e] = __uint_as_float(s2[1]);
            }
            const int n = a + 16 * p + 8 * lh;
            if (!live) continue;
            if (vec && n + 8 <= h.dim) {
              *reinterpret_cast<uint4 *>(o + n) =
                  make_uint4(f2bf2(v[0], v[1]), f2bf2(v[2], v[3]), f2bf2(v[4], v[5]), f2bf2(v[6], v[7]));
            } else {
#pragma unroll
              for (int e = 0; e < 8; ++e)
                if (n + e < h.dim) o[n + e] = f2bf(v[e]);
            }
          }
        } else {
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            const int n = a + 8 * q + 4 * lh;
            if (!live) continue;
            if (vec && n + 4 <= h.dim) {
              *reinterpret_cast<float4 *>(o + n) =
                  make_float4(acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]);
            } else {
#pragma unroll
              for (int e = 0; e < 4; ++e)
                if (n + e < h.dim) o[n + e] = acc[i][j][4 * q + e];
            }
          }
        }
      }
    }
  }
}

template <typename T, int BA, int BB, int WA, int WB, int ST, bool KRA, bool KRB, int EPI>
__global__ __launch_bounds__(64 * WA * WB) void head_gemm_kernel(Gemm g, HeadArgs h) {
  constexpr int WAVES = WA * WB, TA = BA / WA / 32, TB = BB / WB / 32;
  typedef Side<T, BA, KRA, WAVES> SA;
  typedef Side<T, BB, KRB, WAVES> SB;
  constexpr int STAGE = SA::BYTES + SB::BYTES;
  __shared__ __attribute__((aligned(1024))) uint8_t smem[ST * STAGE];
  __shared__ __attribute__((aligned(16))) float2 side_s[EPI == E_STATS || EPI == E_DLOGITS ? BA : 1];

  const int t = threadIdx.x, lane = t & 63;
  const int wave = __builtin_amdgcn_readfirstlane(t >> 6);
  const int wa = wave / WB, wb = wave % WB;
  const int bid = xcd_remap(blockIdx.x, gridDim.x);
  const int tiles = g.tiles_a * g.tiles_b;
  const int split = bid / tiles, tile = bid % tiles;
  // the smaller side of the grid runs fastest, so the larger one's operand is
  // read by workgroups that run together
  const int ta = g.tiles_a <= g.tiles_b ? tile % g.tiles_a : tile / g.tiles_b;
  const int tb = g.tiles_a <= g.tiles_b ? tile / g.tiles_a : tile % g.tiles_b;
  const int a0 = ta * BA, b0 = tb * BB;
  const int nkt = (g.k_ext + SA::KT - 1) / SA::KT;
  const int kt0 = (int)((int64_t)nkt * split / g.splits), kt1 = (int)((int64_t)nkt * (split + 1) / g.splits);
  const int nk = kt1 - kt0;

  load_side<EPI, BA, 64 * WAVES>(g, h, side_s, a0, t);

  SA sa;
  SB sb;
  sa.init(a0, g.a_ext, g.a_ld, wave, lane);
  sb.init(b0, g.b_ext, g.b_ld, wave, lane);
  const int64_t da = SA::k_step(g.a_ld), db = SB::k_step(g.b_ld);
  const uint8_t *pa = static_cast<const uint8_t *>(g.a) + SA::row_base(a0, g.a_ld) + kt0 * da;
  const uint8_t *pb = static_cast<const uint8_t *>(g.b) + SB::row_base(b0, g.b_ld) + kt0 * db;
  const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t *)smem;
  int k_left = g.k_ext - kt0 * SA::KT, issued = 0;
  // Loads past the split's last k-tile read nothing (zeros), so that every
  // k-tile's wait counts the same.
  auto issue = [&] {
    const uint32_t dst = lds0 + (uint32_t)(issued % ST) * STAGE;
    const int left = issued < nk ? k_left : 0;
    sa.issue(pa, dst, left, wave);
    sb.issue(pb, dst + SA::BYTES, left, wave);
    ++issued;
    if (issued < nk) {
      pa += da;
      pb += db;
      k_left -= SA::KT;
    }
  };

  f32x16_t acc[TA][TB];
#pragma unroll
  for (int i = 0; i < TA; ++i)
#pragma unroll
    for (int j = 0; j < TB; ++j)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.0f;

#pragma unroll
  for (int s = 0; s < ST - 1; ++s) issue();
  constexpr int PER = SA::LOADS + SB::LOADS;
  for (int kt = 0; kt < nk; ++kt) {
    // this wave's part of the k-tile has landed and its reads of the last one
    // are done; after the barrier, everyone's
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"((ST - 2) * PER) : "memory");
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
    issue();
    const uint8_t *at = smem + (kt % ST) * STAGE, *bt = at + SA::BYTES;
#pragma unroll
    for (int ks = 0; ks < 4; ++ks) {
      typename Elem<T>::Frag fa[TA], fb[TB];
#pragma unroll
      for (int i = 0; i < TA; ++i) fa[i] = SA::frag(at, (wa * TA + i) * 32, ks, lane);
#pragma unroll
      for (int j = 0; j < TB; ++j) fb[j] = SB::frag(bt, (wb * TB + j) * 32, ks, lane);
#pragma unroll
      for (int i = 0; i < TA; ++i)
#pragma unroll
        for (int j = 0; j < TB; ++j) acc[i][j] = mma(fa[i], fb[j], acc[i][j]);
    }
  }
  // No DMA may outlive the workgroup's LDS, and side_s is read by all waves.
  asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
  __syncthreads();

  const Place<32, 32, 64> at = {a0, a0 + wa * TA * 32, b0 + wb * TB * 32, ta * WA + wa};
  epilogue<T, EPI>(g, h, acc, at, side_s, split, lane);
}

template <typename T, int BA, int BB, int WA, int WB, int ST, bool KRA, bool KRB, int EPI>
hipError_t launch_gemm(Gemm g, const HeadArgs &h, hipStream_t s) {
  g.tiles_a = (g.a_ext + BA - 1) / BA;
  g.tiles_b = (g.b_ext + BB - 1) / BB;
  const int64_t blocks = (int64_t)g.tiles_a * g.tiles_b * g.splits;
  if (blocks == 0) return hipSuccess;
  if (blocks > 0x7fffffff) return hipErrorInvalidValue;
  hapi_launch((head_gemm_kernel<T, BA, BB, WA, WB, ST, KRA, KRB, EPI>), dim3((uint32_t)blocks), dim3(64 * WA * WB), 0, s,
              g, h);
  return hipGetLastError();
}

// The same product on 256 x 256 tiles.  Eight waves, two per SIMD: wave (g, c)
// owns rows 64 g .. + 63 of both 128-row halves of B and rows 32 c .. + 31 of both
// halves of A, 128 accumulator registers.  A k-tile is two steps, each a memory
// slot (fragments of the next 16 MFMAs out of LDS, DMAs of a later k-tile into
// it) and a matrix slot, with a barrier after every slot; the two groups g run one
// slot apart, so one group's MFMAs cover the other's LDS reads.  Two stages of
// 64 KB; half a stage is loaded again as soon as both groups have read it.
template <typename T, bool KRA, bool KRB, int EPI>
__device__ __forceinline__ void big_tile(const Gemm &g, const HeadArgs &h, uint8_t *smem, float2 *side_s, int bid) {
  typedef Side<T, 128, KRA, 8> SA;
  typedef Side<T, 128, KRB, 8> SB;
  constexpr int HALF = SA::BYTES, STAGE = 4 * HALF;  // B halves 0, 1, A halves 0, 1
  typedef typename Elem<T>::Frag Frag;
  const int t = threadIdx.x, lane = t & 63;
  const int wave = __builtin_amdgcn_readfirstlane(t >> 6);
  const int wm = wave >> 2, wn = wave & 3;
  const int tiles = g.tiles_a * g.tiles_b;
  const int split = bid / tiles, tile = bid % tiles;
  const int ta = g.tiles_a <= g.tiles_b ? tile % g.tiles_a : tile / g.tiles_b;
  const int tb = g.tiles_a <= g.tiles_b ? tile / g.tiles_a : tile % g.tiles_b;
  const int a0 = ta * 256, b0 = tb * 256;
  const int nkt = (g.k_ext + SA::KT - 1) / SA::KT;
  const int kt0 = (int)((int64_t)nkt * split / g.splits), kt1 = (int)((int64_t)nkt * (split + 1) / g.splits);
  const int nk = kt1 - kt0;
  load_side<EPI, 256, 512>(g, h, side_s, a0, t);

  SA sa[2];
  SB sb[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    sa[i].init(a0 + 128 * i, g.a_ext, g.a_ld, wave, lane);
    sb[i].init(b0 + 128 * i, g.b_ext, g.b_ld, wave, lane);
  }
  const int64_t da = SA::k_step(g.a_ld), db = SB::k_step(g.b_ld);
  const int64_t ha = SA::row_base(128, g.a_ld), hb = SB::row_base(128, g.b_ld);
  const uint8_t *pa = static_cast<const uint8_t *>(g.a) + SA::row_base(a0, g.a_ld) + kt0 * da;
  const uint8_t *pb = static_cast<const uint8_t *>(g.b) + SB::row_base(b0, g.b_ld) + kt0 * db;
  const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t *)smem;
  int k_left = nk > 0 ? g.k_ext - kt0 * SA::KT : 0, s_kt = 0;
  // The load stream's next k-tile; past the last one loads read nothing.
  auto stream_next = [&] {
    if (++s_kt < nk) {
      pa += da;
      pb += db;
      k_left -= SA::KT;
    } else {
      k_left = 0;
    }
  };
  auto issue_a = [&](uint32_t stage, int i) { sa[i].issue(pa + i * ha, lds0 + stage + (2 + i) * HALF, k_left, wave); };
  auto issue_b = [&](uint32_t stage, int i) { sb[i].issue(pb + i * hb, lds0 + stage + i * HALF, k_left, wave); };

  Frag fb[2][4], fa0[4], fa1[4];
  auto read_b = [&](uint32_t stage, int half) {
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int ks = 0; ks < 4; ++ks)
        fb[i][ks] = SB::frag(smem + stage + half * HALF, wm * 64 + 32 * i, ks, lane);
  };
  auto read_a = [&](uint32_t stage, int half, Frag(&f)[4]) {
#pragma unroll
    for (int ks = 0; ks < 4; ++ks) f[ks] = SA::frag(smem + stage + (2 + half) * HALF, wn * 32, ks, lane);
  };
  auto bar = [&] {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
  };
  // End of a memory slot: this wave's fragments are in registers, and its part of
  // what the next memory slot reads has landed (8 younger DMAs may be in flight).
  auto mem_end = [&] {
    asm volatile("s_waitcnt vmcnt(8) lgkmcnt(0)" ::: "memory");
    bar();
  };
  f32x16_t acc[2][4];
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.0f;
  auto mmas = [&](int half) {
#pragma unroll
    for (int ks = 0; ks < 4; ++ks)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        acc[0][2 * half + i] = mma(fa0[ks], fb[i][ks], acc[0][2 * half + i]);
        acc[1][2 * half + i] = mma(fa1[ks], fb[i][ks], acc[1][2 * half + i]);
      }
    __builtin_amdgcn_sched_barrier(0);
  };

  issue_b(0, 0);
  issue_a(0, 0);
  issue_a(0, 1);
  issue_b(0, 1);
  stream_next();
  issue_b(STAGE, 0);
  issue_a(STAGE, 0);
  issue_a(STAGE, 1);
  uint32_t st = 0;
  mem_end();
  if (wm == 1) bar();  // the second group runs one slot behind
  for (int kt = 0; kt < nk; ++kt) {
    read_b(st, 0);
    read_a(st, 0, fa0);
    read_a(st, 1, fa1);
    issue_b(st ^ STAGE, 1);
    stream_next();
    mem_end();
    mmas(0);
    bar();
    issue_b(st, 0);
    issue_a(st, 0);
    issue_a(st, 1);
    read_b(st, 1);
    mem_end();
    mmas(1);
    if (kt + 1 < nk) bar();
    st ^= STAGE;
  }
  if (wm == 0) bar();
  // No DMA may outlive the workgroup's LDS (the last ones read nothing).
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  const Place<128, 32, 128> at = {a0, a0 + wn * 32, b0 + wm * 64, ta * 4 + wn};
  epilogue<T, EPI>(g, h, acc, at, side_s, split, lane);
}

constexpr int kBigSmem = 8 * 128 * 128;

template <typename T, bool KRA, bool KRB, int EPI>
__global__ __launch_bounds__(512) void head_big_kernel(Gemm g, HeadArgs h) {
  __shared__ __attribute__((aligned(1024))) uint8_t smem[kBigSmem];
  __shared__ __attribute__((aligned(16))) float2 side_s[EPI == E_STATS || EPI == E_DLOGITS ? 256 : 1];
  big_tile<T, KRA, KRB, EPI>(g, h, smem, side_s, xcd_remap(blockIdx.x, gridDim.x));
}

template <typename T, bool KRA, bool KRB, int EPI>
hipError_t launch_big(Gemm g, const HeadArgs &h, hipStream_t s) {
  g.tiles_a = (g.a_ext + 255) / 256;
  g.tiles_b = (g.b_ext + 255) / 256;
  const int64_t blocks = (int64_t)g.tiles_a * g.tiles_b * g.splits;
  if (blocks == 0) return hipSuccess;
  if (blocks > 0x7fffffff) return hipErrorInvalidValue;
  hapi_launch((head_big_kernel<T, KRA, KRB, EPI>), dim3((uint32_t)blocks), dim3(512), 0, s, g, h);
  return hipGetLastError();
}

// ------------------------------------------------------------ small kernels

__device__ __forceinline__ float to_f(uint16_t v) { return bf2f(v); }
__device__ __forceinline__ float to_f(float v) { return v; }
__device__ __forceinline__ void put(uint16_t *p, float v) { *p = f2bf(v); }
__device__ __forceinline__ void put(float *p, float v) { *p = v; }

// out[r][0 .. ld_out) = in[r][0 .. dim), zeros behind; a thread per 16 bytes.
// info (optional): rows whose coefficient is 0 become zeros.
template <typename T>
__global__ __launch_bounds__(256) void stage_kernel(const T *__restrict__ in, int64_t ld_in, T *__restrict__ out,
                                                    int64_t ld_out, int64_t rows, int dim, const float2 *info) {
  constexpr int V = 16 / (int)sizeof(T);
  const int64_t per = ld_out / V;
  const int64_t n = rows * per;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) {
    const int64_t r = i / per;
    const int d = (int)(i - r * per) * V;
    const T *p = in + r * ld_in + d;
    T v[V] = {};
    if (!info || info[r].y != 0.0f) {
      if (d + V <= dim) {
        __builtin_memcpy(v, p, 16);
      } else {
#pragma unroll
        for (int j = 0; j < V; ++j)
          if (d + j < dim) v[j] = p[j];
      }
    }
    uint4 q;
    __builtin_memcpy(&q, v, 16);
    *reinterpret_cast<uint4 *>(out + r * ld_out + d) = q;
  }
}

__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) v += __shfl_xor(v, o, 64);
  return v;
}
__device__ __forceinline__ float wave_max(float v) {
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) v = fmaxf(v, __shfl_xor(v, o, 64));
  return v;
}

// x[row] . w[id] by one wave.
template <typename T>
__device__ __forceinline__ float wave_dot(const T *x, const T *w, int dim, int lane) {
  constexpr int V = 16 / (int)sizeof(T);
  float s = 0.0f;
  for (int d = lane * V; d < dim; d += 64 * V) {
    T a[V], b[V];
    if (d + V <= dim) {
      __builtin_memcpy(a, x + d, 16);
      __builtin_memcpy(b, w + d, 16);
#pragma unroll
      for (int j = 0; j < V; ++j) s = fmaf(to_f(a[j]), to_f(b[j]), s);
    } else {
#pragma unroll
      for (int j = 0; j < V; ++j)
        if (d + j < dim) s = fmaf(to_f(x[d + j]), to_f(w[d + j]), s);
    }
  }
  return wave_sum(s);
}

// Joins a row's partial statistics and forms its loss: 16 rows a block, 64
// threads on a row's parts, then a wave per row for the logits at its targets.
// Merging two (max, sum) pairs rescales the smaller one's sum.
constexpr int kFinishRows = 16;
template <typename T>
__global__ __launch_bounds__(1024) void head_finish_kernel(HeadArgs h) {
  __shared__ float2 ms[16][kFinishRows];
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
  const int64_t r0 = (int64_t)blockIdx.x * kFinishRows;
  const float c = kLog2e * h.inv_t;
  const int64_t row = r0 + (t & 15);
  float m = -INFINITY, s = 0.0f;
  auto merge = [&](float m2, float s2) {
    const float mx = fmaxf(m, m2);
    const float mm = mx == -INFINITY ? 0.0f : mx;
    s = s * __builtin_amdgcn_exp2f((m - mm) * c) + s2 * __builtin_amdgcn_exp2f((m2 - mm) * c);
    m = mx;
  };
  if (row < h.rows)
    for (int p = t >> 4; p < h.parts; p += 64) {
      const float2 v = h.part[(int64_t)p * h.rows + row];
      merge(v.x, v.y);
    }
#pragma unroll
  for (int o = 16; o <= 32; o <<= 1) {
    const float m2 = __shfl_xor(m, o, 64), s2 = __shfl_xor(s, o, 64);
    merge(m2, s2);
  }
  if (lane < 16) ms[wave][lane] = make_float2(m, s);
  __syncthreads();
  // wave w: row w
  const int64_t n = r0 + wave;
  if (n >= h.rows) return;
  m = ms[lane & 15][wave].x;
  s = ms[lane & 15][wave].y;
#pragma unroll
  for (int o = 1; o <= 8; o <<= 1) {
    const float m2 = __shfl_xor(m, o, 64), s2 = __shfl_xor(s, o, 64);
    merge(m2, s2);
  }
  const float l = logf(s);
  if (lane == 0) h.stats[n] = make_float2(m, l);

  const T *x = static_cast<const T *>(h.x_in) + n * h.x_in_ld;
  const T *w = static_cast<const T *>(h.w_in);
  if (!h.teacher) {
    const int64_t id = h.ids[n];
    float loss = 0.0f;
    if (id >= h.classes) {
      loss = NAN;
    } else if (id >= 0) {
      float z = wave_dot(x, w + id * h.w_in_ld, h.dim, lane);
      if (h.bias) z += h.bias[id];
      loss = (m - z) + l;
    }
    if (lane == 0) h.loss[n] = loss;
    return;
  }
  // q = softmax(teacher / T) over the entries that count
  const int64_t *ids = h.ids + n * h.top;
  const float *te = h.teacher + n * h.top;
  float tm = -INFINITY, bad = 0.0f;
  for (int k = lane; k < h.top; k += 64)
    if (ids[k] >= 0) {
      tm = fmaxf(tm, te[k]);
      if (ids[k] >= h.classes || !(te[k] < INFINITY)) bad = 1.0f;
    }
  tm = wave_max(tm);
  bad = wave_max(bad);
  const bool none = tm == -INFINITY;
  float ts = 0.0f;
  for (int k = lane; k < h.top; k += 64)
    if (ids[k] >= 0 && !none) ts += __builtin_amdgcn_exp2f((te[k] - tm) * c);
  ts = wave_sum(ts);
  const float lts = logf(ts);
  float loss = 0.0f;
  for (int k = 0; k < h.top; ++k) {
    const int64_t id = ids[k];
    float z = 0.0f;
    if (id >= 0 && id < h.classes) {
      z = wave_dot(x, w + id * h.w_in_ld, h.dim, lane);
      if (h.bias) z += h.bias[id];
      const float u = (te[k] - tm) * h.inv_t;
      const float q = __builtin_amdgcn_exp2f(u * kLog2e) / ts;
      // an entry without weight adds nothing, whatever its logit
      if (q > 0.0f) loss += q * ((u - lts) + ((m - z) * h.inv_t + l));
    }
    if (lane == 0) h.picked[n * h.top + k] = z;
  }
  if (lane == 0) h.loss[n] = bad != 0.0f ? NAN : none ? 0.0f : h.t * h.t * loss;
}

// Row info of the backward pass, a wave per row: the largest logit m and the
// coefficient over the sum of exp((z - m) / T), so that dz = exp((z - m) / T) times
// it, or (inf, 0) for a row that does not count; distillation's weights q.
__global__ __launch_bounds__(256) void head_info_kernel(HeadArgs h) {
  const int lane = threadIdx.x & 63;
  const int64_t n = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (n >= h.rows_pad) return;
  float2 info = make_float2(INFINITY, 0.0f);
  if (n < h.rows) {
    float coef = h.dloss[n] * h.t;
    bool none;
    float bad = 0.0f;
    if (!h.teacher) {
      none = h.ids[n] < 0;
      if (h.ids[n] >= h.classes) bad = 1.0f;
    } else {
      const int64_t *ids = h.ids + n * h.top;
      const float *te = h.teacher + n * h.top;
      float tm = -INFINITY;
      for (int k = lane; k < h.top; k += 64)
        if (ids[k] >= 0) {
          tm = fmaxf(tm, te[k]);
          if (ids[k] >= h.classes || !(te[k] < INFINITY)) bad = 1.0f;
        }
      tm = wave_max(tm);
      bad = wave_max(bad);
      none = tm == -INFINITY && bad == 0.0f;
      float ts = 0.0f;
      for (int k = lane; k < h.top; k += 64)
        if (ids[k] >= 0 && !none) ts += __builtin_amdgcn_exp2f((te[k] - tm) * kLog2e * h.inv_t);
      ts = wave_sum(ts);
      for (int k = lane; k < h.top; k += 64)
        h.q[n * h.top + k] = ids[k] >= 0 && !none ? __builtin_amdgcn_exp2f((te[k] - tm) * kLog2e * h.inv_t) / ts : 0.0f;
    }
    if (bad != 0.0f) coef = NAN;
    if (!none && coef != 0.0f) {
      const float2 st = h.stats[n];
      info = make_float2(st.x, coef * __builtin_amdgcn_exp2f(-st.y * kLog2e));
    }
  }
  if (lane == 0) h.info[n] = info;
}

// The targets' entries of dz^T: coefficient (p - q), q summed over the row's
// entries of the same class (equal entries write equal values).
template <typename T>
__global__ __launch_bounds__(256) void head_targets_kernel(HeadArgs h) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= h.rows * h.top) return;
  const int64_t n = i / h.top;
  const int64_t id = h.ids[i];
  if (id < h.v0 || id >= h.v0 + h.piece) return;
  const float2 info = h.info[n];
  if (info.y == 0.0f) return;
  float p, q;
  const float coef = h.dloss[n] * h.t;
  if (!h.teacher) {
    p = __builtin_amdgcn_exp2f(-h.loss[n] * kLog2e);
    q = 1.0f;
  } else {
    p = __builtin_amdgcn_exp2f(((h.picked[i] - info.x) * h.inv_t - h.stats[n].y) * kLog2e);
    q = 0.0f;
    for (int k = 0; k < h.top; ++k)
      if (h.ids[n * h.top + k] == id) q += h.q[n * h.top + k];
  }
  put(static_cast<T *>(h.gt) + (id - h.v0) * h.rows_pad + n, coef * (p - q));
}

// dx[n][d] = the splits' partial sums in order, 0 in rows that do not count.
template <typename T>
__global__ __launch_bounds__(256) void head_dx_kernel(HeadArgs h) {
  const int per = (h.dim + 3) / 4;
  const int64_t total = h.rows * per;
  T *dx = static_cast<T *>(h.dx);
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
    const int64_t n = i / per;
    const int d = (int)(i - n * per) * 4;
    float v[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    if (h.info[n].y != 0.0f)
      for (int s = 0; s < h.splits; ++s) {
        const float4 u = *reinterpret_cast<const float4 *>(h.dx_part + ((int64_t)s * h.rows + n) * h.dx_pad + d);
        v[0] += u.x; v[1] += u.y; v[2] += u.z; v[3] += u.w;
      }
    T *o = dx + n * h.dx_ld + d;
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (d + j < h.dim) put(o + j, v[j]);
  }
}

// dbias of 256 classes a block: the row parts' sums of coefficient p in order,
// less the targets' coefficient q.  The block goes through all targets, 256 a
// round, and keeps those of its classes in a list in their order; each thread
// then takes its own class's entries from it.
__global__ __launch_bounds__(256) void head_dbias_kernel(HeadArgs h) {
  __shared__ int cnt[4];
  __shared__ int list_c[256];
  __shared__ float list_v[256];
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
  const int64_t c0 = (int64_t)blockIdx.x * 256;
  const int64_t cls = c0 + t;
  float sum = 0.0f;
  if (cls < h.classes)
    for (int p = 0; p < h.db_parts; ++p) sum += h.db_part[(int64_t)p * h.classes + cls];
  const int64_t total = h.rows * h.top;
  float less = 0.0f;
  for (int64_t i0 = 0; i0 < total; i0 += 256) {
    const int64_t i = i0 + t;
    const int64_t id = i < total ? h.ids[i] : -1;
    const bool hit = id >= c0 && id < c0 + 256;
    const uint64_t mask = __ballot(hit);
    if (lane == 0) cnt[wave] = __popcll(mask);
    __syncthreads();
    int base = 0, n = 0;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      if (w < wave) base += cnt[w];
      n += cnt[w];
    }
    if (n > 0) {
      if (hit) {
        const int at = base + __popcll(mask & ((1ull << lane) - 1));
        const int64_t n1 = i / h.top;
        const float coef = h.info[n1].y != 0.0f ? h.dloss[n1] * h.t : 0.0f;
        list_c[at] = (int)(id - c0);
        list_v[at] = h.teacher ? coef * h.q[i] : coef;
      }
      __syncthreads();
      for (int k = 0; k < n; ++k)
        if (list_c[k] == t) less += list_v[k];
    }
    __syncthreads();
  }
  if (cls < h.classes) h.dbias[cls] = sum - less;
}

int grid_for(int64_t n, int per) {
  const int64_t b = (n + per - 1) / per;
  return (int)(b < 1 ? 1 : b > 16384 ? 16384 : b);
}

// Rows at which the row side of a tile is 128 wide; below, 32.
constexpr int kWideRows = 64;
bool big_rows(int64_t rows) { return rows > 512; }

template <typename T>
hipError_t forward(const HeadArgs &a, hipStream_t s) {
  Gemm g{};
  g.a = a.w; g.a_ld = a.w_ld; g.a_ext = (int)a.classes;
  g.b = a.x; g.b_ld = a.x_ld; g.b_ext = (int)a.rows;
  g.k_ext = a.dim; g.splits = 1;
  if (big_rows(a.rows)) return launch_big<T, false, false, E_STATS>(g, a, s);
  if (a.rows > kWideRows) return launch_gemm<T, 128, 128, 2, 2, 3, false, false, E_STATS>(g, a, s);
  return launch_gemm<T, 128, 32, 4, 1, 4, false, false, E_STATS>(g, a, s);
}
template <typename T>
hipError_t dlogits(const HeadArgs &a, hipStream_t s) {
  Gemm g{};
  g.a = a.x; g.a_ld = a.x_ld; g.a_ext = (int)a.rows;
  g.b = static_cast<const T *>(a.w) + a.v0 * a.w_ld; g.b_ld = a.w_ld; g.b_ext = (int)a.piece;
  g.k_ext = a.dim; g.splits = 1;
  const hipError_t e = big_rows(a.rows) ? launch_big<T, false, false, E_DLOGITS>(g, a, s) :
                       a.rows > kWideRows ? launch_gemm<T, 128, 128, 2, 2, 3, false, false, E_DLOGITS>(g, a, s)
                                          : launch_gemm<T, 32, 128, 1, 4, 4, false, false, E_DLOGITS>(g, a, s);
  if (e != hipSuccess || a.rows == 0) return e;
  hapi_launch(head_targets_kernel<T>, dim3((uint32_t)((a.rows * a.top + 255) / 256)), dim3(256), 0, s, a);
  return hipGetLastError();
}
template <typename T>
hipError_t grads(const HeadArgs &a, hipStream_t s) {
  Gemm g{};
  g.a = static_cast<const T *>(a.w) + a.v0 * a.w_ld; g.a_ld = a.w_ld; g.a_ext = a.dx_pad;
  g.b = a.gt; g.b_ld = a.rows_pad; g.b_ext = (int)a.rows;
  g.k_ext = (int)a.piece; g.splits = a.splits;
  hipError_t e = big_rows(a.rows)  ? launch_big<T, true, true, E_DX>(g, a, s)
                 : a.rows > kWideRows ? launch_gemm<T, 128, 128, 2, 2, 3, true, true, E_DX>(g, a, s)
                                    : launch_gemm<T, 128, 32, 4, 1, 4, true, true, E_DX>(g, a, s);
  if (e != hipSuccess) return e;
  g.a = a.x; g.a_ld = a.x_ld; g.a_ext = a.dx_pad;
  g.b = a.gt; g.b_ld = a.rows_pad; g.b_ext = (int)a.piece;
  g.k_ext = (int)a.rows; g.splits = 1;
  if (big_rows(a.rows)) return launch_big<T, true, false, E_DW>(g, a, s);
  return launch_gemm<T, 128, 128, 2, 2, 3, true, false, E_DW>(g, a, s);
}

}  // namespace

int head_parts(bool, int64_t rows, int64_t classes) {
  if (big_rows(rows)) return (int)((classes + 255) / 256) * 4;
  return (int)((classes + 127) / 128) * (rows > kWideRows ? 2 : 4);
}
int head_db_parts(bool, int64_t rows) {
  if (big_rows(rows)) return (int)((rows + 255) / 256) * 4;
  return rows > kWideRows ? (int)((rows + 127) / 128) * 2 : (int)((rows + 31) / 32);
}
int head_splits(bool, int64_t rows, int dim, int64_t piece) {
  const int64_t br = big_rows(rows) ? 256 : rows > kWideRows ? 128 : 32, ba = big_rows(rows) ? 256 : 128;
  const int64_t tiles = ((rows + br - 1) / br) * ((dim + ba - 1) / ba);
  if (tiles == 0) return 1;
  int64_t s = (512 + tiles - 1) / tiles;           // two workgroups a CU
  const int64_t most = (piece + 511) / 512;        // at least 512 classes each
  s = s < most ? s : most;
  return (int)(s < 1 ? 1 : s);
}

hipError_t launch_head_stage(bool bf16, const void *in, int64_t ld_in, void *out, int64_t ld_out, int64_t rows, int dim,
                             hipStream_t s) {
  if (rows == 0) return hipSuccess;
  const int64_t n = rows * ld_out * (bf16 ? 2 : 4) / 16;
  if (bf16)
    hapi_launch(stage_kernel<uint16_t>, dim3(grid_for(n, 256)), dim3(256), 0, s, (const uint16_t *)in, ld_in,
                (uint16_t *)out, ld_out, rows, dim, (const float2 *)nullptr);
  else
    hapi_launch(stage_kernel<float>, dim3(grid_for(n, 256)), dim3(256), 0, s, (const float *)in, ld_in, (float *)out,
                ld_out, rows, dim, (const float2 *)nullptr);
  return hipGetLastError();
}

hipError_t launch_head_forward(bool bf16, const HeadArgs &a, hipStream_t s) {
  return bf16 ? forward<uint16_t>(a, s) : forward<float>(a, s);
}

hipError_t launch_head_finish(bool bf16, const HeadArgs &a, hipStream_t s) {
  if (a.rows == 0) return hipSuccess;
  const dim3 grid((uint32_t)((a.rows + kFinishRows - 1) / kFinishRows));
  if (bf16) hapi_launch(head_finish_kernel<uint16_t>, grid, dim3(1024), 0, s, a);
  else hapi_launch(head_finish_kernel<float>, grid, dim3(1024), 0, s, a);
  return hipGetLastError();
}

hipError_t launch_head_prepare(bool bf16, const HeadArgs &a, void *xs, int64_t xs_ld, hipStream_t s) {
  if (a.rows == 0) return hipSuccess;
  hapi_launch(head_info_kernel, dim3((uint32_t)((a.rows_pad + 3) / 4)), dim3(256), 0, s, a);
  const int64_t n = a.rows * xs_ld * (bf16 ? 2 : 4) / 16;
  if (bf16)
    hapi_launch(stage_kernel<uint16_t>, dim3(grid_for(n, 256)), dim3(256), 0, s, (const uint16_t *)a.x_in, a.x_in_ld,
                (uint16_t *)xs, xs_ld, a.rows, a.dim, (const float2 *)a.info);
  else
    hapi_launch(stage_kernel<float>, dim3(grid_for(n, 256)), dim3(256), 0, s, (const float *)a.x_in, a.x_in_ld,
                (float *)xs, xs_ld, a.rows, a.dim, (const float2 *)a.info);
  return hipGetLastError();
}

hipError_t launch_head_dlogits(bool bf16, const HeadArgs &a, hipStream_t s) {
  return bf16 ? dlogits<uint16_t>(a, s) : dlogits<float>(a, s);
}

hipError_t launch_head_grads(bool bf16, const HeadArgs &a, hipStream_t s) {
  return bf16 ? grads<uint16_t>(a, s) : grads<float>(a, s);
}

hipError_t launch_head_reduce(bool bf16, const HeadArgs &a, hipStream_t s) {
  if (a.rows > 0) {
    const int64_t n = a.rows * ((a.dim + 3) / 4);
    if (bf16) hapi_launch(head_dx_kernel<uint16_t>, dim3(grid_for(n, 256)), dim3(256), 0, s, a);
    else hapi_launch(head_dx_kernel<float>, dim3(grid_for(n, 256)), dim3(256), 0, s, a);
  }
  if (a.dbias) hapi_launch(head_dbias_kernel, dim3((uint32_t)((a.classes + 255) / 256)), dim3(256), 0, s, a);
  return hipGetLastError();
}

}  // namespace hapi
