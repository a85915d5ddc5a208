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
//              g exp(z - m) / sum less the target's entry, stored transposed, one
//              piece of the classes at a time: a lane owns a class, so the bias's
//              gradient is a sum of its own registers, joined over the rows in 64
//              bits.  A teacher's entries are put in by a small kernel of their own.
//   dx         a = feature, b = row, k = class: dz^T and the weights as they lie,
//              the piece's classes split over workgroups, float32 partial sums.
//   dW         a = feature, b = class, k = row: dz^T and x as they lie; one launch
//              with dx.
//
// float32 uses v_mfma_f32_32x32x2_f32 in the same tiles (128 bytes of k).
// dz is rounded to the operands' type before its two products (the matrix
// cores' bf16 operands; 2^-8 of each entry at most, against 2^-8 of the
// outputs' own rounding); sums, softmax statistics and the bias's gradient are
// float32 or wider throughout.  Up to 32 rows (FEW), where one row's rounding can be
// all of a gradient's, bf16 dz is a sum of two, the second one what the first leaves:
// columns 32 .. 63 of dz^T, further 32 rows to dx's product and further 32 k to dW's,
// whose k-tile holds 64 (a step of 32 x 2048 x 1000 33.5 -> 35.6 us, of 16 x 1024 x
// 32000 81.5 -> 82.5, of 8 x 4096 x 131072 no longer; one row's dW off by 2.6e-4 of its
// length, not 3.8e-4).
//
// Four products of 2 N D V operations in a step, one more than with the logits kept,
// which would be 2 or 4 bytes a logit, written once and read twice.  Bound by the
// matrix pipes: at 8192 x 2048 x 131072 they are busy 78% of the forward product's
// time, 69% of dz's and 76% of the gradients' (their clock, under this load 1.6 to
// 1.9 GHz, included in neither); the k-loop of a 256 x 256 tile takes 2.08k cycles a
// k-tile, its MFMAs 2048.
#include <algorithm>
#include <type_traits>

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

// Tile `tile` of the grid: panels of 8 tiles of its smaller side, each along the whole
// larger one, so that the 32 workgroups an XCD runs at once are 8 x 4 tiles and
// share their operands' k-tiles in its L2 (8192 x 2048 x 131072 forward, one panel
// of all 32: half the L2's requests miss, in panels 19%; the step 14.15 -> 13.79 ms).
__device__ __forceinline__ void place_tile(const Gemm &g, int tile, int &ta, int &tb) {
  const bool a_small = g.tiles_a <= g.tiles_b;
  const int few = a_small ? g.tiles_a : g.tiles_b, many = a_small ? g.tiles_b : g.tiles_a;
  const int p = (int)((uint32_t)tile / (uint32_t)(8 * many));
  const int w = few - 8 * p < 8 ? few - 8 * p : 8;
  const int i = tile - p * 8 * many, m = (int)((uint32_t)i / (uint32_t)w), f = 8 * p + i - m * w;
  ta = a_small ? f : m;
  tb = a_small ? m : f;
}

// What rounding v to bf16 leaves of it (0 where it rounds to inf or NaN).
__device__ __forceinline__ float bf16_rest(float v) {
  const float r = bf2f(f2bf(v));
  return fabsf(r) < INFINITY ? v - r : 0.0f;
}

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
  static constexpr int BYTES = R * 128;
  static constexpr int LOADS = BYTES / 1024 / WAVES;  // DMAs of 1 KB a wave issues per k-tile
  static_assert(LOADS * 1024 * WAVES == BYTES, "whole DMAs per wave");
  static constexpr int KSTEPS = 4;             // MFMA k-steps of a k-tile
  static constexpr int CPR = KR ? R / V : 8;      // 16-byte slots of an LDS row (a power of two)
  static constexpr int RPD = 64 / CPR;            // LDS rows of one DMA
  static_assert(CPR <= 64, "a DMA covers whole LDS rows");

  uint32_t off[LOADS];  // byte offset of this lane from the k-tile's base
  int lk[LOADS];        // this lane's k within the k-tile

  static __device__ __forceinline__ int swz(int row) {
    if constexpr (!KR) return (row >> 1) & 7;
    // 16-bit reads take 32 bytes of each of 4 rows
    if constexpr (KR && sizeof(T) == 2 && CPR >= 16) return 4 * (row & 3);
    if constexpr (KR && sizeof(T) == 2 && CPR == 8) return 4 * ((row >> 1) & 1);
    return 0;
  }
  // r0: the tile's first row (its offset is in the base).  half 0 or 1: the operand's
  // rows are every other 32 of the tile's, starting with that one; -1: all of them.
  __device__ __forceinline__ void init(int r0, int ext, int64_t ld, int wave, int lane, int half = -1) {
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
      const int lr = (wave * LOADS + i) * RPD + lane / CPR;  // LDS row
      const int c = (lane % CPR) ^ swz(lr);                  // 16-byte slot of the memory row
      int r = KR ? c * V : lr;
      if (half >= 0) r = (r >> 5) * 64 + 32 * half + (r & 31);
      lk[i] = KR ? lr : c * V;
      const uint32_t o = KR ? (uint32_t)lr * (uint32_t)ld + r : (uint32_t)r * (uint32_t)ld + c * V;  // < 2^31 bytes
      off[i] = r0 + r < ext ? o * (uint32_t)sizeof(T) : kOob;
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

// What the epilogue needs of the tile's reg side, in LDS.  Forward: the bias of
// its classes, -inf past the last one.  dz: its rows' largest logit and scale, and
// for cross entropy the target class (in the piece; far off if none) and the
// coefficient to take off there, both over the coefficients' unit.
template <int EPI, int BA>
struct SideTable {
  static constexpr int N = EPI == E_STATS || EPI == E_DLOGITS ? BA : 4;
  float m[N];
  float scale[EPI == E_DLOGITS ? BA : 4], coef[EPI == E_DLOGITS ? BA : 4];
  int target[EPI == E_DLOGITS ? BA : 4];
  template <int THREADS>
  __device__ __forceinline__ void load(const Gemm &g, const HeadArgs &h, int a0, int t) {
    if constexpr (EPI == E_STATS)
      for (int i = t; i < BA; i += THREADS) m[i] = a0 + i < g.a_ext ? (h.bias ? h.bias[a0 + i] : 0.0f) : -INFINITY;
    if constexpr (EPI == E_DLOGITS)
      for (int i = t; i < BA; i += THREADS) {
        const int n = a0 + i;
        const float unit = *h.unit;
        const float2 in = n < h.rows_pad ? h.info[n] : make_float2(INFINITY, 0.0f);
        m[i] = in.x;
        scale[i] = in.y / unit;
        if (!h.teacher) {
          const int id = n < h.rows ? h.id32[n] : -1;
          target[i] = id >= 0 ? id - (int)h.v0 : INT32_MIN / 2;
          coef[i] = n < h.rows ? h.cq[n] / unit : 0.0f;
        }
      }
  }
};

// Where a wave's blocks lie: block (i, j) is out[lane(j) + lane % 32][reg(i) + 8 q +
// 4 lh + e] = acc[i][j][4 q + e]; part: which of the reg side's parts the wave holds.
template <int LANE_A, int LANE_B>
struct Place {
  int a0, r0, l0, part;
  __device__ __forceinline__ int reg(int i) const { return r0 + 32 * i; }
  __device__ __forceinline__ int lane(int j) const { return l0 + (j >> 1) * LANE_B + (j & 1) * LANE_A; }
};

// A wave's 32 output rows of L values of type O (a lane's 16 of each block of 32), turned
// in its part of LDS so that a store writes whole rows: put(b, q, v) takes values
// 8 q + 4 lh .. + 3 of block b of the lane's row; rows(f) calls f(row, column, 16
// bytes) with consecutive lanes on consecutive columns.  Stores of the lanes' own
// values would write 32 bytes of 32 rows each, and the L2 takes a request for every
// such piece (dz of 8192 x 2048 x 16384: 525 us, turned 479).
template <typename O, int L>
struct RowsOut {
  static constexpr int PITCH = L * (int)sizeof(O) + 16, V = 16 / (int)sizeof(O), PER = L / V, RPS = 64 / PER;
  static constexpr int BYTES = 32 * PITCH;
  uint8_t *p;
  int lane;
  __device__ __forceinline__ void put(int b, int q, float v0, float v1, float v2, float v3) const {
    uint8_t *d = p + (lane & 31) * PITCH + (32 * b + 8 * q + 4 * (lane >> 5)) * (int)sizeof(O);
    if constexpr (sizeof(O) == 2) *reinterpret_cast<uint2 *>(d) = make_uint2(f2bf2(v0, v1), f2bf2(v2, v3));
    else *reinterpret_cast<float4 *>(d) = make_float4(v0, v1, v2, v3);
  }
  template <typename F>
  __device__ __forceinline__ void rows(F &&f) const {
#pragma unroll
    for (int s = 0; s < 32 / RPS; ++s) {
      const int row = s * RPS + lane / PER, c = lane % PER;
      f(row, c * V, *reinterpret_cast<const uint4 *>(p + row * PITCH + c * 16));
    }
  }
};

// REGS: values of the tile's reg side.
template <typename T, int EPI, int REGS, int TA, int TB, typename P, typename S>
__device__ __forceinline__ void epilogue(const Gemm &g, const HeadArgs &h, f32x16_t (&acc)[TA][TB], const P &at,
                                         const S &side, uint8_t *turn, int split, int lane) {
  const int lh = lane >> 5;
  if constexpr (EPI == E_STATS) {
    const float c = kLog2e * h.inv_t;
    float m[TB], s[TB];
#pragma unroll
    for (int j = 0; j < TB; ++j) m[j] = -INFINITY, s[j] = 0.0f;
    if (h.bias || at.reg(TA) > g.a_ext) {  // else the table holds zeros
#pragma unroll
      for (int i = 0; i < TA; ++i)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const f32x4_t bias = *reinterpret_cast<const f32x4_t *>(side.m + (at.reg(i) - at.a0 + 8 * q + 4 * lh));
#pragma unroll
          for (int j = 0; j < TB; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[i][j][4 * q + e] += bias[e];
        }
    }
#pragma unroll
    for (int i = 0; i < TA; ++i)
#pragma unroll
      for (int j = 0; j < TB; ++j)
#pragma unroll
        for (int r = 0; r < 16; ++r) m[j] = fmaxf(m[j], acc[i][j][r]);
#pragma unroll
    for (int j = 0; j < TB; ++j) {
      m[j] = fmaxf(m[j], __shfl_xor(m[j], 32, 64));
      const float mm = m[j] == -INFINITY ? 0.0f : m[j];  // no class with weight: the sum is 0, not NaN
#pragma unroll
      for (int i = 0; i < TA; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r) s[j] += __builtin_amdgcn_exp2f((acc[i][j][r] - mm) * c);
      s[j] += __shfl_xor(s[j], 32, 64);
      const int row = at.lane(j) + (lane & 31);
      if (lh == 0 && row < g.b_ext && at.part < h.parts) h.part[(int64_t)at.part * h.rows + row] = make_float2(m[j], s[j]);
    }
  }
  if constexpr (EPI == E_DLOGITS) {
    T *gt = static_cast<T *>(h.gt);
    const float c = kLog2e * h.inv_t;
    const RowsOut<T, 32 * TA> out{turn, lane};
    constexpr bool kPair = sizeof(T) == 2 && REGS == 32;  // tiles that few rows may take
#pragma unroll
    for (int j = 0; j < TB; ++j) {
      const int cls = at.lane(j) + (lane & 31);  // in the piece
      if (h.bias) {
        const float bias = cls < g.b_ext ? h.bias[h.v0 + cls] : 0.0f;
#pragma unroll
        for (int i = 0; i < TA; ++i)
#pragma unroll
          for (int r = 0; r < 16; ++r) acc[i][j][r] += bias;
      }
      float sum = 0.0f;
#pragma unroll
      for (int i = 0; i < TA; ++i) {
        const int loc = at.reg(i) - at.a0;
        // a row's target lies in few of the blocks: the others compare nothing
        const int tg = h.teacher ? INT32_MIN / 2 : side.target[loc + (lane & 31)];
        const bool hit = __ballot((unsigned)(tg - at.lane(j)) < 32u) != 0;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const int n = loc + 8 * q + 4 * lh;
          const f32x4_t m = *reinterpret_cast<const f32x4_t *>(side.m + n);
          const f32x4_t sc = *reinterpret_cast<const f32x4_t *>(side.scale + n);
          float v[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) v[e] = __builtin_amdgcn_exp2f((acc[i][j][4 * q + e] - m[e]) * c) * sc[e];
          if (hit) {
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] -= side.target[n + e] == cls ? side.coef[n + e] : 0.0f;
          }
          if (h.db_part) sum += (v[0] + v[1]) + (v[2] + v[3]);
          out.put(i, q, v[0], v[1], v[2], v[3]);
          if constexpr (kPair)
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[i][j][4 * q + e] = bf16_rest(v[e]);
        }
      }
      auto store = [&](int to) {
        out.rows([&](int row, int col, const uint4 &v) {
          const int r = at.lane(j) + row, n = at.reg(0) + col + to;
          if (r < g.b_ext && n < h.rows_pad) *reinterpret_cast<uint4 *>(gt + (int64_t)r * h.rows_pad + n) = v;
        });
      };
      store(0);
      if constexpr (kPair)
        if (h.rows <= kFewRows) {
#pragma unroll
          for (int q = 0; q < 4; ++q)
            out.put(0, q, acc[0][j][4 * q], acc[0][j][4 * q + 1], acc[0][j][4 * q + 2], acc[0][j][4 * q + 3]);
          store(kFewRows);
        }
      if (h.db_part) {
        sum += __shfl_xor(sum, 32, 64);
        if (lh == 0 && cls < g.b_ext && at.part < h.db_parts) h.db_part[(int64_t)at.part * h.classes + h.v0 + cls] = sum;
      }
    }
  }
  if constexpr (EPI == E_DX || EPI == E_DW) {
    // out[row][feature], whole or as one of the float32 partial sums of a split k
    const bool whole = EPI == E_DX ? h.dx_whole : h.w_splits == 1;
    if (!whole) {
      float *o = EPI == E_DX ? h.dx_part + (int64_t)split * h.rows * h.dx_pad
                             : h.dw_part + (int64_t)split * h.piece * h.dx_pad;
      const bool add = EPI == E_DX && !h.first;
      const RowsOut<float, 32 * TA> out{turn, lane};
#pragma unroll
      for (int j = 0; j < TB; ++j) {
#pragma unroll
        for (int i = 0; i < TA; ++i)
#pragma unroll
          for (int q = 0; q < 4; ++q)
            out.put(i, q, acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]);
        out.rows([&](int row, int col, const uint4 &v) {
          const int r = at.lane(j) + row, d = at.reg(0) + col;
          if (r >= g.b_ext || d >= h.dx_pad) return;
          float4 *p = reinterpret_cast<float4 *>(o + (int64_t)r * h.dx_pad + d);
          float4 w = make_float4(__uint_as_float(v.x), __uint_as_float(v.y), __uint_as_float(v.z), __uint_as_float(v.w));
          if (add) {
            const float4 u = *p;
            w.x += u.x; w.y += u.y; w.z += u.z; w.w += u.w;
          }
          *p = w;
        });
      }
      return;
    }
    constexpr int V = 16 / (int)sizeof(T);
    T *o = EPI == E_DX ? static_cast<T *>(h.dx) : static_cast<T *>(h.dw) + h.v0 * h.dw_ld;
    const int64_t ld = EPI == E_DX ? h.dx_ld : h.dw_ld;
    const bool vec = ld % V == 0 && (uintptr_t)o % 16 == 0;
    const float unit = h.rows > 0 ? *h.unit : 0.0f;
    const RowsOut<T, 32 * TA> out{turn, lane};
#pragma unroll
    for (int j = 0; j < TB; ++j) {
      bool none = false;  // a row that does not count: zeros, whatever the weights hold
      if constexpr (EPI == E_DX) {
        const int r = at.lane(j) + (lane & 31);
        none = r >= g.b_ext || h.info[r].y == 0.0f;
      }
#pragma unroll
      for (int i = 0; i < TA; ++i)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          float v[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) v[e] = EPI == E_DX && none ? 0.0f : acc[i][j][4 * q + e] * unit;
          out.put(i, q, v[0], v[1], v[2], v[3]);
        }
      out.rows([&](int row, int col, const uint4 &v) {
        const int r = at.lane(j) + row, d = at.reg(0) + col;
        if (r >= g.b_ext) return;
        T *p = o + (int64_t)r * ld + d;
        if (vec && d + V <= h.dim) {
          *reinterpret_cast<uint4 *>(p) = v;
        } else {
          T w[V];
          __builtin_memcpy(w, &v, 16);
#pragma unroll
          for (int e = 0; e < V; ++e)
            if (d + e < h.dim) p[e] = w[e];
        }
      });
    }
  }
}

// A tile of BA x BB on WA x WB waves.  Two or three stages leave room for more
// workgroups on a CU, whose waves cover each other's waits: 128 x 128 in two stages,
// two workgroups, 302 us for the forward product of 4096 x 768 x 32000; in three
// stages, one workgroup, 371; all of a k-tile's fragments read ahead 486.
// FOLD: B's second 32 rows are what the first ones leave of their values; the sums of
// the two are one.
template <typename T, int BA, int BB, int WA, int WB, int ST, bool KRA, bool KRB, int EPI, bool FOLD = false>
struct RingTile {
  static constexpr int THREADS = 64 * WA * WB, TILE_A = BA, TILE_B = BB;
  static constexpr int SMEM = ST * (BA + BB) * 128;
  typedef SideTable<EPI, BA> Sides;
  static_assert(RowsOut<float, BA / WA>::BYTES * WA * WB <= SMEM, "the epilogue's rows fit the ring");
  // One barrier a k-tile, ST stages of LDS.
  static __device__ __forceinline__ void run(const Gemm &g, const HeadArgs &h, uint8_t *smem, Sides &side, int bid) {
  constexpr int WAVES = WA * WB, TA = BA / WA / 32, TB = BB / WB / 32;
  typedef Side<T, BA, KRA, WAVES> SA;
  typedef Side<T, BB, KRB, WAVES> SB;
  constexpr int STAGE = SA::BYTES + SB::BYTES;

  const int t = threadIdx.x, lane = t & 63;
  const int wave = __builtin_amdgcn_readfirstlane(t >> 6);
  const int wa = wave / WB, wb = wave % WB;
  constexpr bool SPLIT = EPI == E_DX || EPI == E_DW;  // k over several workgroups
  const uint32_t tiles = g.tiles_a * g.tiles_b;
  const int split = SPLIT ? (int)((uint32_t)bid / tiles) : 0, tile = bid - split * (int)tiles;
  int ta, tb;
  place_tile(g, tile, ta, tb);
  const int a0 = ta * BA, b0 = tb * BB;
  const int nkt = (g.k_ext + SA::KT - 1) / SA::KT;
  const int kt0 = SPLIT ? (int)((uint32_t)(nkt * split) / (uint32_t)g.splits) : 0;
  const int kt1 = SPLIT ? (int)((uint32_t)(nkt * (split + 1)) / (uint32_t)g.splits) : nkt;
  const int nk = kt1 - kt0;

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
  side.template load<THREADS>(g, h, a0, t);  // behind the DMAs: their latencies overlap
  constexpr int PER = SA::LOADS + SB::LOADS;
  for (int kt = 0; kt < nk; ++kt) {
    // this wave's part of the k-tile has landed and its reads of the last one
    // are done; after the barrier, everyone's
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"((ST - 2) * PER) : "memory");
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
    const uint8_t *at = smem + (kt % ST) * STAGE, *bt = at + SA::BYTES;
    // Fragments ahead of the MFMAs: a whole k-tile's where a wave has one block
    // (nothing else covers the LDS's latency), else one k-step's.
    constexpr int AHEAD = TA * TB == 1 ? SA::KSTEPS : 1, BUFS = AHEAD == 1 ? 2 : AHEAD;
    typename Elem<T>::Frag fa[BUFS][TA], fb[BUFS][TB];
    auto read = [&](int ks) {
#pragma unroll
      for (int i = 0; i < TA; ++i) fa[ks % BUFS][i] = SA::frag(at, (wa * TA + i) * 32, ks, lane);
#pragma unroll
      for (int j = 0; j < TB; ++j) fb[ks % BUFS][j] = SB::frag(bt, (wb * TB + j) * 32, ks, lane);
    };
#pragma unroll
    for (int ks = 0; ks < AHEAD; ++ks) read(ks);
    __builtin_amdgcn_sched_barrier(0);
    issue();
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int ks = 0; ks < SA::KSTEPS; ++ks) {
      if (AHEAD == 1 && ks + 1 < SA::KSTEPS) read(ks + 1);
      if (AHEAD == 1) __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int i = 0; i < TA; ++i)
#pragma unroll
        for (int j = 0; j < TB; ++j) acc[i][j] = mma(fa[ks % BUFS][i], fb[ks % BUFS][j], acc[i][j]);
      if (AHEAD == 1) __builtin_amdgcn_sched_barrier(0);
    }
  }
  // No DMA may outlive the workgroup's LDS, and the side table is read by all waves.
  asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
  __syncthreads();

  const Place<32, 64> at = {a0, a0 + wa * TA * 32, b0 + wb * TB * 32, ta * WA + wa};
  uint8_t *turn = smem + wave * (SMEM / WAVES);
  if constexpr (FOLD) {
    static_assert(BB == 64 && WB == 1, "a wave has both halves");
    f32x16_t sum[TA][1];
#pragma unroll
    for (int i = 0; i < TA; ++i)
#pragma unroll
      for (int r = 0; r < 16; ++r) sum[i][0][r] = acc[i][0][r] + acc[i][1][r];
    Gemm one = g;
    one.b_ext = (int)h.rows;
    epilogue<T, EPI, BA>(one, h, sum, at, side, turn, split, lane);
  } else {
    epilogue<T, EPI, BA>(g, h, acc, at, side, turn, split, lane);
  }
  }
};

// 32 x 32 tiles for the smallest calls, the k-steps of a k-tile on four waves, whose
// sums the first one adds up in order.  A k-tile costs a workgroup its DMAs, LDS
// reads and MFMAs one after the other (0.25 us with one wave, 0.27 us with four
// waves on a 64 x 64 tile); four waves on one tile have a quarter of each.
template <typename T, int ST, int EPI>
struct TinyTile {
  static constexpr int THREADS = 256, TILE_A = 32, TILE_B = 32;
  typedef Side<T, 32, false, 4> S;
  static constexpr int STAGE = 2 * S::BYTES, SMEM = ST * STAGE;
  static_assert(S::KSTEPS == 4 && S::LOADS == 1, "a k-step and a DMA of each operand to a wave");
  static_assert(SMEM >= 3 * 4096 + RowsOut<float, 32>::BYTES, "the sums and the epilogue's rows fit the ring");
  typedef SideTable<EPI, 32> Sides;
  static __device__ __forceinline__ void run(const Gemm &g, const HeadArgs &h, uint8_t *smem, Sides &side, int bid) {
    const int t = threadIdx.x, lane = t & 63;
    const int wave = __builtin_amdgcn_readfirstlane(t >> 6);
    const int ta = bid % g.tiles_a, tb = bid / g.tiles_a;
    const int a0 = ta * 32, b0 = tb * 32;
    const int nk = (g.k_ext + S::KT - 1) / S::KT;
    S sa, sb;
    sa.init(a0, g.a_ext, g.a_ld, wave, lane);
    sb.init(b0, g.b_ext, g.b_ld, wave, lane);
    const uint8_t *pa = static_cast<const uint8_t *>(g.a) + S::row_base(a0, g.a_ld);
    const uint8_t *pb = static_cast<const uint8_t *>(g.b) + S::row_base(b0, g.b_ld);
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t *)smem;
    int issued = 0;
    auto issue = [&] {  // past the last k-tile: nothing read
      const uint32_t dst = lds0 + (uint32_t)(issued % ST) * STAGE;
      const int left = issued < nk ? g.k_ext - issued * S::KT : 0;
      const int64_t o = issued < nk ? (int64_t)issued * 128 : 0;
      sa.issue(pa + o, dst, left, wave);
      sb.issue(pb + o, dst + S::BYTES, left, wave);
      ++issued;
    };
    f32x16_t acc[1][1];
#pragma unroll
    for (int r = 0; r < 16; ++r) acc[0][0][r] = 0.0f;
#pragma unroll
    for (int s = 0; s < ST - 1; ++s) issue();
    side.template load<THREADS>(g, h, a0, t);
    for (int kt = 0; kt < nk; ++kt) {
      asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"((ST - 2) * 2) : "memory");
      __builtin_amdgcn_sched_barrier(0);
      __builtin_amdgcn_s_barrier();
      asm volatile("" ::: "memory");
      __builtin_amdgcn_sched_barrier(0);
      const uint8_t *at = smem + (kt % ST) * STAGE;
      const typename Elem<T>::Frag fa = S::frag(at, 0, wave, lane), fb = S::frag(at + S::BYTES, 0, wave, lane);
      __builtin_amdgcn_sched_barrier(0);
      issue();
      __builtin_amdgcn_sched_barrier(0);
      acc[0][0] = mma(fa, fb, acc[0][0]);
    }
    // No DMA may outlive the workgroup's LDS, or write to it when it holds the sums.
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
    __syncthreads();
    float *part = reinterpret_cast<float *>(smem);
    if (wave > 0)
#pragma unroll
      for (int r = 0; r < 16; ++r) part[((wave - 1) * 16 + r) * 64 + lane] = acc[0][0][r];
    __syncthreads();
    if (wave > 0) return;
#pragma unroll
    for (int w = 0; w < 3; ++w)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[0][0][r] += part[(w * 16 + r) * 64 + lane];
    const Place<32, 64> at = {a0, a0, b0, ta};
    epilogue<T, EPI, 32>(g, h, acc, at, side, smem + 3 * 4096, 0, lane);
  }
};

// The same product on 256 x 256 tiles.  Eight waves, two per SIMD: wave (g, c)
// owns rows 64 g .. + 63 of both 128-row halves of B and rows 64 c .. + 63 of A, 32 in
// each of its halves (which take every other 32 rows), 128 accumulator registers.  A
// k-tile is two steps, each a memory slot (fragments of the next 16 MFMAs out of LDS,
// DMAs of a later k-tile into it) and a matrix slot, with a barrier after every slot;
// the two groups g run one slot apart, so one group's MFMAs cover the other's LDS
// reads.  Two stages of 64 KB; half a stage is loaded again as soon as both groups
// have read it.
// Not faster: workgroups that stay and take the next tile with its loads in flight
// during the epilogue (4096 x 768 x 32000: forward 212 us against 216, gradients 395
// against 372); 128 x 256 tiles, two workgroups to a CU (forward 320 us and more).
template <typename T, bool KRA, bool KRB, int EPI>
struct BigTile {
  static constexpr int THREADS = 512, TILE_A = 256, TILE_B = 256;
  static constexpr int SMEM = 2 * 512 * 128;
  typedef SideTable<EPI, 256> Sides;
  static __device__ __forceinline__ void run(const Gemm &g, const HeadArgs &h, uint8_t *smem, Sides &side, int bid) {
  typedef Side<T, 128, KRA, 8> SA;
  typedef Side<T, 128, KRB, 8> SB;
  constexpr int HALF = SA::BYTES, STAGE = 4 * HALF;  // B halves 0, 1, A halves 0, 1
  typedef typename Elem<T>::Frag Frag;
  const int t = threadIdx.x, lane = t & 63;
  const int wave = __builtin_amdgcn_readfirstlane(t >> 6);
  const int wm = wave >> 2, wn = wave & 3;
  constexpr bool SPLIT = EPI == E_DX || EPI == E_DW;  // k over several workgroups
  const uint32_t tiles = g.tiles_a * g.tiles_b;
  const int split = SPLIT ? (int)((uint32_t)bid / tiles) : 0, tile = bid - split * (int)tiles;
  int ta, tb;
  place_tile(g, tile, ta, tb);
  const int a0 = ta * 256, b0 = tb * 256;
  const int nkt = (g.k_ext + SA::KT - 1) / SA::KT;
  const int kt0 = SPLIT ? (int)((uint32_t)(nkt * split) / (uint32_t)g.splits) : 0;
  const int kt1 = SPLIT ? (int)((uint32_t)(nkt * (split + 1)) / (uint32_t)g.splits) : nkt;
  const int nk = kt1 - kt0;

  SA sa[2];
  SB sb[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    sa[i].init(a0, g.a_ext, g.a_ld, wave, lane, i);
    sb[i].init(b0 + 128 * i, g.b_ext, g.b_ld, wave, lane);
  }
  const int64_t da = SA::k_step(g.a_ld), db = SB::k_step(g.b_ld);
  const int64_t hb = SB::row_base(128, g.b_ld);
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
  auto issue_a = [&](uint32_t stage, int i) { sa[i].issue(pa, lds0 + stage + (2 + i) * HALF, k_left, wave); };
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
  side.template load<THREADS>(g, h, a0, t);  // behind the DMAs: their latencies overlap
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
  // The last DMAs (they read nothing) write to LDS that the epilogue uses.
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  if constexpr (EPI != E_STATS) __syncthreads();
  const Place<32, 128> at = {a0, a0 + wn * 64, b0 + wm * 64, ta * 4 + wn};
  epilogue<T, EPI, 256>(g, h, acc, at, side, smem + wave * (SMEM / 8), split, lane);
  }
};

// One product a launch.
template <typename Tile>
__global__ __launch_bounds__(Tile::THREADS) void head_product_kernel(Gemm g, HeadArgs h) {
  __shared__ __attribute__((aligned(1024))) uint8_t smem[Tile::SMEM];
  __shared__ __attribute__((aligned(16))) typename Tile::Sides side;
  Tile::run(g, h, smem, side, xcd_remap(blockIdx.x, gridDim.x));
}

// Both products of dz^T in one launch, dx's workgroups first: each fills the
// CUs that the other's last round leaves idle.
template <typename DX, typename DW>
__global__ __launch_bounds__(DX::THREADS) void head_grads_kernel(Gemm gx, Gemm gw, int nx, HeadArgs h) {
  static_assert(DX::THREADS == DW::THREADS, "one block size");
  __shared__ __attribute__((aligned(1024))) uint8_t smem[DX::SMEM > DW::SMEM ? DX::SMEM : DW::SMEM];
  const int b = blockIdx.x;
  typename DX::Sides sx;  // of no use to these epilogues
  typename DW::Sides sw;
  if (b < nx) DX::run(gx, h, smem, sx, xcd_remap(b, nx));
  else DW::run(gw, h, smem, sw, xcd_remap(b - nx, gridDim.x - nx));
}

template <typename Tile>
int64_t count_tiles(Gemm &g) {
  g.tiles_a = (g.a_ext + Tile::TILE_A - 1) / Tile::TILE_A;
  g.tiles_b = (g.b_ext + Tile::TILE_B - 1) / Tile::TILE_B;
  return (int64_t)g.tiles_a * g.tiles_b * g.splits;
}

template <typename Tile>
hipError_t launch_product(Gemm g, const HeadArgs &h, hipStream_t s) {
  const int64_t blocks = count_tiles<Tile>(g);
  if (blocks == 0) return hipSuccess;
  if (blocks > kMaxLaunchThreads / Tile::THREADS) return hipErrorInvalidValue;
  hapi_launch(head_product_kernel<Tile>, dim3((uint32_t)blocks), dim3(Tile::THREADS), 0, s, g, h);
  return hipGetLastError();
}

template <typename DX, typename DW>
hipError_t launch_grads(Gemm gx, Gemm gw, const HeadArgs &h, hipStream_t s) {
  const int64_t nx = count_tiles<DX>(gx), nw = count_tiles<DW>(gw);
  if (nx + nw > kMaxLaunchThreads / DX::THREADS) return hipErrorInvalidValue;
  hapi_launch((head_grads_kernel<DX, DW>), dim3((uint32_t)(nx + nw)), dim3(DX::THREADS), 0, s, gx, gw, (int)nx, h);
  return hipGetLastError();
}

// ------------------------------------------------------------ small kernels

__device__ __forceinline__ float to_f(uint16_t v) { return bf2f(v); }
__device__ __forceinline__ float to_f(float v) { return v; }
__device__ __forceinline__ void put(uint16_t *p, float v) { *p = f2bf(v); }
__device__ __forceinline__ void put(float *p, float v) { *p = v; }

// out[r][0 .. ld_out) = in[r][0 .. dim), zeros behind; a thread per 16 bytes.
template <typename T>
__global__ __launch_bounds__(256) void stage_kernel(const T *__restrict__ in, int64_t ld_in, T *__restrict__ out,
                                                    int64_t ld_out, int64_t rows, int dim) {
  constexpr int V = 16 / (int)sizeof(T);
  const int64_t per = ld_out / V;
  const int64_t n = rows * per;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) {
    const int64_t r = i / per;
    const int d = (int)(i - r * per) * V;
    const T *p = in + r * ld_in + d;
    T v[V] = {};
    if (d + V <= dim) {
      __builtin_memcpy(v, p, 16);
    } else {
#pragma unroll
      for (int j = 0; j < V; ++j)
        if (d + j < dim) v[j] = p[j];
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

// x . w[id] of up to K classes at once by one wave (ids < 0: 0), w's rows ld apart:
// the K rows' loads are in flight together.
template <typename T, int K>
__device__ __forceinline__ void wave_dots(const T *x, const T *w, int64_t ld, const int64_t (&id)[K], int dim, int lane,
                                          float (&s)[K]) {
  constexpr int V = 16 / (int)sizeof(T);
#pragma unroll
  for (int k = 0; k < K; ++k) s[k] = 0.0f;
  for (int d = lane * V; d < dim; d += 64 * V) {
    T a[V], b[K][V];
    if (dim >= V) {
      // the last values come with some of the ones before, which the lane there has
      const int at = d + V <= dim ? d : dim - V;
      __builtin_memcpy(a, x + at, 16);
#pragma unroll
      for (int k = 0; k < K; ++k) __builtin_memcpy(b[k], w + (id[k] < 0 ? 0 : id[k]) * ld + at, 16);
      if (at < d) {
#pragma unroll
        for (int j = 0; j < V; ++j) {
          if (at + j >= d) continue;
          a[j] = 0;
#pragma unroll
          for (int k = 0; k < K; ++k) b[k][j] = 0;
        }
      }
#pragma unroll
      for (int k = 0; k < K; ++k)
#pragma unroll
        for (int j = 0; j < V; ++j) s[k] = fmaf(to_f(a[j]), to_f(b[k][j]), s[k]);
    } else {
#pragma unroll
      for (int k = 0; k < K; ++k)
        for (int j = 0; j < dim; ++j) s[k] = fmaf(to_f(x[j]), to_f(w[(id[k] < 0 ? 0 : id[k]) * ld + j]), s[k]);
    }
  }
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1)
#pragma unroll
    for (int k = 0; k < K; ++k) s[k] += __shfl_xor(s[k], o, 64);
}

// Whether a teacher's logit beside an id is an entry.  One of NaN is, with an error in it.
__device__ __forceinline__ bool is_entry(int64_t id, float logit) { return id >= 0 && logit != -INFINITY; }

// Joins a row's partial statistics and forms its loss: R rows a block, 1024 / R
// threads on a row's parts, then 16 / R waves on the logits at its targets.
// Merging two (max, sum) pairs rescales the smaller one's sum.
template <typename T, int R>
__global__ __launch_bounds__(1024) void head_finish_kernel(HeadArgs h) {
  constexpr int SLICES = 1024 / R, W = 16 / R;
  __shared__ float2 ms[16][R];
  __shared__ float sums[16];
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
  const int64_t r0 = (int64_t)blockIdx.x * R;
  const float c = kLog2e * h.inv_t;
  const int64_t row = r0 + t % R;
  float m = -INFINITY, s = 0.0f;
  auto merge = [&](float m2, float s2) {
    const float mx = fmaxf(m, m2);
    const float mm = mx == -INFINITY ? 0.0f : mx;
    s = s * __builtin_amdgcn_exp2f((m - mm) * c) + s2 * __builtin_amdgcn_exp2f((m2 - mm) * c);
    m = mx;
  };
  if (row < h.rows)
    for (int p0 = t / R; p0 < h.parts; p0 += SLICES * 8) {  // eight parts' loads at a time
      float2 v[8];
#pragma unroll
      for (int i = 0; i < 8; ++i)
        v[i] = p0 + SLICES * i < h.parts ? h.part[(int64_t)(p0 + SLICES * i) * h.rows + row] : make_float2(-INFINITY, 0.0f);
#pragma unroll
      for (int i = 0; i < 8; ++i) merge(v[i].x, v[i].y);
    }
#pragma unroll
  for (int o = R; o <= 32; o <<= 1) {
    const float m2 = __shfl_xor(m, o, 64), s2 = __shfl_xor(s, o, 64);
    merge(m2, s2);
  }
  if (lane < R) ms[wave][lane] = make_float2(m, s);
  __syncthreads();
  // waves W r .. W r + W - 1: row r
  const int part = wave % W;
  const int64_t n = r0 + wave / W;
  const bool live = n < h.rows;
  m = ms[lane & 15][wave / W].x;
  s = ms[lane & 15][wave / W].y;
#pragma unroll
  for (int o = 1; o <= 8; o <<= 1) {
    const float m2 = __shfl_xor(m, o, 64), s2 = __shfl_xor(s, o, 64);
    merge(m2, s2);
  }
  const float l = logf(s);
  if (live && part == 0 && lane == 0) h.stats[n] = make_float2(m, l);

  const T *x = static_cast<const T *>(h.x_in) + n * h.x_in_ld;
  const T *w = static_cast<const T *>(h.w_in);
  if (!h.teacher) {
    if (!live || part > 0) return;
    const int64_t id = h.ids[n];
    float loss = 0.0f;
    if (id >= h.classes) {
      loss = NAN;
    } else if (id >= 0) {
      const int64_t one[1] = {id};
      float z[1];
      wave_dots<T, 1>(x, w, h.w_in_ld, one, h.dim, lane, z);
      if (h.bias) z[0] += h.bias[id];
      loss = (m - z[0]) + l;
    }
    if (lane == 0) h.loss[n] = loss;
    return;
  }
  // q = softmax(teacher / T) over the entries that count
  const int64_t *ids = h.ids + n * h.top;
  const float *te = h.teacher + n * h.top;
  float tm = -INFINITY, bad = 0.0f, loss = 0.0f;
  if (live) {
    for (int k = lane; k < h.top; k += 64)
      if (is_entry(ids[k], te[k])) {
        tm = fmaxf(tm, te[k]);
        if (ids[k] >= h.classes || !(te[k] < INFINITY)) bad = 1.0f;
      }
    tm = wave_max(tm);
    bad = wave_max(bad);
    float ts = 0.0f;
    for (int k = lane; k < h.top; k += 64)
      if (ids[k] >= 0 && tm != -INFINITY) ts += __builtin_amdgcn_exp2f((te[k] - tm) * c);
    ts = wave_sum(ts);
    const float lts = logf(ts);
    // rows of W in flight to a wave (eight leave no registers: 5000 x 300 x 3000, 32
    // entries a row, 86 us against 59)
    constexpr int KB = R == 1 ? 2 : 4;
    for (int k0 = part * KB; k0 < h.top; k0 += W * KB) {
      int64_t id[KB];
      float z[KB];
#pragma unroll
      for (int k = 0; k < KB; ++k) {
        const int64_t v = k0 + k < h.top ? ids[k0 + k] : -1;
        id[k] = v < h.classes ? v : -1;
      }
      wave_dots<T, KB>(x, w, h.w_in_ld, id, h.dim, lane, z);
#pragma unroll
      for (int k = 0; k < KB; ++k) {
        if (k0 + k >= h.top) continue;
        if (id[k] >= 0) {
          if (h.bias) z[k] += h.bias[id[k]];
          const float u = (te[k0 + k] - tm) * h.inv_t;
          const float q = __builtin_amdgcn_exp2f(u * kLog2e) / ts;
          // an entry without weight adds nothing, whatever its logit
          if (q > 0.0f) loss += q * ((u - lts) + ((m - z[k]) * h.inv_t + l));
        }
        if (lane == 0) h.picked[n * h.top + k0 + k] = id[k] >= 0 ? z[k] : 0.0f;
      }
    }
  }
  if (W > 1) {
    if (lane == 0) sums[wave] = loss;
    __syncthreads();
    loss = 0.0f;
#pragma unroll
    for (int i = 0; i < W; ++i) loss += sums[wave / W * W + i];
  }
  if (live && part == 0 && lane == 0) h.loss[n] = bad != 0.0f ? NAN : tm == -INFINITY ? 0.0f : h.t * h.t * loss;
}

// The significand of a coefficient dloss T, of the first entry of a row that counts (1
// if there is none), by the 256 threads of one block, 4096 entries a round.  dz^T holds
// the coefficients over it, and the gradients are multiplied by it in float32: where all
// rows have the same dloss (a mean's), a target's entry of dz is then a power of two
// times p - 1, and not off by the rounding of dloss to 16 bits in every row alike (up
// to 2^-8 of the whole gradient: at 8192 x 2048 x 131072 it was off by 0.0040 of its
// length, and is by 0.0017, its own rounding).  Where they differ any value does as
// well as another: coefficients stay within a factor of two.  Padding in front is
// common (a masked prompt), so the search goes on until it finds a row, while the other
// blocks prepare theirs (2048 of 4096 rows of 32 entries masked: the step 967 -> 975 us;
// no row masked, no longer).
__device__ __forceinline__ void find_unit(const HeadArgs &h) {
  constexpr int U = 16, NONE = INT32_MAX;
  __shared__ int found[2][4];
  const int t = threadIdx.x, total = (int)(h.rows * h.top);  // at most 2^30
  auto coefficient = [&](int i) { return fabsf(h.dloss[(uint32_t)i / (uint32_t)h.top] * h.t); };
  int first = NONE, flip = 0;
  for (int i0 = 0; i0 < total; i0 += 256 * U) {
    // all loads in flight together: past the last entry that one again
    auto entry = [&](int u) { return min(i0 + 256 * u + t, total - 1); };
    int64_t id[U];
#pragma unroll
    for (int u = 0; u < U; ++u) id[u] = h.ids[entry(u)];
    uint32_t named = 0;
#pragma unroll
    for (int u = 0; u < U; ++u) named |= (uint32_t)(id[u] >= 0) << u;
    for (; named && first == NONE; named &= named - 1) {
      const int i = entry(__ffs(named) - 1);
      const float c = coefficient(i);
      if (c > 0.0f && c < INFINITY && (!h.teacher || is_entry(0, h.teacher[i]))) first = i;
    }
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) first = min(first, __shfl_xor(first, o, 64));
    if ((t & 63) == 0) found[flip][t >> 6] = first;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < 4; ++w) first = min(first, found[flip][w]);
    if (first != NONE) break;
    flip ^= 1;  // one barrier a round
  }
  if (t == 0)
    *h.unit = first != NONE ? __uint_as_float((__float_as_uint(coefficient(first)) & 0x7fffffu) | 0x3f800000u) : 1.0f;
}

// What the backward pass needs of a row, a wave per row: its largest logit m and
// the coefficient over the sum of exp((z - m) / T), so that dz = exp((z - m) / T)
// times it, or (inf, 0) for a row that does not count; the targets as 32-bit
// classes (-1: none) with the weight to take off there; and a copy of x whose rows
// that do not count are zero, so that nothing they hold reaches a sum.
// Few rows of 16 bits: x and zeros up to row 32, then the same again.
// The first block finds the coefficients' unit.
template <typename T>
__global__ __launch_bounds__(256) void head_prepare_kernel(HeadArgs h, T *__restrict__ xs, int64_t xs_ld) {
  constexpr int V = 16 / (int)sizeof(T);
  if (blockIdx.x == 0) {
    find_unit(h);
    return;
  }
  const int lane = threadIdx.x & 63;
  const int64_t n = (int64_t)(blockIdx.x - 1) * 4 + (threadIdx.x >> 6);
  if (n >= h.rows_pad) return;
  float2 info = make_float2(INFINITY, 0.0f);
  const bool pair = sizeof(T) == 2 && h.rows <= kFewRows;
  if (pair && n >= h.rows && n < kFewRows)
    for (int d = lane * V; d < xs_ld; d += 64 * V) {
      *reinterpret_cast<uint4 *>(xs + n * xs_ld + d) = make_uint4(0, 0, 0, 0);
      *reinterpret_cast<uint4 *>(xs + (n + kFewRows) * xs_ld + d) = make_uint4(0, 0, 0, 0);
    }
  if (n < h.rows) {
    const int64_t *ids = h.ids + n * h.top;
    float coef = h.dloss[n] * h.t;
    float bad = 0.0f;
    bool none;
    float tm = -INFINITY, ts = 1.0f;
    if (!h.teacher) {
      none = ids[0] < 0;
      if (ids[0] >= h.classes) bad = 1.0f;
    } else {
      const float *te = h.teacher + n * h.top;
      for (int k = lane; k < h.top; k += 64)
        if (is_entry(ids[k], te[k])) {
          tm = fmaxf(tm, te[k]);
          if (ids[k] >= h.classes || !(te[k] < INFINITY)) bad = 1.0f;
        }
      tm = wave_max(tm);
      bad = wave_max(bad);
      none = tm == -INFINITY && bad == 0.0f;
      ts = 0.0f;
      for (int k = lane; k < h.top; k += 64)
        if (ids[k] >= 0 && !none) ts += __builtin_amdgcn_exp2f((te[k] - tm) * kLog2e * h.inv_t);
      ts = wave_sum(ts);
    }
    if (bad != 0.0f) coef = NAN;
    const bool counts = !none && coef != 0.0f;
    if (counts) {
      const float2 st = h.stats[n];
      info = make_float2(st.x, coef * __builtin_amdgcn_exp2f(-st.y * kLog2e));
    }
    for (int k = lane; k < h.top; k += 64) {
      const float te = h.teacher ? h.teacher[n * h.top + k] : 0.0f;
      const bool entry = counts && is_entry(ids[k], te) && ids[k] < h.classes;
      h.id32[n * h.top + k] = entry ? (int)ids[k] : -1;
      const float q = h.teacher ? __builtin_amdgcn_exp2f((te - tm) * kLog2e * h.inv_t) / ts : 1.0f;
      h.cq[n * h.top + k] = entry ? coef * q : 0.0f;
    }
    const T *p = static_cast<const T *>(h.x_in) + n * h.x_in_ld;
    for (int d = lane * V; d < xs_ld; d += 64 * V) {
      T v[V] = {};
      if (counts) {
        if (d + V <= h.dim) {
          __builtin_memcpy(v, p + d, 16);
        } else {
#pragma unroll
          for (int j = 0; j < V; ++j)
            if (d + j < h.dim) v[j] = p[d + j];
        }
      }
      uint4 q;
      __builtin_memcpy(&q, v, 16);
      *reinterpret_cast<uint4 *>(xs + n * xs_ld + d) = q;
      if (pair) *reinterpret_cast<uint4 *>(xs + (n + kFewRows) * xs_ld + d) = q;
    }
  }
  if (lane == 0) h.info[n] = info;
}

// Distillation, 256 threads a block.  Blocks [0, nt): the targets' entries of dz^T,
// coefficient p less the weights of the row's entries of this class (entries of one
// class write equal values).  The others (first piece, with a bias): what the
// targets take off dbias, 128 classes and one slice of the entries each, as further
// parts behind the row parts of db_part.  A block goes through its slice, 2048 a
// round, keeps the entries of its classes in a list in a fixed order, and two
// threads a class each take every other entry of the list.  (One block for all
// entries of its classes: 63 us for 131,072 entries and 32,000 classes with dx's
// reduction, targets' entries 12; in eight slices 18 and 36.)
constexpr int kBiasRound = 2048;
template <typename T>
__global__ __launch_bounds__(256) void head_targets_kernel(HeadArgs h, int nt) {
  __shared__ int cnt[4];
  __shared__ uint8_t list_c[kBiasRound];
  __shared__ float list_v[kBiasRound];
  __shared__ double half_s[kBiasClasses];
  const int t = threadIdx.x;
  if ((int)blockIdx.x < nt) {
    const int64_t i = (int64_t)blockIdx.x * 256 + t;
    if (i >= h.rows * h.top) return;
    const int id = h.id32[i];
    if (id < h.v0 || id >= h.v0 + h.piece) return;
    const int64_t n = i / h.top;
    const float2 info = h.info[n];
    float v = __builtin_amdgcn_exp2f((h.picked[i] - info.x) * h.inv_t * kLog2e) * info.y;
    for (int k = 0; k < h.top; ++k)
      if (h.id32[n * h.top + k] == id) v -= h.cq[n * h.top + k];
    v /= *h.unit;
    T *p = static_cast<T *>(h.gt) + (id - h.v0) * h.rows_pad + n;
    put(p, v);
    if (sizeof(T) == 2 && h.rows <= kFewRows) put(p + kFewRows, bf16_rest(v));
    return;
  }
  const int lane = t & 63, wave = t >> 6;
  const int b = blockIdx.x - nt, slice = b % h.bias_slices;
  const int c0 = b / h.bias_slices * kBiasClasses;
  const int mine = t % kBiasClasses, second = t / kBiasClasses;
  const int64_t total = h.rows * h.top;
  const int64_t per = (total + h.bias_slices * 4 - 1) / (h.bias_slices * 4) * 4;  // whole 16 bytes
  const int64_t lo = slice * per, hi = lo + per < total ? lo + per : total;
  double sum = 0.0;
  int4 nx[2];
  auto fetch = [&](int64_t i0) {
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int64_t i = i0 + u * (kBiasRound / 2) + 4 * t;
      if (i + 4 <= hi) {
        nx[u] = *reinterpret_cast<const int4 *>(h.id32 + i);
      } else {
        int v[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) v[k] = i + k < hi ? h.id32[i + k] : -1;
        nx[u] = make_int4(v[0], v[1], v[2], v[3]);
      }
    }
  };
  fetch(lo);
  for (int64_t i0 = lo; i0 < hi; i0 += kBiasRound) {
    const int id[8] = {nx[0].x - c0, nx[0].y - c0, nx[0].z - c0, nx[0].w - c0,
                       nx[1].x - c0, nx[1].y - c0, nx[1].z - c0, nx[1].w - c0};
    fetch(i0 + kBiasRound);
    int n = 0;
#pragma unroll
    for (int k = 0; k < 8; ++k) n += (unsigned)id[k] < (unsigned)kBiasClasses;
    int before = n;  // entries up to this lane's
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int u = __shfl_up(before, o, 64);
      if (lane >= o) before += u;
    }
    if (lane == 63) cnt[wave] = before;
    __syncthreads();
    int at = before - n, all = 0;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      if (w < wave) at += cnt[w];
      all += cnt[w];
    }
#pragma unroll
    for (int k = 0; k < 8; ++k)
      if ((unsigned)id[k] < (unsigned)kBiasClasses) {
        list_c[at] = (uint8_t)id[k];
        list_v[at] = h.cq[i0 + (k >> 2) * (kBiasRound / 2) + 4 * t + (k & 3)];
        ++at;
      }
    __syncthreads();
#pragma unroll 4
    for (int k = second; k < all; k += 2)
      if (list_c[k] == mine) sum -= list_v[k];
    // the next round's counts are written before its first barrier and its list
    // behind it, this round's counts read before the last barrier
  }
  __syncthreads();
  if (second) half_s[mine] = sum;
  __syncthreads();
  if (!second && c0 + mine < h.classes)
    h.db_part[(int64_t)(h.db_parts + slice) * h.classes + c0 + mine] = (float)((sum + half_s[mine]) / (double)*h.unit);
}

// out[r][d] = unit times the splits' partial sums in order, 0 in rows that do not
// count (info, if given); block b of nb.
constexpr int kReduceThreads = 512;
template <typename T>
__device__ __forceinline__ void reduce_rows(const float *part, int splits, int64_t rows, int dim, int pad, T *out, int64_t ld,
                                            float unit, const float2 *info, int b, int nb) {
  const int per = (dim + 3) / 4;
  const int64_t total = rows * per;
  for (int64_t i = (int64_t)b * kReduceThreads + threadIdx.x; i < total; i += (int64_t)nb * kReduceThreads) {
    const int64_t n = i / per;
    const int d = (int)(i - n * per) * 4;
    float v[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    if (!info || info[n].y != 0.0f)
      for (int s = 0; s < splits; ++s) {
        const float4 u = *reinterpret_cast<const float4 *>(part + ((int64_t)s * rows + n) * pad + d);
        v[0] += u.x; v[1] += u.y; v[2] += u.z; v[3] += u.w;
      }
    T *o = out + n * ld + d;
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (d + j < dim) put(o + j, v[j] * unit);
  }
}

// In blocks [0, nx) of the launch dx from its partial sums, in [nx, nx + nw) dW from
// its (where there are any).  In the others dbias, 128 classes a block: the sums of
// its parts (the rows', and for distillation the targets', which cancel much of them:
// in 64 bits), four threads a class, in order, so that results do not vary.
template <typename T>
__global__ __launch_bounds__(kReduceThreads) void head_reduce_kernel(HeadArgs h, int nx, int nw) {
  __shared__ double sums[4][kBiasClasses];
  const int t = threadIdx.x, b = blockIdx.x;
  const float unit = h.rows > 0 ? *h.unit : 0.0f;
  if (b < nx) {
    reduce_rows(h.dx_part, h.splits, h.rows, h.dim, h.dx_pad, static_cast<T *>(h.dx), h.dx_ld, unit, h.info, b, nx);
    return;
  }
  if (b < nx + nw) {
    reduce_rows(h.dw_part, h.w_splits, h.classes, h.dim, h.dx_pad, static_cast<T *>(h.dw), h.dw_ld, unit,
                (const float2 *)nullptr, b - nx, nw);
    return;
  }
  const int64_t c0 = (int64_t)(b - nx - nw) * kBiasClasses;
  const int slice = t / kBiasClasses, mine = t % kBiasClasses;
  const int parts = h.db_parts + h.bias_slices;
  double sum = 0.0;
  if (c0 + mine < h.classes)
    for (int p = slice; p < parts; p += 4) sum += h.db_part[(int64_t)p * h.classes + c0 + mine];
  sums[slice][mine] = sum;
  __syncthreads();
  if (slice == 0 && c0 + mine < h.classes)
    h.dbias[c0 + mine] = (float)(((sums[0][mine] + sums[1][mine]) + (sums[2][mine] + sums[3][mine])) * (double)unit);
}

int grid_for(int64_t n, int per) {
  const int64_t b = (n + per - 1) / per;
  return (int)(b < 1 ? 1 : b > 16384 ? 16384 : b);
}

// ---------------------------------------------------------------- variants

// Stages of the 64 x 64 tiles: three, and three workgroups to a CU; float32, bound by
// its MFMAs, is better with four workgroups of two stages (512 x 1024 x 10,007 step
// 367 us against 380; bf16 1000 x 1024 x 5000 112 us against 93 the other way round).
template <typename T>
constexpr int kSmallStages = sizeof(T) == 2 ? 3 : 2;
template <typename T, int EPI>
struct Tiles;
template <typename T>
struct Tiles<T, E_STATS> {
  typedef BigTile<T, false, false, E_STATS> Big;
  typedef RingTile<T, 128, 128, 2, 2, 2, false, false, E_STATS> Mid;
  typedef RingTile<T, 64, 64, 2, 2, kSmallStages<T>, false, false, E_STATS> Small;
  typedef RingTile<T, 128, 32, 4, 1, 7, false, false, E_STATS> Few;
  typedef RingTile<T, 64, 64, 2, 2, 8, false, false, E_STATS> Deep;
  typedef TinyTile<T, 8, E_STATS> Tiny;
};
template <typename T>
struct Tiles<T, E_DLOGITS> {
  typedef BigTile<T, false, false, E_DLOGITS> Big;
  typedef RingTile<T, 128, 128, 2, 2, 2, false, false, E_DLOGITS> Mid;
  typedef RingTile<T, 64, 64, 2, 2, kSmallStages<T>, false, false, E_DLOGITS> Small;
  typedef RingTile<T, 32, 128, 1, 4, 7, false, false, E_DLOGITS> Few;
  typedef RingTile<T, 64, 64, 2, 2, 8, false, false, E_DLOGITS> Deep;
  typedef TinyTile<T, 8, E_DLOGITS> Tiny;
};
template <typename T>
struct Tiles<T, E_DX> {
  typedef BigTile<T, true, true, E_DX> Big;
  typedef RingTile<T, 128, 128, 2, 2, 2, true, true, E_DX> Mid;
  typedef RingTile<T, 64, 64, 2, 2, kSmallStages<T>, true, true, E_DX> Small;
  typedef std::conditional_t<sizeof(T) == 2, RingTile<T, 128, 64, 4, 1, 3, true, true, E_DX, true>,
                             RingTile<T, 128, 32, 4, 1, 4, true, true, E_DX>> Few;
};
template <typename T>
struct Tiles<T, E_DW> {
  typedef BigTile<T, true, false, E_DW> Big;
  typedef RingTile<T, 128, 128, 2, 2, 2, true, false, E_DW> Mid;
  typedef RingTile<T, 64, 64, 2, 2, kSmallStages<T>, true, false, E_DW> Small;
};

template <typename T, int EPI>
hipError_t product(Variant v, const Gemm &g, const HeadArgs &a, hipStream_t s) {
  typedef Tiles<T, EPI> X;
  switch (v) {
    case BIG: return launch_product<typename X::Big>(g, a, s);
    case MID: return launch_product<typename X::Mid>(g, a, s);
    case SMALL:
      // no more than one workgroup to a CU: seven k-tiles in flight, not two
      if (ceil_div(g.a_ext, 64) * ceil_div(g.b_ext, 64) <= kCus) return launch_product<typename X::Deep>(g, a, s);
      return launch_product<typename X::Small>(g, a, s);
    case TINY: return launch_product<typename X::Tiny>(g, a, s);
    default: return launch_product<typename X::Few>(g, a, s);
  }
}

template <typename T>
hipError_t forward(const HeadArgs &a, hipStream_t s) {
  Gemm g{};
  g.a_ld = a.w_ld;
  g.b = a.x; g.b_ld = a.x_ld; g.b_ext = (int)a.rows;
  g.k_ext = a.dim; g.splits = 1;
  for (int64_t c0 = 0; c0 < a.classes;) {
    const HeadLaunch l = head_forward_launch(sizeof(T) == 2, a.rows, a.classes, c0);
    g.a = static_cast<const T *>(a.w) + c0 * a.w_ld;
    g.a_ext = (int)l.classes;
    HeadArgs h = a;
    if (a.bias) h.bias += c0;
    h.part += (int64_t)l.part * a.rows;
    h.parts = l.parts;
    const hipError_t e = product<T, E_STATS>(l.v, g, h, s);
    if (e != hipSuccess) return e;
    c0 += l.classes;
  }
  return hipSuccess;
}
template <typename T>
hipError_t finish(const HeadArgs &a, hipStream_t s) {
  // As many waves to a row as leave a block to every CU: its entries' dots are what takes
  // the time (256 x 1024 x 32000, 32 entries a row: 9.5 us with a row a block, 15.2 with
  // four, 39.8 with sixteen; 1000 rows 23.8, 19.5 and 39.9; 4096 rows 98, 79 and 64: the
  // more rows to a block, the wider are the reads of the parts).
  const dim3 block(1024);
  if (a.rows <= kCus) hapi_launch((head_finish_kernel<T, 1>), dim3((uint32_t)a.rows), block, 0, s, a);
  else if (a.rows <= 4 * kCus) hapi_launch((head_finish_kernel<T, 4>), dim3((uint32_t)ceil_div(a.rows, 4)), block, 0, s, a);
  else hapi_launch((head_finish_kernel<T, 16>), dim3((uint32_t)ceil_div(a.rows, 16)), block, 0, s, a);
  return hipGetLastError();
}
template <typename T>
hipError_t dlogits(const HeadArgs &a, hipStream_t s) {
  if (a.rows == 0) return hipSuccess;
  Gemm g{};
  g.a = a.x; g.a_ld = a.x_ld; g.a_ext = (int)a.rows;
  g.b = static_cast<const T *>(a.w) + a.v0 * a.w_ld; g.b_ld = a.w_ld; g.b_ext = (int)a.piece;
  g.k_ext = a.dim; g.splits = 1;
  const Variant v = head_variant(sizeof(T) == 2, a.rows, a.classes);
  const int64_t c = v == BIG && sizeof(T) == 2 ? head_big_classes(a.rows, a.piece) : a.piece;
  g.b_ext = (int)c;
  hipError_t e = product<T, E_DLOGITS>(v, g, a, s);
  if (e == hipSuccess && c < a.piece) {
    HeadArgs rest = a;
    rest.v0 += c;
    rest.gt = static_cast<T *>(a.gt) + c * a.rows_pad;
    g.b = static_cast<const T *>(g.b) + c * a.w_ld;
    g.b_ext = (int)(a.piece - c);
    e = product<T, E_DLOGITS>(MID, g, rest, s);
  }
  if (e != hipSuccess || !a.teacher) return e;
  const int64_t nt = ceil_div(a.rows * a.top, 256);
  const int64_t nb = a.db_part && a.first ? ceil_div(a.classes, kBiasClasses) * a.bias_slices : 0;
  if (nt + nb > kMaxLaunchThreads / 256) return hipErrorInvalidValue;
  hapi_launch(head_targets_kernel<T>, dim3((uint32_t)(nt + nb)), dim3(256), 0, s, a, (int)nt);
  return hipGetLastError();
}
template <typename T>
hipError_t grads(const HeadArgs &a, hipStream_t s) {
  Gemm x{}, w{};
  x.a = static_cast<const T *>(a.w) + a.v0 * a.w_ld; x.a_ld = a.w_ld; x.a_ext = a.dx_pad;
  x.b = a.gt; x.b_ld = a.rows_pad; x.b_ext = (int)a.rows;
  x.k_ext = (int)a.piece; x.splits = a.splits;
  w.a = a.x; w.a_ld = a.x_ld; w.a_ext = a.dx_pad;
  w.b = a.gt; w.b_ld = a.rows_pad; w.b_ext = (int)a.piece;
  w.k_ext = (int)a.rows; w.splits = a.w_splits;
  if (sizeof(T) == 2 && a.rows > 0 && a.rows <= kFewRows) {  // dz's second halves
    x.b_ext = 2 * kFewRows;
    w.k_ext = 2 * kFewRows;
  }
  typedef Tiles<T, E_DX> X;
  typedef Tiles<T, E_DW> W;
  Variant v = head_variant(sizeof(T) == 2, a.rows, a.classes);
  if (v == TINY) v = a.rows <= kFewRows ? FEW : SMALL;
  switch (v) {
    case BIG: return launch_grads<typename X::Big, typename W::Big>(x, w, a, s);
    case MID: return launch_grads<typename X::Mid, typename W::Mid>(x, w, a, s);
    case SMALL: return launch_grads<typename X::Small, typename W::Small>(x, w, a, s);
    default:
      // Many tiles of dW: in a launch of their own, where more of them fit a CU
      // (8 x 4096 x 131072: 1279 us in one launch, 82 KB of LDS each; apart dW takes 324).
      if (!head_few_apart(a.dim, a.piece))
        return launch_grads<typename X::Few, typename W::Small>(x, w, a, s);
      {
        const hipError_t e = launch_product<typename X::Few>(x, a, s);
        return e != hipSuccess ? e : launch_product<typename W::Mid>(w, a, s);
      }
  }
}
}  // namespace

hipError_t launch_head_stage(bool bf16, const void *in, int64_t ld_in, void *out, int64_t ld_out, int64_t rows, int dim,
                             hipStream_t s) {
  if (rows == 0) return hipSuccess;
  const int64_t n = rows * ld_out * (bf16 ? 2 : 4) / 16;
  if (bf16)
    hapi_launch(stage_kernel<uint16_t>, dim3(grid_for(n, 256)), dim3(256), 0, s, (const uint16_t *)in, ld_in,
                (uint16_t *)out, ld_out, rows, dim);
  else
    hapi_launch(stage_kernel<float>, dim3(grid_for(n, 256)), dim3(256), 0, s, (const float *)in, ld_in, (float *)out,
                ld_out, rows, dim);
  return hipGetLastError();
}

hipError_t launch_head_forward(bool bf16, const HeadArgs &a, hipStream_t s) {
  return bf16 ? forward<uint16_t>(a, s) : forward<float>(a, s);
}

hipError_t launch_head_finish(bool bf16, const HeadArgs &a, hipStream_t s) {
  if (a.rows == 0) return hipSuccess;
  return bf16 ? finish<uint16_t>(a, s) : finish<float>(a, s);
}

hipError_t launch_head_prepare(bool bf16, const HeadArgs &a, void *xs, int64_t xs_ld, hipStream_t s) {
  if (a.rows == 0) return hipSuccess;
  const dim3 grid((uint32_t)((a.rows_pad + 3) / 4) + 1);
  if (bf16) hapi_launch(head_prepare_kernel<uint16_t>, grid, dim3(256), 0, s, a, (uint16_t *)xs, xs_ld);
  else hapi_launch(head_prepare_kernel<float>, grid, dim3(256), 0, s, a, (float *)xs, xs_ld);
  return hipGetLastError();
}

hipError_t launch_head_dlogits(bool bf16, const HeadArgs &a, hipStream_t s) {
  return bf16 ? dlogits<uint16_t>(a, s) : dlogits<float>(a, s);
}

hipError_t launch_head_grads(bool bf16, const HeadArgs &a, hipStream_t s) {
  return bf16 ? grads<uint16_t>(a, s) : grads<float>(a, s);
}

hipError_t launch_head_reduce(bool bf16, const HeadArgs &a, hipStream_t s) {
  auto blocks = [&](int64_t rows) { return (int)std::min<int64_t>(ceil_div(rows * ((a.dim + 3) / 4), kReduceThreads), 2048); };
  const int nx = a.rows > 0 && !a.dx_whole ? blocks(a.rows) : 0;
  const int nw = a.w_splits > 1 ? blocks(a.classes) : 0;
  const int nb = a.dbias ? (int)ceil_div(a.classes, kBiasClasses) : 0;
  if (nx + nw + nb == 0) return hipSuccess;
  const dim3 grid((uint32_t)(nx + nw + nb));
  if (bf16) hapi_launch(head_reduce_kernel<uint16_t>, grid, dim3(kReduceThreads), 0, s, a, nx, nw);
  else hapi_launch(head_reduce_kernel<float>, grid, dim3(kReduceThreads), 0, s, a, nx, nw);
  return hipGetLastError();
}

}  // namespace hapi
