// Device helpers of the cross attention's kernels: tiles of rows in LDS, their
// fragments for the matrix cores, and the outputs' stores.
//
// Every product is out^T[a][b] = sum_k A[a][k] B[k][b] on 32 x 32 blocks: lane l holds
// column b = l % 32, its registers rows a = 8 q + 4 (l / 32) + e (register 4 q + e).
// A block of scores, columns owned by lanes, is the next product's B operand as it is:
// of 16 k, the lane's half lh holds k = 4 lh + 0 .. 3 and 8 + 4 lh + 0 .. 3, and the A
// operand is read from LDS in that order (by_column).
#pragma once

#include <type_traits>

#include "block.h"
#include "gemm_util.h"

namespace hapi {
namespace {

typedef float f32x8_t __attribute__((ext_vector_type(8)));
typedef short s16x4_t __attribute__((ext_vector_type(4)));

template <typename T>
struct Elem;
template <>
struct Elem<uint16_t> {
  typedef bf16x8_t Frag;  // 8 values of k
};
template <>
struct Elem<float> {
  typedef f32x8_t Frag;
};

__device__ __forceinline__ f32x16_t mma(bf16x8_t a, bf16x8_t b, f32x16_t c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}
// 16 k as eight products of 2: the pairing of k with lane halves is that of the bf16 one.
__device__ __forceinline__ f32x16_t mma(f32x8_t a, f32x8_t b, f32x16_t c) {
#pragma unroll
  for (int j = 0; j < 8; ++j) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a[j], b[j], c, 0, 0, 0);
  return c;
}
// A block of one value: the forward pass' scores start from it in bf16, which subtracts a
// row's reference without an instruction of its own.
__device__ __forceinline__ f32x16_t block_of(float v) {
  f32x16_t z;
#pragma unroll
  for (int r = 0; r < 16; ++r) z[r] = v;
  return z;
}
__device__ __forceinline__ f32x16_t zeros() { return block_of(0.0f); }
// Registers 8 j .. 8 j + 7 of a block as an operand of 16 k, rounded to T.
template <typename T>
__device__ __forceinline__ typename Elem<T>::Frag operand(const f32x16_t &s, int j) {
  typename Elem<T>::Frag f;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    if constexpr (sizeof(T) == 2) f[e] = (__bf16)s[8 * j + e];
    else f[e] = s[8 * j + e];
  }
  return f;
}

// The waves to a SIMD that a kernel's registers are to leave room for: `want`, or as many as
// fit with the workgroup's LDS of a CU's 160 KB, if fewer.
constexpr int least_waves(int want, int waves, int lds) {
  const int fit = (160 * 1024 / lds * waves + 3) / 4;
  return fit < 1 ? 1 : fit < want ? fit : want;
}

// acc += A(0) f[0] + A(1) f[1], 32 values of k.  In float32 the products are summed by
// themselves first: a row's sum over thousands of keys is then one of block sums, with a
// rounding for each 32 keys and not for each two (1 x 200 x 16384, heads of 128: o off by
// 6.2e-7 of its length, so 4.6e-7, dq by 1.2e-6 and 7.5e-7).
template <typename T, typename A>
__device__ __forceinline__ void add_products(f32x16_t &acc, A &&a, const typename Elem<T>::Frag (&f)[2]) {
  if constexpr (sizeof(T) == 2) {
    acc = mma(a(0), f[0], acc);
    acc = mma(a(1), f[1], acc);
  } else {
    f32x16_t t = mma(a(0), f[0], zeros());
    t = mma(a(1), f[1], t);
#pragma unroll
    for (int i = 0; i < 16; ++i) acc[i] += t[i];
  }
}

// ROWS rows of DP values in LDS, 16-byte slots permuted within a row so that both
// ways of reading spread over the banks; a DMA writes slots in order, so the
// permutation is in the address each lane loads from.
template <typename T, int DP, int ROWS>
struct Tile {
  static constexpr int V = 16 / (int)sizeof(T), CPR = DP / V, PITCH = DP * (int)sizeof(T);
  static constexpr int BYTES = ROWS * PITCH, DMAS = BYTES / 1024;  // of 64 slots each
  static_assert(DMAS * 1024 == BYTES, "whole DMAs");

  static __device__ __forceinline__ int swz(int row) {
    if constexpr (CPR == 4 || CPR == 12) return (row >> 2) & 3;
    if constexpr (CPR == 24) return (row >> 1) & 7;
    if constexpr (CPR == 8) return ((row >> 1) & 1) << 2 | ((row >> 2) & 3);
    // 16-bit columns are read as 64 bytes of each of 8 rows, 32-bit ones as 128 of 2
    if constexpr (sizeof(T) == 2) return (row & 3) << 2 | ((row >> 2) & 3);
    return ((row >> 2) & 1) << 3 | ((row >> 3) & 1) << 2 | (row & 3);
  }
  typedef typename Elem<T>::Frag Frag;
  // Row r + lane % 32, values 16 ks + 8 lh .. + 7.
  static __device__ __forceinline__ Frag by_row(const uint8_t *tile, int r, int ks, int lane) {
    const int row = r + (lane & 31), lh = lane >> 5;
    if constexpr (sizeof(T) == 2) {
      return *reinterpret_cast<const Frag *>(tile + row * PITCH + (((2 * ks + lh) ^ swz(row)) * 16));
    } else {
      typedef float f32x4_t __attribute__((ext_vector_type(4)));
      const f32x4_t lo = *reinterpret_cast<const f32x4_t *>(tile + row * PITCH + (((4 * ks + 2 * lh) ^ swz(row)) * 16));
      const f32x4_t hi = *reinterpret_cast<const f32x4_t *>(tile + row * PITCH + (((4 * ks + 2 * lh + 1) ^ swz(row)) * 16));
      return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
    }
  }
  // Column d + lane % 32, rows r + 4 lh + 0 .. 3 and r + 8 + 4 lh + 0 .. 3.
  static __device__ __forceinline__ Frag by_column(const uint8_t *tile, int r, int d, int lane) {
    const int lh = lane >> 5;
    if constexpr (sizeof(T) == 2) {
      // 16 lanes read 4 rows of 16 columns, lane i getting column i's four
      const int i = lane & 15, col = d + (lane & 16) + 4 * (i & 3);
      union {
        s16x4_t h[2];
        Frag f;
      } u;
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int row = r + 8 * e + 4 * lh + (i >> 2);
        const uint8_t *p = tile + row * PITCH + (((col >> 3) ^ swz(row)) * 16) + (col & 7) * 2;
        u.h[e] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
            (__attribute__((address_space(3))) s16x4_t *)(__attribute__((address_space(3))) void *)p);
      }
      return u.f;
    } else {
      const int col = d + (lane & 31);
      Frag f;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int row = r + 8 * (j >> 2) + 4 * lh + (j & 3);
        f[j] = *reinterpret_cast<const float *>(tile + row * PITCH + (((col >> 2) ^ swz(row)) * 16) + (col & 3) * 4);
      }
      return f;
    }
  }
};

// How WAVES waves bring a tile's rows to LDS: this lane's byte offsets from the tile's
// first row.
template <typename T, int DP, int ROWS, int WAVES>
struct Loader {
  typedef hapi::Tile<T, DP, ROWS> Tile;
  static constexpr int LOADS = Tile::DMAS / WAVES;
  static_assert(LOADS * WAVES == Tile::DMAS, "as many DMAs to every wave");
  uint32_t off[LOADS];
  int row[LOADS];
  // stride: elements between rows
  __device__ __forceinline__ void init(int64_t stride, int dim, int wave, int lane) {
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
      const int slot = (wave * LOADS + i) * 64 + lane;
      row[i] = slot / Tile::CPR;
      const int c = (slot % Tile::CPR) ^ Tile::swz(row[i]);
      off[i] = c * Tile::V < dim ? (uint32_t)((row[i] * stride + c * Tile::V) * (int64_t)sizeof(T)) : kOob;
    }
  }
  // keep: a bit for each row; the others are zeros.
  __device__ __forceinline__ void issue(const void *base, uint32_t lds, uint64_t keep, int wave) const {
    const u32x4_t srd = make_srd(base);
#pragma unroll
    for (int i = 0; i < LOADS; ++i)
      lds_dma16(srd, lds + (wave * LOADS + i) * 1024, (keep >> row[i]) & 1 ? off[i] : kOob, 0);
  }
  // The tile's rows are the rows list[0 .. ROWS) of base, within 2^31 bytes of it.
  static __device__ __forceinline__ void gather(const void *base, int64_t stride, int dim, const int *list, uint32_t lds, uint64_t keep, int wave,
                                                int lane) {
    const u32x4_t srd = make_srd(base);
    const uint32_t to = __builtin_amdgcn_readfirstlane(lds + wave * LOADS * 1024), ld = (uint32_t)stride * (uint32_t)sizeof(T);
#pragma unroll 1  // rare, and its offsets would take registers from the kernel's loop
    for (int i = 0; i < LOADS; ++i) {
      const int slot = (wave * LOADS + i) * 64 + lane, r = slot / Tile::CPR, c = (slot % Tile::CPR) ^ Tile::swz(r);
      const bool there = ((keep >> r) & 1) && c * Tile::V < dim;
      lds_dma16(srd, to + i * 1024, there ? (uint32_t)list[r] * ld + (uint32_t)(c * 16) : kOob, 0);
    }
  }
};

// Until at most N of this wave's loads and DMAs are in flight and its LDS reads are done.
// The builtin, not asm: the compiler then knows that what was loaded before a loop has
// arrived; it would else wait for it at its first use in every turn, and so for the DMAs
// that the turn has just started.
template <int N>
__device__ __forceinline__ void wait_loads() {
  static_assert(N >= 0 && N < 64, "vmcnt range");
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt((N & 15) | ((N >> 4) << 14) | (7 << 4));
  __builtin_amdgcn_sched_barrier(0);
}

// The keys of a tile of BN: a bit for each, of all of them and of the first `left`.
template <int BN>
constexpr uint64_t kAllKeys = BN == 64 ? ~0ull : (1ull << (BN & 63)) - 1;
template <int BN>
constexpr uint64_t key_bits(int64_t left) {
  return left >= BN ? kAllKeys<BN> : left > 0 ? (1ull << left) - 1 : 0;
}

// A wave's 8 values of k of a row in memory: values 16 ks + 8 lh .. + 7, zeros past dim
// (whole 16-byte slots are inside or outside).  The row needs its elements' alignment only:
// o lies where the forward pass was told to write it (loads of 16 bytes need no more here).
template <typename T>
__device__ __forceinline__ typename Elem<T>::Frag row_frag(const T *row, int ks, int lh, int dim, bool there) {
  typedef typename Elem<T>::Frag Frag;
  const int d = 16 * ks + 8 * lh;
  Frag f;
#pragma unroll
  for (int e = 0; e < 8; ++e) f[e] = 0;
  if constexpr (sizeof(T) == 2) {
    if (there && d < dim) __builtin_memcpy(&f, row + d, 16);
  } else {
    typedef float f32x4_t __attribute__((ext_vector_type(4)));
    f32x4_t h[2] = {};
#pragma unroll
    for (int i = 0; i < 2; ++i)
      if (there && d + 4 * i < dim) __builtin_memcpy(&h[i], row + d + 4 * i, 16);
    f = __builtin_shufflevector(h[0], h[1], 0, 1, 2, 3, 4, 5, 6, 7);
  }
  return f;
}

// Four values of a row from d on; vec: the row's places allow one store.
template <typename T>
__device__ __forceinline__ void store4(T *row, int d, int dim, bool vec, float v0, float v1, float v2, float v3) {
  if (vec) {
    if (d >= dim) return;
    if constexpr (sizeof(T) == 2) *reinterpret_cast<uint2 *>(row + d) = make_uint2(f2bf2(v0, v1), f2bf2(v2, v3));
    else *reinterpret_cast<float4 *>(row + d) = make_float4(v0, v1, v2, v3);
    return;
  }
  const float v[4] = {v0, v1, v2, v3};
#pragma unroll
  for (int e = 0; e < 4; ++e)
    if (d + e < dim) {
      if constexpr (sizeof(T) == 2) row[d + e] = f2bf(v[e]);
      else row[d + e] = v[e];
    }
}

// A wave's 32 rows of out^T, acc[d] the values 32 d + 8 q + 4 lh + e of row lane % 32, times
// `by`, to memory: to is this lane's row (null: none), vec what of a row can be stored at
// once.  16-bit rows that allow 16 bytes at once are turned in `turn`, the wave's part of
// the LDS, and stored whole to consecutive lanes; stores of the lanes' own values would be
// up to 16 bytes of each of 32 rows, and the L2 takes a request for every such piece.
// PAIRS: so are rows that allow two values but not four.  Forward and dq, which store more
// than they read where rows are many: 16 x 3182 x 97, 16 + 8 heads of 86, 253 us, so 146, and
// 429, so 310; dk and dv gained nothing, and 8 bytes a lane (64 x 64 x 197, heads of 60) are
// faster as they are, forward 14.3 us for 15.6.
template <typename T, int DB>
struct RowsOut {
  static constexpr bool TURNS = sizeof(T) == 2;  // 32-bit values make 32 bytes of a row as they are
  static constexpr int PITCH = 32 * DB * (int)sizeof(T) + 16, BYTES = TURNS ? 32 * PITCH : 0;
  // Rows from LDS, N values a lane.
  template <int N>
  static __device__ __forceinline__ void rows(T *to, int dim, const uint8_t *turn, int lane) {
    typedef std::conditional_t<N == 8, uint4, uint32_t> Slot;
    constexpr int PER = 32 * DB / N;  // slots of a row
    const uint64_t mine = (uint64_t)(uintptr_t)to;
#pragma unroll
    for (int i = 0; i < 32 * PER / 64; ++i) {
      const int slot = i * 64 + lane, row = slot / PER, c = slot % PER;
      const uint32_t lo = __shfl((uint32_t)mine, row, 64), hi = __shfl((uint32_t)(mine >> 32), row, 64);
      T *p = reinterpret_cast<T *>((uintptr_t)((uint64_t)hi << 32 | lo));
      const Slot v = *reinterpret_cast<const Slot *>(turn + row * PITCH + c * sizeof(Slot));
      if (p && c * N < dim) *reinterpret_cast<Slot *>(p + c * N) = v;
    }
  }
  template <bool PAIRS>
  static __device__ __forceinline__ void store(const f32x16_t (&acc)[DB], float by, T *to, int dim, int vec, uint8_t *turn, int lane) {
    const int lh = lane >> 5;
    if (!TURNS || !(vec & 2 || (PAIRS && vec == 4))) {
      if (to) {
#pragma unroll
        for (int d = 0; d < DB; ++d)
#pragma unroll
          for (int q = 0; q < 4; ++q)
            store4<T>(to, 32 * d + 8 * q + 4 * lh, dim, vec & 1, acc[d][4 * q] * by, acc[d][4 * q + 1] * by, acc[d][4 * q + 2] * by,
                      acc[d][4 * q + 3] * by);
      }
      return;
    }
    if constexpr (TURNS) {
#pragma unroll
      for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          uint8_t *at = turn + (lane & 31) * PITCH + (32 * d + 8 * q + 4 * lh) * (int)sizeof(T);
          const float v0 = acc[d][4 * q] * by, v1 = acc[d][4 * q + 1] * by, v2 = acc[d][4 * q + 2] * by, v3 = acc[d][4 * q + 3] * by;
          *reinterpret_cast<uint2 *>(at) = make_uint2(f2bf2(v0, v1), f2bf2(v2, v3));
        }
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      if (!PAIRS || vec & 2) rows<8>(to, dim, turn, lane);
      else rows<2>(to, dim, turn, lane);
    }
  }
};

constexpr float kLog2e = 1.4426950408889634f;

// A workgroup's part of the problem: tiles of one key head run together on one XCD and
// share its keys and values in the L2.
struct Place {
  int tile, split, pair, b, kh;
};
__device__ __forceinline__ Place place(const AttendArgs &a, int tiles) {
  const int id = xcd_remap(blockIdx.x, gridDim.x), rest = __builtin_amdgcn_readfirstlane(id / tiles);
  Place p;
  p.tile = id - rest * tiles;
  p.pair = __builtin_amdgcn_readfirstlane(rest / a.splits);
  p.split = rest - p.pair * a.splits;
  p.b = __builtin_amdgcn_readfirstlane(p.pair / a.kv_heads);
  p.kh = p.pair - p.b * a.kv_heads;
  return p;
}

// Entry b of lens, within 0 .. most.
__device__ __forceinline__ int clamped(const int64_t *lens, int b, int most) {
  if (!lens) return most;
  const int64_t n = lens[b];
  return n < 0 ? 0 : n < most ? (int)n : most;
}

}  // namespace
}  // namespace hapi
