// Cross attention, backward, without atomics, so that results do not vary.  With
// p = exp(scale (s - m) - l) from the forward pass's statistics:
//   dv = p^T dout, dp = dout v^T, ds = p (dp - delta), delta = sum of dout o,
//   dq = scale ds k, dk = scale ds^T q.
//
// dq: rows and waves as in the forward pass.  A wave keeps its rows' q and dout in
// registers and forms S^T and dP^T of each tile of keys; dS^T is the operand of
// dq^T = K^T dS^T as it is, K^T read transposed from LDS.  It also forms delta.
// dk, dv: a wave keeps 32 keys, k and v in registers, and walks the rows of all query
// heads that share them (their sum is that of its registers): S = Q K^T and dP = dout
// V^T own a key in a lane, so P and dS are the operands of dv^T = dout^T P and
// dk^T = Q^T dS as they are.
// Few rows: all three in one kernel, below.
//
// Scores and dP are formed in both of the first two, seven products where five would do if
// the parts of dq could be added by atomics or went through memory (4 bytes of each value
// for every 128 keys).  P and dS are rounded to the operands' type for the matrix
// cores; all sums are float32.
//
// Bound by the matrix pipes: 2 x 4096 x 4096, 16 + 4 heads of 128 in bf16, dq 418 to 429
// us, 0.96 to 0.99 PF/s of its three products, pipes busy 54%; dk and dv 581 to 597 us, 0.92 to
// 0.95 PF/s of four, 50%.
// float32 of 3 x 77 x 1021, 12 + 4 heads of 80: 31 and 38 us, 43% and 50%.
#include <type_traits>

#include "attend.h"

namespace hapi {
namespace {

constexpr int kFewKeys = 128;

// Where a call has few rows, the roundings of its P and dS to bf16 do not average (a row
// of one token against two keys: dq off by 0.0028 of its length, so 0.0017).  FINE kernels
// multiply by what the rounding left, too: this, as operands.
__device__ __forceinline__ void keep_rest(f32x16_t &s) {
#pragma unroll
  for (int i = 0; i < 16; ++i) s[i] -= (float)(__bf16)s[i];
}

// How many of n keys a mask leaves, or more than kFewKeys as soon as it is that many.  The
// first kFewKeys of them to list (or null), in order.
__device__ __forceinline__ int kept_keys(const uint8_t *mask, int n, int lane, int *list) {
  int kept = 0;
  auto count = [&](auto loads, int k) {  // loads in flight, of 64 keys each
    constexpr int N = decltype(loads)::value;
    bool on[N];
#pragma unroll
    for (int i = 0; i < N; ++i) on[i] = k + 64 * i + lane < n && mask[k + 64 * i + lane] != 0;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const uint64_t bits = __ballot(on[i]);
      if (list && bits != 0 && kept < kFewKeys) {
        const int at = kept + __popcll(bits & ((1ull << lane) - 1));
        if (on[i] && at < kFewKeys) list[at] = k + 64 * i + lane;
      }
      kept += __popcll(bits);
    }
  };
  count(std::integral_constant<int, 4>(), 0);  // most masks are told by these
  for (int k = 256; k < n && kept <= kFewKeys; k += 1024) count(std::integral_constant<int, 16>(), k);
  return __builtin_amdgcn_readfirstlane(kept);
}

template <typename T, int DP, int RW, int KW, int BN, bool FINE>
__global__ __launch_bounds__(64 * RW * KW, least_waves(sizeof(T) == 2 ? (DP <= 64 && RW > 1 ? 3 : 2) : DP <= 64 ? 2 : 1, RW * KW, KW * 4 * hapi::Tile<T, DP, BN>::BYTES)) void attend_dq_kernel(AttendArgs a) {
  typedef hapi::Tile<T, DP, BN> Tile;
  typedef Loader<T, DP, BN, RW> Load;
  typedef typename Elem<T>::Frag Frag;
  constexpr int KS = DP / 16, DB = DP / 32, NT = BN / 32, STAGE = 2 * Tile::BYTES;
  static_assert(kFewKeys % BN == 0, "whole tiles of listed keys");
  __shared__ __attribute__((aligned(1024))) uint8_t smem[KW * 2 * STAGE];
  __shared__ int list[kFewKeys];  // keys that a mask leaves

  const int t = threadIdx.x, lane = t & 63, col = lane & 31, lh = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(t >> 6), wr = wave % RW, wk = wave / RW;
  const int rows = a.q_len * a.group, tiles = (rows + 32 * RW - 1) / (32 * RW);
  const Place at = place(a, tiles);
  const int tile = at.tile, split = at.split, pair = at.pair, b = at.b, kh = at.kh;
  const int q_valid = clamped(a.q_lens, b, a.q_len), kv_valid = clamped(a.kv_lens, b, a.kv_len);

  const int r = (tile * RW + wr) * 32 + col;
  const int qi = r / a.group, qg = r - qi * a.group;
  const bool counts = qi < q_valid;
  const int64_t h = kh * a.group + qg;
  const T *qp = static_cast<const T *>(a.q) + (int64_t)b * a.q_st[0] + (int64_t)qi * a.q_st[1] + h * a.q_st[2];
  const T *gp = static_cast<const T *>(a.dout) + (int64_t)b * a.g_st[0] + (int64_t)qi * a.g_st[1] + h * a.g_st[2];
  const T *op = static_cast<const T *>(a.o) + (int64_t)b * a.o_st[0] + (int64_t)qi * a.o_st[1] + h * a.o_st[2];
  Frag qf[KS], gf[KS];
  float delta = 0.0f;
#pragma unroll
  for (int ks = 0; ks < KS; ++ks) {
    qf[ks] = row_frag<T>(qp, ks, lh, a.dim, counts);
    gf[ks] = row_frag<T>(gp, ks, lh, a.dim, counts);
    const Frag of = row_frag<T>(op, ks, lh, a.dim, counts);
#pragma unroll
    for (int e = 0; e < 8; ++e) delta = fmaf((float)gf[ks][e], (float)of[e], delta);
  }
  delta += __shfl_xor(delta, 32, 64);
  // a row without a key has m = l = -inf: its p are to be 0
  float m = INFINITY, l2 = 0.0f;
  if (counts) {
    const float2 st = a.stats[((int64_t)b * a.q_len + qi) * a.heads + h];
    if (st.x != -INFINITY) m = st.x, l2 = st.y * kLog2e;
  }

  // Of few keys that a mask leaves of many, only they are brought, one after another in the
  // tiles, as long as 32-bit offsets reach them all: a walk over every tile, which each
  // workgroup made twice, took longer than all keys do (a step with 100 keys left: float32 1 x
  // 20 x 16384, 8 heads of 64, 655 us, now 143, and 118 with all of them; 2 x 300 x 16384, 8 +
  // 2 heads of 128 in bf16, 434, now 215, and 250).
  bool few = kv_valid <= kFewKeys, listed = false;
  int keys = kv_valid;
  if (!few && a.mask) {
    const int kept = kept_keys(a.mask + (int64_t)b * a.kv_len, kv_valid, lane, wave == 0 ? list : nullptr);
    few = kept <= kFewKeys;
    const int64_t ld = a.k_st[1] > a.v_st[1] ? a.k_st[1] : a.v_st[1];
    listed = few && (kv_valid * ld + a.dim) * (int64_t)sizeof(T) < (int64_t)kOob - 16;
    if (listed) keys = kept;
    __syncthreads();
  }
  keys = __builtin_amdgcn_readfirstlane(keys);
  const int key_tiles = tile * RW * 32 < q_valid * a.group ? (keys + BN - 1) / BN : 0;
  Load lk, lv;
  lk.init(a.k_st[1], a.dim, wr, lane);
  lv.init(a.v_st[1], a.dim, wr, lane);
  const T *kp = static_cast<const T *>(a.k) + (int64_t)b * a.k_st[0] + (int64_t)kh * a.k_st[2];
  const T *vp = static_cast<const T *>(a.v) + (int64_t)b * a.v_st[0] + (int64_t)kh * a.v_st[2];
  const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t *)smem + wk * 2 * STAGE;

  // the keys of tile kt that take part
  auto bits_of = [&](int kt) {
    uint64_t keep = key_bits<BN>(keys - (int64_t)kt * BN);
    if (a.mask && !listed) {
      const bool in = (keep >> lane) & 1;
      keep &= __ballot(in && a.mask[(int64_t)b * a.kv_len + (int64_t)kt * BN + (in ? lane : 0)] != 0);
    }
    return keep;
  };
  auto bring = [&](int kt, uint64_t keep, int buf) {
    const uint32_t at = lds0 + buf * STAGE;
    if (listed) {
      Load::gather(kp, a.k_st[1], a.dim, list + kt * BN, at, keep, wr, lane);
      Load::gather(vp, a.v_st[1], a.dim, list + kt * BN, at + Tile::BYTES, keep, wr, lane);
      return;
    }
    lk.issue(kp + (int64_t)kt * BN * a.k_st[1], at, keep, wr);
    lv.issue(vp + (int64_t)kt * BN * a.v_st[1], at + Tile::BYTES, keep, wr);
  };
  auto meet = [&]() {
    wait_loads<0>();
    if constexpr (RW > 1) __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
  };
  // p (dp - less) of 32 keys, 0 for those that take no part
  auto scores = [&](const uint8_t *kt, int n, uint64_t keep, float less) {
    const uint8_t *vt = kt + Tile::BYTES;
    f32x16_t s = zeros(), dp = zeros();
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      if (DP == 96 && ks == KS - 1 && 16 * ks >= a.dim) break;  // heads of 80: five sixths of 96
      s = mma(Tile::by_row(kt, 32 * n, ks, lane), qf[ks], s);
      dp = mma(Tile::by_row(vt, 32 * n, ks, lane), gf[ks], dp);
    }
#pragma unroll
    for (int i = 0; i < 16; ++i) s[i] = __builtin_amdgcn_exp2f(fmaf(s[i] - m, a.c, -l2)) * (dp[i] - less);
    if (keep != kAllKeys<BN>) {
      const uint32_t bits = (uint32_t)(keep >> (32 * n)) >> (4 * lh);
#pragma unroll
      for (int i = 0; i < 16; ++i)
        if (!(bits >> (8 * (i >> 2) + (i & 3)) & 1)) s[i] = 0.0f;
    }
    return s;
  };

  // Of few keys delta is formed again, as the sum of p dp, from all of them: o as it was
  // rounded is off by up to 2^-8, which dp - delta shows the more, the fewer keys there are
  // to average it (bf16, 4 keys: dq off by 0.0030 of its length, so 0.0024; past 128 keys
  // it adds less than a tenth of what rounding dS does), and of one key dS is 0, as
  // its score is formed here as the forward pass formed m.
  if (few) {
    float sum = 0.0f;
    for (int kt = 0; kt < key_tiles; ++kt) {
      const uint64_t keep = bits_of(kt);
      if (keep == 0) continue;
      meet();  // the tile before has been read
      bring(kt, keep, 0);
      meet();
#pragma unroll 1
      for (int n = 0; n < NT; ++n) {
        const f32x16_t s = scores(smem + wk * 2 * STAGE, n, keep, 0.0f);
#pragma unroll
        for (int i = 0; i < 16; ++i) sum += s[i];
      }
    }
    delta = sum + __shfl_xor(sum, 32, 64);
    meet();
  }
  if (split == 0 && wk == 0 && r < rows && lh == 0) a.delta[(int64_t)pair * rows + r] = delta;

  // the split's tiles of keys; wave wk takes every KW-th
  const int t0 = (int)((int64_t)key_tiles * split / a.splits), t1 = (int)((int64_t)key_tiles * (split + 1) / a.splits);
  const int steps = (t1 - t0 + KW - 1) / KW;
  uint64_t keep = 0;
  auto issue = [&](int step) {
    const int kt = t0 + step * KW + wk;
    keep = kt < t1 ? bits_of(kt) : 0;
    if (kt < t1) bring(kt, keep, step & 1);
  };
  f32x16_t dq[DB];
#pragma unroll
  for (int d = 0; d < DB; ++d) dq[d] = zeros();
  if (steps > 0) issue(0);
  for (int step = 0; step < steps; ++step) {
    meet();
    const uint64_t now = keep;
    if (step + 1 < steps) issue(step + 1);
    __builtin_amdgcn_sched_barrier(0);
    if (now == 0) continue;
    const uint8_t *kt = smem + wk * 2 * STAGE + (step & 1) * STAGE;
#pragma unroll 1
    for (int n = 0; n < NT; ++n) {
      f32x16_t s = scores(kt, n, now, delta);
#pragma unroll
      for (int turn = 0; turn < (FINE ? 2 : 1); ++turn) {
        const Frag ds[2] = {operand<T>(s, 0), operand<T>(s, 1)};
#pragma unroll
        for (int d = 0; d < DB; ++d)
          add_products<T>(dq[d], [&](int j) { return Tile::by_column(kt, 32 * n + 16 * j, 32 * d, lane); }, ds);
        if (FINE) keep_rest(s);
      }
    }
  }
  __syncthreads();  // the tiles' place is used again
  if constexpr (KW > 1) {
    // the waves that share rows: the others' sums to the first one, a register of all
    // lanes after another, in the tiles' place
    static_assert((KW - 1) * RW * DB * 16 * 256 <= KW * 2 * STAGE, "the tiles' place");
    float *box = reinterpret_cast<float *>(smem);
    if (wk > 0) {
      float *to = box + ((wk - 1) * RW + wr) * DB * 1024 + lane;
#pragma unroll
      for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) to[(16 * d + i) * 64] = dq[d][i];
    }
    __syncthreads();
#pragma unroll
    for (int w = 0; w < KW - 1; ++w) {
      if (wk > 0) break;
      const float *from = box + (w * RW + wr) * DB * 1024 + lane;
#pragma unroll
      for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) dq[d][i] += from[(16 * d + i) * 64];
    }
    __syncthreads();  // one wave of rows may be ahead of another
  }
  if (KW > 1 && wk > 0) return;
  if (a.splits > 1) {
    if (r >= rows) return;
    float *p = a.part + (((int64_t)split * a.pairs + pair) * rows + r) * a.dim4;
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int e = 32 * d + 8 * q + 4 * lh;
        if (e < a.dim4) *reinterpret_cast<float4 *>(p + e) = make_float4(dq[d][4 * q], dq[d][4 * q + 1], dq[d][4 * q + 2], dq[d][4 * q + 3]);
      }
    return;
  }
  T *y = static_cast<T *>(a.dq) + (int64_t)b * a.dq_st[0] + (int64_t)qi * a.dq_st[1] + h * a.dq_st[2];
  typedef RowsOut<T, DB> Out;
  static_assert(RW * Out::BYTES <= KW * 2 * STAGE, "the tiles' place");
  Out::template store<true>(dq, a.scale, r < rows ? y : nullptr, a.dim, a.dq_vec, smem + wr * Out::BYTES, lane);
}

// How WAVES waves bring tiles of rows, q and dout, to LDS.  The rows are the tokens of a
// group's heads, so a lane's offsets from the tile's first token depend on that row's head
// in the group: the same for every tile where the group's heads divide a tile.
template <typename T, int DP, int BM, int WAVES>
struct RowLoader {
  typedef hapi::Tile<T, DP, BM> Tile;
  static constexpr int LOADS = Tile::DMAS / WAVES;
  static_assert(LOADS * WAVES == Tile::DMAS, "as many DMAs to every wave");
  uint32_t q_off[LOADS], g_off[LOADS];
  __device__ __forceinline__ void offsets(const AttendArgs &a, int g0, int wave, int lane) {
    const uint32_t qt_ld = (uint32_t)a.q_st[1] * sizeof(T), qh_ld = (uint32_t)a.q_st[2] * sizeof(T);
    const uint32_t gt_ld = (uint32_t)a.g_st[1] * sizeof(T), gh_ld = (uint32_t)a.g_st[2] * sizeof(T);
    const uint32_t magic = (1u << 20) / (uint32_t)a.group + 1;  // n / group of n < group + 64 <= 576 as n * magic >> 20
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
      const int slot = (wave * LOADS + i) * 64 + lane, lr = slot / Tile::CPR;
      const uint32_t d = ((slot % Tile::CPR) ^ Tile::swz(lr)) * Tile::V;
      const uint32_t n = (uint32_t)(g0 + lr), di = (n * magic) >> 20, dg = n - di * (uint32_t)a.group;
      q_off[i] = d < (uint32_t)a.dim ? di * qt_ld + dg * qh_ld + d * (uint32_t)sizeof(T) : kOob;
      g_off[i] = d < (uint32_t)a.dim ? di * gt_ld + dg * gh_ld + d * (uint32_t)sizeof(T) : kOob;
    }
  }
  __device__ __forceinline__ void init(const AttendArgs &a, int wave, int lane) { offsets(a, 0, wave, lane); }
  // Row tile rt of `valid` rows to lds; q's rows, then dout's.  qb, gb: the group's first head.
  __device__ __forceinline__ void issue(const AttendArgs &a, const T *qb, const T *gb, int rt, int valid, uint32_t lds, int wave, int lane) {
    const int r0 = rt * BM, i0 = __builtin_amdgcn_readfirstlane(r0 / a.group);
    if (BM % a.group != 0) offsets(a, r0 - i0 * a.group, wave, lane);
    const u32x4_t qs = make_srd(qb + (int64_t)i0 * a.q_st[1]), gs = make_srd(gb + (int64_t)i0 * a.g_st[1]);
    const uint32_t to = __builtin_amdgcn_readfirstlane(lds + wave * LOADS * 1024);
    const int left = valid - r0;
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
      const bool in = ((wave * LOADS + i) * 64 + lane) / Tile::CPR < left;
      lds_dma16(qs, to + i * 1024, in ? q_off[i] : kOob, 0);
      lds_dma16(gs, to + Tile::BYTES + i * 1024, in ? g_off[i] : kOob, 0);
    }
  }
};

// BM rows at a time past 4 x 32 keys.  float32 products add to dk and dv directly: sums by
// themselves as in dq and o take registers that 128-value heads do not have (2 x 1000 x 1000,
// 8 heads: 210 us, so 166) and gain little on what the products' own roundings leave (2 x
// 4096 rows to a key: dk off by 6.6e-7 of its length, so 8.2e-7).
template <typename T, int DP, int BM, bool FINE>
__global__ __launch_bounds__(256, sizeof(T) == 4 ? 1 : (DP <= 64 ? 3 : 2) - (FINE && DP > 32)) void attend_dkv_kernel(AttendArgs a) {
  typedef hapi::Tile<T, DP, BM> Tile;
  typedef typename Elem<T>::Frag Frag;
  constexpr int KS = DP / 16, DB = DP / 32, STAGE = 2 * Tile::BYTES, LOADS = Tile::DMAS / 4;
  static_assert(LOADS * 4 == Tile::DMAS && BM <= 64, "as many DMAs to every wave");
  __shared__ __attribute__((aligned(1024))) uint8_t smem[2 * STAGE];
  __shared__ __attribute__((aligned(16))) float side[2][3][BM];  // less m, l log2(e), delta

  const int t = threadIdx.x, lane = t & 63, col = lane & 31, lh = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(t >> 6);
  const int rows = a.q_len * a.group, tiles = (a.kv_len + 127) / 128;
  const Place at = place(a, tiles);
  const int tile = at.tile, split = at.split, pair = at.pair, b = at.b, kh = at.kh;
  const int q_valid = clamped(a.q_lens, b, a.q_len), kv_valid = clamped(a.kv_lens, b, a.kv_len);

  // this lane's key
  const int key = tile * 128 + wave * 32 + col;
  bool counts = key < kv_valid;
  if (a.mask && counts) counts = a.mask[(int64_t)b * a.kv_len + key] != 0;
  const T *kp = static_cast<const T *>(a.k) + (int64_t)b * a.k_st[0] + (int64_t)key * a.k_st[1] + (int64_t)kh * a.k_st[2];
  const T *vp = static_cast<const T *>(a.v) + (int64_t)b * a.v_st[0] + (int64_t)key * a.v_st[1] + (int64_t)kh * a.v_st[2];
  const int valid = tile * 128 < kv_valid ? q_valid * a.group : 0, row_tiles = (valid + BM - 1) / BM;
  const int t0 = (int)((int64_t)row_tiles * split / a.splits), t1 = (int)((int64_t)row_tiles * (split + 1) / a.splits);
  const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t *)smem;
  const T *qb = static_cast<const T *>(a.q) + (int64_t)b * a.q_st[0] + (int64_t)kh * a.group * a.q_st[2];
  const T *gb = static_cast<const T *>(a.dout) + (int64_t)b * a.g_st[0] + (int64_t)kh * a.group * a.g_st[2];
  RowLoader<T, DP, BM, 4> load;
  load.init(a, wave, lane);
  auto issue = [&](int rt, int buf) { load.issue(a, qb, gb, rt, valid, lds0 + buf * STAGE, wave, lane); };
  // The rows' statistics: looked at only when they are stored, so that they are on their
  // way during a tile's products.
  float2 st;
  float sd;
  auto load_side = [&](int rt) {
    const int r = rt * BM + t;
    st = make_float2(-INFINITY, 0.0f), sd = 0.0f;
    if (t < BM && r < valid) {
      const int qi = r / a.group;
      st = a.stats[((int64_t)b * a.q_len + qi) * a.heads + kh * a.group + (r - qi * a.group)];
      sd = a.delta[(int64_t)pair * rows + r];
    }
  };
  // rows that do not count, and those without a key (m = l = -inf), have p = 0
  auto store_side = [&](int buf) {
    const bool some = st.x != -INFINITY;
    if (t < BM) side[buf][0][t] = some ? -st.x : -INFINITY, side[buf][1][t] = some ? -st.y * kLog2e : 0.0f, side[buf][2][t] = -sd;
  };

  f32x16_t dk[DB], dv[DB];
#pragma unroll
  for (int d = 0; d < DB; ++d) dk[d] = zeros(), dv[d] = zeros();
  Frag kf[KS], vf[KS];
  if (t0 < t1) issue(t0, 0);
#pragma unroll
  for (int ks = 0; ks < KS; ++ks) {
    kf[ks] = row_frag<T>(kp, ks, lh, a.dim, counts);
    vf[ks] = row_frag<T>(vp, ks, lh, a.dim, counts);
  }
  if (t0 < t1) {
    load_side(t0);
    store_side(0);
  }
  for (int rt = t0; rt < t1; ++rt) {
    const int buf = (rt - t0) & 1;
    wait_loads<0>();
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
    if (rt + 1 < t1) {
      load_side(rt + 1);
      issue(rt + 1, buf ^ 1);
    }
    __builtin_amdgcn_sched_barrier(0);
    const uint8_t *qt = smem + buf * STAGE, *gt = qt + Tile::BYTES;
#pragma unroll 1
    for (int n = 0; n < BM / 32; ++n) {
      typedef float f32x4_t __attribute__((ext_vector_type(4)));
      // bf16 scores start from less m, which subtracts it without an instruction
      constexpr bool FROM_M = sizeof(T) == 2;
      f32x16_t s = zeros(), dp = zeros();
      if constexpr (FROM_M) {
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const f32x4_t x = *reinterpret_cast<const f32x4_t *>(&side[buf][0][32 * n + 8 * q + 4 * lh]);
#pragma unroll
          for (int e = 0; e < 4; ++e) s[4 * q + e] = x[e];
        }
      }
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        if (DP == 96 && ks == KS - 1 && 16 * ks >= a.dim) break;
        s = mma(Tile::by_row(qt, 32 * n, ks, lane), kf[ks], s);
        dp = mma(Tile::by_row(gt, 32 * n, ks, lane), vf[ks], dp);
      }
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int at = 32 * n + 8 * q + 4 * lh;
        f32x4_t less_m = {};
        if constexpr (!FROM_M) less_m = *reinterpret_cast<const f32x4_t *>(&side[buf][0][at]);
        const f32x4_t less_l = *reinterpret_cast<const f32x4_t *>(&side[buf][1][at]);
        const f32x4_t less_delta = *reinterpret_cast<const f32x4_t *>(&side[buf][2][at]);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int i = 4 * q + e;
          s[i] = __builtin_amdgcn_exp2f(fmaf(FROM_M ? s[i] : s[i] + less_m[e], a.c, less_l[e]));
          dp[i] = s[i] * (dp[i] + less_delta[e]);
        }
      }
#pragma unroll
      for (int turn = 0; turn < (FINE ? 2 : 1); ++turn) {
        const Frag p[2] = {operand<T>(s, 0), operand<T>(s, 1)}, ds[2] = {operand<T>(dp, 0), operand<T>(dp, 1)};
#pragma unroll
        for (int d = 0; d < DB; ++d)
#pragma unroll
          for (int j = 0; j < 2; ++j) dv[d] = mma(Tile::by_column(gt, 32 * n + 16 * j, 32 * d, lane), p[j], dv[d]);
#pragma unroll
        for (int d = 0; d < DB; ++d)
#pragma unroll
          for (int j = 0; j < 2; ++j) dk[d] = mma(Tile::by_column(qt, 32 * n + 16 * j, 32 * d, lane), ds[j], dk[d]);
        if (FINE) keep_rest(s), keep_rest(dp);
      }
    }
    if (rt + 1 < t1) store_side(buf ^ 1);
  }
  if (!counts) {  // whatever the rows hold (0 times NaN)
#pragma unroll
    for (int d = 0; d < DB; ++d) dk[d] = zeros(), dv[d] = zeros();
  }
  if (a.splits > 1) {
    if (key >= a.kv_len) return;
    const int64_t all = (int64_t)a.pairs * a.kv_len;
    float *p = a.part + (((int64_t)split * 2) * all + (int64_t)pair * a.kv_len + key) * a.dim4;
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int e = 32 * d + 8 * q + 4 * lh;
        if (e >= a.dim4) continue;
        *reinterpret_cast<float4 *>(p + e) = make_float4(dk[d][4 * q], dk[d][4 * q + 1], dk[d][4 * q + 2], dk[d][4 * q + 3]);
        *reinterpret_cast<float4 *>(p + all * a.dim4 + e) = make_float4(dv[d][4 * q], dv[d][4 * q + 1], dv[d][4 * q + 2], dv[d][4 * q + 3]);
      }
    return;
  }
  T *yk = static_cast<T *>(a.dk) + (int64_t)b * a.dk_st[0] + (int64_t)key * a.dk_st[1] + (int64_t)kh * a.dk_st[2];
  T *yv = static_cast<T *>(a.dv) + (int64_t)b * a.dv_st[0] + (int64_t)key * a.dv_st[1] + (int64_t)kh * a.dv_st[2];
  typedef RowsOut<T, DB> Out;
  constexpr int HALF = 2 * STAGE >= 8 * Out::BYTES ? 4 * Out::BYTES : 0;  // places of their own, or one after the other
  static_assert(4 * Out::BYTES <= 2 * STAGE, "the tiles' place");
  __syncthreads();
  Out::template store<false>(dk, a.scale, key < a.kv_len ? yk : nullptr, a.dim, a.dk_vec, smem + wave * Out::BYTES, lane);
  Out::template store<false>(dv, 1.0f, key < a.kv_len ? yv : nullptr, a.dim, a.dv_vec, smem + HALF + wave * Out::BYTES, lane);
}

// dk and dv of 128-value heads in 16 bits.  A wave that kept 32 keys' k, v, dk and dv would
// take 366 registers, one wave to a SIMD, and dk and dv in kernels of their own form the
// scores and their exponentials twice (2 x 4096 x 4096, 16 + 4 heads: 890 us, 415 + 300
// us).  Here two waves share 32 keys: each forms P and dS of one half of a tile's 64 rows,
// passes them on in LDS as operands, and sums half the values of dk and dv over all 64.
// A tile's products with P and dS are those of the step after the one that forms them, so
// that they stand beside the next exponentials, which need nothing of them.
// FINE: a tile has two turns, the second one's P and dS are what rounding the first one's
// left; LDS has no place for both at once.
template <bool FINE>
__global__ __launch_bounds__(512, 2) void attend_dkv_pair_kernel(AttendArgs a) {
  typedef uint16_t T;
  constexpr int DP = 128, BM = 64, KS = DP / 16, DB = 2, WAVES = 8;
  typedef hapi::Tile<T, DP, BM> Tile;
  typedef typename Elem<T>::Frag Frag;
  constexpr int STAGE = 2 * Tile::BYTES, LOADS = Tile::DMAS / WAVES;
  static_assert(LOADS * WAVES == Tile::DMAS, "as many DMAs to every wave");
  __shared__ __attribute__((aligned(1024))) uint8_t smem[3 * STAGE];
  // P and dS: [key group][half of the rows][16 rows][P, dS][lane]
  __shared__ __attribute__((aligned(1024))) uint8_t passed[4 * 2 * 2 * 2 * 1024];
  __shared__ __attribute__((aligned(16))) float side[2][3][BM];  // less m, l log2(e), delta

  const int t = threadIdx.x, lane = t & 63, col = lane & 31, lh = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(t >> 6), kg = wave & 3, half = wave >> 2;
  const int rows = a.q_len * a.group, tiles = (a.kv_len + 127) / 128;
  const Place at = place(a, tiles);
  const int tile = at.tile, split = at.split, pair = at.pair, b = at.b, kh = at.kh;
  const int q_valid = clamped(a.q_lens, b, a.q_len), kv_valid = clamped(a.kv_lens, b, a.kv_len);

  // this lane's key
  const int key = tile * 128 + kg * 32 + col;
  bool counts = key < kv_valid;
  if (a.mask && counts) counts = a.mask[(int64_t)b * a.kv_len + key] != 0;
  const T *kp = static_cast<const T *>(a.k) + (int64_t)b * a.k_st[0] + (int64_t)key * a.k_st[1] + (int64_t)kh * a.k_st[2];
  const T *vp = static_cast<const T *>(a.v) + (int64_t)b * a.v_st[0] + (int64_t)key * a.v_st[1] + (int64_t)kh * a.v_st[2];

  const int valid = tile * 128 < kv_valid ? q_valid * a.group : 0, row_tiles = (valid + BM - 1) / BM;
  const int t0 = (int)((int64_t)row_tiles * split / a.splits), t1 = (int)((int64_t)row_tiles * (split + 1) / a.splits);
  const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t *)smem;
  const T *qb = static_cast<const T *>(a.q) + (int64_t)b * a.q_st[0] + (int64_t)kh * a.group * a.q_st[2];
  const T *gb = static_cast<const T *>(a.dout) + (int64_t)b * a.g_st[0] + (int64_t)kh * a.group * a.g_st[2];
  RowLoader<T, DP, BM, WAVES> load;
  load.init(a, wave, lane);
  auto issue = [&](int rt, int buf) { load.issue(a, qb, gb, rt, valid, lds0 + buf * STAGE, wave, lane); };
  float2 st;
  float sd;
  auto load_side = [&](int rt) {
    const int r = rt * BM + t;
    st = make_float2(-INFINITY, 0.0f), sd = 0.0f;
    if (t < BM && r < valid) {
      const int qi = r / a.group;
      st = a.stats[((int64_t)b * a.q_len + qi) * a.heads + kh * a.group + (r - qi * a.group)];
      sd = a.delta[(int64_t)pair * rows + r];
    }
  };
  auto store_side = [&](int buf) {
    const bool some = st.x != -INFINITY;
    if (t < BM) side[buf][0][t] = some ? -st.x : -INFINITY, side[buf][1][t] = some ? -st.y * kLog2e : 0.0f, side[buf][2][t] = -sd;
  };

  f32x16_t dk[DB], dv[DB];
#pragma unroll
  for (int d = 0; d < DB; ++d) dk[d] = zeros(), dv[d] = zeros();
  Frag kf[KS], vf[KS];
  if (t0 < t1) issue(t0, 0);
#pragma unroll
  for (int ks = 0; ks < KS; ++ks) {
    kf[ks] = row_frag<T>(kp, ks, lh, a.dim, counts);
    vf[ks] = row_frag<T>(vp, ks, lh, a.dim, counts);
  }
  if (t0 < t1) {
    load_side(t0);
    store_side(0);
  }
  typedef float f32x4_t __attribute__((ext_vector_type(4)));
  f32x16_t s, dp;  // scores and dP of this wave's half, then P and dS
  uint8_t *const mine = passed + ((kg * 2 + half) * 4) * 1024 + lane * 16;
  auto pass = [&]() {
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      *reinterpret_cast<Frag *>(mine + (2 * j) * 1024) = operand<T>(s, j);
      *reinterpret_cast<Frag *>(mine + (2 * j + 1) * 1024) = operand<T>(dp, j);
    }
  };
  // A step: FORMS the scores of tile `buf` and the probabilities, SUMS the last tile's
  // products.  What a product reads is read two products ahead, and two exponentials'
  // arithmetic stands behind each pair of the sums' products: left to itself the compiler
  // reads right before each product, and puts all exponentials behind the last one.
  auto step = [&](auto forms, auto sums, int buf, int sb, int last) {
    constexpr bool FORMS = decltype(forms)::value, SUMS = decltype(sums)::value;
    constexpr int F = FORMS ? KS : 0, N = F + (SUMS ? 8 : 0), AHEAD = 1;
    const uint8_t *qt = smem + buf * STAGE, *gt = qt + Tile::BYTES, *q_last = smem + last * STAGE, *g_last = q_last + Tile::BYTES;
    Frag row_q[KS], row_g[KS], col_q[8], col_g[8], p[4], ds[4];
    f32x4_t less_l[4], less_delta[4];
    auto rows_of = [&](int q) {
      const int at = 32 * half + 8 * q + 4 * lh;
      less_l[q] = *reinterpret_cast<const f32x4_t *>(&side[sb][1][at]);
      less_delta[q] = *reinterpret_cast<const f32x4_t *>(&side[sb][2][at]);
    };
    auto read = [&](int i) {
      if (i < F) {
        row_q[i] = Tile::by_row(qt, 32 * half, i, lane);
        row_g[i] = Tile::by_row(gt, 32 * half, i, lane);
        return;
      }
      const int c = i - F, r = c >> 1, d = 64 * half + 32 * (c & 1);  // 16 rows from 16 r on, 32 values
      if ((c & 1) == 0) {
        const uint8_t *from = passed + ((kg * 2 + (r >> 1)) * 4 + 2 * (r & 1)) * 1024 + lane * 16;
        p[r] = *reinterpret_cast<const Frag *>(from);
        ds[r] = *reinterpret_cast<const Frag *>(from + 1024);
      }
      col_g[c] = Tile::by_column(g_last, 16 * r, d, lane);
      col_q[c] = Tile::by_column(q_last, 16 * r, d, lane);
    };
    auto probability = [&](int i) {
      s[i] = __builtin_amdgcn_exp2f(fmaf(s[i], a.c, less_l[i >> 2][i & 3]));
      dp[i] = s[i] * (dp[i] + less_delta[i >> 2][i & 3]);
    };
    if (FORMS) {  // scores start from less m
      dp = zeros();
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const f32x4_t x = *reinterpret_cast<const f32x4_t *>(&side[sb][0][32 * half + 8 * q + 4 * lh]);
#pragma unroll
        for (int e = 0; e < 4; ++e) s[4 * q + e] = x[e];
      }
    }
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) read(i);
#pragma unroll
    for (int i = 0; i < N; ++i) {
      if (i + AHEAD < N) read(i + AHEAD);
      __builtin_amdgcn_sched_barrier(0);
      if (i < F) {
        s = mma(row_q[i], kf[i], s);
        dp = mma(row_g[i], vf[i], dp);
      } else {
        const int c = i - F;
        if (FORMS && (c & 1) == 0) rows_of(c >> 1);
        dv[c & 1] = mma(col_g[c], p[c >> 1], dv[c & 1]);
        dk[c & 1] = mma(col_q[c], ds[c >> 1], dk[c & 1]);
        if (FORMS) probability(2 * c), probability(2 * c + 1);
      }
      __builtin_amdgcn_sched_barrier(0);
    }
    if (FORMS && !SUMS) {
#pragma unroll
      for (int q = 0; q < 4; ++q) rows_of(q);
#pragma unroll
      for (int i = 0; i < 16; ++i) probability(i);
    }
  };
  auto meet = [&]() {
    wait_loads<0>();
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
  };
  auto meet_lds = [&]() {  // DMAs and loads stay in flight
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt((63 & 15) | ((63 >> 4) << 14) | (7 << 4));
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
  };
  const std::true_type yes;
  const std::false_type no;
  constexpr int MORE = FINE;
  const int u0 = t0 << MORE, u1 = t1 << MORE;  // turns
  int buf = 0;  // of the turn's tile
  for (int u = u0; u < u1; ++u) {
    const int next = buf == 2 ? 0 : buf + 1, last = buf == 0 ? 2 : buf - 1;
    meet();  // the tile is there; so are the last turn's P and dS
    if (u + 1 < u1) {
      load_side((u + 1) >> MORE);
      issue((u + 1) >> MORE, next);
    }
    __builtin_amdgcn_sched_barrier(0);
    if (u > u0) step(yes, yes, buf, (u - u0) & 1, last);
    else step(yes, no, buf, 0, last);
    if (u & MORE) keep_rest(s), keep_rest(dp);
    meet_lds();  // all have read the last turn's P and dS
    pass();
    if (u + 1 < u1) store_side((u + 1 - u0) & 1);
    buf = next;
  }
  meet();
  if (t0 < t1) step(no, yes, 0, 0, buf == 0 ? 2 : buf - 1);
  if (!counts) {  // whatever the rows hold (0 times NaN)
#pragma unroll
    for (int d = 0; d < DB; ++d) dk[d] = zeros(), dv[d] = zeros();
  }
  const int d0 = 64 * half;
  if (a.splits > 1) {
    if (key >= a.kv_len) return;
    const int64_t all = (int64_t)a.pairs * a.kv_len;
    float *p = a.part + (((int64_t)split * 2) * all + (int64_t)pair * a.kv_len + key) * a.dim4;
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int e = d0 + 32 * d + 8 * q + 4 * lh;
        if (e >= a.dim4) continue;
        *reinterpret_cast<float4 *>(p + e) = make_float4(dk[d][4 * q], dk[d][4 * q + 1], dk[d][4 * q + 2], dk[d][4 * q + 3]);
        *reinterpret_cast<float4 *>(p + all * a.dim4 + e) = make_float4(dv[d][4 * q], dv[d][4 * q + 1], dv[d][4 * q + 2], dv[d][4 * q + 3]);
      }
    return;
  }
  T *yk = static_cast<T *>(a.dk) + (int64_t)b * a.dk_st[0] + (int64_t)key * a.dk_st[1] + (int64_t)kh * a.dk_st[2] + d0;
  T *yv = static_cast<T *>(a.dv) + (int64_t)b * a.dv_st[0] + (int64_t)key * a.dv_st[1] + (int64_t)kh * a.dv_st[2] + d0;
  typedef RowsOut<T, DB> Out;
  static_assert(2 * WAVES * Out::BYTES <= 3 * STAGE, "the tiles' place");
  __syncthreads();
  Out::template store<false>(dk, a.scale, key < a.kv_len ? yk : nullptr, a.dim - d0, a.dk_vec, smem + wave * Out::BYTES, lane);
  Out::template store<false>(dv, 1.0f, key < a.kv_len ? yv : nullptr, a.dim - d0, a.dv_vec, smem + (WAVES + wave) * Out::BYTES, lane);
}

// dq, dk and dv of few rows, 16-bit heads of up to 64 values: a workgroup has all of the
// rows of a group's heads, q and dout in LDS, so that a key's scores are formed once and
// k and v are read once, five products and not seven.  A wave takes blocks of 32 keys, k
// in LDS and v in registers, forms P and dS as dk's and dv's kernel does, and has a
// block's dk and dv when it has been through the rows.  dS goes through LDS to be the
// operand of dq^T = K^T dS^T, which a wave sums over its keys and the workgroup over its
// waves.  A wave's tiles are its own: none waits for another before the last sum.
// 128 x 64 x 197, 12 heads of 64: 57 us, 3.6 TB/s of what it has to move (dq's kernel and
// dk's and dv's: 31 + 48 us); registers leave two workgroups a CU, whose loads and stores
// do not cover each other's products wholly.
template <int DP, int RB, bool FINE>
__global__ __launch_bounds__(256, FINE && DP * RB > 64 ? 1 : 2) void attend_few_rows_kernel(AttendArgs a) {
  typedef uint16_t T;
  typedef typename Elem<T>::Frag Frag;
  typedef float f32x4_t __attribute__((ext_vector_type(4)));
  constexpr int ROWS = 32 * RB, KS = DP / 16, DB = DP / 32, WAVES = 4;
  typedef hapi::Tile<T, DP, ROWS> Rows;
  typedef hapi::Tile<T, DP, 32> Keys;
  typedef hapi::Tile<T, ROWS, 32> Turned;  // dS, a key's rows side by side
  constexpr int TURNS = FINE ? 2 : 1;  // dS, and what its rounding left
  constexpr int OWN = 2 * Keys::BYTES + TURNS * Turned::BYTES;  // a wave's: keys, dS, keys
  __shared__ __attribute__((aligned(1024))) uint8_t smem[2 * Rows::BYTES + WAVES * OWN];
  __shared__ __attribute__((aligned(16))) float side[3][ROWS];  // less m, less l log2(e), less delta
  __shared__ float sums[WAVES][ROWS];

  const int t = threadIdx.x, lane = t & 63, col = lane & 31, lh = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(t >> 6);
  const int rows = a.q_len * a.group;
  const Place at = place(a, 1);
  const int b = at.b, kh = at.kh;
  const int q_valid = clamped(a.q_lens, b, a.q_len), kv_valid = clamped(a.kv_lens, b, a.kv_len);
  const int valid = q_valid * a.group, key_blocks = (a.kv_len + 31) / 32, some_blocks = valid > 0 ? (kv_valid + 31) / 32 : 0;
  const T *kb = static_cast<const T *>(a.k) + (int64_t)b * a.k_st[0] + (int64_t)kh * a.k_st[2];
  const T *vb = static_cast<const T *>(a.v) + (int64_t)b * a.v_st[0] + (int64_t)kh * a.v_st[2];
  const T *qb = static_cast<const T *>(a.q) + (int64_t)b * a.q_st[0] + (int64_t)kh * a.group * a.q_st[2];
  const T *gb = static_cast<const T *>(a.dout) + (int64_t)b * a.g_st[0] + (int64_t)kh * a.group * a.g_st[2];
  const T *ob = static_cast<const T *>(a.o) + (int64_t)b * a.o_st[0] + (int64_t)kh * a.group * a.o_st[2];
  const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t *)smem;
  uint8_t *const own = smem + 2 * Rows::BYTES + wave * OWN;
  const uint32_t own0 = lds0 + 2 * Rows::BYTES + wave * OWN;
  constexpr int TURN = Keys::BYTES, SECOND = Keys::BYTES + TURNS * Turned::BYTES;

  Loader<T, DP, 32, 1> load;
  load.init(a.k_st[1], a.dim, 0, lane);
  Frag vf[KS], vn[KS];  // v of the block, and of the next
  bool counts = false, counts_next = false;  // this lane's key of the block, and of the next
  auto bring = [&](int n, int buf) {
    const int key = n * 32 + col;
    counts_next = key < kv_valid;
    if (a.mask && counts_next) counts_next = a.mask[(int64_t)b * a.kv_len + key] != 0;
    load.issue(kb + (int64_t)n * 32 * a.k_st[1], own0 + (buf ? SECOND : 0), __ballot(counts_next), 0);
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) vn[ks] = row_frag<T>(vb + (int64_t)key * a.v_st[1], ks, lh, a.dim, counts_next);
    __builtin_amdgcn_sched_barrier(0);
  };
  if (some_blocks > 0) {
    constexpr int LOADERS = Rows::DMAS < WAVES ? Rows::DMAS : WAVES;
    if (wave < LOADERS) {
      RowLoader<T, DP, ROWS, LOADERS> rl;
      rl.init(a, wave, lane);
      rl.issue(a, qb, gb, 0, valid, lds0, wave, lane);
    }
  }
  if (wave < some_blocks) bring(wave, 0);
  // the rows' statistics and delta; rows that do not count, and those without a key (m = l =
  // -inf), have p = 0
  constexpr int PER = 256 / ROWS < DP / 8 ? 256 / ROWS : DP / 8;  // threads of a row
  if (t < ROWS * PER) {
    const int r = t / PER, qi = r / a.group, qg = r - qi * a.group;
    const bool there = r < valid;
    const T *gp = gb + (int64_t)qi * a.g_st[1] + (int64_t)qg * a.g_st[2], *op = ob + (int64_t)qi * a.o_st[1] + (int64_t)qg * a.o_st[2];
    float2 st = make_float2(-INFINITY, 0.0f);
    if (there) st = a.stats[((int64_t)b * a.q_len + qi) * a.heads + kh * a.group + qg];
    float delta = 0.0f;
#pragma unroll
    for (int i = 0; i < DP / 8 / PER; ++i) {
      const int d = t % PER + i * PER;  // 8 values
      const Frag g = row_frag<T>(gp, d >> 1, d & 1, a.dim, there), o = row_frag<T>(op, d >> 1, d & 1, a.dim, there);
#pragma unroll
      for (int e = 0; e < 8; ++e) delta = fmaf((float)g[e], (float)o[e], delta);
    }
#pragma unroll
    for (int x = 1; x < PER; x *= 2) delta += __shfl_xor(delta, x, 64);
    if (t % PER == 0) {
      const bool some = st.x != -INFINITY;
      side[0][r] = some ? -st.x : -INFINITY;
      side[1][r] = some ? -st.y * kLog2e : 0.0f;
      side[2][r] = -delta;
    }
  }
  wait_loads<0>();
  __syncthreads();

  const uint8_t *qt = smem, *gt = smem + Rows::BYTES;
  f32x16_t s, dp;
  // P and dP of rows 32 n on; scores start from less m, or from 0 as in the forward pass
  auto scores = [&](auto from_m, int n, const uint8_t *kt) {
    dp = zeros();
    s = zeros();
    if constexpr (decltype(from_m)::value) {
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const f32x4_t x = *reinterpret_cast<const f32x4_t *>(&side[0][32 * n + 8 * q + 4 * lh]);
#pragma unroll
        for (int e = 0; e < 4; ++e) s[4 * q + e] = x[e];
      }
    }
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      s = mma(Rows::by_row(qt, 32 * n, ks, lane), Keys::by_row(kt, 0, ks, lane), s);
      dp = mma(Rows::by_row(gt, 32 * n, ks, lane), vf[ks], dp);
    }
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const f32x4_t less_l = *reinterpret_cast<const f32x4_t *>(&side[1][32 * n + 8 * q + 4 * lh]);
      f32x4_t less_m = {};
      if constexpr (!decltype(from_m)::value) less_m = *reinterpret_cast<const f32x4_t *>(&side[0][32 * n + 8 * q + 4 * lh]);
#pragma unroll
      for (int e = 0; e < 4; ++e) s[4 * q + e] = __builtin_amdgcn_exp2f(fmaf(s[4 * q + e] + less_m[e], a.c, less_l[e]));
    }
  };

  auto take = [&]() {
    counts = counts_next;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) vf[ks] = vn[ks];
  };

  // of few keys delta is the sum of p dp, as in dq's kernel
  bool few = kv_valid <= kFewKeys;
  if (!few && a.mask) few = kept_keys(a.mask + (int64_t)b * a.kv_len, kv_valid, lane, nullptr) <= kFewKeys;
  if (few && some_blocks > 0) {
    f32x16_t sum[RB];
#pragma unroll
    for (int n = 0; n < RB; ++n) sum[n] = zeros();
    for (int kn = wave; kn < some_blocks; kn += WAVES) {
      if (kn > wave) {
        wait_loads<0>();  // the block before has been read
        bring(kn, 0);
      }
      wait_loads<0>();
      take();
      if (!__any(counts)) continue;  // a mask leaves none of the block
#pragma unroll
      for (int n = 0; n < RB; ++n) {
        scores(std::false_type(), n, own);
#pragma unroll
        for (int i = 0; i < 16; ++i) sum[n][i] += counts ? s[i] * dp[i] : 0.0f;
      }
    }
#pragma unroll
    for (int n = 0; n < RB; ++n)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
#pragma unroll
        for (int x = 1; x < 32; x *= 2) sum[n][i] += __shfl_xor(sum[n][i], x, 64);
        if (col == 0) sums[wave][32 * n + 8 * (i >> 2) + 4 * lh + (i & 3)] = sum[n][i];
      }
    if (some_blocks > WAVES && wave < some_blocks) {
      wait_loads<0>();
      bring(wave, 0);
    }
    __syncthreads();
    if (t < ROWS) side[2][t] = -(((sums[0][t] + sums[1][t]) + sums[2][t]) + sums[3][t]);
    wait_loads<0>();
    __syncthreads();
  }

  f32x16_t dq[RB][DB];
#pragma unroll
  for (int n = 0; n < RB; ++n)
#pragma unroll
    for (int d = 0; d < DB; ++d) dq[n][d] = zeros();
  T *const yk = static_cast<T *>(a.dk) + (int64_t)b * a.dk_st[0] + (int64_t)kh * a.dk_st[2];
  T *const yv = static_cast<T *>(a.dv) + (int64_t)b * a.dv_st[0] + (int64_t)kh * a.dv_st[2];
  int buf = 0;
  for (int kn = wave; kn < key_blocks; kn += WAVES, buf ^= 1) {
    f32x16_t dk[DB], dv[DB];
#pragma unroll
    for (int d = 0; d < DB; ++d) dk[d] = zeros(), dv[d] = zeros();
    if (kn < some_blocks) {
      take();
      if (kn + WAVES < some_blocks) bring(kn + WAVES, buf ^ 1);
      const uint8_t *kt = own + (buf ? SECOND : 0);
#pragma unroll
      for (int n = 0; n < RB; ++n) {
        scores(std::true_type(), n, kt);
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const f32x4_t less_delta = *reinterpret_cast<const f32x4_t *>(&side[2][32 * n + 8 * q + 4 * lh]);
#pragma unroll
          for (int e = 0; e < 4; ++e) dp[4 * q + e] = s[4 * q + e] * (dp[4 * q + e] + less_delta[e]);
        }
#pragma unroll
        for (int turn = 0; turn < TURNS; ++turn) {
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            const Frag p = operand<T>(s, j), ds = operand<T>(dp, j);
            // rows 32 n + 16 j + 4 lh + 0 .. 3 and 8 more; a key that takes no part has none
            union {
              Frag f;
              uint2 h[2];
            } u = {ds};
            uint8_t *to = own + TURN + turn * Turned::BYTES + col * Turned::PITCH + 8 * lh;
#pragma unroll
            for (int h = 0; h < 2; ++h)
              *reinterpret_cast<uint2 *>(to + ((4 * n + 2 * j + h) ^ Turned::swz(col)) * 16) = counts ? u.h[h] : make_uint2(0, 0);
#pragma unroll
            for (int d = 0; d < DB; ++d) {
              dv[d] = mma(Rows::by_column(gt, 32 * n + 16 * j, 32 * d, lane), p, dv[d]);
              dk[d] = mma(Rows::by_column(qt, 32 * n + 16 * j, 32 * d, lane), ds, dk[d]);
            }
          }
          if (FINE) keep_rest(s), keep_rest(dp);
        }
      }
      asm volatile("" ::: "memory");  // a wave's LDS accesses are in order
#pragma unroll
      for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int d = 0; d < DB; ++d) {
          const Frag kc = Keys::by_column(kt, 16 * j, 32 * d, lane);
#pragma unroll
          for (int turn = 0; turn < TURNS; ++turn)
#pragma unroll
            for (int n = 0; n < RB; ++n)
              dq[n][d] = mma(kc, Turned::by_column(own + TURN + turn * Turned::BYTES, 16 * j, 32 * n, lane), dq[n][d]);
        }
      wait_loads<0>();  // the next block's: not for the stores that follow
      if (!counts) {  // whatever the rows hold (0 times NaN)
#pragma unroll
        for (int d = 0; d < DB; ++d) dk[d] = zeros(), dv[d] = zeros();
      }
    }
    // turned where this block's keys and dS were
    const int key = kn * 32 + col;
    uint8_t *turn = own + (buf ? TURN : 0);
    typedef RowsOut<T, DB> Out;
    static_assert(Out::BYTES <= Keys::BYTES + Turned::BYTES, "the tiles' place");
    Out::template store<false>(dk, a.scale, key < a.kv_len ? yk + (int64_t)key * a.dk_st[1] : nullptr, a.dim, a.dk_vec, turn, lane);
    asm volatile("" ::: "memory");
    Out::template store<false>(dv, 1.0f, key < a.kv_len ? yv + (int64_t)key * a.dv_st[1] : nullptr, a.dim, a.dv_vec, turn, lane);
    asm volatile("" ::: "memory");
  }

  // dq: the waves' sums, a register of all lanes after another, in the tiles' place
  static_assert(WAVES * RB * DB * 4096 <= sizeof(smem) && RB * DB <= WAVES, "the tiles' place");
  float *const box = reinterpret_cast<float *>(smem);
  __syncthreads();
#pragma unroll
  for (int n = 0; n < RB; ++n)
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
      for (int i = 0; i < 16; ++i) box[((wave * RB + n) * DB + d) * 1024 + i * 64 + lane] = dq[n][d][i];
  __syncthreads();
  if (wave >= RB * DB) return;
  const int n = wave / DB, d = wave % DB, r = 32 * n + col;  // this wave's block
  f32x16_t all[1];
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const float *from = box + wave * 1024 + i * 64 + lane;
    all[0][i] = ((from[0] + from[RB * DB * 1024]) + from[2 * RB * DB * 1024]) + from[3 * RB * DB * 1024];
  }
  const int qi = r / a.group, qg = r - qi * a.group;
  T *y = static_cast<T *>(a.dq) + (int64_t)b * a.dq_st[0] + (int64_t)qi * a.dq_st[1] + (int64_t)(kh * a.group + qg) * a.dq_st[2] + 32 * d;
  asm volatile("" ::: "memory");
  // turned in the place of the first wave's part, which this wave alone has read
  typedef RowsOut<T, 1> Out;
  static_assert(Out::BYTES <= 4096, "a block's place");
  Out::template store<false>(all, a.scale, r < rows ? y : nullptr, a.dim - 32 * d, a.dq_vec, smem + wave * 4096, lane);
}

// Adds the parts: a thread has four values of a row of dq, or of a key's dk (blockIdx.y
// = 0) or dv.
template <typename T, bool DQ>
__global__ __launch_bounds__(256) void attend_sum_kernel(AttendArgs a) {
  const int per = a.dim4 / 4;
  const int64_t rows = DQ ? (int64_t)a.q_len * a.group : a.kv_len, all = rows * a.pairs;
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int64_t row = i / per;
  if (row >= all) return;
  const int d = (int)(i - row * per) * 4;
  const int which = blockIdx.y, each = DQ ? 1 : 2;
  float o[4] = {};
  for (int p0 = 0; p0 < a.splits; p0 += 8) {  // 8 loads in flight
    float4 v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int p = p0 + i < a.splits ? p0 + i : a.splits - 1;
      v[i] = *reinterpret_cast<const float4 *>(a.part + ((p * each + which) * all + row) * a.dim4 + d);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float w = p0 + i < a.splits ? 1.0f : 0.0f;
      o[0] = fmaf(v[i].x, w, o[0]);
      o[1] = fmaf(v[i].y, w, o[1]);
      o[2] = fmaf(v[i].z, w, o[2]);
      o[3] = fmaf(v[i].w, w, o[3]);
    }
  }
  const float scale = DQ || which == 0 ? a.scale : 1.0f;
  const int pair = (int)(row / rows), r = (int)(row - pair * rows), b = pair / a.kv_heads, kh = pair - b * a.kv_heads;
  T *y;
  bool vec;
  if (DQ) {
    const int qi = r / a.group;
    y = static_cast<T *>(a.dq) + (int64_t)b * a.dq_st[0] + (int64_t)qi * a.dq_st[1] + (int64_t)(kh * a.group + r - qi * a.group) * a.dq_st[2];
    vec = a.dq_vec & 1;
  } else {
    const int64_t *st = which ? a.dv_st : a.dk_st;
    y = static_cast<T *>(which ? a.dv : a.dk) + (int64_t)b * st[0] + (int64_t)r * st[1] + (int64_t)kh * st[2];
    vec = (which ? a.dv_vec : a.dk_vec) & 1;
  }
  store4<T>(y, d, a.dim, vec, o[0] * scale, o[1] * scale, o[2] * scale, o[3] * scale);
}

template <typename T, int DP, int RW>
hipError_t dq(const AttendArgs &a, hipStream_t s) {
  constexpr int KW = attend_key_waves(sizeof(T), DP, RW), BN = attend_tile_keys(sizeof(T), DP, KW);
  const int64_t rows = (int64_t)a.q_len * a.group, tiles = ceil_div(rows, 32 * RW);
  const dim3 grid((uint32_t)(tiles * a.splits * a.pairs)), block(64 * RW * KW);
  if constexpr (sizeof(T) == 2) {
    if (attend_fine(a)) hapi_launch(attend_dq_kernel<T, DP, RW, KW, BN, true>, grid, block, 0, s, a);
    else hapi_launch(attend_dq_kernel<T, DP, RW, KW, BN, false>, grid, block, 0, s, a);
  } else {
    hapi_launch(attend_dq_kernel<T, DP, RW, KW, BN, false>, grid, block, 0, s, a);
  }
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.splits == 1) return e;
  hapi_launch(attend_sum_kernel<T, true>, dim3((uint32_t)ceil_div(rows * a.pairs * (a.dim4 / 4), 256)), dim3(256), 0, s, a);
  return hipGetLastError();
}
template <typename T, int DP>
hipError_t dq_rows(const AttendArgs &a, hipStream_t s) {
  const int rw = attend_row_waves((int64_t)a.q_len * a.group);
  return rw == 4 ? dq<T, DP, 4>(a, s) : rw == 2 ? dq<T, DP, 2>(a, s) : dq<T, DP, 1>(a, s);
}
template <typename T>
hipError_t dq_dim(const AttendArgs &a, hipStream_t s) {
  if (a.dim <= 32) return dq_rows<T, 32>(a, s);
  if (a.dim <= 64) return dq_rows<T, 64>(a, s);
  if (a.dim <= 96) return dq_rows<T, 96>(a, s);
  return dq_rows<T, 128>(a, s);
}

template <typename T, int DP>
hipError_t dkv(const AttendArgs &a, hipStream_t s) {
  constexpr int BM = sizeof(T) == 2 ? 64 : 32;
  const dim3 grid((uint32_t)(ceil_div(a.kv_len, 128) * a.splits * a.pairs)), block(256);
  if constexpr (sizeof(T) == 2 && DP == 128) {
    if (attend_fine(a)) hapi_launch(attend_dkv_pair_kernel<true>, grid, dim3(512), 0, s, a);
    else hapi_launch(attend_dkv_pair_kernel<false>, grid, dim3(512), 0, s, a);
  } else if constexpr (sizeof(T) == 2) {
    if (attend_fine(a)) hapi_launch(attend_dkv_kernel<T, DP, BM, true>, grid, block, 0, s, a);
    else hapi_launch(attend_dkv_kernel<T, DP, BM, false>, grid, block, 0, s, a);
  } else {
    hapi_launch(attend_dkv_kernel<T, DP, BM, false>, grid, block, 0, s, a);
  }
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.splits == 1) return e;
  hapi_launch(attend_sum_kernel<T, false>, dim3((uint32_t)ceil_div((int64_t)a.kv_len * a.pairs * (a.dim4 / 4), 256), 2), dim3(256), 0, s, a);
  return hipGetLastError();
}
template <typename T>
hipError_t dkv_dim(const AttendArgs &a, hipStream_t s) {
  if (a.dim <= 32) return dkv<T, 32>(a, s);
  if (a.dim <= 64) return dkv<T, 64>(a, s);
  if (a.dim <= 96) return dkv<T, 96>(a, s);
  return dkv<T, 128>(a, s);
}

template <int DP>
hipError_t few_rows(const AttendArgs &a, hipStream_t s) {
  const dim3 grid((uint32_t)a.pairs), block(256);
  const bool one = a.q_len * a.group <= 32, fine = attend_fine(a);
  if (one && fine) hapi_launch(attend_few_rows_kernel<DP, 1, true>, grid, block, 0, s, a);
  else if (one) hapi_launch(attend_few_rows_kernel<DP, 1, false>, grid, block, 0, s, a);
  else if (fine) hapi_launch(attend_few_rows_kernel<DP, 2, true>, grid, block, 0, s, a);
  else hapi_launch(attend_few_rows_kernel<DP, 2, false>, grid, block, 0, s, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_attend_dq(bool bf16, const AttendArgs &a, hipStream_t s) {
  return bf16 ? dq_dim<uint16_t>(a, s) : dq_dim<float>(a, s);
}
hipError_t launch_attend_few_rows(const AttendArgs &a, hipStream_t s) {
  return a.dim <= 32 ? few_rows<32>(a, s) : few_rows<64>(a, s);
}
hipError_t launch_attend_dkv(bool bf16, const AttendArgs &a, hipStream_t s) {
  return bf16 ? dkv_dim<uint16_t>(a, s) : dkv_dim<float>(a, s);
}

}  // namespace hapi
