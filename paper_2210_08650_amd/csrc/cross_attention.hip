// Cross attention, forward: o = softmax(scale q k^T) v over the keys that take part.
//
// The query heads that share a key head are the rows of one problem (row r: token
// r / group, head r % group), so keys and values are read once for all of them and a
// single token's heads fill a tile together.  A wave owns 32 rows, its queries in
// registers; keys and values pass through LDS in tiles that the waves of a workgroup
// share (several waves on 32 rows: each takes other tiles).  Scores are formed
// transposed, S^T = K Q^T, so that a lane owns one row's: the softmax needs its own
// registers and one exchange with the other half-wave, and the probabilities are the
// next product's operand as they are, o^T = V^T P^T, with V^T read transposed from LDS.
//
// One pass with a running sum about a reference score, which bf16 products'
// accumulators start from: the difference costs no instruction, and it is formed before
// the scale, so that no rounding of ref c is in it.  The reference moves, and what is
// summed is rescaled, only when a tile's largest score goes past it by more than a factor
// of 2^8; a tile whose scores it would have blurred by its size is formed again without it.
// Scores, statistics and sums are float32; probabilities are rounded to the operands' type
// for the matrix cores (2^-8 of each in bf16, the sum is of the unrounded ones), the output
// once.
//
// Bound by the matrix pipes and what stands between their products: 2 x 4096 x 4096, 16 + 4
// heads of 128 in bf16, 304 to 317 us, 0.87 to 0.90 PF/s, pipes busy 47%, exponentials and
// rounding take the issue slots of most others.  By memory where rows are few: 16 x 1 x 8192,
// lengths from three tenths of 8192 to all, 38 us, 4.6 TB/s of the keys that take part; 128 x
// 64 x 197, 12 heads of 64, 24.4 us, 4.2 TB/s.  float32 of 3 x 77 x 1021, heads of 80, 23 us:
// pipes busy 38%, three or four tiles to a wave.
//
// Keys that take no part are zeros in LDS, whatever memory holds, and their scores are
// -inf, so NaN in padding reaches nothing.  Where rows are few, the keys are split over
// workgroups and a second kernel joins the parts.
#include "attend.h"

namespace hapi {
namespace {

// (largest score, log of the sum about it) from the sum about ref.  A row of NaN alone has
// no largest score, and is no row without a key.
__device__ __forceinline__ float2 row_stats(float m, float ref, float sum, float scale) {
  if (m == -INFINITY && sum != sum) m = sum;
  return make_float2(m, m == -INFINITY ? -INFINITY : logf(sum) - (m - ref) * scale);
}

template <typename T, int DP, int RW, int KW, int BN>
__global__ __launch_bounds__(64 * RW * KW, least_waves(sizeof(T) == 2 && DP <= 32 ? 4 : sizeof(T) == 2 || DP <= 96 ? 2 : 1, RW * KW, KW * 4 * hapi::Tile<T, DP, BN>::BYTES)) void attend_forward_kernel(AttendArgs a) {
  typedef hapi::Tile<T, DP, BN> Tile;
  typedef Loader<T, DP, BN, RW> Load;
  typedef typename Elem<T>::Frag Frag;
  constexpr int KS = DP / 16, DB = DP / 32, NT = BN / 32, STAGE = 2 * Tile::BYTES;
  __shared__ __attribute__((aligned(1024))) uint8_t smem[KW * 2 * STAGE];

  const int t = threadIdx.x, lane = t & 63, col = lane & 31, lh = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(t >> 6), wr = wave % RW, wk = wave / RW;
  const int rows = a.q_len * a.group, tiles = (rows + 32 * RW - 1) / (32 * RW);
  const Place at = place(a, tiles);
  const int tile = at.tile, split = at.split, pair = at.pair, b = at.b, kh = at.kh;
  const int q_valid = clamped(a.q_lens, b, a.q_len), kv_valid = clamped(a.kv_lens, b, a.kv_len);

  // this lane's row
  const int r = (tile * RW + wr) * 32 + col;
  const int qi = r / a.group, qg = r - qi * a.group;
  const bool counts = qi < q_valid;
  const T *qp = static_cast<const T *>(a.q) + (int64_t)b * a.q_st[0] + (int64_t)qi * a.q_st[1] + (int64_t)(kh * a.group + qg) * a.q_st[2];
  Frag qf[KS];
#pragma unroll
  for (int ks = 0; ks < KS; ++ks) qf[ks] = row_frag<T>(qp, ks, lh, a.dim, counts);

  // the split's tiles of keys; wave wk takes every KW-th
  const int key_tiles = tile * RW * 32 < q_valid * a.group ? (kv_valid + BN - 1) / BN : 0;
  const int t0 = (int)((int64_t)key_tiles * split / a.splits), t1 = (int)((int64_t)key_tiles * (split + 1) / a.splits);
  const int steps = (t1 - t0 + KW - 1) / KW;
  Load lk, lv;
  lk.init(a.k_st[1], a.dim, wr, lane);
  lv.init(a.v_st[1], a.dim, wr, lane);
  const T *kp = static_cast<const T *>(a.k) + (int64_t)b * a.k_st[0] + (int64_t)kh * a.k_st[2];
  const T *vp = static_cast<const T *>(a.v) + (int64_t)b * a.v_st[0] + (int64_t)kh * a.v_st[2];
  const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t *)smem + wk * 2 * STAGE;

  uint64_t keep = 0;  // of the tile in flight
  auto issue = [&](int step) {
    const int kt = t0 + step * KW + wk;
    keep = kt < t1 ? key_bits<BN>(kv_valid - (int64_t)kt * BN) : 0;
    if (keep && a.mask) {
      const bool in = (keep >> lane) & 1;
      keep &= __ballot(in && a.mask[(int64_t)b * a.kv_len + (int64_t)kt * BN + (in ? lane : 0)] != 0);
    }
    if (kt >= t1) return;
    const uint32_t at = lds0 + (step & 1) * STAGE;
    lk.issue(kp + (int64_t)kt * BN * a.k_st[1], at, keep, wr);
    lv.issue(vp + (int64_t)kt * BN * a.v_st[1], at + Tile::BYTES, keep, wr);
  };

  f32x16_t o[DB];
#pragma unroll
  for (int d = 0; d < DB; ++d) o[d] = zeros();
  // m: the largest score so far; ref: what is subtracted from the scores, the same until
  // a tile goes past it by more than 2^8 in the probabilities; sum: of this half-wave's keys
  float m = -INFINITY, ref = 0.0f, sum = 0.0f;
  // float32 scores are formed by themselves: sums that start at -ref would round by its size
  constexpr bool FROM_REF = sizeof(T) == 2;
  f32x16_t start = zeros();
  bool first = true;
  const float slack = 8.0f / a.c;

  if (steps > 0) issue(0);
  for (int step = 0; step < steps; ++step) {
    // this wave's DMAs have landed and its reads of the last tile are done; after the
    // barrier, everyone's
    wait_loads<0>();
    if constexpr (RW > 1) __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
    const uint64_t now = keep;
    if (step + 1 < steps) issue(step + 1);
    __builtin_amdgcn_sched_barrier(0);
    if (now == 0) continue;  // the same for all waves of wk
    const uint8_t *kt = smem + wk * 2 * STAGE + (step & 1) * STAGE, *vt = kt + Tile::BYTES;
    f32x16_t s[NT];  // scores, FROM_REF: less ref
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      if (DP == 96 && ks == KS - 1 && 16 * ks >= a.dim) break;  // heads of 80: five sixths of 96
#pragma unroll
      for (int n = 0; n < NT; ++n) s[n] = mma(Tile::by_row(kt, 32 * n, ks, lane), qf[ks], ks > 0 ? s[n] : FROM_REF ? start : zeros());
    }
    // -inf for keys that take no part; the row's largest
    auto masked = [&]() {
      if (now != kAllKeys<BN>) {
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          const uint32_t bits = (uint32_t)(now >> (32 * n)) >> (4 * lh);
#pragma unroll
          for (int i = 0; i < 16; ++i)
            if (!(bits >> (8 * (i >> 2) + (i & 3)) & 1)) s[n][i] = -INFINITY;
        }
      }
      float mx = -INFINITY;
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int i = 0; i < 16; ++i) mx = fmaxf(mx, s[n][i]);
      return fmaxf(mx, __shfl_xor(mx, 32, 64));
    };
    auto subtract = [&](float by) {
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int i = 0; i < 16; ++i) s[n][i] -= by;
    };
    const float mx = masked();
    // the first key of a row sets its ref, whatever its size
    const bool moves = (FROM_REF ? mx : mx - ref) > slack || (first && mx > -INFINITY);
    float top = FROM_REF ? ref + mx : mx;
    if (__any(moves)) {
      bool less_ref = FROM_REF;  // what s is
      // Scores less a ref far below 0 that are themselves nearer to it have lost their low
      // bits to its size (2^-24 of it; down to 2^-32 in the probabilities that is less than
      // 2^-16 of them): they are formed again by themselves, with q from memory (a loop about
      // both, with q in its registers: 2 x 4096 x 4096 348 us for 308; whenever ref moves: 435
      // us for scores that spread over 10 units, 311 so).
      if (FROM_REF && __any(moves && !first && ref * a.c < -32.0f && -ref > 2.0f * fabsf(top))) {
        less_ref = false;
#pragma unroll
        for (int n = 0; n < NT; ++n) s[n] = zeros();
#pragma unroll 1
        for (int ks = 0; ks < KS; ++ks) {
          const Frag f = row_frag<T>(qp, ks, lh, a.dim, counts);
#pragma unroll
          for (int n = 0; n < NT; ++n) s[n] = mma(Tile::by_row(kt, 32 * n, ks, lane), f, s[n]);
        }
        top = masked();
      }
      const float to = moves ? top : ref;
      const float alpha = first ? 1.0f : __builtin_amdgcn_exp2f((ref - to) * a.c);
      if (FROM_REF) subtract(less_ref ? to - ref : to);
      first = first && !moves;
      ref = to;
      start = block_of(-ref);
      sum *= alpha;
#pragma unroll
      for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[d][i] *= alpha;
    }
    m = fmaxf(m, top);
    if (!FROM_REF) subtract(ref);
    // Probabilities of 32 keys are summed by themselves: the roundings of thousands of equal
    // ones to a running sum would all go one way (16384 keys: off by 1.1e-4 of it, so 4e-6).
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      float own = 0.0f;
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        s[n][i] = __builtin_amdgcn_exp2f(s[n][i] * a.c);
        own += s[n][i];
      }
      sum += own;
    }
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      const Frag p[2] = {operand<T>(s[n], 0), operand<T>(s[n], 1)};
#pragma unroll
      for (int d = 0; d < DB; ++d)
        add_products<T>(o[d], [&](int j) { return Tile::by_column(vt, 32 * n + 16 * j, 32 * d, lane); }, p);
    }
  }
  sum += __shfl_xor(sum, 32, 64);
  __syncthreads();  // the tiles' place is used again
  if constexpr (KW > 1) {
    // the waves that share rows: the others' sums to the first one's, a register of all
    // lanes after another, in the tiles' place
    constexpr int REGS = 3 + 16 * DB;
    static_assert((KW - 1) * RW * REGS * 256 <= KW * 2 * STAGE, "the tiles' place");
    float *box = reinterpret_cast<float *>(smem);
    if (wk > 0) {
      float *to = box + ((wk - 1) * RW + wr) * REGS * 64 + lane;
      to[0] = ref, to[64] = sum, to[128] = m;
#pragma unroll
      for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) to[(3 + 16 * d + i) * 64] = o[d][i];
    }
    __syncthreads();
#pragma unroll
    for (int w = 0; w < KW - 1; ++w) {
      if (wk > 0) break;
      const float *from = box + (w * RW + wr) * REGS * 64 + lane;
      const float ref2 = from[0], sum2 = from[64], m2 = from[128];
      // a part without a key has no weight, and its ref no say
      const float both = m == -INFINITY ? ref2 : m2 == -INFINITY ? ref : fmaxf(ref, ref2);
      const float w1 = m == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f((ref - both) * a.c);
      const float w2 = m2 == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f((ref2 - both) * a.c);
      ref = both;
      m = fmaxf(m, m2);
      sum = sum * w1 + sum2 * w2;
#pragma unroll
      for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[d][i] = o[d][i] * w1 + from[(3 + 16 * d + i) * 64] * w2;
    }
    __syncthreads();  // one wave of rows may be ahead of another
  }
  if (!counts) {  // padding between rows that count: as a row without keys
    m = -INFINITY, ref = 0.0f, sum = 0.0f;
#pragma unroll
    for (int d = 0; d < DB; ++d) o[d] = zeros();
  }
  if (KW > 1 && wk > 0) return;
  if (a.splits > 1) {
    if (r >= rows) return;
    const int64_t at = ((int64_t)split * a.pairs + pair) * rows + r;
    float *p = a.part + at * a.dim4;
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int e = 32 * d + 8 * q + 4 * lh;
        if (e < a.dim4) *reinterpret_cast<float4 *>(p + e) = make_float4(o[d][4 * q], o[d][4 * q + 1], o[d][4 * q + 2], o[d][4 * q + 3]);
      }
    if (lh == 0) a.part_ml[at] = make_float4(ref, sum, m, 0.0f);
    return;
  }
  const float inv = sum > 0.0f || sum != sum ? 1.0f / sum : 0.0f;
  const int64_t h = kh * a.group + qg;
  T *y = static_cast<T *>(a.y) + (int64_t)b * a.y_st[0] + (int64_t)qi * a.y_st[1] + h * a.y_st[2];
  typedef RowsOut<T, DB> Out;
  static_assert(RW * Out::BYTES <= KW * 2 * STAGE, "the tiles' place");
  Out::template store<true>(o, inv, r < rows ? y : nullptr, a.dim, a.y_vec, smem + wr * Out::BYTES, lane);
  if (r >= rows) return;
  if (lh == 0) a.stats[((int64_t)b * a.q_len + qi) * a.heads + h] = row_stats(m, ref, sum, a.scale);
}

// Joins a row's parts: a thread has four of its values.
template <typename T>
__global__ __launch_bounds__(256) void attend_join_kernel(AttendArgs a) {
  const int per = a.dim4 / 4;
  const int64_t rows = (int64_t)a.q_len * a.group, all = rows * a.pairs;
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int64_t row = i / per;
  if (row >= all) return;
  const int d = (int)(i - row * per) * 4;
  float m = -INFINITY, ref = 0.0f, sum = 0.0f, o[4] = {};
  for (int p0 = 0; p0 < a.splits; p0 += 8) {  // the loads of 8 parts in flight
    float4 ml[8], v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int p = p0 + i < a.splits ? p0 + i : a.splits - 1;
      ml[i] = a.part_ml[p * all + row];
      v[i] = *reinterpret_cast<const float4 *>(a.part + (p * all + row) * a.dim4 + d);
    }
    // parts without a key have no weight, and their ref no say
    float both = m > -INFINITY ? ref : -INFINITY;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if (p0 + i >= a.splits) ml[i].z = -INFINITY;
      if (ml[i].z > -INFINITY) both = fmaxf(both, ml[i].x);
    }
    if (both == -INFINITY) both = 0.0f;
    const float w0 = m > -INFINITY ? __builtin_amdgcn_exp2f((ref - both) * a.c) : 0.0f;
    sum *= w0;
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] *= w0;
    ref = both;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float w = ml[i].z > -INFINITY ? __builtin_amdgcn_exp2f((ml[i].x - ref) * a.c) : 0.0f;
      m = fmaxf(m, ml[i].z);
      sum = fmaf(ml[i].y, w, sum);
      o[0] = fmaf(v[i].x, w, o[0]);
      o[1] = fmaf(v[i].y, w, o[1]);
      o[2] = fmaf(v[i].z, w, o[2]);
      o[3] = fmaf(v[i].w, w, o[3]);
    }
  }
  const float inv = sum > 0.0f || sum != sum ? 1.0f / sum : 0.0f;
  const int pair = (int)(row / rows), r = (int)(row - pair * rows), qi = r / a.group;
  const int b = pair / a.kv_heads;
  const int64_t h = (int64_t)(pair - b * a.kv_heads) * a.group + (r - qi * a.group);
  T *y = static_cast<T *>(a.y) + (int64_t)b * a.y_st[0] + (int64_t)qi * a.y_st[1] + h * a.y_st[2];
  store4<T>(y, d, a.dim, a.y_vec & 1, o[0] * inv, o[1] * inv, o[2] * inv, o[3] * inv);
  if (d == 0) a.stats[((int64_t)b * a.q_len + qi) * a.heads + h] = row_stats(m, ref, sum, a.scale);
}

// Rows of any layout to 16-byte aligned ones, a slot of 16 bytes a thread.
template <typename T>
__global__ __launch_bounds__(256) void attend_stage_kernel(StageArgs a) {
  constexpr int V = 16 / (int)sizeof(T);
  const int per = a.ld / V;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < a.count * per; i += (int64_t)gridDim.x * 256) {
    const int64_t row = i / per;
    const int d = (int)(i - row * per) * V;
    const int64_t tok = row / a.heads, b = tok / a.tokens;
    const T *p = static_cast<const T *>(a.in) + b * a.st[0] + (tok - b * a.tokens) * a.st[1] + (row - tok * a.heads) * a.st[2];
    T v[V];
#pragma unroll
    for (int e = 0; e < V; ++e) v[e] = d + e < a.dim ? p[d + e] : T{};
    __builtin_memcpy(static_cast<T *>(a.out) + row * a.ld + d, v, 16);
  }
}

template <typename T, int DP, int RW>
hipError_t forward(const AttendArgs &a, hipStream_t s) {
  constexpr int KW = attend_key_waves(sizeof(T), DP, RW), BN = attend_tile_keys(sizeof(T), DP, KW);
  const int64_t rows = (int64_t)a.q_len * a.group, tiles = ceil_div(rows, 32 * RW);
  hapi_launch(attend_forward_kernel<T, DP, RW, KW, BN>, dim3((uint32_t)(tiles * a.splits * a.pairs)), dim3(64 * RW * KW), 0, s, a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.splits == 1) return e;
  hapi_launch(attend_join_kernel<T>, dim3((uint32_t)ceil_div(rows * a.pairs * (a.dim4 / 4), 256)), dim3(256), 0, s, a);
  return hipGetLastError();
}

template <typename T, int DP>
hipError_t forward_rows(const AttendArgs &a, hipStream_t s) {
  const int rw = attend_row_waves((int64_t)a.q_len * a.group);
  return rw == 4 ? forward<T, DP, 4>(a, s) : rw == 2 ? forward<T, DP, 2>(a, s) : forward<T, DP, 1>(a, s);
}

template <typename T>
hipError_t forward_dim(const AttendArgs &a, hipStream_t s) {
  if (a.dim <= 32) return forward_rows<T, 32>(a, s);
  if (a.dim <= 64) return forward_rows<T, 64>(a, s);
  if (a.dim <= 96) return forward_rows<T, 96>(a, s);
  return forward_rows<T, 128>(a, s);
}

}  // namespace

hipError_t launch_attend_forward(bool bf16, const AttendArgs &a, hipStream_t s) {
  return bf16 ? forward_dim<uint16_t>(a, s) : forward_dim<float>(a, s);
}

hipError_t launch_attend_stage(bool bf16, const StageArgs &a, hipStream_t s) {
  const int64_t slots = a.count * (a.ld / (bf16 ? 8 : 4)), want = ceil_div(slots, 256);
  if (want == 0) return hipSuccess;
  const dim3 grid((uint32_t)(want < 16384 ? want : 16384)), block(256);
  if (bf16) hapi_launch(attend_stage_kernel<uint16_t>, grid, block, 0, s, a);
  else hapi_launch(attend_stage_kernel<float>, grid, block, 0, s, a);
  return hipGetLastError();
}

}  // namespace hapi
