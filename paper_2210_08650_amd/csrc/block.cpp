// Entry points of the trained block: argument checks, workspace layout and the
// launches of the gradients' norm and clipping, of the rotary positions and of the
// cross attention.  Declared in hapi.h.
#include <algorithm>
#include <cmath>
#include <new>
#include <vector>

#include "block.h"
#include "host_checks.h"

namespace hapi {
namespace {

// ----------------------------------------------------------------- gradients

constexpr int kMaxTensors = 1 << 20;
constexpr int64_t kMaxTensorSize = (int64_t)1 << 38;  // a launch's segments are a 32-bit number

int check_gradients(const hapi_gradient_desc *d) {
  if (!d) return fail(HAPI_E_INVAL, "desc is NULL");
  if (d->reserved) return fail(HAPI_E_INVAL, "reserved must be 0");
  if (d->count < 0) return fail(HAPI_E_INVAL, "count must be >= 0");
  if (d->count > kMaxTensors) return fail(HAPI_E_UNSUPPORTED, "%d tensors (at most 2^20)", d->count);
  if (!(d->max_norm > 0.0f) || !std::isfinite(d->max_norm)) return fail(HAPI_E_INVAL, "max_norm must be finite and > 0");
  if (d->count == 0) return HAPI_OK;
  if (!d->grads || !d->sizes || !d->dtypes) return fail(HAPI_E_INVAL, "grads, sizes or dtypes is NULL");
  for (int i = 0; i < d->count; ++i) {
    if (d->dtypes[i] != HAPI_F32 && d->dtypes[i] != HAPI_BF16) return fail(HAPI_E_INVAL, "unknown dtype %d of tensor %d", d->dtypes[i], i);
    if (d->sizes[i] < 0) return fail(HAPI_E_INVAL, "size of tensor %d must be >= 0", i);
    if (d->sizes[i] > kMaxTensorSize) return fail(HAPI_E_UNSUPPORTED, "tensor %d has more than 2^38 values", i);
    if (d->sizes[i] == 0) continue;
    const uintptr_t align = d->dtypes[i] == HAPI_BF16 ? 2 : 4;
    if (!d->grads[i]) return fail(HAPI_E_INVAL, "grads[%d] is NULL", i);
    if ((uintptr_t)d->grads[i] % align) return fail(HAPI_E_INVAL, "grads[%d] must be %d-byte aligned", i, (int)align);
    if (d->out && !d->out[i]) return fail(HAPI_E_INVAL, "out[%d] is NULL", i);
    if (d->out && (uintptr_t)d->out[i] % align) return fail(HAPI_E_INVAL, "out[%d] must be %d-byte aligned", i, (int)align);
  }
  return HAPI_OK;
}

struct Range {
  uintptr_t lo, hi;
};

// No value is written twice, or read after it was written as another tensor's: a
// tensor listed twice would be scaled twice, and by blocks that race.
int check_outputs_apart(const hapi_gradient_desc *d) {
  std::vector<Range> out;
  out.reserve(d->count);
  auto range = [&](const void *p, int i) {
    const uintptr_t lo = (uintptr_t)p;
    return Range{lo, lo + (uintptr_t)d->sizes[i] * (d->dtypes[i] == HAPI_BF16 ? 2 : 4)};
  };
  for (int i = 0; i < d->count; ++i)
    if (d->sizes[i] > 0) out.push_back(range(d->out ? d->out[i] : d->grads[i], i));
  const auto below = [](const Range &a, const Range &b) { return a.lo < b.lo; };
  if (!std::is_sorted(out.begin(), out.end(), below)) std::sort(out.begin(), out.end(), below);
  for (size_t i = 1; i < out.size(); ++i)
    if (out[i].lo < out[i - 1].hi) return fail(HAPI_E_INVAL, "two of the tensors that are written overlap");
  for (int i = 0; d->out && i < d->count; ++i) {
    if (d->sizes[i] == 0 || d->out[i] == d->grads[i]) continue;
    const Range g = range(d->grads[i], i);
    auto next = std::upper_bound(out.begin(), out.end(), g, below);  // the first that starts behind g's start
    if ((next != out.end() && next->lo < g.hi) || (next != out.begin() && (next - 1)->hi > g.lo))
      return fail(HAPI_E_INVAL, "grads[%d] overlaps a tensor that is written", i);
  }
  return HAPI_OK;
}

int64_t gradient_workspace(const hapi_gradient_desc *d) {
  const int64_t launches = std::max<int64_t>(1, ceil_div(d->count, kGradTensors));
  return up((launches + 1) * kGradBlocks * (int64_t)sizeof(double), kAlign);
}

// The next launch's tensors from i on (those without values left out); its blocks, 0: none.
int next_gradients(const hapi_gradient_desc *d, int &i, GradArgs &a) {
  a.count = 0;
  for (uint32_t &f : a.f32) f = 0;
  int64_t total = 0;
  for (; i < d->count && a.count < kGradTensors; ++i) {
    if (d->sizes[i] == 0) continue;
    a.in[a.count] = d->grads[i];
    a.out[a.count] = d->out ? d->out[i] : const_cast<void *>(d->grads[i]);
    a.size[a.count] = d->sizes[i];
    if (d->dtypes[i] == HAPI_F32) a.f32[a.count >> 5] |= 1u << (a.count & 31);
    total += d->sizes[i];
    ++a.count;
  }
  // Segments that fill the blocks, of 2048 to 32,768 values: a block's first loads
  // wait for its search of the tensor (32,768 always: 2 million values in two float32
  // tensors 5.5 + 10.7 us, so 4.0 + 6.8).
  a.seg_size = 32768;
  while (a.seg_size > 2048 && total / a.seg_size < 2 * kGradBlocks) a.seg_size /= 2;
  int64_t seg = 0;
  for (int t = 0; t < a.count; ++t) {
    a.seg[t] = (int32_t)seg;
    seg += ceil_div(a.size[t], a.seg_size);
  }
  a.seg[a.count] = (int32_t)seg;
  return (int)std::min<int64_t>(seg, kGradBlocks);
}

int run_gradients(const hapi_gradient_desc *d, float *norm, bool clip) {
  TRY(check_gradients(d));
  TRY(check_ptr(norm, 4, "norm"));
  if (clip) TRY(check_outputs_apart(d));
  TRY(check_workspace(d->workspace, d->workspace_bytes, gradient_workspace(d)));
  TRY(check_stream(d->stream));
  hipStream_t s = static_cast<hipStream_t>(d->stream);
  double *part = static_cast<double *>(d->workspace);
  GradArgs a;
  a.max_norm = d->max_norm;
  int64_t parts = 0;
  int launches = 0;
  for (int i = 0; i < d->count;) {
    const int blocks = next_gradients(d, i, a);
    if (blocks == 0) break;
    a.part = part + parts;
    a.parts = 0;
    a.norm = nullptr;
    HIP_TRY(launch_grad_squares(a, blocks, s));
    parts += blocks;
    ++launches;
  }
  if (launches > kGradSumLaunches) {
    double *joined = part + (int64_t)ceil_div(d->count, kGradTensors) * kGradBlocks;
    HIP_TRY(launch_grad_join(part, parts, joined, s));
    part = joined;
    parts = std::min<int64_t>(parts, kGradBlocks);
  }
  if (!clip || launches == 0) {
    HIP_TRY(launch_grad_norm(part, parts, norm, s));
    return HAPI_OK;
  }
  for (int i = 0; i < d->count;) {
    const int blocks = next_gradients(d, i, a);
    if (blocks == 0) break;
    a.part = part;
    a.parts = parts;
    a.norm = norm;
    norm = nullptr;
    HIP_TRY(launch_grad_clip(a, blocks, s));
  }
  return HAPI_OK;
}

// ------------------------------------------------------------------- layouts

constexpr int64_t kMaxExtent = (int64_t)1 << 31;
constexpr int64_t kMaxStride = (int64_t)1 << 40;

// Elements between batch entries, tokens and heads; three zeros: [batch, tokens, heads, dim].
int read_strides(const int64_t *in, int64_t tokens, int64_t heads, int64_t dim, const char *name, int64_t *out) {
  if (in[0] == 0 && in[1] == 0 && in[2] == 0) {
    out[2] = dim;
    out[1] = heads * dim;
    out[0] = tokens * out[1];
    return HAPI_OK;
  }
  for (int i = 0; i < 3; ++i) {
    if (in[i] < 0) return fail(HAPI_E_INVAL, "strides of %s must be >= 0", name);
    if (in[i] > kMaxStride) return fail(HAPI_E_UNSUPPORTED, "strides of %s must be <= 2^40", name);
    out[i] = in[i];
  }
  return HAPI_OK;
}

// Whether no two values of a tensor share a place, as one that is written must.
int check_apart(const int64_t *stride, int64_t batch, int64_t tokens, int64_t heads, int64_t dim, const char *name) {
  struct {
    int64_t stride, extent;
  } d[3] = {{stride[0], batch}, {stride[1], tokens}, {stride[2], heads}};
  std::sort(d, d + 3, [](const auto &a, const auto &b) { return a.stride < b.stride; });
  if (batch == 0 || tokens == 0 || heads == 0) return HAPI_OK;
  __int128 span = dim;
  for (const auto &x : d) {
    if (x.extent == 1) continue;
    if (x.stride < span) return fail(HAPI_E_INVAL, "strides of %s let its values overlap", name);
    span += (__int128)x.stride * (x.extent - 1);
  }
  return HAPI_OK;
}

// -------------------------------------------------------------------- rotary

struct Rotary {
  bool bf16;
  int esz, v;
  RotaryArgs a;
  int64_t batch;
};

int read_rotary(const hapi_rotary_desc *d, Rotary &r) {
  if (!d) return fail(HAPI_E_INVAL, "desc is NULL");
  if (d->dtype != HAPI_F32 && d->dtype != HAPI_BF16) return fail(HAPI_E_INVAL, "unknown dtype %d", d->dtype);
  if (d->reserved) return fail(HAPI_E_INVAL, "reserved must be 0");
  if (d->head_dim < 1) return fail(HAPI_E_INVAL, "head_dim must be >= 1");
  if (d->head_dim > kRotaryMaxDim) return fail(HAPI_E_UNSUPPORTED, "head_dim %d (at most %d)", d->head_dim, kRotaryMaxDim);
  if (d->heads < 0 || d->kv_heads < 0 || d->heads + (int64_t)d->kv_heads < 1)
    return fail(HAPI_E_INVAL, "heads and kv_heads must be >= 0, one of them >= 1");
  if (d->batch < 0 || d->length < 0) return fail(HAPI_E_INVAL, "batch and length must be >= 0");
  if (d->axes < 0 || d->axes > kRotaryAxes) return fail(HAPI_E_INVAL, "axes must be in [0, %d]", kRotaryAxes);
  if (d->neighbours != 0 && d->neighbours != 1) return fail(HAPI_E_INVAL, "neighbours must be 0 or 1");
  if (d->norm != 0 && d->norm != 1) return fail(HAPI_E_INVAL, "norm must be 0 or 1");
  if (!(d->eps >= 0.0f) || !std::isfinite(d->eps)) return fail(HAPI_E_INVAL, "eps must be finite and >= 0");
  r = Rotary{};
  RotaryArgs &a = r.a;
  int64_t pairs = 0;
  for (int i = 0; i < kRotaryAxes; ++i) {
    if (i >= d->axes ? d->sections[i] != 0 : d->sections[i] < 1)
      return fail(HAPI_E_INVAL, "sections must be >= 1 on each axis, and 0 past the last one");
    a.first[i] = (int32_t)std::min<int64_t>(pairs, kRotaryMaxDim);
    pairs += d->sections[i];
  }
  if (2 * pairs > d->head_dim) return fail(HAPI_E_INVAL, "the sections' %lld pairs exceed head_dim", (long long)pairs);
  if (d->batch >= kMaxExtent || d->length >= kMaxExtent || d->heads >= 1 << 20 || d->kv_heads >= 1 << 20 ||
      (__int128)d->batch * d->length * (d->heads + d->kv_heads) >= kMaxExtent)
    return fail(HAPI_E_UNSUPPORTED, "batch * length * (heads + kv_heads) must be below 2^31");
  r.bf16 = d->dtype == HAPI_BF16;
  r.esz = r.bf16 ? 2 : 4;
  r.batch = d->batch;
  a.heads[0] = d->heads;
  a.heads[1] = d->kv_heads;
  a.tokens = d->batch * d->length;
  a.len = (int32_t)d->length;
  a.dim = d->head_dim;
  a.pairs = (int32_t)pairs;
  a.axes = d->axes;
  a.eps = d->eps;
  a.inv_dim = 1.0f / (float)d->head_dim;
  a.norm = d->norm;
  a.neighbours = d->neighbours;
  TRY(read_strides(d->q_stride, d->length, d->heads, d->head_dim, "q", a.x_st[0]));
  TRY(read_strides(d->k_stride, d->length, d->kv_heads, d->head_dim, "k", a.x_st[1]));
  TRY(read_strides(d->q_out_stride, d->length, d->heads, d->head_dim, "q_out", a.y_st[0]));
  TRY(read_strides(d->k_out_stride, d->length, d->kv_heads, d->head_dim, "k_out", a.y_st[1]));
  // As many values at once as the pairs' two sides and what is not rotated divide into
  // (128 x 197 tokens of 24 heads of 64 in bf16: 32 us, one value at a time 61); neighbours
  // lie together with what is not rotated.
  const int64_t side = d->neighbours ? 0 : pairs, rest = d->head_dim - 2 * side;
  r.v = r.bf16 ? 8 : 4;
  while (r.v > 1 && (side % r.v != 0 || rest % (2 * r.v) != 0)) r.v /= 2;
  // A lane forms the sines of its pairs one after another, so few vectors are shared by
  // more lanes, down to two pairs each (1 x 197 tokens: 3.9 us, with 8 pairs 5.7; backward
  // 5.5 and 8.5), until the CUs have 1024 lanes each (12 x 197: 11.5 us with 4 pairs, 12.9
  // with 2).
  const int64_t heads = (int64_t)d->heads + d->kv_heads;
  const auto lanes_of = [&](int v) {
    int n = 4;
    while (n < 64 && n * 2 * v < d->head_dim) n *= 2;
    return n;
  };
  while (r.v > 2 && a.tokens * heads * lanes_of(r.v) < kCus * 1024) r.v /= 2;
  // Up to 8 heads a lane, so that it forms sines and cosines once for them, as long as
  // the CUs' 2048 lanes each are filled (1 x 197 tokens with all 12 heads a lane: 13.6 us
  // where one takes 5.7; 3 x 4099 tokens in float32: 46.1 and, with 8, 45.2).
  const int lanes = lanes_of(r.v);
  const int64_t each = std::max<int64_t>(1, std::min<int64_t>(8, a.tokens * heads * lanes / (kCus * 2048)));
  for (int w = 0; w < 2; ++w) a.head_groups[w] = (int32_t)ceil_div(a.heads[w], each);
  return HAPI_OK;
}

int64_t rotary_workspace(const Rotary &r) { return r.a.norm ? up((int64_t)kRotaryParts * 2 * r.a.dim * 4, kAlign) : 0; }

// The inputs that both directions read, and the gammas.
int check_rotary_inputs(const hapi_rotary_desc *d, Rotary &r, const float *q_gamma, const float *k_gamma,
                        const int64_t *positions, const double *freq, const int64_t *lens) {
  const float *gamma[2] = {q_gamma, k_gamma};
  static const char *const names[2] = {"q_gamma", "k_gamma"};
  for (int w = 0; w < 2; ++w) {
    if (r.a.norm && r.a.heads[w] > 0) TRY(check_ptr(gamma[w], 4, names[w]));
    else if (gamma[w]) return fail(HAPI_E_INVAL, "%s is given, and not used", names[w]);
    r.a.gamma[w] = gamma[w];
  }
  if (d->axes > 0) {
    TRY(check_ptr(freq, 8, "freq"));
    if (r.a.tokens > 0) TRY(check_ptr(positions, 8, "positions"));
  }
  if (lens && (uintptr_t)lens % 8) return fail(HAPI_E_INVAL, "lens must be 8-byte aligned");
  r.a.positions = positions;
  r.a.freq = freq;
  r.a.lens = lens;
  return HAPI_OK;
}

// Tensors of q and k, which must be there where there are heads of them.
int check_both(const Rotary &r, const void *q, const void *k, const char *q_name, const char *k_name) {
  if (r.a.heads[0] > 0) TRY(check_ptr(q, r.esz, q_name));
  else if (q) return fail(HAPI_E_INVAL, "%s without heads", q_name);
  if (r.a.heads[1] > 0) TRY(check_ptr(k, r.esz, k_name));
  else if (k) return fail(HAPI_E_INVAL, "%s without kv_heads", k_name);
  return HAPI_OK;
}

// Outputs in place of inputs: each in its own input's, with the same strides; q and k are
// worked on at once, so neither is written where the other is read or written.
int check_places(const Rotary &r, const void *const (&in)[2], const int64_t (&in_st)[2][3], const void *const (&out)[2],
                 const int64_t (&out_st)[2][3], const char *const (&in_name)[2], const char *const (&out_name)[2]) {
  for (int w = 0; w < 2; ++w) {
    if (r.a.heads[w] == 0) continue;
    const int64_t extent[3] = {r.batch, r.a.len, r.a.heads[w]};
    for (int i = 0; in[w] == out[w] && i < 3; ++i)
      if (extent[i] > 1 && in_st[w][i] != out_st[w][i])
        return fail(HAPI_E_INVAL, "%s may be %s only where their strides are the same", out_name[w], in_name[w]);
    if (r.a.heads[1 - w] > 0 && in[0] != in[1] && out[w] == in[1 - w])
      return fail(HAPI_E_INVAL, "%s must not be %s", out_name[w], in_name[1 - w]);
  }
  if (r.a.heads[0] > 0 && r.a.heads[1] > 0 && in[0] != in[1] && out[0] == out[1])
    return fail(HAPI_E_INVAL, "%s and %s are the same", out_name[0], out_name[1]);
  return HAPI_OK;
}

// ----------------------------------------------------------- cross attention

struct Attend {
  bool bf16;
  int esz, v;  // bytes of a value, values of 16 bytes
  AttendArgs a;
  int64_t batch;
  bool stage_q, stage_k, stage_v, stage_o;  // copied to aligned rows; dout lies as o does
  int64_t ld;                               // of those
  int fwd_splits, dkv_splits;
  int64_t bytes_fwd, bytes_bwd;
  int64_t o_q, o_k, o_v, o_o, o_g, o_part, o_ml, o_delta;  // byte offsets into the workspace
};

int read_attend(const hapi_attention_desc *d, Attend &t) {
  if (!d) return fail(HAPI_E_INVAL, "desc is NULL");
  if (d->dtype != HAPI_F32 && d->dtype != HAPI_BF16) return fail(HAPI_E_INVAL, "unknown dtype %d", d->dtype);
  if (d->reserved) return fail(HAPI_E_INVAL, "reserved must be 0");
  if (d->head_dim < 1) return fail(HAPI_E_INVAL, "head_dim must be >= 1");
  if (d->head_dim > kAttendMaxDim) return fail(HAPI_E_UNSUPPORTED, "head_dim %d (at most %d)", d->head_dim, kAttendMaxDim);
  if (d->heads < 1 || d->kv_heads < 1 || d->heads % d->kv_heads)
    return fail(HAPI_E_INVAL, "heads must be a multiple of kv_heads, both >= 1");
  if (d->heads > 1 << 20) return fail(HAPI_E_UNSUPPORTED, "%d heads (at most 2^20)", d->heads);
  if (d->heads / d->kv_heads > kAttendMaxGroup)
    return fail(HAPI_E_UNSUPPORTED, "%d heads share a key head (at most %d)", d->heads / d->kv_heads, kAttendMaxGroup);
  if (d->batch < 0 || d->q_len < 0 || d->kv_len < 0) return fail(HAPI_E_INVAL, "batch, q_len and kv_len must be >= 0");
  if (!(d->scale >= 0.0f && d->scale <= 0x1p126f)) return fail(HAPI_E_INVAL, "scale must be in (0, 2^126], or 0");  // times log2(e) it is finite
  t = Attend{};
  AttendArgs &a = t.a;
  constexpr int64_t kMaxRows = (int64_t)1 << 30, kMaxTiles = (int64_t)1 << 24;  // 2^32 threads are too many for a launch
  const int64_t group = d->heads / d->kv_heads;
  if (d->batch > kMaxRows || d->q_len > kMaxRows || d->kv_len > kMaxRows || d->q_len * group > kMaxRows)
    return fail(HAPI_E_UNSUPPORTED, "batch, kv_len and q_len times heads / kv_heads must be at most 2^30");
  const int64_t pairs = d->batch * d->kv_heads, rows = d->q_len * group;
  const int rw = attend_row_waves(rows);
  // tiles of keys of bf16 heads past 96 values have 512 threads, others 256
  const int64_t key_tiles_most = d->dtype == HAPI_BF16 && d->head_dim > 96 ? kMaxTiles / 2 : kMaxTiles;
  if (pairs >= kMaxTiles || ceil_div(rows, 32 * rw) * pairs >= kMaxTiles || ceil_div(d->kv_len, 128) * pairs >= key_tiles_most)
    return fail(HAPI_E_UNSUPPORTED, "too many tiles of queries or keys (2^24, or 2^23 of keys of bf16 heads past 96 values)");
  t.bf16 = d->dtype == HAPI_BF16;
  t.esz = t.bf16 ? 2 : 4;
  t.v = 16 / t.esz;
  t.batch = d->batch;
  a.q_len = (int32_t)d->q_len;
  a.kv_len = (int32_t)d->kv_len;
  a.heads = d->heads;
  a.kv_heads = d->kv_heads;
  a.group = (int32_t)group;
  a.dim = d->head_dim;
  a.dim4 = (int32_t)up(d->head_dim, 4);
  a.pairs = (int32_t)pairs;
  a.scale = d->scale != 0.0f ? d->scale : 1.0f / std::sqrt((float)d->head_dim);
  a.c = (float)((double)a.scale * 1.4426950408889634);
  TRY(read_strides(d->q_stride, d->q_len, d->heads, d->head_dim, "q", a.q_st));
  TRY(read_strides(d->k_stride, d->kv_len, d->kv_heads, d->head_dim, "k", a.k_st));
  TRY(read_strides(d->v_stride, d->kv_len, d->kv_heads, d->head_dim, "v", a.v_st));
  TRY(read_strides(d->o_stride, d->q_len, d->heads, d->head_dim, "o", a.o_st));
  // An extent of one has no stride: whatever is given, it costs no copy and no narrow store.
  const int64_t extents[2][3] = {{d->batch, d->q_len, d->heads}, {d->batch, d->kv_len, d->kv_heads}};
  for (int i = 0; i < 3; ++i) {
    if (extents[0][i] == 1) a.q_st[i] = a.o_st[i] = 0;
    if (extents[1][i] == 1) a.k_st[i] = a.v_st[i] = 0;
  }
  // The kernels read whole 16-byte slots, at 32-bit offsets from a tile's first token.
  const auto staged = [&](const int64_t *st, int64_t heads) {
    return d->head_dim % t.v != 0 || st[0] % t.v != 0 || st[1] % t.v != 0 || st[2] % t.v != 0 || st[1] > 1 << 20 ||
           st[2] * heads * t.esz >= (int64_t)1 << 30;
  };
  t.stage_q = staged(a.q_st, group);
  t.stage_k = staged(a.k_st, 1);
  t.stage_v = staged(a.v_st, 1);
  t.stage_o = staged(a.o_st, group);
  t.ld = up(d->head_dim, t.v);

  // Few rows: the keys over as many workgroups as fill the CUs, some tiles to each wave.
  const int padded = (int)up(d->head_dim, 32), kw = attend_key_waves(t.esz, padded, rw), bn = attend_tile_keys(t.esz, padded, kw);
  // Two workgroups a CU, and one of float32 heads past 64 values, whose registers leave no more
  // (but for the forward pass of 65 to 96 values, which would run two).
  const int64_t wgs = ceil_div(rows, 32 * rw) * pairs, want = (!t.bf16 && padded > 64 ? 1 : 2) * kCus;
  // A float32 tile's products take eight times as long as a bf16 one's, so one of them is
  // worth a part of its own; of the others four.  Forward and join with 1, 2, 4 and 16 of
  // them: 1 x 1 x 8192, 16 + 4 heads of 128, 21, 21, 18 and 32 us; 4 x 8 x 2000, 8 + 2 heads
  // of 96, 15, 13, 14 and 37; 1 x 300 x 600, 4 heads of 128, 14, 14, 17 and 19.  float32, 3 x
  // 77 x 1021, 12 + 4 heads of 80: the same with 1 and 4; 2 x 100 x 500, 8 heads of 128, 16 and
  // 28.
  const int64_t key_tiles = ceil_div(d->kv_len, bn), least = t.bf16 ? 4 : 1;
  t.fwd_splits = wgs == 0 ? 1 : (int)std::max<int64_t>(1, std::min<int64_t>({want / wgs, key_tiles / (least * kw), 64}));
  const int64_t dkv_want = padded > 96 ? kCus : want;  // one workgroup a CU
  const int64_t kwgs = ceil_div(d->kv_len, 128) * pairs, row_tiles = ceil_div(rows, t.bf16 ? 64 : 32);
  t.dkv_splits = kwgs == 0 ? 1 : (int)std::max<int64_t>(1, std::min<int64_t>({dkv_want / kwgs, row_tiles / least, 64}));

  const int64_t all = pairs * rows, keys = pairs * d->kv_len;
  int64_t o = 0;
  auto take = [&](int64_t bytes) {
    const int64_t at = o;
    o += up(bytes, kAlign);
    return at;
  };
  t.o_q = take(t.stage_q ? all * t.ld * t.esz : 0);
  t.o_k = take(t.stage_k ? keys * t.ld * t.esz : 0);
  t.o_v = take(t.stage_v ? keys * t.ld * t.esz : 0);
  const int64_t shared = o;
  t.o_ml = take(t.fwd_splits > 1 ? t.fwd_splits * all * 16 : 0);
  take(t.fwd_splits > 1 ? t.fwd_splits * all * a.dim4 * 4 : 0);
  t.bytes_fwd = o;
  o = shared;
  t.o_o = take(t.stage_o ? all * t.ld * t.esz : 0);
  t.o_g = take(t.stage_o ? all * t.ld * t.esz : 0);
  t.o_delta = take(all * 4);
  t.o_part = o;  // dq's, then dk's and dv's
  take(std::max<int64_t>(t.fwd_splits > 1 ? t.fwd_splits * all * a.dim4 * 4 : 0, t.dkv_splits > 1 ? t.dkv_splits * 2 * keys * a.dim4 * 4 : 0));
  t.bytes_bwd = o;
  return HAPI_OK;
}

int check_attend_inputs(const Attend &t, const void *q, const void *k, const void *v, const int64_t *q_lens,
                        const int64_t *kv_lens, const uint8_t *mask) {
  if (t.a.q_len > 0) TRY(check_ptr(q, t.stage_q ? t.esz : 16, "q"));
  if (t.a.kv_len > 0) {
    TRY(check_ptr(k, t.stage_k ? t.esz : 16, "k"));
    TRY(check_ptr(v, t.stage_v ? t.esz : 16, "v"));
  }
  if ((uintptr_t)q_lens % 8) return fail(HAPI_E_INVAL, "q_lens must be 8-byte aligned");
  if ((uintptr_t)kv_lens % 8) return fail(HAPI_E_INVAL, "kv_lens must be 8-byte aligned");
  return HAPI_OK;
}

// What of every row can be stored at once: bit 0, four values; bit 1, 16 bytes; bit 2, two
// values.
int at_once(const Attend &t, const void *p, const int64_t *st) {
  const auto fits = [&](int n) { return t.a.dim % n == 0 && st[0] % n == 0 && st[1] % n == 0 && st[2] % n == 0 && (uintptr_t)p % (n * t.esz) == 0; };
  return (fits(4) ? 1 : 0) | (fits(t.v) ? 2 : 0) | (fits(2) ? 4 : 0);
}

// A copy of in, [batch][tokens][heads], with aligned rows, and its strides.
int stage_rows(const Attend &t, const void *in, int64_t *st, int64_t tokens, int64_t heads, void *out, hipStream_t s) {
  StageArgs g;
  g.in = in;
  g.out = out;
  for (int i = 0; i < 3; ++i) g.st[i] = st[i];
  g.count = t.batch * tokens * heads;
  g.tokens = (int32_t)tokens;
  g.heads = (int32_t)heads;
  g.dim = t.a.dim;
  g.ld = (int32_t)t.ld;
  HIP_TRY(launch_attend_stage(t.bf16, g, s));
  st[2] = t.ld;
  st[1] = heads * t.ld;
  st[0] = tokens * st[1];
  return HAPI_OK;
}

int stage_inputs(Attend &t, const void *q, const void *k, const void *v, uint8_t *base, hipStream_t s) {
  AttendArgs &a = t.a;
  a.q = q;
  a.k = k;
  a.v = v;
  if (t.stage_q) {
    a.q = base + t.o_q;
    TRY(stage_rows(t, q, a.q_st, a.q_len, a.heads, base + t.o_q, s));
  }
  if (t.stage_k) {
    a.k = base + t.o_k;
    TRY(stage_rows(t, k, a.k_st, a.kv_len, a.kv_heads, base + t.o_k, s));
  }
  if (t.stage_v) {
    a.v = base + t.o_v;
    TRY(stage_rows(t, v, a.v_st, a.kv_len, a.kv_heads, base + t.o_v, s));
  }
  return HAPI_OK;
}

}  // namespace

}  // namespace hapi

using namespace hapi;

extern "C" {

int64_t hapi_gradient_workspace_bytes(const hapi_gradient_desc *desc) {
  TRY(check_gradients(desc));
  return gradient_workspace(desc);
}

int hapi_gradient_norm(const hapi_gradient_desc *desc, float *norm) { return run_gradients(desc, norm, false); }

int hapi_gradient_clip(const hapi_gradient_desc *desc, float *norm) {
  try {
    return run_gradients(desc, norm, true);
  } catch (const std::bad_alloc &) {
    return fail(HAPI_E_NOMEM, "no host memory to compare the tensors' addresses");
  }
}

int64_t hapi_rotary_workspace_bytes(const hapi_rotary_desc *desc) {
  Rotary r;
  TRY(read_rotary(desc, r));
  return rotary_workspace(r);
}

int hapi_rotary_forward(const hapi_rotary_desc *desc, const void *q, const void *k, const float *q_gamma, const float *k_gamma,
                        const int64_t *positions, const double *freq, const int64_t *lens, void *q_out, void *k_out) {
  Rotary r;
  TRY(read_rotary(desc, r));
  TRY(check_rotary_inputs(desc, r, q_gamma, k_gamma, positions, freq, lens));
  if (r.a.tokens == 0) return HAPI_OK;
  TRY(check_both(r, q, k, "q", "k"));
  TRY(check_both(r, q_out, k_out, "q_out", "k_out"));
  TRY(check_apart(r.a.y_st[0], r.batch, r.a.len, r.a.heads[0], r.a.dim, "q_out"));
  TRY(check_apart(r.a.y_st[1], r.batch, r.a.len, r.a.heads[1], r.a.dim, "k_out"));
  TRY(check_places(r, {q, k}, r.a.x_st, {q_out, k_out}, r.a.y_st, {"q", "k"}, {"q_out", "k_out"}));
  TRY(check_stream(desc->stream));
  r.a.x[0] = q;
  r.a.x[1] = k;
  r.a.y[0] = q_out;
  r.a.y[1] = k_out;
  HIP_TRY(launch_rotary_forward(r.bf16, r.v, r.a, static_cast<hipStream_t>(desc->stream)));
  return HAPI_OK;
}

int hapi_rotary_backward(const hapi_rotary_desc *desc, const void *dq_out, const void *dk_out, const void *q, const void *k,
                         const float *q_gamma, const float *k_gamma, const int64_t *positions, const double *freq,
                         const int64_t *lens, void *dq, void *dk, float *dq_gamma, float *dk_gamma) {
  Rotary r;
  TRY(read_rotary(desc, r));
  TRY(check_rotary_inputs(desc, r, q_gamma, k_gamma, positions, freq, lens));
  if (r.a.tokens > 0) {
    TRY(check_both(r, dq_out, dk_out, "dq_out", "dk_out"));
    TRY(check_both(r, dq, dk, "dq", "dk"));
    if (r.a.norm) TRY(check_both(r, q, k, "q", "k"));
    TRY(check_apart(r.a.x_st[0], r.batch, r.a.len, r.a.heads[0], r.a.dim, "dq"));
    TRY(check_apart(r.a.x_st[1], r.batch, r.a.len, r.a.heads[1], r.a.dim, "dk"));
  }
  float *const dgamma[2] = {dq_gamma, dk_gamma};
  static const char *const names[2] = {"dq_gamma", "dk_gamma"};
  for (int w = 0; w < 2; ++w) {
    if (r.a.norm && r.a.heads[w] > 0) TRY(check_ptr(dgamma[w], 4, names[w]));
    else if (dgamma[w]) return fail(HAPI_E_INVAL, "%s is given, and nothing to write", names[w]);
    r.a.dgamma[w] = dgamma[w];
  }
  TRY(check_workspace(desc->workspace, desc->workspace_bytes, rotary_workspace(r)));
  if (r.a.tokens > 0) {
    TRY(check_places(r, {dq_out, dk_out}, r.a.y_st, {dq, dk}, r.a.x_st, {"dq_out", "dk_out"}, {"dq", "dk"}));
    if (r.a.norm) TRY(check_places(r, {q, k}, r.a.x_st, {dq, dk}, r.a.x_st, {"q", "k"}, {"dq", "dk"}));
  }
  TRY(check_stream(desc->stream));
  r.a.x[0] = q;
  r.a.x[1] = k;
  r.a.dy[0] = dq_out;
  r.a.dy[1] = dk_out;
  r.a.y[0] = dq;
  r.a.y[1] = dk;
  r.a.part = static_cast<float *>(desc->workspace);
  if (r.a.tokens == 0 && !r.a.norm) return HAPI_OK;
  HIP_TRY(launch_rotary_backward(r.bf16, r.v, r.a, static_cast<hipStream_t>(desc->stream)));
  return HAPI_OK;
}

int64_t hapi_cross_attention_workspace_bytes(const hapi_attention_desc *desc, int32_t backward) {
  Attend t;
  TRY(read_attend(desc, t));
  return backward ? std::max(t.bytes_fwd, t.bytes_bwd) : t.bytes_fwd;
}

int hapi_cross_attention_forward(const hapi_attention_desc *desc, const void *q, const void *k, const void *v,
                                 const int64_t *q_lens, const int64_t *kv_lens, const uint8_t *mask, void *o, float *stats) {
  Attend t;
  TRY(read_attend(desc, t));
  if (t.batch == 0 || t.a.q_len == 0) return HAPI_OK;
  AttendArgs &a = t.a;
  TRY(check_attend_inputs(t, q, k, v, q_lens, kv_lens, mask));
  TRY(check_ptr(o, t.esz, "o"));
  TRY(check_ptr(stats, 8, "stats"));
  TRY(check_apart(a.o_st, t.batch, a.q_len, a.heads, a.dim, "o"));
  TRY(check_workspace(desc->workspace, desc->workspace_bytes, t.bytes_fwd));
  TRY(check_stream(desc->stream));
  hipStream_t s = static_cast<hipStream_t>(desc->stream);
  uint8_t *base = static_cast<uint8_t *>(desc->workspace);
  TRY(stage_inputs(t, q, k, v, base, s));
  a.q_lens = q_lens;
  a.kv_lens = kv_lens;
  a.mask = mask;
  a.y = o;
  for (int i = 0; i < 3; ++i) a.y_st[i] = a.o_st[i];
  a.y_vec = at_once(t, o, a.o_st);
  a.stats = reinterpret_cast<float2 *>(stats);
  a.splits = t.fwd_splits;
  a.part_ml = reinterpret_cast<float4 *>(base + t.o_ml);
  a.part = reinterpret_cast<float *>(base + t.o_ml + up((int64_t)t.fwd_splits * a.pairs * a.q_len * a.group * 16, kAlign));
  HIP_TRY(launch_attend_forward(t.bf16, a, s));
  return HAPI_OK;
}

int hapi_cross_attention_backward(const hapi_attention_desc *desc, const void *q, const void *k, const void *v,
                                  const int64_t *q_lens, const int64_t *kv_lens, const uint8_t *mask, const void *o,
                                  const float *stats, const void *dout, void *dq, void *dk, void *dv) {
  Attend t;
  TRY(read_attend(desc, t));
  AttendArgs &a = t.a;
  if (t.batch == 0 || (a.q_len == 0 && a.kv_len == 0)) return HAPI_OK;
  TRY(check_attend_inputs(t, q, k, v, q_lens, kv_lens, mask));
  if (a.q_len > 0) {
    TRY(check_ptr(o, t.esz, "o"));
    TRY(check_ptr(stats, 8, "stats"));
    TRY(check_ptr(dout, t.stage_o ? t.esz : 16, "dout"));
    TRY(check_ptr(dq, t.esz, "dq"));
    TRY(check_apart(a.q_st, t.batch, a.q_len, a.heads, a.dim, "dq"));
  }
  if (a.kv_len > 0) {
    TRY(check_ptr(dk, t.esz, "dk"));
    TRY(check_ptr(dv, t.esz, "dv"));
    TRY(check_apart(a.k_st, t.batch, a.kv_len, a.kv_heads, a.dim, "dk"));
    TRY(check_apart(a.v_st, t.batch, a.kv_len, a.kv_heads, a.dim, "dv"));
  }
  TRY(check_workspace(desc->workspace, desc->workspace_bytes, t.bytes_bwd));
  TRY(check_stream(desc->stream));
  hipStream_t s = static_cast<hipStream_t>(desc->stream);
  uint8_t *base = static_cast<uint8_t *>(desc->workspace);
  a.dq = dq;
  a.dk = dk;
  a.dv = dv;
  for (int i = 0; i < 3; ++i) {
    a.dq_st[i] = a.q_st[i];
    a.dk_st[i] = a.k_st[i];
    a.dv_st[i] = a.v_st[i];
    a.g_st[i] = a.o_st[i];
  }
  a.dq_vec = at_once(t, dq, a.dq_st);
  a.dk_vec = at_once(t, dk, a.dk_st);
  a.dv_vec = at_once(t, dv, a.dv_st);
  TRY(stage_inputs(t, q, k, v, base, s));
  a.o = o;
  a.dout = dout;
  if (t.stage_o && a.q_len > 0) {
    a.o = base + t.o_o;
    a.dout = base + t.o_g;
    TRY(stage_rows(t, o, a.o_st, a.q_len, a.heads, base + t.o_o, s));
    TRY(stage_rows(t, dout, a.g_st, a.q_len, a.heads, base + t.o_g, s));
  }
  a.q_lens = q_lens;
  a.kv_lens = kv_lens;
  a.mask = mask;
  a.stats = reinterpret_cast<float2 *>(const_cast<float *>(stats));
  a.delta = reinterpret_cast<float *>(base + t.o_delta);
  a.part = reinterpret_cast<float *>(base + t.o_part);
  if (attend_few_rows(t.bf16, a) && ((t.fwd_splits == 1 && t.dkv_splits == 1) || 4 * a.pairs >= 3 * kCus)) {
    a.splits = 1;
    HIP_TRY(launch_attend_few_rows(a, s));
    return HAPI_OK;
  }
  if (a.q_len > 0) {
    a.splits = t.fwd_splits;
    HIP_TRY(launch_attend_dq(t.bf16, a, s));
  }
  if (a.kv_len > 0) {
    a.splits = t.dkv_splits;
    HIP_TRY(launch_attend_dkv(t.bf16, a, s));
  }
  return HAPI_OK;
}

}  // extern "C"
