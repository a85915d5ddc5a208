// Drives the host side of the trained block's operators (argument checks, split rules,
// workspace layout, the sequence of launches) under AddressSanitizer and UBSan, with
// stand-ins for the kernel launchers that check what each is handed: every scratch
// region inside the workspace, no two of them overlapping, every grid within a launch's
// limits.  No address is read or written.  Prints "OK <checks>".
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <deque>
#include <string>
#include <vector>

#include "block.h"

static long g_checks = 0;
#define EXPECT(cond)                                                                            \
  do {                                                                                          \
    ++g_checks;                                                                                 \
    if (!(cond)) {                                                                              \
      std::fprintf(stderr, "FAILED %s at line %d: %s\n", #cond, __LINE__, hapi_last_error());   \
      std::exit(2);                                                                             \
    }                                                                                           \
  } while (0)

// The device that streams and calls are on: no GPU is asked.
static int g_stream_device = 0;
extern "C" hipError_t hipStreamGetDevice(hipStream_t, hipDevice_t *d) {
  *d = g_stream_device;
  return hipSuccess;
}
extern "C" hipError_t hipGetDevice(int *d) {
  *d = 0;
  return hipSuccess;
}

namespace {
uint8_t *const kWs = reinterpret_cast<uint8_t *>((uintptr_t)1 << 46);
void *const kAt = reinterpret_cast<void *>((uintptr_t)1 << 45);  // any tensor
int64_t g_ws_bytes = 0;
struct Region {
  const char *name;
  int64_t lo, hi;
};
std::vector<Region> g_regions;
bool in_ws(const void *p) {
  const int64_t o = (int64_t)((uintptr_t)p - (uintptr_t)kWs);
  return o >= 0 && o < g_ws_bytes;
}
const char *unique() {  // of a region that no later launch names again
  static std::deque<std::string> names;
  names.push_back("#" + std::to_string(names.size()));
  return names.back().c_str();
}
void region(const char *name, const void *p, int64_t bytes, int64_t align = 16) {
  const Region r{name, (int64_t)((uintptr_t)p - (uintptr_t)kWs), (int64_t)((uintptr_t)p - (uintptr_t)kWs) + bytes};
  EXPECT(bytes > 0 && r.lo >= 0 && r.lo % align == 0 && r.hi <= g_ws_bytes);
  for (const Region &o : g_regions) {
    if (!std::strcmp(o.name, name)) {
      EXPECT(o.lo == r.lo);
      return;
    }
    EXPECT(r.hi <= o.lo || o.hi <= r.lo);
  }
  g_regions.push_back(r);
}
void forget(const char *name) {
  for (size_t i = 0; i < g_regions.size(); ++i)
    if (!std::strcmp(g_regions[i].name, name)) g_regions.erase(g_regions.begin() + (long)i--);
}
int g_stage, g_forward, g_dq, g_dkv, g_rotary, g_squares, g_clip, g_join, g_norm;
int64_t g_values, g_parts;
constexpr int64_t kBlocks = ((int64_t)1 << 32) / 256;
}  // namespace

namespace hapi {
hipError_t launch_grad_squares(const GradArgs &a, int blocks, hipStream_t) {
  EXPECT(blocks >= 1 && blocks <= kGradBlocks && a.count >= 1 && a.count <= kGradTensors);
  region(unique(), a.part, (int64_t)blocks * 8, 8);
  EXPECT(a.seg[0] == 0);
  for (int t = 0; t < a.count; ++t) {
    EXPECT(a.size[t] > 0 && (int64_t)(a.seg[t + 1] - a.seg[t]) == ceil_div(a.size[t], a.seg_size));
    g_values += a.size[t];
  }
  EXPECT(blocks <= a.seg[a.count]);
  g_parts += blocks;
  ++g_squares;
  return hipSuccess;
}
hipError_t launch_grad_clip(const GradArgs &a, int blocks, hipStream_t) {
  EXPECT(blocks >= 1 && blocks <= kGradBlocks && a.parts >= 1 && in_ws(a.part) && in_ws(a.part + a.parts - 1));
  EXPECT(a.parts <= (int64_t)hapi::kGradSumLaunches * hapi::kGradBlocks && (a.norm != nullptr) == (g_clip == 0));
  for (int t = 0; t < a.count; ++t) g_values -= a.size[t];
  ++g_clip;
  return hipSuccess;
}
hipError_t launch_grad_join(const double *part, int64_t parts, double *out, hipStream_t) {
  EXPECT(parts == g_parts && part == (const double *)kWs && out >= part + parts && in_ws(out + kGradBlocks - 1));
  ++g_join;
  return hipSuccess;
}
hipError_t launch_grad_norm(const double *part, int64_t parts, float *, hipStream_t) {
  EXPECT(parts == 0 || (in_ws(part) && in_ws(part + parts - 1)));
  ++g_norm;
  return hipSuccess;
}
static void check_rotary(bool bf16, int v, const RotaryArgs &a) {
  EXPECT(v >= 1 && v <= (bf16 ? 8 : 4) && a.dim <= kRotaryMaxDim && 2 * a.pairs <= a.dim);
  if (!a.neighbours) EXPECT(a.pairs % v == 0 && (v == 1 || (a.dim - 2 * a.pairs) % (2 * v) == 0));
  else EXPECT(v == 1 || a.dim % (2 * v) == 0);
  for (int w = 0; w < 2; ++w) {
    EXPECT((a.heads[w] == 0) == (a.head_groups[w] == 0) && a.head_groups[w] <= a.heads[w]);
    EXPECT(a.tokens * a.head_groups[w] < (int64_t)1 << 31);
  }
  ++g_rotary;
}
hipError_t launch_rotary_forward(bool bf16, int v, const RotaryArgs &a, hipStream_t) {
  check_rotary(bf16, v, a);
  return hipSuccess;
}
hipError_t launch_rotary_backward(bool bf16, int v, const RotaryArgs &a, hipStream_t) {
  check_rotary(bf16, v, a);
  if (a.norm) region("part", a.part, (int64_t)2 * kRotaryParts * a.dim * 4);
  return hipSuccess;
}
hipError_t launch_attend_stage(bool bf16, const StageArgs &a, hipStream_t) {
  const int64_t esz = bf16 ? 2 : 4;
  EXPECT(a.ld % (16 / esz) == 0 && a.ld >= a.dim);
  if (a.count > 0) {
    region(unique(), a.out, a.count * a.ld * esz);
  }
  ++g_stage;
  return hipSuccess;
}
// Reads of 16 bytes at 32-bit offsets from a tile's first token.
static void check_rows(const int64_t *st, int64_t heads, int64_t rows, int64_t esz) {
  const int64_t v = 16 / esz;
  EXPECT(st[0] % v == 0 && st[1] % v == 0 && st[2] % v == 0);
  EXPECT((rows * st[1] + heads * st[2]) * esz + 4096 < (int64_t)1 << 31);
}
static void check_attend(bool bf16, const AttendArgs &a, bool back) {
  const int64_t esz = bf16 ? 2 : 4;
  if (a.q_len > 0) check_rows(a.q_st, a.group, 65, esz);
  check_rows(a.k_st, 0, 65, esz);
  check_rows(a.v_st, 0, 65, esz);
  if (back && a.q_len > 0) {
    check_rows(a.o_st, a.group, 65, esz);
    check_rows(a.g_st, a.group, 65, esz);
  }
  EXPECT(a.splits >= 1 && a.splits <= 64 && a.group * a.kv_heads == a.heads && a.dim4 % 4 == 0 && a.dim4 >= a.dim);
  EXPECT(a.scale > 0 && a.c > 0);
}
hipError_t launch_attend_forward(bool bf16, const AttendArgs &a, hipStream_t) {
  check_attend(bf16, a, false);
  const int64_t rows = (int64_t)a.q_len * a.group;
  EXPECT(ceil_div(rows, 32 * attend_row_waves(rows)) * a.splits * a.pairs <= kBlocks);
  if (a.splits > 1) {
    region("ml", a.part_ml, a.splits * a.pairs * rows * 16);
    region("part", a.part, a.splits * a.pairs * rows * a.dim4 * 4);
    EXPECT(ceil_div(rows * a.pairs * (a.dim4 / 4), 256) <= kBlocks);
  }
  ++g_forward;
  return hipSuccess;
}
hipError_t launch_attend_dq(bool bf16, const AttendArgs &a, hipStream_t) {
  check_attend(bf16, a, true);
  const int64_t rows = (int64_t)a.q_len * a.group;
  EXPECT(ceil_div(rows, 32 * attend_row_waves(rows)) * a.splits * a.pairs <= kBlocks);
  region("delta", a.delta, a.pairs * rows * 4);
  if (a.splits > 1) region("dq", a.part, a.splits * a.pairs * rows * a.dim4 * 4);
  forget("dq");
  ++g_dq;
  return hipSuccess;
}
hipError_t launch_attend_dkv(bool bf16, const AttendArgs &a, hipStream_t) {
  check_attend(bf16, a, true);
  const int64_t rows = (int64_t)a.q_len * a.group;
  // 512 threads for 128 keys of bf16 heads past 96 values, else 256; all of a launch: 32 bits
  EXPECT(ceil_div(a.kv_len, 128) * a.splits * a.pairs * (bf16 && a.dim > 96 ? 512 : 256) <= kMaxLaunchThreads);
  if (rows > 0) region("delta", a.delta, a.pairs * rows * 4);
  if (a.splits > 1) region("dkv", a.part, a.splits * 2 * a.pairs * (int64_t)a.kv_len * a.dim4 * 4);
  ++g_dkv;
  return hipSuccess;
}
hipError_t launch_attend_few_rows(const AttendArgs &a, hipStream_t) {
  check_attend(true, a, true);
  const int64_t rows = (int64_t)a.q_len * a.group;
  EXPECT(rows >= 1 && rows <= 64 && a.dim <= 64 && a.kv_len >= 1 && a.splits == 1 && a.pairs <= kBlocks);
  ++g_dq;
  ++g_dkv;
  return hipSuccess;
}
}  // namespace hapi

static void attention(int dtype, int64_t b, int64_t q, int64_t k, int heads, int kv, int dim, int layout) {
  hapi_attention_desc d = {};
  d.dtype = dtype;
  d.head_dim = dim;
  d.heads = heads;
  d.kv_heads = kv;
  d.batch = b;
  d.q_len = q;
  d.kv_len = k;
  if (layout == 1) {  // [batch, heads, tokens, dim + 8]
    const int64_t ld = dim + 8;
    const int64_t qs[3] = {heads * q * ld, ld, q * ld}, ks[3] = {kv * k * ld, ld, k * ld};
    for (int i = 0; i < 3; ++i) d.q_stride[i] = d.o_stride[i] = qs[i], d.k_stride[i] = d.v_stride[i] = ks[i];
  }
  if (layout == 2) {  // token strides past what a tile's offsets hold
    const int64_t t = ((int64_t)1 << 20) + 8;
    const int64_t qs[3] = {(q + 1) * t, t, dim + 8}, ks[3] = {(k + 1) * t, t, dim + 8};
    for (int i = 0; i < 3; ++i) d.q_stride[i] = d.o_stride[i] = qs[i], d.k_stride[i] = d.v_stride[i] = ks[i];
  }
  const int64_t fwd = hapi_cross_attention_workspace_bytes(&d, 0), both = hapi_cross_attention_workspace_bytes(&d, 1);
  if (fwd == HAPI_E_UNSUPPORTED) {
    EXPECT(both == HAPI_E_UNSUPPORTED);
    return;
  }
  EXPECT(fwd >= 0 && both >= fwd);
  d.workspace = kWs;
  float *f = static_cast<float *>(kAt);
  g_regions.clear();
  d.workspace_bytes = g_ws_bytes = fwd;
  int n = g_forward;
  EXPECT(hapi_cross_attention_forward(&d, kAt, kAt, kAt, nullptr, nullptr, nullptr, kAt, f) == HAPI_OK);
  EXPECT(g_forward - n == (b > 0 && q > 0));
  if (fwd > 0 && b > 0 && q > 0) {
    d.workspace_bytes = fwd - 256;
    EXPECT(hapi_cross_attention_forward(&d, kAt, kAt, kAt, nullptr, nullptr, nullptr, kAt, f) == HAPI_E_NOMEM);
  }
  g_regions.clear();
  d.workspace_bytes = g_ws_bytes = both;
  const int nq = g_dq, nk = g_dkv;
  EXPECT(hapi_cross_attention_backward(&d, kAt, kAt, kAt, nullptr, nullptr, nullptr, kAt, f, kAt, kAt, kAt, kAt) == HAPI_OK);
  EXPECT(g_dq - nq == (b > 0 && q > 0) && g_dkv - nk == (b > 0 && k > 0));
  g_stream_device = 1;
  if (b > 0 && q > 0)
    EXPECT(hapi_cross_attention_forward(&d, kAt, kAt, kAt, nullptr, nullptr, nullptr, kAt, f) == HAPI_E_INVAL);
  g_stream_device = 0;
}

static void rotary(int dtype, int64_t b, int64_t l, int heads, int kv, int dim, int axes, int each, int neighbours, int norm) {
  hapi_rotary_desc d = {};
  d.dtype = dtype;
  d.head_dim = dim;
  d.heads = heads;
  d.kv_heads = kv;
  d.batch = b;
  d.length = l;
  d.axes = axes;
  for (int i = 0; i < axes; ++i) d.sections[i] = each;
  d.neighbours = neighbours;
  d.norm = norm;
  d.eps = 1e-6f;
  const int64_t need = hapi_rotary_workspace_bytes(&d);
  EXPECT(need >= 0 && (need > 0) == (norm != 0));
  d.workspace = kWs;
  d.workspace_bytes = g_ws_bytes = need;
  g_regions.clear();
  float *f = static_cast<float *>(kAt);
  const float *gq = norm && heads ? f : nullptr, *gk = norm && kv ? f : nullptr;
  void *q = heads ? kAt : nullptr, *k = kv ? kAt : nullptr;
  const int64_t *pos = axes ? static_cast<int64_t *>(kAt) : nullptr;
  const double *freq = axes ? static_cast<double *>(kAt) : nullptr;
  const int n = g_rotary;
  EXPECT(hapi_rotary_forward(&d, q, k, gq, gk, pos, freq, nullptr, q, k) == HAPI_OK);
  EXPECT(hapi_rotary_backward(&d, q, k, q, k, gq, gk, pos, freq, nullptr, q, k, const_cast<float *>(gq), const_cast<float *>(gk)) == HAPI_OK);
  EXPECT(g_rotary - n == (b * l > 0) + (b * l > 0 || norm));
}

static void gradients(int count, int64_t size, int zeros_every, bool in_place) {
  std::vector<const void *> in(count);
  std::vector<void *> out(count);
  std::vector<int64_t> sizes(count);
  std::vector<int32_t> types(count);
  const int64_t apart = (size * 4 + 4096) * 2;
  int64_t values = 0;
  for (int i = 0; i < count; ++i) {
    // neither in order of their addresses nor next to their outputs
    const int64_t at = (int64_t)(((int64_t)i * 7919) % count) * apart;
    in[i] = static_cast<uint8_t *>(kAt) + at;
    out[i] = in_place ? const_cast<void *>(in[i]) : static_cast<uint8_t *>(kAt) + at + apart / 2;
    sizes[i] = zeros_every && i % zeros_every == 0 ? 0 : size;
    types[i] = i % 2 ? HAPI_BF16 : HAPI_F32;
    values += sizes[i];
  }
  hapi_gradient_desc d = {};
  d.count = count;
  d.grads = in.data();
  d.out = in_place && count % 2 ? nullptr : out.data();
  d.sizes = sizes.data();
  d.dtypes = types.data();
  d.max_norm = 1.0f;
  const int64_t need = hapi_gradient_workspace_bytes(&d);
  EXPECT(need > 0);
  d.workspace = kWs;
  d.workspace_bytes = g_ws_bytes = need;
  float *norm = static_cast<float *>(kAt);
  g_regions.clear();
  g_squares = g_clip = g_join = g_norm = 0;
  g_values = g_parts = 0;
  EXPECT(hapi_gradient_clip(&d, norm) == HAPI_OK);
  EXPECT(g_values == 0 && g_squares == g_clip && (g_norm == 1) == (values == 0) && (g_join == 1) == (g_squares > hapi::kGradSumLaunches));
  g_regions.clear();
  g_squares = g_join = g_norm = 0;
  g_values = g_parts = 0;
  EXPECT(hapi_gradient_norm(&d, norm) == HAPI_OK);
  EXPECT(g_values == values && g_norm == 1);
  d.workspace_bytes = need - 256;
  EXPECT(hapi_gradient_norm(&d, norm) == HAPI_E_NOMEM);
}

int main() {
  const int64_t lengths[] = {0, 1, 2, 31, 32, 33, 64, 65, 127, 128, 129, 197, 1000, 4097, 70000, 1 << 20, (int64_t)1 << 30};
  const int heads[][2] = {{1, 1}, {12, 12}, {16, 4}, {7, 1}, {512, 1}, {96, 2}};
  const int dims[] = {1, 3, 8, 32, 33, 40, 64, 72, 80, 96, 100, 127, 128};
  for (int dtype : {HAPI_F32, HAPI_BF16})
    for (int64_t q : lengths)
      for (int64_t k : lengths)
        for (const auto &h : heads)
          for (int dim : dims)
            for (int64_t b : {(int64_t)0, (int64_t)1, (int64_t)5, (int64_t)1 << 16})
              for (int layout = 0; layout < 3; ++layout) {
                // sizes whose bytes a 63-bit number holds
                if (((double)q * h[0] + (double)k * h[1]) * (double)b * dim * (layout == 2 ? 1e6 / dim : 1.0) > 1e15) continue;
                attention(dtype, b, q, k, h[0], h[1], dim, layout);
              }
  for (int dtype : {HAPI_F32, HAPI_BF16})
    for (int64_t b : {0, 1, 7, 128})
      for (int64_t l : {0, 1, 197, 4099})
        for (const auto &h : heads)
          for (int dim : {1, 2, 7, 16, 33, 64, 80, 128, 255, 256})
            for (int axes = 0; axes <= 4; ++axes)
              for (int each : {1, 5, 8, 16})
                for (int flags = 0; flags < 4; ++flags)
                  if (2 * axes * each <= dim) {
                    rotary(dtype, b, l, h[0], h[1], dim, axes, each, flags & 1, flags >> 1);
                    rotary(dtype, b, l, h[0], 0, dim, axes, each, flags & 1, flags >> 1);
                    rotary(dtype, b, l, 0, h[1], dim, axes, each, flags & 1, flags >> 1);
                  }
  for (int count : {0, 1, 2, 119, 120, 121, 480, 481, 600, 5000})
    for (int64_t size : {(int64_t)1, (int64_t)8, (int64_t)1000, (int64_t)100003, (int64_t)1 << 22, (int64_t)1 << 30})
      for (int zeros : {0, 1, 2, 3})
        for (bool in_place : {true, false}) gradients(count, size, zeros, in_place);
  std::printf("OK %ld\n", g_checks);
  return 0;
}
