// Drives the host side of the trained tail (argument checks, tile rules, workspace
// layout, the sequence of launches) under AddressSanitizer and UBSan, with stand-ins
// for the kernel launchers that check what each is handed: every scratch region
// inside the workspace, no two of them overlapping, every count within the
// kernels' index types.  No address is read or written.  Prints "OK <calls>".
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <initializer_list>
#include <vector>

#include "tail.h"

static long g_calls = 0;
#define EXPECT(cond)                                                                            \
  do {                                                                                          \
    ++g_calls;                                                                                  \
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
int64_t g_ws_bytes = 0;
struct Region {
  const char *name;
  int64_t lo, hi;
};
std::vector<Region> g_regions;
void region(const char *name, const void *p, int64_t bytes) {
  if (bytes == 0) return;
  const Region r{name, (int64_t)((uintptr_t)p - (uintptr_t)kWs), (int64_t)((uintptr_t)p - (uintptr_t)kWs) + bytes};
  EXPECT(bytes > 0 && r.lo >= 0 && r.lo % 16 == 0 && r.hi <= g_ws_bytes);
  for (const Region &o : g_regions) {
    if (!std::strcmp(o.name, name)) {
      EXPECT(o.lo == r.lo && o.hi == r.hi);
      return;
    }
    EXPECT(r.hi <= o.lo || o.hi <= r.lo);
  }
  g_regions.push_back(r);
}
bool in_ws(const void *p) {
  const int64_t o = (int64_t)((uintptr_t)p - (uintptr_t)kWs);
  return o >= 0 && o < g_ws_bytes;
}
int g_fwd, g_finish, g_prepare, g_reduce, g_grads;
int64_t g_next_class;
}  // namespace

namespace hapi {
static int64_t tile_of(bool bf16, const HeadArgs &a) {
  const Variant v = head_variant(bf16, a.rows, a.classes);
  return v == BIG ? 256 : v == MID ? 128 : v == SMALL ? 64 : 32;
}
static void check_operands(bool bf16, const HeadArgs &a) {
  const int64_t esz = bf16 ? 2 : 4, v = 16 / esz;
  EXPECT(a.x_ld % v == 0 && a.w_ld % v == 0 && a.x_ld >= a.dim && a.w_ld >= a.dim && a.dx_pad >= a.dim);
  EXPECT(a.x_ld * 256 * esz < (int64_t)1 << 31 && a.w_ld * 256 * esz < (int64_t)1 << 31 && a.rows_pad * 64 * esz < (int64_t)1 << 31);
  if (in_ws(a.w)) region("w", a.w, a.classes * a.w_ld * esz);
  if (in_ws(a.x)) region("x", a.x, a.rows * a.x_ld * esz);
  const int64_t t = tile_of(bf16, a);
  EXPECT(ceil_div(a.rows, t) * ceil_div(a.classes, t) < (int64_t)1 << 31);
}
hipError_t launch_head_stage(bool bf16, const void *, int64_t ld_in, void *out, int64_t ld_out, int64_t rows, int dim,
                             hipStream_t) {
  EXPECT(in_ws(out) && ld_in >= dim && ld_out >= dim && rows >= 0);
  EXPECT((int64_t)((uintptr_t)out - (uintptr_t)kWs) + rows * ld_out * (bf16 ? 2 : 4) <= g_ws_bytes);
  return hipSuccess;
}
hipError_t launch_head_forward(bool bf16, const HeadArgs &a, hipStream_t) {
  check_operands(bf16, a);
  region("part", a.part, (int64_t)a.parts * a.rows * 8);
  if (head_variant(bf16, a.rows, a.classes) == BIG) {
    const int64_t c = head_big_classes(a.rows, a.classes);
    EXPECT(c > 0 && c <= a.classes && (c == a.classes || c % 256 == 0));
    EXPECT(c / 64 + ceil_div(a.classes - c, 128) * 2 <= a.parts + 3);
  }
  ++g_fwd;
  return hipSuccess;
}
hipError_t launch_head_finish(bool, const HeadArgs &a, hipStream_t) {
  region("part", a.part, (int64_t)a.parts * a.rows * 8);
  ++g_finish;
  return hipSuccess;
}
hipError_t launch_head_prepare(bool bf16, const HeadArgs &a, void *xs, int64_t xs_ld, hipStream_t) {
  EXPECT(xs == a.x && xs_ld == a.x_ld && a.rows_pad >= a.rows && a.rows_pad % kHeadRowPad == 0);
  check_operands(bf16, a);
  if (bf16 && a.rows > 0 && a.rows <= kFewRows) {  // x twice
    g_regions.pop_back();
    region("x", a.x, 2 * kFewRows * a.x_ld * 2);
  }
  region("info", a.info, a.rows_pad * 8);
  region("unit", a.unit, 4);
  region("id32", a.id32, a.rows * a.top * 4);
  region("cq", a.cq, a.rows * a.top * 4);
  g_next_class = 0;
  ++g_prepare;
  return hipSuccess;
}
static int64_t g_piece;
hipError_t launch_head_dlogits(bool bf16, const HeadArgs &a, hipStream_t) {
  EXPECT(a.v0 == g_next_class && a.piece >= 1 && a.v0 + a.piece <= a.classes && a.first == (a.v0 == 0));
  if (a.first) g_piece = a.piece;
  EXPECT(a.piece <= g_piece && (a.piece == g_piece || a.v0 + a.piece == a.classes) && (a.v0 % kHeadPiece == 0));
  g_next_class = a.v0 + a.piece;
  region("gt", a.gt, g_piece * a.rows_pad * (bf16 ? 2 : 4));
  if (a.db_part) region("db", a.db_part, (int64_t)(a.db_parts + (a.teacher ? a.bias_slices : 0)) * a.classes * 4);
  EXPECT(ceil_div(a.rows * a.top, 256) + ceil_div(a.classes, kBiasClasses) * a.bias_slices < (int64_t)1 << 31);
  return hipSuccess;
}
hipError_t launch_head_grads(bool bf16, const HeadArgs &a, hipStream_t) {
  EXPECT(a.splits >= 1 && a.splits <= 64 && a.w_splits >= 1 && a.w_splits <= 16);
  EXPECT(a.w_splits == 1 || a.piece == a.classes);
  EXPECT(a.dx_whole == (a.splits == 1 && g_piece == a.classes));
  const int64_t kt = bf16 ? 64 : 32;
  EXPECT(ceil_div(g_piece, kt) * a.splits < (int64_t)1 << 31 && ceil_div(a.rows, kt) * a.w_splits < (int64_t)1 << 31);
  if (!a.dx_whole) region("dx", a.dx_part, (int64_t)a.splits * a.rows * a.dx_pad * 4);
  if (a.w_splits > 1) region("dw", a.dw_part, (int64_t)a.w_splits * a.classes * a.dx_pad * 4);
  ++g_grads;
  return hipSuccess;
}
hipError_t launch_head_reduce(bool, const HeadArgs &a, hipStream_t) {
  EXPECT(g_next_class == a.classes);
  ++g_reduce;
  return hipSuccess;
}
static int g_norm;
hipError_t launch_norm_forward(bool, const NormArgs &, hipStream_t) {
  ++g_norm;
  return hipSuccess;
}
hipError_t launch_norm_backward(bool, const NormArgs &a, hipStream_t) {
  region("norm", a.part, (int64_t)kNormParts * 2 * a.dim * 4);
  ++g_norm;
  return hipSuccess;
}
}  // namespace hapi

static void *fake(int i) { return reinterpret_cast<void *>(((uintptr_t)1 << 45) + ((uintptr_t)i << 20)); }
static float *ffake(int i) { return static_cast<float *>(fake(i)); }

static void head(int dtype, int64_t rows, int dim, int64_t classes, int top, int64_t pad_x, int64_t pad_w, bool bias) {
  hapi_head_desc d{};
  d.dtype = dtype;
  d.rows = rows;
  d.dim = dim;
  d.classes = classes;
  d.top = top;
  d.temperature = top ? 2.0f : 1.0f;
  d.x_stride = pad_x ? dim + pad_x : 0;
  d.w_stride = pad_w ? dim + pad_w : 0;
  const int64_t f = hapi_head_workspace_bytes(&d, 0), b = hapi_head_workspace_bytes(&d, 1);
  EXPECT(f >= 0 && b >= f);
  const int64_t *ids = static_cast<const int64_t *>(fake(4));
  float *bi = bias ? ffake(3) : nullptr;
  for (int dir = 0; dir < 2; ++dir) {
    g_regions.clear();
    g_fwd = g_finish = g_prepare = g_grads = g_reduce = 0;
    g_ws_bytes = dir ? b : f;
    d.workspace = kWs;
    d.workspace_bytes = (size_t)g_ws_bytes;
    auto call = [&] {
      if (dir == 0)
        return top ? hapi_distill_forward(&d, fake(1), fake(2), bi, ids, ffake(5), ffake(6), ffake(7), ffake(8))
                   : hapi_xent_forward(&d, fake(1), fake(2), bi, ids, ffake(6), ffake(7));
      return top ? hapi_distill_backward(&d, fake(1), fake(2), bi, ids, ffake(5), ffake(7), ffake(8), ffake(9), fake(10),
                                         fake(11), bias ? ffake(12) : nullptr)
                 : hapi_xent_backward(&d, fake(1), fake(2), bi, ids, ffake(6), ffake(7), ffake(9), fake(10), fake(11),
                                      bias ? ffake(12) : nullptr);
    };
    EXPECT(call() == HAPI_OK);
    if (dir == 0) EXPECT(g_fwd == (rows > 0) && g_finish == (rows > 0));
    else EXPECT(g_prepare == 1 && g_grads >= 1 && g_reduce == 1);
    // a byte less than it uses, another device, a workspace off its alignment: refused,
    // nothing launched
    g_fwd = g_prepare = 0;
    int64_t used = 0;
    for (const Region &r : g_regions) used = r.hi > used ? r.hi : used;
    EXPECT(used > 0 || (dir == 0 && rows == 0));
    if (used > 0) {
      d.workspace_bytes = (size_t)used - 1;
      EXPECT(call() == HAPI_E_NOMEM && std::strlen(hapi_last_error()) > 0);
      d.workspace_bytes = (size_t)g_ws_bytes;
      d.workspace = kWs + 128;
      EXPECT(call() == HAPI_E_INVAL);
      d.workspace = nullptr;
      EXPECT(call() == HAPI_E_NOMEM);
      d.workspace = kWs;
      g_stream_device = 1;
      EXPECT(call() == HAPI_E_INVAL);
      g_stream_device = 0;
    }
    EXPECT(g_fwd == 0 && g_prepare == 0);
  }
}

int main() {
  for (int dtype : {HAPI_F32, HAPI_BF16})
    for (int64_t rows : {0, 1, 7, 32, 33, 100, 1000, 4097, 100001, 1 << 20})
      for (int dim : {1, 8, 100, 768, 4096, 1 << 18})
        for (int64_t classes : {1, 10, 257, 1000, 50021, 131072, 1 << 24})
          for (int top : {0, 1, 33, 1024})
            for (int pad : {0, 1, 8}) head(dtype, rows, dim, classes, top, pad, pad == 8 ? 1 : pad, top != 33);
  head(HAPI_F32, 1 << 20, 1 << 20, 1 << 24, 1024, 0, 0, true);

  hapi_head_desc h{};
  h.dtype = HAPI_BF16;
  h.rows = 4;
  h.dim = 64;
  h.classes = 100;
  h.temperature = 1.0f;
  auto refuses = [&](auto set, int code) {
    hapi_head_desc x = h;
    set(x);
    EXPECT(hapi_head_workspace_bytes(&x, 1) == code);
  };
  EXPECT(hapi_head_workspace_bytes(nullptr, 0) == HAPI_E_INVAL);
  refuses([](hapi_head_desc &x) { x.dtype = 7; }, HAPI_E_INVAL);
  refuses([](hapi_head_desc &x) { x.rows = -1; }, HAPI_E_INVAL);
  refuses([](hapi_head_desc &x) { x.rows = INT64_MAX; }, HAPI_E_UNSUPPORTED);
  refuses([](hapi_head_desc &x) { x.dim = INT32_MIN; }, HAPI_E_INVAL);
  refuses([](hapi_head_desc &x) { x.dim = INT32_MAX; }, HAPI_E_UNSUPPORTED);
  refuses([](hapi_head_desc &x) { x.classes = INT64_MAX; }, HAPI_E_UNSUPPORTED);
  refuses([](hapi_head_desc &x) { x.classes = INT64_MIN; }, HAPI_E_INVAL);
  refuses([](hapi_head_desc &x) { x.x_stride = INT64_MAX; }, HAPI_E_UNSUPPORTED);
  refuses([](hapi_head_desc &x) { x.w_stride = INT64_MIN; }, HAPI_E_INVAL);
  refuses([](hapi_head_desc &x) { x.top = INT32_MAX; }, HAPI_E_UNSUPPORTED);
  refuses([](hapi_head_desc &x) { x.top = -1; }, HAPI_E_INVAL);
  refuses([](hapi_head_desc &x) { x.top = 2, x.temperature = 0.0f; }, HAPI_E_INVAL);
  refuses([](hapi_head_desc &x) { x.top = 2, x.temperature = 1e-45f; }, HAPI_E_INVAL);

  for (int dtype : {HAPI_F32, HAPI_BF16})
    for (int64_t rows : {(int64_t)0, (int64_t)1, (int64_t)25216, (int64_t)1 << 40})
      for (int dim : {1, 768, 1111, 16384}) {
        hapi_norm_desc d{};
        d.dtype = dtype;
        d.rows = rows;
        d.dim = dim;
        g_regions.clear();
        g_ws_bytes = hapi_layernorm_workspace_bytes(&d);
        EXPECT(g_ws_bytes > 0);
        d.workspace = kWs;
        d.workspace_bytes = (size_t)g_ws_bytes;
        EXPECT(hapi_layernorm_forward(&d, fake(1), ffake(2), ffake(3), fake(4), ffake(5), ffake(6)) == HAPI_OK);
        EXPECT(hapi_layernorm_backward(&d, fake(1), fake(2), ffake(3), ffake(4), ffake(5), fake(6), ffake(7), ffake(8)) ==
               HAPI_OK);
        d.rows = INT64_MAX;
        EXPECT(hapi_layernorm_workspace_bytes(&d) == HAPI_E_UNSUPPORTED);
        d.rows = rows;
        d.x_stride = INT64_MIN;
        EXPECT(hapi_layernorm_workspace_bytes(&d) == HAPI_E_INVAL);
        d.x_stride = INT64_MAX;
        EXPECT(hapi_layernorm_workspace_bytes(&d) == (rows > 0 ? HAPI_E_UNSUPPORTED : g_ws_bytes));
      }
  std::printf("OK %ld\n", g_calls);
  return 0;
}
