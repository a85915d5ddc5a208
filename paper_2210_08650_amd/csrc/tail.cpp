// Entry points of the trained tail: argument checks, workspace layout and the
// launches of layer norm and of the classifier's losses.  Declared in hapi.h.
#include <algorithm>
#include <cmath>

#include "host_checks.h"
#include "tail.h"

namespace hapi {

// As many rows to every block, up to four: gamma and beta are read once, and
// there are blocks enough for the CUs (25,216 x 768: 15.2 us with one, 14.8 with
// two, 15.3 with four, 17.0 with eight).
int64_t norm_forward_blocks(int64_t want, int threads) {
  const int64_t iters = std::max<int64_t>(1, std::min<int64_t>(4, want / 1536));
  return std::min(ceil_div(want, iters), kMaxLaunchThreads / threads);
}

// ------------------------------------------------------------------ tile rules

Variant head_variant(bool bf16, int64_t rows, int64_t classes) {
  // The smallest calls spread over the CUs: up to two workgroups of 32 x 32 tiles each
  // (forward product of 128 x 2048 x 1000 7.9 us, in 64 x 64 tiles 13.6; of
  // 8 x 768 x 1000 5.4 us, in 32 x 128 tiles 8.4).
  if (ceil_div(rows, 32) * ceil_div(classes, 32) <= 2 * kCus) return TINY;
  if (rows <= kFewRows) return FEW;
  const int64_t big = ceil_div(rows, 256) * ceil_div(classes, 256), mid = ceil_div(rows, 128) * ceil_div(classes, 128),
                small = ceil_div(rows, 64) * ceil_div(classes, 64);
  double tb, tm, ts;
  if (bf16) {
    // 27.5, 19 and 10.3 us a round of 256, 512 and 768 workgroups at 768 features
    // (4096 x 768 x 32000); the last round less when it holds one to a CU.  The rule
    // takes their ratios for every width.
    tb = 27.5 * (double)ceil_div(big, kCus);
    tm = 19.0 * (double)(mid / (2 * kCus)) + (mid % (2 * kCus) == 0 ? 0.0 : mid % (2 * kCus) <= kCus ? 12.0 : 19.0);
    const int64_t r = small % (3 * kCus);
    ts = 10.3 * (double)(small / (3 * kCus)) + (r == 0 ? 0.0 : r <= kCus ? 5.0 : r <= 2 * kCus ? 7.5 : 10.3);
  } else {
    // the matrix pipes are the bound: a CU's workgroups take turns on them
    tb = 16.0 * (double)ceil_div(big, kCus);
    tm = 4.25 * (double)ceil_div(mid, kCus);
    ts = 1.06 * (double)ceil_div(small, kCus);
  }
  return tb <= tm && tb <= ts ? BIG : tm <= ts ? MID : SMALL;
}

// The classes that 256 x 256 tiles take, the others going to 128 x 128 tiles in a
// launch of their own: whole rounds of the large ones, where what is left of a
// round costs more in them (1000 x 520 x 50,021, 784 tiles: 75 us; 768 of them and 56
// small ones 60 + 10).  A part is 64 classes (or rows, for dbias) in either.
int64_t head_big_classes(int64_t rows, int64_t classes) {
  const int64_t rt = ceil_div(rows, 256), tiles = rt * ceil_div(classes, 256);
  const int64_t whole = tiles / kCus * kCus / rt * 256;  // classes of the whole rounds
  if (whole == 0 || whole >= classes) return classes;
  const int64_t mid = ceil_div(rows, 128) * ceil_div(classes - whole, 128);
  // rounds as in head_variant(): 19 us for 512 of them, 27.5 for 256 large ones
  const double tm = 19.0 * (double)(mid / (2 * kCus)) + (mid % (2 * kCus) <= kCus ? 12.0 : 19.0);
  return tm + 3.0 < 27.5 * (double)(ceil_div(tiles, kCus) - tiles / kCus) ? whole : classes;
}

int head_parts(bool bf16, int64_t rows, int64_t classes) {
  switch (head_variant(bf16, rows, classes)) {
    case BIG:  // a tile's parts past these are empty, and not written
    case MID: return (int)ceil_div(classes, 128) * 2;
    case SMALL: return (int)ceil_div(classes, 64) * 2;
    case TINY: return (int)ceil_div(classes, 32);
    default: return (int)ceil_div(classes, 128) * 4;
  }
}
HeadLaunch head_forward_launch(bool bf16, int64_t rows, int64_t classes, int64_t c0) {
  HeadLaunch l;
  l.v = head_variant(bf16, rows, classes);
  int64_t end = classes;
  if (l.v == BIG && bf16) {
    const int64_t big = head_big_classes(rows, classes);
    if (c0 < big) end = big;
    else l.v = MID;
  }
  // No more threads than a launch takes: 131,072 rows of 4,194,304 classes, 2^23 tiles
  // of 512 threads, are two.
  const int64_t threads = l.v == BIG ? 512 : 256, tile_rows = l.v == BIG ? 256 : l.v == MID ? 128 : l.v == SMALL ? 64 : 32,
                tile_classes = l.v == BIG ? 256 : l.v == MID || l.v == FEW ? 128 : l.v == SMALL ? 64 : 32;
  const int64_t most = kMaxLaunchThreads / threads / std::max<int64_t>(ceil_div(rows, tile_rows), 1) * tile_classes;
  l.classes = std::min(end - c0, most);
  l.part = (int)(c0 / (l.v == BIG || l.v == MID ? 64 : 32));
  l.parts = head_parts(bf16, rows, classes) - l.part;
  return l;
}
int head_db_parts(bool bf16, int64_t rows, int64_t classes) {
  switch (head_variant(bf16, rows, classes)) {
    case BIG:
    case MID: return (int)ceil_div(rows, 128) * 2;
    case SMALL: return (int)ceil_div(rows, 64) * 2;
    default: return (int)ceil_div(rows, 32);
  }
}
namespace {
struct GradTiles {
  Variant v;
  int64_t nx, nw;  // tiles of dx and of dW
};
GradTiles grad_tiles(bool bf16, int64_t rows, int dim, int64_t classes, int64_t piece) {
  GradTiles t;
  t.v = head_variant(bf16, rows, classes);
  if (t.v == TINY) t.v = rows <= kFewRows ? FEW : SMALL;
  const int64_t br = t.v == BIG ? 256 : t.v == MID ? 128 : t.v == SMALL ? 64 : 32;
  const int64_t ba = t.v == BIG ? 256 : t.v == SMALL ? 64 : 128, bc = t.v == BIG ? 256 : t.v == MID ? 128 : 64;
  t.nx = ceil_div(rows, br) * ceil_div(dim, ba);
  t.nw = ceil_div(piece, bc) * ceil_div(dim, t.v == FEW ? 64 : ba);
  return t;
}
}  // namespace

bool head_few_apart(int dim, int64_t piece) { return ceil_div(dim, 64) * ceil_div(piece, 64) > 4 * kCus; }

// dW's rows split over workgroups where its tiles leave CUs idle (few classes, many
// rows), at least 8 k-tiles to each; its partial sums are of all classes, so with one
// piece of them only.  256 x 256 tiles up to one a CU (a step of 1000 x 1024 x 10000 in
// two splits 129 us, in one 114), others up to two (2048 x 768 x 1000 51 us, one 55).
int head_w_splits(bool bf16, int64_t rows, int dim, int64_t classes, int64_t piece) {
  if (piece < classes) return 1;
  const GradTiles t = grad_tiles(bf16, rows, dim, classes, piece);
  const int64_t most = ceil_div(rows, bf16 ? 64 : 32) / 8, want = (t.v == BIG ? 1 : 2) * kCus / std::max<int64_t>(t.nw, 1);
  return (int)std::max<int64_t>(1, std::min<int64_t>(std::min(most, want), 16));
}

// Slices of the entries: 512 blocks or more, of 128 classes and one slice each.
int head_bias_slices(int64_t classes) {
  return (int)std::max<int64_t>(8, std::min<int64_t>(64, 512 / ceil_div(classes, kBiasClasses)));
}

int head_splits(bool bf16, int64_t rows, int dim, int64_t classes, int64_t piece, int w_splits) {
  const GradTiles tiles = grad_tiles(bf16, rows, dim, classes, piece);
  const Variant v = tiles.v;
  // few rows: dW has a launch of its own where it has many tiles
  const int64_t nx = tiles.nx, nw = v == FEW && head_few_apart(dim, piece) ? 0 : tiles.nw * w_splits;
  if (nx == 0) return 1;
  const int64_t kt = bf16 ? 64 : 32;
  const double kx = (double)ceil_div(piece, kt), kw = (double)ceil_div(rows, kt) / w_splits + 4.0;
  // The launch's time in a workgroup's k-tiles: dx's rounds over as many workgroups as
  // run at once, then dW's as places come free; and the partial sums' way through
  // memory.
  const int64_t cus = kCus * (v == MID ? 2 : v == SMALL ? (bf16 ? 3 : 4) : 1);
  double best = 0.0;
  int64_t pick = 1;
  for (int64_t s = 1; s <= 64 && s * 4 <= (int64_t)kx + 3; ++s) {
    const double lx = kx / (double)s + 4.0;
    const int64_t n = nx * s, full = n / cus, rest = n % cus;
    const double t0 = (double)full * lx, t1 = t0 + lx;
    // earliest time by which the places have run all of dW's workgroups: the early
    // ones' k-th round of them, with what the late ones have done by then
    double end = rest ? t1 : t0;
    if (nw > 0)
      for (int64_t k = std::max<int64_t>(1, (int64_t)((double)nw / cus) - 1);; ++k) {
        const double t = t0 + (double)k * kw;
        const int64_t late = t > t1 ? (int64_t)((t - t1) / kw) : 0;
        if ((cus - rest) * k + rest * late < nw) continue;
        end = std::max(end, t);
        break;
      }
    // one split of one piece is stored whole
    const double bytes = s == 1 && piece >= classes ? 0.0 : (double)s * (double)rows * (double)dim * 8.0;
    const double ktile_bytes = v == BIG ? 8.0e6 : v == MID ? 3.0e6 : 1.0e6;  // memory traffic in a k-tile's time
    const double cost = end + bytes / ktile_bytes;
    if (s == 1 || cost < best) {
      best = cost;
      pick = s;
    }
  }
  return (int)pick;
}

namespace {

constexpr int64_t kMaxRows = (int64_t)1 << 20;
constexpr int64_t kMaxLd = (int64_t)1 << 20;     // a tile's rows lie within 2^31 bytes of its first
constexpr int64_t kMaxClasses = (int64_t)1 << 24;
constexpr int kMaxTop = 1024;
constexpr float kMinTemperature = 0x1p-60f;  // T^2, 1 / T and the exponent's log2(e) / T stay normal numbers
// Of dz^T: one piece of the classes, or kHeadPiece classes where those are more (1 GiB at
// 2^20 rows in float32).
constexpr int64_t kPieceBytes = (int64_t)256 << 20;

// ---------------------------------------------------------------- layer norm

struct Norm {
  bool bf16;
  size_t esz;
  NormArgs a;
};

int read_norm(const hapi_norm_desc *d, Norm &n) {
  if (!d) return fail(HAPI_E_INVAL, "desc is NULL");
  if (d->dtype != HAPI_F32 && d->dtype != HAPI_BF16) return fail(HAPI_E_INVAL, "unknown dtype %d", d->dtype);
  if (d->reserved) return fail(HAPI_E_INVAL, "reserved must be 0");
  if (d->rows < 0) return fail(HAPI_E_INVAL, "rows must be >= 0");
  if (d->dim < 1) return fail(HAPI_E_INVAL, "dim must be >= 1");
  if (d->dim > kNormMaxDim) return fail(HAPI_E_UNSUPPORTED, "dim %d (at most %d)", d->dim, kNormMaxDim);
  if ((d->x_stride != 0 && d->x_stride < d->dim) || (d->y_stride != 0 && d->y_stride < d->dim))
    return fail(HAPI_E_INVAL, "a row stride must be 0 or >= dim");
  if (!(d->eps >= 0.0f) || !std::isfinite(d->eps)) return fail(HAPI_E_INVAL, "eps must be finite and >= 0");
  n.bf16 = d->dtype == HAPI_BF16;
  n.esz = n.bf16 ? 2 : 4;
  n.a = NormArgs{};
  n.a.rows = d->rows;
  n.a.dim = d->dim;
  n.a.eps = d->eps;
  n.a.x_ld = d->x_stride ? d->x_stride : d->dim;
  n.a.y_ld = d->y_stride ? d->y_stride : d->dim;
  // element offsets are 64 bits; the bytes of a tensor must be too
  const int64_t most = ((int64_t)1 << 60) / std::max(n.a.x_ld, n.a.y_ld);
  if (d->rows > most) return fail(HAPI_E_UNSUPPORTED, "rows times stride exceeds 2^60");
  return HAPI_OK;
}

int64_t norm_workspace(const Norm &n) { return up((int64_t)kNormParts * 2 * n.a.dim * 4, kAlign); }

// ---------------------------------------------------------------- classifier

struct Head {
  bool bf16;
  int esz, v;  // bytes of an element, elements of 16 bytes
  HeadArgs a;
  bool stage_x, stage_w;
  int64_t piece;     // classes of a piece
  int64_t bytes_fwd, bytes_bwd;
  // byte offsets into the workspace
  int64_t o_part, o_xs, o_ws, o_info, o_unit, o_id, o_cq, o_gt, o_db, o_dx, o_dw;
};

int read_head(const hapi_head_desc *d, Head &h) {
  if (!d) return fail(HAPI_E_INVAL, "desc is NULL");
  if (d->dtype != HAPI_F32 && d->dtype != HAPI_BF16) return fail(HAPI_E_INVAL, "unknown dtype %d", d->dtype);
  if (d->rows < 0) return fail(HAPI_E_INVAL, "rows must be >= 0");
  if (d->dim < 1 || d->classes < 1) return fail(HAPI_E_INVAL, "dim and classes must be >= 1");
  if (d->top < 0) return fail(HAPI_E_INVAL, "top must be >= 0");
  if (!(d->temperature >= kMinTemperature && d->temperature <= 1.0f / kMinTemperature))
    return fail(HAPI_E_INVAL, "temperature must be in [2^-60, 2^60]");
  if (d->top == 0 && d->temperature != 1.0f) return fail(HAPI_E_INVAL, "cross entropy has temperature 1");
  if ((d->x_stride != 0 && d->x_stride < d->dim) || (d->w_stride != 0 && d->w_stride < d->dim))
    return fail(HAPI_E_INVAL, "a row stride must be 0 or >= dim");
  if (d->rows > kMaxRows) return fail(HAPI_E_UNSUPPORTED, "%lld rows (at most 2^20)", (long long)d->rows);
  if (d->classes > kMaxClasses) return fail(HAPI_E_UNSUPPORTED, "%lld classes (at most 2^24)", (long long)d->classes);
  if (d->top > kMaxTop) return fail(HAPI_E_UNSUPPORTED, "top %d (at most %d)", d->top, kMaxTop);
  const int64_t x_ld = d->x_stride ? d->x_stride : d->dim, w_ld = d->w_stride ? d->w_stride : d->dim;
  if (x_ld > kMaxLd || w_ld > kMaxLd) return fail(HAPI_E_UNSUPPORTED, "dim and row strides must be <= 2^20");
  h = Head{};
  h.bf16 = d->dtype == HAPI_BF16;
  h.esz = h.bf16 ? 2 : 4;
  h.v = 16 / h.esz;
  HeadArgs &a = h.a;
  a.rows = d->rows;
  a.classes = d->classes;
  a.dim = d->dim;
  a.top = d->top > 0 ? d->top : 1;
  a.t = d->temperature;
  a.inv_t = 1.0f / d->temperature;
  a.x_in_ld = x_ld;
  a.w_in_ld = w_ld;
  a.rows_pad = up(std::max<int64_t>(d->rows, 1), kHeadRowPad);
  a.dx_pad = (int)up(d->dim, h.v);
  // The products read whole 16-byte slots: other widths and strides are copied
  // to padded rows first.
  h.stage_x = d->dim % h.v != 0 || x_ld % h.v != 0;
  h.stage_w = d->dim % h.v != 0 || w_ld % h.v != 0;
  a.x_ld = h.stage_x ? a.dx_pad : x_ld;
  a.w_ld = h.stage_w ? a.dx_pad : w_ld;
  a.parts = head_parts(h.bf16, d->rows, d->classes);
  // Pieces of equal size, as few as keep dz^T within kPieceBytes.
  const int64_t most = std::max<int64_t>(kPieceBytes / (a.rows_pad * h.esz) / kHeadPiece * kHeadPiece, kHeadPiece);
  const int64_t pieces = (d->classes + most - 1) / most;
  h.piece = std::min(up((d->classes + pieces - 1) / pieces, kHeadPiece), up(d->classes, kHeadPiece));
  a.db_parts = head_db_parts(h.bf16, d->rows, d->classes);
  a.w_splits = head_w_splits(h.bf16, d->rows, d->dim, d->classes, h.piece);
  a.splits = head_splits(h.bf16, d->rows, d->dim, d->classes, h.piece, a.w_splits);
  a.dx_whole = a.splits == 1 && h.piece >= d->classes;
  a.bias_slices = d->top > 0 && d->rows > 0 ? head_bias_slices(d->classes) : 0;  // without rows nothing writes them

  const int64_t xs = up(d->rows * a.dx_pad * h.esz, kAlign), ws = up(d->classes * a.dx_pad * h.esz, kAlign);
  int64_t o = 0;
  auto take = [&](int64_t bytes) {
    const int64_t at = o;
    o += up(bytes, kAlign);
    return at;
  };
  h.o_ws = take(h.stage_w ? ws : 0);
  h.o_xs = take(h.stage_x ? xs : 0);
  h.o_part = take((int64_t)a.parts * d->rows * 8);
  h.bytes_fwd = o;
  o = h.o_xs;
  // up to kFewRows rows of 16 bits: x twice
  take(h.bf16 && d->rows > 0 && d->rows <= kFewRows ? up((int64_t)2 * kFewRows * a.dx_pad * h.esz, kAlign) : xs);
  h.o_info = take(a.rows_pad * 8);
  h.o_unit = take(4);
  h.o_id = take(d->rows * a.top * 4);
  h.o_cq = take(d->rows * a.top * 4);
  h.o_gt = take(h.piece * a.rows_pad * h.esz);
  h.o_db = take((int64_t)(a.db_parts + a.bias_slices) * d->classes * 4);
  h.o_dx = take(a.dx_whole ? 0 : (int64_t)a.splits * d->rows * a.dx_pad * 4);
  h.o_dw = take(a.w_splits > 1 ? (int64_t)a.w_splits * d->classes * a.dx_pad * 4 : 0);
  h.bytes_bwd = o;
  return HAPI_OK;
}

// The caller's x and w, where the products can read them as they are.
int check_head_inputs(const hapi_head_desc *d, const Head &h, const void *x, const void *w, const float *bias,
                      const int64_t *ids, const char *ids_name) {
  if (d->rows > 0) {
    TRY(check_ptr(x, h.stage_x ? h.esz : 16, "x"));
    TRY(check_ptr(ids, 8, ids_name));
  }
  TRY(check_ptr(w, h.stage_w ? h.esz : 16, "weight"));
  if (bias) TRY(check_ptr(bias, 4, "bias"));
  return HAPI_OK;
}

int head_forward(const hapi_head_desc *d, Head &h, const void *x, const void *w, const float *bias, const int64_t *ids,
                 const float *teacher, float *loss, float *stats, float *picked) {
  if (d->rows == 0) return HAPI_OK;
  TRY(check_ptr(loss, 4, "loss"));
  TRY(check_ptr(stats, 8, "stats"));
  TRY(check_workspace(d->workspace, d->workspace_bytes, h.bytes_fwd));
  TRY(check_stream(d->stream));
  hipStream_t s = static_cast<hipStream_t>(d->stream);
  uint8_t *base = static_cast<uint8_t *>(d->workspace);
  HeadArgs &a = h.a;
  a.x_in = x;
  a.w_in = w;
  a.x = h.stage_x ? base + h.o_xs : x;
  a.w = h.stage_w ? base + h.o_ws : w;
  a.bias = bias;
  a.ids = ids;
  a.teacher = teacher;
  a.loss = loss;
  a.stats = reinterpret_cast<float2 *>(stats);
  a.picked = picked;
  a.part = reinterpret_cast<float2 *>(base + h.o_part);
  if (h.stage_w) HIP_TRY(launch_head_stage(h.bf16, w, a.w_in_ld, base + h.o_ws, a.w_ld, a.classes, a.dim, s));
  if (h.stage_x) HIP_TRY(launch_head_stage(h.bf16, x, a.x_in_ld, base + h.o_xs, a.x_ld, a.rows, a.dim, s));
  HIP_TRY(launch_head_forward(h.bf16, a, s));
  HIP_TRY(launch_head_finish(h.bf16, a, s));
  return HAPI_OK;
}

int head_backward(const hapi_head_desc *d, Head &h, const void *x, const void *w, const float *bias, const int64_t *ids,
                  const float *teacher, const float *stats, const float *picked, const float *dloss, void *dx, void *dw,
                  float *dbias) {
  if (d->rows > 0) {
    TRY(check_ptr(stats, 8, "stats"));
    TRY(check_ptr(dloss, 4, "dloss"));
    TRY(check_ptr(dx, h.esz, "dx"));
  }
  TRY(check_ptr(dw, h.esz, "dweight"));
  if (dbias) {
    if (!bias) return fail(HAPI_E_INVAL, "dbias without a bias");
    TRY(check_ptr(dbias, 4, "dbias"));
  }
  TRY(check_workspace(d->workspace, d->workspace_bytes, h.bytes_bwd));
  TRY(check_stream(d->stream));
  hipStream_t s = static_cast<hipStream_t>(d->stream);
  uint8_t *base = static_cast<uint8_t *>(d->workspace);
  HeadArgs &a = h.a;
  a.x_in = x;
  a.w_in = w;
  a.x = base + h.o_xs;
  a.x_ld = a.dx_pad;
  a.w = h.stage_w ? base + h.o_ws : w;
  a.bias = bias;
  a.ids = ids;
  a.teacher = teacher;
  a.stats = reinterpret_cast<float2 *>(const_cast<float *>(stats));
  a.picked = const_cast<float *>(picked);
  a.dloss = dloss;
  a.info = reinterpret_cast<float2 *>(base + h.o_info);
  a.unit = reinterpret_cast<float *>(base + h.o_unit);
  a.id32 = reinterpret_cast<int32_t *>(base + h.o_id);
  a.cq = reinterpret_cast<float *>(base + h.o_cq);
  a.gt = base + h.o_gt;
  a.db_part = dbias ? reinterpret_cast<float *>(base + h.o_db) : nullptr;
  a.dx_part = reinterpret_cast<float *>(base + h.o_dx);
  a.dw_part = reinterpret_cast<float *>(base + h.o_dw);
  a.dx = dx;
  a.dw = dw;
  a.dx_ld = a.x_in_ld;
  a.dw_ld = a.w_in_ld;
  a.dbias = dbias;
  if (h.stage_w) HIP_TRY(launch_head_stage(h.bf16, w, a.w_in_ld, base + h.o_ws, a.w_ld, a.classes, a.dim, s));
  HIP_TRY(launch_head_prepare(h.bf16, a, base + h.o_xs, a.x_ld, s));
  for (int64_t v0 = 0; v0 < a.classes; v0 += h.piece) {
    a.v0 = v0;
    a.piece = std::min(h.piece, a.classes - v0);
    a.first = v0 == 0;
    HIP_TRY(launch_head_dlogits(h.bf16, a, s));
    HIP_TRY(launch_head_grads(h.bf16, a, s));
  }
  HIP_TRY(launch_head_reduce(h.bf16, a, s));
  return HAPI_OK;
}

}  // namespace
}  // namespace hapi

using namespace hapi;

extern "C" {

int64_t hapi_layernorm_workspace_bytes(const hapi_norm_desc *desc) {
  Norm n;
  TRY(read_norm(desc, n));
  return norm_workspace(n);
}

int hapi_layernorm_forward(const hapi_norm_desc *desc, const void *x, const float *gamma, const float *beta, void *y,
                           float *mean, float *rstd) {
  Norm n;
  TRY(read_norm(desc, n));
  if (desc->rows == 0) return HAPI_OK;
  TRY(check_ptr(x, n.esz, "x"));
  TRY(check_ptr(gamma, 4, "gamma"));
  TRY(check_ptr(beta, 4, "beta"));
  TRY(check_ptr(y, n.esz, "y"));
  TRY(check_ptr(mean, 4, "mean"));
  TRY(check_ptr(rstd, 4, "rstd"));
  TRY(check_stream(desc->stream));
  n.a.x = x;
  n.a.gamma = gamma;
  n.a.beta = beta;
  n.a.y = y;
  n.a.mean = mean;
  n.a.rstd = rstd;
  HIP_TRY(launch_norm_forward(n.bf16, n.a, static_cast<hipStream_t>(desc->stream)));
  return HAPI_OK;
}

int hapi_layernorm_backward(const hapi_norm_desc *desc, const void *dy, const void *x, const float *gamma,
                            const float *mean, const float *rstd, void *dx, float *dgamma, float *dbeta) {
  Norm n;
  TRY(read_norm(desc, n));
  if (desc->rows > 0) {
    TRY(check_ptr(dy, n.esz, "dy"));
    TRY(check_ptr(x, n.esz, "x"));
    TRY(check_ptr(gamma, 4, "gamma"));
    TRY(check_ptr(mean, 4, "mean"));
    TRY(check_ptr(rstd, 4, "rstd"));
    TRY(check_ptr(dx, n.esz, "dx"));
  }
  TRY(check_ptr(dgamma, 4, "dgamma"));
  TRY(check_ptr(dbeta, 4, "dbeta"));
  TRY(check_workspace(desc->workspace, desc->workspace_bytes, norm_workspace(n)));
  TRY(check_stream(desc->stream));
  n.a.dy = dy;
  n.a.x = x;
  n.a.gamma = gamma;
  n.a.mean = const_cast<float *>(mean);
  n.a.rstd = const_cast<float *>(rstd);
  n.a.dx = dx;
  n.a.dgamma = dgamma;
  n.a.dbeta = dbeta;
  n.a.part = static_cast<float *>(desc->workspace);
  HIP_TRY(launch_norm_backward(n.bf16, n.a, static_cast<hipStream_t>(desc->stream)));
  return HAPI_OK;
}

int64_t hapi_head_workspace_bytes(const hapi_head_desc *desc, int32_t backward) {
  Head h;
  TRY(read_head(desc, h));
  return backward ? std::max(h.bytes_fwd, h.bytes_bwd) : h.bytes_fwd;
}

int hapi_xent_forward(const hapi_head_desc *desc, const void *x, const void *weight, const float *bias,
                      const int64_t *targets, float *loss, float *stats) {
  Head h;
  TRY(read_head(desc, h));
  if (desc->top != 0) return fail(HAPI_E_INVAL, "cross entropy needs top = 0");
  TRY(check_head_inputs(desc, h, x, weight, bias, targets, "targets"));
  return head_forward(desc, h, x, weight, bias, targets, nullptr, loss, stats, nullptr);
}

int hapi_xent_backward(const hapi_head_desc *desc, const void *x, const void *weight, const float *bias,
                       const int64_t *targets, const float *loss, const float *stats, const float *dloss, void *dx,
                       void *dweight, float *dbias) {
  Head h;
  TRY(read_head(desc, h));
  if (desc->top != 0) return fail(HAPI_E_INVAL, "cross entropy needs top = 0");
  TRY(check_head_inputs(desc, h, x, weight, bias, targets, "targets"));
  if (desc->rows > 0) TRY(check_ptr(loss, 4, "loss"));  // of the interface, not read
  return head_backward(desc, h, x, weight, bias, targets, nullptr, stats, nullptr, dloss, dx, dweight, dbias);
}

int hapi_distill_forward(const hapi_head_desc *desc, const void *x, const void *weight, const float *bias,
                         const int64_t *ids, const float *teacher, float *loss, float *stats, float *picked) {
  Head h;
  TRY(read_head(desc, h));
  if (desc->top < 1) return fail(HAPI_E_INVAL, "distillation needs top >= 1");
  TRY(check_head_inputs(desc, h, x, weight, bias, ids, "ids"));
  if (desc->rows > 0) {
    TRY(check_ptr(teacher, 4, "teacher"));
    TRY(check_ptr(picked, 4, "picked"));
  }
  return head_forward(desc, h, x, weight, bias, ids, teacher, loss, stats, picked);
}

int hapi_distill_backward(const hapi_head_desc *desc, const void *x, const void *weight, const float *bias,
                          const int64_t *ids, const float *teacher, const float *stats, const float *picked,
                          const float *dloss, void *dx, void *dweight, float *dbias) {
  Head h;
  TRY(read_head(desc, h));
  if (desc->top < 1) return fail(HAPI_E_INVAL, "distillation needs top >= 1");
  TRY(check_head_inputs(desc, h, x, weight, bias, ids, "ids"));
  if (desc->rows > 0) {
    TRY(check_ptr(teacher, 4, "teacher"));
    TRY(check_ptr(picked, 4, "picked"));
  }
  return head_backward(desc, h, x, weight, bias, ids, teacher, stats, picked, dloss, dx, dweight, dbias);
}

}  // extern "C"
