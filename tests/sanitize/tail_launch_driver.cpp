// Walks layer norm's grids, and the launches that the forward product of the trained
// tail's classifier is made of, from one row and class to the largest sizes: these
// cover the classes once, and their parts lie within the partial statistics to the last
// one, with no more room than there is; all are launches that the device takes.  Host
// code only.  Prints "OK <launches>".
#include <cstdio>
#include <cstdlib>
#include <initializer_list>

#include "tail.h"

// The launchers, which nothing here calls.
namespace hapi {
int fail(int code, const char *, ...) { return code; }
#define NONE \
  { return hipErrorNotSupported; }
hipError_t launch_norm_forward(bool, const NormArgs &, hipStream_t) NONE
hipError_t launch_norm_backward(bool, const NormArgs &, hipStream_t) NONE
hipError_t launch_head_stage(bool, const void *, int64_t, void *, int64_t, int64_t, int, hipStream_t) NONE
hipError_t launch_head_forward(bool, const HeadArgs &, hipStream_t) NONE
hipError_t launch_head_finish(bool, const HeadArgs &, hipStream_t) NONE
hipError_t launch_head_prepare(bool, const HeadArgs &, void *, int64_t, hipStream_t) NONE
hipError_t launch_head_dlogits(bool, const HeadArgs &, hipStream_t) NONE
hipError_t launch_head_grads(bool, const HeadArgs &, hipStream_t) NONE
hipError_t launch_head_reduce(bool, const HeadArgs &, hipStream_t) NONE
}  // namespace hapi

using namespace hapi;

static long g_launches = 0;
static int64_t g_rows, g_classes;
#define EXPECT(cond)                                                                              \
  do {                                                                                            \
    if (!(cond)) {                                                                                \
      std::fprintf(stderr, "FAILED %s at line %d, %lld rows, %lld classes\n", #cond, __LINE__,    \
                   (long long)g_rows, (long long)g_classes);                                      \
      std::exit(2);                                                                               \
    }                                                                                             \
  } while (0)

// What the kernels of each variant take: classes and rows of a tile, classes of a part.
struct Tile {
  int64_t classes, rows, part, threads;
};
static Tile tile(Variant v) {
  switch (v) {
    case BIG: return {256, 256, 64, 512};
    case MID: return {128, 128, 64, 256};
    case SMALL: return {64, 64, 32, 256};
    case FEW: return {128, 32, 32, 256};
    default: return {32, 32, 32, 256};
  }
}

static void walk(bool bf16, int64_t rows, int64_t classes) {
  g_rows = rows;
  g_classes = classes;
  const int parts = head_parts(bf16, rows, classes);
  int64_t c0 = 0, next_part = 0;
  while (c0 < classes) {
    const HeadLaunch l = head_forward_launch(bf16, rows, classes, c0);
    const Tile t = tile(l.v);
    EXPECT(l.classes > 0 && c0 + l.classes <= classes);
    const bool last = c0 + l.classes == classes;
    // a launch's threads are a 32-bit number
    EXPECT(ceil_div(l.classes, t.classes) * ceil_div(rows, t.rows) * t.threads <= (int64_t)UINT32_MAX);
    EXPECT(last || l.classes % t.classes == 0);  // whole tiles, so whole parts
    EXPECT(l.part == next_part && l.parts == parts - l.part && l.parts > 0);
    // parts that the launch's tiles have classes for: all of what is left by the last one
    const int64_t holds = ceil_div(l.classes, t.part);
    EXPECT(holds <= l.parts && (!last || l.parts - holds < t.classes / t.part));
    next_part += holds;
    c0 += l.classes;
    ++g_launches;
  }
}

int main() {
  for (bool bf16 : {false, true}) {
    for (int64_t rows : {1, 2, 31, 32, 33, 64, 65, 128, 129, 255, 256, 257, 600, 700, 1000, 1300, 4096, 8192, 65537, 131072,
                         1 << 20})
      for (int64_t classes : {1, 31, 32, 33, 100, 129, 257, 1000, 5003, 10007, 22100, 32000, 33000, 50021, 131072, 524288,
                              2100001, 4194309, 1 << 24})
        walk(bf16, rows, classes);
    for (int64_t rows = 1; rows < 3000; rows += 37)
      for (int64_t classes = 1; classes < 200000; classes += 1 + classes / 9) walk(bf16, rows, classes);
  }
  // Layer norm's forward grid: threads a launch takes, and no block without rows.
  g_classes = 0;
  for (int threads : {256, 512})
    for (int64_t want : {(int64_t)1, (int64_t)2, (int64_t)1535, (int64_t)6145, (int64_t)1 << 26, ((int64_t)1 << 26) + 5,
                         (int64_t)1 << 40, (int64_t)1 << 60}) {
      g_rows = want;
      const int64_t blocks = norm_forward_blocks(want, threads);
      EXPECT(blocks >= 1 && blocks <= want && blocks * threads <= (int64_t)UINT32_MAX);
      ++g_launches;
    }
  std::printf("OK %ld\n", g_launches);
  return 0;
}
