// Walks the tiles of keys that the cross attention's kernels go through: each tile's bits
// are its own keys and no others, and a tile without a missing key has all of them set,
// which is what lets it skip the masking.  Prints "OK <checks>".
#include <cstdio>
#include <cstdlib>

#include "attend.h"

static long g_checks = 0;
#define EXPECT(cond)                                                          \
  do {                                                                        \
    ++g_checks;                                                               \
    if (!(cond)) {                                                            \
      std::fprintf(stderr, "FAILED %s at line %d\n", #cond, __LINE__);        \
      std::exit(2);                                                           \
    }                                                                         \
  } while (0)

template <int BN>
static void walk() {
  for (int64_t keys = 0; keys < 1000; ++keys) {
    int64_t seen = 0;
    for (int64_t tile = -1; tile < keys / BN + 3; ++tile) {
      const int64_t left = keys - (tile < 0 ? keys + 5 : tile * BN);  // and past the last key
      const uint64_t bits = hapi::key_bits<BN>(left);
      EXPECT((bits & ~hapi::kAllKeys<BN>) == 0);
      EXPECT((bits == hapi::kAllKeys<BN>) == (left >= BN));
      for (int i = 0; i < BN; ++i) EXPECT((bits >> i & 1) == (i < left));
      if (tile >= 0) seen += __builtin_popcountll(bits);
    }
    EXPECT(seen == keys);
  }
  EXPECT(hapi::key_bits<BN>((int64_t)1 << 40) == hapi::kAllKeys<BN> && __builtin_popcountll(hapi::kAllKeys<BN>) == BN);
}

int main() {
  walk<32>();
  walk<64>();
  std::printf("OK %ld\n", g_checks);
  return 0;
}
