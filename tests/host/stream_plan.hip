// The index arithmetic of streamed attention (csrc/stream.h) on the host, every case against
// its definition: which key tiles rows have, which keys are read for them, which workgroup
// has which piece.  Test infrastructure only.
#include <cstdio>
#include <cstdlib>
#include <set>
#include <string>
#include <vector>

#include "../../paper_2607_06631_amd/csrc/stream.h"

using namespace dif;

static long g_cases = 0;
#define NEED(c, ...)                    \
  do {                                  \
    if (!(c)) {                         \
      std::printf(__VA_ARGS__);         \
      std::printf(": %s\n", #c);        \
      std::exit(1);                     \
    }                                   \
  } while (0)

template <int BN>
static void tiles(const SeenMask& m, int p0, int p1, int keys) {
  ++g_cases;
  std::vector<int> rows_of(keys, 0);   // rows that see a key
  for (int p = p0; p <= p1; ++p) {
    if (m.block > 0 && p < 0) continue;
    const int64_t e = m.block > 0 ? ((int64_t)(p / m.block) + 1) * m.block : keys;
    for (int j = 0; j < keys && j < e; ++j)
      if (m.window == 0 || j >= e - m.window || j < m.sinks) ++rows_of[j];
  }
  const Extent<BN, true> ex = extent<BN, true>(m, p0, p1, keys);
#define WHO "block %d window %d sinks %d rows %d .. %d of %d keys, tile %d key %d -> %d", m.block, m.window, m.sinks, p0, p1, keys
  std::set<int> have;
  for (int t = 0; t < ex.ntiles; ++t) {
    const int i = ex.tile(t);
    NEED(have.insert(i).second, WHO, i, 0, 0);
    int some = 0;
    for (int k = i * BN; k < (i + 1) * BN; ++k) some += k < keys && rows_of[k] > 0;
    NEED(!ex.whole(i) || some == BN, WHO, i, some, 0);
    // (tiles that the kernels take without masks are copied as whole ones)
    const Seen a = seen_by(m, p0, keys), b = seen_by(m, p1, keys);
    NEED(ex.whole(i) || !((i + 1) * BN <= a.end && (i * BN >= b.start || (i + 1) * BN <= ex.sinks)), WHO, i, some, 0);
    for (int k = i * BN; k < (i + 1) * BN; ++k) {
      NEED(ex.sees(k) == (k < keys && rows_of[k] > 0), WHO, i, k, 0);
      const int n = ex.nearest(i, k);
      NEED(n / BN == i && n < keys && (!ex.sees(k) || n == k), WHO, i, k, n);
    }
    if (some == 0) NEED(ex.before(i) >= 0 && rows_of[ex.before(i)] > 0, WHO, i, 0, ex.before(i));
  }
  // without gaps: each key read in place of one that no row sees is seen
  if (!(m.window > 0 && m.window < m.block)) {
    const Extent<BN, false> plain = extent<BN, false>(m, p0, p1, keys);
    NEED(plain.ntiles == ex.ntiles, WHO, 0, 0, 0);
    for (int t = 0; t < ex.ntiles; ++t)
      for (int i = ex.tile(t), k = i * BN; k < (i + 1) * BN; ++k)
        NEED(rows_of[plain.nearest(i, k)] > 0 && plain.whole(i) == ex.whole(i) && plain.sees(k) == ex.sees(k), WHO, i, k, 0);
  }
  for (int j = 0; j < keys; ++j) NEED(rows_of[j] == 0 || have.count(j / BN), WHO, j / BN, j, 0);
}

static void all_tiles() {
  const int some[] = {0, 1, 2, 3, 5, 7, 16, 20, 31, 32, 33, 50, 64, 65, 100, 130, 200, 300};
  for (int block : some)
    for (int window : some)
      for (int sinks : {0, 1, 5, 32, 40, 70, 200}) {
        if (sinks && !window) continue;
        const SeenMask m{block, window, sinks};
        for (int keys : {0, 1, 15, 32, 33, 64, 90, 128, 197, 290})
          for (int p0 : {-70, -3, 0, 1, 15, 30, 63, 64, 100, 150, 289})
            for (int n : {1, 2, 6, 16, 40, 128, 256}) {
              if (p0 >= keys) continue;
              tiles<32>(m, p0, std::min(p0 + n, keys) - 1 < p0 ? p0 : std::min(p0 + n, keys) - 1, keys);
              tiles<64>(m, p0, std::min(p0 + n, keys) - 1 < p0 ? p0 : std::min(p0 + n, keys) - 1, keys);
            }
      }
}

// Every piece of every head has one workgroup of the launch, whose size is that of the most there may be.
static void all_turns() {
  for (int heads : {1, 2, 3, 5, 7, 8, 12, 13, 16, 40, 41, 64, 100, 128})
    for (int pieces = 1; pieces < 9000; pieces += pieces < 140 ? 1 : pieces < 1000 ? 17 : 501)
      for (int64_t spare : {0, 1, 1000}) {
        ++g_cases;
        const int64_t grid = turns((int64_t)pieces * heads + spare, heads);
        std::vector<char> seen((size_t)pieces * heads, 0);
        for (int64_t b = 0; b < grid; ++b) {
          int i, h;
          if (!turn_of((int)b, pieces, heads, &i, &h)) continue;
          NEED(i >= 0 && i < pieces && h >= 0 && h < heads, "pieces %d heads %d workgroup %lld", pieces, heads, (long long)b);
          NEED(!seen[(size_t)h * pieces + i]++, "pieces %d heads %d workgroup %lld twice", pieces, heads, (long long)b);
        }
        for (char c : seen) NEED(c == 1, "pieces %d heads %d of %lld", pieces, heads, (long long)grid);
      }
}

int main(int argc, char** argv) {
  const std::string what = argc > 1 ? argv[1] : "";
  if (what == "tiles") all_tiles();
  else if (what == "turns") all_turns();
  else return 2;
  std::printf("%ld cases passed\n", g_cases);
  return 0;
}
