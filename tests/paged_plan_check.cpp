// Host check of the paged attention's work plan: parts cover the longest sequence, counts fit
// the grids, and a workspace taken for the largest call serves every smaller one.
#include <cmath>
#include <cstdio>

#include "splits.hpp"

using namespace spectra;

#define CHECK(c)                                                                                                   \
  do {                                                                                                             \
    if (!(c)) {                                                                                                    \
      std::printf("%s:%d: %s (batch %d n_new %lld heads %d/%d max_new %d max_tokens %lld)\n", __FILE__, __LINE__,  \
                  #c, batch, (long long)n_new, q, kv, max_new, (long long)max_tokens);                             \
      return 1;                                                                                                    \
    }                                                                                                              \
  } while (0)

static uint64_t state = 88172645463325252ull;
static int64_t pick(int64_t lo, int64_t hi) {  // spread over the logarithm
  state ^= state << 13, state ^= state >> 7, state ^= state << 17;
  const double u = (double)(state >> 11) / 9007199254740992.0;
  const int64_t v = (int64_t)std::exp(std::log((double)lo) + u * std::log((double)(hi + 1) / (double)lo));
  return v < lo ? lo : v > hi ? hi : v;
}

int main() {
  for (int it = 0; it < 200000; ++it) {
    const int kv = (int)pick(1, 64), n_qh = (int)pick(1, 16), q = kv * n_qh;
    const int batch = (int)pick(1, 2000), max_new = (int)pick(1, 20000);
    const int64_t n_new = pick(1, (int64_t)batch * max_new < 1000000 ? (int64_t)batch * max_new : 1000000);
    const int64_t max_tokens = pick(1, 2000000);
    const int rows = pick(1, 2) == 1 ? 12 : 16;
    const PagedPlan p = paged_plan(batch, n_new, q, kv, max_new, max_tokens, rows);
    CHECK(p.split.parts >= 1 && p.split.parts <= 64 && p.split.slots * p.split.parts >= max_tokens);
    CHECK(p.split.slots * (p.split.parts - 1) < max_tokens);
    CHECK(p.units == 0 || p.split.slots % PAGED_STEP == 0);
    CHECK(p.scan_tokens * n_qh <= rows && (p.units > 0) == (max_new > p.scan_tokens));
    CHECK(p.scan_tokens > 0 || n_new >= (int64_t)batch * max_new || rows / n_qh == 0);
    CHECK(p.scan_at <= p.part_at && p.part_at <= p.bytes);
    // units of every sequence: the worst cut of n_new tokens into `batch` sequences
    const int64_t all = n_new < (int64_t)batch * max_new ? n_new : (int64_t)batch * max_new;
    CHECK(p.units == 0 || p.units * PAGED_ROWS >= all * n_qh);
    const size_t room = paged_workspace_bytes(batch, n_new, q, kv, max_new, max_tokens);
    CHECK(room >= p.bytes);
    const int64_t tiles = ceil_div(max_tokens, 64), groups = (int64_t)batch * kv;
    for (int per_cu = 1; per_cu <= 3; ++per_cu) {
      const Split s = paged_scan_split(groups, tiles, per_cu);
      CHECK(s.n_chunks <= paged_scan_chunks(groups, tiles) && (int64_t)s.n_chunks * s.tiles_per_chunk >= tiles);
      CHECK(s.tiles_per_chunk % SCAN_WAVES == 0);
    }
    // any smaller call
    const int b2 = (int)pick(1, batch), m2 = (int)pick(1, max_new);
    const int64_t t2 = pick(1, max_tokens), n2 = pick(1, n_new);
    CHECK(paged_plan(b2, n2, q, kv, m2, t2, rows).bytes <= room);
    CHECK(paged_workspace_bytes(b2, n2, q, kv, m2, t2) <= room);
  }
  std::printf("OK\n");
  return 0;
}
