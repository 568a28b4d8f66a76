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
    CHECK(p.plan_at <= p.scan_at && p.scan_at <= p.part_at && p.part_at <= p.bytes);
    // units of every sequence: the worst cut of n_new tokens into `batch` sequences
    const int64_t all = n_new < (int64_t)batch * max_new ? n_new : (int64_t)batch * max_new;
    CHECK(p.units == 0 || p.units * PAGED_ROWS >= all * n_qh);
    const size_t room = paged_workspace_bytes(batch, n_new, q, kv, max_new, max_tokens);
    CHECK(room >= p.bytes);
    // the scan's chunks, their length found from the sequences' tiles as on the device
    for (int per_cu = 1; per_cu <= 3; ++per_cu) {
      const int64_t items = paged_scan_items(kv, per_cu);
      int64_t total = 0, chunks = 0, each[40];
      const int nb = batch < 40 ? batch : 40;
      for (int i = 0; i < nb; ++i) total += each[i] = ceil_div(pick(1, max_tokens), 64);
      const int64_t whole = items - (nb < items ? nb : items) / 2;
      int64_t tpc = ceil_div(ceil_div(total, whole), SCAN_WAVES) * SCAN_WAVES;
      if (tpc < PAGED_SCAN_LEAST) tpc = PAGED_SCAN_LEAST;
      for (int i = 0; i < nb; ++i) chunks += ceil_div(each[i], tpc);
      CHECK(chunks <= items + nb && chunks * kv <= paged_scan_chunks(nb, kv, ceil_div(max_tokens, 64)));
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
