// Host check of what a paged attention call's plan has to hold for any sequences that keep its bounds:
// a unit of 256 rows for every started one of every sequence that is not scanned, and for the scan's
// chunks, whatever the workgroups of a CU, the items of the launch and the room of the workspace.
#include <cmath>
#include <cstdio>
#include <vector>

#include "splits.hpp"

using namespace spectra;

static uint64_t state = 0x9E3779B97F4A7C15ull;
static int64_t pick(int64_t lo, int64_t hi) {  // spread over the logarithm
  state ^= state << 13, state ^= state >> 7, state ^= state << 17;
  const double u = (double)(state >> 11) / 9007199254740992.0;
  const int64_t v = (int64_t)std::exp(std::log((double)lo) + u * std::log((double)(hi + 1) / (double)lo));
  return v < lo ? lo : v > hi ? hi : v;
}

int main() {
  for (int it = 0; it < 60000; ++it) {
    const int kv = (int)pick(1, 64), n_qh = (int)pick(1, 16), q = kv * n_qh, rows = pick(1, 2) == 1 ? 12 : 16;
    const int batch = (int)pick(1, 300);
    const int64_t max_tokens = pick(1, 1000000);
    std::vector<int64_t> n(batch);
    int64_t sum = 0, most = 0;
    const int kind = (int)pick(1, 4);
    const int64_t top = pick(1, 3000);
    for (auto& x : n) {
      if (kind == 1) x = pick(1, top);                       // ragged
      if (kind == 2) x = pick(1, 2) == 1 ? 0 : pick(1, top);  // some without tokens
      if (kind == 3) x = pick(1, 4) * PAGED_ROWS / n_qh + 1;  // a row or more past whole units
      if (kind == 4) x = rows / n_qh + 1;                     // just past the scan's
      sum += x;
      most = x > most ? x : most;
    }
    if (sum == 0) continue;
    const int max_new = (int)(most + (pick(1, 3) == 1 ? pick(1, 50) : 0));
    const int64_t n_new = sum + (pick(1, 3) == 1 ? pick(1, 1000) : 0);  // rows behind the last sequence
    const PagedPlan p = paged_plan(batch, n_new, q, kv, max_new, max_tokens, rows);
    int64_t units = 0;
    for (int64_t x : n)
      if (x > p.scan_tokens) units += ceil_div(x * n_qh, PAGED_ROWS);
    if (units > p.units) {
      std::printf("units %lld > %lld (batch %d n_new %lld heads %d/%d max_new %d)\n", (long long)units, (long long)p.units, batch,
                  (long long)n_new, q, kv, max_new);
      return 1;
    }
    // the scan's chunks, their length found from the sequences' tiles as on the device
    for (int per_cu = 1; per_cu <= PAGED_SCAN_PER_CU; ++per_cu) {
      const int64_t items = paged_scan_items(kv, per_cu);
      int64_t total = 0, chunks = 0;
      std::vector<int64_t> each(batch);
      for (auto& e : each) total += e = ceil_div(pick(1, max_tokens), 64);
      const int64_t whole = items - (batch < items ? batch : items) / 2;
      int64_t tpc = ceil_div(ceil_div(total, whole), SCAN_WAVES) * SCAN_WAVES;
      if (tpc < PAGED_SCAN_LEAST) tpc = PAGED_SCAN_LEAST;
      for (int64_t e : each) chunks += ceil_div(e, tpc);
      if (chunks > items + batch || chunks * kv > paged_scan_chunks(batch, kv, ceil_div(max_tokens, 64))) {
        std::printf("chunks %lld (batch %d kv %d per_cu %d max_tokens %lld)\n", (long long)chunks, batch, kv, per_cu, (long long)max_tokens);
        return 1;
      }
    }
  }
  std::printf("OK\n");
  return 0;
}
