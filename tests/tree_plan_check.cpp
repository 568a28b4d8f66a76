// Host check of the drafted trees' work plan: every unit has its workgroups, the workspace lies as it is sized, serves every
// smaller call of as many heads, and holds little more than the largest plan of its counts.
#include <cmath>
#include <cstdio>
#include <initializer_list>

#include "splits.hpp"

using namespace spectra;

#define CHECK(c)                                                                                                   \
  do {                                                                                                             \
    if (!(c)) {                                                                                                    \
      std::printf("%s:%d: %s (batch %d n_new %lld heads %d x %d max_new %d max_tokens %lld)\n", __FILE__, __LINE__, \
                  #c, batch, (long long)n_new, kv, n_qh, max_new, (long long)max_tokens);                          \
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
    const int kv = (int)pick(1, 1200), n_qh = (int)pick(1, 16), batch = (int)pick(1, 16384), max_new = (int)pick(1, 64);
    const int64_t n_new = pick(1, (int64_t)batch * max_new + 5), max_tokens = pick(1, 2000000);
    const size_t room = tree_workspace_bytes(batch, n_new, n_qh, kv, max_new, max_tokens);
    for (const bool f32 : {false, true}) {
      const TreePlan p = tree_plan(batch, n_new, n_qh, kv, max_new, max_tokens, f32);
      CHECK(p.bytes <= room);
      CHECK(p.plan_at <= p.rows_at && p.rows_at <= p.part_at && p.part_at <= p.bytes);
      CHECK((p.units > 0) == (max_new > p.scan_tokens) && (!f32 || p.scan_tokens == max_new));
      CHECK(p.scan_tokens > 0 || n_new >= (int64_t)batch * max_new);
      if (p.scan_tokens == 0) continue;
      const int64_t rows = 16 * p.nb;
      // sequences cut out of the new tokens one after the other: units, their places in the plan, and their chunks
      const int nb = batch < 50 ? batch : 50;
      int64_t first = 0, units = 0, work = 0, last = -1, n_units[50], tiles[50];
      for (int b = 0; b < nb; ++b) {
        const int64_t most = n_new - first < p.scan_tokens ? n_new - first : p.scan_tokens, n = most > 0 ? pick(1, most) : 0;
        n_units[b] = ceil_div(n * n_qh, rows);
        tiles[b] = ceil_div(pick(1, max_tokens), 64);
        if (n_units[b] > 0) {
          CHECK(first * n_qh / rows + b > last);
          last = first * n_qh / rows + b + n_units[b] - 1;
        }
        units += n_units[b];
        work += n_units[b] * tiles[b];
        first += n;
      }
      CHECK(last < tree_units(batch, n_new, n_qh, (int)rows));
      const int64_t whole = p.want - (units < p.want ? units : p.want) / 2;
      int64_t each = ceil_div(ceil_div(work, whole), 4) * 4, chunks = 0;
      if (each < 4) each = 4;
      for (int b = 0; b < nb; ++b) chunks += n_units[b] * ceil_div(tiles[b], each);
      CHECK(chunks <= p.items);
      CHECK((size_t)p.items * kv * rows * SCAN_PART_BYTES <= p.part_at - p.rows_at);
    }
    // any smaller call
    const int b2 = (int)pick(1, batch), m2 = (int)pick(1, max_new);
    const int64_t t2 = pick(1, max_tokens), n2 = pick(1, n_new);
    CHECK(tree_workspace_bytes(b2, n2, n_qh, kv, m2, t2) <= room);
    for (const bool f32 : {false, true}) CHECK(tree_plan(b2, n2, n_qh, kv, m2, t2, f32).bytes <= room);
    // and no more than twice the largest plan of these counts (that of one new token less included), and the parts
    size_t most = 0;
    for (const bool f32 : {false, true})
      for (const int64_t n : {n_new, n_new < (int64_t)batch * max_new ? n_new : (int64_t)batch * max_new - 1}) {
        const size_t bytes = n > 0 ? tree_plan(batch, n, n_qh, kv, max_new, max_tokens, f32).bytes : 0;
        most = bytes > most ? bytes : most;
      }
    const size_t parts = (int64_t)max_new * n_qh > TREE_FEW_ROWS ? 2 * N_CU * PAGED_PART_BYTES : 0;
    CHECK(room <= 2 * most + parts + 4096);
  }
  std::printf("OK\n");
  return 0;
}
