// Host check of the block selection's work plan: launches cover the tokens, scores and the heads' best lie where the
// workspace has room for them, chunks cover the blocks, and no selection asks for more than the scores' room.
#include <cmath>
#include <cstdio>

#include "splits.hpp"

using namespace spectra;

#define CHECK(c)                                                                                                   \
  do {                                                                                                             \
    if (!(c)) {                                                                                                    \
      std::printf("%s:%d: %s (batch %d n_new %lld heads %d x %d max_tokens %lld from %lld)\n", __FILE__, __LINE__,  \
                  #c, batch, (long long)n_new, kv, n_qh, (long long)max_tokens, (long long)from);                  \
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
  for (int it = 0; it < 100000; ++it) {
    const int kv = (int)pick(1, 2000), n_qh = (int)pick(1, 16), batch = (int)pick(1, 16384);
    const int64_t n_new = pick(1, ((int64_t)1 << 21) / (kv * n_qh)), max_tokens = pick(1, (int64_t)1 << 30);
    int64_t from = 0;
    const SelectPlan p = select_plan(n_new, kv * n_qh, kv, max_tokens);
    CHECK(p.pitch % SELECT_STEP == 0 && p.pitch * 64 >= max_tokens && p.scores_at % 64 == 0);
    CHECK(p.many == (n_new * kv > SELECT_FEW_PAIRS) && p.tokens >= 1);
    const int64_t least = (int64_t)kv * n_qh * p.pitch;
    CHECK(p.floats - p.scores_at <= (least > SELECT_SCORES ? least : SELECT_SCORES));
    int pitch_log2 = 0;
    while (1 << pitch_log2 < n_qh) ++pitch_log2;
    for (int slabs = 0; from < n_new && slabs < 20; ++slabs) {
      const int64_t tokens = p.tokens < n_new - from ? p.tokens : n_new - from;
      const SelectSlab s = select_slab(p, tokens, batch, kv, pitch_log2);
      const int tg = s.columns >> pitch_log2;
      CHECK(tg >= 1 && s.chunks >= 1 && s.chunks <= SELECT_MOST_CHUNKS && s.steps * s.chunks * SELECT_STEP >= p.pitch);
      CHECK(s.steps * (s.chunks - 1) * SELECT_STEP < p.pitch && (!s.both || s.chunks == 1));
      CHECK(tokens * kv * n_qh * s.chunks <= p.scores_at);
      CHECK(tokens * (p.many ? kv : kv * n_qh) * p.pitch <= p.floats - p.scores_at);
      // units of sequences cut out of the launch's tokens one after the other, their last among them
      int64_t first = 0, last = -1;
      for (int b = 0; b < (batch < 40 ? batch : 40) && first < tokens; ++b) {
        const int64_t n = pick(1, tokens - first), base = first / tg + b;
        CHECK(base > last);
        last = base + ceil_div(n, tg) - 1;
        first += n;
      }
      CHECK(last < s.units);
      from += tokens;
    }
    from = -1;
    const int64_t n2 = pick(1, n_new), t2 = pick(1, max_tokens);
    CHECK(select_plan(n2, kv * n_qh, kv, t2).floats <= p.floats);
  }
  std::printf("OK\n");
  return 0;
}
