// Prints how a paged attention call's work is cut: units of 256 rows, parts of the slots, slots of
// a part, and the new tokens up to which a sequence is scanned.
// Arguments: batch n_new query_heads kv_heads max_new max_tokens scan_rows.
#include <cstdio>
#include <cstdlib>

#include "splits.hpp"

int main(int argc, char** argv) {
  if (argc != 8) return 2;
  const spectra::PagedPlan p = spectra::paged_plan(std::atoi(argv[1]), std::atoll(argv[2]), std::atoi(argv[3]), std::atoi(argv[4]),
                                                   std::atoi(argv[5]), std::atoll(argv[6]), std::atoi(argv[7]));
  std::printf("%lld %d %lld %d\n", (long long)p.units, p.split.parts, (long long)p.split.slots, p.scan_tokens);
  return 0;
}
