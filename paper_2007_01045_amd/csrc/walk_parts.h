// How walks of dk and dv are cut into parts (docs_plan in attention_window.h): the numbers alone, for the device and for a test on the host.
#pragma once

namespace dapple {

// The blocks of a part: one of `units` shares of the walks of all heads (`all` blocks a head), `least` at least.  Tens of millions of rows
// that see each other have shares beyond an int; a walk has fewer than 2^23 blocks (query heads times blocks of 32 rows), so 2^30
// cuts none, either.
constexpr int walk_share(unsigned long long all, int heads, int units, int least) {
  const unsigned long long share = (all * heads + units - 1) / units, most = 1ULL << 30;
  return share < (unsigned long long)least ? least : (int)(share < most ? share : most);
}
constexpr int walk_parts(int n, int share) { return n > share ? (n + share - 1) / share : 1; }

}  // namespace dapple
