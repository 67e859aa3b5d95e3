#include "seen.hpp"

#include <algorithm>

namespace cs {

bool tree_ok(const int32_t* parents, int32_t n) {
  for (int32_t i = 0; i < n; ++i)
    if (parents[i] < -1 || parents[i] >= i) return false;
  return true;
}

int32_t tree_words(const int32_t* parents, int32_t n, int64_t prefix, std::vector<uint32_t>& out) {
  const int64_t w0 = prefix / 32;
  const int32_t words = static_cast<int32_t>((prefix + n - 1) / 32 - w0 + 1);
  const size_t base = out.size();
  out.resize(base + static_cast<size_t>(n) * words);
  const int bit0 = static_cast<int>(prefix % 32);
  for (int32_t i = 0; i < n; ++i) {
    uint32_t* row = out.data() + base + static_cast<size_t>(i) * words;
    if (parents[i] < 0) {
      std::fill(row, row + words, 0u);
      row[0] = (1u << bit0) - 1u;   // the cached tokens of the first word
    } else {
      std::copy_n(out.data() + base + static_cast<size_t>(parents[i]) * words, words, row);
    }
    const int at = bit0 + i;
    row[at / 32] |= 1u << (at % 32);
  }
  return words;
}

void tree_depths(const int32_t* parents, int32_t n, int32_t* out) {
  for (int32_t i = 0; i < n; ++i) out[i] = parents[i] < 0 ? 0 : out[parents[i]] + 1;
}

}  // namespace cs
