#include "seen.hpp"

#include <algorithm>

namespace cs {

int32_t rows_split(const std::vector<int64_t>& lens, int32_t n_kv_heads, int32_t n_cus) {
  int64_t keys = 0, longest = 0;
  for (const int64_t n : lens) {
    keys += n;
    longest = std::max(longest, n);
  }
  if (longest <= 64 * kDecodeSubSplits) return 64;
  const int64_t share = keys * n_kv_heads / n_cus;   // of a CU
  for (const int64_t most : {2 * n_cus, 3 * n_cus, 4 * n_cus}) {   // twice the workgroups
    for (int32_t split = 32; split <= 1024; split += 32) {
      const int64_t item = static_cast<int64_t>(kDecodeSubSplits) * split;
      if (item > std::max<int64_t>(2 * share, 1024)) break;
      int64_t items = 0;
      for (const int64_t n : lens) items += (n + item - 1) / item;
      if (2 * items * n_kv_heads <= most) return split;
    }
  }
  return 1024;
}

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
