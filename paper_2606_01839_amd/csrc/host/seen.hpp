// Host plans of the attention whose rows are not a conversation's last tokens in causal order: trees of
// drafted tokens, and rows that see every token (an encoder's states). No HIP here.
#pragma once

#include <cstdint>
#include <vector>

#include "host_state.hpp"

namespace cs {

// What the rows of a batch entry see: every key before `clear`, and of the others those whose bits are set in the
// row's words (none: `words` = 0, and clear = the conversation's length). Word w of a row stands for keys 32 (clear / 32
// + w) .. + 31, bit b for key 32 (clear / 32 + w) + b: aligned to absolute keys, as the kernels meet them.
struct SeenMask {
  int32_t clear;
  int32_t off;      // first word of the entry's rows, [q_len][words]
  int32_t words;    // a row
  int32_t rec;      // first record of the entry's work items (rows kernel)
};

// A work item of the rows kernel: keys [k0, k0 + kDecodeSubSplits x split) of a batch entry.
struct SeenItem {
  int32_t conv;
  int32_t k0;
};

// Keys per wave of the rows kernel for a batch of conversations: the smallest multiple of 32 whose items (workgroups of
// kDecodeSubSplits waves, one a CU, over all kv heads) fit one round of the CUs, or one and a half, or two, with items of at most twice a
// CU's share of the keys; where there is none, 1024. In a batch whose longest conversation has at most 512 tokens each is one item (a pool that
// holds no longer ones has no records). Items that just fill a round are the best that there is: 16 trees of 8
// on 1k-9k tokens (32 query and 8 kv heads of 128) take 38.4 us with 232 items, 46-49 with 304-560, 44-80 with 184-128; one of 12
// on 100k 72.1 with 248, 85-120 with 320-3128. Beyond two rounds fewer items, with fewer records, are better: 64 on
// 8k-32k 727 us with 1248, 744 with 1500; 200 on 300-5000 243 with 1600, 283 with 2248.
int32_t rows_split(const std::vector<int64_t>& lens, int32_t n_kv_heads, int32_t n_cus);

// Tokens a tree may have (what bounds it: n^2 / 8 bytes of words).
constexpr int kMaxDraft = 1024;

// Whether parents[0 .. n) is a tree's: each -1 or an earlier token.
bool tree_ok(const int32_t* parents, int32_t n);

// Words of the rows of a tree of n tokens behind `prefix` cached ones, appended to `out`; returns the words a row. A
// token sees what its parent sees, and itself.
int32_t tree_words(const int32_t* parents, int32_t n, int64_t prefix, std::vector<uint32_t>& out);

// Depth of each token (0: its parent is -1).
void tree_depths(const int32_t* parents, int32_t n, int32_t* out);

}  // namespace cs
