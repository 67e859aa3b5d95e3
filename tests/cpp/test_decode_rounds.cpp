// plan_decode_rounds: the plan of plan_decode_filling, or longer items that fit one or two rounds of the CUs.
#include <cstdio>
#include <cstdlib>
#include <vector>

#include "host/host_state.hpp"

#define CHECK(x)                                                                  \
  do {                                                                            \
    if (!(x)) {                                                                   \
      std::printf("%s:%d: failed: %s\n", __FILE__, __LINE__, #x);                 \
      std::exit(1);                                                               \
    }                                                                             \
  } while (0)

static int64_t workgroups(const std::vector<int64_t>& lens, int hkv, int split) {
  int64_t n = 0;
  for (int64_t L : lens) n += (L + 8 * split - 1) / (8 * split);
  return n * hkv;
}

int main() {
  std::srand(77);
  int one = 0, two = 0;
  for (int trial = 0; trial < 600; ++trial) {
    const int n = 1 + std::rand() % (std::rand() % 3 ? 8 : 70), hkv = 1 << (std::rand() % 4);
    const int top = std::rand() % 4 ? 9000 : 120000;
    std::vector<int32_t> slots(n);
    std::vector<int64_t> lens(n);
    for (int i = 0; i < n; ++i) {
      slots[i] = i;
      lens[i] = 1 + std::rand() % (std::rand() % 8 ? top : 900);
    }
    const cs::DecodePlan base = cs::plan_decode_filling(slots, lens, hkv, 4096, 256);
    const cs::DecodePlan p = cs::plan_decode_rounds(slots, lens, hkv, 4096, 256);
    int64_t total = 0;
    std::vector<char> seen(p.order.size(), 0);
    for (int i = 0; i < n; ++i) {
      CHECK(p.convs[i].slot == i && p.convs[i].len == lens[i] && p.convs[i].item_start == total);
      CHECK(static_cast<int64_t>(p.convs[i].n_splits - 1) * 8 * p.split_tokens < lens[i]);
      CHECK(static_cast<int64_t>(p.convs[i].n_splits) * 8 * p.split_tokens >= lens[i]);
      CHECK(lens[i] > 1024 || p.convs[i].n_splits == 1 || base.split_tokens < 128);
      total += p.convs[i].n_splits;
    }
    CHECK(p.n_items == total && p.order.size() == static_cast<size_t>(total) && p.single_item == (total == n));
    for (int32_t it : p.order) {
      CHECK(it >= 0 && it < total && !seen[it]);
      seen[it] = 1;
    }
    // a wave takes at most 1024 keys, a record's room is never exceeded
    CHECK(p.split_tokens % 32 == 0 && p.split_tokens <= 1024 && p.n_items <= base.n_items);
    const int64_t wg = workgroups(lens, hkv, base.split_tokens);
    if (wg <= 256) {
      CHECK(p.split_tokens == base.split_tokens);
      continue;
    }
    const bool fits1 = base.split_tokens < 512 && workgroups(lens, hkv, 512) <= 256;
    const bool fits2 = base.split_tokens < 384 && workgroups(lens, hkv, 384) <= 512;
    if (!fits1 && !fits2) {
      CHECK(p.split_tokens == base.split_tokens);
      continue;
    }
    const int64_t room = fits1 ? 256 : 512;
    ++(fits1 ? one : two);
    CHECK(p.split_tokens > base.split_tokens && workgroups(lens, hkv, p.split_tokens) <= room);
    CHECK(p.split_tokens == base.split_tokens + 32 || workgroups(lens, hkv, p.split_tokens - 32) > room);
  }
  CHECK(one > 30 && two > 30);
  std::printf("passed (%d in one round, %d in two)\n", one, two);
  return 0;
}
