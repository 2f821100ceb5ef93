// Host model of which tokens a batch's sequences have, against their definition: whatever the counts and lengths are.
#include <cstdio>
#include <cstdlib>
#include <random>
#include <vector>

#include "../paper_2605_12471_amd/csrc/pcache.h"

using namespace kvfold;

#define CHECK(x)                                          \
  do {                                                    \
    if (!(x)) {                                           \
      std::printf("%s:%d: %s\n", __FILE__, __LINE__, #x); \
      std::exit(1);                                       \
    }                                                     \
  } while (0)

// Token i of a sequence lies at position len - count + i, with the counts that the device holds; the first max_new of them take part.
static void positions() {
  for (int first : {0, 3, 50})
    for (int count : {0, 1, 2, 5, 40, 50})
      for (int len : {0, 1, 4, 5, 39, 40, 41, 100, 1000})
        for (int max_new : {1, 2, 5, 39, 40, 60}) {
          const PagedSeq q = paged_seq(first, first + count, len, 100, max_new, 1000);
          CHECK(q.first == first && q.n == (count < max_new ? count : max_new) && q.len >= 0 && q.len <= len);
          for (int i = 0; i < q.n; ++i) {
            const int at = q.len - q.n + i, want = len - count + i;
            CHECK(want >= 0 ? at == want : at < 0);
          }
        }
}

// A token belongs to the sequence that holds it, if it has a position there and counts; running sums that do not ascend end the search inside them.
static void tokens() {
  std::mt19937 rng(5);
  auto any = [&](int lo, int hi) { return lo + (int)(rng() % (unsigned)(hi - lo + 1)); };
  for (int i = 0; i < 3000; ++i) {
    const int seqs = any(1, 40), lead = any(0, 3), max_new = any(1, 9);
    std::vector<int32_t> cu(seqs + 1), lens(seqs);
    cu[0] = lead;
    for (int s = 0; s < seqs; ++s) {
      cu[s + 1] = cu[s] + (any(0, 2) ? any(0, 12) : 0);
      lens[s] = any(0, 20);
    }
    const int n_tokens = cu[seqs] + any(0, 4);
    for (int t = 0; t < n_tokens; ++t) {
      bool want = false;
      for (int s = 0; s < seqs; ++s)
        if (cu[s] <= t && t < cu[s + 1]) want = t - cu[s] < max_new && lens[s] - (cu[s + 1] - t) >= 0;
      CHECK(paged_token(cu.data(), lens.data(), 0, seqs, n_tokens, max_new, 1000, t) == want);
    }
    for (int t = 0; t < seqs; ++t) CHECK(paged_token(nullptr, lens.data(), t, t + 1, seqs, 1, 1000, t) == (lens[t] > 0));
    const int64_t slots[] = {0, 99, 100, -1, INT64_MIN, INT64_MAX};
    for (int t = 0; t < 6; ++t) CHECK(paged_one(slots, 100, t) == (t < 2 ? t + 1 : t) && paged_one(nullptr, 100, t) == t + 1);
    for (auto& x : cu) x = any(0, 3) ? any(-5, 60) : any(0, 1) ? INT32_MIN : INT32_MAX;
    for (auto& x : lens) x = any(0, 3) ? any(-5, 60) : any(0, 1) ? INT32_MIN : INT32_MAX;
    for (int t = 0; t < n_tokens; ++t) (void)paged_token(cu.data(), lens.data(), 0, seqs, n_tokens, max_new, 1000, t);
  }
}

int main() {
  positions();
  tokens();
  std::puts("ok: positions, tokens");
}
