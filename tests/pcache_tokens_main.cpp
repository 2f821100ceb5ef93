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

int main() {
  positions();
  std::puts("ok: positions");
}
