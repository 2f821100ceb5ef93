// Host model of the eviction in place: chunks of 64 kept rows, handed out in order, each run in two halves (all rows read; then, once the chunks that it
// waits for have read theirs, written) in any order that the waits allow.
#include <algorithm>
#include <cstdio>
#include <cstdlib>
#include <random>
#include <vector>

#include "../paper_2605_12471_amd/csrc/weigh.h"

using namespace kvfold;

#define CHECK(x)                                                       \
  do {                                                                 \
    if (!(x)) {                                                        \
      std::printf("%s:%d: %s\n", __FILE__, __LINE__, #x);              \
      std::exit(1);                                                    \
    }                                                                  \
  } while (0)

static void layout() {
  for (int64_t heads : {1, 3, 8})
    for (int64_t keep : {1, 63, 64, 65, 1000, 20000}) {
      const EvictLayout l = evict_layout(heads, keep, keep + 500);
      CHECK(l.chunks * kEvictRows >= keep && (l.chunks - 1) * kEvictRows < keep);
      CHECK(l.weights == l.kept + (size_t)(heads * keep) && l.before == l.weights + (size_t)(heads * keep));
      CHECK(l.read == l.before + (size_t)(heads * (l.chunks + 1)) && l.next == l.read + (size_t)(heads * l.chunks) && l.counts == l.next + 1);
      CHECK(l.pieces * kEvictPiece >= keep + 500 && l.more == l.counts + (size_t)(512 * heads * l.pieces) && l.state == l.more + (size_t)(heads * l.pieces));
      CHECK(l.words == l.state + (size_t)(4 * heads));
    }
}

static void move(std::mt19937& rng, int len, int keep) {
  std::vector<int> all((size_t)len), cache((size_t)len);
  for (int i = 0; i < len; ++i) all[(size_t)i] = cache[(size_t)i] = i;
  std::shuffle(all.begin(), all.end(), rng);
  std::vector<int> kept(all.begin(), all.begin() + keep);
  std::sort(kept.begin(), kept.end());
  const int chunks = (keep + kEvictRows - 1) / kEvictRows;
  std::vector<int> before((size_t)chunks + 1);
  for (int c = 0; c <= chunks; ++c) before[(size_t)c] = (int)(std::lower_bound(kept.begin(), kept.end(), c * kEvictRows) - kept.begin());
  std::vector<std::vector<int>> held((size_t)chunks);
  std::vector<int> state((size_t)chunks, 0);  // 0: not handed out, 1: has read, 2: done
  int next = 0, done = 0, running = 0;
  const int resident = 1 + (int)(rng() % 6);
  while (done < chunks) {
    // what can go on: the next chunk, if there is room for it, and any that waits for nobody
    std::vector<int> ready;
    if (next < chunks && running < resident) ready.push_back(-1);
    for (int c = 0; c < next; ++c) {
      if (state[(size_t)c] != 1) continue;
      bool wait = false;
      for (int other = before[(size_t)c] / kEvictRows; other < c && other * kEvictRows < before[(size_t)c + 1]; ++other) wait = wait || state[(size_t)other] == 0;
      if (!wait) ready.push_back(c);
    }
    CHECK(!ready.empty());  // nobody waits for ever
    const int c = ready[rng() % ready.size()];
    if (c < 0) {
      const int end = std::min(keep, (next + 1) * kEvictRows);
      for (int i = next * kEvictRows; i < end; ++i) held[(size_t)next].push_back(cache[(size_t)kept[(size_t)i]]);
      state[(size_t)next++] = 1;
      ++running;
    } else {
      for (size_t i = 0; i < held[(size_t)c].size(); ++i) cache[(size_t)c * kEvictRows + i] = held[(size_t)c][i];
      state[(size_t)c] = 2;
      --running;
      ++done;
    }
  }
  for (int i = 0; i < keep; ++i) CHECK(cache[(size_t)i] == kept[(size_t)i]);
}

int main() {
  layout();
  std::mt19937 rng(1);
  for (int round = 0; round < 3000; ++round) {
    const int len = 1 + (int)(rng() % 1500);
    move(rng, len, 1 + (int)(rng() % (unsigned)len));
  }
  std::printf("ok: layout, moving in place\n");
}
