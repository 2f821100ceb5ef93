// Host model of rules that the kernels and their launches take from the headers that this file includes: who writes the 8-bit cache's ring of bf16 rows,
// whom a chunk of an eviction in place waits for (workgroups run in any order that the rules allow), and how weighing wavefronts are shared out.
#include <algorithm>
#include <cstdio>
#include <cstdlib>
#include <random>
#include <vector>

#include "../paper_2605_12471_amd/csrc/qcache.h"
#include "../paper_2605_12471_amd/csrc/weigh.h"

using namespace kvfold;

#define CHECK(x)                                                       \
  do {                                                                 \
    if (!(x)) {                                                        \
      std::printf("%s:%d: %s\n", __FILE__, __LINE__, #x);              \
      std::exit(1);                                                    \
    }                                                                  \
  } while (0)

// A layer's ring: in place r % 128 the row that lies there, and whether it is the one that counts as row r.
static void ring() {
  std::mt19937 rng(1);
  constexpr int N = kQRing * kQBlock;
  for (int round = 0; round < 4000; ++round) {
    QLength length;
    std::vector<int64_t> place(N, -1), name;  // name[r]: the row that was appended as row r, each its own
    // since: from where on any place can be gone back to -- the beginning of the block before the last one that rows were appended to, or where a rewind
    // has gone in front of that
    int64_t names = 0, since = 0;
    for (int turn = 0; turn < 12; ++turn) {
      if (rng() % 4 == 0) {
        const int64_t to = rng() % 3 == 0 ? (int64_t)(rng() % (length.len / kQBlock + 1)) * kQBlock : std::max<int64_t>(0, length.len - (int64_t)(rng() % 80));
        const bool whole = to % kQBlock == 0;
        // what can be gone back to: whole blocks, and places whose incomplete block's rows lie in the ring
        bool there = true;
        for (int64_t r = to / kQBlock * kQBlock; r < to; ++r) there = there && place[(size_t)(r % N)] == name[(size_t)r];
        CHECK(length.can_truncate(to) == (whole || to >= since));
        CHECK(!length.can_truncate(to) || whole || there);
        if (!length.can_truncate(to)) continue;
        since = std::min(since, to);
        length.truncate(to);
        name.resize((size_t)to);
        continue;
      }
      const int64_t prev = length.len, n = 1 + rng() % (rng() % 2 ? 20 : 400), end = prev + n;
      for (int64_t r = prev; r < end; ++r) name.push_back(names++);
      const QRingWriters w(prev, n);
      auto write = [&](int64_t block) {
        for (int64_t r = std::max(prev, block * kQBlock); r < std::min(end, (block + 1) * kQBlock); ++r) place[(size_t)(r % N)] = name[(size_t)r];
      };
      auto read = [&]() {  // the first block's earlier rows, if it is whole now and is made codes
        if (w.earlier && (w.first + 1) * kQBlock <= end)
          for (int64_t r = w.first * kQBlock; r < prev; ++r) CHECK(place[(size_t)(r % N)] == name[(size_t)r]);
      };
      std::vector<int64_t> order;
      for (int64_t b = w.first; b <= w.last; ++b) order.push_back(b);
      std::shuffle(order.begin(), order.end(), rng);
      // the first block's workgroup in three parts, among the others in any order
      const size_t at = (size_t)(std::find(order.begin(), order.end(), w.first) - order.begin());
      order.erase(order.begin() + (long)at);
      size_t cut[3];
      for (size_t& c : cut) c = rng() % (order.size() + 1);
      std::sort(cut, cut + 3);
      for (size_t i = 0; i <= order.size(); ++i) {
        if (i == cut[0] && w.itself(w.first)) write(w.first);
        if (i == cut[1]) read();
        if (i == cut[2] && w.taken_over() > w.first) write(w.taken_over());
        if (i < order.size() && w.itself(order[i])) write(order[i]);
      }
      length.append(n);
      since = std::max(since, (w.last - 1) * kQBlock);
      CHECK(length.len == end);
      for (int64_t r = std::max(prev, (w.last - (kQRing - 1)) * kQBlock); r < end; ++r) CHECK(place[(size_t)(r % N)] == name[(size_t)r]);
      for (int64_t r = end / kQBlock * kQBlock; r < end; ++r) CHECK(place[(size_t)(r % N)] == name[(size_t)r]);
    }
  }
}

// 128 rows are left of 300 and only codes of them: their last block cannot be gone back into.
static void rewound_to_codes() {
  QLength l;
  l.append(300);
  CHECK(l.can_truncate(236) && l.can_truncate(193) && !l.can_truncate(191) && l.can_truncate(128));
  l.truncate(128);
  l.append(10);
  CHECK(!l.can_truncate(74) && !l.can_truncate(127) && l.can_truncate(128) && l.can_truncate(129) && l.can_truncate(64));
  l.append(190);
  CHECK(l.can_truncate(264) && l.can_truncate(257) && !l.can_truncate(255) && l.can_truncate(192));
}

static void move(std::mt19937& rng, int len, int keep) {
  std::vector<int> all((size_t)len), cache((size_t)len);
  for (int i = 0; i < len; ++i) all[(size_t)i] = cache[(size_t)i] = i;
  std::shuffle(all.begin(), all.end(), rng);
  std::vector<int> kept(all.begin(), all.begin() + keep);
  std::sort(kept.begin(), kept.end());
  const int chunks = (keep + kEvictRows - 1) / kEvictRows;
  std::vector<uint32_t> before((size_t)chunks + 1);
  for (int c = 0; c <= chunks; ++c) before[(size_t)c] = (uint32_t)(std::lower_bound(kept.begin(), kept.end(), c * kEvictRows) - kept.begin());
  std::vector<std::vector<int>> held((size_t)chunks);
  std::vector<int> state((size_t)chunks, 0);  // 1: handed out, 2: read, 3: written
  int next = 0, running = 0;
  const int resident = 1 + (int)(rng() % 8);
  for (int done = 0; done < chunks;) {
    std::vector<int> ready;
    if (next < chunks && running < resident) ready.push_back(next);
    for (int c = 0; c < next; ++c) {
      const EvictWaits w = evict_waits(before[(size_t)c], before[(size_t)c + 1], c);
      CHECK(w.to <= c);
      bool free = state[(size_t)c] == 1 || state[(size_t)c] == 2;
      if (state[(size_t)c] == 2)
        for (int other = w.from; other < w.to; ++other) free = free && state[(size_t)other] >= 2;
      if (free) ready.push_back(c);
    }
    CHECK(!ready.empty());  // nobody waits for ever
    const int c = ready[rng() % ready.size()], row0 = c * kEvictRows, end = std::min(keep, row0 + kEvictRows);
    switch (++state[(size_t)c]) {
      case 1:
        ++next, ++running;
        break;
      case 2:
        for (int i = row0; i < end; ++i) held[(size_t)c].push_back(cache[(size_t)kept[(size_t)i]]);
        break;
      case 3:
        for (int i = row0; i < end; ++i) cache[(size_t)i] = held[(size_t)c][(size_t)(i - row0)];
        --running, ++done;
    }
  }
  for (int i = 0; i < keep; ++i) CHECK(cache[(size_t)i] == kept[(size_t)i]);
}

// The same share of a chip, whatever its CUs are.
static void weighing() {
  for (int n_cu : {32, 64, 256, 304})
    for (int64_t wgs = 1; wgs < 1000; ++wgs) {
      CHECK(weigh_shares_rows(true, n_cu, wgs, 8) == ((double)wgs < 1.5 * n_cu) && weigh_shares_rows(false, n_cu, wgs, 4) == (wgs < n_cu));
      CHECK(!weigh_shares_rows(true, n_cu, wgs, 7) && !weigh_shares_rows(false, n_cu, wgs, 3));
    }
}

int main() {
  ring();
  weighing();
  rewound_to_codes();
  std::mt19937 rng(2);
  for (int round = 0; round < 3000; ++round) {
    const int len = 1 + (int)(rng() % 1500);
    move(rng, len, 1 + (int)(rng() % (unsigned)len));
  }
  std::printf("ok: ring, rewinding, weighing, moving in place\n");
}
