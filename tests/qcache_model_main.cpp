// Host model of the cache held in 8 bits: where its elements lie, who writes the ring, what can be rewound, and the launch plans.
#include <cstdio>
#include <cstdlib>
#include <random>
#include <vector>

#include "../paper_2605_12471_amd/csrc/kvfold_plan.h"
#include "../paper_2605_12471_amd/csrc/qcache.h"

using namespace kvfold;

#define CHECK(x)                                                       \
  do {                                                                 \
    if (!(x)) {                                                        \
      std::printf("%s:%d: %s\n", __FILE__, __LINE__, #x);              \
      std::exit(1);                                                    \
    }                                                                  \
  } while (0)

static kvfold_config_t config(int hq, int hkv, int d, int chunk, int64_t capacity) {
  kvfold_config_t c{};
  c.struct_size = sizeof c;
  c.n_layers = 2;
  c.n_q_heads = hq;
  c.n_kv_heads = hkv;
  c.head_dim = d;
  c.chunk_tokens = chunk;
  c.capacity_tokens = capacity;
  c.dtype = KVFOLD_BF16;
  return c;
}

// Every element of a block has a place of its own.
static void layout() {
  for (int kg = 0; kg < 4; ++kg)
    for (int e = 0; e < 16; ++e) {
      const int key = q_key(kg, e);
      CHECK(key >= 0 && key < kQBlock && q_key_group(key) == kg && q_key_element(key) == e);
    }
  for (int d : {64, 128}) {
    std::vector<int> k((size_t)kQBlock * d), v(k.size());
    for (int key = 0; key < kQBlock; ++key)
      for (int col = 0; col < d; ++col) {
        ++k.at((size_t)q_k_piece(col / 16, key) * 16 + col % 16);
        ++v.at((size_t)q_v_piece(d, q_key_group(key), col) * 16 + q_key_element(key));
      }
    for (size_t i = 0; i < k.size(); ++i) CHECK(k[i] == 1 && v[i] == 1);
    // what the decoding kernel's lanes load: all rows of its four tiles, all columns and keys
    std::vector<int> seen((size_t)kQBlock);
    for (int t = 0; t < 4; ++t)
      for (int c16 = 0; c16 < 16; ++c16) {
        const int row = 32 * (c16 >> 3) + 4 * (c16 >> 2 & 1) + 8 * t + (c16 & 3);
        ++seen.at((size_t)row);
        CHECK(q_key_group(row) == c16 >> 2 && q_key_element(row) == 4 * t + (c16 & 3));  // row 4 kg + e of the tile: the keys of group kg
        CHECK(q_k_piece(4 * (d / 64 - 1) + 3, row) < kQBlock * d / 16);
      }
    for (int n : seen) CHECK(n == 1);
  }
}

// The append's blocks: which workgroup writes a ring slot, and that none writes what another still reads.
static void ring() {
  std::mt19937 rng(1);
  for (int round = 0; round < 20000; ++round) {
    const int64_t prev = rng() % 400, n = 1 + rng() % 500, end = prev + n, first = prev / kQBlock, last = (end - 1) / kQBlock;
    const int64_t over = last - (last - first) % kQRing;
    std::vector<int64_t> writer(kQRing, -1), holds(kQRing, -1);
    auto write = [&](int64_t by, int64_t block) {
      CHECK(writer[(size_t)(block % kQRing)] == -1);
      writer[(size_t)(block % kQRing)] = by;
      holds[(size_t)(block % kQRing)] = block;
    };
    for (int64_t b = first; b <= last; ++b) {
      const bool later = b != first && (b - first) % kQRing == 0;
      if (b + kQRing > last && !later) write(b, b);
      if (b == first && over > first) write(b, over);
    }
    for (int64_t b = last; b > last - kQRing && b >= first; --b) CHECK(holds[(size_t)(b % kQRing)] == b);
    // the first block's earlier rows are read by its own workgroup, the only one to write their slot
    if (prev % kQBlock) CHECK(writer[(size_t)(first % kQRing)] == -1 || writer[(size_t)(first % kQRing)] == first);
  }
}

// A ring of rows beside the bookkeeping: whatever can be rewound to has its incomplete block's rows there.
static void rewinding() {
  std::mt19937 rng(2);
  for (int round = 0; round < 300; ++round) {
    QLength l;
    std::vector<int64_t> row(kQRing * kQBlock, -1);
    for (int turn = 0; turn < 60; ++turn) {
      if (rng() % 3) {
        const int64_t n = 1 + rng() % (rng() % 2 ? 5 : 200), last = (l.len + n - 1) / kQBlock;
        for (int64_t t = l.len; t < l.len + n; ++t)
          if (t / kQBlock + kQRing > last) row[(size_t)(t % (kQRing * kQBlock))] = t;
        l.append(n);
      } else {
        const int64_t to = rng() % 2 ? l.len - (int64_t)(rng() % 70) : (int64_t)(rng() % (l.len + 1));
        if (l.can_truncate(to)) l.truncate(to);
        CHECK(!l.can_truncate(l.len + 1) && !l.can_truncate(-1) && l.can_truncate(l.len / kQBlock * kQBlock));
      }
      for (int64_t t = l.len / kQBlock * kQBlock; t < l.len; ++t) CHECK(row[(size_t)(t % (kQRing * kQBlock))] == t);
      if (l.len > 64 && l.ring_from == 0) CHECK(l.can_truncate(l.len - 64));
    }
  }
  QLength l;
  l.append(1000);
  for (int64_t back = 0; back <= 64; ++back) CHECK(l.can_truncate(1000 - back));
}

static void plans() {
  std::mt19937 rng(3);
  for (int round = 0; round < 20000; ++round) {
    const int hkv = 1 + rng() % 16, hq = hkv * (1 + rng() % 16), d = rng() % 2 ? 64 : 128, chunk = 1 + rng() % (rng() % 2 ? 20 : 4096);
    const int64_t capacity = chunk + rng() % 100000;
    const kvfold_config_t c = config(hq, hkv, d, chunk, capacity);
    CHECK(validate_qconfig(&c) == KVFOLD_OK);
    const int n = 1 + rng() % chunk;
    const int64_t len = n + rng() % (capacity - n + 1), ws = workspace_rows(&c);
    const QPlan p = make_qplan(c, 256, ws, n, len);
    const int blocks = (int)((len + kQBlock - 1) / kQBlock);
    CHECK(p.n_splits >= 1 && p.n_splits <= kMaxSplits && p.blocks_per_split >= 1);
    CHECK((int64_t)(p.n_splits - 1) * p.blocks_per_split < blocks && (int64_t)p.n_splits * p.blocks_per_split >= blocks);  // no piece without a block
    CHECK(p.n_splits == 1 || (int64_t)p.n_splits * n * hq <= ws);
    CHECK(p.n_wgs == hkv * p.wgs_per_head * p.n_splits);
    CHECK(p.decode ? n * (hq / hkv) <= 16 && p.wgs_per_head == 1 : p.wgs_per_head * p.waves_per_wg >= p.units_per_head && (p.wgs_per_head - 1) * p.waves_per_wg < p.units_per_head);
    const QLayout l = q_layout(c);
    CHECK(l.blocks * kQBlock >= capacity && l.codes % 256 == 0 && l.scales % 256 == 0 && l.ring % 256 == 0);
    CHECK(l.layer == 2 * l.codes + l.scales + 2 * l.ring);
  }
}

int main() {
  layout();
  ring();
  rewinding();
  plans();
  std::printf("ok: layout, ring, rewinding, plans\n");
}
