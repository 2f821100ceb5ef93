// Host model of the cache in pages: what a batch's numbers are refused for, the parts of its workspace, the pieces of the keys, the list of a batch's work inside
// its bounds, and sequences from whatever the device holds.
#include <cstdio>
#include <cstdlib>
#include <random>
#include <vector>

#include "../paper_2605_12471_amd/csrc/pcache.h"

using namespace kvfold;

#define CHECK(x)                                                       \
  do {                                                                 \
    if (!(x)) {                                                        \
      std::printf("%s:%d: %s\n", __FILE__, __LINE__, #x);              \
      std::exit(1);                                                    \
    }                                                                  \
  } while (0)

static kvfold_pcache_config_t config(int hq, int hkv, int d, int page, int n_pages, int dtype) {
  kvfold_pcache_config_t c{};
  c.struct_size = sizeof c;
  c.n_layers = 1;
  c.n_q_heads = hq;
  c.n_kv_heads = hkv;
  c.head_dim = d;
  c.page_tokens = page;
  c.n_pages = n_pages;
  c.dtype = dtype;
  return c;
}

static kvfold_batch_t batch(int seqs, int tokens, int max_new, int64_t max_len, int64_t table) {
  kvfold_batch_t b{};
  b.struct_size = sizeof b;
  b.n_seqs = seqs;
  b.n_tokens = tokens;
  b.max_new = max_new;
  b.max_len = max_len;
  b.table_stride = table;
  return b;
}

static void refusals() {
  const kvfold_pcache_config_t c = config(8, 2, 128, 64, 1000, KVFOLD_BF16);
  CHECK(validate_pconfig(&c) == KVFOLD_OK);
  const kvfold_batch_t good = batch(4, 40, 10, 1000, 20);
  CHECK(validate_batch(c, &good) == KVFOLD_OK);
  CHECK(validate_batch(c, nullptr) == KVFOLD_ERR_INVALID_ARG);
  auto with = [&](auto change) {
    kvfold_batch_t b = good;
    change(b);
    return validate_batch(c, &b);
  };
  CHECK(with([](kvfold_batch_t& b) { b.struct_size = 4; }) == KVFOLD_ERR_INVALID_ARG);
  CHECK(with([](kvfold_batch_t& b) { b.n_seqs = -1; }) == KVFOLD_ERR_INVALID_ARG);
  CHECK(with([](kvfold_batch_t& b) { b.n_tokens = -1; }) == KVFOLD_ERR_INVALID_ARG);
  CHECK(with([](kvfold_batch_t& b) { b.max_new = 0; }) == KVFOLD_ERR_INVALID_ARG);
  CHECK(with([](kvfold_batch_t& b) { b.max_len = 0; }) == KVFOLD_ERR_INVALID_ARG);
  CHECK(with([](kvfold_batch_t& b) { b.table_stride = 0; }) == KVFOLD_ERR_INVALID_ARG);
  CHECK(with([](kvfold_batch_t& b) { b.q_stride = 1028; }) == KVFOLD_ERR_INVALID_ARG);
  CHECK(with([](kvfold_batch_t& b) { b.q_stride = 1016; }) == KVFOLD_ERR_INVALID_ARG);
  CHECK(with([](kvfold_batch_t& b) { b.q_stride = -8; }) == KVFOLD_ERR_INVALID_ARG);
  CHECK(with([](kvfold_batch_t& b) { b.kv_stride = 248; }) == KVFOLD_ERR_INVALID_ARG);
  CHECK(with([](kvfold_batch_t& b) { b.kv_stride = 264; }) == KVFOLD_OK);
  CHECK(with([](kvfold_batch_t& b) { b.q_stride = 1024, b.kv_stride = 256; }) == KVFOLD_OK);
  CHECK(with([](kvfold_batch_t& b) { b.kv_stride = (int64_t)1 << 32; }) == KVFOLD_ERR_UNSUPPORTED);
  CHECK(with([](kvfold_batch_t& b) { b.q_stride = (int64_t)1 << 62; }) == KVFOLD_ERR_UNSUPPORTED);
  CHECK(with([](kvfold_batch_t& b) { b.max_len = ((int64_t)1 << 30) + 1; }) == KVFOLD_ERR_UNSUPPORTED);
  CHECK(with([](kvfold_batch_t& b) { b.max_len = (int64_t)1 << 30; }) == KVFOLD_OK);
  CHECK(with([](kvfold_batch_t& b) { b.table_stride = (int64_t)1 << 31; }) == KVFOLD_ERR_UNSUPPORTED);
  CHECK(with([](kvfold_batch_t& b) { b.n_seqs = (1 << 20) + 1; }) == KVFOLD_ERR_UNSUPPORTED);
  CHECK(with([](kvfold_batch_t& b) { b.n_tokens = 1 << 27; }) == KVFOLD_ERR_UNSUPPORTED);
}

// Whatever the device holds: inside the bounds
static void sequences() {
  const int odd[] = {INT32_MIN, INT32_MIN + 1, -5, -1, 0, 1, 7, 99, 100, 101, INT32_MAX - 1, INT32_MAX};
  for (int from : odd)
    for (int to : odd)
      for (int len : odd)
        for (int tokens : {1, 100})
          for (int max_new : {1, 60, 100})
            for (int max_len : {1, 100, 1 << 30}) {
              const PagedSeq q = paged_seq(from, to, len, tokens, max_new, max_len);
              CHECK(q.first >= 0 && q.n >= 0 && q.n <= max_new && q.first + q.n <= tokens && q.len >= 0 && q.len <= max_len);
              if (0 <= from && from <= to && to <= tokens && to - from <= max_new && 0 <= len && len <= max_len)
                CHECK(q.first == from && q.n == to - from && q.len == len);
            }
  for (int len : {0, 1, 127, 128, 129, 1 << 30})
    for (int piece : {128, 256, 1 << 20}) CHECK(paged_pieces(len, piece) >= 1 && ((int64_t)paged_pieces(len, piece) * piece >= len) && (len == 0 || (int64_t)(paged_pieces(len, piece) - 1) * piece < len));
}

// A plan against batches inside its numbers: what its list and its partial results have room for is enough, whichever length of a piece the device takes.
static void plans() {
  std::mt19937 rng(11);
  auto any = [&](int lo, int hi) { return lo + (int)(rng() % (unsigned)(hi - lo + 1)); };
  const int heads[][2] = {{4, 1}, {8, 2}, {7, 1}, {32, 8}, {40, 2}, {3, 3}, {64, 1}};
  int prompts = 0, cut = 0;
  for (int i = 0; i < 6000; ++i) {
    const auto& h = heads[any(0, 6)];
    const int page = 16 << any(0, 4), G = h[0] / h[1];
    const kvfold_pcache_config_t c = config(h[0], h[1], any(0, 1) ? 128 : 64, page, 100000, any(0, 1) ? KVFOLD_BF16 : KVFOLD_F32);
    const int seqs = any(1, i % 3 ? 20 : 400), top = any(0, 2) ? any(1, 40) : any(1, 700), longest = 1 << any(4, 16);
    std::vector<int> n(seqs), len(seqs);
    int tokens = 0, max_new = 1, max_len = 1;
    for (int s = 0; s < seqs; ++s) {
      n[s] = any(0, top);
      len[s] = n[s] + any(0, longest);
      tokens += n[s];
      max_new = std::max(max_new, n[s]);
      max_len = std::max(max_len, len[s]);
    }
    const kvfold_batch_t b = batch(seqs, tokens + any(0, 9), max_new + any(0, 3), max_len + any(0, 1000), (max_len + 1000) / page + 1);
    CHECK(validate_batch(c, &b) == KVFOLD_OK);
    const PagedPlan pl = make_pplan(c, 256, b);
    CHECK(pl.counters >= (size_t)seqs * h[1] * kPagedMeetStride * 4 && pl.counters % 256 == 0 && pl.list % 256 == 0);
    CHECK(pl.bytes >= pl.counters + pl.list + (size_t)pl.rows * (c.head_dim + 2) * 4 && pl.rows <= kPagedMaxRows);
    CHECK(pl.n_pieces >= 1);
    if (pl.decode) {
      CHECK(pl.unit_rows <= 16 && pl.unit_rows >= std::min(max_new, tokens) * G && pl.piece % 128 == 0 && pl.n_pieces <= kPagedMaxPieces);
      for (int s = 0; s < seqs; ++s) CHECK(paged_pieces(len[s], pl.piece) <= pl.n_pieces);
      CHECK(pl.n_pieces == 1 || pl.rows == (int64_t)seqs * h[1] * pl.n_pieces * pl.unit_rows);
      CHECK(pl.shared == 0.f || (!pl.from_end && seqs > 1 && (int64_t)seqs * h[1] < 256 && (int64_t)seqs * h[1] * pl.n_pieces <= 2 * kPagedMostWgs));  // (pieces are longer than pl.piece then)
      continue;
    }
    ++prompts;
    auto items = [&](int keys) {
      int64_t count = 0;
      for (int s = 0; s < seqs; ++s)
        for (int64_t r = 0; r < (int64_t)n[s] * G; r += pl.unit_rows) {
          const int64_t last = std::min<int64_t>(r + pl.unit_rows, (int64_t)n[s] * G), seen = len[s] - n[s] + (last - 1) / G + 1;
          count += paged_pieces((int)seen, keys);
        }
      return count;
    };
    const int tiles = (max_len + 63) / 64, most = (std::max(tiles, 2) + 1) / 2 * 2;
    CHECK(items(most * 64) <= pl.blocks && pl.blocks <= pl.items);  // in one piece each: always room
    CHECK(pl.list >= kPromptHead + (size_t)pl.items * sizeof(PromptItem) + (size_t)pl.blocks * 4);
    if (pl.n_pieces > 1) {
      CHECK(pl.rows == (int64_t)b.n_tokens * h[0] * pl.n_pieces);
      const int least = (most + pl.n_pieces - 1) / pl.n_pieces;
      for (int x = std::max(least, pl.shortest); x < most; x += any(1, 9)) {
        const int keys = (x + 1) / 2 * 2 * 64;
        for (int s = 0; s < seqs; ++s) CHECK(paged_pieces(len[s], keys) <= pl.n_pieces);
      }
      ++cut;
    }
  }
  CHECK(prompts > 1000 && cut > 300);
  // the largest numbers: nothing overflows
  for (int d : {64, 128})
    for (int type : {KVFOLD_BF16, KVFOLD_F32}) {
      const kvfold_pcache_config_t c = config(32, 8, d, 16, (1 << 27) - 1, type);
      CHECK(validate_pconfig(&c) == KVFOLD_OK);
      for (int seqs : {1, 1 << 20})  // (times 8 KV heads: as many as there may be)
        for (int tokens : {1, 1 << 20, 1 << 23})
          for (int max_new : {1, 4, 100, 1 << 23})
            for (int64_t len : {(int64_t)1, (int64_t)5000, (int64_t)1 << 30}) {
              const kvfold_batch_t b = batch(seqs, tokens, max_new, len, 1 << 26);
              CHECK(validate_batch(c, &b) == KVFOLD_OK);
              const PagedPlan pl = make_pplan(c, 256, b);
              CHECK(pl.rows >= 0 && pl.rows <= kPagedMaxRows && pl.bytes >= pl.counters && pl.bytes < (size_t)1 << 36 && pl.items * 8 < (int64_t)1 << 24);  // (256 threads each: below 2^32)
              CHECK(pl.n_pieces >= 1 && (!pl.decode || (pl.piece >= 128 && (int64_t)pl.piece * pl.n_pieces >= std::min<int64_t>(len, 1 << 30))));
            }
    }
}

int main() {
  refusals();
  sequences();
  plans();
  std::puts("ok: refusals, sequences, plans");
}
