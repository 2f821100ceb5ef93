// Attention weights by key, and the eviction of keys by them (kvfold_cache_weigh, kvfold_cache_evict).
#pragma once
#include <stddef.h>
#include <stdint.h>

#include "kvfold_consts.h"

namespace kvfold {

constexpr int kEvictRows = 64;     // rows that a workgroup moves
constexpr int kEvictPiece = 8192;  // rows that a workgroup looks through where a KV head has several

// Whether wavefronts that weigh the same keys share out the rows, units of 32 of them: where workgroups of 128 keys, wgs of them, leave CUs without
// work (measured: weigh.hip, launch_width()).
inline bool weigh_shares_rows(bool bf16, int n_cu, int64_t wgs, int units) { return bf16 ? 2 * wgs < 3 * (int64_t)n_cu && units >= 8 : wgs < n_cu && units >= 4; }

// The caller's workspace of an eviction, in words: kept rows' indices and weights [Hkv][n_keep], per chunk of kEvictRows rows the number of kept
// rows in front of it [Hkv][chunks + 1] and whether its rows have been read [Hkv][chunks], the next chunk to move; for pieces of long
// caches the counts of a digit's values [2][Hkv][pieces][256], the rows known to be kept [Hkv][pieces], and what is known of the smallest kept
// weight [2][Hkv][2].
struct EvictLayout {
  int64_t chunks, pieces;
  size_t kept, weights, before, read, next, counts, more, state, words;
};
inline EvictLayout evict_layout(int64_t n_kv_heads, int64_t n_keep, int64_t capacity) {
  EvictLayout l;
  l.chunks = (n_keep + kEvictRows - 1) / kEvictRows;
  l.pieces = (capacity + kEvictPiece - 1) / kEvictPiece;
  const size_t rows = (size_t)(n_kv_heads * n_keep), chunks = (size_t)(n_kv_heads * l.chunks);
  l.kept = 0;
  l.weights = l.kept + rows;
  l.before = l.weights + rows;
  l.read = l.before + chunks + (size_t)n_kv_heads;
  l.next = l.read + chunks;
  l.counts = l.next + 1;
  l.more = l.counts + 2 * 256 * (size_t)(n_kv_heads * l.pieces);
  l.state = l.more + (size_t)(n_kv_heads * l.pieces);
  l.words = l.state + 4 * (size_t)n_kv_heads;
  return l;
}

// The chunks [from, to) that a chunk, moved in place, waits for: in front of it, with kept rows that lie where it writes.  front, behind: how many kept rows
// lie before its first place and before the place behind its last.
struct EvictWaits {
  int from, to;
};
KVFOLD_HD EvictWaits evict_waits(uint32_t front, uint32_t behind, int chunk) {
  const int end = (int)((behind + kEvictRows - 1) / kEvictRows);
  return EvictWaits{(int)(front / kEvictRows), end < chunk ? end : chunk};
}

}  // namespace kvfold

#if defined(__HIP__)
#include "kvfold_internal.h"

namespace kvfold {

struct WeighParams {
  const void* q;       // [n][Hq][d]
  const void* k;       // layer base, [Hkv][cap][d]
  const float* lse;    // [Hq][n], natural logarithms
  float* weights;      // [Hkv][cap]
  const float *rope_cos, *rope_sin;  // of the queries, [n][d/2], or nullptr
  int64_t capacity;
  int32_t n_tokens, n_q_heads, n_kv_heads, group, len;  // len: rows of the layer, the chunk's n_tokens the last of them
  int32_t add;
  float scale_log2e;
  FastDiv by_group;
};
hipError_t launch_weigh(const WeighParams& p, int head_dim, bool bf16, int n_cu, hipStream_t s);

struct EvictParams {
  const float* weights;     // [Hkv][from_capacity]
  const unsigned char* from[2];  // K, V: layer base, [Hkv][from_capacity][row_bytes]
  unsigned char* to[2];
  float* to_weights;        // [Hkv][to_capacity] or nullptr
  int32_t* kept;            // [Hkv][n_keep]
  uint32_t* workspace;
  EvictLayout ws;
  int64_t from_capacity, to_capacity;
  int32_t n_kv_heads, row_bytes, len, n_sink, n_recent, n_keep;
  int32_t in_place;
};
hipError_t launch_evict(const EvictParams& p, hipStream_t s);

}  // namespace kvfold
#endif
