// What the prompt kernels of the cache in pages have in common: which rows are a workgroup's, and its tiles' way from the pages into LDS.
#pragma once
#include "pcache.h"
#include "wave_ops.h"

namespace kvfold {

// The workgroup's packed rows [row0, row0 + unit_rows) of a sequence and KV head, and the keys that its piece has.
struct PromptWork {
  int seq, row0, rows;      // rows: packed rows of the sequence
  PagedSeq sq;
  int g, piece, n_pieces;   // n_pieces: of the keys that the workgroup's last row sees
  int key_begin, key_end;
  bool any;
};

// The sequence whose workgroups begin at or before block b, the last of those that do: 64 candidates a step, one a lane.
__device__ __forceinline__ int prompt_find(const PAttnParams& p, int64_t b, int l) {
  int lo = 0, n = p.n_seqs;
  while (n > 1) {
    const int step = (n + 63) >> 6, i = lo + l * step;
    bool before = false;
    if (l * step < n) before = paged_first_block(p.cu_new[i], i, p.group, p.unit_rows) <= b;
    const uint64_t which = __ballot(before);
    const int k = which ? 63 - __builtin_clzll(which) : 0;
    lo += k * step;
    n = n - k * step < step ? n - k * step : step;
  }
  return __builtin_amdgcn_readfirstlane(lo);
}

// Blocks come heaviest first: a prompt's last rows see the most keys.
__device__ __forceinline__ PromptWork prompt_work(const PAttnParams& p, unsigned id, int l) {
  PromptWork k;
  const int b_piece = (int)quot(id, p.by_kv_heads);  // (KV heads side by side: with eight, each on its own XCD)
  k.g = (int)id - b_piece * p.n_kv_heads;
  const int n = (int)quot((unsigned)b_piece, p.by_units);
  k.piece = n;
  const int64_t b = p.n_units - 1 - (b_piece - n * p.n_units);
  int from, to, len;
  if (p.cu_new) {
    k.seq = prompt_find(p, b, l);
    from = ((ConstPtr<int32_t>)(uintptr_t)p.cu_new)[k.seq];
    to = ((ConstPtr<int32_t>)(uintptr_t)p.cu_new)[k.seq + 1];
  } else {  // (one row a sequence: more than 16 query heads share a KV head)
    int lo = 0, hi = p.n_seqs;
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (paged_first_block(mid, mid, p.group, p.unit_rows) <= b)
        lo = mid;
      else
        hi = mid;
    }
    k.seq = lo;
    from = lo;
    to = lo + 1;
  }
  len = ((ConstPtr<int32_t>)(uintptr_t)p.lens)[k.seq];
  k.sq = paged_seq(from, to, len, p.n_tokens, p.max_new, p.max_len);
  const int64_t in_seq = b - paged_first_block(from, k.seq, p.group, p.unit_rows);
  k.rows = k.sq.n * p.group;
  k.any = in_seq >= 0 && in_seq * p.unit_rows < k.rows;
  k.row0 = k.any ? (int)in_seq * p.unit_rows : 0;
  const int last = k.row0 + p.unit_rows < k.rows ? k.row0 + p.unit_rows : k.rows;
  int seen = k.sq.len - k.sq.n + (k.rows ? (int)quot((unsigned)(last - 1), p.by_group) : 0) + 1;
  if (seen < 0) seen = 0;
  k.n_pieces = paged_pieces(seen, p.piece);
  if (k.piece >= k.n_pieces) k.any = false;
  k.key_begin = k.piece * p.piece;
  k.key_end = k.key_begin + p.piece < seen ? k.key_begin + p.piece : seen;
  return k;
}

// The page numbers of 64 runs of 16 keys, one a lane, and which of them are pages.
struct PageWindow {
  int number = -1;
  uint64_t there = 0;
  __device__ __forceinline__ void fetch(const PAttnParams& p, const int32_t* table, int key0, int key_end, int l) {
    const int key = key0 + 16 * l;
    number = -1;
    if (key < key_end) number = table[(unsigned)key >> p.page_log2];
    there = __ballot((unsigned)number < (unsigned)p.n_pages);
  }
};

}  // namespace kvfold
