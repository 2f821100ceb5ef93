// What the prompt kernels of the cache in pages have in common: which work is a workgroup's, and the page numbers of its tiles.
#pragma once
#include "pcache.h"
#include "wave_ops.h"

namespace kvfold {

// A workgroup's work: an item of the list, for a KV head.
struct PromptWork {
  PagedSeq sq;
  int seq, row0, rows;  // rows: packed rows of the sequence
  int g, piece, n_pieces;
  int key_begin, key_end;
  bool any;
};
__device__ __forceinline__ PromptWork prompt_item(const PAttnParams& p, int n, int g) {
  const ConstPtr<int32_t> x = (ConstPtr<int32_t>)(uintptr_t)(p.items + n);
  PromptWork k;
  k.g = g;
  k.seq = x[0];
  k.sq.first = x[1];
  k.sq.n = x[2];
  k.sq.len = x[3];
  k.rows = x[2] * p.group;
  k.row0 = x[4];
  k.key_begin = x[5];
  k.key_end = x[6];
  k.piece = x[7] & 0xffff;
  k.n_pieces = x[7] >> 16;
  k.any = true;
  return k;
}
// KV heads side by side: with eight, each on its own XCD.  (An item is fetched before it is known whether it is there: the list has room for all that may be asked for.)
__device__ __forceinline__ PromptWork prompt_work(const PAttnParams& p, unsigned id) {
  const int n = (int)quot(id, p.by_kv_heads);
  PromptWork k = prompt_item(p, n, (int)id - n * p.n_kv_heads);
  k.any = n < ((ConstPtr<int32_t>)(uintptr_t)p.list_head)[0];
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
