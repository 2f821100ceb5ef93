// The cache in pages: what its kernels, its planner and the host model of both share.
#pragma once
#include <stddef.h>
#include <stdint.h>

#include "kvfold_consts.h"
#include "kvfold_plan.h"

namespace kvfold {

constexpr int64_t kPagedMaxRows = 1 << 20;  // (row, piece) pairs of a workspace
constexpr int kPagedMeetStride = 16;        // words from one unit's counter to the next: a line's
constexpr int kPagedMaxPieces = 128;        // of a sequence's keys
constexpr int kPagedLongestPiece = 2048;    // keys (decode)
constexpr int64_t kPagedMostWgs = 2048;     // of a decoding step whose lengths decide: many find that they have no piece (4096: 27.1 us for the first 24.2 in pcache_plan.cpp, 1024: 27.0; under a max_len that was the longest sequence's)

int validate_pconfig(const kvfold_pcache_config_t* c);
size_t pcache_layer_bytes(const kvfold_pcache_config_t& c);  // K and V
// What can be told from a batch's numbers, without its pointers
int validate_batch(const kvfold_pcache_config_t& c, const kvfold_batch_t* b);

struct PagedPlan {
  bool decode;           // at most 16 packed rows per sequence and KV head: the kernel that deals keys to wavefronts
  int unit_rows;         // packed rows of a workgroup (decode: of a sequence and KV head)
  int units_per_wave;    // prompts: 32-row units of a wavefront
  bool from_end;         // decode: a sequence's last piece is whole, and its first what is left
  int64_t blocks, items;  // prompts: blocks of rows per KV head, and these with a piece of their keys each, at most
  int places, shortest, step;  // PromptPlanParams
  float cost_once, cost_piece, cost_merge;
  int n_pieces;          // of the keys, at most
  int piece;             // decode: keys of one, a multiple of 128; where lengths decide, the fewest
  float shared;          // decode: steps of 128 keys of a piece for each that the sequences have, together; 0: the lengths do not decide
  int64_t rows;          // of partial results
  size_t counters;       // bytes in front of them: of the counters by which pieces meet,
  size_t list;           // prompts: and of the work's list
  size_t bytes;          // of the workspace
};
PagedPlan make_pplan(const kvfold_pcache_config_t& c, int n_cu, const kvfold_batch_t& b);

// Prompts: a block of rows of a sequence and a piece of the keys that its last row sees.  The list of them is made on the device, from the lengths there, in front of the
// attention (pcache_rows.hip); its head says how many there are.
struct PromptItem {
  int32_t seq, first, n, len;  // the sequence, its new tokens among the packed ones, its length
  int32_t row0;                // the block's first packed (token, query head) row
  int32_t key_begin, key_end;  // the piece
  int32_t piece;               // its number, and how many the block has in all << 16
};
static_assert(sizeof(PromptItem) == 32, "an item is fetched at once");
constexpr int kPromptHead = 64;     // bytes in front of the list: the number of items, and of blocks to merge
constexpr int kPromptMaxPieces = 64;

// The pieces of `len` keys, one at least
KVFOLD_HD int paged_pieces(int len, int piece) {
  const int n = (int)(((unsigned)len + (unsigned)piece - 1) / (unsigned)piece);
  return n < 1 ? 1 : n;
}

// A sequence's new tokens and its length from what the device holds, inside the batch's bounds whatever that is: tokens [first, first + n) exist, n <= max_new,
// 0 <= len <= max_len.  Token i has the position len - n + i: where there are more than max_new, the length ends behind the last that counts (at 0, where that lies in front of
// the first position).
struct PagedSeq {
  int first, n, len;
};
KVFOLD_HD PagedSeq paged_seq(int from, int to, int len, int n_tokens, int max_new, int max_len) {
  PagedSeq q;
  q.first = from < 0 ? 0 : from > n_tokens ? n_tokens : from;
  const int end = to < q.first ? q.first : to > n_tokens ? n_tokens : to;
  q.n = end - q.first < max_new ? end - q.first : max_new;
  const int beyond = end - q.first - q.n;
  q.len = len < 0 ? 0 : len > max_len ? max_len : len;
  q.len = q.len > beyond ? q.len - beyond : 0;
  return q;
}

// Without running sums: the end of sequence s's tokens, which begin at s.  It has one, where rows are stored (slots) if that has a place: an assignment that could not be made
// leaves it none.
KVFOLD_HD int paged_one(const int64_t* slots, int64_t n_places, int s) { return slots && (uint64_t)slots[s] >= (uint64_t)n_places ? s : s + 1; }

// Whether packed token t is one of a sequence's that have a position.  The sequence is the last that begins at t or in front of it, of [s, hi) (the running sums ascend;
// where they do not, some sequence in there).
KVFOLD_HD bool paged_token(const int32_t* cu_new, const int32_t* lens, int s, int hi, int n_tokens, int max_new, int max_len, int t) {
  while (hi - s > 1) {
    const int mid = (int)((unsigned)(s + hi) >> 1);
    if (cu_new[mid] <= t)
      s = mid;
    else
      hi = mid;
  }
  const PagedSeq q = paged_seq(cu_new ? cu_new[s] : s, cu_new ? cu_new[s + 1] : s + 1, lens[s], n_tokens, max_new, max_len);
  const int i = t - q.first;
  return i >= 0 && i < q.n && i >= q.n - q.len;
}

}  // namespace kvfold

#if defined(__HIP__)
#include <hip/hip_runtime.h>

namespace kvfold {

struct AssignParams {
  const int32_t *lens, *n_new, *free_pages, *n_free;
  int32_t *tables, *lens_after, *cu_new, *positions, *n_free_after, *status;
  int64_t* slots;
  int64_t table_stride, n_slots;
  int32_t n_seqs, page_log2, n_pages;
};
hipError_t launch_assign(const AssignParams& p, int n_cu, hipStream_t s);

// The list of a batch's work, made by one workgroup
struct PromptPlanParams {
  const int32_t *lens, *cu_new;
  const int64_t* slots;  // nullptr: nothing is stored
  int64_t all_places;    // of the cache
  int32_t* head;      // [0] items, [1] blocks to merge
  PromptItem* items;  // nullptr: no list is asked for
  int32_t* merges;    // behind them: the first pieces of blocks that have several
  int32_t n_seqs, n_tokens, max_new, max_len, group, unit_rows, max_items, max_merges, n_pieces, n_kv_heads;  // (the two bounds hold for sequences that overlap, too)
  int32_t n_places, n_cu;  // workgroups that the GPU has room for; and with a CU each
  int32_t shortest, step;  // tiles of a piece, at least, and that it is a multiple of
  float cost_once, cost_piece, cost_merge;  // in tiles: of a workgroup besides its tiles, of a piece besides that, of cutting at all
};
struct PAppendParams {
  const void *k, *v;  // [n_tokens][Hkv][d] at token_bytes
  const int32_t *lens, *cu_new;  // of the batch whose packed tokens [first, first + n_tokens) these are; lens = nullptr: the places alone decide
  int32_t n_seqs, all_tokens, max_new, max_len, first;
  void *k_pages, *v_pages;
  const int64_t* slots;
  int64_t token_bytes;
  int64_t n_places;
  int32_t n_tokens, n_kv_heads, row_bytes, page_log2;
};
hipError_t launch_pappend(const PAppendParams& p, const PromptPlanParams& plan, hipStream_t s);

struct PAttnParams {
  const void* q;
  const void *k_new, *v_new;  // nullptr: the new rows are in the pages
  void *k_pages, *v_pages;    // of the layer
  void* out;
  float* lse;
  const int32_t *tables, *lens, *cu_new;
  const int64_t* slots;
  uint32_t* counters;  // zero between steps
  float *part_o, *part_ml;
  const int32_t* list_head;  // prompts
  const PromptItem* items;
  const int32_t* merges;
  int64_t table_stride, q_stride, kv_stride;  // (the latter two in elements)
  int64_t n_places;
  uint64_t page_bytes;  // of K or V of a page
  int32_t n_seqs, n_tokens, max_new, max_len;  // (max_len: also what a row of the tables can name)
  int32_t n_q_heads, n_kv_heads, group, page_log2, n_pages;
  int32_t n_pieces, piece, unit_rows;
  int32_t n_units;   // decode: sequences times KV heads; prompts: items at most
  int32_t n_blocks, n_cu;  // prompts: blocks of rows, at most
  int32_t from_end;  // decode: PagedPlan,
  float shared;      // as here
  float scale_log2e, from_log2, stale;  // its reciprocal, and 2^16 in its units
  FastDiv by_group, by_units, by_kv_heads;
};
hipError_t launch_attn_pdecode(const PAttnParams& p, int head_dim, bool bf16, hipStream_t s);
hipError_t launch_attn_prompt(const PAttnParams& p, int head_dim, bool bf16, int units_per_wave, hipStream_t s);
hipError_t prepare_attn_prompt(int head_dim, bool bf16);
hipError_t prepare_attn_prompt_f32(int head_dim);
hipError_t launch_attn_prompt_f32(const PAttnParams& p, int head_dim, hipStream_t s);
hipError_t launch_pmerge(const PAttnParams& p, int head_dim, bool bf16, hipStream_t s);

// Read-only arguments by scalar loads (nobody writes them while the kernel runs)
template <class T>
using ConstPtr = const __attribute__((address_space(4))) T*;

}  // namespace kvfold
#endif
