// Host decisions of the cache in pages.  No HIP in this file.
#include <algorithm>
#include <cmath>

#include "pcache.h"

namespace kvfold {

int validate_pconfig(const kvfold_pcache_config_t* c) {
  if (!c || c->struct_size != sizeof(kvfold_pcache_config_t)) return KVFOLD_ERR_INVALID_ARG;
  if (c->n_layers < 1 || c->n_q_heads < 1 || c->n_kv_heads < 1 || c->n_pages < 1 || c->page_tokens < 1 || c->device < 0 || !(c->softmax_scale >= 0.f) ||
      !std::isfinite(c->softmax_scale))
    return KVFOLD_ERR_INVALID_ARG;
  if (c->kv_buffer && (reinterpret_cast<uintptr_t>(c->kv_buffer) & 255)) return KVFOLD_ERR_INVALID_ARG;
  if (elem_size(c->dtype) == 0) return KVFOLD_ERR_UNSUPPORTED;
  if (c->head_dim != 64 && c->head_dim != 128) return KVFOLD_ERR_UNSUPPORTED;
  if (c->n_q_heads % c->n_kv_heads || c->n_kv_heads > 32767 || c->n_q_heads > 1 << 20) return KVFOLD_ERR_UNSUPPORTED;
  if (c->page_tokens < 16 || c->page_tokens > 256 || (c->page_tokens & (c->page_tokens - 1))) return KVFOLD_ERR_UNSUPPORTED;
  if ((int64_t)c->n_pages * c->page_tokens >= (int64_t)1 << 31) return KVFOLD_ERR_UNSUPPORTED;
  // (all bytes in 64 bits: n_layers < 2^31 times a page pool's at most 2^31 * 2^15 * 2^9 * 2)
  if ((double)c->n_layers * (double)pcache_layer_bytes(*c) > 9e18) return KVFOLD_ERR_UNSUPPORTED;
  return KVFOLD_OK;
}

size_t pcache_layer_bytes(const kvfold_pcache_config_t& c) {
  return 2u * (size_t)c.n_pages * (size_t)c.n_kv_heads * (size_t)c.page_tokens * (size_t)c.head_dim * (size_t)elem_size(c.dtype);
}

int validate_batch(const kvfold_pcache_config_t& c, const kvfold_batch_t* b) {
  if (!b || b->struct_size != sizeof(kvfold_batch_t)) return KVFOLD_ERR_INVALID_ARG;
  if (b->n_seqs < 0 || b->n_tokens < 0 || b->max_new < 1 || b->max_len < 1 || b->table_stride < 1 || b->q_stride < 0 || b->kv_stride < 0)
    return KVFOLD_ERR_INVALID_ARG;
  const int64_t unit = 16 / elem_size(c.dtype), wide = (int64_t)c.n_q_heads * c.head_dim, narrow = (int64_t)c.n_kv_heads * c.head_dim;
  if (b->q_stride % unit || b->kv_stride % unit || (b->q_stride && b->q_stride < wide) || (b->kv_stride && b->kv_stride < narrow)) return KVFOLD_ERR_INVALID_ARG;
  if (b->max_len > (int64_t)1 << 30 || b->table_stride >= (int64_t)1 << 31 || (int64_t)b->n_tokens * c.n_q_heads > (int64_t)1 << 28 || b->n_seqs > 1 << 20 ||
      (int64_t)b->n_seqs * c.n_kv_heads > (int64_t)1 << 23 || b->kv_stride > (int64_t)1 << 31 || (b->q_stride >> 3) > ((int64_t)1 << 31) / std::max(b->n_tokens, 1))
    return KVFOLD_ERR_UNSUPPORTED;
  return KVFOLD_OK;
}

PagedPlan make_pplan(const kvfold_pcache_config_t& c, int n_cu, const kvfold_batch_t& b) {
  const int G = c.n_q_heads / c.n_kv_heads;
  const int64_t max_new = std::min<int64_t>(b.max_new, std::max(b.n_tokens, 1)), len = std::min(b.max_len, b.table_stride * c.page_tokens);
  const int64_t steps = (len + 127) / 128;  // (pieces are whole steps of 128 keys)
  PagedPlan pl{};
  pl.decode = max_new * G <= 16;
  int64_t pieces;
  const int64_t units = std::max<int64_t>(1, (int64_t)b.n_seqs * c.n_kv_heads);
  if (pl.decode) {
    pl.unit_rows = (int)max_new * G;
    pl.units_per_wave = 1;
    // (a bound wider than the lengths makes pieces longer: one sequence of 4000 keys under a max_len of 4096 10.1 us, of 131072 25.8)
    // Where pieces are many the whole ones come first, else the way to the first keys counts (attn_pdecode.hip)
    pl.from_end = units >= n_cu;
    pieces = std::max((n_cu + units - 1) / units, (len + kPagedLongestPiece - 1) / kPagedLongestPiece);
    auto bounded = [&](int64_t n) { return std::max<int64_t>(1, std::min<int64_t>({n, kPagedMaxRows / (units * pl.unit_rows), steps, kPagedMaxPieces})); };
    // Few sequences of unlike lengths: a long one in pieces of a CU's share of all keys, which the device finds, instead of those that it would have among equals (16 sequences of 10 to
    // 16000 keys, 32 heads on 8, 41.7 -> 24.2 us, of 4 new tokens 46 -> 29.5; fp32 of 100 to 8000 84 -> 37; equal ones within 3 %, 12 of 1000 to 3000 19.4 -> 23.7).
    const int64_t more = bounded(std::min<int64_t>((len + 255) / 256, kPagedMostWgs / units));
    pieces = bounded(pieces);
    if (!pl.from_end && b.n_seqs > 1 && more > pieces) {
      pieces = more;
      pl.shared = (float)c.n_kv_heads / (float)n_cu;
    }
    pl.piece = (int)((steps + pieces - 1) / pieces) * 128;
    pl.n_pieces = paged_pieces((int)len, pl.piece);
    pl.rows = pl.n_pieces > 1 ? units * pl.n_pieces * pl.unit_rows : 0;
  } else {
    const int64_t rows_a_seq = (int64_t)b.n_tokens * G / std::max(b.n_seqs, 1);
    const bool bf16 = c.dtype == KVFOLD_BF16;
    // (the average of all sequences, those without new tokens among them, and max_len: what the host knows.  One prompt of 4096 tokens 151 us, beside 255 sequences of one new token
    // each, with one unit a wavefront, 243; 1000 tokens under a max_len of 1000 32.7, under 4096, with two, 40.0)
    pl.units_per_wave = bf16 && rows_a_seq > 128 && len > 1024 ? 2 : 1;
    pl.unit_rows = kUnitsPerWg * kRowsPerUnit * pl.units_per_wave;
    // Blocks of rows: a sequence's last one is filled up.  Pieces: no shorter than a place's share of all tiles (pcache_rows.hip), so that there are at most as many more
    // as there are places, and those that the device's estimate of the tiles leaves out.
    pl.blocks = (int64_t)b.n_tokens * G / pl.unit_rows + std::min<int64_t>(b.n_seqs, b.n_tokens);
    pl.places = pl.units_per_wave == 2 ? n_cu : 2 * n_cu;
    // (a tile of bf16, two units a wavefront: 1.6 us; one, and two workgroups a CU: 2.8; of fp32, 64 wide, two workgroups a CU: 7)
    // With what two units cost for one, too, short chunks stayed whole: 64 tokens on 900 keys 33.7 us, cut 21.9 (32 sequences of 20 to 60 on 20 to 900, cut or not, 38.6 and 39.9).
    const bool two = pl.units_per_wave == 2;
    pl.step = two ? 2 : 1;
    pl.shortest = bf16 ? 4 : 1;
    pl.cost_once = two ? 5 : bf16 ? 2 : 1;
    pl.cost_piece = two ? 8 : bf16 ? 4 : 0.5f;
    pl.cost_merge = two ? 8 : bf16 ? 1.5f : 1;
    const int64_t rows = (int64_t)b.n_tokens * c.n_q_heads;
    pieces = std::min<int64_t>({kPromptMaxPieces, steps, kPagedMaxRows / std::max<int64_t>(rows, 1)});
    // Whole prompts that fill the GPU are left in one piece: in bf16 the merge costs more than is won (1000 tokens, 32 heads on 8: 33.8 us, in pieces 38), in fp32 less (147, 114).
    if (len <= 2 * max_new && pl.blocks * c.n_kv_heads >= (bf16 ? pl.places / 2 : 2 * pl.places)) pieces = 1;
    pl.n_pieces = (int)std::max<int64_t>(1, pieces);
    pl.items = pl.blocks;
    if (pl.n_pieces > 1) pl.items += std::min<int64_t>(pl.places / c.n_kv_heads + pl.blocks / 8 + 8, pl.blocks * (pl.n_pieces - 1));
    pl.rows = pl.n_pieces > 1 ? rows * pl.n_pieces : 0;
    pl.list = (kPromptHead + (size_t)pl.items * sizeof(PromptItem) + (size_t)pl.blocks * sizeof(int32_t) + 255) / 256 * 256;
  }
  pl.counters = ((size_t)units * kPagedMeetStride * sizeof(uint32_t) + 255) / 256 * 256;  // (always there: steps of either kind share a workspace)
  pl.bytes = pl.counters + pl.list + (((size_t)pl.rows * (size_t)(c.head_dim + 2) * sizeof(float)) + 255) / 256 * 256;
  return pl;
}

}  // namespace kvfold

using namespace kvfold;

extern "C" size_t kvfold_pcache_bytes_required(const kvfold_pcache_config_t* cfg) {
  return validate_pconfig(cfg) == KVFOLD_OK ? (size_t)cfg->n_layers * pcache_layer_bytes(*cfg) : 0;
}
