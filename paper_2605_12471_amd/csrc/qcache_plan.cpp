// Host decisions of the cache held in 8 bits.  No HIP in this file.
#include <algorithm>

#include "kvfold_plan.h"
#include "qcache.h"

namespace kvfold {

int validate_qconfig(const kvfold_config_t* c) {
  const int rc = validate_config(c);
  if (rc != KVFOLD_OK) return rc;
  return c->dtype == KVFOLD_BF16 ? KVFOLD_OK : KVFOLD_ERR_UNSUPPORTED;
}

// Decoding: a wavefront takes a block at a time, so that a piece of 4 r blocks takes r turns, and a workgroup has a CU to itself.  One token, 32 heads on 8,
// captured steps.  Up to eight blocks are one piece's: 300 keys 6.7 us, two pieces 7.5.  Beyond, the fewest pieces with which there are as few turns as a
// workgroup for every CU would take: 4187 keys, 17 pieces of four blocks 7.6, 8 pieces 9.8, 31 of three 7.8; 16K, 32 of eight 9.8, 28 of nine 10.9, 16 12.4; 40K,
// 32 of twenty 18.6, 16 21.7.  Above eight turns memory is what counts, and three quarters of the CUs ask it for no more than it gives: 65K to 131K keys,
// five lengths, both widths, 24 pieces 0.96 of the time of 32 (128K keys 45 to 46 us, 32 pieces 50).
static int64_t decode_splits(int blocks, int64_t per_cu) {
  if (blocks <= 8) return 1;
  const int64_t turns = (blocks + 4 * per_cu - 1) / (4 * per_cu);
  return turns > 8 ? std::max<int64_t>(1, per_cu * 3 / 4) : (blocks + 4 * turns - 1) / (4 * turns);
}

QPlan make_qplan(const kvfold_config_t& c, int n_cu, int64_t ws_rows, int n_tokens, int64_t len_after) {
  const int G = c.n_q_heads / c.n_kv_heads, blocks = (int)((len_after + kQBlock - 1) / kQBlock);
  const int64_t rows = (int64_t)n_tokens * G;
  QPlan pl{};
  pl.decode = rows <= 16;
  pl.units_per_head = units_of_head(n_tokens, G);
  // Chunks: eight wavefronts share what is widened, four come sooner to their end and leave fewer pieces to merge.  64 wide, eight where workgroups of
  // four on every CU would have more than 32 blocks each: 32 heads on 8, 1000 tokens on 8K keys (141 blocks) 103 us, in fours 111 to 122, 100 on 16K (32.3) 35.3, 38.4; 512 on
  // 2048 (20) 36.1, in fours 33.7, on 512 (8) 28.3, 24.3; 4 heads on 1, 256 on 4096 (8.5) 22.0, 18.9.  Up to four units the other four wavefronts only widen:
  // 20 tokens on 32K 27.0, in fours 28.3.  128 wide a workgroup of four has no registers for its share.
  const int64_t blocks_of_fours = (int64_t)c.n_kv_heads * ((pl.units_per_head + 3) / 4) * blocks;
  pl.waves_per_wg = c.head_dim == 64 && pl.units_per_head > 4 && blocks_of_fours <= (int64_t)32 * n_cu ? 4 : 8;
  pl.wgs_per_head = pl.decode ? 1 : (pl.units_per_head + pl.waves_per_wg - 1) / pl.waves_per_wg;
  const int64_t per_split = (int64_t)c.n_kv_heads * pl.wgs_per_head;
  int64_t splits = pl.decode ? decode_splits(blocks, std::min<int64_t>(std::max<int64_t>(1, n_cu / c.n_kv_heads), kMaxSplits)) : std::min<int64_t>((int64_t)n_cu / per_split, blocks);
  splits = std::min<int64_t>(splits, kMaxSplits);
  splits = std::min(splits, ws_rows / ((int64_t)n_tokens * c.n_q_heads));
  splits = std::max<int64_t>(splits, 1);
  pl.blocks_per_split = (int)((blocks + splits - 1) / splits);
  pl.n_splits = (blocks + pl.blocks_per_split - 1) / pl.blocks_per_split;
  pl.n_wgs = (int)(per_split * pl.n_splits);
  // A row's pieces meet in the last one's workgroup, a row a wavefront at a time: up to two of them, and as many pieces as a wavefront has registers
  // for.  Four tokens (16 rows a KV head), 4187 keys 12.1 us, by the merge kernel 10.8; 28 heads on 4, one token (seven rows) 8.8 both ways.
  pl.meet = pl.decode && rows <= 8 && pl.n_splits > 1 && pl.n_splits <= kMeetSplits;
  return pl;
}

}  // namespace kvfold
