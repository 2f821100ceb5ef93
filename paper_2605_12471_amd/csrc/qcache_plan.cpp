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

// Pieces of the keys until the chip is full: two workgroups a CU, as both kernels are compiled for.
QPlan make_qplan(const kvfold_config_t& c, int n_cu, int64_t ws_rows, int n_tokens, int64_t len_after) {
  const int G = c.n_q_heads / c.n_kv_heads, blocks = (int)((len_after + kQBlock - 1) / kQBlock);
  const int64_t rows = (int64_t)n_tokens * G;
  QPlan pl{};
  pl.decode = rows <= 16;
  pl.units_per_head = units_of_head(n_tokens, G);
  pl.units_per_wave = 1;
  pl.wgs_per_head = pl.decode ? 1 : (pl.units_per_head + kUnitsPerWg * pl.units_per_wave - 1) / (kUnitsPerWg * pl.units_per_wave);
  const int64_t per_split = (int64_t)c.n_kv_heads * pl.wgs_per_head;
  int64_t splits = 2 * (int64_t)n_cu / per_split;
  splits = std::min<int64_t>(splits, pl.decode ? (blocks + 3) / 4 : blocks);  // (decoding deals a piece's blocks to four wavefronts)
  splits = std::min<int64_t>(splits, kMaxSplits);
  splits = std::min(splits, ws_rows / ((int64_t)n_tokens * c.n_q_heads));
  splits = std::max<int64_t>(splits, 1);
  pl.blocks_per_split = (int)((blocks + splits - 1) / splits);
  pl.n_splits = (blocks + pl.blocks_per_split - 1) / pl.blocks_per_split;
  pl.n_wgs = (int)(per_split * pl.n_splits);
  return pl;
}

}  // namespace kvfold
