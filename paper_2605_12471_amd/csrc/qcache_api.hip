// Host side of the cache held in 8 bits (kvfold_qcache_*): one step = an append kernel where the attention kernel does not append by itself, the
// attention kernel, and a merge where the keys were cut into pieces that do not meet in it.  Stream-ordered; nothing synchronises or allocates after kvfold_qcache_create.
#include <cmath>
#include <new>
#include <vector>

#include "kvfold_host.h"
#include "qcache.h"

using namespace kvfold;

struct kvfold_qcache {
  kvfold_config_t cfg;
  QLayout layout;
  int n_cu;
  float scale;
  unsigned char* store;
  bool owns_store;
  float *ws_o, *ws_ml;  // partial results of pieces
  int64_t ws_rows;
  uint32_t* meet_count;  // zero between steps (meet.h)
  std::vector<QLength> len;

  QRows rows(int layer) const {
    unsigned char* at = store + (size_t)layer * layout.layer;
    QRows r;
    r.codes[0] = at;
    r.codes[1] = at + layout.codes;
    r.scales = reinterpret_cast<float*>(at + 2 * layout.codes);
    r.ring[0] = reinterpret_cast<__bf16*>(at + 2 * layout.codes + layout.scales);
    r.ring[1] = reinterpret_cast<__bf16*>(at + 2 * layout.codes + layout.scales + layout.ring);
    r.blocks = layout.blocks;
    return r;
  }
  size_t bytes() const { return (size_t)cfg.n_layers * layout.layer; }
};

namespace {

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

// Everything but the memory that `c` is in.
void release(kvfold_qcache* c) {
  if (c->owns_store && c->store) (void)hipFree(c->store);
  if (c->ws_o) (void)hipFree(c->ws_o);
  if (c->ws_ml) (void)hipFree(c->ws_ml);
  if (c->meet_count) (void)hipFree(c->meet_count);
}

// Both null, or both set and aligned.
bool angles_ok(const float* cos, const float* sin) { return cos ? sin && aligned16(cos) && aligned16(sin) : !sin; }

hipError_t append(kvfold_qcache* c, int layer, const void* k, const void* v, int64_t token_stride, int64_t head_stride, int64_t n, const float* cos,
                  const float* sin, hipStream_t s) {
  QAppendParams p;
  p.to = c->rows(layer);
  p.rows[0] = static_cast<const __bf16*>(k);
  p.rows[1] = static_cast<const __bf16*>(v);
  p.token_stride = token_stride;
  p.head_stride = head_stride;
  p.len_prev = c->len[(size_t)layer].len;
  p.n = n;
  p.rope_cos = cos;
  p.rope_sin = sin;
  p.n_kv_heads = c->cfg.n_kv_heads;
  return launch_qappend(p, c->cfg.head_dim, s);
}

}  // namespace

extern "C" {

size_t kvfold_qcache_bytes_required(const kvfold_config_t* cfg) {
  return validate_qconfig(cfg) == KVFOLD_OK ? (size_t)cfg->n_layers * q_layout(*cfg).layer : 0;
}

int kvfold_qcache_create(const kvfold_config_t* cfg, kvfold_qcache_t** out_cache) {
  if (!out_cache) return KVFOLD_ERR_INVALID_ARG;
  *out_cache = nullptr;
  const int rc = validate_qconfig(cfg);
  if (rc != KVFOLD_OK) return rc;
  const size_t need = kvfold_qcache_bytes_required(cfg);
  if (cfg->kv_buffer && cfg->kv_buffer_bytes < need) return KVFOLD_ERR_OOM;

  int n_dev = 0;
  hipError_t e = hipGetDeviceCount(&n_dev);
  if (e != hipSuccess) return hip_fail(e);
  if (cfg->device >= n_dev || cfg->device >= kMaxDevices) return KVFOLD_ERR_INVALID_ARG;
  DeviceGuard guard(cfg->device);
  if (guard.err != hipSuccess) return hip_fail(guard.err);

  kvfold_qcache* c = new (std::nothrow) kvfold_qcache();
  if (!c) return KVFOLD_ERR_OOM;
  try {
    c->len.resize((size_t)cfg->n_layers);
  } catch (...) {
    delete c;
    return KVFOLD_ERR_OOM;
  }
  c->cfg = *cfg;
  c->layout = q_layout(*cfg);
  c->scale = cfg->softmax_scale > 0.f ? cfg->softmax_scale : 1.0f / std::sqrt((float)cfg->head_dim);
  hipDeviceProp_t prop;
  e = hipGetDeviceProperties(&prop, cfg->device);
  c->n_cu = e == hipSuccess && prop.multiProcessorCount > 0 ? prop.multiProcessorCount : 256;
  auto take = [&](size_t bytes) -> void* {
    void* p = nullptr;
    if (e == hipSuccess) e = hipMalloc(&p, bytes);
    return e == hipSuccess ? p : nullptr;
  };
  c->owns_store = !cfg->kv_buffer;
  c->store = static_cast<unsigned char*>(cfg->kv_buffer ? cfg->kv_buffer : take(need));
  c->ws_rows = workspace_rows(cfg);
  if (c->ws_rows > 0) {
    c->ws_o = static_cast<float*>(take((size_t)c->ws_rows * cfg->head_dim * sizeof(float)));
    c->ws_ml = static_cast<float*>(take((size_t)c->ws_rows * 2 * sizeof(float)));
    if (cfg->n_kv_heads <= kMeetUnits) {
      const size_t counters = (size_t)cfg->n_kv_heads * kMeetStride * sizeof(uint32_t);
      c->meet_count = static_cast<uint32_t*>(take(counters));
      if (e == hipSuccess) e = clear_device(c->meet_count, counters);
    }
  }
  if (e != hipSuccess) {
    release(c);
    delete c;
    return hip_fail(e);
  }
  *out_cache = c;
  return KVFOLD_OK;
}

int kvfold_qcache_destroy(kvfold_qcache_t* c) {
  if (!c) return KVFOLD_OK;
  int rc = KVFOLD_OK;
  {
    DeviceGuard guard(c->cfg.device);
    if (guard.err != hipSuccess) rc = hip_fail(guard.err);
    const hipError_t e = hipDeviceSynchronize();
    if (e != hipSuccess) rc = hip_fail(e);
    release(c);
  }
  delete c;
  return rc;
}

int64_t kvfold_qcache_length(const kvfold_qcache_t* c, int layer) {
  if (!c) return KVFOLD_ERR_INVALID_ARG;
  if (layer < 0 || layer >= c->cfg.n_layers) return KVFOLD_ERR_BAD_LAYER;
  return c->len[(size_t)layer].len;
}

int kvfold_qcache_truncate(kvfold_qcache_t* c, int layer, int64_t new_len) {
  if (!c || new_len < 0) return KVFOLD_ERR_INVALID_ARG;
  if (layer < -1 || layer >= c->cfg.n_layers) return KVFOLD_ERR_BAD_LAYER;
  const size_t from = layer < 0 ? 0 : (size_t)layer, to = layer < 0 ? c->len.size() : from + 1;
  for (size_t i = from; i < to; ++i)
    if (!c->len[i].can_truncate(new_len)) return KVFOLD_ERR_POSITION;
  for (size_t i = from; i < to; ++i) c->len[i].truncate(new_len);
  return KVFOLD_OK;
}

int kvfold_qcache_append(kvfold_qcache_t* c, int layer, const void* k, const void* v, int64_t token_stride, int64_t head_stride, int64_t n_tokens,
                         int64_t pos_offset, const float* rope_cos, const float* rope_sin, void* stream) {
  if (!c || n_tokens < 0 || (n_tokens > 0 && (!k || !v))) return KVFOLD_ERR_INVALID_ARG;
  const kvfold_config_t& f = c->cfg;
  if (layer < 0 || layer >= f.n_layers) return KVFOLD_ERR_BAD_LAYER;
  if (!angles_ok(rope_cos, rope_sin) || !aligned16(k) || !aligned16(v) || token_stride < 0 || head_stride < 0 || (token_stride | head_stride) & 7)
    return KVFOLD_ERR_INVALID_ARG;
  QLength& len = c->len[(size_t)layer];
  if (pos_offset != len.len) return KVFOLD_ERR_POSITION;
  if (n_tokens > f.capacity_tokens - len.len) return KVFOLD_ERR_CAPACITY;
  if (n_tokens == 0) return KVFOLD_OK;
  const size_t extent = ((size_t)(n_tokens - 1) * (size_t)token_stride + (size_t)(f.n_kv_heads - 1) * (size_t)head_stride + (size_t)f.head_dim) * 2;
  if (!apart(c->store, c->bytes(), k, extent) || !apart(c->store, c->bytes(), v, extent)) return KVFOLD_ERR_INVALID_ARG;
  DeviceGuard guard(f.device);
  if (guard.err != hipSuccess) return hip_fail(guard.err);
  const hipError_t e = append(c, layer, k, v, token_stride, head_stride, n_tokens, rope_cos, rope_sin, static_cast<hipStream_t>(stream));
  if (e != hipSuccess) return hip_fail(e);
  len.append(n_tokens);
  return KVFOLD_OK;
}

int kvfold_qcache_step(kvfold_qcache_t* c, int layer, const void* q, const void* k_new, const void* v_new, int32_t n_tokens, int64_t pos_offset,
                       const float* rope_cos, const float* rope_sin, void* out, float* lse, void* stream) {
  if (!c || !q || !k_new || !v_new || !out) return KVFOLD_ERR_INVALID_ARG;
  const kvfold_config_t& f = c->cfg;
  if (layer < 0 || layer >= f.n_layers) return KVFOLD_ERR_BAD_LAYER;
  if (n_tokens < 1 || n_tokens > f.chunk_tokens || !angles_ok(rope_cos, rope_sin)) return KVFOLD_ERR_INVALID_ARG;
  QLength& len = c->len[(size_t)layer];
  if (pos_offset != len.len) return KVFOLD_ERR_POSITION;
  if (len.len + n_tokens > f.capacity_tokens) return KVFOLD_ERR_CAPACITY;
  if (!aligned16(q) || !aligned16(k_new) || !aligned16(v_new) || !aligned16(out) || reinterpret_cast<uintptr_t>(lse) & 3) return KVFOLD_ERR_INVALID_ARG;
  // Results are stored while other rows' queries and angles are still read: on the rows' own queries they may lie, nowhere else there.
  const size_t wide = (size_t)n_tokens * f.n_q_heads * f.head_dim * 2, sums = (size_t)n_tokens * f.n_q_heads * sizeof(float);
  const size_t angles = (size_t)n_tokens * (f.head_dim / 2) * sizeof(float);
  bool ok = out == q || apart(q, wide, out, wide);
  if (lse) ok = ok && apart(q, wide, lse, sums) && apart(out, wide, lse, sums);
  for (const float* a : {rope_cos, rope_sin})
    if (a) ok = ok && apart(a, angles, out, wide) && (!lse || apart(a, angles, lse, sums));
  ok = ok && apart(c->store, c->bytes(), out, wide) && (!lse || apart(c->store, c->bytes(), lse, sums));
  // (and the cache is written while the inputs are read)
  const size_t narrow = (size_t)n_tokens * f.n_kv_heads * f.head_dim * 2;
  ok = ok && apart(c->store, c->bytes(), q, wide) && apart(c->store, c->bytes(), k_new, narrow) && apart(c->store, c->bytes(), v_new, narrow);
  if (!ok) return KVFOLD_ERR_INVALID_ARG;

  DeviceGuard guard(f.device);
  if (guard.err != hipSuccess) return hip_fail(guard.err);
  hipStream_t s = static_cast<hipStream_t>(stream);
  const QPlan pl = make_qplan(f, c->n_cu, c->ws_rows, n_tokens, len.len + n_tokens);

  QAttnParams p;
  AttnParams& a = p.a;
  a = AttnParams{};
  a.q = q;
  a.out = out;
  a.lse = lse;
  a.part_o = c->ws_o;
  a.part_ml = c->ws_ml;
  a.n_tokens = n_tokens;
  a.n_q_heads = f.n_q_heads;
  a.n_kv_heads = f.n_kv_heads;
  a.group = f.n_q_heads / f.n_kv_heads;
  a.capacity = f.capacity_tokens;
  a.len_prev = len.len;
  a.n_splits = pl.n_splits;
  a.tiles_per_split = pl.blocks_per_split;
  a.units_per_head = pl.units_per_head;
  a.wgs_per_head = pl.wgs_per_head;
  a.n_wgs = pl.n_wgs;
  a.scale_log2e = c->scale * 1.4426950408889634f;
  a.rope_cos = rope_cos;
  a.rope_sin = rope_sin;
  const bool meet = pl.meet && c->meet_count;
  a.meet_count = meet ? c->meet_count : nullptr;
  finish_attn_params(a, pl.decode);
  p.c = c->rows(layer);

  // Rows that fill no block are appended by the attention kernel, where one workgroup alone reads a head's last block and its results lie apart from them:
  // these are stored while other heads' rows are still read.  37 tokens on 32K keys 47.5 us for 51, 32 on 4187 24.1 for 27.
  bool inside = pl.wgs_per_head == 1 && len.len / kQBlock == (len.len + n_tokens) / kQBlock;
  for (const void* rows : {k_new, v_new}) inside = inside && apart(rows, narrow, out, wide) && (!lse || apart(rows, narrow, lse, sums));
  p.k_new = inside ? static_cast<const __bf16*>(k_new) : nullptr;
  p.v_new = inside ? static_cast<const __bf16*>(v_new) : nullptr;
  const int64_t row = (int64_t)f.n_kv_heads * f.head_dim;
  hipError_t e = inside ? hipSuccess : append(c, layer, k_new, v_new, row, f.head_dim, n_tokens, rope_cos, rope_sin, s);
  if (e != hipSuccess) return hip_fail(e);
  e = pl.decode ? launch_attn_qdecode(p, f.head_dim, s) : launch_attn_q(p, f.head_dim, pl.waves_per_wg, s);
  if (e != hipSuccess) return hip_fail(e);
  if (pl.n_splits > 1 && !meet) {
    CombineParams cp;
    cp.part_o = c->ws_o;
    cp.part_ml = c->ws_ml;
    cp.out = out;
    cp.lse = lse;
    cp.n_rows = n_tokens * f.n_q_heads;
    cp.n_tokens = n_tokens;
    cp.n_q_heads = f.n_q_heads;
    cp.head_dim = f.head_dim;
    cp.n_splits = pl.n_splits;
    cp.out_is_bf16 = 1;
    e = launch_combine(cp, s);
    if (e != hipSuccess) return hip_fail(e);
  }
  len.append(n_tokens);
  return KVFOLD_OK;
}

int kvfold_qcache_read(kvfold_qcache_t* c, int layer, int64_t first, int64_t n_tokens, float* k_out, float* v_out, void* stream) {
  if (!c || first < 0 || n_tokens < 0 || !aligned16(k_out) || !aligned16(v_out)) return KVFOLD_ERR_INVALID_ARG;
  if (layer < 0 || layer >= c->cfg.n_layers) return KVFOLD_ERR_BAD_LAYER;
  const int64_t len = c->len[(size_t)layer].len;
  if (first > len || n_tokens > len - first) return KVFOLD_ERR_POSITION;
  if (n_tokens == 0 || (!k_out && !v_out)) return KVFOLD_OK;
  const size_t bytes = (size_t)n_tokens * c->cfg.n_kv_heads * c->cfg.head_dim * sizeof(float);
  if ((k_out && !apart(c->store, c->bytes(), k_out, bytes)) || (v_out && !apart(c->store, c->bytes(), v_out, bytes)) ||
      (k_out && v_out && !apart(k_out, bytes, v_out, bytes)))
    return KVFOLD_ERR_INVALID_ARG;
  DeviceGuard guard(c->cfg.device);
  if (guard.err != hipSuccess) return hip_fail(guard.err);
  QReadParams p;
  p.from = c->rows(layer);
  p.out[0] = k_out;
  p.out[1] = v_out;
  p.first = first;
  p.n = n_tokens;
  p.len = len;
  p.n_kv_heads = c->cfg.n_kv_heads;
  const hipError_t e = launch_qread(p, c->cfg.head_dim, static_cast<hipStream_t>(stream));
  return e == hipSuccess ? KVFOLD_OK : hip_fail(e);
}

}  // extern "C"
