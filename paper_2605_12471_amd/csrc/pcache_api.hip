// Host side of the cache in pages (kvfold_pcache_*).  A step is one launch where every sequence has few rows, else the rows' way to their places, the attention
// kernel, and a merge where the keys were cut into pieces.  Stream-ordered; nothing synchronises or allocates after kvfold_pcache_create.
#include <cmath>
#include <new>

#include "kvfold_host.h"
#include "pcache.h"

using namespace kvfold;

struct kvfold_pcache {
  kvfold_pcache_config_t cfg;
  int n_cu, page_log2;
  float scale;
  unsigned char* store;
  bool owns_store;

  size_t bytes() const { return (size_t)cfg.n_layers * pcache_layer_bytes(cfg); }
  unsigned char* rows(int layer, bool v) const { return store + (size_t)layer * pcache_layer_bytes(cfg) + (v ? pcache_layer_bytes(cfg) / 2 : 0); }
  int es() const { return elem_size(cfg.dtype); }
  int64_t places() const { return (int64_t)cfg.n_pages * cfg.page_tokens; }
};

namespace {

bool aligned(const void* p, size_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

struct Range {
  const void* at;
  size_t bytes;
};
bool all_apart(const Range& a, const Range* others, int n) {
  for (int i = 0; i < n; ++i)
    if (a.at && a.bytes && others[i].at && others[i].bytes && !apart(a.at, a.bytes, others[i].at, others[i].bytes)) return false;
  return true;
}

// Bytes of n tokens' rows of `heads` heads at `stride` elements
size_t extent(int64_t n, int64_t stride, int64_t heads, int64_t d, int es) { return n < 1 ? 0 : ((size_t)(n - 1) * (size_t)stride + (size_t)(heads * d)) * (size_t)es; }

// Rows to their places; `plan`: of the step that they are part of, whose sequences they have to belong to (lens = nullptr: of none)
hipError_t append_rows(const kvfold_pcache* c, int layer, const void* k, const void* v, int64_t kv_stride, const int64_t* slots, int32_t n, const PromptPlanParams& plan,
                       hipStream_t s) {
  PAppendParams p;
  p.lens = plan.lens;
  p.cu_new = plan.cu_new;
  p.n_seqs = plan.n_seqs;
  p.all_tokens = plan.n_tokens;
  p.max_new = plan.max_new;
  p.max_len = plan.max_len;
  p.first = 0;
  p.k = k;
  p.v = v;
  p.k_pages = c->rows(layer, false);
  p.v_pages = c->rows(layer, true);
  p.slots = slots;
  p.token_bytes = kv_stride * c->es();
  p.n_places = c->places();
  p.n_tokens = n;
  p.n_kv_heads = c->cfg.n_kv_heads;
  p.row_bytes = c->cfg.head_dim * c->es();
  p.page_log2 = c->page_log2;
  return launch_pappend(p, plan, s);
}

}  // namespace

extern "C" {

int kvfold_pcache_create(const kvfold_pcache_config_t* cfg, kvfold_pcache_t** out_cache) {
  if (!out_cache) return KVFOLD_ERR_INVALID_ARG;
  *out_cache = nullptr;
  const int rc = validate_pconfig(cfg);
  if (rc != KVFOLD_OK) return rc;
  const size_t need = kvfold_pcache_bytes_required(cfg);
  if (cfg->kv_buffer && cfg->kv_buffer_bytes < need) return KVFOLD_ERR_OOM;
  int n_dev = 0;
  hipError_t e = hipGetDeviceCount(&n_dev);
  if (e != hipSuccess) return hip_fail(e);
  if (cfg->device >= n_dev || cfg->device >= kMaxDevices) return KVFOLD_ERR_INVALID_ARG;
  DeviceGuard guard(cfg->device);
  if (guard.err != hipSuccess) return hip_fail(guard.err);
  kvfold_pcache* c = new (std::nothrow) kvfold_pcache();
  if (!c) return KVFOLD_ERR_OOM;
  c->cfg = *cfg;
  while ((1 << c->page_log2) < cfg->page_tokens) ++c->page_log2;
  c->scale = cfg->softmax_scale > 0.f ? cfg->softmax_scale : 1.0f / std::sqrt((float)cfg->head_dim);
  hipDeviceProp_t prop;
  e = hipGetDeviceProperties(&prop, cfg->device);
  c->n_cu = e == hipSuccess && prop.multiProcessorCount > 0 ? prop.multiProcessorCount : 256;
  if (e == hipSuccess) e = prepare_attn_prompt(cfg->head_dim, cfg->dtype == KVFOLD_BF16);
  c->owns_store = !cfg->kv_buffer;
  if (cfg->kv_buffer) {
    c->store = static_cast<unsigned char*>(cfg->kv_buffer);
  } else if (e == hipSuccess) {
    void* store = nullptr;
    e = hipMalloc(&store, need);
    c->store = static_cast<unsigned char*>(store);
  }
  if (e != hipSuccess) {
    delete c;
    return hip_fail(e);
  }
  *out_cache = c;
  return KVFOLD_OK;
}

int kvfold_pcache_destroy(kvfold_pcache_t* c) {
  if (!c) return KVFOLD_OK;
  int rc = KVFOLD_OK;
  {
    DeviceGuard guard(c->cfg.device);
    if (guard.err != hipSuccess) rc = hip_fail(guard.err);
    hipError_t e = hipDeviceSynchronize();
    if (e != hipSuccess) rc = hip_fail(e);
    if (c->owns_store && c->store) e = hipFree(c->store);
    if (e != hipSuccess) rc = hip_fail(e);
  }
  delete c;
  return rc;
}

int kvfold_pcache_view(const kvfold_pcache_t* c, int layer, void** k_dev, void** v_dev) {
  if (!c) return KVFOLD_ERR_INVALID_ARG;
  if (layer < 0 || layer >= c->cfg.n_layers) return KVFOLD_ERR_BAD_LAYER;
  if (k_dev) *k_dev = c->rows(layer, false);
  if (v_dev) *v_dev = c->rows(layer, true);
  return KVFOLD_OK;
}

int kvfold_pcache_assign(const kvfold_pcache_t* c, int32_t n_seqs, const int32_t* lens, const int32_t* n_new, const int32_t* free_pages, const int32_t* n_free,
                         int32_t* tables, int64_t table_stride, int32_t* lens_after, int32_t* cu_new, int64_t* slots, int32_t* positions, int64_t n_slots,
                         int32_t* n_free_after, int32_t* status, void* stream) {
  if (!c || n_seqs < 0 || n_slots < 0 || table_stride < 1 || !free_pages || !n_free || !cu_new || !n_free_after || !status) return KVFOLD_ERR_INVALID_ARG;
  if ((n_seqs > 0 && (!lens || !n_new || !tables || !lens_after)) || (n_slots > 0 && !slots)) return KVFOLD_ERR_INVALID_ARG;
  if (n_seqs > 1 << 20 || n_slots >= (int64_t)1 << 31 || table_stride >= (int64_t)1 << 31) return KVFOLD_ERR_UNSUPPORTED;
  for (const void* at : {(const void*)lens, (const void*)n_new, (const void*)free_pages, (const void*)n_free, (const void*)tables, (const void*)lens_after, (const void*)cu_new,
                         (const void*)positions, (const void*)n_free_after, (const void*)status})
    if (!aligned(at, 4)) return KVFOLD_ERR_INVALID_ARG;
  if (!aligned(slots, 8)) return KVFOLD_ERR_INVALID_ARG;
  const size_t seqs = (size_t)n_seqs * 4;
  const Range all[] = {{tables, (size_t)n_seqs * (size_t)table_stride * 4}, {lens_after, seqs}, {cu_new, seqs + 4}, {slots, (size_t)n_slots * 8},
                       {positions, positions ? (size_t)n_slots * 4 : 0}, {n_free_after, 4}, {status, 4},  // results, then inputs
                       {lens, seqs}, {n_new, seqs}, {free_pages, (size_t)c->cfg.n_pages * 4}, {n_free, 4}, {c->store, c->bytes()}};
  for (int i = 0; i < 7; ++i)
    if (!all_apart(all[i], all + i + 1, 11 - i)) return KVFOLD_ERR_INVALID_ARG;
  DeviceGuard guard(c->cfg.device);
  if (guard.err != hipSuccess) return hip_fail(guard.err);
  AssignParams p;
  p.lens = lens;
  p.n_new = n_new;
  p.free_pages = free_pages;
  p.n_free = n_free;
  p.tables = tables;
  p.lens_after = lens_after;
  p.cu_new = cu_new;
  p.positions = positions;
  p.n_free_after = n_free_after;
  p.status = status;
  p.slots = slots;
  p.table_stride = table_stride;
  p.n_slots = n_slots;
  p.n_seqs = n_seqs;
  p.page_log2 = c->page_log2;
  p.n_pages = c->cfg.n_pages;
  const hipError_t e = launch_assign(p, c->n_cu, static_cast<hipStream_t>(stream));
  return e == hipSuccess ? KVFOLD_OK : hip_fail(e);
}

size_t kvfold_pcache_workspace_bytes(const kvfold_pcache_t* c, const kvfold_batch_t* batch) {
  if (!c || validate_batch(c->cfg, batch) != KVFOLD_OK) return 0;
  return make_pplan(c->cfg, c->n_cu, *batch).bytes;
}

int kvfold_pcache_append(const kvfold_pcache_t* c, int layer, const void* k, const void* v, int64_t kv_stride, const int64_t* slots, int32_t n_tokens, void* stream) {
  if (!c || n_tokens < 0 || kv_stride < 0 || (n_tokens > 0 && (!k || !v || !slots))) return KVFOLD_ERR_INVALID_ARG;
  if (layer < 0 || layer >= c->cfg.n_layers) return KVFOLD_ERR_BAD_LAYER;
  const int64_t narrow = (int64_t)c->cfg.n_kv_heads * c->cfg.head_dim;
  if (kv_stride % (16 / c->es()) || (kv_stride && kv_stride < narrow) || !aligned(k, 16) || !aligned(v, 16) || !aligned(slots, 8)) return KVFOLD_ERR_INVALID_ARG;
  if (kv_stride > (int64_t)1 << 31) return KVFOLD_ERR_UNSUPPORTED;
  if (n_tokens == 0) return KVFOLD_OK;
  const int64_t stride = kv_stride ? kv_stride : narrow;
  const size_t rows = extent(n_tokens, stride, c->cfg.n_kv_heads, c->cfg.head_dim, c->es());
  const Range inputs[] = {{k, rows}, {v, rows}, {slots, (size_t)n_tokens * 8}};
  if (!all_apart({c->store, c->bytes()}, inputs, 3)) return KVFOLD_ERR_INVALID_ARG;
  DeviceGuard guard(c->cfg.device);
  if (guard.err != hipSuccess) return hip_fail(guard.err);
  const hipError_t e = append_rows(c, layer, k, v, stride, slots, n_tokens, PromptPlanParams{}, static_cast<hipStream_t>(stream));
  return e == hipSuccess ? KVFOLD_OK : hip_fail(e);
}

int kvfold_pcache_step(const kvfold_pcache_t* c, int layer, const kvfold_batch_t* b, const void* q, const void* k_new, const void* v_new, void* out, float* lse,
                       void* workspace, size_t workspace_bytes, void* stream) {
  if (!c) return KVFOLD_ERR_INVALID_ARG;
  const kvfold_pcache_config_t& f = c->cfg;
  int rc = validate_batch(f, b);
  if (rc != KVFOLD_OK) return rc;
  if (layer < 0 || layer >= f.n_layers) return KVFOLD_ERR_BAD_LAYER;
  const bool fresh = b->slots != nullptr;
  if ((fresh && (!k_new || !v_new)) || (!fresh && (k_new || v_new))) return KVFOLD_ERR_INVALID_ARG;
  if (!b->cu_new && (b->n_tokens != b->n_seqs || b->max_new != 1)) return KVFOLD_ERR_INVALID_ARG;
  if (b->n_seqs == 0 || b->n_tokens == 0) return KVFOLD_OK;
  if (!q || !out || !workspace || !b->tables || !b->lens) return KVFOLD_ERR_INVALID_ARG;
  if (!aligned(q, 16) || !aligned(k_new, 16) || !aligned(v_new, 16) || !aligned(out, 16) || !aligned(lse, 4) || !aligned(workspace, 256) || !aligned(b->tables, 4) ||
      !aligned(b->lens, 4) || !aligned(b->cu_new, 4) || !aligned(b->slots, 8))
    return KVFOLD_ERR_INVALID_ARG;
  const PagedPlan pl = make_pplan(f, c->n_cu, *b);
  if (workspace_bytes < pl.bytes) return KVFOLD_ERR_OOM;
  const int64_t q_stride = b->q_stride ? b->q_stride : (int64_t)f.n_q_heads * f.head_dim, kv_stride = b->kv_stride ? b->kv_stride : (int64_t)f.n_kv_heads * f.head_dim;
  const size_t seqs = (size_t)b->n_seqs * 4, tokens = (size_t)b->n_tokens, narrow = extent(b->n_tokens, kv_stride, f.n_kv_heads, f.head_dim, c->es());
  const Range all[] = {{out, tokens * (size_t)f.n_q_heads * (size_t)f.head_dim * (size_t)c->es()}, {lse, lse ? tokens * (size_t)f.n_q_heads * 4 : 0},
                       {workspace, pl.bytes}, {c->store, c->bytes()},  // what is written, then what is read
                       {q, extent(b->n_tokens, q_stride, f.n_q_heads, f.head_dim, c->es())}, {k_new, fresh ? narrow : 0}, {v_new, fresh ? narrow : 0},
                       {b->tables, (size_t)b->n_seqs * (size_t)b->table_stride * 4}, {b->lens, seqs}, {b->cu_new, b->cu_new ? seqs + 4 : 0},
                       {b->slots, fresh ? tokens * 8 : 0}};
  for (int i = 0; i < 4; ++i)
    if (!all_apart(all[i], all + i + 1, 10 - i)) return KVFOLD_ERR_INVALID_ARG;

  DeviceGuard guard(f.device);
  if (guard.err != hipSuccess) return hip_fail(guard.err);
  hipStream_t s = static_cast<hipStream_t>(stream);
  const bool bf16 = f.dtype == KVFOLD_BF16;
  PAttnParams p;
  p.q = q;
  p.k_new = pl.decode && fresh ? k_new : nullptr;
  p.v_new = pl.decode && fresh ? v_new : nullptr;
  p.k_pages = c->rows(layer, false);
  p.v_pages = c->rows(layer, true);
  p.out = out;
  p.lse = lse;
  p.tables = b->tables;
  p.lens = b->lens;
  p.cu_new = b->cu_new;
  p.slots = b->slots;
  p.counters = static_cast<uint32_t*>(workspace);
  unsigned char* list = static_cast<unsigned char*>(workspace) + pl.counters;
  p.list_head = reinterpret_cast<int32_t*>(list);
  p.items = reinterpret_cast<PromptItem*>(list + kPromptHead);
  p.merges = reinterpret_cast<int32_t*>(list + kPromptHead + (size_t)pl.items * sizeof(PromptItem));
  p.n_blocks = (int32_t)pl.blocks;
  p.n_cu = c->n_cu;
  p.from_end = pl.from_end;
  p.shared = pl.shared;
  p.part_o = reinterpret_cast<float*>(list + pl.list);
  p.part_ml = p.part_o + pl.rows * f.head_dim;
  p.table_stride = b->table_stride;
  p.q_stride = q_stride;
  p.kv_stride = kv_stride;
  p.n_places = c->places();
  p.page_bytes = pcache_layer_bytes(f) / 2 / (size_t)f.n_pages;
  p.n_seqs = b->n_seqs;
  p.n_tokens = b->n_tokens;
  p.max_new = b->max_new < b->n_tokens ? b->max_new : b->n_tokens;
  const int64_t named = b->table_stride * f.page_tokens;
  p.max_len = (int32_t)(b->max_len < named ? b->max_len : named);
  p.n_q_heads = f.n_q_heads;
  p.n_kv_heads = f.n_kv_heads;
  p.group = f.n_q_heads / f.n_kv_heads;
  p.page_log2 = c->page_log2;
  p.n_pages = f.n_pages;
  p.n_pieces = pl.n_pieces;
  p.piece = pl.piece;
  p.unit_rows = pl.unit_rows;
  p.n_units = pl.decode ? b->n_seqs * f.n_kv_heads : (int32_t)pl.items;
  p.scale_log2e = c->scale * 1.4426950408889634f;
  p.from_log2 = 1.0f / p.scale_log2e;
  p.stale = 16.0f * p.from_log2;
  p.by_group = fast_div(p.group);
  p.by_units = fast_div(p.n_units);
  p.by_kv_heads = fast_div(f.n_kv_heads);
  hipError_t e;
  if (pl.decode) {
    e = launch_attn_pdecode(p, f.head_dim, bf16, s);
  } else {
    PromptPlanParams plan;
    plan.lens = b->lens;
    plan.cu_new = b->cu_new;
    plan.slots = b->slots;
    plan.all_places = c->places();
    plan.head = reinterpret_cast<int32_t*>(list);
    plan.items = reinterpret_cast<PromptItem*>(list + kPromptHead);
    plan.n_seqs = b->n_seqs;
    plan.n_tokens = b->n_tokens;
    plan.max_new = p.max_new;
    plan.max_len = p.max_len;
    plan.group = p.group;
    plan.unit_rows = pl.unit_rows;
    plan.max_items = (int32_t)pl.items;
    plan.max_merges = (int32_t)pl.blocks;
    plan.n_pieces = pl.n_pieces;
    plan.n_kv_heads = f.n_kv_heads;
    plan.merges = const_cast<int32_t*>(p.merges);
    plan.n_places = pl.places;
    plan.n_cu = c->n_cu;
    plan.shortest = pl.shortest;
    plan.step = pl.step;
    plan.cost_once = pl.cost_once;
    plan.cost_piece = pl.cost_piece;
    plan.cost_merge = pl.cost_merge;
    e = append_rows(c, layer, k_new, v_new, kv_stride, b->slots, fresh ? b->n_tokens : 0, plan, s);
    if (e == hipSuccess) e = launch_attn_prompt(p, f.head_dim, bf16, pl.units_per_wave, s);
    if (e == hipSuccess && pl.n_pieces > 1) e = launch_pmerge(p, f.head_dim, bf16, s);
  }
  return e == hipSuccess ? KVFOLD_OK : hip_fail(e);
}

}  // extern "C"
