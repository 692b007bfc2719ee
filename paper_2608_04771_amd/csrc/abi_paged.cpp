// C ABI of the operators over a paged KV cache: host-side argument validation,
// workspace sizing and launches, in the manner of abi.cpp.
#include "reco.h"

#include <hip/hip_runtime.h>
#include <math.h>
#include <stddef.h>
#include <stdint.h>

#include "abi_common.hpp"
#include "paged.hpp"

namespace {

// Positions rounded up to a tile, and sums of two of them, stay inside int32.
constexpr int64_t kMaxCapacity = int64_t{1} << 29;
constexpr int64_t kMaxQueryRows = int64_t{1} << 28;   // of one KV head in a run

bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

int64_t capacity_of(const reco_paged_cache_t *c) { return static_cast<int64_t>(c->max_pages) * c->page_rows; }

int row_bytes_of(const reco_paged_cache_t *c) { return c->head_dim * (c->dtype == RECO_F32 ? 4 : 2); }

bool paged_ok(const reco_paged_cache_t *c) {
  return c && c->k && c->v && c->pages && c->len && c->n_layers >= 1 && c->batch >= 1 && c->n_kv_heads >= 1 &&
         c->n_pages >= 1 && c->page_rows >= 1 && c->max_pages >= 1 && aligned16(c->k) && aligned16(c->v) &&
         aligned16(c->weight);
}

reco_status_t paged_supported(const reco_paged_cache_t *c) {
  if (c->head_dim != 64 && c->head_dim != 128) return RECO_ERR_UNSUPPORTED;
  if (c->dtype != RECO_F32 && c->dtype != RECO_BF16) return RECO_ERR_UNSUPPORTED;
  if (c->page_rows < 16 || c->page_rows > 4096 || (c->page_rows & (c->page_rows - 1))) return RECO_ERR_UNSUPPORTED;
  if (capacity_of(c) > kMaxCapacity) return RECO_ERR_UNSUPPORTED;
  return RECO_OK;
}

bool paged_layers_ok(const reco_paged_cache_t *c, int32_t layer0, int32_t n_layers) {
  return layer0 >= 0 && n_layers >= 1 && static_cast<int64_t>(layer0) + n_layers <= c->n_layers;
}

// Units of a call, or 0 where they do not fit a grid dimension.
int units_of(const reco_paged_cache_t *c, int32_t n_layers) {
  if (n_layers < 1) return 0;
  const int64_t rest = static_cast<int64_t>(c->batch) * c->n_kv_heads;
  if (rest > 65535 || rest * n_layers > 65535) return 0;
  return static_cast<int>(rest * n_layers);
}

int group_of(const reco_paged_cache_t *c, int32_t n_q_heads) {
  if (n_q_heads < 1 || n_q_heads % c->n_kv_heads != 0) return -1;
  return n_q_heads / c->n_kv_heads;
}

reco::PagedCache paged_cache(const reco_paged_cache_t *c, int32_t layer0, int32_t n_layers, int32_t *dev_err) {
  reco::PagedCache p{};
  p.k = c->k;
  p.v = c->v;
  p.pages = c->pages;
  p.len = c->len;
  p.weight = c->weight;
  p.dev_err = dev_err;
  p.layer0 = layer0;
  p.n_layers = n_layers;
  p.batch = c->batch;
  p.hkv = c->n_kv_heads;
  p.n_pages = c->n_pages;
  p.by_hkv = reco::FastDiv(c->n_kv_heads);
  p.by_batch = reco::FastDiv(c->batch);
  p.page_shift = __builtin_ctz(static_cast<unsigned>(c->page_rows));
  p.max_pages = c->max_pages;
  p.cap = static_cast<int>(capacity_of(c));
  return p;
}

}  // namespace

extern "C" {

// ---------------------------------------------------------------- decode
size_t reco_paged_decode_attn_workspace_size(const reco_paged_cache_t *cache, int32_t n_layers, int32_t n_q_heads) {
  if (!paged_ok(cache) || paged_supported(cache) != RECO_OK) return 0;
  const int units = units_of(cache, n_layers), G = group_of(cache, n_q_heads);
  if (units < 1 || G < 1 || G > 16) return 0;
  return reco::paged_decode_workspace_bytes(units, static_cast<int>(capacity_of(cache)), G, cache->head_dim,
                                            cache->weight != nullptr, reco::current_compute_units());
}

reco_status_t reco_paged_decode_attn(const reco_paged_cache_t *cache, int32_t layer0, int32_t n_layers, const void *q,
                                     int32_t n_q_heads, float scale, int32_t sinks, int32_t window, const void *k_new,
                                     const void *v_new, void *out, float *lse, void *ws, size_t ws_bytes,
                                     int32_t *dev_err, hipStream_t stream) {
  if (!paged_ok(cache) || !q || !out || sinks < 0 || window < 0 || !isfinite(scale)) return RECO_ERR_INVALID_ARG;
  if ((k_new == nullptr) != (v_new == nullptr)) return RECO_ERR_INVALID_ARG;
  if (!aligned16(q) || !aligned16(out) || !aligned16(k_new) || !aligned16(v_new)) return RECO_ERR_INVALID_ARG;
  if (!paged_layers_ok(cache, layer0, n_layers)) return RECO_ERR_INVALID_ARG;
  const int units = units_of(cache, n_layers), G = group_of(cache, n_q_heads);
  if (units < 1 || G < 1) return RECO_ERR_INVALID_ARG;
  const reco_status_t st = paged_supported(cache);
  if (st != RECO_OK) return st;
  if (G > 16) return RECO_ERR_UNSUPPORTED;
  const int cus = reco::current_compute_units();

  reco::PagedDecodeParams p{};
  p.c = paged_cache(cache, layer0, n_layers, dev_err);
  const size_t need =
      reco::paged_decode_workspace_bytes(units, p.c.cap, G, cache->head_dim, cache->weight != nullptr, cus);
  if (!ws || ws_bytes < need || (reinterpret_cast<uintptr_t>(ws) & 255)) return RECO_ERR_WORKSPACE;
  p.q = q;
  p.k_new = k_new;
  p.v_new = v_new;
  p.out = out;
  p.lse = lse;
  p.group = G;
  p.by_group = reco::FastDiv(G);
  p.cus = cus;
  p.sinks = sinks;
  p.window = window;
  p.scale_log2 = scale * 1.4426950408889634f;
  p.splits = reco::paged_decode_splits(units, reco::paged_span_tiles(p.c.cap, sinks, window), cus);
  p.by_splits = reco::FastDiv(p.splits);
  if (!reco::paged_decode_fits_grid(p)) return RECO_ERR_UNSUPPORTED;
  reco::paged_decode_place(p, cache->head_dim, ws);
  return reco::hip_status(reco::launch_paged_decode(p, cache->dtype, cache->head_dim, stream));
}

// ---------------------------------------------------------------- prefill
size_t reco_paged_prefill_attn_workspace_size(const reco_paged_cache_t *cache, int32_t n_layers, int32_t n_q_heads,
                                              int32_t n_tokens) {
  if (!paged_ok(cache) || paged_supported(cache) != RECO_OK) return 0;
  const int units = units_of(cache, n_layers), G = group_of(cache, n_q_heads);
  if (units < 1 || G < 1 || G > 16 || n_tokens < 1 || static_cast<int64_t>(n_tokens) * G > kMaxQueryRows) return 0;
  return reco::prefill_workspace_bytes(units, n_tokens, static_cast<int>(capacity_of(cache)), G, cache->head_dim,
                                       reco::prefill_tile_rows(cache->dtype), reco::current_compute_units());
}

reco_status_t reco_paged_prefill_attn(const reco_paged_cache_t *cache, int32_t layer0, int32_t n_layers,
                                      const void *q, int32_t n_q_heads, int32_t n_tokens, const int32_t *n_new,
                                      float scale, int32_t sinks, int32_t window, const void *k_new,
                                      const void *v_new, void *out, float *lse, void *ws, size_t ws_bytes,
                                      int32_t *dev_err, hipStream_t stream) {
  if (!paged_ok(cache) || !q || !k_new || !v_new || !out || sinks < 0 || window < 0 || !isfinite(scale))
    return RECO_ERR_INVALID_ARG;
  if (!aligned16(q) || !aligned16(out) || !aligned16(k_new) || !aligned16(v_new)) return RECO_ERR_INVALID_ARG;
  if (!paged_layers_ok(cache, layer0, n_layers) || n_tokens < 1) return RECO_ERR_INVALID_ARG;
  const int units = units_of(cache, n_layers), G = group_of(cache, n_q_heads);
  if (units < 1 || G < 1) return RECO_ERR_INVALID_ARG;
  const reco_status_t st = paged_supported(cache);
  if (st != RECO_OK) return st;
  if (G > 16 || static_cast<int64_t>(n_tokens) * G > kMaxQueryRows) return RECO_ERR_UNSUPPORTED;
  const int cus = reco::current_compute_units();

  reco::PagedPrefillParams p{};
  p.c = paged_cache(cache, layer0, n_layers, dev_err);
  const int tile_rows = reco::prefill_tile_rows(cache->dtype);
  const size_t need = reco::prefill_workspace_bytes(units, n_tokens, p.c.cap, G, cache->head_dim, tile_rows, cus);
  if (!ws || ws_bytes < need || (reinterpret_cast<uintptr_t>(ws) & 255)) return RECO_ERR_WORKSPACE;
  p.q = q;
  p.k_new = k_new;
  p.v_new = v_new;
  p.n_new = n_new;
  p.out = out;
  p.lse = lse;
  p.group = G;
  p.by_group = reco::FastDiv(G);
  p.tokens = n_tokens;
  p.rows = reco::prefill_rows(units, n_tokens, G, p.c.cap, window, cache->dtype, cus);
  p.blocks = reco::prefill_blocks(n_tokens, G, p.rows);
  p.splits = p.rows == reco::kPrefillRows
                 ? reco::prefill_splits(units, p.blocks, p.c.cap, sinks, window, tile_rows, cus) : 1;
  p.sinks = sinks;
  p.window = window;
  p.scale_log2 = scale * 1.4426950408889634f;
  p.by_splits = reco::FastDiv(p.splits);
  if (!reco::prefill_fits_grid(p)) return RECO_ERR_UNSUPPORTED;
  reco::prefill_pieces(p, units, cus);
  reco::prefill_place(p, cache->head_dim, ws);
  return reco::hip_status(reco::launch_paged_prefill(p, cache->dtype, cache->head_dim, stream));
}

// ---------------------------------------------------------------- eviction
size_t reco_paged_evict_workspace_size(const reco_paged_cache_t *cache, int32_t n_layers) {
  if (!paged_ok(cache) || paged_supported(cache) != RECO_OK) return 0;
  const int units = units_of(cache, n_layers);
  if (units < 1) return 0;
  return reco::paged_evict_workspace_bytes(units, static_cast<int>(capacity_of(cache)), row_bytes_of(cache), true);
}

reco_status_t reco_paged_evict(const reco_paged_cache_t *cache, int32_t layer0, int32_t n_layers,
                               const int32_t *budget, int64_t budget_layer_stride, int32_t sinks, int32_t recent,
                               int32_t *kept_idx, void *ws, size_t ws_bytes, int32_t *dev_err, hipStream_t stream) {
  if (!paged_ok(cache) || !cache->weight || !budget || budget_layer_stride < 0) return RECO_ERR_INVALID_ARG;
  if (sinks < 0 || recent < 0) return RECO_ERR_INVALID_ARG;
  if (!paged_layers_ok(cache, layer0, n_layers)) return RECO_ERR_INVALID_ARG;
  const int units = units_of(cache, n_layers);
  if (units < 1) return RECO_ERR_INVALID_ARG;
  const reco_status_t st = paged_supported(cache);
  if (st != RECO_OK) return st;

  reco::PagedEvictParams p{};
  p.c = paged_cache(cache, layer0, n_layers, dev_err);
  const size_t need = reco::paged_evict_workspace_bytes(units, p.c.cap, row_bytes_of(cache), kept_idx == nullptr);
  if (!ws || ws_bytes < need || (reinterpret_cast<uintptr_t>(ws) & 255)) return RECO_ERR_WORKSPACE;
  p.budget = budget;
  p.budget_stride = budget_layer_stride;
  p.sinks = sinks;
  p.recent = recent;
  p.idx = kept_idx;
  reco::paged_evict_place(p, units, row_bytes_of(cache), ws);
  return reco::hip_status(reco::launch_paged_evict(p, cache->dtype, cache->head_dim, stream));
}

}  // extern "C"
