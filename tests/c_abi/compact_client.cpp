// The eviction's compaction alone, on state that the caller sets: what a workgroup does
// whose wait for earlier chunks of its unit ends in vain cannot be brought about by whole
// evictions.
#include "paged.hpp"
#include "reco.h"

extern "C" {

int compact_state() { return reco::kEvictState; }
int compact_chunk_rows(int row_bytes) { return reco::evict_chunk_rows(row_bytes); }

// idx [units][capacity], kept [units], state [units][compact_state() + chunks of capacity],
// all on the device; max_spins 0: the product's own.
int compact_alone(const reco_paged_cache_t *c, int32_t *idx, int32_t *kept, int32_t *state, int max_spins,
                  int32_t *dev_err, hipStream_t stream) {
  const int row_bytes = c->head_dim * (c->dtype == RECO_F32 ? 4 : 2);
  reco::PagedEvictParams p{};
  p.c.k = c->k;
  p.c.v = c->v;
  p.c.pages = c->pages;
  p.c.len = c->len;
  p.c.weight = c->weight;
  p.c.dev_err = dev_err;
  p.c.n_layers = c->n_layers;
  p.c.batch = c->batch;
  p.c.hkv = c->n_kv_heads;
  p.c.n_pages = c->n_pages;
  p.c.by_hkv = reco::FastDiv(c->n_kv_heads);
  p.c.by_batch = reco::FastDiv(c->batch);
  p.c.page_shift = __builtin_ctz(static_cast<unsigned>(c->page_rows));
  p.c.max_pages = c->max_pages;
  p.c.cap = c->max_pages * c->page_rows;
  p.idx = idx;
  reco::paged_evict_place(p, c->n_layers * c->batch * c->n_kv_heads, row_bytes, nullptr);   // rows and workers
  p.kept = kept;
  p.state = state;
  if (max_spins > 0) p.max_spins = max_spins;
  return static_cast<int>(reco::launch_evict_compact(p, row_bytes, stream));
}

}  // extern "C"
