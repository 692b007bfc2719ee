// Launch interface of the kernels over a paged KV cache (paged_decode.hip,
// paged_prefill.hip, paged_evict.hip).  Not part of the public ABI.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace reco {

// Division by a number that the host knows: n / d for 0 <= n < 2^28 and n d < 2^36.  The
// compiler's own takes some 35 instructions in a row, which short kernels wait for.
struct FastDiv {
  uint64_t m;
  int d;

  FastDiv() = default;
  explicit FastDiv(int divisor) : m(((uint64_t{1} << 36) + divisor - 1) / divisor), d(divisor) {}
  __host__ __device__ int of(int n) const { return static_cast<int>((static_cast<uint64_t>(static_cast<uint32_t>(n)) * m) >> 36); }
  __host__ __device__ int rest(int n) const { return n - of(n) * d; }
};

// A unit is (layer of the call, sequence, KV head) in this order, so that the query heads
// of unit u start at u * group and its cache unit is layer0 * batch * hkv + u.
// A page holds 1 << page_shift rows (16 or more) of one unit; cap = max_pages << page_shift.
struct PagedCache {
  void *k;                // [n_pages][page rows][D]
  void *v;
  const int32_t *pages;   // [cache layers][batch][hkv][max_pages]
  int32_t *len;           // [cache layers][batch][hkv]
  float *weight;          // nullable [cache layers][batch][hkv][cap]
  int32_t *dev_err;
  FastDiv by_hkv, by_batch;
  int layer0, n_layers, batch, hkv, n_pages, page_shift, max_pages, cap;

  __host__ __device__ size_t unit(int u) const { return static_cast<size_t>(layer0) * batch * hkv + u; }
  __host__ __device__ int sequence(int u) const { return by_batch.rest(by_hkv.of(u)); }
};

// ---- attention of one new token ---------------------------------------------
struct PagedDecodeParams {
  PagedCache c;
  const void *q;          // [n_layers][batch][hq][D]
  const void *k_new;      // nullable [n_layers][batch][hkv][D]
  const void *v_new;
  void *out;              // [n_layers][batch][hq][D]
  float *lse;             // nullable [n_layers][batch][hq]
  float *part_o;          // [units][splits][group][D]
  float *part_ml;         // [units][splits][2][group]  (maxima, sums)
  int32_t *len_in;        // [units]  lengths before the append, for the weights
  float *logits;          // [units][group][logit_pitch]  log2-domain logits, where weights are kept
  int64_t logit_pitch;
  bool held_logits;       // in the workgroup instead
  FastDiv by_splits, by_group;
  int group, splits, cus;
  int sinks, window;      // window 0: every row is visible
  float scale_log2;       // logit scale * log2(e)
};
// Most tiles of kPagedTile rows that a call's tokens see.
constexpr int kPagedTile = 32;
constexpr int kPagedMaxSplits = 128;
int paged_span_tiles(int capacity, int sinks, int window);
int paged_decode_splits(int units, int span_tiles, int compute_units);
size_t paged_decode_workspace_bytes(int units, int capacity, int group, int head_dim, bool weights, int compute_units);
// Places the parts of a call's workspace; p.splits, p.group and p.c.cap are set.
void paged_decode_place(PagedDecodeParams &p, int head_dim, void *ws);
// Workgroups that the weights of a call's unit take, and whether they fit a grid.
constexpr int kPagedWeightRows = 1024;
int paged_weight_chunks(const PagedDecodeParams &p);
bool paged_decode_fits_grid(const PagedDecodeParams &p);
hipError_t launch_paged_decode(const PagedDecodeParams &p, int dtype, int head_dim, hipStream_t s);

// ---- attention of a run of new tokens -------------------------------------------
constexpr int kPrefillRows = 128;        // query rows of a workgroup
constexpr int kPrefillLongRows = 256;    // of one for long bf16 runs
constexpr int kPrefillMaxSplits = 64;
constexpr int kPrefillAppendRows = 128;  // of a workgroup that appends
constexpr int kXcds = 8;
struct PagedPrefillParams {
  PagedCache c;
  const void *q;          // [n_layers][batch][hq][tokens][D]
  const void *k_new;      // [n_layers][batch][hkv][tokens][D]
  const void *v_new;
  const int32_t *n_new;   // nullable [batch]: real tokens of each sequence
  void *out;              // [n_layers][batch][hq][tokens][D]
  float *lse;             // nullable [n_layers][batch][hq][tokens]
  int32_t *len_in;        // [units]  lengths before the append
  float *part_o;          // [units][blocks][splits][kPrefillRows][D]
  float *part_ml;         // [units][blocks][splits][2][kPrefillRows]
  FastDiv by_splits, by_group, by_near;
  int group, tokens, blocks, splits;
  int rows;               // of a block: kPrefillRows, or kPrefillLongRows with one split
  int pieces;             // of a unit's blocks, each for one XCD, where there are many; else 0
  int near;               // blocks of a piece
  bool spread;            // a piece's blocks are every pieces-th, not neighbours
  int sinks, window;
  float scale_log2;
};
int prefill_blocks(int tokens, int group, int rows);
int prefill_rows(int units, int tokens, int group, int capacity, int window, int dtype, int compute_units);
constexpr int prefill_tile_rows(int dtype) { return dtype == 0 ? 32 : 64; }   // keys of a tile: fp32, bf16
int prefill_splits(int units, int blocks, int capacity, int sinks, int window, int tile_rows, int compute_units);
size_t prefill_workspace_bytes(int units, int tokens, int capacity, int group, int head_dim, int tile_rows,
                               int compute_units);
constexpr int kDeviceUnits = 256;        // compute units of a whole MI355X
void prefill_pieces(PagedPrefillParams &p, int units, int compute_units = kDeviceUnits);
bool prefill_fits_grid(const PagedPrefillParams &p);
void prefill_place(PagedPrefillParams &p, int head_dim, void *ws);
hipError_t launch_paged_prefill(const PagedPrefillParams &p, int dtype, int head_dim, hipStream_t s);

// ---- eviction -----------------------------------------------------------------
struct PagedEvictParams {
  PagedCache c;           // with weights
  const int32_t *budget;  // [batch], or [n_layers][batch] with budget_stride = batch
  int64_t budget_stride;
  int32_t *idx;           // [units][cap]  kept rows (the caller's buffer or the workspace)
  bool idx_wanted;        // the caller's: written for units that keep everything, too
  int32_t *kept;          // [units]  rows after the call, or -1 where nothing moves
  int32_t *state;         // [units][state_pitch]  chunks taken, loaded in order, stored, and loaded (one flag each)
  int64_t state_pitch;
  int sinks, recent;
  int chunk_rows;         // rows of a chunk of the compaction
  int workers;            // its workgroups for a unit
  int max_spins;          // of a workgroup that waits for earlier chunks
};
constexpr int kEvictState = 3;
constexpr int kEvictSpins = 1 << 20;         // of a microsecond or so
constexpr int kEvictWorkers = 32;
constexpr int evict_chunk_rows(int row_bytes) { return 32768 / row_bytes; }
size_t paged_evict_workspace_bytes(int units, int capacity, int row_bytes, bool need_idx);
void paged_evict_place(PagedEvictParams &p, int units, int row_bytes, void *ws);
hipError_t launch_paged_evict(const PagedEvictParams &p, int dtype, int head_dim, hipStream_t s);
// The compaction alone, of units whose kept rows, counts and state are set.
hipError_t launch_evict_compact(const PagedEvictParams &p, int row_bytes, hipStream_t s);

}  // namespace reco
