// Device-side helpers shared by the kernels over a paged KV cache.
#pragma once

#include "paged.hpp"
#include "reco_device.hpp"

#include <math.h>

namespace reco {

constexpr int kDevAppendOverflow = 1, kDevBadScore = 3, kDevBadLength = 5, kDevBadPage = 7, kDevBadBudget = 8,
              kDevStalled = 9;

// Table entries are read through the scalar unit where their index is the same
// in all lanes: no kernel writes the table.
typedef const __attribute__((address_space(4))) int32_t const_i32;
__device__ __forceinline__ const_i32 *as_const(const int32_t *p) {
  return reinterpret_cast<const_i32 *>(reinterpret_cast<uintptr_t>(p));
}

// One unit of a paged cache with n cached rows.  Only ids of pages that hold cached
// rows are used; one outside the pool becomes its last page and is noted.
struct PagedUnit {
  const_i32 *table;
  int n_pages, shift, last;
  unsigned worst;

  __device__ __forceinline__ PagedUnit(const PagedCache &c, size_t cunit, int n)
      : table(as_const(c.pages + cunit * static_cast<size_t>(c.max_pages))), n_pages(c.n_pages), shift(c.page_shift),
        last(max(n - 1, 0)), worst(0) {}
  // The table's entry for `row` (the same in all lanes), or for the last cached row
  // where that comes first.  Without a branch, so that several are on their way at once.
  __device__ __forceinline__ int entry(int row) const { return table[min(row, last) >> shift]; }
  // The pool's row of `row`, by its entry.
  __device__ __forceinline__ size_t row_at(int entry, int row) {
    worst = max(worst, static_cast<unsigned>(entry));
    const unsigned id = min(static_cast<unsigned>(entry), static_cast<unsigned>(n_pages - 1));
    return (static_cast<size_t>(id) << shift) + static_cast<size_t>(row & ((1 << shift) - 1));
  }
  __device__ __forceinline__ bool bad() const { return worst >= static_cast<unsigned>(n_pages); }
};

// The rows that a token at row n_tot - 1 sees: [0, sink_end) and [lo, n_tot), as
// a list of tiles (first the sinks', then the window's).
struct SeenTiles {
  int n_tot, lo, sink_end;
  int sink_tiles, skip, total;

  __device__ __forceinline__ SeenTiles(int n, int sinks, int window) : n_tot(n) {
    lo = window > 0 && n > window ? n - window : 0;
    sink_end = sinks < lo ? sinks : lo;
    const int first = lo / kPagedTile;
    const int st = (sink_end + kPagedTile - 1) / kPagedTile;
    sink_tiles = st < first ? st : first;
    skip = first - sink_tiles;
    total = (n + kPagedTile - 1) / kPagedTile - skip;
  }
  __device__ __forceinline__ int tile(int i) const { return i < sink_tiles ? i : i + skip; }
  __device__ __forceinline__ bool sees(int row) const { return row < n_tot && (row >= lo || row < sink_end); }
  // Whether all rows of the tile at row kb are cached and seen.
  __device__ __forceinline__ bool whole(int kb, int n_cache) const {
    return kb + kPagedTile <= n_cache && (kb >= lo || kb + kPagedTile <= sink_end);
  }
};

}  // namespace reco
