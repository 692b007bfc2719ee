// Work split of the kernels over a paged cache and the workspaces it implies
// (host code).
#include "paged.hpp"

#include "decode_plan.hpp"
#include "rope.hpp"

namespace reco {

namespace {
size_t aligned(size_t bytes) { return (bytes + 255) / 256 * 256; }
size_t logit_pitch(int capacity) { return (static_cast<size_t>(capacity) + 1 + kPagedTile - 1) / kPagedTile * kPagedTile; }
size_t partial_bytes(int units, int splits, int group, int head_dim) {
  return aligned(static_cast<size_t>(units) * splits * group * (static_cast<size_t>(head_dim) + 2) * sizeof(float));
}
}  // namespace

int paged_span_tiles(int capacity, int sinks, int window) {
  const int64_t all = (static_cast<int64_t>(capacity) + 1 + kPagedTile - 1) / kPagedTile;
  if (window == 0) return static_cast<int>(all);
  // the sinks' tiles, and a window's, which may begin and end inside a tile
  const int64_t seen = (static_cast<int64_t>(sinks) + kPagedTile - 1) / kPagedTile +
                       (static_cast<int64_t>(window) + 2 * kPagedTile - 2) / kPagedTile;
  return static_cast<int>(seen < all ? seen : all);
}

// The rule of the dense cache (decode_plan.cpp) on the rows that can be visible; twice
// its splits, two workgroups on a compute unit, where units shorter than capacity may
// leave others to finish alone (128 units of 4K-32K rows: 217 -> 194 us) and a split
// keeps 64 tiles, which costs even units little (112 of 8.7K: 82 -> 83 us).
int paged_decode_splits(int units, int span_tiles, int compute_units) {
  const int splits = decode_splits(units, span_tiles * kDecodeTile - 1, compute_units);
  const bool more = splits > 1 && units <= compute_units && 2 * splits <= kPagedMaxSplits && span_tiles / (2 * splits) >= 64;
  return more ? 2 * splits : splits;
}

size_t paged_decode_workspace_bytes(int units, int capacity, int group, int head_dim, bool weights,
                                    int compute_units) {
  // a window takes no more splits than the whole cache does
  const int splits = paged_decode_splits(units, paged_span_tiles(capacity, 0, 0), compute_units);
  size_t bytes = partial_bytes(units, splits, group, head_dim) + aligned(static_cast<size_t>(units) * sizeof(int32_t));
  if (weights) bytes += static_cast<size_t>(units) * group * logit_pitch(capacity) * sizeof(float);
  return bytes;
}

int paged_weight_chunks(const PagedDecodeParams &p) {
  if (!p.c.weight) return 0;
  const int64_t rows = static_cast<int64_t>(paged_span_tiles(p.c.cap, p.sinks, p.window)) * kPagedTile;
  return static_cast<int>((rows + kPagedWeightRows - 1) / kPagedWeightRows);
}

bool paged_decode_fits_grid(const PagedDecodeParams &p) {
  const int64_t units = static_cast<int64_t>(p.c.n_layers) * p.c.batch * p.c.hkv;
  return units * (p.group + paged_weight_chunks(p)) < (int64_t{1} << 24);   // of 256 threads
}

void paged_decode_place(PagedDecodeParams &p, int head_dim, void *ws) {
  const int units = p.c.n_layers * p.c.batch * p.c.hkv;
  char *at = static_cast<char *>(ws);
  p.part_o = reinterpret_cast<float *>(at);
  p.part_ml = p.part_o + static_cast<size_t>(units) * p.splits * p.group * head_dim;
  at += partial_bytes(units, p.splits, p.group, head_dim);
  p.len_in = reinterpret_cast<int32_t *>(at);
  at += aligned(static_cast<size_t>(units) * sizeof(int32_t));
  p.logits = p.c.weight ? reinterpret_cast<float *>(at) : nullptr;
  p.logit_pitch = static_cast<int64_t>(logit_pitch(p.c.cap));
}

int prefill_blocks(int tokens, int group, int rows) {
  return static_cast<int>((static_cast<int64_t>(tokens) * group + rows - 1) / rows);
}

// Blocks of 256 rows for bf16, whose eight waves share a tile, where a block sees many
// keys (1,024 by what the call can know: 2,048 tokens of 32 units of 4 heads 204 -> 191 us
// against blocks of 128; prompts of 200 to 512 tokens 40 -> 45) and the blocks fill the
// last round of two workgroups on every compute unit, or it is one of many (at 1.5 rounds,
// 2,452 tokens of 16 units of 5 heads, 181 -> 213 us; at 4, 8,192 of 16 of 4, 1,178 -> 1,066).
int prefill_rows(int units, int tokens, int group, int capacity, int window, int dtype, int compute_units) {
  if (dtype != 1) return kPrefillRows;
  const int64_t blocks = static_cast<int64_t>(units) * prefill_blocks(tokens, group, kPrefillLongRows);
  const int64_t round = 2 * static_cast<int64_t>(compute_units), rounds = (blocks + round - 1) / round;
  const int own = tokens < capacity ? tokens : capacity;
  int keys = capacity - own / 2;
  if (window > 0 && window < keys) keys = window;
  const bool even = blocks >= 3 * round || 8 * blocks >= 7 * rounds * round;
  return keys >= 1024 && even ? kPrefillLongRows : kPrefillRows;
}

// Key tiles are split where there are too few blocks of query rows for two workgroups
// on every compute unit, into pieces of at least six tiles of bf16 (32 tokens over 9,645
// rows of 4 units of 7 heads: 30.0 us per call by twos, 31.3 by fours, 27.1 by sixes, 30.3 by
// eights) or one of fp32, whose products take sixteen times as long (90 tokens of 2 units of
// 4 heads: 28 us by twos, 22 by ones).
int prefill_splits(int units, int blocks, int capacity, int sinks, int window, int tile_rows, int compute_units) {
  int64_t rows = capacity;
  if (window > 0) {
    const int64_t seen = static_cast<int64_t>(sinks) + window + 2 * kPrefillRows;
    if (seen < rows) rows = seen;
  }
  int64_t splits = 2 * static_cast<int64_t>(compute_units) / (static_cast<int64_t>(units) * blocks);
  const int64_t pieces = rows / (tile_rows == prefill_tile_rows(0) ? tile_rows : 6 * tile_rows);
  if (splits > pieces) splits = pieces;
  if (splits > kPrefillMaxSplits) splits = kPrefillMaxSplits;
  return splits < 1 ? 1 : static_cast<int>(splits);
}

size_t prefill_workspace_bytes(int units, int tokens, int capacity, int group, int head_dim, int tile_rows,
                               int compute_units) {
  const int blocks = prefill_blocks(tokens, group, kPrefillRows);
  const int splits = prefill_splits(units, blocks, capacity, 0, 0, tile_rows, compute_units);   // a window takes no more
  size_t bytes = aligned(static_cast<size_t>(units) * sizeof(int32_t));
  if (splits > 1)
    bytes += static_cast<size_t>(units) * blocks * splits * kPrefillRows * (static_cast<size_t>(head_dim) + 2) * sizeof(float);
  return bytes;
}

// Where every XCD has four rounds of its compute units and more, a piece is up to one
// round's blocks of a unit, and a quarter of that at least: as many as leave the XCDs with
// the same number of pieces, or nearly.  A partition of the device has fewer compute units,
// and its workgroups take eight turns all the same.  Without a window a block's work grows with its place, so a piece takes blocks
// from everywhere (its XCD's others wait for none: 8,192 tokens of 16 units of 4 heads
// 1,601 -> 1,066 us); with one, neighbours see the same keys.
void prefill_pieces(PagedPrefillParams &p, int units, int compute_units) {
  const int64_t all = static_cast<int64_t>(units) * p.blocks;
  p.pieces = p.near = 0;
  p.spread = p.window == 0 || p.window >= p.tokens;
  p.by_near = FastDiv(1);
  if (p.splits > 1 || all < 4 * static_cast<int64_t>(compute_units)) return;
  const int round = compute_units < kXcds ? 1 : compute_units / kXcds;
  double least = 1e30;
  for (int near = round; near >= (round + 3) / 4; --near) {
    const int pieces = (p.blocks + near - 1) / near;
    const int size = (p.blocks + pieces - 1) / pieces;
    const int64_t turns = (static_cast<int64_t>(units) * pieces + kXcds - 1) / kXcds;
    const double cost = static_cast<double>(turns * kXcds * size) / static_cast<double>(all);
    if (cost > 0.97 * least) continue;                   // smaller pieces have to be worth it
    least = cost;
    p.pieces = pieces;
    p.near = size;
  }
  p.by_near = FastDiv(p.near);
}

bool prefill_fits_grid(const PagedPrefillParams &p) {
  const int64_t units = static_cast<int64_t>(p.c.n_layers) * p.c.batch * p.c.hkv;
  const int64_t most = int64_t{1} << 24;                 // workgroups of 256 threads
  const int64_t chunks = p.tokens / kPrefillAppendRows + 1;
  return units * (static_cast<int64_t>(p.blocks) * p.splits + chunks) < most / 4 &&   // of 512, and pieces rounded up
         chunks + (p.splits > 1 ? static_cast<int64_t>(p.blocks) * 16 : 0) < most;
}

void prefill_place(PagedPrefillParams &p, int head_dim, void *ws) {
  const size_t units = static_cast<size_t>(p.c.n_layers) * p.c.batch * p.c.hkv;
  char *at = static_cast<char *>(ws);
  p.len_in = reinterpret_cast<int32_t *>(at);
  at += aligned(units * sizeof(int32_t));
  p.part_o = reinterpret_cast<float *>(at);
  p.part_ml = p.part_o + units * p.blocks * p.splits * kPrefillRows * head_dim;
}

int shared_blocks(int batch, int group, int groups) {
  const int64_t rows = static_cast<int64_t>(batch) * group + static_cast<int64_t>(groups) * (kSharedRows - 1);
  return static_cast<int>(rows / kSharedRows);            // each group's last block may not be whole
}

int shared_span_rows(int capacity, int sinks, int window) {
  const int64_t seen = window == 0 ? capacity : static_cast<int64_t>(sinks) + window;
  return static_cast<int>(seen < capacity ? seen : capacity);
}

// A workgroup for every compute unit shares the common rows of `jobs` (layers and KV heads), nine
// tenths of them at least, and no number where few units have a second one: up to 1.4 for
// each one split more is taken (32 sequences in 8 groups, 4 layers, 144 blocks: 288 workgroups
// 325 us, 432 of them 282; two for every unit write and join more parts: 128 rows of 28 heads a
// group, 8 layers, 64 blocks: 256 workgroups 170 us, 512 of them 195).  A split keeps 256 rows
// of what a call may see, of fp32, whose products take sixteen times as long, a tile.
int shared_splits(int jobs, int blocks, int span_rows, int dtype, int compute_units) {
  const int64_t each = static_cast<int64_t>(jobs) * blocks;
  int64_t splits = compute_units / each;
  if (splits < 1 || 10 * each * splits < 9 * compute_units) {
    ++splits;
    if (each * splits > compute_units && 10 * each * splits < 14 * compute_units) ++splits;
  }
  const int least = dtype == 0 ? prefill_tile_rows(0) : 256;
  if (splits > span_rows / least) splits = span_rows / least;
  if (splits > kSharedMaxSplits) splits = kSharedMaxSplits;
  return splits < 1 ? 1 : static_cast<int>(splits);
}

// A workgroup for every compute unit shares the sequences' own rows, too.
int shared_cell_wgs(int cells, int compute_units) { return (compute_units + cells - 1) / cells; }

// A sequence's even share of its cell's waves, twice that, for longer ones, and two more for
// the waves that it has in part.  Still longer ones make all waves' shares larger.
int shared_own_parts(int batch, int cell_wgs) {
  const int sequences = batch < kSharedCell ? batch : kSharedCell;
  const int64_t parts = 2 * ((4 * static_cast<int64_t>(cell_wgs) + sequences - 1) / sequences) + 2;
  return parts < kSharedMaxSplits ? static_cast<int>(parts) : kSharedMaxSplits;
}

size_t paged_shared_workspace_bytes(int jobs, int batch, int group, int groups, int capacity, int head_dim, int dtype,
                                    int compute_units) {
  // a window takes no more splits than the whole cache does
  const int blocks = shared_blocks(batch, group, groups), cells = jobs * ((batch + kSharedCell - 1) / kSharedCell);
  const size_t parts = static_cast<size_t>(shared_splits(jobs, blocks, capacity, dtype, compute_units)) +
                       shared_own_parts(batch, shared_cell_wgs(cells, compute_units));
  return parts * jobs * batch * group * (static_cast<size_t>(head_dim) + 2) * sizeof(float);
}

void paged_shared_place(PagedSharedParams &p, int head_dim, void *ws) {
  const int64_t jobs = static_cast<int64_t>(p.c.n_layers) * p.c.hkv * p.splits;
  p.common_wgs = static_cast<int>((jobs + kXcds - 1) / kXcds * kXcds * p.blocks);
  p.own_items = p.c.n_layers * p.c.hkv * p.by_chunks.d * p.cell_wgs;
  p.own_wgs = (p.own_items + kXcds - 1) / kXcds * kXcds;
  p.part_o = static_cast<float *>(ws);
  p.part_ml = p.part_o + static_cast<size_t>(p.splits + p.own_parts) * p.rows * head_dim;
}

// Workgroups of 256 threads, what FastDiv divides, and a cell's tiles.
bool paged_shared_fits_grid(const PagedSharedParams &p) {
  const int64_t most = int64_t{1} << 24, units = static_cast<int64_t>(p.c.n_layers) * p.c.batch * p.c.hkv;
  const int64_t jobs = static_cast<int64_t>(p.c.n_layers) * p.c.hkv * p.splits + kXcds;
  const int64_t cells = static_cast<int64_t>(p.c.n_layers) * p.c.hkv * p.by_chunks.d;
  const int64_t sequences = p.c.batch < kSharedCell ? p.c.batch : kSharedCell;
  return jobs * p.blocks + cells * p.cell_wgs < most && units * p.group < most &&
         sequences * (p.c.cap / kPagedTile + 4) < (int64_t{1} << 31);
}

// An appended run of up to eight tokens is one workgroup's, which then sets the lengths itself
// and is as wide as one can be (5 tokens of 4 sequences, 32 layers of 48 rows: 16.0 us with
// 256 threads, 12 with 1,024); other runs go by fours.  Rows that the kernel before has left
// are in the last cache, and what is made of them fits beside them, unless they are many
// (36 heads, past the caches and through them: 2,848 tokens 15.6 and 12.0 us, 8,192 27.1 and
// 26.0, 12,000 36.1 and 42.1).
void rope_plan(RopeParams &p, int row_bytes) {
  const int most = p.c.k && p.tokens <= kRopeMaxBlock ? kRopeMaxBlock : kRopeBlock;
  p.block = 1;
  while (p.block < p.tokens && p.block < most) p.block *= 2;
  const int64_t rows = static_cast<int64_t>(p.layers) * p.batch * p.tokens * (p.heads + (p.c.k ? 2 * p.c.hkv : 0));
  p.far = rows * row_bytes > (int64_t{64} << 20);
}

static int64_t evict_state_pitch(int capacity, int row_bytes) {
  const int rows = evict_chunk_rows(row_bytes);
  return kEvictState + (static_cast<int64_t>(capacity) + rows - 1) / rows;
}

size_t paged_evict_workspace_bytes(int units, int capacity, int row_bytes, bool need_idx) {
  const size_t n = static_cast<size_t>(units);
  size_t bytes = aligned(n * sizeof(int32_t)) + aligned(n * evict_state_pitch(capacity, row_bytes) * sizeof(int32_t));
  if (need_idx) bytes += n * capacity * sizeof(int32_t);
  return bytes;
}

void paged_evict_place(PagedEvictParams &p, int units, int row_bytes, void *ws) {
  char *at = static_cast<char *>(ws);
  p.kept = reinterpret_cast<int32_t *>(at);
  at += aligned(static_cast<size_t>(units) * sizeof(int32_t));
  p.state = reinterpret_cast<int32_t *>(at);
  p.state_pitch = evict_state_pitch(p.c.cap, row_bytes);
  at += aligned(static_cast<size_t>(units) * p.state_pitch * sizeof(int32_t));
  p.idx_wanted = p.idx != nullptr;
  if (!p.idx) p.idx = reinterpret_cast<int32_t *>(at);
  p.chunk_rows = evict_chunk_rows(row_bytes);
  // A workgroup for each chunk, up to where a few units alone fill the device; those of
  // units that keep everything, or fewer rows, end at once.
  const int64_t chunks = p.state_pitch - kEvictState;
  p.workers = static_cast<int>(chunks < kEvictWorkers ? chunks : kEvictWorkers);
  p.max_spins = kEvictSpins;
}

}  // namespace reco
