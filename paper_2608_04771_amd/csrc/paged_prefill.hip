// GQA attention of a run of new tokens over ragged units of a paged KV cache
// (gfx950): causal, with an optional sliding window and sinks.
//
//   token t of a sequence, at row p = L + t, sees the rows j <= p with
//   j < sinks or j > p - window;   out = softmax(scale <q, k_j>) v_j over them
//
// The n tokens' G query heads of one KV head make n * G query rows (row t * G + g),
// so a group shares its K and V.  A workgroup takes 128 of them, or 256, 32 a wave, and walks
// the key tiles that any of them sees: tiles of the cached rows (in pages), then tiles
// of the new rows (as the caller gives them; other workgroups put them into their
// pages).  Per tile a wave computes
//   S^T = K_tile . Q^T           (32 keys x 32 rows per block)
//   O^T += V_tile^T . P^T        (32 columns of the head x 32 rows per block)
// so that a row's softmax lies in two lanes, the values of S^T are the operand P^T as
// they are, and rescaling O needs nothing from other lanes.  Statistics and outputs
// are fp32; P alone is rounded to the cache's type, as its operand has to be.  Where
// there are few query rows, their key tiles are split over several workgroups and
// joined by the second kernel.
//
// Long runs are bound by the matrix units and what feeds them: 16,384 tokens of a 7B
// layer in a window of 4,096 take 860 us (the median; 838 at best), 980 TFLOP/s, where a
// large library product reaches 1,190 on the same card.  No one part is the rest: without the loads to
// LDS it takes 18% less, without the reads of K 18%, of V 6%, without the exponentials
// 6%.  64 rows a wave (half the LDS reads) need more registers than a wave has and copy
// (1,110 us on chunks that took 786 then); two tiles in flight by halves of a workgroup, 985.
// The careful pass over blocks with infinities or NaN (below) is compiled into the same
// kernel and costs every call registers: at head_dim 128 bf16 245 vector registers, 233
// without it, fp32 256 and 106 more in memory, 245 without; at 64 bf16 237 and 147, fp32 219
// and 169.
#include "paged_device.hpp"
#include "paged_tiles.hpp"

#include <type_traits>

namespace reco {

namespace {

using namespace tiles32;

constexpr int kRows = kPrefillRows;          // query rows of a workgroup
constexpr int kWaitLoads = 0x0f70;           // vmcnt(0)
constexpr float kSlack = 8.f;                // log2 units that a maximum may grow before O follows

// Which of the rows at and behind `base` the token at row pos does not see.  The bounds
// are taken relative to base once, so that rows compare as constants.
struct Hidden {
  int end, low, sinks;

  __device__ __forceinline__ Hidden(int base, int end_, int pos, int sinks_, int window)
      : end(min(end_, pos + 1) - base), low(window > 0 ? pos - window - base : -1 - base), sinks(sinks_ - base) {}
  __device__ __forceinline__ bool at(int c) const { return c >= end || (c <= low && c >= sinks); }
};

// What one unit's call sees: cached rows in tiles of KT from row 0, new rows in tiles
// of KT from row L.
template <int KT>
struct Run {
  int L, n, old_tiles;

  __device__ __forceinline__ Run(int len, int tokens) : L(len), n(tokens), old_tiles((len + KT - 1) / KT) {}
  __device__ __forceinline__ int tile_of(int row) const { return row < L ? row / KT : old_tiles + (row - L) / KT; }
  __device__ __forceinline__ int start(int tile) const { return tile < old_tiles ? tile * KT : L + (tile - old_tiles) * KT; }
  __device__ __forceinline__ int end(int tile) const { return min(start(tile) + KT, tile < old_tiles ? L : L + n); }
};

// What a block of query rows sees, as a list of tiles: the sinks', then those of its
// windows up to its last token.
template <int KT>
struct Seen {
  Run<KT> run;
  int lo, s_end;                             // rows [0, s_end) and [lo, ...)
  int sink_tiles, skip, total;

  __device__ __forceinline__ Seen(const Run<KT> &r, int t_lo, int t_hi, int sinks, int window) : run(r) {
    lo = window > 0 ? max(0, run.L + t_lo - window + 1) : 0;
    s_end = min(sinks, lo);
    const int first = run.tile_of(lo);
    sink_tiles = s_end > 0 ? min(run.tile_of(s_end - 1) + 1, first) : 0;
    skip = first - sink_tiles;
    total = run.tile_of(run.L + t_hi) + 1 - skip;
  }
  __device__ __forceinline__ int tile(int i) const { return i < sink_tiles ? i : i + skip; }
};

// Key tiles on their way to LDS, which loads fill without registers between.  Each
// lane holds the place of 16 rows of the list's tiles, so 64 / (KT / 16) tiles at a
// time; the table's entries of the batch after are on their way meanwhile.
template <typename T, int D, int NW = kWaves>
struct Stager {
  using C = Cfg<T, D, NW>;
  static constexpr int KT = C::keys;
  static constexpr int kGroups = KT / 16;
  static constexpr int kBatch = kWave / kGroups;   // tiles
  const unsigned char *k, *v, *knew, *vnew;
  const int32_t *table;
  const Seen<KT> &seen;
  int n_pages, shift, tokens, end, wave, lane;
  unsigned worst;                            // id, of rows that are cached
  uint64_t place;                            // of this lane's 16 rows: a byte offset
  int coming;                                // the entry for the same lane of the next batch
  unsigned koff[C::insts], voff[C::insts];   // within 16 rows

  // Tiles [.., end) of the list.
  __device__ __forceinline__ Stager(const PagedPrefillParams &p, size_t cunit, int unit, const Seen<KT> &seen_, int end_,
                                    int wave_, int lane_)
      : k(static_cast<const unsigned char *>(p.c.k)), v(static_cast<const unsigned char *>(p.c.v)),
        knew(static_cast<const unsigned char *>(p.k_new) + static_cast<size_t>(unit) * p.tokens * C::row_bytes),
        vnew(static_cast<const unsigned char *>(p.v_new) + static_cast<size_t>(unit) * p.tokens * C::row_bytes),
        table(p.c.pages + cunit * static_cast<size_t>(p.c.max_pages)), seen(seen_), n_pages(p.c.n_pages),
        shift(p.c.page_shift), tokens(p.tokens), end(end_), wave(wave_), lane(lane_), worst(0) {
    start();
  }
  // Before the list's first tile.
  __device__ __forceinline__ void start() {
#pragma unroll
    for (int i = 0; i < C::insts; ++i) place_in(i, piece(i) % 16 + lane / C::lanes_per_row);
  }

  // A wave's i-th load of a tile takes wave_rows rows from this one on.
  __device__ __forceinline__ int piece(int i) const { return (i * NW + wave) * C::wave_rows; }
  // Lane offsets of the i-th load, from row `in` of the 16.
  __device__ __forceinline__ void place_in(int i, int in) {
    const int row = piece(i) + lane / C::lanes_per_row, c = lane % C::lanes_per_row;
    koff[i] = in * C::row_bytes + (c ^ C::k_swap(row)) * 16;
    voff[i] = in * C::row_bytes + (c ^ C::v_swap(row)) * 16;
  }
  __device__ __forceinline__ int tile(int i) const { return seen.tile(min(i, end - 1)); }
  // This lane's tile of the batch that starts at tile i, and its rows there.
  __device__ __forceinline__ int row_of(int i, bool &old) const {
    const int t = tile(i + lane / kGroups);
    old = t < seen.run.old_tiles;
    return (old ? t : t - seen.run.old_tiles) * KT + lane % kGroups * 16;
  }
  __device__ __forceinline__ void ask(int i) {
    bool old;
    const int row = row_of(i, old);
    coming = old ? table[min(row, seen.run.L - 1) >> shift] : 0;
  }
  // The batch that starts at tile i, whose entries were asked for, and the one after.
  __device__ __forceinline__ void batch(int i) {
    bool old;
    const int row = row_of(i, old);
    worst = max(worst, static_cast<unsigned>(coming));
    const unsigned id = min(static_cast<unsigned>(coming), static_cast<unsigned>(n_pages - 1));
    const unsigned in = old ? row & ((1u << shift) - 1u) : min(row, (tokens - 1) & ~15);
    place = ((static_cast<uint64_t>(id) << shift) + in) * C::row_bytes;
    ask(i + kBatch);
  }
  // A tile's rows.  Those past its end are other rows of the pool or of the run.
  struct Place {
    const unsigned char *k, *v;
    uint64_t at[C::insts];
  };
  __device__ __forceinline__ Place find(int i) const {
    const int at_i = min(i, end - 1);
    const bool old = seen.tile(at_i) < seen.run.old_tiles;
    Place w{old ? k : knew, old ? v : vnew, {}};
#pragma unroll
    for (int j = 0; j < C::insts; ++j) {
      const int from = (at_i & (kBatch - 1)) * kGroups + piece(j) / 16;
      w.at[j] = static_cast<uint64_t>(static_cast<unsigned>(__builtin_amdgcn_readlane(static_cast<int>(place >> 32), from))) << 32 |
                static_cast<unsigned>(__builtin_amdgcn_readlane(static_cast<int>(place), from));
    }
    return w;
  }
  __device__ __forceinline__ void load_k(const Place &w, int j, unsigned char *buf) const {
    __builtin_amdgcn_global_load_lds((global_u32 *)(w.k + w.at[j] + koff[j]), (lds_u32 *)(buf + piece(j) * C::row_bytes), 16, 0, 0);
  }
  __device__ __forceinline__ void load_v(const Place &w, int j, unsigned char *buf) const {
    __builtin_amdgcn_global_load_lds((global_u32 *)(w.v + w.at[j] + voff[j]), (lds_u32 *)(buf + piece(j) * C::row_bytes), 16, 0, 0);
  }
  // Ahead of load(i): what seldom happens there, the places of a new batch ...
  __device__ __forceinline__ void turn(int i) {
    if (i < end && (i & (kBatch - 1)) == 0) batch(i);
  }
  // ... and the offsets of a run's last tile, whose rows past the last place must not be
  // read (no tile of the list comes after it).
  __device__ __forceinline__ void trim(int i) {
    const int t = tile(i);
    const int row0 = (t - seen.run.old_tiles) * KT;
    if (t < seen.run.old_tiles || row0 + KT <= tokens) return;
#pragma unroll
    for (int j = 0; j < C::insts; ++j) {
      const int base = min((row0 + piece(j)) & ~15, (tokens - 1) & ~15);
      place_in(j, min(piece(j) % 16 + lane / C::lanes_per_row, tokens - 1 - base));
    }
  }
  // Rows of V that no token of the block sees count for nothing, whatever they hold.
  __device__ __forceinline__ bool mixed(int i) const {
    const int t = tile(i);
    const int from = seen.run.start(t), to = seen.run.end(t);
    return to - from < KT || (from < seen.lo && to > seen.s_end);
  }
  __device__ __forceinline__ void clean(int i, unsigned char *vbuf) const {
    const int t = tile(i);
    const int from = seen.run.start(t), to = seen.run.end(t);
#pragma unroll
    for (int j = 0; j < C::insts; ++j) {
      const int row = from + piece(j) + lane / C::lanes_per_row;
      if (!(row < to && (row >= seen.lo || row < seen.s_end)))
        *reinterpret_cast<u32x4v *>(vbuf + piece(j) * C::row_bytes + lane * 16) = u32x4v{0, 0, 0, 0};
    }
  }
  // f(16 bytes) for what this lane loaded of V.
  template <typename F>
  __device__ __forceinline__ void each_piece(unsigned char *vbuf, F f) const {
#pragma unroll
    for (int j = 0; j < C::insts; ++j) f(*reinterpret_cast<u32x4v *>(vbuf + piece(j) * C::row_bytes + lane * 16));
  }
};

// Whether any of the values is an infinity or a NaN: all bits of its exponent are set.
template <typename T>
__device__ __forceinline__ bool odd_word(unsigned w) {
  if (sizeof(T) == 4) return (w & 0x7f800000u) == 0x7f800000u;
  return (w & 0x7f800000u) == 0x7f800000u || (w & 0x7f80u) == 0x7f80u;
}
template <typename T>
__device__ __forceinline__ unsigned even_word(unsigned w) {      // with zeros in their place
  if (sizeof(T) == 4) return odd_word<T>(w) ? 0u : w;
  return ((w & 0x7f800000u) == 0x7f800000u ? 0u : w & 0xffff0000u) | ((w & 0x7f80u) == 0x7f80u ? 0u : w & 0xffffu);
}

// A wave's 32 rows from row0 on, of `rows`, divided by their sums and written whole
// through LDS (`stage`: 32 rows of its own).  head0: query head 0 of the group.
template <typename T, int D>
__device__ __forceinline__ void write_rows(const PagedPrefillParams &p, unsigned char *stage,
                                           const f32x16_t (&o)[Cfg<T, D>::dtiles], float m, float l, size_t head0,
                                           int row0, int rows, int lane) {
  using C = Cfg<T, D>;
  const int half = lane >> 5, col = lane & 31;
  const float inv = l == 0.f ? 0.f : 1.f / l;
  const auto place = [&](int row) {
    const int t = p.by_group.of(row);
    return (head0 + (row - t * p.group)) * static_cast<size_t>(p.tokens) + t;
  };
#pragma unroll
  for (int dt = 0; dt < C::dtiles; ++dt) {
#pragma unroll
    for (int e = 0; e < 16; e += 4) {
      const int byte = (dt * 32 + acc_row(e, half)) * static_cast<int>(sizeof(T));
      T *at = reinterpret_cast<T *>(stage + col * C::row_bytes + (byte ^ ((col & 7) * 16)));
#pragma unroll
      for (int j = 0; j < 4; ++j) at[j] = from_f32<T>(o[dt][e + j] * inv);
    }
  }
  if (p.lse && half == 0 && row0 + col < rows) p.lse[place(row0 + col)] = l == 0.f ? -INFINITY : (m + log2f(l)) * kLn2;
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
#pragma unroll
  for (int k = 0; k < 32 / C::wave_rows; ++k) {
    const int in = k * C::wave_rows + lane / C::lanes_per_row;
    if (row0 + in >= rows) break;
    reinterpret_cast<u32x4v *>(p.out)[place(row0 + in) * C::lanes_per_row + lane % C::lanes_per_row] =
        *reinterpret_cast<const u32x4v *>(stage + in * C::row_bytes + ((lane % C::lanes_per_row) ^ (in & 7)) * 16);
  }
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
}

// Puts rows [first, first + kAppendRows) of a unit's run into their pages; a unit's rows are
// appended together or, where they or their pages do not fit, not at all.  The rows come
// while it is found out where they go.  Attention may go on meanwhile: it has no use for
// rows of the cache past L (against a kernel after the attention, prompts of 200 to 512
// tokens take 4 us less of 39 per call, 16,384 tokens 6 us more of 850).  Returns whether the unit's rows
// are stored.
constexpr int kAppendRows = kPrefillAppendRows;

template <typename T, int D, int NT>
__device__ __forceinline__ bool append_run(const PagedPrefillParams &p, int unit, int first, int L) {
  const int tid = threadIdx.x;
  constexpr int kLanes = D * (int)sizeof(T) / 16, kEach = kAppendRows * kLanes / NT;
  u32x4v k[kEach], v[kEach];
#pragma unroll
  for (int i = 0; i < kEach; ++i) {
    const int row = min(first + (tid + i * NT) / kLanes, p.tokens - 1);
    const size_t at = (static_cast<size_t>(unit) * p.tokens + row) * kLanes + tid % kLanes;
    k[i] = reinterpret_cast<const u32x4v *>(p.k_new)[at];
    v[i] = reinterpret_cast<const u32x4v *>(p.v_new)[at];
  }
  const size_t cunit = p.c.unit(unit);
  const int given = p.n_new ? p.n_new[p.c.sequence(unit)] : p.tokens;
  const int n = given < 0 || given > p.tokens ? 0 : given;
  if (first >= n || L < 0 || L > p.c.cap) return false;
  const bool reporting = first == 0 && tid == 0;
  if (n > p.c.cap - L) {
    if (reporting) report(p.c.dev_err, kDevAppendOverflow);
    return false;
  }
  const int32_t *table = p.c.pages + cunit * static_cast<size_t>(p.c.max_pages);
  const int shift = p.c.page_shift;
  int id[kEach];
#pragma unroll
  for (int i = 0; i < kEach; ++i) id[i] = table[min(L + first + (tid + i * NT) / kLanes, L + n - 1) >> shift];
  bool bad = false;
  for (int g = (L >> shift) + tid; g <= (L + n - 1) >> shift; g += NT)
    if (static_cast<unsigned>(table[g]) >= static_cast<unsigned>(p.c.n_pages)) bad = true;
  if (__syncthreads_or(bad)) {
    if (reporting) report(p.c.dev_err, kDevBadPage);
    return false;
  }
#pragma unroll
  for (int i = 0; i < kEach; ++i) {
    const int t = first + (tid + i * NT) / kLanes;
    if (t >= n) break;
    const size_t at = ((static_cast<size_t>(id[i]) << shift) + ((L + t) & ((1 << shift) - 1))) * kLanes + tid % kLanes;
    reinterpret_cast<u32x4v *>(p.c.k)[at] = k[i];
    reinterpret_cast<u32x4v *>(p.c.v)[at] = v[i];
  }
  if (p.c.weight && tid < kAppendRows && first + tid < n) p.c.weight[cunit * p.c.cap + L + first + tid] = 0.f;
  return true;
}

template <typename T, int D, int NW>
__global__ __launch_bounds__(NW * kWave, 2) void prefill_kernel(PagedPrefillParams p) {
  using C = Cfg<T, D, NW>;
  using In = Stager<T, D, NW>;
  constexpr int kRows = 32 * NW;
  using M = Mma32<T>;
  using frag = typename M::frag;
  constexpr int KT = C::keys;
  // arrays of their own, so that reads of one need not wait for loads into another
  __shared__ __attribute__((aligned(1024))) unsigned char k0[C::stage], v0[C::stage], k1[C::stage], v1[C::stage];

  const int lane = threadIdx.x & (kWave - 1);
  const int wave = __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x) / kWave);
  const int half = lane >> 5;
  const int col = lane & 31;
  const int units = p.c.n_layers * p.c.batch * p.c.hkv;
  // Workgroups go to the XCDs in turn.  Where there are many, a piece of a unit's blocks,
  // which see mostly the same keys, takes its turn on one XCD and shares its L2.
  // Where there are few, all units' longest blocks come first (768 fp32 blocks, 1.5 rounds
  // of two on a compute unit: 330 -> 230 us; 256 in two splits each, all at once: 54 -> 47),
  // unless a unit is rather splits than blocks, which then lie together (48 uneven units of
  // 2 blocks in 5 splits: 61 us, 68 the other way).
  int unit = blockIdx.y, block = blockIdx.x, split = 0;
  int chunk = -1;                                        // of the rows to append, after all blocks
  if (p.pieces > 0) {
    const int attending = (units * p.pieces + kXcds - 1) / kXcds * kXcds * p.near;
    const int slot = blockIdx.x / kXcds;
    const int turn = p.by_near.of(slot), pos = p.by_near.rest(slot);
    const int piece = turn * kXcds + blockIdx.x % kXcds;
    unit = piece / p.pieces;
    block = p.spread ? piece % p.pieces + p.pieces * pos : piece % p.pieces * p.near + pos;
    const int more = static_cast<int>(blockIdx.x) - attending;
    if (more >= 0) {
      unit = more % units;
      chunk = more / units;
    } else if (unit >= units || block >= p.blocks) {
      return;
    }
  } else if (p.splits == 1 || p.blocks > p.splits) {
    unit = p.by_splits.of(blockIdx.x);
    block = blockIdx.y;
    split = p.by_splits.rest(blockIdx.x);
    if (block >= p.blocks) chunk = block - p.blocks;
  } else {
    block = p.by_splits.of(blockIdx.x);
    split = p.by_splits.rest(blockIdx.x);
  }
  if (chunk >= 0) {
    append_run<T, D, NW * kWave>(p, unit, chunk * kAppendRows, p.c.len[p.c.unit(unit)]);
    return;
  }
  block = p.blocks - 1 - block;                          // the longest first
  const size_t cunit = p.c.unit(unit);

  const int len_in = p.c.len[cunit];
  const int given = p.n_new ? p.n_new[p.c.sequence(unit)] : p.tokens;
  const int n = given < 0 || given > p.tokens ? 0 : given;
  if (block == 0 && split == 0 && threadIdx.x == 0) {
    p.len_in[unit] = len_in;                               // for the second kernel, which changes len
    if (len_in < 0 || len_in > p.c.cap || n != given) report(p.c.dev_err, kDevBadLength);
  }
  const int G = p.group;
  const int r0 = block * kRows;
  if (r0 >= n * G) return;
  const Run<KT> run(len_in < 0 ? 0 : min(len_in, p.c.cap), n);
  const int L = run.L;
  const int t_lo = p.by_group.of(r0), t_hi = p.by_group.of(min(r0 + kRows - 1, n * G - 1));

  const Seen<KT> seen(run, t_lo, t_hi, p.sinks, p.window);
  const int per_split = p.by_splits.of(seen.total + p.splits - 1);
  const int i0 = split * per_split;
  const int i1 = min(seen.total, i0 + per_split);

  // This lane's query row.
  const int r = r0 + wave * 32 + col;
  const int t = p.by_group.of(min(r, p.tokens * G - 1));
  const int pos = L + t;
  const size_t head0 = static_cast<size_t>(unit) * G;
  const size_t qrow = (head0 + (min(r, p.tokens * G - 1) - t * G)) * static_cast<size_t>(p.tokens) + t;
  frag qf[C::qk_steps];
  {
    const T *src = reinterpret_cast<const T *>(p.q) + qrow * D + half * (D / 2);
#pragma unroll
    for (int c = 0; c < C::qk_steps; ++c) {
      qf[c] = load_frag(src + c * M::kpl);
      if (p.scale_log2 < 0.f) qf[c] = M::negated(qf[c]);   // so that the largest product is the largest logit
    }
  }
  const float scale = fmaxf(fabsf(p.scale_log2), 0x1p-126f);   // times a hidden row's -inf, 0 would be NaN

  In in(p, cunit, unit, seen, i1, wave, lane);

  float m_run, l_run;                                    // m in units of the scaled logits
  f32x16_t o[C::dtiles];
  const int kat = k_base<T, D>(lane), vat = v_base<T, D>(lane);
  __shared__ int s_odd[2][NW];

  // A token that does not see a row gives it the weight 0, which makes a NaN of an
  // infinity or a NaN.  Tiles that not all tokens see whole are looked through for such
  // values; where there are any, the block is done once more, carefully: they are taken
  // out of the tile, and what they give is added for each of the wave's tokens apart.
  // (A branch in the ordinary loop costs it 4%: 902 -> 942 us for 16,384 tokens of a 7B
  // layer in a window of 4,096.)
  bool odd = false;
  const auto add_odd = [&](unsigned char *vbuf, f32x16_t (&s)[C::blocks], int start, int end,
                           float ref) __attribute__((always_inline)) {
    constexpr int kParts = C::blocks * C::pv_steps;
    const int w0 = min(r0 + wave * 32, p.tokens * G - 1), w1 = min(r0 + wave * 32 + 31, p.tokens * G - 1);
    for (int u = p.by_group.of(w0); u <= p.by_group.of(w1); ++u) {
      const Hidden hidden(start + 4 * half, end, L + u, p.sinks, p.window);
#pragma unroll
      for (int dt = 0; dt < C::dtiles; ++dt) {
        f32x16_t sum;
#pragma unroll
        for (int e = 0; e < 16; ++e) sum[e] = 0.f;
#pragma unroll
        for (int q = 0; q < kParts; ++q) {
          const int row = M::kpl == 8 ? 16 * q : 8 * (q / 4) + q % 4;
          frag vf = v_frag32<T, D>(vbuf + (vat ^ (dt * 32 * (int)sizeof(T))) + row * C::row_bytes), pf;
#pragma unroll
          for (int j = 0; j < M::kpl; ++j) {
            const int e = q * M::kpl + j;
            const float w = fast_exp2(fmaf(s[e / 16][e % 16], scale, -ref));
            const bool counts = !hidden.at(acc_row(e, 0));
            if constexpr (M::kpl == 1) {
              vf = counts && odd_word<T>(__float_as_uint(vf)) ? vf : 0.f;
              pf = w;
            } else {
              const __bf16 x = vf[j];
              vf[j] = counts && odd_word<T>(__builtin_bit_cast(unsigned short, x)) ? x : static_cast<__bf16>(0.f);
              pf[j] = static_cast<__bf16>(w);
            }
          }
          sum = M::mma(vf, pf, sum);
        }
#pragma unroll
        for (int e = 0; e < 16; ++e) o[dt][e] = t == u ? o[dt][e] + sum[e] : o[dt][e];
      }
    }
  };

  // Tile i, in kbuf and vbuf once its loads are done; tile i + 1 goes to kto and vto.
  const auto step = [&](auto careful, int i, unsigned char *kbuf, unsigned char *vbuf, unsigned char *kto,
                        unsigned char *vto) __attribute__((always_inline)) {
    constexpr bool kCareful = decltype(careful)::value;
    in.turn(i + 1);
    in.trim(i + 1);
    const int tile = seen.tile(i);
    const int start = run.start(tile), end = run.end(tile);
    // Whether every token of the block sees the whole tile.
    const bool whole = end - start == KT && end - 1 <= L + t_lo &&
                       (p.window == 0 || start > L + t_hi - p.window || end <= p.sinks);
    __builtin_amdgcn_s_waitcnt(kWaitLoads);
    if (!whole) {                                         // each wave looks after what it loaded
      if (in.mixed(i)) in.clean(i, vbuf);
      if (kCareful) odd = false;
      in.each_piece(vbuf, [&](const u32x4v &x) { odd |= odd_word<T>(x[0]) | odd_word<T>(x[1]) | odd_word<T>(x[2]) | odd_word<T>(x[3]); });
      if (kCareful && lane == 0) s_odd[i & 1][wave] = 0;
      if (kCareful && odd) s_odd[i & 1][wave] = 1;
    }
    __syncthreads();                                      // tile i is there, and no one reads tile i - 1

    // S^T, with operands read ahead of their products, and between the products the
    // next tile asked for, piece by piece.
    f32x16_t s[C::blocks];
#pragma unroll
    for (int kb = 0; kb < C::blocks; ++kb) {
#pragma unroll
      for (int e = 0; e < 16; ++e) s[kb][e] = 0.f;
    }
    constexpr int kSteps = C::blocks * C::qk_steps, kAhead = M::kpl == 8 ? 8 : 16, kEach = kSteps / C::insts;
    const typename In::Place from = in.find(i + 1);
    frag kf[2][kAhead];
    const auto read_k = [&](int q) {
#pragma unroll
      for (int c = 0; c < kAhead; ++c) {
        const int z = q * kAhead + c, b = z % C::qk_steps * M::kpl * (int)sizeof(T);
        kf[q & 1][c] = load_frag(reinterpret_cast<const T *>(kbuf + (kat ^ (b & ~15)) + (b & 15) + z / C::qk_steps * 32 * C::row_bytes));
      }
    };
    read_k(0);
#pragma unroll
    for (int z = 0; z < kSteps; ++z) {
      if (z % kAhead == 0 && z + kAhead < kSteps) read_k(z / kAhead + 1);
      if (z % kAhead == 0) __builtin_amdgcn_sched_barrier(0);
      s[z / C::qk_steps] = M::mma(kf[z / kAhead & 1][z % kAhead], qf[z % C::qk_steps], s[z / C::qk_steps]);
      if (z % kEach == 0) {
        in.load_k(from, z / kEach, kto);
        in.load_v(from, z / kEach, vto);
      }
      __builtin_amdgcn_sched_barrier(0);
    }
    constexpr int kParts = C::blocks * C::pv_steps;
    frag vf[2][C::dtiles];
    const auto read_v = [&](int q) {
      const int row = M::kpl == 8 ? 16 * q : 8 * (q / 4) + q % 4;
#pragma unroll
      for (int dt = 0; dt < C::dtiles; ++dt)
        vf[q & 1][dt] = v_frag32<T, D>(vbuf + (vat ^ (dt * 32 * (int)sizeof(T))) + row * C::row_bytes);
    };
    read_v(0);

    if (!whole) {
      const Hidden hidden(start + 4 * half, end, pos, p.sinks, p.window);
#pragma unroll
      for (int kb = 0; kb < C::blocks; ++kb) {
#pragma unroll
        for (int e = 0; e < 16; ++e) s[kb][e] = hidden.at(kb * 32 + acc_row(e, 0)) ? -INFINITY : s[kb][e];
      }
    }
    float top = -INFINITY;
#pragma unroll
    for (int kb = 0; kb < C::blocks; ++kb) {
#pragma unroll
      for (int e = 0; e < 16; ++e) top = fmaxf(top, s[kb][e]);
    }
    top = fmaxf(top, shfl_xor(top, 32)) * scale;
    // The reference of the exponentials follows the maximum only where it grew by more
    // than kSlack (P then stays below 2^kSlack, with the same relative precision), so
    // that O is seldom rescaled.
    if (__any(top > m_run + kSlack)) {
      const float m_new = fmaxf(m_run, top);
      const float alpha = fast_exp2(m_run - (m_new == -INFINITY ? 0.f : m_new));
      l_run *= alpha;
      m_run = m_new;
#pragma unroll
      for (int dt = 0; dt < C::dtiles; ++dt) {
#pragma unroll
        for (int e = 0; e < 16; ++e) o[dt][e] *= alpha;
      }
    }
    // O^T: part q takes kpl elements of every lane, slot j of which is row
    // 8 (e / 4) + 4 half + e % 4 of S^T for e = q * kpl + j; the exponentials of a part
    // lie between the products of the part before.
    const float ref = m_run == -INFINITY ? 0.f : m_run;
    if (kCareful && !whole) {
      int any = 0;
#pragma unroll
      for (int w = 0; w < NW; ++w) any |= s_odd[i & 1][w];
      if (any) {                                          // the same for the workgroup
        add_odd(vbuf, s, start, end, ref);
        __syncthreads();
        in.each_piece(vbuf, [](u32x4v &x) { x = u32x4v{even_word<T>(x[0]), even_word<T>(x[1]), even_word<T>(x[2]), even_word<T>(x[3])}; });
        __syncthreads();
        read_v(0);
      }
    }
    const auto weigh = [&](int q, int j) {
      const int e = q * M::kpl + j;
      const float w = fast_exp2(fmaf(s[e / 16][e % 16], scale, -ref));
      l_run += w;
      return w;
    };
    frag pf[2];
    const auto put = [&](int q, int j) {
      if constexpr (M::kpl == 1) pf[q & 1] = weigh(q, j);
      else pf[q & 1][j] = static_cast<__bf16>(weigh(q, j));
    };
#pragma unroll
    for (int j = 0; j < M::kpl; ++j) put(0, j);
#pragma unroll
    for (int q = 0; q < kParts; ++q) {
      if (q + 1 < kParts) read_v(q + 1);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int dt = 0; dt < C::dtiles; ++dt) {
        o[dt] = M::mma(vf[q & 1][dt], pf[q & 1], o[dt]);
        if (q + 1 < kParts) {
#pragma unroll
          for (int j = dt * M::kpl / C::dtiles; j < (dt + 1) * M::kpl / C::dtiles; ++j) put(q + 1, j);
        }
        __builtin_amdgcn_sched_barrier(0);
      }
    }
  };
  const auto walk = [&](auto careful) __attribute__((always_inline)) {
    m_run = -INFINITY;
    l_run = 0.f;
#pragma unroll
    for (int dt = 0; dt < C::dtiles; ++dt) {
#pragma unroll
      for (int i = 0; i < 16; ++i) o[dt][i] = 0.f;
    }
    if (i0 < i1) {
      in.ask(i0 & -In::kBatch);
      in.batch(i0 & -In::kBatch);
      in.trim(i0);
      const typename In::Place from = in.find(i0);
#pragma unroll
      for (int j = 0; j < C::insts; ++j) {
        in.load_k(from, j, k0);
        in.load_v(from, j, v0);
      }
      for (int i = i0; i < i1; i += 2) {
        step(careful, i, k0, v0, k1, v1);
        if (i + 1 < i1) step(careful, i + 1, k1, v1, k0, v0);
      }
    }
    __builtin_amdgcn_s_waitcnt(kWaitLoads);
  };
  walk(std::false_type{});
  if (__syncthreads_or(odd)) {
    in.start();
    walk(std::true_type{});
    __syncthreads();
  }
  if (in.worst >= static_cast<unsigned>(p.c.n_pages)) report(p.c.dev_err, kDevBadPage);

  const float l_tot = l_run + shfl_xor(l_run, 32);
  if (p.splits > 1) {
    // partials stay in the lanes' order, so that they are written and read whole
    const size_t part = (static_cast<size_t>(unit) * p.blocks + block) * p.splits + split;
    if (half == 0) {
      p.part_ml[part * 2 * kRows + wave * 32 + col] = m_run;
      p.part_ml[part * 2 * kRows + kRows + wave * 32 + col] = l_tot;
    }
    float4 *po = reinterpret_cast<float4 *>(p.part_o + (part * kRows + wave * 32) * D) + lane;
#pragma unroll
    for (int dt = 0; dt < C::dtiles; ++dt) {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        po[(dt * 4 + e) * kWave] = make_float4(o[dt][4 * e], o[dt][4 * e + 1], o[dt][4 * e + 2], o[dt][4 * e + 3]);
    }
    return;
  }
  unsigned char *mine = wave < NW / 2 ? (wave < NW / 4 ? k0 : v0) : (wave < 3 * NW / 4 ? k1 : v1);
  write_rows<T, D>(p, mine + wave % (NW / 4) * 32 * C::row_bytes, o, m_run, l_tot, head0,
                   r0 + wave * 32, n * G, lane);
}

// Where there are splits: joins them (workgroups [0, merges) of a unit) and puts the new
// rows into their pages (the others).
constexpr int kMergeRows = 32;               // a wave's rows, and a quarter of a 32-column block each thread

template <typename T, int D>
__global__ __launch_bounds__(256) void prefill_finish_kernel(PagedPrefillParams p, int merges) {
  const int tid = threadIdx.x;
  const int G = p.group;
  const int unit = blockIdx.y;
  if (static_cast<int>(blockIdx.x) < merges) {
    constexpr int kDt = D / 32;
    const int dt = blockIdx.x % kDt, w32 = blockIdx.x / kDt % (kRows / kMergeRows);
    const int block = blockIdx.x / (kDt * (kRows / kMergeRows));
    const int given = p.n_new ? p.n_new[p.c.sequence(unit)] : p.tokens;
    const int n = given < 0 || given > p.tokens ? 0 : given;
    if (block * kRows + w32 * kMergeRows >= n * G) return;
    // The splits' weights of the rows: eight threads a row.
    __shared__ float s_w[kPrefillMaxSplits][kMergeRows];
    const size_t part = (static_cast<size_t>(unit) * p.blocks + block) * p.splits;
    const int lane = tid & (kWave - 1);
    {
      constexpr int kPer = 256 / kMergeRows, kEach = kPrefillMaxSplits / kPer;
      const int row_of = tid / kPer, sub = tid % kPer;
      const float *ml = p.part_ml + part * 2 * kRows + w32 * kMergeRows + row_of;
      float m[kEach], l[kEach];
      float top = -INFINITY, sum = 0.f;
#pragma unroll
      for (int i = 0; i < kEach; ++i) {
        const int s = sub + i * kPer;
        m[i] = s < p.splits ? ml[static_cast<size_t>(s) * 2 * kRows] : -INFINITY;
        l[i] = s < p.splits ? ml[static_cast<size_t>(s) * 2 * kRows + kRows] : 0.f;
        top = fmaxf(top, m[i]);
      }
#pragma unroll
      for (int d = 1; d < kPer; d <<= 1) top = fmaxf(top, shfl_xor(top, d));
      const float ref = top == -INFINITY ? 0.f : top;
#pragma unroll
      for (int i = 0; i < kEach; ++i) {
        m[i] = fast_exp2(m[i] - ref);
        sum += l[i] * m[i];
      }
#pragma unroll
      for (int d = 1; d < kPer; d <<= 1) sum += shfl_xor(sum, d);
      const float inv = sum == 0.f ? 0.f : 1.f / sum;
#pragma unroll
      for (int i = 0; i < kEach; ++i) s_w[sub + i * kPer][row_of] = m[i] * inv;
      const int r = block * kRows + w32 * kMergeRows + row_of;
      if (p.lse && dt == 0 && sub == 0 && r < n * G)
        p.lse[(static_cast<size_t>(unit) * G + p.by_group.rest(r)) * static_cast<size_t>(p.tokens) + p.by_group.of(r)] =
            sum == 0.f ? -INFINITY : (ref + log2f(sum)) * kLn2;
    }
    __syncthreads();
    const int row_of = lane & 31, e = tid / kWave;
    const int r = block * kRows + w32 * kMergeRows + row_of;
    const float4 *po = reinterpret_cast<const float4 *>(p.part_o + (part * kRows + w32 * kMergeRows) * D) +
                       (dt * 4 + e) * kWave + lane;
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 8
    for (int s = 0; s < p.splits; ++s) {
      const float w = s_w[s][row_of];
      const float4 x = po[static_cast<size_t>(s) * kRows * (D / 4)];
      acc.x += x.x * w;
      acc.y += x.y * w;
      acc.z += x.z * w;
      acc.w += x.w * w;
    }
    if (r >= n * G) return;
    const int t = p.by_group.of(r);
    const size_t row = (static_cast<size_t>(unit) * G + (r - t * G)) * static_cast<size_t>(p.tokens) + t;
    T *dst = reinterpret_cast<T *>(p.out) + row * D + dt * 32 + acc_row(4 * e, lane >> 5);
    dst[0] = from_f32<T>(acc.x);
    dst[1] = from_f32<T>(acc.y);
    dst[2] = from_f32<T>(acc.z);
    dst[3] = from_f32<T>(acc.w);
    return;
  }
  const int first = (blockIdx.x - merges) * kAppendRows, L = p.len_in[unit];
  if (append_run<T, D, 256>(p, unit, first, L) && first == 0 && tid == 0)
    p.c.len[p.c.unit(unit)] = L + (p.n_new ? p.n_new[p.c.sequence(unit)] : p.tokens);
}

// Where there are none, the first kernel's last workgroups have put the rows, and what
// is left are the lengths, which no one reads any more.
__global__ __launch_bounds__(kWave) void prefill_len_kernel(PagedPrefillParams p) {
  const int unit = blockIdx.x;
  const size_t cunit = p.c.unit(unit);
  const int L = p.c.len[cunit];
  const int n = p.n_new ? p.n_new[p.c.sequence(unit)] : p.tokens;
  if (n < 1 || n > p.tokens || L < 0 || L > p.c.cap || n > p.c.cap - L) return;
  const int32_t *table = p.c.pages + cunit * static_cast<size_t>(p.c.max_pages);
  bool bad = false;
  for (int g = (L >> p.c.page_shift) + threadIdx.x; g <= (L + n - 1) >> p.c.page_shift; g += kWave)
    bad |= static_cast<unsigned>(table[g]) >= static_cast<unsigned>(p.c.n_pages);
  if (!__any(bad) && threadIdx.x == 0) p.c.len[cunit] = L + n;
}

template <typename T, int D>
hipError_t launch_typed(const PagedPrefillParams &p, hipStream_t s) {
  const int units = p.c.n_layers * p.c.batch * p.c.hkv;
  const int chunks = (p.tokens + kAppendRows - 1) / kAppendRows;
  const dim3 grid = p.pieces > 0 ? dim3((units * p.pieces + kXcds - 1) / kXcds * kXcds * p.near + units * chunks)
                    : p.splits == 1 ? dim3(units, p.blocks + chunks)
                    : p.blocks > p.splits ? dim3(units * p.splits, p.blocks) : dim3(p.blocks * p.splits, units);
  if constexpr (sizeof(T) == 2) {
    if (p.rows == kPrefillLongRows)
      hipLaunchKernelGGL((prefill_kernel<T, D, 8>), grid, dim3(8 * kWave), 0, s, p);
  }
  if (p.rows == kRows)
    hipLaunchKernelGGL((prefill_kernel<T, D, 4>), grid, dim3(4 * kWave), 0, s, p);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  if (p.splits > 1) {
    const int merges = p.blocks * (kRows / kMergeRows) * (D / 32);
    hipLaunchKernelGGL((prefill_finish_kernel<T, D>), dim3(merges + chunks, units), dim3(256), 0, s, p, merges);
  } else {
    hipLaunchKernelGGL(prefill_len_kernel, dim3(units), dim3(kWave), 0, s, p);
  }
  return hipGetLastError();
}

}  // namespace

hipError_t launch_paged_prefill(const PagedPrefillParams &p, int dtype, int head_dim, hipStream_t s) {
  if (dtype == 0) {
    if (head_dim == 64) return launch_typed<float, 64>(p, s);
    return launch_typed<float, 128>(p, s);
  }
  if (head_dim == 64) return launch_typed<bf16_t, 64>(p, s);
  return launch_typed<bf16_t, 128>(p, s);
}

}  // namespace reco
