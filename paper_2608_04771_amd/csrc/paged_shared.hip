// GQA attention of one new token of every sequence over a paged KV cache (gfx950), where
// sequences come in groups whose first rows are the same ones:
//
//   out = softmax(scale <q, k_j>) v_j over the rows j that the token sees,
//   rows j < shared[group] being those of the group's first sequence.
//
// Softmax over two sets of rows is joined from each set's (max, sum, output), so a group's
// query rows (sequence * G + head, of one layer and KV head) take the rows that all of
// them see together, once, and each unit its other rows alone:
//   common  [0, min(sinks, c)) and [c, shared), c the largest window start of the group
//   own     [max(lo, sinks), c) of the shared rows, the rows from `shared` on, the new one
// One launch has both kinds of workgroups, so that neither kind's last ones leave the
// device idle; the second joins their parts and commits the append.
//
// The common part has 128 query rows a workgroup, 32 a wave, and key tiles (64 rows of bf16, 32 of
// fp32) that the waves share through LDS,
//   S^T = K_tile . Q^T (32 keys x 32 rows),   O^T += V_tile^T . P^T.
// The own part has 16 padded query heads and tiles of 32 keys that are a wave's own.
// Statistics and outputs are fp32; P alone is rounded to the cache's type, as its operand
// has to be: a weight is off by half a step, 2^-8 of it at most.
//
// What bounds it, per call (both kernels, and the least time of its bytes at 6.6 TB/s):
//   32 sequences of 28 heads on 4, 16,384 common rows and 256 to 2,048 own ones, 8 layers: 877 MB,
//   161 + 8 us, 133: memory.  The two blocks of query rows read the common rows at 1.0 times
//   their bytes from memory and again from L2, 7 TB/s into the units together; the matrix
//   units work in 19% of the cycles, the vector units in 23, both in 5.
//   16 sequences in 4 groups, window 4,096, 4 layers: 368 MB, 75 + 5 us, 56: 426 MB, since the
//   common rows begin at the group's last window start, and what lies between a sequence's own
//   start and that one it reads alone (a choice: rows that some do not see would have to be
//   masked by each query row's start, and kept from its sums in V); and the ends of ragged groups.
//   128 sequences of 32 heads, 4,096 common rows and up to 400 own ones: 125 MB and 9 GFLOP,
//   32 + 7 us, 19: products, exponentials and loads in turn, and 4,096 rows of 8 parts and more.
//   8 sequences, 8,190 common rows: 62 MB, 16 + 5 us, 9.3: the way to the first tile (lengths,
//   page ids, keys: three round trips, 4 us) and the last one's way out.
// fp32 is bound by its products, a sixteenth of bf16's rate: where a block has up to 64 query rows, the
// waves that would have none share the others' (21 sequences in 8 groups, 15,366 rows: 596 us with
// one wave at work, 367).  Of fp32 rows of 128, 43 registers are kept in memory.
// Not kept: 256 query rows and 8 waves a workgroup with four stages (200 us for the first call, 188
// then), 32-key tiles in bf16 and three waves a SIMD (410, by registers in memory), own rows two
// tiles ahead (233, likewise), one wave's own rows as items of their own (181 to 185), and a
// priority of its own for either kind of workgroup (no difference).
#include "paged_device.hpp"
#include "paged_tiles.hpp"

namespace reco {

namespace {

constexpr int kNW = 4;                       // waves of a workgroup
constexpr int kRows = kSharedRows;           // query rows of one
static_assert(kRows == 32 * kNW, "32 rows a wave");
constexpr int kMix = 32;                     // compute units of an XCD (by 1: 217 us, by 16 or 64: the same)
constexpr int wait_loads(int n) { return 0x0f70 | (n & 15) | (n >> 4) << 14; }   // vmcnt(n)
constexpr float kSlack = 8.f;                // log2 units that a maximum may grow before O follows

// Loads to LDS of 16 or 4 bytes a lane, from `from` (the same in all lanes) + `at`, to the LDS
// address `to` on.  In assembly, because the compiler makes reads of LDS wait for all loads
// of its own kind that are on their way there; these are waited for by their number, and its
// own waits for other loads only become longer by them.  No register receives anything.
__device__ __forceinline__ void load_to_lds16(const void *from, unsigned at, unsigned to) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(to), "v"(at), "s"(from) : "m0");
}
__device__ __forceinline__ void load_to_lds4(const void *from, unsigned at, unsigned to) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, %2" ::"s"(to), "v"(at), "s"(from) : "m0", "memory");
}
__device__ __forceinline__ unsigned lds_address(const void *p) {
  return __builtin_amdgcn_readfirstlane(static_cast<unsigned>(reinterpret_cast<uintptr_t>((const __attribute__((address_space(3))) unsigned char *)p)));
}
// A barrier for what waves have waited for themselves (__syncthreads waits for all loads).
__device__ __forceinline__ void barrier() {
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// f over all 64 lanes, by the vector unit alone (a shuffle goes through the LDS unit, some
// 100 cycles each, which every workgroup would wait for before its first load).
template <typename F>
__device__ __forceinline__ int wave_all(int v, F f) {
  const float x = wave_fold(__int_as_float(v), [&](float a, float b) { return __int_as_float(f(__float_as_int(a), __float_as_int(b))); });
  return __builtin_amdgcn_readfirstlane(__float_as_int(x));
}

// What a workgroup needs first, asked for at once where it fits a wave: the list of groups,
// their counts of shared rows and the lengths of a layer's and KV head's units.
struct Asked {
  int from, to, shared, len;
};
__device__ __forceinline__ int ask_len(const PagedSharedParams &p, int layer, int head, int b) {
  return p.c.len[p.c.unit((layer * p.c.batch + b) * p.c.hkv + head)];
}
__device__ __forceinline__ Asked ask_first(const PagedSharedParams &p, int layer, int head, int lane) {
  Asked a;
  a.from = p.first[min(lane, p.groups)];
  a.to = p.first[min(lane + 1, p.groups)];
  a.shared = p.shared[layer * p.shared_stride + min(lane, p.groups - 1)];
  a.len = ask_len(p, layer, head, min(lane, p.c.batch - 1));
  return a;
}

// Whether the list of groups ascends from 0 to the batch.
__device__ __forceinline__ bool groups_ascend(const PagedSharedParams &p, int from0, int to0, int lane) {
  const auto good = [&](int i, int from, int to) {
    return i >= p.groups || (from <= to && from >= 0 && to <= p.c.batch && (i > 0 || from == 0) && (i + 1 < p.groups || to == p.c.batch));
  };
  bool ok = good(lane, from0, to0);
#pragma unroll 4
  for (int i = kWave + lane; i < p.groups; i += kWave) ok = ok & good(i, p.first[i], p.first[i + 1]);
  return __all(ok);
}

// One group of sequences [from, to), and its place in the list.
struct Group {
  int id, from, to;
  int row0;             // of the block that was looked for
};

// The group of block `block` (of kRows query rows each, groups in order) of a list that ascends;
// id is -1 where there is none.  A group's blocks begin where all before it would end, had each
// kRows - 1 rows more, so that no one has to count them.
__device__ __forceinline__ Group find_group(const PagedSharedParams &p, const Asked &asked, int block, int lane) {
  const auto begins = [&](int id, int from) { return (from * p.group + id * (kRows - 1)) / kRows; };
  Group g;
  if (p.groups <= kWave) {
    const uint64_t here = __ballot(lane < p.groups && block >= begins(lane, asked.from) && block < begins(lane + 1, asked.to));
    if (here == 0) return Group{-1, 0, 0, 0};
    g.id = __builtin_ctzll(here);
    g.from = __builtin_amdgcn_readlane(asked.from, g.id);
    g.to = __builtin_amdgcn_readlane(asked.to, g.id);
  } else {
    int low = 0, high = p.groups - 1;                     // the last group that begins here or before
    while (low < high) {
      const int mid = (low + high + 1) / 2;
      if (begins(mid, p.first[mid]) <= block) low = mid;
      else high = mid - 1;
    }
    g = Group{low, p.first[low], p.first[low + 1], 0};
  }
  g.row0 = (block - begins(g.id, g.from)) * kRows;
  if (g.row0 >= (g.to - g.from) * p.group) g.id = -1;
  return g;
}

// What the sequences of a group see together of one layer and KV head.
struct Common {
  int rows;             // shared ones
  int sinks, start;     // [0, sinks) and [start, rows)
};

__device__ __forceinline__ Common common_rows(const PagedSharedParams &p, const Asked &asked, const Group &g, int layer,
                                              int head, int lane, bool reporting) {
  const int extra = p.k_new ? 1 : 0;
  int least = p.c.cap, start = 0;
  const auto count = [&](int len) {
    const int n = max(0, min(len, p.c.cap));
    least = min(least, n);
    if (p.window > 0) start = max(start, n + extra - p.window);
  };
  if (lane >= g.from && lane < g.to) count(asked.len);
  for (int b = max(g.from, kWave) + lane; b < g.to; b += kWave) count(ask_len(p, layer, head, b));
  least = wave_all(least, [](int a, int b) { return min(a, b); });
  const int given = g.id < kWave ? __builtin_amdgcn_readlane(asked.shared, g.id) : p.shared[layer * p.shared_stride + g.id];
  Common c;
  c.rows = max(0, min(given, least));
  if (reporting && c.rows != given) report(p.c.dev_err, kDevBadLength);
  c.start = p.window > 0 ? min(wave_all(start, [](int a, int b) { return max(a, b); }), c.rows) : 0;
  c.sinks = min(p.sinks, c.start);
  return c;
}

// A tile of KT rows in a list that covers ranges of rows, one after the other: its first row,
// its range's rows, and which range that is.
struct TileAt {
  int row, from, to, range;
};
template <int KT>
__device__ __forceinline__ int tiles_of(int from, int to) { return to > from ? (to + KT - 1) / KT - from / KT : 0; }
template <int KT>
__device__ __forceinline__ TileAt tile_at(int i, int from0, int to0, int from1, int to1, int from2, int to2) {
  const int until0 = tiles_of<KT>(from0, to0), until1 = until0 + tiles_of<KT>(from1, to1);
  const bool past0 = i >= until0, past1 = i >= until1;
  const int from = past1 ? from2 : past0 ? from1 : from0;
  const int to = past1 ? to2 : past0 ? to1 : to0;
  return TileAt{(from / KT + i - (past1 ? until1 : past0 ? until0 : 0)) * KT, from, to, past1 ? 2 : past0 ? 1 : 0};
}

// What a group sees together: the rows [0, sinks) and [start, rows).
template <int KT>
struct CommonTiles {
  int sinks, start, rows, total;

  __device__ __forceinline__ explicit CommonTiles(const Common &c)
      : sinks(c.sinks), start(c.start), rows(c.rows), total(tiles_of<KT>(0, c.sinks) + tiles_of<KT>(c.start, c.rows)) {}
  __device__ __forceinline__ TileAt at(int i) const {
    // (readfirstlane keeps the choice one of values: of addresses, it would be made in memory)
    const int s = __builtin_amdgcn_readfirstlane(sinks), a = __builtin_amdgcn_readfirstlane(start),
              r = __builtin_amdgcn_readfirstlane(rows);
    return tile_at<KT>(i, 0, s, a, r, r, r);
  }
};

// ------------------------------------------------------------------ common rows
// Key tiles on their way to LDS, which loads fill without registers between.  Each lane
// holds the place of 16 rows of the list's tiles; the table's entries of the batch after go
// to LDS meanwhile (a load to a register would have to wait for all rows on their way).
template <typename T, int D>
struct Feed {
  using C = tiles32::Cfg<T, D, kNW>;
  static constexpr int KT = C::keys;
  static constexpr int kGroups = KT / 16;
  static constexpr int kBatch = kWave / kGroups;         // tiles
  using List = CommonTiles<KT>;
  const unsigned char *k, *v;
  const int32_t *table;
  const List &list;
  int n_pages, shift, begin, end, wave, lane;
  int *entries;                              // [kWave] in LDS, the wave's own
  unsigned entries_at;
  unsigned worst;                            // id, of rows that are seen
  uint64_t place;                            // of this lane's 16 rows: a byte offset
  unsigned koff[C::insts], voff[C::insts];   // within 16 rows

  // Tiles [begin, end) of the list.
  __device__ __forceinline__ Feed(const PagedSharedParams &p, size_t cunit, const List &list_, int begin_, int end_,
                                  int *entries_, int wave_, int lane_)
      : k(static_cast<const unsigned char *>(p.c.k)), v(static_cast<const unsigned char *>(p.c.v)),
        table(p.c.pages + cunit * static_cast<size_t>(p.c.max_pages)), list(list_), n_pages(p.c.n_pages),
        shift(p.c.page_shift), begin(begin_), end(end_), wave(wave_), lane(lane_), entries(entries_),
        entries_at(lds_address(entries_)), worst(0) {
#pragma unroll
    for (int i = 0; i < C::insts; ++i) {
      const int row = piece(i) + lane / C::lanes_per_row, c = lane % C::lanes_per_row;
      koff[i] = row % 16 * C::row_bytes + (c ^ C::k_swap(row)) * 16;
      voff[i] = row % 16 * C::row_bytes + (c ^ C::v_swap(row)) * 16;
    }
  }
  // A wave's i-th load of a tile takes wave_rows rows from this one on.
  __device__ __forceinline__ int piece(int i) const { return (i * kNW + wave) * C::wave_rows; }
  // The first of this lane's 16 rows in the batch that starts at tile i, and whether any is seen.
  __device__ __forceinline__ int row_of(int i, bool &seen) const {
    const TileAt a = list.at(min(i + lane / kGroups, end - 1));
    const int row = a.row + lane % kGroups * 16;
    seen = row < a.to && row + 16 > a.from;
    return row;
  }
  __device__ __forceinline__ unsigned entry_of(int i) const {
    bool seen;
    const int row = row_of(i, seen);
    return seen ? static_cast<unsigned>(row >> shift) * 4u : 0u;
  }
  __device__ __forceinline__ void ask(int i) { load_to_lds4(table, entry_of(i), entries_at); }
  // The batch that starts at tile i, by its entries, and the one after.
  __device__ __forceinline__ void batch(int i, int entry) {
    bool seen;
    const int row = row_of(i, seen);
    if (seen) worst = max(worst, static_cast<unsigned>(entry));
    const unsigned id = min(static_cast<unsigned>(entry), static_cast<unsigned>(n_pages - 1));
    place = ((static_cast<uint64_t>(id) << shift) + (row & ((1u << shift) - 1u))) * C::row_bytes;
    // The entry has come from LDS before the load that overwrites it there is sent, which
    // the compiler does not know to write LDS.
    asm volatile("s_waitcnt lgkmcnt(0)" : "+v"(entry));
    ask(i + kBatch);
  }
  __device__ __forceinline__ void first() {
    batch(begin, *reinterpret_cast<const int32_t *>(reinterpret_cast<const char *>(table) + entry_of(begin)));
  }
  __device__ __forceinline__ void turn(int i) {
    if (i < end && ((i - begin) & (kBatch - 1)) == 0) batch(i, entries[lane]);
  }
  // Where tile i's loads begin.  Past the end they are made all the same, so that what is on
  // its way can be counted, but of one piece.
  struct Place {
    uint64_t at[C::insts];
    unsigned lanes;
  };
  __device__ __forceinline__ Place find(int i) const {
    const int at_i = min(i, end - 1);
    Place w;
    w.lanes = i < end ? ~0u : 0u;
#pragma unroll
    for (int j = 0; j < C::insts; ++j) {
      const int from = ((at_i - begin) & (kBatch - 1)) * kGroups + piece(j) / 16;
      w.at[j] = static_cast<uint64_t>(static_cast<unsigned>(__builtin_amdgcn_readlane(static_cast<int>(place >> 32), from))) << 32 |
                static_cast<unsigned>(__builtin_amdgcn_readlane(static_cast<int>(place), from));
    }
    return w;
  }
  __device__ __forceinline__ void load_k(const Place &w, int j, unsigned to) const {
    load_to_lds16(k + w.at[j], koff[j] & w.lanes, to + piece(j) * C::row_bytes);
  }
  __device__ __forceinline__ void load_v(const Place &w, int j, unsigned to) const {
    load_to_lds16(v + w.at[j], voff[j] & w.lanes, to + piece(j) * C::row_bytes);
  }
  // Rows of V outside the range count for nothing, whatever they hold.
  __device__ __forceinline__ void clean(const TileAt &a, unsigned char *vbuf) const {
#pragma unroll
    for (int j = 0; j < C::insts; ++j) {
      const int row = a.row + piece(j) + lane / C::lanes_per_row;
      if (row < a.from || row >= a.to)
        *reinterpret_cast<u32x4v *>(vbuf + piece(j) * C::row_bytes + lane * 16) = u32x4v{0, 0, 0, 0};
    }
  }
};

// LDS of a workgroup: four buffers, of the common part's K and V of two tiles, or of a
// wave's tile each.
template <typename T, int D>
constexpr int area_bytes() {
  const int a = tiles32::Cfg<T, D, kNW>::stage, b = tiles16::Cfg<T, D>::wave_stage;
  return a > b ? a : b;
}

// A split of a block of query rows.
struct Block {
  int layer, head, lh, split;
  Group g;
  Common seen;
};

// kWays waves have 32 query rows together: each forms S from its part of D, all add them up through
// LDS and weigh the same rows, and each forms its columns of O (of two with the same ones,
// from half of the tile's rows).
template <typename T, int D, int kWays>
__device__ __forceinline__ void attend_block(const PagedSharedParams &p, const Block &at, unsigned char *k0, unsigned char *v0,
                                             unsigned char *k1, unsigned char *v1, int *entries) {
  using namespace tiles32;
  using C = tiles32::Cfg<T, D, kNW>;
  using In = Feed<T, D>;
  using M = Mma32<T>;
  using frag = typename M::frag;
  constexpr int KT = C::keys;
  constexpr int kQk = C::qk_steps / kWays;                // a wave's, of a block of S
  constexpr int kD = C::dtiles > kWays ? C::dtiles / kWays : 1, kColumns = C::dtiles / kD, kHalves = kWays / kColumns > 1 ? 2 : 1;
  static_assert(kWays == 1 || (C::blocks == 1 && M::kpl == 1), "fp32's tiles");
  const int lane = threadIdx.x & (kWave - 1);
  const int wave = __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x) / kWave);
  const int half = lane >> 5;
  const int col = lane & 31;
  const int part = wave % kWays;                          // of D
  const int dt0 = kWays > 1 ? part % kColumns * kD : 0, key_half = kHalves > 1 ? part / kColumns : 0;
  const int layer = at.layer, head = at.head, lh = at.lh, split = at.split;
  const Group &g = at.g;
  const int rows = (g.to - g.from) * p.group;

  const typename In::List list(at.seen);
  const int per_split = p.by_splits.of(list.total + p.splits - 1);
  const int i0 = split * per_split;
  const int i1 = min(list.total, i0 + per_split);

  // This lane's query row.
  const int wave_row = g.row0 + wave / kWays * 32;
  const bool active = wave_row < rows;
  const int r = min(wave_row + col, rows - 1);
  const int b = g.from + p.by_group.of(r);
  const size_t qrow = (static_cast<size_t>(layer * p.c.batch + b) * p.c.hkv + head) * p.group + p.by_group.rest(r);
  frag qf[kQk];
  {
    const T *src = reinterpret_cast<const T *>(p.q) + qrow * D + half * (D / 2) + part * kQk * M::kpl;
#pragma unroll
    for (int c = 0; c < kQk; ++c) {
      qf[c] = load_frag(src + c * M::kpl);
      if (p.scale_log2 < 0.f) qf[c] = M::negated(qf[c]);   // so that the largest product is the largest logit
    }
  }
  const float scale = fmaxf(fabsf(p.scale_log2), 0x1p-126f);   // times a hidden row's -inf, 0 would be NaN

  In in(p, p.c.unit((layer * p.c.batch + g.from) * p.c.hkv + head), list, i0, i1, entries + wave * kWave, wave, lane);
  float m_run = -INFINITY, l_run = 0.f;                  // m in units of the scaled logits
  f32x16_t o[kD];
#pragma unroll
  for (int dt = 0; dt < kD; ++dt) {
#pragma unroll
    for (int i = 0; i < 16; ++i) o[dt][i] = 0.f;
  }
  const int kat = k_base<T, D>(lane) ^ (part * kQk * M::kpl * (int)sizeof(T));
  const int vat = (v_base<T, D>(lane) ^ (dt0 * 32 * (int)sizeof(T))) + key_half * (16 * C::row_bytes);

  // Tile i, in kbuf and vbuf once its loads are done.  The next tile's V goes to vto, where the
  // last tile's was, while S is formed, and the K of the one after to kbuf, while O is: so
  // each has a tile and a half's time to come in two buffers.  `ahead`: the next tile's place,
  // then that of the one after.
  constexpr int kHalf = C::insts;                         // a wave's loads of a tile's K or V
  typename In::Place ahead;
  const auto step = [&](int i, unsigned char *kbuf, unsigned char *vbuf, unsigned kto, unsigned vto, bool turning)
                        __attribute__((always_inline)) {
    const TileAt tile = list.at(i);
    const bool whole = tile.row >= tile.from && tile.row + KT <= tile.to;
    __builtin_amdgcn_s_waitcnt(wait_loads(2 * kHalf));    // K
    barrier();                                            // is there, and no one reads the last tile's V
    f32x16_t s[C::blocks];
    constexpr int kSteps = C::blocks * kQk, kAhead = M::kpl == 8 || kSteps < 16 ? 8 : 16, kEach = kSteps / C::insts;
    float ref = 0.f;
    if (!active) {
#pragma unroll
      for (int j = 0; j < C::insts; ++j) in.load_v(ahead, j, vto);
    } else {
      // S^T, with operands read ahead of their products, and between the products the next
      // V asked for, piece by piece.  The blocks take turns, so that a product does not wait
      // for the one before.
#pragma unroll
      for (int kb = 0; kb < C::blocks; ++kb) {
#pragma unroll
        for (int e = 0; e < 16; ++e) s[kb][e] = 0.f;
      }
      frag kf[2][kAhead];
      const auto read_k = [&](int q) {
#pragma unroll
        for (int c = 0; c < kAhead; ++c) {
          const int z = q * kAhead + c, byte = z / C::blocks * M::kpl * (int)sizeof(T);
          kf[q & 1][c] = load_frag(reinterpret_cast<const T *>(kbuf + (kat ^ (byte & ~15)) + (byte & 15) + z % C::blocks * 32 * C::row_bytes));
        }
      };
      read_k(0);
#pragma unroll
      for (int z = 0; z < kSteps; ++z) {
        if (z % kAhead == 0 && z + kAhead < kSteps) read_k(z / kAhead + 1);
        if (z % kAhead == 0) __builtin_amdgcn_sched_barrier(0);
        s[z % C::blocks] = M::mma(kf[z / kAhead & 1][z % kAhead], qf[z / C::blocks], s[z % C::blocks]);
        if (z % kEach == 0) in.load_v(ahead, z / kEach, vto);
        __builtin_amdgcn_sched_barrier(0);
      }
      if constexpr (kWays > 1) {
        // All waves are past their reads of K, whose place the parts of S take; their sum has one order.
        constexpr int kRounds = kNW * kWave * 64 / C::stage > 1 ? kNW * kWave * 64 / C::stage : 1, kRegs = 16 / kRounds;
        float4 *parts = reinterpret_cast<float4 *>(kbuf);
#pragma unroll
        for (int rd = 0; rd < kRounds; ++rd) {
          barrier();
#pragma unroll
          for (int e = rd * kRegs; e < (rd + 1) * kRegs; e += 4)
            parts[(wave * (kRegs / 4) + e / 4 % (kRegs / 4)) * kWave + lane] = make_float4(s[0][e], s[0][e + 1], s[0][e + 2], s[0][e + 3]);
          barrier();
#pragma unroll
          for (int e = rd * kRegs; e < (rd + 1) * kRegs; e += 4) {
            float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (int w = 0; w < kWays; ++w) {
              const float4 x = parts[((wave - part + w) * (kRegs / 4) + e / 4 % (kRegs / 4)) * kWave + lane];
              sum = w == 0 ? x : make_float4(sum.x + x.x, sum.y + x.y, sum.z + x.z, sum.w + x.w);
            }
            s[0][e] = sum.x;
            s[0][e + 1] = sum.y;
            s[0][e + 2] = sum.z;
            s[0][e + 3] = sum.w;
          }
        }
      }
      if (!whole) {
        const int low = tile.from - tile.row - 4 * half, high = tile.to - tile.row - 4 * half;
#pragma unroll
        for (int kb = 0; kb < C::blocks; ++kb) {
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            const int c = kb * 32 + acc_row(e, 0);
            s[kb][e] = c < low || c >= high ? -INFINITY : s[kb][e];
          }
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
        for (int dt = 0; dt < kD; ++dt) {
#pragma unroll
          for (int e = 0; e < 16; ++e) o[dt][e] *= alpha;
        }
      }
      ref = m_run == -INFINITY ? 0.f : m_run;
    }
    __builtin_amdgcn_s_waitcnt(wait_loads(2 * kHalf));    // V
    if (!whole) in.clean(tile, vbuf);                     // each wave looks after what it loaded
    barrier();                                            // is there, and no one reads K any more
    if (turning) in.turn(i + 2);
    ahead = in.find(i + 2);
    if (!active) {
#pragma unroll
      for (int j = 0; j < C::insts; ++j) in.load_k(ahead, j, kto);
      return;
    }
    constexpr int kParts = C::blocks * C::pv_steps / kHalves;
    frag vf[2][kD];
    const auto read_v = [&](int q) {
      const int row = M::kpl == 8 ? 16 * q : 8 * (q / 4) + q % 4;
#pragma unroll
      for (int dt = 0; dt < kD; ++dt)
        vf[q & 1][dt] = v_frag32<T, D>(vbuf + (vat ^ (dt * 32 * (int)sizeof(T))) + row * C::row_bytes);
    };
    read_v(0);

    // O^T: part q takes kpl elements of every lane, slot j of which is row
    // 8 (e / 4) + 4 half + e % 4 of S^T for e = q * kpl + j; the exponentials of a part
    // lie between the products of the part before, as the loads do.
    const auto weigh = [&](int q, int j) {
      const int e = q * M::kpl + j;
      const float w = fast_exp2(fmaf(s[e / 16][e % 16], scale, -ref));
      l_run += w;
      return w;
    };
    frag pf[2];
    const auto put = [&](int q, int j) {
      if constexpr (kHalves > 1) {
        const float low = weigh(q, j), high = weigh(q + kParts, j);
        pf[q & 1] = key_half ? high : low;
      } else if constexpr (M::kpl == 1) pf[q & 1] = weigh(q, j);
      else pf[q & 1][j] = static_cast<__bf16>(weigh(q, j));
    };
#pragma unroll
    for (int j = 0; j < M::kpl; ++j) put(0, j);
#pragma unroll
    for (int q = 0; q < kParts; ++q) {
      if (q + 1 < kParts) read_v(q + 1);
      __builtin_amdgcn_sched_barrier(0);
      constexpr int kApart = kParts / C::insts > 0 ? kParts / C::insts : 1, kTogether = kApart * C::insts > kParts ? 2 : 1;
#pragma unroll
      for (int dt = 0; dt < kD; ++dt) {
        o[dt] = M::mma(vf[q & 1][dt], pf[q & 1], o[dt]);
        if (dt == 0 && q % kApart == 0) {
#pragma unroll
          for (int j = q / kApart * kTogether; j < (q / kApart + 1) * kTogether && j < C::insts; ++j) in.load_k(ahead, j, kto);
        }
        if (q + 1 < kParts) {
#pragma unroll
          for (int j = dt * M::kpl / kD; j < (dt + 1) * M::kpl / kD; ++j) put(q + 1, j);
        }
        __builtin_amdgcn_sched_barrier(0);
      }
    }
  };
  if (i0 < i1) {
    in.first();
    const unsigned at_k0 = lds_address(k0), at_v0 = lds_address(v0), at_k1 = lds_address(k1), at_v1 = lds_address(v1);
    ahead = in.find(i0);
#pragma unroll
    for (int j = 0; j < C::insts; ++j) in.load_k(ahead, j, at_k0);
#pragma unroll
    for (int j = 0; j < C::insts; ++j) in.load_v(ahead, j, at_v0);
    ahead = in.find(i0 + 1);
#pragma unroll
    for (int j = 0; j < C::insts; ++j) in.load_k(ahead, j, at_k1);
    static_assert(In::kBatch % 2 == 0, "batches begin at an even step");
    for (int i = i0; i < i1; i += 2) {
      step(i, k0, v0, at_k0, at_v1, true);
      if (i + 1 < i1) step(i + 1, k1, v1, at_k1, at_v0, false);
    }
  }
  __builtin_amdgcn_s_waitcnt(wait_loads(0));              // LDS is another workgroup's afterwards
  if (in.worst >= static_cast<unsigned>(p.c.n_pages)) report(p.c.dev_err, kDevBadPage);

  const float l_tot = l_run + shfl_xor(l_run, 32);
  if constexpr (kHalves > 1) {
    if (i0 < i1) {
      float4 *halves = reinterpret_cast<float4 *>(k0);
      barrier();                                          // of all waves' loads and reads
#pragma unroll
      for (int e = 0; e < 4 && key_half; ++e)
        halves[(part % kColumns * 4 + e) * kWave + lane] = make_float4(o[0][4 * e], o[0][4 * e + 1], o[0][4 * e + 2], o[0][4 * e + 3]);
      barrier();
#pragma unroll
      for (int e = 0; e < 4 && !key_half; ++e) {
        const float4 x = halves[(part % kColumns * 4 + e) * kWave + lane];
        o[0][4 * e] += x.x;
        o[0][4 * e + 1] += x.y;
        o[0][4 * e + 2] += x.z;
        o[0][4 * e + 3] += x.w;
      }
    }
    if (key_half) return;
  }
  if (wave_row + col >= rows) return;
  const size_t to = static_cast<size_t>(split) * p.rows +
                      (static_cast<size_t>(lh) * p.c.batch + g.from) * p.group + wave_row + col;
  if (half == 0 && part == 0) {
    p.part_ml[2 * to] = m_run;
    p.part_ml[2 * to + 1] = l_tot;
  }
  if (i0 >= i1) return;                                   // without tiles, sum 0: not read
  float4 *po = reinterpret_cast<float4 *>(p.part_o + to * D) + half + dt0 * 8;
#pragma unroll
  for (int dt = 0; dt < kD; ++dt) {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      po[dt * 8 + 2 * e] = make_float4(o[dt][4 * e], o[dt][4 * e + 1], o[dt][4 * e + 2], o[dt][4 * e + 3]);
  }
}

template <typename T, int D>
__device__ __forceinline__ void attend_common(const PagedSharedParams &p, int id, unsigned char *k0, unsigned char *v0,
                                              unsigned char *k1, unsigned char *v1, int *entries) {
  const int lane = threadIdx.x & (kWave - 1);
  // The blocks of a layer, KV head and split take their turn on one XCD, beside each other,
  // so that those of a group share the keys' way through its L2.
  const int slot = id / kXcds;
  const int turn = p.by_blocks.of(slot), block = p.by_blocks.rest(slot);
  const int job = turn * kXcds + id % kXcds;
  const int lh = p.by_splits.of(job), split = p.by_splits.rest(job);
  const int layer = p.c.by_hkv.of(lh), head = p.c.by_hkv.rest(lh);
  if (layer >= p.c.n_layers) return;
  const Asked asked = ask_first(p, layer, head, lane);
  if (!groups_ascend(p, asked.from, asked.to, lane)) return;
  const Group g = find_group(p, asked, block, lane);
  if (g.id < 0) return;
  const Block at{layer, head, lh, split, g, common_rows(p, asked, g, layer, head, lane, threadIdx.x == 0 && split == 0 && g.row0 == 0)};
  // fp32's products take so long that few rows' ones are dealt to all waves; of bf16 one wave keeps up
  // with memory (8 sequences of 4 heads: 23.4 us, 23.5 with a tile's rows dealt to all; 26 of 5, whose
  // second block has two rows: 125 and 135).
  if constexpr (sizeof(T) == 4) {
    const int here = (g.to - g.from) * p.group - g.row0;
    if (here <= 32) return attend_block<T, D, 4>(p, at, k0, v0, k1, v1, entries);
    if (here <= 64) return attend_block<T, D, 2>(p, at, k0, v0, k1, v1, entries);
  }
  attend_block<T, D, 1>(p, at, k0, v0, k1, v1, entries);
}

// ------------------------------------------------------------------ units' own rows
// A cell is up to kSharedCell sequences of one layer and KV head.  Their own tiles, one
// sequence after the other, are dealt evenly to the cell's waves, also of ragged sequences; a
// sequence's part of a wave is a part of its own for the join.  Of one sequence there are
// own_parts of them at most, 4 where a cell has as many sequences as waves: one that is longer
// than 3 even shares makes every wave's share a third of itself, and leaves some waves nothing
// (8 heads, 128 sequences of 20 own rows, one of 2,048: 69 us a call, 17 with as many rows dealt
// evenly; one of 8,192: 198 and 20).
struct Cell {
  int n[kSharedCell];           // rows with the new one
  int rows[kSharedCell];        // shared ones
  int start[kSharedCell];       // of the rows that the sequence's group sees together
  int lead[kSharedCell];        // the group's first sequence
  int until[kSharedCell];       // tiles of the sequences up to this one
  int sums[kNW], most;
};

// The rows of a sequence with n of them that are not its group's common ones: shared rows that
// not all see, sinks behind the shared rows, and its own.
struct OwnRows {
  int from0, to0, from1, to1, from2, to2;

  __device__ __forceinline__ OwnRows(const PagedSharedParams &p, int n, int rows, int start) {
    const int lo = p.window > 0 && n > p.window ? n - p.window : 0;
    from0 = max(lo, min(p.sinks, start));
    to0 = start;
    from1 = rows;
    to1 = min(p.sinks, lo);
    from2 = max(rows, lo);
    to2 = n;
  }
  __device__ __forceinline__ int tiles() const {
    return tiles_of<kPagedTile>(from0, to0) + tiles_of<kPagedTile>(from1, to1) + tiles_of<kPagedTile>(from2, to2);
  }
  __device__ __forceinline__ TileAt at(int i) const { return tile_at<kPagedTile>(i, from0, to0, from1, to1, from2, to2); }
};

// Inclusive sums over the lanes: within sixteens, then over them.
template <int CTRL, int ROWS>
__device__ __forceinline__ int dpp_add(int v) {
  return v + __builtin_amdgcn_update_dpp(0, v, CTRL, ROWS, 0xf, false);
}
__device__ __forceinline__ int wave_sums(int v) {
  v = dpp_add<0x111, 0xf>(v);                             // the lane 1, 2, 4, 8 before
  v = dpp_add<0x112, 0xf>(v);
  v = dpp_add<0x114, 0xf>(v);
  v = dpp_add<0x118, 0xf>(v);
  v = dpp_add<0x142, 0xa>(v);                             // lane 15 to the next sixteen, 31 to the next two
  return dpp_add<0x143, 0xc>(v);
}

// Whether the list of groups is good (without it every sequence's rows are its own), all
// tiles, and the most of a sequence.
struct CellSum {
  bool ok;
  int total, most;
};

// Fills the cell that is the whole batch, in few groups.  Every wave writes what it reads,
// the same as the others, so that none has to wait for another (128 sequences in one group:
// 42.5 us a call, 47.7 with all waves together), but the groups take their turns here, some
// 100 cycles each (64 sequences in 16 groups: 17.9 us, 14.3 together; 8 groups: the same).
__device__ __forceinline__ CellSum fill_whole_cell(const PagedSharedParams &p, Cell &cell, int layer, int head, int lane) {
  constexpr int kEach = kSharedCell / kWave;
  const int extra = p.k_new ? 1 : 0, per = (p.c.batch + kWave - 1) / kWave;      // sequences of a lane, neighbours
  Asked asked;
  asked.from = p.first[min(lane, p.groups)];
  asked.to = p.first[min(lane + 1, p.groups)];
  asked.shared = p.shared[layer * p.shared_stride + min(lane, p.groups - 1)];
  int cached[kEach], rows[kEach], start[kEach], lead[kEach], tiles[kEach];
#pragma unroll
  for (int j = 0; j < kEach; ++j) cached[j] = j < per ? ask_len(p, layer, head, min(lane * per + j, p.c.batch - 1)) : 0;
  CellSum sum;
  sum.ok = groups_ascend(p, asked.from, asked.to, lane);
#pragma unroll
  for (int j = 0; j < kEach; ++j) {
    cached[j] = max(0, min(cached[j], p.c.cap));
    rows[j] = start[j] = 0;
    lead[j] = lane * per + j;
  }
  for (int k = 0; sum.ok && k < p.groups; ++k) {
    const int from = __builtin_amdgcn_readlane(asked.from, k), to = __builtin_amdgcn_readlane(asked.to, k);
    int least = p.c.cap, most = 0;
#pragma unroll
    for (int j = 0; j < kEach; ++j) {
      const int b = lane * per + j;
      if (j < per && b >= from && b < to) {
        least = min(least, cached[j]);
        most = max(most, cached[j] + extra - p.window);
      }
    }
    least = wave_all(least, [](int a, int b) { return min(a, b); });
    if (p.window > 0) most = wave_all(most, [](int a, int b) { return max(a, b); });
    const int r = max(0, min(__builtin_amdgcn_readlane(asked.shared, k), least));
#pragma unroll
    for (int j = 0; j < kEach; ++j) {
      const int b = lane * per + j;
      const bool here = b >= from && b < to;
      rows[j] = here ? r : rows[j];
      start[j] = here && p.window > 0 ? max(0, min(most, r)) : start[j];
      lead[j] = here ? from : lead[j];
    }
  }
  int all = 0, most = 0;
#pragma unroll
  for (int j = 0; j < kEach; ++j) {
    tiles[j] = j < per && lane * per + j < p.c.batch ? OwnRows(p, cached[j] + extra, rows[j], start[j]).tiles() : 0;
    all += tiles[j];
    most = max(most, tiles[j]);
  }
  int until = wave_sums(all);
  sum.total = __builtin_amdgcn_readlane(until, kWave - 1);
  sum.most = wave_all(most, [](int a, int b) { return max(a, b); });
  until -= all;
#pragma unroll
  for (int j = 0; j < kEach; ++j) {
    const int b = lane * per + j;
    if (j >= per) break;
    until += tiles[j];
    if (b < p.c.batch) {
      cell.n[b] = cached[j] + extra;
      cell.rows[b] = rows[j];
      cell.start[b] = start[j];
      cell.lead[b] = lead[j];
      cell.until[b] = until;
    }
  }
  return sum;
}

// Fills any cell, by all waves together.
__device__ __forceinline__ CellSum fill_cell(const PagedSharedParams &p, Cell &cell, int layer, int head, int b0, int nb) {
  constexpr int kEach = kSharedCell / (kNW * kWave);
  const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = tid / kWave;
  const int extra = p.k_new ? 1 : 0;
  const Asked asked = ask_first(p, layer, head, lane);
  for (int i = tid; i < kSharedCell; i += kNW * kWave) {
    cell.rows[i] = p.c.cap;
    cell.start[i] = 0;
  }
  if (tid == 0) cell.most = 0;
  __syncthreads();

  // The group of sequence b: the last one that begins there or before.
  const auto group_of = [&](int b) {
    int low = 0, high = p.groups - 1;
    while (low < high) {
      const int mid = (low + high + 1) / 2;
      if (p.first[mid] <= b) low = mid;
      else high = mid - 1;
    }
    return low;
  };
  const bool ok = groups_ascend(p, asked.from, asked.to, lane);
  // Sequences of groups that reach into the cell, also those outside of it, by the place of
  // their group's first sequence in it.
  int begin = 0, end = p.c.batch;
  if (ok && nb < p.c.batch) {
    begin = p.first[group_of(b0)];
    end = p.first[group_of(b0 + nb - 1) + 1];
  }
  for (int b = begin + tid; ok && b < end; b += kNW * kWave) {
    const int len = wave == 0 && b == lane ? asked.len : ask_len(p, layer, head, b);   // (not where begin > 0)
    const int id = group_of(b), from = p.first[id];
    const int at = max(from, b0) - b0, n = max(0, min(len, p.c.cap));
    atomicMin(&cell.rows[at], n);
    if (p.window > 0) atomicMax(&cell.start[at], n + extra - p.window);
    if (b >= b0 && b < b0 + nb) {
      cell.lead[b - b0] = from;
      cell.until[b - b0] = id;
    }
  }
  __syncthreads();
  int n[kEach], rows[kEach], start[kEach], lead[kEach], tiles[kEach], sum = 0, most = 0;
#pragma unroll
  for (int i = 0; i < kEach; ++i) {
    const int at = tid * kEach + i, b = b0 + at;
    n[i] = rows[i] = start[i] = tiles[i] = 0;
    lead[i] = b;
    if (at < nb) {
      n[i] = max(0, min(ask_len(p, layer, head, b), p.c.cap)) + extra;
      if (ok) {
        lead[i] = cell.lead[at];
        const int given = p.shared[layer * p.shared_stride + cell.until[at]], place = max(lead[i], b0) - b0;
        rows[i] = max(0, min(given, cell.rows[place]));
        start[i] = p.window > 0 ? min(cell.start[place], rows[i]) : 0;
      }
      tiles[i] = OwnRows(p, n[i], rows[i], start[i]).tiles();
    }
    sum += tiles[i];
    most = max(most, tiles[i]);
  }
  // tiles up to each sequence: over the lanes, then the waves
  int until = wave_sums(sum);
  if (lane == kWave - 1) cell.sums[wave] = until;
  if (most > 0) atomicMax(&cell.most, most);
  __syncthreads();
  int total = 0;
#pragma unroll
  for (int w = 0; w < kNW; ++w) {
    until += w < wave ? cell.sums[w] : 0;
    total += cell.sums[w];
  }
  until -= sum;
#pragma unroll
  for (int i = 0; i < kEach; ++i) {
    const int at = tid * kEach + i;
    until += tiles[i];
    cell.n[at] = n[i];
    cell.rows[at] = rows[i];
    cell.start[at] = start[i];
    cell.lead[at] = lead[i];
    cell.until[at] = until;
  }
  __syncthreads();
  return CellSum{ok, __builtin_amdgcn_readfirstlane(total), __builtin_amdgcn_readfirstlane(cell.most)};
}

template <typename T, int D>
__device__ __forceinline__ void attend_own(const PagedSharedParams &p, int id, unsigned char *a0, unsigned char *a1,
                                           unsigned char *a2, unsigned char *a3, Cell &cell) {
  using namespace tiles16;
  using C = tiles16::Cfg<T, D>;
  using MF = Mfma<T>;
  using frag = typename MF::frag;
  const int lane = threadIdx.x & (kWave - 1);
  const int wave = __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x) / kWave);
  const int col = lane & 15;
  const int grp = lane >> 4;
  const int cid = p.by_cell.of(id), turn_of = p.by_cell.rest(id);     // the cell, and which of its workgroups
  const int lh = p.by_chunks.of(cid), b0 = p.by_chunks.rest(cid) * kSharedCell;
  const int layer = p.c.by_hkv.of(lh), head = p.c.by_hkv.rest(lh);
  const int nb = min(kSharedCell, p.c.batch - b0);
  const CellSum sum = p.c.batch <= kSharedCell && p.groups <= 8 ? fill_whole_cell(p, cell, layer, head, lane)
                                                                 : fill_cell(p, cell, layer, head, b0, nb);
  const size_t row0 = (static_cast<size_t>(lh) * p.c.batch + b0) * p.group;       // of the parts

  // Even shares, and of no sequence more parts than there are places.
  const int waves = p.cell_wgs * kNW, w = turn_of * kNW + wave;
  const int share = max(max((sum.total + waves - 1) / waves, (sum.most + p.own_parts - 2) / (p.own_parts - 1)), 1);
  const auto no_part = [&](int slot, int b, int g) {
    float *ml = p.part_ml + 2 * (static_cast<size_t>(slot) * p.rows + row0 + static_cast<size_t>(b) * p.group + g);
    ml[0] = -INFINITY;
    ml[1] = 0.f;
  };
  if (turn_of == 0) {
    if (!sum.ok && threadIdx.x == 0) report(p.c.dev_err, kDevBadGroup);
    // places without a part: of sequences without tiles, and the common ones where there are no groups
    for (int i = threadIdx.x; i < nb * p.group; i += kNW * kWave) {
      const int b = p.by_group.of(i), g = p.by_group.rest(i);
      if (cell.until[b] == (b > 0 ? cell.until[b - 1] : 0))
        for (int k = 0; k < p.own_parts; ++k) no_part(p.splits + k, b, g);
      if (!sum.ok)
        for (int k = 0; k < p.splits; ++k) no_part(k, b, g);
    }
  }
  const int x0 = w * share, x1 = min(sum.total, x0 + share);
  const int mine = x1 - x0;                               // tiles of the wave
  if (mine <= 0) return;
  unsigned char *stage = wave < 2 ? (wave == 0 ? a0 : a1) : (wave == 2 ? a2 : a3);

  // Where the wave's tiles lie: each lane holds the place of 16 rows, so 32 tiles at a
  // time; the table's entries of the batch after are on their way meanwhile.
  constexpr int kBatch = kWave / 2;
  struct Tile {
    int b, row, from, to;       // the sequence and, from bit 16 on, the range of its list; rows
  };
  const auto locate = [&](int k) {
    const int x = x0 + min(k, mine - 1);
    int b = 0, end = nb - 1;                              // the first sequence whose tiles reach past x
    while (__any(b < end)) {
      const int mid = (b + end) >> 1;
      const bool past = cell.until[mid] > x;
      end = past ? mid : end;
      b = past ? b : min(mid + 1, end);
    }
    const TileAt at = OwnRows(p, cell.n[b], cell.rows[b], cell.start[b]).at(x - (b > 0 ? cell.until[b - 1] : 0));
    return Tile{b | at.range << 16, at.row, at.from, at.to};
  };
  Tile here, next;
  unsigned worst = 0;
  int coming = 0;
  uint64_t place = 0;
  const int extra = p.k_new ? 1 : 0;
  const auto ask = [&](int batch) {
    next = locate(batch * kBatch + lane / 2);
    const int b = next.b & 0xffff, row = next.row + lane % 2 * 16;
    const bool cached = row < min(next.to, cell.n[b] - extra) && row + 16 > next.from;
    const size_t cunit = p.c.unit((layer * p.c.batch + (next.b >> 16 == 0 ? cell.lead[b] : b0 + b)) * p.c.hkv + head);
    coming = cached ? p.c.pages[cunit * static_cast<size_t>(p.c.max_pages) + (row >> p.c.page_shift)] : 0;
  };
  const auto turn = [&](int batch) {
    here = next;
    const int row = here.row + lane % 2 * 16;
    const unsigned page = min(static_cast<unsigned>(coming), static_cast<unsigned>(p.c.n_pages - 1));
    worst = max(worst, static_cast<unsigned>(coming));
    place = ((static_cast<uint64_t>(page) << p.c.page_shift) + (row & ((1 << p.c.page_shift) - 1))) * C::row_bytes;
    if (mine > (batch + 1) * kBatch) ask(batch + 1);
  };
  struct Where {
    uint64_t at[2];
  };
  const auto find = [&](int k) {
    Where w;
#pragma unroll
    for (int hf = 0; hf < 2; ++hf) {
      const int from = (k & (kBatch - 1)) * 2 + hf;
      w.at[hf] = static_cast<uint64_t>(static_cast<unsigned>(__builtin_amdgcn_readlane(static_cast<int>(place >> 32), from))) << 32 |
                 static_cast<unsigned>(__builtin_amdgcn_readlane(static_cast<int>(place), from));
    }
    return w;
  };
  // The sequence that the wave is at, its part's number, and its softmax; what the next tile
  // needs beside its rows (another sequence's queries, the new row) comes with them.
  struct Uniform {
    int b, range, row, from, to;
    bool fresh;                 // the new row is in it
  };
  const auto info = [&](int k) {
    const int from_lane = (k & (kBatch - 1)) * 2, b = __builtin_amdgcn_readlane(here.b, from_lane);
    Uniform u{b & 0xffff, b >> 16, __builtin_amdgcn_readlane(here.row, from_lane), __builtin_amdgcn_readlane(here.from, from_lane),
              __builtin_amdgcn_readlane(here.to, from_lane), false};
    u.fresh = extra && u.range == 2 && u.row + kTile >= u.to;      // a sequence's last tile holds it
    return u;
  };
  // Rows outside the range are masked where they are used; loads take one of its rows in
  // their place, so that short ranges cost what they hold (of sixteen that are all outside,
  // one; 167 sequences of 20 own rows, 3 layers, window 368: 65 us with all rows loaded, 55).
  // The new row is put where it belongs in LDS.
  const auto load = [&](Rows<T, D> &reg, const void *pool, const Where &w, const Uniform &u) {
    const int low = u.from - u.row, high = u.to - u.row - (u.fresh ? 2 : 1);
#pragma unroll
    for (int j = 0; j < C::insts; ++j) {
      constexpr int kHalf = C::insts / 2;
      const int hf = j / kHalf, row = j % kHalf * C::rows_per_inst + lane / C::lanes_per_row;
      const int from = max(0, min(low - 16 * hf, 15)), to = max(0, min(high - 16 * hf, 15));
      reg[j] = __builtin_nontemporal_load(reinterpret_cast<const u32x4v *>(
          static_cast<const unsigned char *>(pool) + w.at[hf] + max(from, min(row, to)) * C::row_bytes + lane % C::lanes_per_row * 16));
    }
  };
  // (fp32 has no registers for the next queries beside the present ones and waits for them)
  constexpr bool kQueriesAhead = sizeof(T) == 2;
  frag qf[C::qk_steps], q_next[kQueriesAhead ? C::qk_steps : 1];
  uint4 kfresh, vfresh;
  const auto unit_of = [&](const Uniform &u) { return static_cast<size_t>(layer * p.c.batch + b0 + u.b) * p.c.hkv + head; };
  const auto load_queries = [&](auto &to, const Uniform &u) {
    const T *qrow = reinterpret_cast<const T *>(p.q) + (unit_of(u) * p.group + min(col, p.group - 1)) * D + grp * C::dq;
#pragma unroll
    for (int c = 0; c < C::qk_steps; ++c) to[c] = load_frag(qrow + c * C::kpl);
  };
  const auto load_more = [&](const Uniform &u, bool queries) {
    if constexpr (kQueriesAhead) {
      if (queries) load_queries(q_next, u);
    }
    if (u.fresh) {
      const size_t at = unit_of(u) * C::lanes_per_row + lane % C::lanes_per_row;
      kfresh = reinterpret_cast<const uint4 *>(p.k_new)[at];
      vfresh = reinterpret_cast<const uint4 *>(p.v_new)[at];
    }
  };
  float m_run, l_run;
  f32x4_t o[C::dtiles];
  int number = 0;
  const auto begin = [&](const Uniform &u) {
    if constexpr (kQueriesAhead) {
#pragma unroll
      for (int c = 0; c < C::qk_steps; ++c) qf[c] = q_next[c];
    } else {
      load_queries(qf, u);
    }
    m_run = -INFINITY;
    l_run = 0.f;
#pragma unroll
    for (int dt = 0; dt < C::dtiles; ++dt) o[dt] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  };
  const auto finish = [&](int seq) {
    const float l_tot = group4_sum(l_run);
    if (col < p.group) {
      const size_t part = static_cast<size_t>(p.splits + number) * p.rows + row0 + static_cast<size_t>(seq) * p.group + col;
      if (grp == 0) {
        p.part_ml[2 * part] = m_run;
        p.part_ml[2 * part + 1] = l_tot;
      }
#pragma unroll
      for (int dt = 0; dt < C::dtiles; ++dt)
        *reinterpret_cast<float4 *>(p.part_o + part * D + dt * 16 + 4 * grp) =
            make_float4(o[dt][0], o[dt][1], o[dt][2], o[dt][3]);
      if (number == 0) {                                  // the places of parts that there are not
        const int until = cell.until[seq], parts = until <= x1 ? 1 : (until - 1) / share - w + 1;
        for (int i = parts + grp; i < p.own_parts; i += 4) no_part(p.splits + i, seq, col);
      }
    }
    number = 0;
  };

  Rows<T, D> kreg, vreg;
  Uniform now, then;
  const auto attend = [&](int k) {
    const bool more = k + 1 < mine;
    if (((k + 1) & (kBatch - 1)) == 0 && more) turn((k + 1) / kBatch);
    const Where place_of = find(k + 1);
    then = info(k + 1);
    if (!more) then.b = now.b;
    const int kb = now.row, from = now.from, to = now.to, n_cache = to - 1;   // of a tile with the new row
    const bool whole = kb >= from && kb + kTile <= to && !now.fresh;
#pragma unroll
    for (int j = 0; j < C::insts; ++j) {
      const int r = j * C::rows_per_inst + lane / C::lanes_per_row;
      *reinterpret_cast<u32x4v *>(stage + r * C::k_stride + (lane % C::lanes_per_row) * 16) = kreg[j];
    }
    if (now.fresh && lane < C::lanes_per_row)
      *reinterpret_cast<uint4 *>(stage + (n_cache - kb) * C::k_stride + lane * 16) = kfresh;
    const uint4 v_row = vfresh;
    if (more) load(kreg, p.c.k, place_of, then);
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    f32x4_t s[2];
#pragma unroll
    for (int hf = 0; hf < 2; ++hf) {
      const T *krow = reinterpret_cast<const T *>(stage + (hf * 16 + col) * C::k_stride) + grp * C::dq;
      s[hf] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int c = 0; c < C::qk_steps; ++c) s[hf] = MF::mma(load_frag(krow + c * C::kpl), qf[c], s[hf]);
    }
    // V's rows take the place of K's, which other lanes read: the compiler must not put
    // the writes first (a wave's LDS accesses are done in order, so nothing waits).
    asm volatile("" ::: "memory");

    float x[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = s[e >> 2][e & 3] * p.scale_log2;
    if (!whole) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int row = kb + (e >> 2) * 16 + 4 * grp + (e & 3);
        x[e] = row >= from && row < to ? x[e] : -INFINITY;
      }
    }
    float top = x[0];
#pragma unroll
    for (int e = 1; e < 8; ++e) top = fmaxf(top, x[e]);
    top = group4_max(top);
    if (__any(top > m_run + kSlack)) {                    // as in the common part
      const float m_new = fmaxf(m_run, top);
      const float alpha = fast_exp2(m_run - (m_new == -INFINITY ? 0.f : m_new));
      l_run *= alpha;
      m_run = m_new;
#pragma unroll
      for (int dt = 0; dt < C::dtiles; ++dt) {
#pragma unroll
        for (int e = 0; e < 4; ++e) o[dt][e] *= alpha;
      }
    }
    const float ref = m_run == -INFINITY ? 0.f : m_run;   // logits of -inf alone have no weight
    float pv[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      pv[e] = fast_exp2(x[e] - ref);
      l_run += pv[e];
    }
    if (!whole) {                                         // a NaN that is not seen, times 0, would be NaN
#pragma unroll
      for (int j = 0; j < C::insts; ++j) {
        const int row = kb + j * C::rows_per_inst + lane / C::lanes_per_row;
        const unsigned keep = row >= from && row < to ? ~0u : 0u;
        vreg[j] &= u32x4v{keep, keep, keep, keep};
      }
    }
#pragma unroll
    for (int j = 0; j < C::insts; ++j) {
      const int r = j * C::rows_per_inst + lane / C::lanes_per_row;
      uint2 *dst = reinterpret_cast<uint2 *>(stage + r * C::v_stride + (lane % C::lanes_per_row) * 16);
      dst[0] = make_uint2(vreg[j][0], vreg[j][1]);
      dst[1] = make_uint2(vreg[j][2], vreg[j][3]);
    }
    if (now.fresh && lane < C::lanes_per_row) {
      uint2 *dst = reinterpret_cast<uint2 *>(stage + (n_cache - kb) * C::v_stride + lane * 16);
      dst[0] = make_uint2(v_row.x, v_row.y);
      dst[1] = make_uint2(v_row.z, v_row.w);
    }
    if (more) {
      load(vreg, p.c.v, place_of, then);
      load_more(then, then.b != now.b);
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
#pragma unroll
    for (int dt = 0; dt < C::dtiles; ++dt) {
#pragma unroll
      for (int c = 0; c < C::pv_ops; ++c) o[dt] = MF::mma(v_frag<T, D>(stage, c, grp, dt, col), p_frag<T>(pv, c), o[dt]);
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  };
  ask(0);
  turn(0);
  const Where first = find(0);
  now = info(0);
  load(kreg, p.c.k, first, now);
  load(vreg, p.c.v, first, now);
  load_more(now, true);
  number = w - (now.b > 0 ? __builtin_amdgcn_readfirstlane(cell.until[now.b - 1]) : 0) / share;   // waves before that had some of it
  begin(now);
  for (int k = 0; k < mine; ++k) {
    attend(k);
    if (then.b != now.b) {
      finish(now.b);
      begin(then);
    }
    now = then;
  }
  finish(now.b);
  if (worst >= static_cast<unsigned>(p.c.n_pages)) report(p.c.dev_err, kDevBadPage);
}

template <typename T, int D>
__global__ __launch_bounds__(kNW * kWave, 2) void shared_attn_kernel(PagedSharedParams p) {
  // arrays of their own, so that reads of one need not wait for loads into another
  __shared__ __attribute__((aligned(1024))) unsigned char a0[area_bytes<T, D>()], a1[area_bytes<T, D>()],
      a2[area_bytes<T, D>()], a3[area_bytes<T, D>()];
  __shared__ Cell cell;
  // Common and own workgroups take turns, kMix on each XCD: the ones wait for products, the
  // others for memory.
  const int xcd = blockIdx.x % kXcds;
  int slot = blockIdx.x / kXcds;
  bool common;
  const int turns = min(p.common_wgs, p.own_wgs) / (kXcds * kMix);
  if (slot < 2 * kMix * turns) {
    const int t = slot / kMix;
    common = t % 2 == 0;
    slot = t / 2 * kMix + slot % kMix;
  } else {
    slot -= kMix * turns;
    common = slot < p.common_wgs / kXcds;
    if (!common) slot -= p.common_wgs / kXcds - kMix * turns;
  }
  const int id = slot * kXcds + xcd;
  if (common) attend_common<T, D>(p, id, a0, a1, a2, a3, cell.n);
  else if (id < p.own_items) attend_own<T, D>(p, id, a0, a1, a2, a3, cell);
}

// ------------------------------------------------------------------ the join
// D / 4 threads have a row, kSub times where there are many parts.  Query head 0 of a unit
// commits the append.
constexpr int kJoinThreads = 256;

// f over each 16 or 32 lanes, in every lane.
template <int LANES, typename F>
__device__ __forceinline__ float lanes_fold(float v, F f) {
  static_assert(LANES == 16 || LANES == 32, "a row's lanes");
  v = f(v, dpp<kDppXor1>(v));
  v = f(v, dpp<kDppXor2>(v));
  v = f(v, dpp<kDppHalfMirror>(v));
  v = f(v, dpp<kDppMirror>(v));
  if (LANES == 32) {
    const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = f(__uint_as_float(a[0]), __uint_as_float(a[1]));
  }
  return v;
}

template <typename T, int D, int kSub>
__global__ __launch_bounds__(kJoinThreads) void shared_join_kernel(PagedSharedParams p) {
  constexpr int kLanes = D / 4, kEach = kLanes * kSub, kPer = kJoinThreads / kEach;   // rows of a workgroup
  constexpr int kMost = kSharedMaxParts / kSub;                                       // parts of a thread
  __shared__ __attribute__((aligned(16))) float s_acc[kSub > 1 ? kSub : 1][kSub > 1 ? D : 1];
  __shared__ float s_w[kPer][kSharedMaxParts];
  const int tid = threadIdx.x;
  const int lane = tid % kLanes, sub = tid / kLanes % kSub, in = tid / kEach;
  const size_t row = static_cast<size_t>(blockIdx.x) * kPer + in;
  const bool real = row < p.rows;
  const int S = p.splits + p.own_parts;
  // rows are (layer, KV head, sequence, query head); units (layer, sequence, KV head)
  const int flat = static_cast<int>(real ? row : 0);
  const int lhb = p.by_group.of(flat), qi = p.by_group.rest(flat);
  const int lh = p.c.by_batch.of(lhb), b = p.c.by_batch.rest(lhb);
  const int layer = p.c.by_hkv.of(lh), head = p.c.by_hkv.rest(lh);
  const int unit = (layer * p.c.batch + b) * p.c.hkv + head;
  const size_t cunit = p.c.unit(unit);
  const bool commits = real && sub == 0 && qi == 0;
  const int len_in = commits ? p.c.len[cunit] : 0;        // (asked for first: its page waits for it)

  // Few rows' parts are asked for together with their statistics; of many, whose places are
  // mostly empty, those alone that there are.
  constexpr int kAhead = kSub > 1 ? (kMost < 8 ? kMost : 8) : 0;
  float4 x[kAhead + 1];
  const float *po = p.part_o + row * D + lane * 4;
#pragma unroll
  for (int i = 0; i < kAhead; ++i) {
    const int s = sub + i * kSub;
    x[i] = real && s < S ? *reinterpret_cast<const float4 *>(po + static_cast<size_t>(s) * p.rows * D) : make_float4(0.f, 0.f, 0.f, 0.f);
  }
  constexpr int kTurns = (kSharedMaxParts + kLanes - 1) / kLanes;
  float m[kTurns], l[kTurns];
#pragma unroll
  for (int i = 0; i < kTurns; ++i) {
    const int s = lane + i * kLanes;
    const bool there = real && s < S;
    const float2 ml = there ? reinterpret_cast<const float2 *>(p.part_ml)[static_cast<size_t>(s) * p.rows + row] : make_float2(-INFINITY, 0.f);
    m[i] = ml.x;
    l[i] = ml.y;
  }
  using Four = std::conditional_t<sizeof(T) == 2, uint2, uint4>;           // elements of a thread
  Four k_row{}, v_row{};
  int page = 0;
  if (commits && p.k_new) {
    const size_t from = static_cast<size_t>(unit) * kLanes + lane;
    k_row = reinterpret_cast<const Four *>(p.k_new)[from];
    v_row = reinterpret_cast<const Four *>(p.v_new)[from];
    page = p.c.pages[cunit * static_cast<size_t>(p.c.max_pages) + (max(0, min(len_in, p.c.cap - 1)) >> p.c.page_shift)];
  }
  float M = -INFINITY, L = 0.f;
#pragma unroll
  for (int i = 0; i < kTurns; ++i) M = fmaxf(M, m[i]);
  M = lanes_fold<kLanes>(M, [](float a, float b) { return fmaxf(a, b); });
  const float ref = M == -INFINITY ? 0.f : M;
#pragma unroll
  for (int i = 0; i < kTurns; ++i) {
    m[i] = fast_exp2(m[i] - ref);
    L += l[i] * m[i];
    // a part without rows has no output
    if (sub == 0 && lane + i * kLanes < kSharedMaxParts) s_w[in][lane + i * kLanes] = l[i] == 0.f ? 0.f : m[i];
  }
  L = lanes_fold<kLanes>(L, [](float a, float b) { return a + b; });
  __syncthreads();
  const float inv = L == 0.f ? 0.f : 1.f / L;
  float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
  const auto add = [&](int s, const float4 &y) {
    const float w = s_w[in][s] * inv;
    acc.x += w == 0.f ? 0.f : w * y.x;
    acc.y += w == 0.f ? 0.f : w * y.y;
    acc.z += w == 0.f ? 0.f : w * y.z;
    acc.w += w == 0.f ? 0.f : w * y.w;
  };
#pragma unroll
  for (int i = 0; i < kAhead; ++i) {
    if (sub + i * kSub < S) add(sub + i * kSub, x[i]);
  }
#pragma unroll 4
  for (int s = sub + kAhead * kSub; s < S; s += kSub)
    if (real && s_w[in][s] != 0.f) add(s, *reinterpret_cast<const float4 *>(po + static_cast<size_t>(s) * p.rows * D));
  if constexpr (kSub > 1) {
    *reinterpret_cast<float4 *>(&s_acc[sub][lane * 4]) = acc;
    __syncthreads();
    if (sub > 0) return;
#pragma unroll
    for (int i = 1; i < kSub; ++i) {
      const float4 y = *reinterpret_cast<const float4 *>(&s_acc[i][lane * 4]);
      acc.x += y.x;
      acc.y += y.y;
      acc.z += y.z;
      acc.w += y.w;
    }
  }
  if (!real) return;
  const size_t oq = static_cast<size_t>(unit) * p.group + qi;
  const T y[4] = {from_f32<T>(acc.x), from_f32<T>(acc.y), from_f32<T>(acc.z), from_f32<T>(acc.w)};
  reinterpret_cast<Four *>(p.out)[oq * kLanes + lane] = __builtin_bit_cast(Four, y);
  if (p.lse && lane == 0) p.lse[oq] = L == 0.f ? -INFINITY : (M + log2f(L)) * kLn2;
  if (!commits) return;
  int code = 0;
  if (len_in < 0 || len_in > p.c.cap) code = kDevBadLength;
  else if (p.k_new && len_in == p.c.cap) code = kDevAppendOverflow;
  else if (p.k_new && static_cast<unsigned>(page) >= static_cast<unsigned>(p.c.n_pages)) code = kDevBadPage;
  if (code && lane == 0) report(p.c.dev_err, code);
  if (code || !p.k_new) return;
  const size_t at = ((static_cast<size_t>(page) << p.c.page_shift) + (len_in & ((1 << p.c.page_shift) - 1))) * kLanes + lane;
  reinterpret_cast<Four *>(p.c.k)[at] = k_row;
  reinterpret_cast<Four *>(p.c.v)[at] = v_row;
  if (lane == 0) p.c.len[cunit] = len_in + 1;
}

template <typename T, int D, int kSub>
hipError_t launch_join(const PagedSharedParams &p, hipStream_t s) {
  constexpr int kPer = kJoinThreads / (D / 4 * kSub);
  hipLaunchKernelGGL((shared_join_kernel<T, D, kSub>), dim3((p.rows + kPer - 1) / kPer), dim3(kJoinThreads), 0, s, p);
  return hipGetLastError();
}

template <typename T, int D>
hipError_t launch_typed(const PagedSharedParams &p, hipStream_t s) {
  hipLaunchKernelGGL((shared_attn_kernel<T, D>), dim3(p.common_wgs + p.own_wgs), dim3(kNW * kWave), 0, s, p);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  // Few rows of many parts have a workgroup each (8 sequences of 32 heads, 32 splits: 23.0 us a call,
  // 38.7 without; 165 sequences of 32 heads, 2 layers: 40.0, and 55.5 if theirs had).
  if (p.splits + p.own_parts > 8 && p.rows < 2048) return launch_join<T, D, kJoinThreads / (D / 4)>(p, s);
  return launch_join<T, D, 1>(p, s);
}

}  // namespace

hipError_t launch_paged_shared(const PagedSharedParams &p, int dtype, int head_dim, hipStream_t s) {
  if (dtype == 0) {
    if (head_dim == 64) return launch_typed<float, 64>(p, s);
    return launch_typed<float, 128>(p, s);
  }
  if (head_dim == 64) return launch_typed<bf16_t, 64>(p, s);
  return launch_typed<bf16_t, 128>(p, s);
}

}  // namespace reco
