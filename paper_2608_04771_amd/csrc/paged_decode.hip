// GQA attention of one new token over ragged units of a paged KV cache (gfx950),
// with an optional sliding window, sinks and accumulated attention weights.
//
//   out_g = sum_j p_gj v_j,  p_g = softmax over the seen rows j of scale <q_g, k_j>
//   weight_j += sum_g p_gj
//
// A unit's seen rows are a list of 32-row tiles, cut into `splits` stretches, one
// workgroup each, whose waves take tiles in turn.  Per tile a wave computes
//   S^T = K_tile . Q^T          (16 keys x 16 padded queries per instruction)
//   O^T += V_tile^T . P^T       (16 columns of the head x 16 queries)
// where a lane's four S^T values are the operand P^T wants of it, so P stays in
// registers; K and V go through LDS once each.  Softmax is online, in the log2
// domain, with fp32 maxima, sums and outputs; P alone is rounded to the cache's
// type, as its operand has to be.  It is bound by the rows' bytes.
// Of 28 layers of a 7B shape, 9,645 rows, 83 us or 6.7 TB/s.
//
// Weights need each row's softmax normalised over all splits, which is known only
// at the end: the tiles keep their logits, in LDS where one workgroup has the unit
// and they fit, else in memory (4 bytes per row and query, against 4 D or 8 D of K
// and V), and that workgroup, or the merge kernel's later ones, turn them into weights,
// row by row in the order of the queries, so sums do not depend on scheduling.
#include "paged_device.hpp"
#include "paged_tiles.hpp"

#include <type_traits>

namespace reco {

namespace {

using namespace tiles16;

// Where a unit's new row goes, or that it goes nowhere (the first such code is reported).
template <typename T, int D>
__device__ __forceinline__ bool append_row(const PagedDecodeParams &p, size_t cunit, int len_in, size_t *at) {
  int code = 0;
  if (len_in < 0 || len_in > p.c.cap) code = kDevBadLength;
  else if (p.k_new && len_in == p.c.cap) code = kDevAppendOverflow;
  if (code == 0 && p.k_new) {
    PagedUnit u(p.c, cunit, len_in + 1);
    *at = u.row_at(u.entry(len_in), len_in) * D;
    if (u.bad()) code = kDevBadPage;
  }
  if (code && threadIdx.x == 0) report(p.c.dev_err, code);
  return code == 0 && p.k_new;
}

// Weights of four rows from `row` on: their probabilities summed over the queries.
// seen: what the token sees; n: the rows cached before the call; fresh: row n was appended.
// logits: query 0's of these rows, the others pitch apart.  What the rows had is asked for
// first, so that it comes with the logits.
__device__ __forceinline__ void add_weights(float *weight, const float *logits, int64_t pitch, int group, int row,
                                            const SeenTiles &seen, int n, int cap, bool fresh, const float *top,
                                            const float *inv) {
  float old[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) old[i] = weight[min(row + i, cap - 1)];
  float w[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
  for (int g = 0; g < group; ++g) {
    const float4 x = *reinterpret_cast<const float4 *>(logits + g * pitch);
    w[0] += fast_exp2(x.x - top[g]) * inv[g];
    w[1] += fast_exp2(x.y - top[g]) * inv[g];
    w[2] += fast_exp2(x.z - top[g]) * inv[g];
    w[3] += fast_exp2(x.w - top[g]) * inv[g];
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int j = row + i;
    if (seen.sees(j) && (j < n || fresh)) weight[j] = j < n ? old[i] + w[i] : w[i];
  }
}

template <typename T, int D>
__global__ __launch_bounds__(kSplitWaves * kWave, (Cfg<T, D>::min_wgs)) void paged_split_kernel(PagedDecodeParams p) {
  using C = Cfg<T, D>;
  using MF = Mfma<T>;
  using frag = typename MF::frag;
  constexpr int kThreads = kSplitWaves * kWave;
  __shared__ __attribute__((aligned(16))) unsigned char smem[C::smem()];

  const int lane = threadIdx.x & (kWave - 1);
  const int wave = __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x) / kWave);
  const int col = lane & 15;
  const int grp = lane >> 4;
  const int split = blockIdx.x, unit = blockIdx.y;
  const size_t cunit = p.c.unit(unit);
  const size_t oq0 = static_cast<size_t>(unit) * p.group;

  const int len_in = p.c.len[cunit];
  const int n_cache = len_in < 0 ? 0 : (len_in > p.c.cap ? p.c.cap : len_in);
  const bool append = p.k_new != nullptr;
  const SeenTiles seen(n_cache + (append ? 1 : 0), p.sinks, p.window);
  const T *knew = append ? reinterpret_cast<const T *>(p.k_new) + static_cast<size_t>(unit) * D : nullptr;
  const T *vnew = append ? reinterpret_cast<const T *>(p.v_new) + static_cast<size_t>(unit) * D : nullptr;

  const int per_split = p.by_splits.of(seen.total + p.splits - 1);
  const int i0 = split * per_split;
  const int i1 = min(seen.total, i0 + per_split);

  frag qf[C::qk_steps];
  {
    const T *qrow = reinterpret_cast<const T *>(p.q) + (oq0 + col) * D + grp * C::dq;
#pragma unroll
    for (int c = 0; c < C::qk_steps; ++c) qf[c] = col < p.group ? load_frag(qrow + c * C::kpl) : zero_frag(frag{});
  }

  float m_run = -INFINITY;
  float l_run = 0.f;
  f32x4_t o[C::dtiles];
#pragma unroll
  for (int dt = 0; dt < C::dtiles; ++dt) o[dt] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  unsigned char *stage = smem + wave * C::wave_stage;
  extern __shared__ __attribute__((aligned(16))) float s_logits[];   // [tiles][group][kTile] where they are held
  float *logits = p.logits ? p.logits + (static_cast<size_t>(unit) * p.group + col) * p.logit_pitch + 4 * grp : nullptr;

  // Where the wave's tiles lie: each lane holds the place of 16 rows, so 32 tiles at a
  // time; the table's entries of the batch after are on their way meanwhile.
  constexpr int kBatch = kWave / 2;
  const int mine = i1 - i0 - wave > 0 ? (i1 - i0 - wave + kSplitWaves - 1) / kSplitWaves : 0;   // tiles of the wave
  const int32_t *table = p.c.pages + cunit * static_cast<size_t>(p.c.max_pages);
  const auto tile_of = [&](int k) { return seen.tile(i0 + wave + kSplitWaves * min(k, mine - 1)); };
  const auto row_of = [&](int batch) { return tile_of(batch * kBatch + lane / 2) * kTile + lane % 2 * 16; };
  unsigned worst = 0;
  int coming = 0;
  uint64_t place = 0;
  const auto ask = [&](int batch) { coming = table[max(min(row_of(batch), n_cache - 1), 0) >> p.c.page_shift]; };
  const auto turn = [&](int batch) {
    const unsigned id = min(static_cast<unsigned>(coming), static_cast<unsigned>(p.c.n_pages - 1));
    worst = max(worst, static_cast<unsigned>(coming));
    place = ((static_cast<uint64_t>(id) << p.c.page_shift) + (row_of(batch) & ((1 << p.c.page_shift) - 1))) * C::row_bytes;
    ask(batch + 1);
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
  // Rows of K or V of a tile.  Rows past the last cached one are others of the pool and
  // are masked where they are used; the new row is put where it belongs in LDS.
  const auto load = [&](Rows<T, D> &reg, const void *pool, const Where &w) {
#pragma unroll
    for (int j = 0; j < C::insts; ++j)
      reg[j] = __builtin_nontemporal_load(reinterpret_cast<const u32x4v *>(
          static_cast<const unsigned char *>(pool) + w.at[j / (C::insts / 2)] + j % (C::insts / 2) * (kWave * 16) + lane * 16));
  };
  const auto fresh_row = [&](const T *row) {
    return append ? *reinterpret_cast<const uint4 *>(reinterpret_cast<const unsigned char *>(row) + lane % C::lanes_per_row * 16)
                  : make_uint4(0, 0, 0, 0);
  };
  const uint4 kfresh = fresh_row(knew), vfresh = fresh_row(vnew);

  Rows<T, D> kreg, vreg;
  const auto attend = [&](int k) {
    const int kb = tile_of(k) * kTile;
    const bool whole = seen.whole(kb, n_cache);
    const bool holds_new = append && kb <= n_cache && n_cache < kb + kTile;
    const bool more = k + 1 < mine;
    if (((k + 1) & (kBatch - 1)) == 0) turn((k + 1) / kBatch);
    const Where next = find(k + 1);
#pragma unroll
    for (int j = 0; j < C::insts; ++j) {
      const int r = j * C::rows_per_inst + lane / C::lanes_per_row;
      *reinterpret_cast<u32x4v *>(stage + r * C::k_stride + (lane % C::lanes_per_row) * 16) = kreg[j];
    }
    if (more) load(kreg, p.c.k, next);
    if (holds_new && lane < C::lanes_per_row)
      *reinterpret_cast<uint4 *>(stage + (n_cache - kb) * C::k_stride + lane * 16) = kfresh;
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
      for (int e = 0; e < 8; ++e) x[e] = seen.sees(kb + (e >> 2) * 16 + 4 * grp + (e & 3)) ? x[e] : -INFINITY;
    }
    float top = x[0];
#pragma unroll
    for (int e = 1; e < 8; ++e) top = fmaxf(top, x[e]);
    if (p.c.weight && col < p.group) {
      const float4 a = make_float4(x[0], x[1], x[2], x[3]), b = make_float4(x[4], x[5], x[6], x[7]);
      if (p.held_logits) {
        float *to = s_logits + ((i0 + wave + kSplitWaves * k) * p.group + col) * kTile + 4 * grp;
        *reinterpret_cast<float4 *>(to) = a;
        *reinterpret_cast<float4 *>(to + 16) = b;
      } else {
        *reinterpret_cast<float4 *>(logits + kb) = a;
        *reinterpret_cast<float4 *>(logits + kb + 16) = b;
      }
    }
    const float m_new = fmaxf(m_run, group4_max(top));
    const float ref = m_new == -INFINITY ? 0.f : m_new;   // logits of -inf alone have no weight
    const float alpha = fast_exp2(m_run - ref);
    float pv[8];
    float sum = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      pv[e] = fast_exp2(x[e] - ref);
      sum += pv[e];
    }
    l_run = l_run * alpha + sum;
    m_run = m_new;
#pragma unroll
    for (int dt = 0; dt < C::dtiles; ++dt) {
#pragma unroll
      for (int e = 0; e < 4; ++e) o[dt][e] *= alpha;
    }

    if (!whole) {                                         // a NaN that is not seen, times 0, would be NaN
#pragma unroll
      for (int j = 0; j < C::insts; ++j) {
        const unsigned keep = seen.sees(kb + j * C::rows_per_inst + lane / C::lanes_per_row) ? ~0u : 0u;
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
    if (more) load(vreg, p.c.v, next);
    if (holds_new && lane < C::lanes_per_row) {
      uint2 *dst = reinterpret_cast<uint2 *>(stage + (n_cache - kb) * C::v_stride + lane * 16);
      dst[0] = make_uint2(vfresh.x, vfresh.y);
      dst[1] = make_uint2(vfresh.z, vfresh.w);
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
#pragma unroll
    for (int dt = 0; dt < C::dtiles; ++dt) {
#pragma unroll
      for (int c = 0; c < C::pv_ops; ++c) o[dt] = MF::mma(v_frag<T, D>(stage, c, grp, dt, col), p_frag<T>(pv, c), o[dt]);
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  };

  if (mine > 0) {
    ask(0);
    turn(0);
    const Where first = find(0);
    load(kreg, p.c.k, first);
    load(vreg, p.c.v, first);
    for (int k = 0; k < mine; ++k) attend(k);
  }
  if (worst >= static_cast<unsigned>(p.c.n_pages) && n_cache > 0) report(p.c.dev_err, kDevBadPage);

  const float l_tot = group4_sum(l_run);
  __threadfence_block();                                  // logits, before other waves read them
  __syncthreads();
  float *mw = reinterpret_cast<float *>(smem);            // [kSplitWaves][16]
  float *lw = mw + kSplitWaves * 16;                               // [kSplitWaves][16]
  float *ow = lw + kSplitWaves * 16;                               // [kSplitWaves][16][merge_pitch]
  if (grp == 0) {
    mw[wave * 16 + col] = m_run;
    lw[wave * 16 + col] = l_tot;
  }
#pragma unroll
  for (int dt = 0; dt < C::dtiles; ++dt)
    *reinterpret_cast<float4 *>(ow + (wave * 16 + col) * C::merge_pitch + dt * 16 + 4 * grp) =
        make_float4(o[dt][0], o[dt][1], o[dt][2], o[dt][3]);
  __syncthreads();
  const auto merged = [&](int qi, int d, float &M, float &L) {
    M = -INFINITY;
#pragma unroll
    for (int w = 0; w < kSplitWaves; ++w) M = fmaxf(M, mw[w * 16 + qi]);
    L = 0.f;
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
    const float ref = M == -INFINITY ? 0.f : M;
#pragma unroll
    for (int w = 0; w < kSplitWaves; ++w) {
      const float e = fast_exp2(mw[w * 16 + qi] - ref);
      const float4 v = *reinterpret_cast<const float4 *>(ow + (w * 16 + qi) * C::merge_pitch + d);
      acc.x += v.x * e;
      acc.y += v.y * e;
      acc.z += v.z * e;
      acc.w += v.w * e;
      L += lw[w * 16 + qi] * e;
    }
    return acc;
  };

  if (p.splits > 1) {
    const size_t part = static_cast<size_t>(unit) * p.splits + split;
    float *po = p.part_o + part * p.group * D;
    float *pml = p.part_ml + part * 2 * p.group;
    for (int idx = threadIdx.x; idx < p.group * (D / 4); idx += kThreads) {
      const int qi = idx / (D / 4);
      const int d = (idx - qi * (D / 4)) * 4;
      float M, L;
      const float4 acc = merged(qi, d, M, L);
      *reinterpret_cast<float4 *>(po + qi * D + d) = acc;
      if (d == 0) {
        pml[qi] = M;
        pml[p.group + qi] = L;
      }
    }
    if (split == 0 && threadIdx.x == 0) p.len_in[unit] = len_in;
    return;
  }

  // The workgroup holds its unit's whole softmax.
  __shared__ float s_top[16], s_inv[16];
  for (int idx = threadIdx.x; idx < p.group * (D / 4); idx += kThreads) {
    const int qi = idx / (D / 4);
    const int d = (idx - qi * (D / 4)) * 4;
    float M, L;
    const float4 acc = merged(qi, d, M, L);
    const float inv = L == 0.f ? 0.f : 1.f / L;
    T *dst = reinterpret_cast<T *>(p.out) + (oq0 + qi) * D + d;
    dst[0] = from_f32<T>(acc.x * inv);
    dst[1] = from_f32<T>(acc.y * inv);
    dst[2] = from_f32<T>(acc.z * inv);
    dst[3] = from_f32<T>(acc.w * inv);
    if (d == 0) {
      if (p.lse) p.lse[oq0 + qi] = L == 0.f ? -INFINITY : (M + log2f(L)) * kLn2;
      s_top[qi] = M == -INFINITY ? 0.f : M;
      s_inv[qi] = inv;
    }
  }
  // No one reads row n_cache of the cache or changes len in this call before here.
  size_t at = 0;
  const bool put = append_row<T, D>(p, cunit, len_in, &at);
  if (put) {
    for (int d = threadIdx.x; d < D; d += kThreads) {
      reinterpret_cast<T *>(p.c.k)[at + d] = knew[d];
      reinterpret_cast<T *>(p.c.v)[at + d] = vnew[d];
    }
    if (threadIdx.x == 0) p.c.len[cunit] = len_in + 1;
  }
  if (!p.c.weight) return;
  __syncthreads();
  const float *lg = p.logits + static_cast<size_t>(unit) * p.group * p.logit_pitch;
  float *weight = p.c.weight + cunit * p.c.cap;
  for (int k = threadIdx.x; k < seen.total * (kTile / 4); k += kThreads) {
    const int i = k / (kTile / 4), in = k % (kTile / 4) * 4;
    const int row = seen.tile(i) * kTile + in;
    if (p.held_logits)
      add_weights(weight, s_logits + i * p.group * kTile + in, kTile, p.group, row, seen, n_cache, p.c.cap, put, s_top, s_inv);
    else
      add_weights(weight, lg + row, p.logit_pitch, p.group, row, seen, n_cache, p.c.cap, put, s_top, s_inv);
  }
}

// Joins the splits.  Workgroups [0, units * group) take one query head of one unit
// each: every split's slice is asked for at once, together with the statistics, and
// the weighted slices meet in LDS; query head 0 of a unit commits the append.  The
// others, where weights are kept, take kPagedWeightRows seen rows of a unit each.
constexpr int kMergeThreads = 256;
static_assert(kPagedWeightRows == kMergeThreads * 4, "four rows a thread");

template <typename T, int D>
__global__ __launch_bounds__(kMergeThreads) void paged_merge_kernel(PagedDecodeParams p, int weight_chunks) {
  constexpr int kTPS = D / 4;                             // threads per split slice
  constexpr int kSG = kMergeThreads / kTPS;               // slices read together
  constexpr int kMaxPer = kPagedMaxSplits / kSG;
  constexpr int kWaves = kMergeThreads / kWave;
  __shared__ float s_w[kPagedMaxSplits];
  __shared__ float s_red[2][kWaves];
  __shared__ __attribute__((aligned(16))) float s_acc[kSG][D];
  __shared__ float s_top[16], s_inv[16];

  const int tid = threadIdx.x;
  const int lane = tid & (kWave - 1);
  const int wave = tid / kWave;
  const int S = p.splits, G = p.group;
  const int units = p.c.n_layers * p.c.batch * p.c.hkv;
  const int id = blockIdx.x;
  const bool merging = id < units * G;
  const int unit = merging ? p.by_group.of(id) : (id - units * G) / weight_chunks;
  const size_t cunit = p.c.unit(unit);
  const float *pml = p.part_ml + static_cast<size_t>(unit) * S * 2 * G;

  if (!merging) {
    const int len_in = p.len_in[unit];                    // len itself changes during this kernel
    const int n = len_in < 0 ? 0 : (len_in > p.c.cap ? p.c.cap : len_in);
    const SeenTiles seen(n + (p.k_new ? 1 : 0), p.sinks, p.window);
    const int k = ((id - units * G) % weight_chunks) * kMergeThreads + tid;
    if ((k - tid) / (kTile / 4) >= seen.total) return;    // the same for the workgroup
    for (int g = wave; g < G; g += kWaves) {
      const float m0 = lane < S ? pml[lane * 2 * G + g] : -INFINITY;
      const float l0 = lane < S ? pml[lane * 2 * G + G + g] : 0.f;
      const float m1 = lane + kWave < S ? pml[(lane + kWave) * 2 * G + g] : -INFINITY;
      const float l1 = lane + kWave < S ? pml[(lane + kWave) * 2 * G + G + g] : 0.f;
      const float M = wave_max(fmaxf(m0, m1));
      const float ref = M == -INFINITY ? 0.f : M;
      const float L = wave_sum(l0 * fast_exp2(m0 - ref) + l1 * fast_exp2(m1 - ref));
      if (lane == 0) {
        s_top[g] = ref;
        s_inv[g] = L == 0.f ? 0.f : 1.f / L;
      }
    }
    __syncthreads();
    if (k / (kTile / 4) >= seen.total) return;
    bool fresh = false;
    if (p.k_new && len_in >= 0 && len_in < p.c.cap) {
      PagedUnit u(p.c, cunit, len_in + 1);
      u.row_at(u.entry(len_in), len_in);
      fresh = !u.bad();
    }
    const int row = seen.tile(k / (kTile / 4)) * kTile + k % (kTile / 4) * 4;
    add_weights(p.c.weight + cunit * p.c.cap, p.logits + static_cast<size_t>(unit) * G * p.logit_pitch + row, p.logit_pitch,
                G, row, seen, n, p.c.cap, fresh, s_top, s_inv);
    return;
  }

  const int qi = id - unit * G;
  const bool append = p.k_new != nullptr && qi == 0;
  const int len_in = qi == 0 ? p.c.len[cunit] : 0;
  T krow = T{}, vrow = T{};
  if (append && tid < D) {
    krow = reinterpret_cast<const T *>(p.k_new)[static_cast<size_t>(unit) * D + tid];
    vrow = reinterpret_cast<const T *>(p.v_new)[static_cast<size_t>(unit) * D + tid];
  }
  const int sg = tid / kTPS;
  const int dv = (tid % kTPS) * 4;
  const float *po = p.part_o + (static_cast<size_t>(unit) * S * G + qi) * D;
  float4 part[kMaxPer];
#pragma unroll
  for (int i = 0; i < kMaxPer; ++i) {
    const int sp = sg + kSG * i;
    part[i] = sp < S ? *reinterpret_cast<const float4 *>(po + static_cast<size_t>(sp) * G * D + dv)
                     : make_float4(0.f, 0.f, 0.f, 0.f);
  }
  const float m_t = tid < S ? pml[tid * 2 * G + qi] : -INFINITY;
  const float l_t = tid < S ? pml[tid * 2 * G + G + qi] : 0.f;

  float v = wave_max(m_t);
  if (lane == 0) s_red[0][wave] = v;
  __syncthreads();
  float M = s_red[0][0];
#pragma unroll
  for (int w = 1; w < kWaves; ++w) M = fmaxf(M, s_red[0][w]);
  const float e_t = fast_exp2(m_t - (M == -INFINITY ? 0.f : M));
  v = wave_sum(l_t * e_t);
  if (lane == 0) s_red[1][wave] = v;
  __syncthreads();
  float L = 0.f;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) L += s_red[1][w];
  if (tid < kPagedMaxSplits) s_w[tid] = L == 0.f ? 0.f : e_t / L;
  __syncthreads();

  float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
  for (int i = 0; i < kMaxPer; ++i) {
    const int sp = sg + kSG * i;
    const float w = sp < S ? s_w[sp] : 0.f;
    acc.x += w * part[i].x;
    acc.y += w * part[i].y;
    acc.z += w * part[i].z;
    acc.w += w * part[i].w;
  }
  *reinterpret_cast<float4 *>(&s_acc[sg][dv]) = acc;
  __syncthreads();
  const size_t oq = static_cast<size_t>(unit) * G + qi;
  if (tid < D) {
    float o = 0.f;
#pragma unroll
    for (int g = 0; g < kSG; ++g) o += s_acc[g][tid];
    reinterpret_cast<T *>(p.out)[oq * D + tid] = from_f32<T>(o);
  }
  if (p.lse && tid == 0) p.lse[oq] = L == 0.f ? -INFINITY : (M + log2f(L)) * kLn2;
  if (qi != 0) return;
  size_t at = 0;
  if (!append_row<T, D>(p, cunit, len_in, &at)) return;
  if (tid < D) {
    reinterpret_cast<T *>(p.c.k)[at + tid] = krow;
    reinterpret_cast<T *>(p.c.v)[at + tid] = vrow;
  }
  if (tid == 0) p.c.len[cunit] = len_in + 1;
}

constexpr int kLdsBytes = 160 * 1024;        // of a compute unit

template <typename T, int D>
hipError_t launch_typed(const PagedDecodeParams &p, hipStream_t s) {
  const int units = p.c.n_layers * p.c.batch * p.c.hkv;
  // Logits are held in LDS where one workgroup has a unit's whole softmax and they fit
  // beside its stages, twice on a compute unit where there are more units than those:
  // writes among the reads cost them much of their rate (256 units of 4,225 rows and
  // 4 heads, whose logits are 3% of the bytes: 110 us through memory, 90 held).
  PagedDecodeParams q = p;
  const int64_t room = (units > p.cus ? kLdsBytes / 2 : kLdsBytes) - Cfg<T, D>::smem() - 1024;
  const int64_t need = p.c.weight && p.splits == 1
                           ? static_cast<int64_t>(paged_span_tiles(p.c.cap, p.sinks, p.window)) * p.group * kTile * 4 : 0;
  q.held_logits = need > 0 && need <= room;
  const int held = q.held_logits ? static_cast<int>(need) : 0;
  hipLaunchKernelGGL((paged_split_kernel<T, D>), dim3(p.splits, units), dim3(kSplitWaves * kWave), held, s, q);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || p.splits == 1) return e;         // one split: finished in place
  const int chunks = paged_weight_chunks(p);
  hipLaunchKernelGGL((paged_merge_kernel<T, D>), dim3(units * (p.group + chunks)), dim3(kMergeThreads), 0, s, p,
                     chunks);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_paged_decode(const PagedDecodeParams &p, int dtype, int head_dim, hipStream_t s) {
  if (dtype == 0) {
    if (head_dim == 64) return launch_typed<float, 64>(p, s);
    return launch_typed<float, 128>(p, s);
  }
  if (head_dim == 64) return launch_typed<bf16_t, 64>(p, s);
  return launch_typed<bf16_t, 128>(p, s);
}

}  // namespace reco
