// Eviction from a paged KV cache by accumulated attention weight (gfx950).
//
// select: one 1024-thread workgroup per unit.  The rows to choose from lie between
//   the sinks and the recent rows; the k-th largest of their weights is found with
//   an exact radix select on the fp32 bit patterns (weights are not negative, so
//   they order like their bits): histograms of 11, 11 and 10 bits give the value
//   theta and how many rows equal to it are still needed, the first ones.  Each
//   wave owns a stretch of rows, 64 at a time, so ballots and one sum over the
//   waves' counts give every kept row its place.  Up to kHeld weights a thread stay
//   in registers.
// compact: moves row idx[p] to row p, K, V and weight, in chunks of 32 KB of K and of V
//   that a unit's workgroups take in ascending order.  idx[p] >= p, so a chunk's places
//   hold rows that it or an earlier chunk moves: a workgroup loads its chunk into
//   registers, says so, waits until all earlier chunks of the unit are loaded, and
//   stores.  Loading waits for nothing and chunks are taken in order by workgroups that
//   run, so the wait ends whatever the order of dispatch.  It is bounded all the same:
//   a workgroup that waits in vain (its workspace is another call's, too) stores nothing
//   and reports it, and len changes only once all chunks are stored.  It is bound by the rows'
//   bytes (112 units, 9,516 of 16,384 rows of 2 x 256 bytes: 225 us, 4.9 TB/s; with
//   chunks of 16 KB 248); a chunk of rows that stay where they are is not read.
#include "paged_device.hpp"

namespace reco {

namespace {

constexpr int kSelThreads = 1024;
constexpr int kSelWaves = kSelThreads / kWave;
constexpr int kHeld = 16;                    // weights a thread keeps in registers
constexpr int kCopies = 4;                   // copies of each histogram bin
constexpr int kMaxBins = 2048;

// Sum of the lanes up to this one: within rows of 16 lanes, then rows 1 and 3 take the
// last lane of the row before, and the upper half the last of the lower.
__device__ __forceinline__ int wave_incl_scan(int v) {
  v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xf, 0xf, false);   // row_shr 1, 2, 4, 8
  v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xa, 0xf, false);   // row_bcast 15
  v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xc, 0xf, false);   // row_bcast 31
  return v;
}

__global__ __launch_bounds__(kSelThreads) void evict_select_kernel(PagedEvictParams p) {
  __shared__ __attribute__((aligned(16))) int hists[2][kMaxBins * kCopies];   // in turn
  __shared__ int wsum[kSelWaves];
  __shared__ int2 wcount[kSelWaves];
  __shared__ int s_bin, s_krem, s_bad;

  const int unit = blockIdx.x;
  const size_t cunit = p.c.unit(unit);
  const int seq = p.c.by_hkv.of(unit);                 // of all layers
  const int lc = p.c.by_batch.of(seq), b = p.c.by_batch.rest(seq);
  const int tid = threadIdx.x;
  const int lane = tid & (kWave - 1);
  const int wave = tid / kWave;
  int32_t *idx = p.idx + static_cast<size_t>(unit) * p.c.cap;

  const int L = p.c.len[cunit];
  const int m = p.budget[static_cast<int64_t>(lc) * p.budget_stride + b];
  int code = 0;
  if (L < 0 || L > p.c.cap) code = kDevBadLength;
  else if (m < 1 || static_cast<int64_t>(p.sinks) + p.recent > m) code = kDevBadBudget;
  if (code || L <= m) {
    if (!code && p.idx_wanted)
      for (int j = tid; j < L; j += kSelThreads) idx[j] = j;
    if (tid == 0) {
      if (code) report(p.c.dev_err, code);
      p.kept[unit] = -1;
    }
    return;
  }
  if (tid == 0) s_bad = 0;
  for (int i = tid; i < 2 * kMaxBins * kCopies / 4; i += kSelThreads) reinterpret_cast<int4 *>(hists)[i] = make_int4(0, 0, 0, 0);

  const int lo = p.sinks, hi = L - p.recent;           // the rows to choose from
  const int k = m - p.sinks - p.recent;                // of them
  const float *weight = p.c.weight + cunit * p.c.cap;
  const int turns = (L + kSelThreads - 1) / kSelThreads;
  const int j0 = wave * turns * kWave + lane;
  const bool held = turns <= kHeld;
  bool bad = false;
  const auto bits = [&](int j) {
    uint32_t u = j >= lo && j < hi ? __float_as_uint(weight[j]) : 0u;
    if (u == 0x80000000u) u = 0;                       // -0 ranks as +0
    if ((u >> 31) || u > 0x7f800000u) bad = true;      // negative or NaN
    return u;
  };
  uint32_t kept_bits[kHeld];
  if (held) {
#pragma unroll
    for (int i = 0; i < kHeld; ++i) kept_bits[i] = i < turns ? bits(j0 + i * kWave) : 0u;
  }
  // f(bits, row) for every row of this lane, in order and by whole waves; rows past L come too.
  const auto for_each = [&](auto f) {
    if (held) {
#pragma unroll
      for (int i = 0; i < kHeld; ++i)
        if (i < turns) f(kept_bits[i], j0 + i * kWave);
    } else {
#pragma unroll 4
      for (int i = 0; i < turns; ++i) f(bits(j0 + i * kWave), j0 + i * kWave);
    }
  };
  __syncthreads();                                     // the histograms are clear, and s_bad
  // The unit's pages, which the compaction then trusts.
  int page_bad = 0;
  const int32_t *table = p.c.pages + cunit * static_cast<size_t>(p.c.max_pages);
  for (int g = tid; g < ((L - 1) >> p.c.page_shift) + 1; g += kSelThreads)
    if (static_cast<unsigned>(table[g]) >= static_cast<unsigned>(p.c.n_pages)) page_bad = 1;
  if (page_bad) atomicOr(&s_bad, 2);

  uint32_t prefix = 0, pmask = 0;
  int krem = k;
  const int shifts[3] = {21, 10, 0};
  const int nbits[3] = {11, 11, 10};
  for (int pass = 0; pass < 3; ++pass) {
    const int sh = shifts[pass];
    const int nb = 1 << nbits[pass];
    int *hist = hists[pass & 1];
    if (pass == 1)                                       // for the last pass
      for (int i = tid; i < (1 << 10) * kCopies / 4; i += kSelThreads) reinterpret_cast<int4 *>(hists[0])[i] = make_int4(0, 0, 0, 0);
    for_each([&](uint32_t u, int j) {
      if (j >= lo && j < hi && (u & pmask) == prefix) atomicAdd(&hist[((u >> sh) & (nb - 1)) * kCopies + lane % kCopies], 1);
    });
    if (bad) atomicOr(&s_bad, 1);
    __syncthreads();
    if (s_bad || k == 0) break;
    // Find the bin of the krem-th largest: thread t has bins 2t and 2t + 1, or bin t alone.
    static_assert(kCopies == 4 && kMaxBins == 2 * kSelThreads, "one int4 per bin, at most two bins per thread");
    const auto count = [&](int bin) {
      const int4 c = reinterpret_cast<const int4 *>(hist)[bin];
      return c.x + c.y + c.z + c.w;
    };
    const bool two = nb == kMaxBins;
    const int first = two ? count(2 * tid) : count(tid);
    const int second = two ? count(2 * tid + 1) : 0;
    const int incl = wave_incl_scan(first + second);
    if (lane == kWave - 1) wsum[wave] = incl;
    __syncthreads();
    const int wincl = wave_incl_scan(lane < kSelWaves ? wsum[lane] : 0);
    const int total = __shfl(wincl, kSelWaves - 1, kWave);
    const int before = wave == 0 ? 0 : __shfl(wincl, wave - 1, kWave);
    const int above = total - before - incl;           // rows in the bins of later threads
    if (above < krem && krem <= above + first + second) {
      const bool in_second = krem <= above + second;
      s_bin = two ? 2 * tid + (in_second ? 1 : 0) : tid;
      s_krem = krem - above - (in_second ? 0 : second);
    }
    __syncthreads();
    prefix |= static_cast<uint32_t>(s_bin) << sh;
    pmask |= static_cast<uint32_t>(nb - 1) << sh;
    krem = s_krem;
  }
  if (s_bad) {
    if (tid == 0) {
      report(p.c.dev_err, s_bad & 2 ? kDevBadPage : kDevBadScore);
      p.kept[unit] = -1;
    }
    return;
  }

  // Keep what is safe, weights above theta, and the first `need` equal to it.
  const uint32_t theta = k == 0 ? 0xffffffffu : prefix;
  const int need = k == 0 ? 0 : krem;
  const auto safe = [&](int j) { return j < lo || (j >= hi && j < L); };
  int n_keep = 0, n_eq = 0;                              // of this wave
  for_each([&](uint32_t u, int j) {
    const bool cand = j >= lo && j < hi;
    n_keep += __popcll(__ballot(safe(j) || (cand && u > theta)));
    n_eq += __popcll(__ballot(cand && u == theta));
  });
  if (lane == 0) wcount[wave] = make_int2(n_keep, n_eq);
  __syncthreads();
  int eq = 0, pos = 0;                                   // rows equal to theta, and kept ones, so far
  for (int w = 0; w < wave; ++w) {
    pos += wcount[w].x;
    eq += wcount[w].y;
  }
  pos += min(eq, need);
  const uint64_t below = (1ull << lane) - 1;
  for_each([&](uint32_t u, int j) {
    const bool cand = j >= lo && j < hi;
    const bool is_eq = cand && u == theta;
    const uint64_t eq_mask = __ballot(is_eq);
    const bool keep = safe(j) || (cand && u > theta) || (is_eq && eq + __popcll(eq_mask & below) < need);
    const uint64_t keep_mask = __ballot(keep);
    if (keep) idx[pos + __popcll(keep_mask & below)] = j;
    pos += __popcll(keep_mask);
    eq += __popcll(eq_mask);
  });
  int32_t *state = p.state + static_cast<size_t>(unit) * p.state_pitch;
  for (int i = tid; i < kEvictState + (m + p.chunk_rows - 1) / p.chunk_rows; i += kSelThreads) state[i] = 0;
  if (tid == 0) p.kept[unit] = m;
}

constexpr int kCompThreads = 256;
// LDS that no one uses keeps three workgroups on a compute unit: fewer or more of them
// cost rate (all 28 layers of a 7B shape, per call: 257 us with 2.6 on a compute unit, 268
// with 1.3; in chunks of 16 KB 280 with 2.6, 308 with 7.9).
constexpr int kCompLds = 48 * 1024;

__device__ __forceinline__ int relaxed_load(const int32_t *p) {
  return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

template <int ROWB>
__global__ __launch_bounds__(kCompThreads) void evict_compact_kernel(PagedEvictParams p) {
  constexpr int kLanesPerRow = ROWB / 16;
  constexpr int kRowsPerPass = kCompThreads / kLanesPerRow;
  constexpr int kPasses = evict_chunk_rows(ROWB) / kRowsPerPass;
  constexpr int kRows = kPasses * kRowsPerPass;
  static_assert(kRows <= kCompThreads, "a weight a thread");
  __shared__ int s_ticket, s_known, s_stalled;

  const int unit = blockIdx.x;
  const int tid = threadIdx.x;
  const size_t cunit = p.c.unit(unit);
  const int m = p.kept[unit];
  if (m < 0) return;
  const int32_t *idx = p.idx + static_cast<size_t>(unit) * p.c.cap;
  const int32_t *table = p.c.pages + cunit * static_cast<size_t>(p.c.max_pages);
  const int shift = p.c.page_shift, mask = (1 << shift) - 1;
  int32_t *ticket = p.state + static_cast<size_t>(unit) * p.state_pitch;
  int32_t *prefix = ticket + 1;                          // chunks before this one are known to be loaded
  int32_t *stored = ticket + 2;                          // chunks that are, or are being, stored
  int32_t *loaded = ticket + kEvictState;
  unsigned char *k = reinterpret_cast<unsigned char *>(p.c.k) + tid % kLanesPerRow * 16;
  unsigned char *v = reinterpret_cast<unsigned char *>(p.c.v) + tid % kLanesPerRow * 16;
  float *weight = p.c.weight + cunit * p.c.cap;
  const auto at = [&](int row) { return ((static_cast<size_t>(table[row >> shift]) << shift) + (row & mask)) * ROWB; };

  // A chunk, and before which one all are known to be loaded: the same for the whole
  // workgroup, so that its waves together wait for every chunk between the two.
  const auto take = [&] {
    const int chunk = atomicAdd(ticket, 1), before = relaxed_load(prefix);
    s_ticket = chunk;
    s_known = before;
  };
  if (tid == 0) {
    s_stalled = 0;
    take();
  }
  __syncthreads();
  int mine = 0;                                          // chunks that this workgroup stores
  for (;;) {
    const int c = s_ticket, known = s_known;
    const int r0 = c * kRows;
    if (r0 >= m) break;                                  // the same for the workgroup
    const int last = min(r0 + kRows, m) - 1;
    const bool moves = idx[last] != last;
    int from[kPasses], wfrom = 0;
#pragma unroll
    for (int i = 0; i < kPasses; ++i) from[i] = idx[min(r0 + i * kRowsPerPass + tid / kLanesPerRow, last)];
    if (tid < kRows) wfrom = idx[min(r0 + tid, last)];
    u32x4v kr[kPasses], vr[kPasses];
    float w = 0.f;
    if (moves) {
#pragma unroll
      for (int i = 0; i < kPasses; ++i) {
        const size_t o = at(from[i]);
        kr[i] = __builtin_nontemporal_load(reinterpret_cast<const u32x4v *>(k + o));
        vr[i] = __builtin_nontemporal_load(reinterpret_cast<const u32x4v *>(v + o));
      }
      if (tid < kRows) w = weight[wfrom];
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");     // the rows are in registers
    __syncthreads();
    if (tid == 0) {
      __hip_atomic_store(&loaded[c], 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      take();
    }
    // Bounded, so that a workspace that another call writes meanwhile cannot hang the device.
    int spins = 0;
    for (int f = known + tid; f < c && spins <= p.max_spins; f += kCompThreads)
      while (!relaxed_load(&loaded[f]) && ++spins <= p.max_spins) __builtin_amdgcn_s_sleep(1);
    if (spins > p.max_spins) s_stalled = 1;
    __syncthreads();
    if (s_stalled) {                                     // rows that this chunk's would replace may still be wanted
      if (tid == 0) report(p.c.dev_err, kDevStalled);
      return;
    }
    // Nothing keeps the chunk from being stored now: whoever counts the unit's last one
    // sets its length, beside the stores.
    ++mine;
    int count = 0;
    if (tid == 0) {
      atomicMax(prefix, c);
      if (s_ticket * kRows >= m) count = atomicAdd(stored, mine) + mine;
    }
    if (moves) {
#pragma unroll
      for (int i = 0; i < kPasses; ++i) {
        const int row = r0 + i * kRowsPerPass + tid / kLanesPerRow;
        if (row <= last) {
          const size_t o = at(row);
          __builtin_nontemporal_store(kr[i], reinterpret_cast<u32x4v *>(k + o));
          __builtin_nontemporal_store(vr[i], reinterpret_cast<u32x4v *>(v + o));
        }
      }
      if (r0 + tid <= last && tid < kRows) weight[r0 + tid] = w;
    }
    if (tid == 0 && count == (m + kRows - 1) / kRows) p.c.len[cunit] = m;
  }
}

}  // namespace

hipError_t launch_paged_evict(const PagedEvictParams &p, int dtype, int head_dim, hipStream_t s) {
  const int units = p.c.n_layers * p.c.batch * p.c.hkv;
  hipLaunchKernelGGL(evict_select_kernel, dim3(units), dim3(kSelThreads), 0, s, p);
  hipError_t e = hipGetLastError();
  return e != hipSuccess ? e : launch_evict_compact(p, head_dim * (dtype == 0 ? 4 : 2), s);
}

hipError_t launch_evict_compact(const PagedEvictParams &p, int rowb, hipStream_t s) {
  const dim3 grid(p.c.n_layers * p.c.batch * p.c.hkv, p.workers);
  if (rowb == 128) hipLaunchKernelGGL(evict_compact_kernel<128>, grid, dim3(kCompThreads), kCompLds, s, p);
  else if (rowb == 256) hipLaunchKernelGGL(evict_compact_kernel<256>, grid, dim3(kCompThreads), kCompLds, s, p);
  else hipLaunchKernelGGL(evict_compact_kernel<512>, grid, dim3(kCompThreads), kCompLds, s, p);
  return hipGetLastError();
}

}  // namespace reco
