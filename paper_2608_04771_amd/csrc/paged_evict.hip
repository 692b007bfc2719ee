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
// compact: one workgroup per unit and 128-byte column of K or V, or per unit's
//   weights, moves row idx[p] to row p in ascending chunks.  idx[p] >= p, so a
//   chunk's rows, once all are loaded, can be stored over anything that earlier
//   chunks held, and rows that later chunks read lie behind.
#include "paged_device.hpp"

namespace reco {

namespace {

constexpr int kSelThreads = 1024;
constexpr int kSelWaves = kSelThreads / kWave;
constexpr int kHeld = 16;                    // weights a thread keeps in registers
constexpr int kCopies = 4;                   // copies of each histogram bin
constexpr int kMaxBins = 2048;

__device__ __forceinline__ int wave_incl_scan(int v, int lane) {
#pragma unroll
  for (int d = 1; d < kWave; d <<= 1) {
    const int o = __shfl_up(v, d, kWave);
    if (lane >= d) v += o;
  }
  return v;
}

__global__ __launch_bounds__(kSelThreads) void evict_select_kernel(PagedEvictParams p) {
  __shared__ __attribute__((aligned(16))) int hist[kMaxBins * kCopies];
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
  __syncthreads();

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
    for (int i = tid; i < nb * kCopies / 4; i += kSelThreads) reinterpret_cast<int4 *>(hist)[i] = make_int4(0, 0, 0, 0);
    __syncthreads();
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
    const int incl = wave_incl_scan(first + second, lane);
    if (lane == kWave - 1) wsum[wave] = incl;
    __syncthreads();
    const int wincl = wave_incl_scan(lane < kSelWaves ? wsum[lane] : 0, lane);
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
  if (tid == 0) p.kept[unit] = m;
}

constexpr int kCompThreads = 256;
constexpr int kSliceBytes = 128;
constexpr int kLanesPerRow = kSliceBytes / 16;
constexpr int kRowsPerPass = kCompThreads / kLanesPerRow;
constexpr int kRowsPerThread = 8;
constexpr int kChunkRows = kRowsPerPass * kRowsPerThread;

template <int ROWB>
__global__ __launch_bounds__(kCompThreads) void evict_compact_kernel(PagedEvictParams p) {
  constexpr int kSlices = ROWB / kSliceBytes;
  const int unit = blockIdx.x;
  const int job = blockIdx.y;                            // K slices, V slices, weights
  const size_t cunit = p.c.unit(unit);
  const int m = p.kept[unit];
  if (m < 0) return;
  const int32_t *idx = p.idx + static_cast<size_t>(unit) * p.c.cap;
  const int32_t *table = p.c.pages + cunit * static_cast<size_t>(p.c.max_pages);
  const int shift = p.c.page_shift, mask = (1 << shift) - 1;

  if (job == 2 * kSlices) {
    float *weight = p.c.weight + cunit * p.c.cap;
    for (int c0 = 0; c0 < m; c0 += kCompThreads * 8) {
      float x[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = weight[idx[min(c0 + i * kCompThreads + (int)threadIdx.x, m - 1)]];
      __syncthreads();
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int d = c0 + i * kCompThreads + threadIdx.x;
        if (d < m) weight[d] = x[i];
      }
    }
    if (threadIdx.x == 0) p.c.len[cunit] = m;
    return;
  }
  unsigned char *base = reinterpret_cast<unsigned char *>(job < kSlices ? p.c.k : p.c.v) +
                        (job % kSlices) * kSliceBytes + (threadIdx.x % kLanesPerRow) * 16;
  const int rrow = threadIdx.x / kLanesPerRow;
  const auto at = [&](int row) {
    return base + ((static_cast<size_t>(table[row >> shift]) << shift) + (row & mask)) * ROWB;
  };
  for (int c0 = 0; c0 < m; c0 += kChunkRows) {
    u32x4v v[kRowsPerThread];
#pragma unroll
    for (int i = 0; i < kRowsPerThread; ++i)
      v[i] = *reinterpret_cast<const u32x4v *>(at(idx[min(c0 + i * kRowsPerPass + rrow, m - 1)]));
    __syncthreads();   // every row of this chunk is loaded before any of its places is overwritten
#pragma unroll
    for (int i = 0; i < kRowsPerThread; ++i) {
      const int d = c0 + i * kRowsPerPass + rrow;
      if (d < m) *reinterpret_cast<u32x4v *>(at(d)) = v[i];
    }
  }
}

}  // namespace

hipError_t launch_paged_evict(const PagedEvictParams &p, int dtype, int head_dim, hipStream_t s) {
  const int units = p.c.n_layers * p.c.batch * p.c.hkv;
  hipLaunchKernelGGL(evict_select_kernel, dim3(units), dim3(kSelThreads), 0, s, p);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const int rowb = head_dim * (dtype == 0 ? 4 : 2);
  const dim3 grid(units, 2 * (rowb / kSliceBytes) + 1);
  if (rowb == 128) hipLaunchKernelGGL(evict_compact_kernel<128>, grid, dim3(kCompThreads), 0, s, p);
  else if (rowb == 256) hipLaunchKernelGGL(evict_compact_kernel<256>, grid, dim3(kCompThreads), 0, s, p);
  else hipLaunchKernelGGL(evict_compact_kernel<512>, grid, dim3(kCompThreads), 0, s, p);
  return hipGetLastError();
}

}  // namespace reco
