// Rotation of query and key rows by their positions (gfx950), and the append of the
// rotated keys, and of values as they are, to the pages of their units.
//
//   a_i = pos[axis(i)] inv_freq[i];   (x_i, y_i) <- (x_i cos a_i - y_i sin a_i, x_i sin a_i + y_i cos a_i)
//
// A workgroup takes a block of tokens of one sequence and layer, all heads of them, so
// that an angle is computed once for all heads: in turns, pos (inv_freq / 2 pi) in 64
// bits, of which the whole turns are dropped exactly, so that far positions lose
// nothing; sine and cosine of the rest in fp32, rows in fp32 between their loads and
// stores.  A thread holds 16 bytes of each end of its pairs, of one token, and goes
// through the heads.  Bound by the rows' bytes: 16,384 tokens of 32 heads in bf16, 269 MB in 48 us
// (5.6 TB/s; a copy reaches 4.9), with K and V of 16,384 tokens appended besides, 302 MB in 68 us
// (4.5 TB/s: writes go to pages) and 5 us for the lengths; fp32, half as many tokens: 50 us, and
// 70 and 5.  One token takes 2.6 us, of 32
// sequences with its append 5.8: a launch and the round trips to positions, page ids and rows.
// Blocks of 2, 8, 16 or 32 tokens and 512 or 1,024 threads were slower on long runs.
#include "paged_device.hpp"
#include "rope.hpp"

namespace reco {

namespace {

template <typename T, int D, int THREADS>
struct Cfg {
  static constexpr int vec = 16 / (int)sizeof(T);        // elements of a load, pairs of a thread
  static constexpr int per_row = D / (2 * vec);          // threads of a row
  static constexpr int rows = THREADS / per_row;         // of a turn of the workgroup
};

template <typename T>
struct Vec {
  T x[16 / sizeof(T)];
};
template <typename T>
__device__ __forceinline__ Vec<T> unpack(u32x4v w) { return __builtin_bit_cast(Vec<T>, w); }
template <typename T>
__device__ __forceinline__ u32x4v pack(const Vec<T> &v) { return __builtin_bit_cast(u32x4v, v); }

template <typename T>
__device__ __forceinline__ void turn_pair(T x, T y, float2 turn, T &u, T &w) {
  const float g = to_f32(x), o = to_f32(y);
  u = from_f32<T>(g * turn.x - o * turn.y);
  w = from_f32<T>(g * turn.y + o * turn.x);
}

// Real tokens of a sequence; a bad count is none.
__device__ __forceinline__ int new_tokens(const RopeParams &p, int b, bool &bad) {
  const int given = p.n_new ? p.n_new[b] : p.tokens;
  bad = given < 0 || given > p.tokens;
  return bad ? 0 : given;
}

// What stops n rows from being appended behind L ones, in the order of the checks.
__device__ __forceinline__ int append_code(const PagedCache &c, int L, int n, bool bad_page) {
  if (L < 0 || L > c.cap) return kDevBadLength;
  if (n > c.cap - L) return kDevAppendOverflow;
  return bad_page && n > 0 ? kDevBadPage : 0;
}

template <typename T, int D, bool kAppend, int THREADS, bool kFar>
__global__ __launch_bounds__(THREADS) void rope_kernel(RopeParams p) {
  using C = Cfg<T, D, THREADS>;
  __shared__ __attribute__((aligned(16))) float2 s_turn[kRopeMaxBlock][D / 2];
  extern __shared__ __attribute__((aligned(16))) int64_t s_to[];     // [hkv][block]  element of the pool, or -1
  const int tid = threadIdx.x;
  const int b = blockIdx.y, l = blockIdx.z;
  const int t0 = blockIdx.x * p.block;
  bool bad;
  const int n = new_tokens(p, b, bad);
  if (bad && t0 == 0 && l == 0 && tid == 0) report(p.dev_err, kDevBadLength);
  const bool all = p.tokens <= p.block;                   // the workgroup has whole runs, and sets the lengths
  if (t0 >= n && !(kAppend && all)) return;

  // Where this thread's elements lie, and its token.
  const int sub = tid % C::per_row;
  const int slot = tid / C::per_row;
  const int at_t = slot & (p.block - 1);
  const int t = t0 + at_t;
  const int step = C::rows / p.block;                     // heads of a turn
  // Two pieces of the row, of neighbouring threads beside each other: of halves the two ends
  // of the same pairs, or two of what passes; of neighbouring pairs any two.
  const int half = p.pairs ? D / 2 : p.rot / 2;
  const bool low = sub * C::vec < half;
  const int e0 = low ? sub * C::vec : p.rot + sub * C::vec - half;
  const int e1 = low ? half + e0 : e0 + (D - p.rot) / 2;
  const bool turns0 = e0 < p.rot, turns1 = e1 < p.rot;
  const int rows = p.heads + (kAppend ? 2 * p.c.hkv : 0);
  const bool real = t < n;

  const T *q = nullptr, *k = nullptr, *v = nullptr;
  if (p.heads) q = p.q.at<const T>(l, b, t);
  if (kAppend) {
    k = p.k.at<const T>(l, b, t);
    v = p.v.at<const T>(l, b, t);
  }
  const auto source = [&](int r) {
    if (kAppend && r >= p.heads) {
      const int h = r - p.heads;
      return h < p.c.hkv ? k + h * p.k.head : v + (h - p.c.hkv) * p.v.head;
    }
    return q + r * p.q.head;
  };
  // One row of a thread comes while another goes.  More of them on their way made long runs
  // slower (16,384 tokens of 36 heads: 71 us by ones, 80 by twos, 82 by fours without turns).
  constexpr int kAhead = 1;
  u32x4v lo_a[kAhead], hi_a[kAhead], lo_b[kAhead], hi_b[kAhead];
  const auto load = [&](int r0, u32x4v (&lo)[kAhead], u32x4v (&hi)[kAhead]) {
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      const int r = r0 + i * step;
      if (real && r < rows) {
        const T *src = source(r);
        const u32x4v *x = reinterpret_cast<const u32x4v *>(src + e0), *y = reinterpret_cast<const u32x4v *>(src + e1);
        lo[i] = kFar ? __builtin_nontemporal_load(x) : *x;
        hi[i] = kFar ? __builtin_nontemporal_load(y) : *y;
      }
    }
  };
  const int first = slot / p.block;
  load(first, lo_a, hi_a);

  for (int i = tid; i < p.block * (p.rot / 2); i += THREADS) {
    const int pair = i % (p.rot / 2), tt = i / (p.rot / 2);
    if (t0 + tt >= n) break;
    const int axis = static_cast<int>(p.axis[pair / 32] >> (2 * (pair % 32))) & 3;
    const int pos = p.pos[(static_cast<size_t>(axis) * p.batch + b) * p.tokens + t0 + tt];
    constexpr double kPerTurn = 0.15915494309189533577;   // 1 / (2 pi)
    const double turn = static_cast<double>(pos) * (static_cast<double>(p.freq[pair]) * kPerTurn);
    float s, c;
    sincospif(2.f * static_cast<float>(turn - rint(turn)), &s, &c);
    s_turn[tt][pair] = make_float2(c, s);
  }
  if (kAppend) {
    const int shift = p.c.page_shift;
    for (int i = tid; i < p.c.hkv * p.block; i += THREADS) {
      const int tt = i & (p.block - 1), h = i / p.block;
      const size_t cunit = p.c.unit((l * p.batch + b) * p.c.hkv + h);
      const int L = p.c.len[cunit], row = L + t0 + tt;
      int64_t to = -1;
      if (t0 + tt < n && L >= 0 && L <= p.c.cap && t0 + tt < p.c.cap - L) {
        const int id = p.c.pages[cunit * static_cast<size_t>(p.c.max_pages) + (row >> shift)];
        if (static_cast<unsigned>(id) < static_cast<unsigned>(p.c.n_pages))
          to = ((static_cast<int64_t>(id) << shift) + (row & ((1 << shift) - 1))) * D;
        if (to >= 0 && p.c.weight) p.c.weight[cunit * p.c.cap + row] = 0.f;
      }
      s_to[i] = to;
    }
  }
  __syncthreads();
  if (kAppend && all) {
    for (int h = tid; h < p.c.hkv; h += THREADS) {
      const size_t cunit = p.c.unit((l * p.batch + b) * p.c.hkv + h);
      const int L = p.c.len[cunit];
      bool bad_page = false;
      for (int tt = 0; tt < n; ++tt) bad_page |= s_to[h * p.block + tt] < 0;
      const int code = append_code(p.c, L, n, bad_page);
      if (code) report(p.dev_err, code);
      else if (n > 0) p.c.len[cunit] = L + n;
    }
  }
  // The angles of this thread's pairs; with neighbouring pairs half of them are its second piece's.
  float2 turn[C::vec];
#pragma unroll
  for (int j = 0; j < C::vec; ++j) {
    const int pair = !p.pairs ? e0 + j : j < C::vec / 2 ? e0 / 2 + j : e1 / 2 + j - C::vec / 2;
    turn[j] = s_turn[at_t][min(pair, D / 2 - 1)];
  }

  const auto put = [&](int r0, const u32x4v (&lo)[kAhead], const u32x4v (&hi)[kAhead]) {
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      const int r = r0 + i * step;
      if (!real || r >= rows) break;
      const int h = r - p.heads;
      T *dst;
      bool turned = true;
      if (kAppend && h >= 0) {
        const bool key = h < p.c.hkv;
        const int64_t to = s_to[(key ? h : h - p.c.hkv) * p.block + at_t];
        if (to < 0) continue;
        dst = static_cast<T *>(key ? p.c.k : p.c.v) + to;
        turned = key;
      } else {
        dst = p.q_out.at<T>(l, b, t) + r * p.q_out.head;
      }
      u32x4v a = lo[i], z = hi[i];
      if (turned) {
        const Vec<T> x = unpack<T>(a), y = unpack<T>(z);
        Vec<T> u, w;
        if (p.pairs) {
#pragma unroll
          for (int j = 0; j < C::vec / 2; ++j) {
            turn_pair(x.x[2 * j], x.x[2 * j + 1], turn[j], u.x[2 * j], u.x[2 * j + 1]);
            turn_pair(y.x[2 * j], y.x[2 * j + 1], turn[C::vec / 2 + j], w.x[2 * j], w.x[2 * j + 1]);
          }
        } else {
#pragma unroll
          for (int j = 0; j < C::vec; ++j) turn_pair(x.x[j], y.x[j], turn[j], u.x[j], w.x[j]);
        }
        a = turns0 ? pack<T>(u) : a;
        z = turns1 ? pack<T>(w) : z;
      }
      *reinterpret_cast<u32x4v *>(dst + e0) = a;
      *reinterpret_cast<u32x4v *>(dst + e1) = z;
    }
  };
  for (int r0 = first; r0 < rows; r0 += 2 * kAhead * step) {
    load(r0 + kAhead * step, lo_b, hi_b);
    put(r0, lo_a, hi_a);
    load(r0 + 2 * kAhead * step, lo_a, hi_a);
    put(r0 + kAhead * step, lo_b, hi_b);
  }
}

// The lengths after a run of more tokens than a workgroup's, whose rows the other kernel
// has put where their pages are good.
constexpr int kRopeLenThreads = 256;

__global__ __launch_bounds__(kRopeLenThreads) void rope_len_kernel(RopeParams p) {
  const int unit = blockIdx.x;
  const size_t cunit = p.c.unit(unit);
  bool bad;
  const int L = p.c.len[cunit], n = new_tokens(p, p.c.sequence(unit), bad);
  bool bad_page = false;
  if (L >= 0 && L <= p.c.cap && n <= p.c.cap - L && n > 0) {
    const int32_t *table = p.c.pages + cunit * static_cast<size_t>(p.c.max_pages);
#pragma unroll 4
    for (int g = (L >> p.c.page_shift) + threadIdx.x; g <= (L + n - 1) >> p.c.page_shift; g += kRopeLenThreads)
      bad_page |= static_cast<unsigned>(table[g]) >= static_cast<unsigned>(p.c.n_pages);
  }
  bad_page = __syncthreads_or(bad_page);
  if (threadIdx.x) return;
  const int code = append_code(p.c, L, n, bad_page);
  if (code) report(p.dev_err, code);
  else if (n > 0) p.c.len[cunit] = L + n;
}

template <typename T, int D, bool kAppend>
hipError_t launch_rows(const RopeParams &p, hipStream_t s) {
  const dim3 grid((p.tokens + p.block - 1) / p.block, p.batch, p.layers);
  const size_t lds = kAppend ? static_cast<size_t>(p.c.hkv) * p.block * sizeof(int64_t) : 0;
  if constexpr (kAppend) {
    if (p.tokens <= p.block) {
      hipLaunchKernelGGL((rope_kernel<T, D, true, kRopeWide, false>), grid, dim3(kRopeWide), lds, s, p);
      return hipGetLastError();
    }
  }
  if (p.far) hipLaunchKernelGGL((rope_kernel<T, D, kAppend, kRopeThreads, true>), grid, dim3(kRopeThreads), lds, s, p);
  else hipLaunchKernelGGL((rope_kernel<T, D, kAppend, kRopeThreads, false>), grid, dim3(kRopeThreads), lds, s, p);
  return hipGetLastError();
}

template <typename T, int D>
hipError_t launch_typed(const RopeParams &p, hipStream_t s) {
  if (!p.c.k) return launch_rows<T, D, false>(p, s);
  const hipError_t e = launch_rows<T, D, true>(p, s);
  if (e != hipSuccess || p.tokens <= p.block) return e;
  hipLaunchKernelGGL(rope_len_kernel, dim3(p.layers * p.batch * p.c.hkv), dim3(kRopeLenThreads), 0, s, p);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_rope(const RopeParams &p, int dtype, int head_dim, hipStream_t s) {
  if (dtype == 0) {
    if (head_dim == 64) return launch_typed<float, 64>(p, s);
    return launch_typed<float, 128>(p, s);
  }
  if (head_dim == 64) return launch_typed<bf16_t, 64>(p, s);
  return launch_typed<bf16_t, 128>(p, s);
}

}  // namespace reco
