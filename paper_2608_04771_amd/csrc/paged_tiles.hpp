// Tiles of keys as the attention kernels over a paged cache lay them out in LDS, and the
// matrix instructions' operands in them: tiles16 for few query rows, where every wave
// has tiles of its own, tiles32 for many, where a workgroup's waves share them.
#pragma once

#include "paged_device.hpp"

namespace reco {

typedef short i16x4_t __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) i16x4_t lds_i16x4_t;

namespace tiles16 {

constexpr int kTile = kPagedTile;
constexpr int kSplitWaves = 4;                        // waves of a workgroup

template <typename T, int D>
struct Cfg {
  using MF = Mfma<T>;
  static constexpr int kpl = MF::kPerLane;
  static constexpr int dq = D / 4;                  // head-dim elements per lane group for Q.K
  static constexpr int qk_steps = dq / kpl;
  static constexpr int dtiles = D / 16;
  static constexpr int pv_ops = kTile / MF::kPerOp;
  static constexpr int row_bytes = D * (int)sizeof(T);
  static constexpr int k_stride = row_bytes + 16;   // LDS pitches, free of bank conflicts
  static constexpr int v_stride = row_bytes + 8;
  static constexpr int wave_stage = kTile * k_stride;
  static constexpr int merge_pitch = D + 4;
  static constexpr int lanes_per_row = row_bytes / 16;
  static constexpr int rows_per_inst = kWave / lanes_per_row;
  static constexpr int insts = kTile / rows_per_inst;   // 1 KB loads per tile of K or V
  static constexpr int min_wgs = sizeof(T) == 4 && D == 128 ? 1 : 2;
  static constexpr int smem() {
    const int a = kSplitWaves * wave_stage, b = kSplitWaves * 16 * (2 + merge_pitch) * 4;
    return a > b ? a : b;
  }
};

template <typename T, int D>
using Rows = u32x4v[Cfg<T, D>::insts];

// V^T operand of instruction c: lane (col, grp) holds column dt * 16 + col of the
// rows of elements e = c * kpl + j, row (e / 4) * 16 + 4 * grp + e % 4.  bf16 takes
// them with two transposing LDS reads of four rows each.
template <typename T, int D>
__device__ __forceinline__ typename Mfma<T>::frag v_frag(const unsigned char *stage, int c, int grp, int dt, int col) {
  using C = Cfg<T, D>;
  typename Mfma<T>::frag a;
  if constexpr (C::kpl == 1) {
    const int row = (c >> 2) * 16 + 4 * grp + (c & 3);
    a = *reinterpret_cast<const float *>(stage + row * C::v_stride + (dt * 16 + col) * 4);
  } else {
    const int row = 32 * c + 4 * grp + col / 4;
    const int at = (dt * 16 + 4 * (col % 4)) * 2;
    const i16x4_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4_t *)(stage + row * C::v_stride + at));
    const i16x4_t hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4_t *)(stage + (row + 16) * C::v_stride + at));
    const short v[8] = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
#pragma unroll
    for (int j = 0; j < 8; ++j) a[j] = __builtin_bit_cast(__bf16, v[j]);
  }
  return a;
}

template <typename T>
__device__ __forceinline__ typename Mfma<T>::frag p_frag(const float (&pv)[8], int c) {
  if constexpr (Mfma<T>::kPerLane == 1) return pv[c];
  else return pack_frag8(pv);
}

}  // namespace tiles16

namespace tiles32 {

typedef __attribute__((__vector_size__(16 * sizeof(float)))) float f32x16_t;
typedef __attribute__((address_space(3))) unsigned int lds_u32;
typedef const __attribute__((address_space(1))) unsigned int global_u32;

constexpr int kWaves = 4;

// 32x32 fragments: lane l has 8 (bf16) or 1 (fp32) consecutive contraction elements of
// row or column l % 32, group l / 32; the result holds rows 8 (i / 4) + 4 (l / 32) + i % 4
// of column l % 32.
template <typename T>
struct Mma32;
template <>
struct Mma32<bf16_t> {
  static constexpr int kpl = 8;
  static constexpr int keys = 64;            // of a tile
  using frag = bf16x8_t;
  __device__ __forceinline__ static f32x16_t mma(frag a, frag b, f32x16_t c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
  }
  __device__ __forceinline__ static frag negated(frag a) {
    const uint4 u = __builtin_bit_cast(uint4, a);
    constexpr unsigned k = 0x80008000u;
    return __builtin_bit_cast(frag, make_uint4(u.x ^ k, u.y ^ k, u.z ^ k, u.w ^ k));
  }
};
template <>
struct Mma32<float> {
  static constexpr int kpl = 1;
  static constexpr int keys = 32;
  using frag = float;
  __device__ __forceinline__ static f32x16_t mma(frag a, frag b, f32x16_t c) {
    return __builtin_amdgcn_mfma_f32_32x32x2f32(a, b, c, 0, 0, 0);
  }
  __device__ __forceinline__ static frag negated(frag a) { return -a; }
};

template <typename T, int D, int NW = kWaves>
struct Cfg {
  using M = Mma32<T>;
  static constexpr int keys = M::keys;
  static constexpr int blocks = keys / 32;               // S^T blocks of a tile
  static constexpr int qk_steps = D / 2 / M::kpl;
  static constexpr int dtiles = D / 32;
  static constexpr int pv_steps = 16 / M::kpl;           // per block
  static constexpr int row_bytes = D * (int)sizeof(T);
  static constexpr int stage = keys * row_bytes;         // of K or V, without padding
  static constexpr int lanes_per_row = row_bytes / 16;
  static constexpr int wave_rows = kWave / lanes_per_row;   // rows a wave's load takes
  static constexpr int insts = keys * row_bytes / (NW * kWave * 16);
  static constexpr int chunks = lanes_per_row;           // 16-byte pieces of a row
  // Rows lie in LDS as they are loaded, so their pieces are permuted instead, by what
  // makes the rows that are read together fall on different banks.
  __device__ __forceinline__ static int k_swap(int row) { return chunks >= 16 ? row & 15 : (row >> 1) & 7; }
  __device__ __forceinline__ static int v_swap(int row) {
    if (sizeof(T) == 4) return ((row >> 2) & 1) << 3;
    return (chunks >= 16 ? row & 3 : (row >> 1) & 1) << 2;
  }
};

// The row of a result element within its 32.
__device__ __forceinline__ int acc_row(int i, int half) { return 8 * (i / 4) + 4 * half + (i & 3); }

// Where a lane reads operands of K rows [0, 32): step c is at this ^ (c kpl sizeof(T)).
template <typename T, int D>
__device__ __forceinline__ int k_base(int lane) {
  using C = Cfg<T, D>;
  const int col = lane & 31, half = lane >> 5;
  return col * C::row_bytes + ((half * (C::chunks / 2)) ^ C::k_swap(col)) * 16;
}
// And of V rows [0, 16): columns [32 dt, 32 dt + 32) are at this ^ (32 dt sizeof(T)).
// bf16 takes them by two transposing reads of four rows each, in which lane i of 16
// gets column i.
template <typename T, int D>
__device__ __forceinline__ int v_base(int lane) {
  using C = Cfg<T, D>;
  const int half = lane >> 5;
  if (sizeof(T) == 4) return 4 * half * C::row_bytes + ((((lane & 31) / 4) ^ C::v_swap(4 * half)) * 16) + (lane & 3) * 4;
  const int row = 4 * half + (lane & 15) / 4, c = (lane & 16) / 8 + (lane & 3) / 2;
  return row * C::row_bytes + ((c ^ C::v_swap(row)) * 16) + (lane & 1) * 8;
}
template <typename T, int D>
__device__ __forceinline__ typename Mma32<T>::frag v_frag32(const unsigned char *at) {
  if constexpr (sizeof(T) == 4) {
    return *reinterpret_cast<const float *>(at);
  } else {
    const i16x4_t a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4_t *)at);
    const i16x4_t b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4_t *)(at + 8 * Cfg<T, D>::row_bytes));
    const short v[8] = {a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
    bf16x8_t f;
#pragma unroll
    for (int j = 0; j < 8; ++j) f[j] = __builtin_bit_cast(__bf16, v[j]);
    return f;
  }
}

}  // namespace tiles32

}  // namespace reco
