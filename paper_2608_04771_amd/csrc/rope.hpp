// Launch interface of the kernel that rotates rows by their positions and appends
// them to a paged cache (rope_append.hip).  Not part of the public ABI.
#pragma once

#include "paged.hpp"

namespace reco {

// Rows of head_dim elements; strides in elements.
struct RowsOf {
  void *data;
  int64_t layer, seq, head, token;

  template <typename T>
  __host__ __device__ T *at(int64_t l, int64_t b, int64_t t) const {
    return static_cast<T *>(data) + l * layer + b * seq + t * token;
  }
};

constexpr int kRopeThreads = 256;
constexpr int kRopeWide = 1024;      // of a workgroup that has a sequence's whole run
constexpr int kRopeMaxAxes = 4;      // two bits a pair
constexpr int kRopeBlock = 4;        // tokens of a workgroup
constexpr int kRopeMaxBlock = 8;     // of one that has a whole run

struct RopeParams {
  const float *freq;      // [rot / 2]
  const int32_t *pos;     // [axes][batch][tokens]
  uint64_t axis[2];       // of pair i: bits 2 (i % 32) of word i / 32
  int rot;                // rotated elements of a row, 0: none
  bool pairs;             // pair i is (2 i, 2 i + 1), else (i, i + rot / 2)

  RowsOf q, q_out;        // heads rows a token; none where heads is 0
  RowsOf k, v;            // c.hkv rows a token, where c.k is set
  PagedCache c;           // k null: nothing to append
  const int32_t *n_new;   // nullable [batch]
  int32_t *dev_err;
  int heads, layers, batch, tokens;
  int block;              // tokens of a workgroup, a power of two
  bool far;               // the rows are not in a cache
};

// Sets block and far; the rows' numbers are set.
void rope_plan(RopeParams &p, int row_bytes);
hipError_t launch_rope(const RopeParams &p, int dtype, int head_dim, hipStream_t s);

}  // namespace reco
