// What the kernels that turn queries and keys share (rotary.hip, memory_rows.hip).
#pragma once
#include "kernels.h"

namespace cfdetr {

namespace {

// A unit is two runs of 16 bytes of one head, as far apart as what they are runs of allows: run j of either half of the
// rotated features, or of either half of those behind.  Neighbouring threads then have neighbouring
// runs, and with pairs half a head apart a unit holds whole pairs.  One unit a thread: with two in turn
// 20,000 rows of 2 x 768 columns take 26.3 us and not 24.8, 51,200 of 2 x 384 34.5 and not 31.3.
template <typename T>
struct Runs;
template <>
struct Runs<bf16_t> {
  static constexpr int kRun = 8;
  typedef uint4 Piece;
  Piece v[2];
  __device__ __forceinline__ void get(float (&x)[2][kRun]) const {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const uint32_t w[4] = {v[h].x, v[h].y, v[h].z, v[h].w};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        x[h][2 * i] = __uint_as_float(w[i] << 16);
        x[h][2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
      }
    }
  }
  __device__ __forceinline__ void put(const float (&x)[2][kRun]) {
#pragma unroll
    for (int h = 0; h < 2; ++h)
      v[h] = make_uint4(pack_bf16x2(x[h][0], x[h][1]), pack_bf16x2(x[h][2], x[h][3]), pack_bf16x2(x[h][4], x[h][5]), pack_bf16x2(x[h][6], x[h][7]));
  }
};
template <>
struct Runs<float> {
  static constexpr int kRun = 4;
  typedef float4 Piece;
  Piece v[2];
  __device__ __forceinline__ void get(float (&x)[2][kRun]) const {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      x[h][0] = v[h].x;
      x[h][1] = v[h].y;
      x[h][2] = v[h].z;
      x[h][3] = v[h].w;
    }
  }
  __device__ __forceinline__ void put(const float (&x)[2][kRun]) {
#pragma unroll
    for (int h = 0; h < 2; ++h) v[h] = make_float4(x[h][0], x[h][1], x[h][2], x[h][3]);
  }
};

}  // namespace

}  // namespace cfdetr
