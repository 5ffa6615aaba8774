// Rotary positions of queries and keys (operator of a differential encoder layer).
//
// Pair i of a head, i < n = rot_dim / 2, is turned by the angle pos[axis(i)] freq[i]:
//   (a, b) -> (a cos - b sin, a sin + b cos),
// (a, b) being features (i, i + n) or (2i, 2i + 1) of the head; the features from rot_dim on stay.
// Queries are multiplied by q_scale before they are rounded, so that a softmax scale costs neither
// a second rounding nor an operation in the attention.
//
// Bound by memory: every feature is read and written once.  The angles are those of a row, the same for
// all its heads and for queries and keys, so a workgroup takes some rows, works their sines and cosines
// out once into LDS, and its threads, whose features are on their way meanwhile, turn them.
// A position times a frequency is thousands of turns for a far token: the product and its whole
// turns are taken in 64 bits (32 bits lose 0.06 radians at 10^6), what is left of a turn goes through
// the 32-bit functions of half turns.
#include <algorithm>

#include "kernels.h"

namespace cfdetr {

namespace {

constexpr int kThreads = 256;

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

// Units of a row: those of its query heads, then those of its key heads.
template <typename T, bool INTERLEAVED>
__global__ __launch_bounds__(kThreads) void rotary_kernel(
    const T* q, const T* k, const float* __restrict__ pos, const double* __restrict__ freq, T* q_out,
    T* k_out, int q_ld, int k_ld, int qo_ld, int ko_ld, int m_host, const int32_t* __restrict__ m_ptr, float q_scale,
    int rows_wg, int units_row, int units_q, int d_head, int n, int n_axes) {
  constexpr int RUN = Runs<T>::kRun;
  typedef typename Runs<T>::Piece Piece;
  extern __shared__ float2 turns[];   // [rows_wg][n] cosine and sine
  const int M = m_ptr ? *m_ptr : m_host;
  const int row0 = blockIdx.x * rows_wg;
  const int rows = min(rows_wg, M - row0);
  if (rows <= 0) return;
  const int tid = threadIdx.x;
  const int per_head = d_head / (2 * RUN);
  Runs<T> f;
  const int r = tid / units_row, u = tid - r * units_row;
  const bool mine = r < rows, is_q = u < units_q;
  const int head_run = is_q ? u : u - units_q;
  const int head = head_run / per_head, j = RUN * (head_run - head * per_head);
  const bool rotated = j < n;
  const int first = head * d_head + (rotated ? j : n + j);   // where the first run starts in the row
  const int apart = rotated ? n : d_head / 2 - n;            // and the second behind it
  if (mine) {
    const T* const src = (is_q ? q + (size_t)(row0 + r) * q_ld : k + (size_t)(row0 + r) * k_ld) + first;
    f.v[0] = *reinterpret_cast<const Piece*>(src);
    f.v[1] = *reinterpret_cast<const Piece*>(src + apart);
  }
  for (int a = tid; a < rows * n; a += kThreads) {
    const int row = a / n, i = a - row * n;
    const int axis = 2 * i >= n ? n_axes - 1 : 0;
    double t = (double)pos[(size_t)(row0 + row) * n_axes + axis] * freq[i] * 0.15915494309189533577;
    t -= rint(t);
    float s, c;
    sincospif(2.0f * (float)t, &s, &c);
    turns[a] = make_float2(c, s);
  }
  __syncthreads();
  if (!mine) return;
  float x[2][RUN];
  f.get(x);
  if (rotated) {
    const float2* const t0 = turns + r * n + (INTERLEAVED ? j / 2 : j);
#pragma unroll
    for (int p = 0; p < RUN; ++p) {
      // pair p of the unit: the runs' elements p, or two neighbours, the second half of the pairs in the second run
      const int h = 2 * p / RUN, e = 2 * p % RUN;
      float& a = INTERLEAVED ? x[h][e] : x[0][p];
      float& b = INTERLEAVED ? x[h][e + 1] : x[1][p];
      const float2 t = t0[INTERLEAVED ? (h ? n / 2 : 0) + e / 2 : p];
      const float ra = fmaf(a, t.x, -(b * t.y)), rb = fmaf(a, t.y, b * t.x);
      a = ra;
      b = rb;
    }
  }
  if (is_q) {
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int p = 0; p < RUN; ++p) x[h][p] *= q_scale;
  }
  f.put(x);
  T* const dst = (is_q ? q_out + (size_t)(row0 + r) * qo_ld : k_out + (size_t)(row0 + r) * ko_ld) + first;
  *reinterpret_cast<Piece*>(dst) = f.v[0];
  *reinterpret_cast<Piece*>(dst + apart) = f.v[1];
}

template <typename T, bool INTERLEAVED>
hipError_t launch(const RotaryArgs& a, hipStream_t s) {
  const int heads = a.k ? 2 * a.heads : a.heads;
  const int units_q = a.heads * a.d_head / (2 * Runs<T>::kRun), units_row = heads * a.d_head / (2 * Runs<T>::kRun);
  const int rows_wg = std::max(1, kThreads / units_row), n = a.rot_dim / 2;
  const int64_t grid = ((int64_t)a.m_capacity + rows_wg - 1) / rows_wg;
  if (grid * kThreads > 0xFFFFFFFFLL) return hipErrorInvalidValue;   // more threads than a launch has
  hipLaunchKernelGGL((rotary_kernel<T, INTERLEAVED>), dim3((unsigned)grid), dim3(kThreads), (size_t)rows_wg * n * sizeof(float2), s,
                     static_cast<const T*>(a.q), static_cast<const T*>(a.k), a.pos, a.freq, static_cast<T*>(a.q_out),
                     static_cast<T*>(a.k_out), a.q_ld, a.k_ld, a.qo_ld, a.ko_ld, a.m_capacity, a.m_ptr, a.q_scale, rows_wg,
                     units_row, units_q, a.d_head, n, a.n_axes);
  return hipGetLastError();
}

// Positions of a run's rows: the centres of their cells in units of the finest level's cells, (row, column).
__global__ __launch_bounds__(256) void cell_positions_kernel(const int32_t* __restrict__ first, int n_first,
                                                             const int32_t* __restrict__ second, int finest,
                                                             const int32_t* __restrict__ m_ptr, int m_host, float2* __restrict__ pos) {
  const int M = m_ptr ? *m_ptr : m_host;
  const int m = blockIdx.x * 256 + threadIdx.x;
  if (m >= M) return;
  const int32_t t = m < n_first ? first[m] : second[m - n_first];
  const float cells = (float)(1 << (finest - tok_level(t)));
  pos[m] = make_float2(((float)tok_row(t) + 0.5f) * cells, ((float)tok_col(t) + 0.5f) * cells);
}

}  // namespace

hipError_t launch_rotary(const RotaryArgs& a, bool use_bf16, hipStream_t s) {
  if (a.rot_dim % 16 != 0 || a.d_head % 16 != 0) return hipErrorInvalidValue;   // whole runs in either half
  if (use_bf16) return a.interleaved ? launch<bf16_t, true>(a, s) : launch<bf16_t, false>(a, s);
  return a.interleaved ? launch<float, true>(a, s) : launch<float, false>(a, s);
}

hipError_t launch_cell_positions(const int32_t* first, int n_first, const int32_t* second, int finest, const int32_t* m_ptr,
                                 int m_capacity, float* pos, hipStream_t s) {
  hipLaunchKernelGGL(cell_positions_kernel, dim3((m_capacity + 255) / 256), dim3(256), 0, s, first, n_first, second, finest, m_ptr,
                     m_capacity, reinterpret_cast<float2*>(pos));
  return hipGetLastError();
}

}  // namespace cfdetr
