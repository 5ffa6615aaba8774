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
constexpr int kUnit = 16;   // features of one thread and step: 8 pairs

template <typename T>
struct Features;
template <>
struct Features<bf16_t> {   // 16 features as two runs of 8
  uint4 lo, hi;
  __device__ __forceinline__ void load(const bf16_t* a, const bf16_t* b) {
    lo = *reinterpret_cast<const uint4*>(a);
    hi = *reinterpret_cast<const uint4*>(b);
  }
  __device__ __forceinline__ void store(bf16_t* a, bf16_t* b) const {
    *reinterpret_cast<uint4*>(a) = lo;
    *reinterpret_cast<uint4*>(b) = hi;
  }
  __device__ __forceinline__ void get(float (&x)[kUnit]) const {
    const uint32_t w[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      x[2 * i] = __uint_as_float(w[i] << 16);
      x[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
    }
  }
  __device__ __forceinline__ void put(const float (&x)[kUnit]) {
    lo = make_uint4(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(x[4], x[5]), pack_bf16x2(x[6], x[7]));
    hi = make_uint4(pack_bf16x2(x[8], x[9]), pack_bf16x2(x[10], x[11]), pack_bf16x2(x[12], x[13]), pack_bf16x2(x[14], x[15]));
  }
};
template <>
struct Features<float> {
  float4 v[4];
  __device__ __forceinline__ void load(const float* a, const float* b) {
    v[0] = *reinterpret_cast<const float4*>(a);
    v[1] = *reinterpret_cast<const float4*>(a + 4);
    v[2] = *reinterpret_cast<const float4*>(b);
    v[3] = *reinterpret_cast<const float4*>(b + 4);
  }
  __device__ __forceinline__ void store(float* a, float* b) const {
    *reinterpret_cast<float4*>(a) = v[0];
    *reinterpret_cast<float4*>(a + 4) = v[1];
    *reinterpret_cast<float4*>(b) = v[2];
    *reinterpret_cast<float4*>(b + 4) = v[3];
  }
  __device__ __forceinline__ void get(float (&x)[kUnit]) const {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[4 * i] = v[i].x;
      x[4 * i + 1] = v[i].y;
      x[4 * i + 2] = v[i].z;
      x[4 * i + 3] = v[i].w;
    }
  }
  __device__ __forceinline__ void put(const float (&x)[kUnit]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = make_float4(x[4 * i], x[4 * i + 1], x[4 * i + 2], x[4 * i + 3]);
  }
};

// A unit is 8 pairs of one head (its 16 features), or 16 features behind the rotated ones.
// Half layout: the runs of 8 start at 8u and n + 8u; otherwise the 16 features are consecutive.
// Units of a row: those of its query heads, then those of its key heads.
template <typename T, bool INTERLEAVED, int U>
__global__ __launch_bounds__(kThreads) void rotary_kernel(
    const T* q, const T* k, const float* __restrict__ pos, const double* __restrict__ freq, T* q_out,
    T* k_out, int q_ld, int k_ld, int qo_ld, int ko_ld, int m_host, const int32_t* __restrict__ m_ptr, float q_scale,
    int rows_wg, int units_row, int units_q, int d_head, int n, int n_axes) {
  extern __shared__ float2 turns[];   // [rows_wg][n] cosine and sine
  const int M = m_ptr ? *m_ptr : m_host;
  const int row0 = blockIdx.x * rows_wg;
  const int rows = min(rows_wg, M - row0);
  if (rows <= 0) return;
  const int tid = threadIdx.x;
  const int per_head = d_head / kUnit;
  Features<T> f[U];
  const T* src[U];
  int first[U], second[U], at[U];   // run starts within the row; where its angles are, -1: none
  bool is_q[U];
  int r_of[U];
#pragma unroll
  for (int i = 0; i < U; ++i) {
    const int unit = tid + kThreads * i;
    const int r = unit / units_row;
    r_of[i] = r;
    if (r >= rows) continue;
    int u = unit - r * units_row;
    is_q[i] = u < units_q;
    if (!is_q[i]) u -= units_q;
    const int head = u / per_head, j = u - head * per_head;
    const bool rotated = 8 * j < n;
    at[i] = rotated ? r * n + 8 * j : -1;
    if (INTERLEAVED || !rotated) {
      first[i] = head * d_head + kUnit * j;
      second[i] = first[i] + 8;
    } else {
      first[i] = head * d_head + 8 * j;
      second[i] = first[i] + n;
    }
    src[i] = is_q[i] ? q + (size_t)(row0 + r) * q_ld : k + (size_t)(row0 + r) * k_ld;
    f[i].load(src[i] + first[i], src[i] + second[i]);
  }
  for (int a = tid; a < rows * n; a += kThreads) {
    const int r = a / n, i = a - r * n;
    const int axis = 2 * i >= n ? n_axes - 1 : 0;
    double t = (double)pos[(size_t)(row0 + r) * n_axes + axis] * freq[i] * 0.15915494309189533577;
    t -= rint(t);
    float s, c;
    sincospif(2.0f * (float)t, &s, &c);
    turns[a] = make_float2(c, s);
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < U; ++i) {
    if (r_of[i] >= rows) continue;
    float x[kUnit];
    f[i].get(x);
    if (at[i] >= 0) {
#pragma unroll
      for (int p = 0; p < 8; ++p) {
        const float2 t = turns[at[i] + p];
        float& a = x[INTERLEAVED ? 2 * p : p];
        float& b = x[INTERLEAVED ? 2 * p + 1 : p + 8];
        const float ra = fmaf(a, t.x, -(b * t.y)), rb = fmaf(a, t.y, b * t.x);
        a = ra;
        b = rb;
      }
    }
    if (is_q[i]) {
#pragma unroll
      for (int p = 0; p < kUnit; ++p) x[p] *= q_scale;
    }
    f[i].put(x);
    T* const dst = is_q[i] ? q_out + (size_t)(row0 + r_of[i]) * qo_ld : k_out + (size_t)(row0 + r_of[i]) * ko_ld;
    f[i].store(dst + first[i], dst + second[i]);
  }
}

template <typename T, bool INTERLEAVED, int U>
hipError_t launch(const RotaryArgs& a, hipStream_t s) {
  const int heads = a.k ? 2 * a.heads : a.heads;
  const int units_q = a.heads * a.d_head / kUnit, units_row = heads * a.d_head / kUnit;
  const int rows_wg = std::max(1, kThreads * U / units_row), n = a.rot_dim / 2;
  const int grid = (a.m_capacity + rows_wg - 1) / rows_wg;
  hipLaunchKernelGGL((rotary_kernel<T, INTERLEAVED, U>), dim3(grid), dim3(kThreads), (size_t)rows_wg * n * sizeof(float2), s,
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
  if (a.rot_dim % kUnit != 0 || a.d_head % kUnit != 0) return hipErrorInvalidValue;
  if (use_bf16) return a.interleaved ? launch<bf16_t, true, 2>(a, s) : launch<bf16_t, false, 2>(a, s);
  return a.interleaved ? launch<float, true, 2>(a, s) : launch<float, false, 2>(a, s);
}

hipError_t launch_cell_positions(const int32_t* first, int n_first, const int32_t* second, int finest, const int32_t* m_ptr,
                                 int m_capacity, float* pos, hipStream_t s) {
  hipLaunchKernelGGL(cell_positions_kernel, dim3((m_capacity + 255) / 256), dim3(256), 0, s, first, n_first, second, finest, m_ptr,
                     m_capacity, reinterpret_cast<float2*>(pos));
  return hipGetLastError();
}

}  // namespace cfdetr
