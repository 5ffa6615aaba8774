// Attention of one new token of every stream over the tokens that its stream holds in a paged memory:
//   out[h] = sum_t softmax_t(scale q[h] . k[t, h / G]) v[t, h / G],   G = heads / key heads.
//
// One pass over keys and values, with a running maximum and sum.  Every key and value is read once for the G query
// heads that share it: 2 G operations a byte in bf16, so memory bounds it.
#include "kernels.h"
#include "stream_memory.h"

namespace cfdetr {

namespace {

constexpr int kThreads = 256, kWaves = kThreads / 64;

// 16 bytes of a row as numbers, and their products with a query's.
template <typename T>
struct Piece;
template <>
struct Piece<bf16_t> {
  static constexpr int kN = 8;
  static __device__ __forceinline__ void get(const uint4& v, float (&x)[kN]) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[2 * i] = __uint_as_float(w[i] << 16);
      x[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
    }
  }
  static __device__ __forceinline__ uint4 put(const float (&x)[kN]) {
    return make_uint4(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(x[4], x[5]), pack_bf16x2(x[6], x[7]));
  }
};
template <>
struct Piece<float> {
  static constexpr int kN = 4;
  static __device__ __forceinline__ void get(const uint4& v, float (&x)[kN]) {
    x[0] = __uint_as_float(v.x);
    x[1] = __uint_as_float(v.y);
    x[2] = __uint_as_float(v.z);
    x[3] = __uint_as_float(v.w);
  }
  static __device__ __forceinline__ uint4 put(const float (&x)[kN]) {
    return make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3]));
  }
};

// A workgroup has a stream, a key head and up to GP of its query heads.  LPH lanes hold a row's 16-byte pieces, so that a
// wavefront takes 64 / LPH tokens at a time, each group of lanes with a running maximum, sum and row of its own; the groups'
// results are brought to one maximum and added at the end.
template <typename T, int DH, int GP>
__global__ __launch_bounds__(kThreads) void memory_attention_kernel(MemoryAttentionArgs a) {
  constexpr int N = Piece<T>::kN, LPH = DH / N, TPW = 64 / LPH;
  __shared__ float s_m[kWaves][TPW][GP], s_l[kWaves][TPW][GP];
  __shared__ float s_o[kWaves][TPW][GP][DH];
  __shared__ int s_bad;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int b = blockIdx.x, kh = blockIdx.y, G = a.heads / a.kv_heads;
  if (tid == 0) s_bad = 0;
  __syncthreads();
  for (int i = tid; i < a.B; i += kThreads) {
    const int2 span = a.span[i];
    if (span_is_bad(span.x, span.y, a.page_bits, a.cols)) s_bad = 1;
  }
  __syncthreads();
  if (s_bad) {
    if (tid == 0) *a.err_flag = 1;
    return;
  }
  const int first = a.span[b].x, held = a.span[b].y;
  const int group = lane / LPH, c = lane % LPH;
  float q[GP][N], acc[GP][N], m[GP], l[GP];
  int head[GP];
#pragma unroll
  for (int g = 0; g < GP; ++g) {
    head[g] = kh * G + min((int)blockIdx.z * GP + g, G - 1);   // (a group's last heads again, where there are fewer)
    Piece<T>::get(*reinterpret_cast<const uint4*>(static_cast<const T*>(a.q) + (size_t)b * a.q_ld + head[g] * DH + c * N), q[g]);
    m[g] = -INFINITY;
    l[g] = 0.f;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      q[g][i] *= a.scale2;
      acc[g][i] = 0.f;
    }
  }
  const int32_t* const table = a.table + (size_t)b * a.cols;
  for (int t0 = wave * TPW; t0 < held; t0 += kWaves * TPW) {
    const int t = t0 + group;
    bool open = t < held;
    size_t slot = 0;
    if (open) {
      const int p = first + t, id = table[ring_column(p >> a.page_bits, a.cols)];
      if ((unsigned)id >= (unsigned)a.n_pages) {
        *a.err_flag = 1;
        open = false;
      } else {
        slot = ((size_t)id << a.page_bits) + (p & ((1 << a.page_bits) - 1));
        if (a.mask && a.mask[slot] == 0) open = false;
      }
    }
    uint4 kp = make_uint4(0, 0, 0, 0), vp = kp;
    if (open) {
      kp = *reinterpret_cast<const uint4*>(static_cast<const T*>(a.k) + slot * a.k_ld + kh * DH + c * N);
      vp = *reinterpret_cast<const uint4*>(static_cast<const T*>(a.v) + slot * a.v_ld + kh * DH + c * N);
    }
    float k[N], v[N];
    Piece<T>::get(kp, k);
    Piece<T>::get(vp, v);
#pragma unroll
    for (int g = 0; g < GP; ++g) {
      float s = 0.f;
#pragma unroll
      for (int i = 0; i < N; ++i) s = fmaf(q[g][i], k[i], s);
#pragma unroll
      for (int o = 1; o < LPH; o <<= 1) s += __shfl_xor(s, o);
      if (!open) s = -INFINITY;
      const float top = fmaxf(m[g], s), ref = top == -INFINITY ? 0.f : top;
      const float keep = __builtin_amdgcn_exp2f(m[g] - ref), w = __builtin_amdgcn_exp2f(s - ref);
      m[g] = top;
      l[g] = fmaf(l[g], keep, w);
#pragma unroll
      for (int i = 0; i < N; ++i) acc[g][i] = fmaf(acc[g][i], keep, w * v[i]);
    }
  }
#pragma unroll
  for (int g = 0; g < GP; ++g) {
    if (c == 0) {
      s_m[wave][group][g] = m[g];
      s_l[wave][group][g] = l[g];
    }
#pragma unroll
    for (int i = 0; i < N; ++i) s_o[wave][group][g][c * N + i] = acc[g][i];
  }
  __syncthreads();
  for (int i = tid; i < GP * LPH; i += kThreads) {
    const int g = i / LPH, cc = i % LPH;
    if ((int)blockIdx.z * GP + g >= G) continue;
    float top = -INFINITY, sum = 0.f, row[N] = {};
    for (int w = 0; w < kWaves; ++w)
      for (int j = 0; j < TPW; ++j) top = fmaxf(top, s_m[w][j][g]);
    const float ref = top == -INFINITY ? 0.f : top;
    for (int w = 0; w < kWaves; ++w)
      for (int j = 0; j < TPW; ++j) {
        const float f = __builtin_amdgcn_exp2f(s_m[w][j][g] - ref);
        sum = fmaf(s_l[w][j][g], f, sum);
#pragma unroll
        for (int e = 0; e < N; ++e) row[e] = fmaf(s_o[w][j][g][cc * N + e], f, row[e]);
      }
    const float inv = sum != 0.f ? 1.0f / sum : 0.f;
#pragma unroll
    for (int e = 0; e < N; ++e) row[e] *= inv;
    *reinterpret_cast<uint4*>(static_cast<T*>(a.out) + (size_t)b * a.out_ld + (kh * G + blockIdx.z * GP + g) * DH + cc * N) = Piece<T>::put(row);
  }
}

template <typename T, int DH>
hipError_t launch(const MemoryAttentionArgs& a, hipStream_t s) {
  const int G = a.heads / a.kv_heads;
  if (G == 1)
    hipLaunchKernelGGL((memory_attention_kernel<T, DH, 1>), dim3(a.B, a.kv_heads, 1), dim3(kThreads), 0, s, a);
  else
    hipLaunchKernelGGL((memory_attention_kernel<T, DH, 2>), dim3(a.B, a.kv_heads, (G + 1) / 2), dim3(kThreads), 0, s, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_memory_attention(const MemoryAttentionArgs& a, int d_head, bool use_bf16, hipStream_t s) {
  if (d_head == 64) return use_bf16 ? launch<bf16_t, 64>(a, s) : launch<float, 64>(a, s);
  if (d_head == 32) return use_bf16 ? launch<bf16_t, 32>(a, s) : launch<float, 32>(a, s);
  return hipErrorInvalidValue;
}

}  // namespace cfdetr
