// The step between two blocks of a differential encoder layer, in one pass over the rows:
//   y = post(block);  x' = res_scale x + gate * y;  normed = pre(x')
// post and pre: LayerNorm, root-mean-square norm, or none; gate: one vector, one for every frame, or none.
//
// Bound by memory: an element of x and of the block is read once, one of x' and of the normed row
// written once; the row stays in registers between its norms.  Sums, means and variances are 32-bit, the
// variance that of the centred values.  A row belongs to 16, 32 or 64 lanes, the most that its quads
// of columns fill, so that narrow rows leave no lanes idle.
#include <algorithm>

#include "kernels.h"

namespace cfdetr {

namespace {

constexpr int kThreads = 256;

// Sum over the LANES lanes of a row, delivered to all of them (the steps of wave_sum that stay inside).
template <int LANES>
__device__ __forceinline__ float row_sum(float v) {
  if constexpr (LANES == 64) return wave_sum(v);
  typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
  if constexpr (LANES == 32) {
    const u32x2 p = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = __uint_as_float(p[0]) + __uint_as_float(p[1]);
  }
  auto from = [&](int old, auto ctrl, auto banks) {
    return __builtin_amdgcn_update_dpp(old, __float_as_int(v), decltype(ctrl)::value, 0xF, decltype(banks)::value, false);
  };
  const auto all = std::integral_constant<int, 0xF>{};
  v += __int_as_float(from(0, std::integral_constant<int, 0x128>{}, all));   // row_ror:8
  v += __int_as_float(from(from(0, std::integral_constant<int, 0x104>{}, std::integral_constant<int, 0x5>{}),
                           std::integral_constant<int, 0x114>{}, std::integral_constant<int, 0xA>{}));
  v += __int_as_float(from(0, std::integral_constant<int, 0x4E>{}, all));    // quad_perm [2, 3, 0, 1]
  v += __int_as_float(from(0, std::integral_constant<int, 0xB1>{}, all));    // quad_perm [1, 0, 3, 2]
  return v;
}

__device__ __forceinline__ float4 load_quad(const float* p) { return *reinterpret_cast<const float4*>(p); }
__device__ __forceinline__ float4 load_quad(const bf16_t* p) {
  const uint2 w = *reinterpret_cast<const uint2*>(p);
  return make_float4(__uint_as_float(w.x << 16), __uint_as_float(w.x & 0xFFFF0000u), __uint_as_float(w.y << 16),
                     __uint_as_float(w.y & 0xFFFF0000u));
}
// fp32 rows go past the caches' replacement: the rows are next read behind two matrix products (64,000 rows of 384 columns 65 ->
// 61 us, 20,000 of 768 42.4 -> 40.3; with such loads of x as well the smaller ones, which the caches hold, lose a third).
__device__ __forceinline__ void store_quad(float* p, const float4& v) {
  const f32x4 w = {v.x, v.y, v.z, v.w};
  __builtin_nontemporal_store(w, reinterpret_cast<f32x4*>(p));
}
__device__ __forceinline__ void store_quad(bf16_t* p, const float4& v) {
  *reinterpret_cast<uint2*>(p) = make_uint2(pack_bf16x2(v.x, v.y), pack_bf16x2(v.z, v.w));
}

// A norm of the row that LANES lanes hold in quads (quad lane + LANES j in v[j], zeros beyond `quads`), in place.
template <int LANES, int NQ>
__device__ __forceinline__ void norm_row(float4 (&v)[NQ], NormKind kind, const float4 (&g)[NQ], const float4 (&b)[NQ], int lane,
                                         int quads, float inv_d, float eps) {
  float mean = 0.f;
  if (kind == NormKind::kLayer) {
    float sum = 0.f;
#pragma unroll
    for (int j = 0; j < NQ; ++j) sum += (v[j].x + v[j].y) + (v[j].z + v[j].w);
    mean = row_sum<LANES>(sum) * inv_d;
  }
  float sq = 0.f;
#pragma unroll
  for (int j = 0; j < NQ; ++j)
    if (lane + LANES * j < quads) {
      v[j] = make_float4(v[j].x - mean, v[j].y - mean, v[j].z - mean, v[j].w - mean);
      sq += fmaf(v[j].x, v[j].x, v[j].y * v[j].y) + fmaf(v[j].z, v[j].z, v[j].w * v[j].w);
    }
  const float r = rsqrtf(row_sum<LANES>(sq) * inv_d + eps);
  if (kind == NormKind::kLayer) {
#pragma unroll
    for (int j = 0; j < NQ; ++j)
      v[j] = make_float4(fmaf(v[j].x * r, g[j].x, b[j].x), fmaf(v[j].y * r, g[j].y, b[j].y), fmaf(v[j].z * r, g[j].z, b[j].z),
                         fmaf(v[j].w * r, g[j].w, b[j].w));
  } else {
#pragma unroll
    for (int j = 0; j < NQ; ++j) v[j] = make_float4(v[j].x * r * g[j].x, v[j].y * r * g[j].y, v[j].z * r * g[j].z, v[j].w * r * g[j].w);
  }
}

template <typename TBlock, typename TOut, int LANES, int NQ>
__global__ __launch_bounds__(kThreads) void norm_residual_kernel(NormResidualArgs a, int m_host) {
  constexpr int kRows = 64 / LANES;   // rows of a wavefront
  const int lane = threadIdx.x & (LANES - 1);
  const int d = a.d, quads = d >> 2;
  const float inv_d = 1.0f / (float)d;
  int M = a.m_ptr ? *a.m_ptr : m_host;
  if (a.cu != nullptr) {
    // a gate for every frame: offsets that are none are refused, and rows behind the last frame are left alone
    const int l = threadIdx.x & 63;
    const int lo = l < a.B ? a.cu[l] : 0, hi = l < a.B ? a.cu[l + 1] : 0;
    if (__any(l < a.B && (hi < lo || lo < 0 || hi > M || (l == 0 && lo != 0)))) {
      if (blockIdx.x == 0 && threadIdx.x == 0) *a.err_flag = 1;
      return;
    }
    M = a.cu[a.B];
  }
  int row = (blockIdx.x * (kThreads / 64) + (threadIdx.x >> 6)) * kRows + (threadIdx.x & 63) / LANES;
  const int step = gridDim.x * (kThreads / 64) * kRows;
  const TBlock* const block = static_cast<const TBlock*>(a.block);
  float4 post_g[NQ], post_b[NQ], gate[NQ], pre_g[NQ], pre_b[NQ];
  auto vec = [&](float4(&to)[NQ], const float* from, float value) {
#pragma unroll
    for (int j = 0; j < NQ; ++j) {
      const int i = lane + LANES * j;
      to[j] = from != nullptr && i < quads ? load_quad(from + 4 * i) : make_float4(value, value, value, value);
    }
  };
  if (row >= M) return;
  float4 x[NQ], y[NQ], xn[NQ], yn[NQ];
  auto rows = [&](float4(&xs)[NQ], float4(&ys)[NQ], int m) {
#pragma unroll
    for (int j = 0; j < NQ; ++j) {
      const int i = lane + LANES * j;
      xs[j] = ys[j] = make_float4(0.f, 0.f, 0.f, 0.f);
      if (i < quads) {
        xs[j] = load_quad(a.x + (size_t)m * d + 4 * i);
        ys[j] = load_quad(block + (size_t)m * d + 4 * i);
      }
    }
  };
  rows(x, y, row);
  vec(post_g, a.post_g, 1.f);
  vec(post_b, a.post_b, 0.f);
  vec(pre_g, a.pre_g, 1.f);
  vec(pre_b, a.pre_b, 0.f);
  int frame = -1;
  if (a.cu == nullptr) vec(gate, a.gate, 1.f);
  for (;;) {
    const int behind = row + step;
    if (behind < M) rows(xn, yn, behind);
    if (a.cu != nullptr) {
      const int f = frame_of_token(a.cu, a.B, row);
      if (f != frame) {
        frame = f;
        vec(gate, a.gate + (size_t)f * d, 1.f);
      }
    }
    if (a.post != NormKind::kNone) norm_row<LANES, NQ>(y, a.post, post_g, post_b, lane, quads, inv_d, a.eps);
#pragma unroll
    for (int j = 0; j < NQ; ++j) {
      const int i = lane + LANES * j;
      x[j] = make_float4(fmaf(a.res_scale, x[j].x, gate[j].x * y[j].x), fmaf(a.res_scale, x[j].y, gate[j].y * y[j].y),
                         fmaf(a.res_scale, x[j].z, gate[j].z * y[j].z), fmaf(a.res_scale, x[j].w, gate[j].w * y[j].w));
      if (i < quads) store_quad(a.x_out + (size_t)row * d + 4 * i, x[j]);
      else x[j] = make_float4(0.f, 0.f, 0.f, 0.f);
    }
    if (a.pre != NormKind::kNone) {
      norm_row<LANES, NQ>(x, a.pre, pre_g, pre_b, lane, quads, inv_d, a.eps);
      TOut* const to = a.normed2 != nullptr && row >= a.split_row ? static_cast<TOut*>(a.normed2) + (size_t)(row - a.split_row) * d
                                                                  : static_cast<TOut*>(a.normed) + (size_t)row * d;
#pragma unroll
      for (int j = 0; j < NQ; ++j) {
        const int i = lane + LANES * j;
        if (i < quads) store_quad(to + 4 * i, x[j]);
      }
    }
    if (behind >= M) return;
    row = behind;
#pragma unroll
    for (int j = 0; j < NQ; ++j) {
      x[j] = xn[j];
      y[j] = yn[j];
    }
  }
}

constexpr int kRowGroups = 8;

template <typename TBlock, typename TOut, int LANES, int NQ>
void go(const NormResidualArgs& a, int m_capacity, hipStream_t s) {
  const int rows_wg = kThreads / LANES;
  const int grid = std::min((m_capacity + rows_wg - 1) / rows_wg, kRowGroups * cu_count());
  hipLaunchKernelGGL((norm_residual_kernel<TBlock, TOut, LANES, NQ>), dim3(grid), dim3(kThreads), 0, s, a, m_capacity);
}

// Lanes of a row by its quads of columns (a multiple of 16, up to 256).
template <typename TBlock, typename TOut>
hipError_t by_width(const NormResidualArgs& a, int m_capacity, hipStream_t s) {
  const int quads = a.d / 4;
  if (quads % 16 != 0 || quads > 256 || quads < 16) return hipErrorInvalidValue;
  if (quads == 16) go<TBlock, TOut, 16, 1>(a, m_capacity, s);
  else if (quads == 32) go<TBlock, TOut, 32, 1>(a, m_capacity, s);
  else if (quads == 48) go<TBlock, TOut, 16, 3>(a, m_capacity, s);
  else if (quads == 64) go<TBlock, TOut, 64, 1>(a, m_capacity, s);
  else if (quads <= 96) go<TBlock, TOut, 32, 3>(a, m_capacity, s);
  else if (quads <= 128) go<TBlock, TOut, 64, 2>(a, m_capacity, s);
  else if (quads <= 192) go<TBlock, TOut, 64, 3>(a, m_capacity, s);
  else go<TBlock, TOut, 64, 4>(a, m_capacity, s);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_norm_residual(const NormResidualArgs& a, bool block_is_bf16, bool normed_is_bf16, int m_capacity, hipStream_t s) {
  if (block_is_bf16) return normed_is_bf16 ? by_width<bf16_t, bf16_t>(a, m_capacity, s) : by_width<bf16_t, float>(a, m_capacity, s);
  return normed_is_bf16 ? hipErrorInvalidValue : by_width<float, float>(a, m_capacity, s);
}

}  // namespace cfdetr
