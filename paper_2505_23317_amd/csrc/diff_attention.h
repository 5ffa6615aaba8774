// What the kernels of the differential attention share (diff_attention.hip, diff_tiles.hip).
#pragma once
#include <type_traits>

#include "kernels.h"

namespace cfdetr {

namespace {

constexpr int kThreads = 256;   // four wavefronts
constexpr int kUnitKeys = 32;   // keys of one step of a wavefront

__device__ __forceinline__ int swap_bits_2_3(int i) { return (i & ~12) | ((i & 4) << 1) | ((i & 8) >> 1); }

// Where the frames of a batch lie: lane l of every wavefront holds the offsets of frames 2l and 2l + 1
// (the merged run of the encoder has two sequences for each of up to 64 cameras).
struct Frames {
  int q[3], k[3];
  bool bad;   // a negative length, or an end beyond the rows: the whole call is refused
};
__device__ __forceinline__ Frames frames_of(const int32_t* __restrict__ cu_q, const int32_t* __restrict__ cu_k, int B, int n_q, int n_k) {
  const int l = 2 * (threadIdx.x & 63);
  Frames f;
  bool bad = false;
#pragma unroll
  for (int i = 0; i < 3; ++i) {
    f.q[i] = cu_q[min(l + i, B)];
    f.k[i] = cu_k[min(l + i, B)];
    bad |= f.q[i] < 0 || f.k[i] < 0 || f.q[i] > n_q || f.k[i] > n_k || (i > 0 && (f.q[i] < f.q[i - 1] || f.k[i] < f.k[i - 1]));
  }
  f.bad = __any(bad || (l == 0 && (f.q[0] != 0 || f.k[0] != 0)));
  return f;
}
// Sum of v over this lane and those before it: inside the vector unit, within rows of 16, then row 0 into 1 and 2 into 3,
// then 1 into 2 and 3.
__device__ __forceinline__ int sum_upto(int v) {
  auto from = [&](auto ctrl, auto rows) { return __builtin_amdgcn_update_dpp(0, v, decltype(ctrl)::value, decltype(rows)::value, 0xF, false); };
  const auto all = std::integral_constant<int, 0xF>{};
  v += from(std::integral_constant<int, 0x111>{}, all);   // row_shr:1, 2, 4, 8
  v += from(std::integral_constant<int, 0x112>{}, all);
  v += from(std::integral_constant<int, 0x114>{}, all);
  v += from(std::integral_constant<int, 0x118>{}, all);
  v += from(std::integral_constant<int, 0x142>{}, std::integral_constant<int, 0xA>{});   // row_bcast:15
  v += from(std::integral_constant<int, 0x143>{}, std::integral_constant<int, 0xC>{});   // row_bcast:31
  return v;
}
// The frame that piece `id` belongs to, where a frame has pieces[0 or 1] of them (lane's two frames, `upto` their sum_upto); `id`
// becomes the piece's number within it.  -1: there are fewer.
__device__ __forceinline__ int frame_of_piece(const int (&pieces)[2], int upto, int& id) {
  const uint64_t in = __ballot(upto > id);
  if (in == 0) return -1;
  const int l = __ffsll((unsigned long long)in) - 1;
  const int first = __builtin_amdgcn_readlane(pieces[0], l);
  id -= __builtin_amdgcn_readlane(upto, l) - first - __builtin_amdgcn_readlane(pieces[1], l);
  if (id < first) return 2 * l;
  id -= first;
  return 2 * l + 1;
}
// The pieces of a frame, `all` of them, that an XCD has: an eighth, in order.  Which eighth moves on by one from frame to frame (turn =
// XCD + frame), so that the rounding does not give one XCD more of every frame: 12 frames of 300 queries with 6 heads are
// 18 tiles of 128 a frame, 24 or 36 an XCD with one and the same turn, a second round on its 32 CUs: 60 us over 1000 keys, and 35 with 27 each.
__device__ __forceinline__ void xcd_share(int all, int turn, int& first, int& count) {
  const int x = turn & 7;
  first = (all >> 3) * x + (((all & 7) * x + 7) >> 3);
  count = (all >> 3) * (x + 1) + (((all & 7) * (x + 1) + 7) >> 3) - first;
}
__device__ __forceinline__ int of_lane_pair(const int (&values)[2], int frame) {
  const int even = __builtin_amdgcn_readlane(values[0], frame >> 1), odd = __builtin_amdgcn_readlane(values[1], frame >> 1);
  return (frame & 1) ? odd : even;
}
__device__ __forceinline__ int of_frame(const int (&offsets)[3], int frame) {
  const int even = __builtin_amdgcn_readlane(offsets[0], frame >> 1), odd = __builtin_amdgcn_readlane(offsets[1], frame >> 1);
  return (frame & 1) ? odd : even;
}
__device__ __forceinline__ int behind_frame(const int (&offsets)[3], int frame) {
  const int even = __builtin_amdgcn_readlane(offsets[1], frame >> 1), odd = __builtin_amdgcn_readlane(offsets[2], frame >> 1);
  return (frame & 1) ? odd : even;
}

// ---- elements --------------------------------------------------------------------------
// bf16: operands of 32x32x16 products, 8 elements a lane and step.  fp32: of 32x32x2 products, one.
// In both, an operand row in LDS or memory is cut into chunks of 16 bytes and a lane of group g (lanes 32 g on)
// has chunk 2c + g of chunk pair c.  S^T = K Q^T leaves a lane with 16 keys of one query.
template <typename T>
struct Elem;
template <>
struct Elem<bf16_t> {
  static constexpr int kChunk = 8;   // elements of 16 bytes
  typedef bf16x8 Frag;
  static __device__ __forceinline__ f32x16 dot(const uint4& k, const uint4& q, f32x16 acc) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(*reinterpret_cast<const bf16x8*>(&k), *reinterpret_cast<const bf16x8*>(&q), acc, 0, 0, 0);
  }
  // LDS row of a key and its values, so that eight consecutive result registers of a lane are eight consecutive keys
  static __device__ __forceinline__ int row_of_key(int key) { return swap_bits_2_3(key); }
  // key of result register r of lane group g
  static __device__ __forceinline__ int key_of(int r, int g) { return 16 * (r >> 3) + 8 * g + (r & 7); }
};
template <>
struct Elem<float> {
  static constexpr int kChunk = 4;
  static __device__ __forceinline__ f32x16 dot(const uint4& k, const uint4& q, f32x16 acc) {
    acc = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(k.x), __uint_as_float(q.x), acc, 0, 0, 0);
    acc = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(k.y), __uint_as_float(q.y), acc, 0, 0, 0);
    acc = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(k.z), __uint_as_float(q.z), acc, 0, 0, 0);
    return __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(k.w), __uint_as_float(q.w), acc, 0, 0, 0);
  }
  static __device__ __forceinline__ int row_of_key(int key) { return key; }
  static __device__ __forceinline__ int key_of(int r, int g) { return 8 * (r >> 2) + 4 * g + (r & 3); }
};

// Order of a row's chunks in LDS.  Keys: 16 rows that are read together lie in all banks.  Values: blocks of 32
// columns, moved so that the rows a product reads together lie in different banks.
template <typename T, int ROWB>
__device__ __forceinline__ int key_chunk(int row, int c) {
  return ROWB == 128 ? c ^ ((row >> 1) & 7) : c ^ (row & 15);
}
template <typename T, int ROWB>
__device__ __forceinline__ int value_block(int row, int b) {
  if constexpr (std::is_same_v<T, float>) return b ^ ((row >> 2) & 1);
  return ROWB == 128 ? b ^ ((row >> 1) & 1) : b ^ (row & 3);
}

// Sum of v over the lanes l and l ^ 32, and the larger of the two.
__device__ __forceinline__ float half_sum(float v) {
  typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
  const u32x2 p = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(p[0]) + __uint_as_float(p[1]);
}
__device__ __forceinline__ float half_max(float v) {
  typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
  const u32x2 p = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(p[0]), __uint_as_float(p[1]));
}

template <typename T, int N>
__device__ __forceinline__ void store_columns(T* to, const float (&x)[N]) {
  static_assert(N % 4 == 0, "whole quads");
  if constexpr (std::is_same_v<T, float>) {
#pragma unroll
    for (int i = 0; i < N / 4; ++i) reinterpret_cast<float4*>(to)[i] = make_float4(x[4 * i], x[4 * i + 1], x[4 * i + 2], x[4 * i + 3]);
  } else if constexpr (N % 8 == 0) {
#pragma unroll
    for (int i = 0; i < N / 8; ++i)
      reinterpret_cast<uint4*>(to)[i] = make_uint4(pack_bf16x2(x[8 * i], x[8 * i + 1]), pack_bf16x2(x[8 * i + 2], x[8 * i + 3]),
                                                   pack_bf16x2(x[8 * i + 4], x[8 * i + 5]), pack_bf16x2(x[8 * i + 6], x[8 * i + 7]));
  } else {
#pragma unroll
    for (int i = 0; i < N / 4; ++i)
      reinterpret_cast<uint2*>(to)[i] = make_uint2(pack_bf16x2(x[4 * i], x[4 * i + 1]), pack_bf16x2(x[4 * i + 2], x[4 * i + 3]));
  }
}

__device__ __forceinline__ void wave_fence() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// A unit of 32 keys with a running maximum, in three parts: the logits of a wavefront's 32 queries, their weights and
// what those make of the sums so far, and the values under the weights.  Keys and values lie in LDS, in rows
// of Elem::row_of_key; `left` of them are keys of the frame, and the values of the others are numbers.
template <typename T, int DH>
__device__ __forceinline__ void unit_logits(const unsigned char* sK, const uint4 (&qf)[2][DH * (int)sizeof(T) / 32], f32x16 (&s)[2]) {
  constexpr int ROWB = 2 * DH * (int)sizeof(T), KS = ROWB / 64;
  const int lane = threadIdx.x & 63, l32 = lane & 31, g = lane >> 5;
#pragma unroll
  for (int m = 0; m < 2; ++m)
#pragma unroll
    for (int r = 0; r < 16; ++r) s[m][r] = 0.f;
#pragma unroll
  for (int c = 0; c < KS; ++c)
#pragma unroll
    for (int m = 0; m < 2; ++m)
      s[m] = Elem<T>::dot(*reinterpret_cast<const uint4*>(sK + l32 * ROWB + key_chunk<T, ROWB>(l32, m * 2 * KS + 2 * c + g) * 16),
                          qf[m][c], s[m]);
}
// The reference of the weights follows the largest logit only once that is kSlack ahead (2^kSlack times the
// others): a quotient is the same for any reference, and with 32 queries in a wavefront some largest logit moves in almost every
// unit, which costs two operations for every sum (4 frames of 300 queries over 1600 to 6400 tokens: 43 -> 41.7 us).
// A weight is then 2^kSlack at most, and a sum of n values under them n 2^kSlack |v|: 32 bits hold it as long as n |v| stays
// below 2^(127 - kSlack), half a step of 2^-8 for the weights' rounding included.  The header promises 2^110.
constexpr float kSlack = 16.f;
template <typename T, int MO>
__device__ __forceinline__ void unit_weights(f32x16 (&s)[2], int left, float scale2, float (&m_run)[2], float (&l_run)[2], f32x16 (&acc)[2][MO]) {
  const int g = (threadIdx.x & 63) >> 5;
  if (left < kUnitKeys) {
#pragma unroll
    for (int m = 0; m < 2; ++m)
#pragma unroll
      for (int r = 0; r < 16; ++r)
        if (Elem<T>::key_of(r, g) >= left) s[m][r] = -INFINITY;
  }
#pragma unroll
  for (int m = 0; m < 2; ++m) {
    float top = s[m][0];
#pragma unroll
    for (int r = 1; r < 16; ++r) top = fmaxf(top, s[m][r]);
    top = half_max(top) * scale2;
    const bool follow = top > m_run[m] + kSlack;
    if (__any(follow)) {
      // (a query alone: what the wavefront's others are does not show in its row)
      const float alpha = follow ? __builtin_amdgcn_exp2f(m_run[m] - top) : 1.0f;
      if (follow) m_run[m] = top;
      l_run[m] *= alpha;
#pragma unroll
      for (int i = 0; i < MO; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[m][i][r] *= alpha;
    }
    const float m_ref = m_run[m] == -INFINITY ? 0.f : m_run[m];   // (every logit of a query may be -infinity so far)
    float sum = 0.f;
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      s[m][r] = __builtin_amdgcn_exp2f(fmaf(s[m][r], scale2, -m_ref));
      sum += s[m][r];
    }
    l_run[m] += sum;
  }
}
template <typename T, int DH>
__device__ __forceinline__ void unit_rows(const unsigned char* sV, const f32x16 (&s)[2], f32x16 (&acc)[2][DH / 16]) {
  constexpr int ROWB = 2 * DH * (int)sizeof(T), MO = DH / 16;
  const int lane = threadIdx.x & 63, l32 = lane & 31, g = lane >> 5;
  if constexpr (std::is_same_v<T, bf16_t>) {
    // A rounding of the weights to bf16: half a step of 2^-8 each, independent between keys and maps (what it does to their
    // difference: diff_tiles.hip).
    typedef __attribute__((ext_vector_type(4))) short s16x4;
    typedef __attribute__((address_space(3))) s16x4* lds4;
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      bf16x8 p[2];
#pragma unroll
      for (int m = 0; m < 2; ++m) {
        uint4 w = make_uint4(pack_bf16x2(s[m][8 * t], s[m][8 * t + 1]), pack_bf16x2(s[m][8 * t + 2], s[m][8 * t + 3]),
                             pack_bf16x2(s[m][8 * t + 4], s[m][8 * t + 5]), pack_bf16x2(s[m][8 * t + 6], s[m][8 * t + 7]));
        p[m] = *reinterpret_cast<bf16x8*>(&w);
      }
#pragma unroll
      for (int i = 0; i < MO; ++i) {
        // values come row by row; the transposing read gives a lane four keys of its column, a group of 16 lanes
        // naming the pieces of four keys by 16 columns
        union {
          s16x4 half[2];
          bf16x8 whole;
        } v;
#pragma unroll
        for (int hh = 0; hh < 2; ++hh) {
          const int row = 16 * t + 8 * hh + 4 * g + ((lane & 15) >> 2);   // of keys 16 t + 8 g + 4 hh on
          v.half[hh] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
              (lds4)(sV + row * ROWB + value_block<T, ROWB>(row, i) * 64 + ((lane >> 4) & 1) * 32 + (lane & 3) * 8));
        }
#pragma unroll
        for (int m = 0; m < 2; ++m) acc[m][i] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v.whole, p[m], acc[m][i], 0, 0, 0);
      }
    }
  } else {
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const int key = Elem<T>::key_of(r, g);
#pragma unroll
      for (int i = 0; i < MO; ++i) {
        const float v = *reinterpret_cast<const float*>(sV + key * ROWB + value_block<T, ROWB>(key, i) * 128 + l32 * 4);
#pragma unroll
        for (int m = 0; m < 2; ++m) acc[m][i] = __builtin_amdgcn_mfma_f32_32x32x2f32(v, s[m][r], acc[m][i], 0, 0, 0);
      }
    }
  }
}

// One 16-byte piece per lane from global memory straight into LDS (1 KB a wavefront at lds_addr, in lane order).  The
// compiler does not count these loads: whoever reads them waits with vmcnt first.
__device__ __forceinline__ void dma16(const void* sbase, uint32_t voff, uint32_t lds_addr) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" : : "s"(__builtin_amdgcn_readfirstlane(lds_addr)), "v"(voff), "s"(sbase) : "memory");
}
__device__ __forceinline__ void dma16(const void* from, uint32_t lds_addr) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" : : "s"(__builtin_amdgcn_readfirstlane(lds_addr)), "v"(from) : "memory");
}
// Which chunk of 16 bytes lies at place `c` of an LDS row of keys, and of values (both orders are their own inverse).
template <typename T, int ROWB>
__device__ __forceinline__ int key_piece(int row, int c) { return key_chunk<T, ROWB>(row, c); }
template <typename T, int ROWB>
__device__ __forceinline__ int value_piece(int row, int c) {
  constexpr int CPB = 2 * (int)sizeof(T);   // chunks of a block of 32 columns
  return value_block<T, ROWB>(row, c / CPB) * CPB + c % CPB;
}

}  // namespace

// The kernel for many queries (diff_tiles.hip), bf16.
hipError_t launch_diff_tiles(const DiffAttentionArgs& a, int d_head, hipStream_t s);

}  // namespace cfdetr
