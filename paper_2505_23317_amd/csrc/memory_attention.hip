// Attention of one new token of every stream over the tokens that its stream holds in a paged memory:
//   out[h] = sum_t softmax_t(scale q[h] . k[t, h / G]) v[t, h / G],   G = heads / key heads.
//
// One pass over keys and values, with a running maximum and sum.  A key and a value are read once for up to 16 query heads that
// share them in bf16 and for up to four in fp32 (the check mode), once more for every further 16 or four: 2 G operations a byte in
// bf16, so memory bounds it.
//
// A stream's tokens are units of 32 positions, cut into pieces of one length for all streams, a workgroup each (lengths are
// known on the device only, so every workgroup works the cut out for itself).  A piece gives a row under its own maximum; a
// stream of one piece is finished there, the rows of the others go to memory and the workgroup that ends last adds
// them up in order.  Units lie on multiples of 32 positions and pages hold 8 or more, so eight consecutive tokens of
// a unit are in one page.
#include <algorithm>
#include <cstddef>
#include <type_traits>

#include "kernels.h"
#include "stream_memory.h"

namespace cfdetr {

namespace {

constexpr int kUnit = kMemoryUnit;
// Measured as replays of a captured call, us; "768 / 4": width 768, four key heads.
// A piece has four units a wavefront at least, a stream of up to ten is not cut: adding the pieces takes 2 us and more, a tile
// 0.4 to 0.6.  One stream of 1,600 tokens, width 768: 10.5 (six units at least 12.2, eight 13.6; six streams of 4,000 to 16,000, 768 / 4,
// then 16.7 and 16.0 instead of 17.5); of 300: 9.1 (cut in two 10.2); 300 of up to 900, 256 wide, 22.0 (uncut up to sixteen 23.1, none 23.5).
constexpr int kLeast = 4, kUncut = 10;
// Eight wavefronts a workgroup, two workgroups a CU: 24 streams of 8,000 to 64,000, 768 / 2, 47.7, 300 of up to 900, 256 wide, 22.0, 1,024 of
// up to 100 18.3, one of 1,600, width 768, 10.5.  Sixteen and one: 49.2, 24.3, 31.3, 13.6; four and four: 51.0, 23.6, 19.2, 9.8.
constexpr int kWaves = 8;
constexpr int kResident = 2;   // workgroups that a CU has room for
constexpr int kMostUnits = 1 << 30;   // of all streams
__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }

// Tiles' slots and open tokens, those of up to 64 of a wavefront's tiles at a time: lane l has tile l's.
struct Tiles {
  int slot[4];     // of token 8 j; those behind it up to 8 j + 7 lie behind it
  uint32_t open;   // bit t: token t is read
};
__device__ __forceinline__ Tiles tiles_of(const MemoryAttentionArgs& a, const int32_t* table, int first, int end, int p0, bool any) {
  Tiles t{};
  if (!any) return t;
  const int lo = max(first - p0, 0), hi = min(end - p0, kUnit);
  t.open = (0xFFFFFFFFu >> (kUnit - hi)) & (0xFFFFFFFFu << lo);
  bool wrong = false;
  int id[4] = {};
#pragma unroll
  for (int j = 0; j < 4; ++j)
    if (t.open >> (8 * j) & 0xFF) id[j] = table[ring_column((p0 + 8 * j) >> a.page_bits, a.cols)];
  uint2 bytes[4] = {};
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    if ((unsigned)id[j] >= (unsigned)a.n_pages) {
      wrong = true;
      id[j] = 0;
      t.open &= ~(0xFFu << (8 * j));
    }
    t.slot[j] = (id[j] << a.page_bits) + ((p0 + 8 * j) & ((1 << a.page_bits) - 1));
    if (a.mask) bytes[j] = *reinterpret_cast<const uint2*>(a.mask + t.slot[j]);
  }
  if (a.mask) {
    uint32_t read = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if (bytes[j].x >> (8 * i) & 0xFF) read |= 1u << (8 * j + i);
        if (bytes[j].y >> (8 * i) & 0xFF) read |= 1u << (8 * j + 4 + i);
      }
    t.open &= read;
  }
  if (wrong) *a.err_flag = 1;
  return t;
}

// Maximum and sum over the lanes l, l ^ 16, l ^ 32, l ^ 48.
template <typename F>
__device__ __forceinline__ float across_quarters(float v, F f) {
  typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
  u32x2 p = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = f(__uint_as_float(p[0]), __uint_as_float(p[1]));
  p = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return f(__uint_as_float(p[0]), __uint_as_float(p[1]));
}

// The reference of the weights follows the largest logit only once that is kSlack ahead (in base 2): rows under the reference are
// multiplied less often.  A weight is 2^kSlack at most; the header promises sums for values below 2^110 / n.
constexpr float kSlack = 16.f;

// A logit in base 2, rounded: not part of a fused multiply-add, so that the largest one less itself is 0 whatever its size.
__device__ __forceinline__ float in_base_2(float s, float scale2) {
#pragma clang fp contract(off)
  return s * scale2;
}
// A fused multiply-add less the reference has what the reference's rounding left, 2^-25 of it: nothing beside kSlack up to here,
// past 2^31 more than a weight can hold.
constexpr float kFar = 1048576.f;

// What a wavefront leaves of its tiles: for row i of its kRows (query heads) a maximum, a sum and a row under that maximum.
template <int ROWS, int DH>
struct Rows {
  float m[ROWS], l[ROWS];
  alignas(16) float o[ROWS][DH];   // (16 bytes are written and read at once)
};
template <typename R>
constexpr bool rows_are_aligned(int bytes) { return offsetof(R, o) % 16 == 0 && bytes % 16 == 0; }

// bf16, several query heads a key head.  A wavefront has 128 bytes of every key and value row, a slab: NH key heads, and up to 16 query heads of each.
// Logits are products of 16 tokens x 32 features x 16 query heads, S^T = K Q^T, which leave lane l query head l mod 16 and tokens
// 4 (l / 16) + r of either half of the tile; these are at once the operand of O^T = V^T P^T if the products' index runs over
// the tokens in that order, so weights never leave their lane.  Two query heads of 16 leave the products 14 parts zeros, and still they cost a
// fraction of the loads' time.  Keys and values go straight into LDS, every wavefront's own, a tile ahead: no barrier in
// the loop.  (Two tiles ahead leave a CU one workgroup, measured with one product of the weights: 24 streams of 8,000 to 64,000, 768 / 2, 50.0 instead of 47.6 us, 1,024 of up
// to 100, 768 / 4, 30.3 instead of 19.1.)
template <int DH>
struct Core16 {
  typedef bf16_t T;
  static constexpr int kWavesSimd = kResident * kWaves / 4;
  static constexpr int kSlabHeads = 64 / DH, kGroup = 16, kRows = kSlabHeads * kGroup;
  static constexpr int kBytes = 2 * kUnit * 128;   // LDS of a tile: keys, values
  typedef Rows<kRows, DH> Result;
  static_assert(sizeof(Result) <= kBytes, "in place of keys and values");
  static_assert(rows_are_aligned<Result>(kBytes), "rows pass 16 bytes at a time");

  static __device__ __forceinline__ void run(const MemoryAttentionArgs& a, unsigned char* lds, int b, int slab, int group, int unit, int step,
                                             int units, int first, int end) {
    constexpr int NH = kSlabHeads, KS = DH / 32, NB = DH / 16;
    const int lane = threadIdx.x & 63, l16 = lane & 15, g = lane >> 4;
    const int G = a.heads / a.kv_heads;
    const int32_t* const table = a.table + (size_t)b * a.cols;
    // the queries' operand: query head l16 of either key head
    uint4 qf[NH][KS];
#pragma unroll
    for (int h = 0; h < NH; ++h) {
      const int kh = slab * NH + h, head = group * kGroup + l16;
      const bool mine = kh < a.kv_heads && head < G;
#pragma unroll
      for (int s = 0; s < KS; ++s) {
        qf[h][s] = make_uint4(0, 0, 0, 0);
        if (mine) qf[h][s] = *reinterpret_cast<const uint4*>(static_cast<const T*>(a.q) + (size_t)b * a.q_ld + (kh * G + head) * DH + 32 * s + 8 * g);
      }
    }
    f32x4 acc[NH][NB];
    float m_run[NH], l_run[NH], ref[NH];   // ref: m_run, or 0 as long as no token is open
    uint64_t far = 0;                      // lanes with a reference past kFar
#pragma unroll
    for (int h = 0; h < NH; ++h) {
      m_run[h] = -INFINITY;
      l_run[h] = ref[h] = 0.f;
#pragma unroll
      for (int n = 0; n < NB; ++n) acc[h][n] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    // Loads: lane l has place l mod 8 of token 8 j + l / 8.  A row's pieces of 16 bytes lie in LDS so that what is read together
    // lies in different banks: key piece c of token t at place c ^ (t / 2 mod 8), values in pairs of pieces, pair c at c ^ (t / 2 mod 4).
    const bool half = (slab + 1) * NH > a.kv_heads;   // (the slab's second key head is none: its first again)
    const int kc = (lane & 7) ^ g, vc = ((((lane & 7) >> 1) ^ g) << 1) | (lane & 1);
    const uint32_t k_step = (uint32_t)a.k_ld * 2, v_step = (uint32_t)a.v_ld * 2;
    const uint32_t k_lane = (uint32_t)(lane >> 3) * k_step + slab * 128, v_lane = (uint32_t)(lane >> 3) * v_step + slab * 128;
    const uint32_t k_even = k_lane + (half ? kc & 3 : kc) * 16, k_odd = k_lane + (half ? kc & 3 : kc ^ 4) * 16;
    const uint32_t v_off = v_lane + (half ? vc & 3 : vc) * 16;
    const unsigned char* const sK = lds;
    const unsigned char* const sV = lds + kUnit * 128;
    const uint32_t lds0 = (uint32_t)(uintptr_t)lds;
    const int p_first = first & ~(kUnit - 1);

#pragma nounroll
    for (; unit < units; unit += 64 * step) {
      const int count = min(64, (units - unit + step - 1) / step);
      const int p_lane = p_first + (unit + lane * step) * kUnit;
      Tiles t = tiles_of(a, table, first, end, p_lane, lane < count);
      // (ordinary loads are waited for here: the compiler does not count those into LDS, and would wait for all of them below)
      asm volatile("" : "+v"(t.slot[0]), "+v"(t.slot[1]), "+v"(t.slot[2]), "+v"(t.slot[3]), "+v"(t.open));
#pragma unroll
      for (int h = 0; h < NH; ++h)
#pragma unroll
        for (int s = 0; s < KS; ++s) asm volatile("" : "+v"(qf[h][s].x), "+v"(qf[h][s].y), "+v"(qf[h][s].z), "+v"(qf[h][s].w));

      auto load = [&](int i) {
        const uint32_t open = __builtin_amdgcn_readlane((int)t.open, i);
        const char *k[4], *v[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const uint64_t slot = (uint32_t)__builtin_amdgcn_readlane(t.slot[j], i);
          k[j] = static_cast<const char*>(a.k) + slot * k_step;
          v[j] = static_cast<const char*>(a.v) + slot * v_step;
        }
        if (open == 0xFFFFFFFFu) {
#pragma unroll
          for (int j = 0; j < 4; ++j) dma16(k[j], j & 1 ? k_odd : k_even, lds0 + j * 1024);
#pragma unroll
          for (int j = 0; j < 4; ++j) dma16(v[j], v_off, lds0 + (4 + j) * 1024);
        } else {
          // tokens that are not read: zeros, from the one place that all such lanes share
          const char* const zeros = static_cast<const char*>(a.zeros);
          const uint32_t mine = open >> (lane >> 3);
#pragma unroll
          for (int j = 0; j < 4; ++j) dma16(mine >> (8 * j) & 1 ? k[j] + (j & 1 ? k_odd : k_even) : zeros, lds0 + j * 1024);
#pragma unroll
          for (int j = 0; j < 4; ++j) dma16(mine >> (8 * j) & 1 ? v[j] + v_off : zeros, lds0 + (4 + j) * 1024);
        }
      };
      load(0);
#pragma nounroll
      for (int i = 0; i < count; ++i) {
        asm volatile("s_waitcnt vmcnt(0)" : : : "memory");
        // all operands at once: the tile's place is free for the next loads before a product is taken, and no product waits for a read
        typedef __attribute__((ext_vector_type(4))) short s16x4;
        typedef __attribute__((address_space(3))) s16x4* lds4;
        bf16x8 kf[NH][2][KS];
        union {
          s16x4 part[2];
          bf16x8 whole;
        } v[NH][NB];
#pragma unroll
        for (int h = 0; h < NH; ++h)
#pragma unroll
          for (int half16 = 0; half16 < 2; ++half16)
#pragma unroll
            for (int c = 0; c < KS; ++c) {
              const int row = 16 * half16 + l16, piece = (h * KS + c) * 4 + g;
              kf[h][half16][c] = *reinterpret_cast<const bf16x8*>(sK + row * 128 + (piece ^ ((row >> 1) & 7)) * 16);
            }
#pragma unroll
        for (int h = 0; h < NH; ++h)
#pragma unroll
          for (int n = 0; n < NB; ++n)
#pragma unroll
            for (int half16 = 0; half16 < 2; ++half16) {
              // the transposing read gives a lane four tokens of its column, 16 lanes naming the pieces of four tokens by 16 columns
              const int row = 16 * half16 + 4 * g + (l16 >> 2);
              v[h][n].part[half16] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)(
                  sV + row * 128 + ((h * NB + n) ^ ((row >> 1) & 3)) * 32 + (lane & 3) * 8));
            }
        asm volatile("s_waitcnt lgkmcnt(0)" : : : "memory");
        if (i + 1 < count) load(i + 1);
        f32x4 s[NH][2];
#pragma unroll
        for (int h = 0; h < NH; ++h)
#pragma unroll
          for (int half16 = 0; half16 < 2; ++half16) {
            s[h][half16] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int c = 0; c < KS; ++c)
              s[h][half16] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[h][half16][c], *reinterpret_cast<const bf16x8*>(&qf[h][c]), s[h][half16], 0, 0, 0);
          }
        const uint32_t open = __builtin_amdgcn_readlane((int)t.open, i);
        union {
          uint32_t part[4];
          bf16x8 whole;
        } w[NH][2];
#pragma unroll
        for (int h = 0; h < NH; ++h) {
          if (open != 0xFFFFFFFFu) {
            const uint32_t mine = open >> (4 * g);
#pragma unroll
            for (int r = 0; r < 4; ++r) {
              if (!(mine >> r & 1)) s[h][0][r] = -INFINITY;
              if (!(mine >> (16 + r) & 1)) s[h][1][r] = -INFINITY;
            }
          }
          // The weights under the reference so far, and beside them whether it is to follow: it seldom is, and the products
          // then need not wait for the maximum.
          float p[8];
          auto weigh = [&] {
            if (__builtin_expect(far == 0, 1)) {
#pragma unroll
              for (int r = 0; r < 8; ++r) p[r] = __builtin_amdgcn_exp2f(fmaf(s[h][r >> 2][r & 3], a.scale2, -ref[h]));
            } else {
#pragma unroll
              for (int r = 0; r < 8; ++r) p[r] = __builtin_amdgcn_exp2f(in_base_2(s[h][r >> 2][r & 3], a.scale2) - ref[h]);
            }
          };
          weigh();
#pragma unroll
          for (int r = 0; r < 8; ++r) asm volatile("" : "+v"(p[r]));
          float top = s[h][0][0];
#pragma unroll
          for (int r = 1; r < 8; ++r) top = fmaxf(top, s[h][r >> 2][r & 3]);
          top = in_base_2(across_quarters(top, [](float x, float y) { return fmaxf(x, y); }), a.scale2);
          const bool follow = top > m_run[h] + kSlack;
          if (__any(follow)) {
            const float alpha = follow ? __builtin_amdgcn_exp2f(m_run[h] - top) : 1.0f;
            if (follow) m_run[h] = ref[h] = top;
            far |= __ballot(fabsf(ref[h]) > kFar);
            l_run[h] *= alpha;
#pragma unroll
            for (int n = 0; n < NB; ++n) acc[h][n] *= alpha;
            weigh();
          }
          float sum = 0.f;
#pragma unroll
          for (int r = 0; r < 8; ++r) sum += p[r];
          l_run[h] += sum;
          // A weight goes into two products, itself rounded to bf16 and what that leaves, rounded to bf16: off by 2^-16 of itself
          // and not by 2^-8, rows by 0.0017 of their size and not by 0.0023 (their own rounding is 0.0017).  The second costs 24 streams
          // of 8,000 to 64,000, 768 / 2, 47.1 -> 47.3 us, one of 1,600, 256 / 4, 10.9 -> 11.4, 300 of up to 900, 256 / 4, 15.5 -> 16.7.
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const uint32_t hi = pack_bf16x2(p[2 * r], p[2 * r + 1]);
            w[h][0].part[r] = hi;
            w[h][1].part[r] = pack_bf16x2(p[2 * r] - __uint_as_float(hi << 16), p[2 * r + 1] - __uint_as_float(hi & 0xFFFF0000u));
          }
        }
#pragma unroll
        for (int of = 0; of < 2; ++of)
#pragma unroll
          for (int h = 0; h < NH; ++h)
#pragma unroll
            for (int n = 0; n < NB; ++n) acc[h][n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v[h][n].whole, w[h][of].whole, acc[h][n], 0, 0, 0);
      }
    }
    // (the LDS of keys and values is free: every read has been waited for)
    Result* const to = reinterpret_cast<Result*>(lds);
#pragma unroll
    for (int h = 0; h < NH; ++h) {
      const float l = across_quarters(l_run[h], [](float x, float y) { return x + y; });
      const int row = h * kGroup + l16;
      if (group * kGroup + l16 >= G) continue;
      if (g == 0) {
        to->m[row] = m_run[h];
        to->l[row] = l;
      }
#pragma unroll
      for (int n = 0; n < NB; ++n) *reinterpret_cast<f32x4*>(&to->o[row][16 * n + 4 * g]) = acc[h][n];
    }
  }
};

// Sum of v over LANES (4, 8 or 16) consecutive lanes, delivered to all of them, inside the vector unit.
template <int LANES>
__device__ __forceinline__ float row_sum(float v) {
  auto from = [&](auto ctrl) { return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), decltype(ctrl)::value, 0xF, 0xF, false)); };
  v += from(std::integral_constant<int, 0xB1>{});    // quad_perm [1, 0, 3, 2]
  v += from(std::integral_constant<int, 0x4E>{});    // quad_perm [2, 3, 0, 1]
  if constexpr (LANES >= 8) v += from(std::integral_constant<int, 0x141>{});    // row_half_mirror: the other quad of eight
  if constexpr (LANES == 16) v += from(std::integral_constant<int, 0x140>{});   // row_mirror: the other eight
  return v;
}

// 16 bytes of a row.
template <typename T>
struct Bytes16;
template <>
struct Bytes16<bf16_t> {
  static constexpr int kN = 8;
  static __device__ __forceinline__ float dot(const uint4& a, const uint4& b) {
    auto two = [](uint32_t x, uint32_t y, float c) {
      return __builtin_amdgcn_fdot2_f32_bf16(*reinterpret_cast<const bf16x2*>(&x), *reinterpret_cast<const bf16x2*>(&y), c, false);
    };
    return two(a.x, b.x, two(a.y, b.y, two(a.z, b.z, two(a.w, b.w, 0.f))));
  }
  static __device__ __forceinline__ void get(const uint4& v, float (&x)[kN]) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[2 * i] = __uint_as_float(w[i] << 16);
      x[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
    }
  }
};
template <>
struct Bytes16<float> {
  static constexpr int kN = 4;
  static __device__ __forceinline__ float dot(const uint4& a, const uint4& b) {
    auto f = [](uint32_t x) { return __uint_as_float(x); };
    return fmaf(f(a.x), f(b.x), fmaf(f(a.y), f(b.y), fmaf(f(a.z), f(b.z), f(a.w) * f(b.w))));
  }
  static __device__ __forceinline__ void get(const uint4& v, float (&x)[kN]) {
    x[0] = __uint_as_float(v.x);
    x[1] = __uint_as_float(v.y);
    x[2] = __uint_as_float(v.z);
    x[3] = __uint_as_float(v.w);
  }
};

// One query head a key head, and fp32 (the check mode): a wavefront has 128 bytes or a head of every row, and up to GROUP query heads of a
// key head.  Lanes hold a row's pieces of 16 bytes, LANES of them a token, so a load takes 64 / LANES tokens; each group of lanes has
// a maximum, sum and row of its own until the end.  Weights stay in 32 bits.
template <typename E, int DH, int GROUP>
struct CoreLanes {
  typedef E T;
  static constexpr int N = Bytes16<E>::kN, kPieces = DH / N;   // of a head
  static constexpr int kWavesSimd = 2;
  static constexpr int kSlabHeads = kPieces < 8 ? 8 / kPieces : 1, kGroup = GROUP, kRows = kSlabHeads * GROUP;
  typedef Rows<kRows, DH> Result;
  static constexpr int kBytes = (sizeof(Result) + 255) / 256 * 256;
  static_assert(rows_are_aligned<Result>(kBytes), "rows pass 16 bytes at a time");

  static __device__ __forceinline__ void run(const MemoryAttentionArgs& a, unsigned char* lds, int b, int slab, int group, int unit, int step,
                                             int units, int first, int end) {
    constexpr int LANES = kSlabHeads * kPieces, TPL = 64 / LANES, LOADS = kUnit / TPL;
    static_assert(LANES >= 8, "the tokens of a load lie behind each other");
    const int lane = threadIdx.x & 63, part = lane / LANES, in_slab = lane % LANES / kPieces, c = lane % kPieces;
    const int G = a.heads / a.kv_heads;
    const int kh = min(slab * kSlabHeads + in_slab, a.kv_heads - 1);   // (a slab's last head again, where there are fewer)
    const int32_t* const table = a.table + (size_t)b * a.cols;
    uint4 q[GROUP];
    float acc[GROUP][N], m[GROUP], l[GROUP];
#pragma unroll
    for (int h = 0; h < GROUP; ++h) {
      const int head = kh * G + min(group * GROUP + h, G - 1);   // (and a group's)
      q[h] = *reinterpret_cast<const uint4*>(static_cast<const T*>(a.q) + (size_t)b * a.q_ld + head * DH + N * c);
      m[h] = -INFINITY;
      l[h] = 0.f;
#pragma unroll
      for (int e = 0; e < N; ++e) acc[h][e] = 0.f;
    }
    const int p_first = first & ~(kUnit - 1);
    const uint32_t column = (kh * DH + N * c) * (uint32_t)sizeof(T);
    const uint32_t k_step = (uint32_t)a.k_ld * (uint32_t)sizeof(T), v_step = (uint32_t)a.v_ld * (uint32_t)sizeof(T);
    const uint32_t k_lane = part * k_step + column, v_lane = part * v_step + column;
    for (; unit < units; unit += 64 * step) {
      const int count = min(64, (units - unit + step - 1) / step);
      const Tiles t = tiles_of(a, table, first, end, p_first + (unit + lane * step) * kUnit, lane < count);
      for (int i = 0; i < count; ++i) {
        const uint32_t open = __builtin_amdgcn_readlane((int)t.open, i);
        uint4 k[LOADS], v[LOADS];
        const char *k_from[LOADS], *v_from[LOADS];
#pragma unroll
        for (int j = 0; j < LOADS; ++j) {
          const uint64_t slot = (uint32_t)__builtin_amdgcn_readlane(t.slot[j * TPL / 8], i) + j * TPL % 8;
          k_from[j] = static_cast<const char*>(a.k) + slot * k_step;
          v_from[j] = static_cast<const char*>(a.v) + slot * v_step;
        }
        if (open == 0xFFFFFFFFu) {
#pragma unroll
          for (int j = 0; j < LOADS; ++j) k[j] = *reinterpret_cast<const uint4*>(k_from[j] + k_lane);
#pragma unroll
          for (int j = 0; j < LOADS; ++j) v[j] = *reinterpret_cast<const uint4*>(v_from[j] + v_lane);
        } else {
          // tokens that are not read: zeros, from the one place that all such lanes share
          const char* const zeros = static_cast<const char*>(a.zeros);
          const uint32_t mine = open >> part;
#pragma unroll
          for (int j = 0; j < LOADS; ++j) k[j] = *reinterpret_cast<const uint4*>(mine >> (j * TPL) & 1 ? k_from[j] + k_lane : zeros);
#pragma unroll
          for (int j = 0; j < LOADS; ++j) v[j] = *reinterpret_cast<const uint4*>(mine >> (j * TPL) & 1 ? v_from[j] + v_lane : zeros);
        }
        float s[GROUP][LOADS];
#pragma unroll
        for (int h = 0; h < GROUP; ++h)
#pragma unroll
          for (int j = 0; j < LOADS; ++j) s[h][j] = in_base_2(row_sum<kPieces>(Bytes16<T>::dot(q[h], k[j])), a.scale2);
        if (open != 0xFFFFFFFFu) {
#pragma unroll
          for (int j = 0; j < LOADS; ++j)
            if (!(open >> (j * TPL + part) & 1))
#pragma unroll
              for (int h = 0; h < GROUP; ++h) s[h][j] = -INFINITY;
        }
#pragma unroll
        for (int h = 0; h < GROUP; ++h) {
          float top = m[h];
#pragma unroll
          for (int j = 0; j < LOADS; ++j) top = fmaxf(top, s[h][j]);
          const float ref = top == -INFINITY ? 0.f : top, keep = __builtin_amdgcn_exp2f(m[h] - ref);
          m[h] = top;
          l[h] *= keep;
#pragma unroll
          for (int e = 0; e < N; ++e) acc[h][e] *= keep;
#pragma unroll
          for (int j = 0; j < LOADS; ++j) {
            s[h][j] = __builtin_amdgcn_exp2f(s[h][j] - ref);
            l[h] += s[h][j];
          }
        }
#pragma unroll
        for (int j = 0; j < LOADS; ++j) {
          float x[N];
          Bytes16<T>::get(v[j], x);
#pragma unroll
          for (int h = 0; h < GROUP; ++h)
#pragma unroll
            for (int e = 0; e < N; ++e) acc[h][e] = fmaf(s[h][j], x[e], acc[h][e]);
        }
      }
    }
    Result* const to = reinterpret_cast<Result*>(lds);
#pragma unroll
    for (int h = 0; h < GROUP; ++h) {
      float top = m[h];
#pragma unroll
      for (int o = LANES; o < 64; o <<= 1) top = fmaxf(top, __shfl_xor(top, o));
      const float f = __builtin_amdgcn_exp2f(m[h] - (top == -INFINITY ? 0.f : top));
      l[h] *= f;
#pragma unroll
      for (int e = 0; e < N; ++e) acc[h][e] *= f;
#pragma unroll
      for (int o = LANES; o < 64; o <<= 1) {
        l[h] += __shfl_xor(l[h], o);
#pragma unroll
        for (int e = 0; e < N; ++e) acc[h][e] += __shfl_xor(acc[h][e], o);
      }
      if (part == 0) {
        const int row = in_slab * GROUP + h;
        if (c == 0) {
          to->m[row] = top;
          to->l[row] = l[h];
        }
#pragma unroll
        for (int e = 0; e < N; e += 4)
          *reinterpret_cast<float4*>(&to->o[row][N * c + e]) = make_float4(acc[h][e], acc[h][e + 1], acc[h][e + 2], acc[h][e + 3]);
      }
    }
  }
};

template <typename T>
__device__ __forceinline__ void store4(T* to, float4 x) {
  if constexpr (std::is_same_v<T, float>) *reinterpret_cast<float4*>(to) = x;
  else *reinterpret_cast<uint2*>(to) = make_uint2(pack_bf16x2(x.x, x.y), pack_bf16x2(x.z, x.w));
}

// Pieces pass between workgroups of any XCD, whose L2s do not see each other's: every one is written past them (stores of device
// scope, waited for before the workgroup is counted) and read past them.  A release and an acquire around the counter would do the
// same for all of an L2: one stream of 200,003 tokens, width 768, 116 us so, 267 with them.
struct Shared {
  __amdgpu_buffer_rsrc_t at;
  typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
  typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
  static constexpr int kDevice = 16;   // sc1
  __device__ explicit Shared(void* p) : at(__builtin_amdgcn_make_buffer_rsrc(p, 0, 0x7FFFFFFF, 0x00027000)) {}
  __device__ __forceinline__ void put(int i, float2 v) const {
    __builtin_amdgcn_raw_buffer_store_b64(u32x2{__float_as_uint(v.x), __float_as_uint(v.y)}, at, i * 8, 0, kDevice);
  }
  __device__ __forceinline__ void put(int i, float4 v) const {
    __builtin_amdgcn_raw_buffer_store_b128(u32x4{__float_as_uint(v.x), __float_as_uint(v.y), __float_as_uint(v.z), __float_as_uint(v.w)}, at, i * 16, 0, kDevice);
  }
  __device__ __forceinline__ float2 get2(int i) const {
    const u32x2 v = __builtin_amdgcn_raw_buffer_load_b64(at, i * 8, 0, kDevice);
    return make_float2(__uint_as_float(v[0]), __uint_as_float(v[1]));
  }
  __device__ __forceinline__ float4 get4(int i) const {
    const u32x4 v = __builtin_amdgcn_raw_buffer_load_b128(at, i * 16, 0, kDevice);
    return make_float4(__uint_as_float(v[0]), __uint_as_float(v[1]), __uint_as_float(v[2]), __uint_as_float(v[3]));
  }
};
// Four columns of a row under a maximum.
struct Sum {
  float m, l;
  float4 o;
  __device__ __forceinline__ void add(const Sum& s) {
    const float top = fmaxf(m, s.m), ref = top == -INFINITY ? 0.f : top;
    const float f = __builtin_amdgcn_exp2f(m - ref), g = __builtin_amdgcn_exp2f(s.m - ref);
    m = top;
    l = fmaf(l, f, s.l * g);
    o = make_float4(fmaf(o.x, f, s.o.x * g), fmaf(o.y, f, s.o.y * g), fmaf(o.z, f, s.o.z * g), fmaf(o.w, f, s.o.w * g));
  }
  template <typename T>
  __device__ __forceinline__ void store(T* to) const {
    const float inv = l != 0.f ? 1.0f / l : 0.f;
    store4(to, make_float4(o.x * inv, o.y * inv, o.z * inv, o.w * inv));
  }
};
// First query head of a slab: slabs go through the key heads and, where a key head has more query heads than a wavefront takes,
// through groups of these, so that the query heads of consecutive slabs lie behind each other.
template <typename Core>
__device__ __forceinline__ int first_head(int slab, int passes, int G) {
  return slab / passes * Core::kSlabHeads * G + slab % passes * Core::kGroup;
}

// How the streams are cut, and which piece a workgroup has.
struct Piece {
  int stream, number, pieces;   // -1: there is no such piece
  int length;                   // of all pieces but a stream's last, in units
  int first, held;              // the stream's span
  bool bad;                     // a span is none, or there are too many units
};
// The wavefronts share the streams, rows of 64 that lie behind each other.  Up to 64 streams every wavefront has them all and needs no
// barrier (one stream of 64 tokens 6.3 us, 7.2 with all three).
template <int NW>
__device__ __forceinline__ Piece find_piece(const MemoryAttentionArgs& a, int piece, int least) {
  constexpr int R = kMemoryMaxStreams / 64 / NW;   // rows of a wavefront, at most
  __shared__ int s_sums[3][NW];
  __shared__ Piece s_found;
  const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6), B = a.B;
  const bool alone = B <= 64;
  const int rows = alone ? 1 : (B + 64 * NW - 1) / (64 * NW), b0 = alone ? 0 : wave * rows * 64;
  Piece p{-1, 0, 0, 0, 0, 0, false};
  int2 span[R];
#pragma unroll
  for (int r = 0; r < R; ++r) {
    if (r >= rows) break;
    const int b = b0 + 64 * r + lane;
    span[r] = b < B ? a.span[b] : make_int2(0, 0);
  }
  int units = 0;   // (of up to 8 streams of 2^24 units)
#pragma unroll
  for (int r = 0; r < R; ++r) {
    if (r >= rows) break;
    if (span_is_bad(span[r].x, span[r].y, a.page_bits, a.cols)) p.bad = true;
    else units += units_of(span[r].x, span[r].y);
  }
  // (the units' thousands tell whether their sum fits 32 bits)
  int total = __builtin_amdgcn_readlane(sum_upto(units), 63), thousands = __builtin_amdgcn_readlane(sum_upto((units + 1023) / 1024), 63);
  if (__any(p.bad)) thousands = kMostUnits;
  if (!alone) {
    if (lane == 0) {
      s_sums[0][wave] = total;
      s_sums[1][wave] = min(thousands, kMostUnits / 1024 + 1);
    }
    if (threadIdx.x == 0) s_found = p;
    __syncthreads();
    total = thousands = 0;
#pragma unroll
    for (int w = 0; w < NW; ++w) {
      total += s_sums[0][w];
      thousands += s_sums[1][w];
    }
    total = uniform(total);
    thousands = uniform(thousands);
  }
  p.bad = thousands > kMostUnits / 1024;
  if (p.bad) return p;
  const int length = cut_length(total, B, a.places, least);
  p.length = length;
  const float per_length = 1.0f / (float)length;
  int pieces[R], upto[R], before = 0;
#pragma unroll
  for (int r = 0; r < R; ++r) {
    if (r >= rows) break;
    pieces[r] = pieces_of(units_of(span[r].x, span[r].y), length, per_length, kUncut * (least / kLeast));
    upto[r] = before + sum_upto(pieces[r]);
    before = __builtin_amdgcn_readlane(upto[r], 63);
  }
  if (!alone) {
    if (lane == 0) s_sums[2][wave] = before;
    __syncthreads();
    for (int w = 0; w < wave; ++w) piece -= s_sums[2][w];
    piece = uniform(piece);
  }
  if (piece >= 0 && piece < before) {
#pragma unroll
    for (int r = 0; r < R; ++r) {
      if (r >= rows) break;
      const uint64_t in = __ballot(upto[r] > piece);
      if (in == 0) continue;
      const int l = __ffsll((unsigned long long)in) - 1;
      p.stream = b0 + 64 * r + l;
      p.pieces = __builtin_amdgcn_readlane(pieces[r], l);
      p.number = piece - (__builtin_amdgcn_readlane(upto[r], l) - p.pieces);
      p.first = __builtin_amdgcn_readlane(span[r].x, l);
      p.held = __builtin_amdgcn_readlane(span[r].y, l);
      break;
    }
    if (!alone && lane == 0) s_found = p;
  }
  if (!alone) {
    __syncthreads();
    p.stream = uniform(s_found.stream);
    p.pieces = uniform(s_found.pieces);
    p.number = uniform(s_found.number);
    p.first = uniform(s_found.first);
    p.held = uniform(s_found.held);
  }
  return p;
}

// n / d for small numbers (n < 2^16), without the long division.
__device__ __forceinline__ int quotient(int n, float one_over_d) { return (int)(((float)n + 0.5f) * one_over_d); }

// Workgroup: one piece of a stream and a.wave_slabs of the slabs; its NW wavefronts have one slab each, and where
// that leaves some over, every second, third, .. tile of it.
template <typename Core, int DH, int NW>
__global__ __launch_bounds__(64 * NW, Core::kWavesSimd) void memory_attention_kernel(MemoryAttentionArgs a) {
  typedef typename Core::T T;
  typedef typename Core::Result Result;
  constexpr int kThreads = 64 * NW, Q = DH / 4;
  __shared__ __attribute__((aligned(1024))) unsigned char smem[std::max(NW * Core::kBytes, kThreads * (int)sizeof(Sum))];
  __shared__ int s_last;
  const int tid = threadIdx.x, wave = uniform(tid >> 6);
  const int G = a.heads / a.kv_heads;
  const int passes = (G + Core::kGroup - 1) / Core::kGroup, slabs = (a.kv_heads + Core::kSlabHeads - 1) / Core::kSlabHeads * passes;
  const int WS = a.wave_slabs, TS = NW / WS, slab_groups = slabs / WS;
  const int number = blockIdx.x / slab_groups, slab_group = blockIdx.x - number * slab_groups;
  const Piece p = find_piece<NW>(a, number, kLeast * TS);
  if (p.bad) {
    if (blockIdx.x == 0 && tid == 0) *a.err_flag = 1;
    return;
  }
  // the row of a stream that holds nothing (there are more workgroups than streams)
  if ((int)blockIdx.x < a.B && a.span[blockIdx.x].y == 0)
    for (int i = tid; i < a.heads * Q; i += kThreads) store4(static_cast<T*>(a.out) + (size_t)blockIdx.x * a.out_ld + 4 * i, make_float4(0.f, 0.f, 0.f, 0.f));
  if (p.stream < 0) return;
  const int b = p.stream, units = units_of(p.first, p.held);
  const int u0 = p.number * p.length, u1 = p.pieces == 1 ? units : min(u0 + p.length, units);
  const int my_slab = slab_group * WS + wave % WS;
  Core::run(a, smem + wave * Core::kBytes, b, my_slab / passes, my_slab % passes, u0 + wave / WS, TS, u1, p.first, p.first + p.held);
  __syncthreads();

  // The wavefronts' rows of a query head to one maximum, and added: a thread has four columns.  The group's query heads lie one
  // behind the other: those of a slab's key heads, or a group of those of one key head.
  const int head0 = first_head<Core>(slab_group * WS, passes, G), heads = min(first_head<Core>((slab_group + 1) * WS, passes, G), a.heads) - head0;
  const int items = heads * Q;
  const float per_key = 1.0f / (float)G;
  const Shared all_ml(a.partial_ml), all_rows(a.partial);
  for (int i = tid; i < items; i += kThreads) {
    const int quad = i % Q, head = head0 + i / Q;
    const int kh = quotient(head, per_key), in_key = head - kh * G;
    const int slab = kh / Core::kSlabHeads * passes + in_key / Core::kGroup, row = kh % Core::kSlabHeads * Core::kGroup + in_key % Core::kGroup;
    Sum sum{-INFINITY, 0.f, make_float4(0.f, 0.f, 0.f, 0.f)};
    for (int part = 0; part < TS; ++part) {
      const Result* const r = reinterpret_cast<const Result*>(smem + (part * WS + slab - slab_group * WS) * Core::kBytes);
      sum.add(Sum{r->m[row], r->l[row], *reinterpret_cast<const float4*>(&r->o[row][4 * quad])});
    }
    if (p.pieces == 1) {
      sum.store(static_cast<T*>(a.out) + (size_t)b * a.out_ld + head * DH + 4 * quad);
    } else {
      const int at = number * a.heads + head;
      if (quad == 0) all_ml.put(at, make_float2(sum.m, sum.l));
      all_rows.put(at * Q + quad, sum.o);
    }
  }
  if (p.pieces == 1) return;
  // the pieces of a stream: the workgroup that ends last adds them up, in order
  asm volatile("s_waitcnt vmcnt(0)" : : : "memory");   // (a piece has arrived in memory before its workgroup is counted)
  __syncthreads();
  if (tid == 0) {
    int32_t* const ticket = a.tickets + (size_t)b * slab_groups + slab_group;
    s_last = __hip_atomic_fetch_add(ticket, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == p.pieces - 1;
    if (s_last) __hip_atomic_store(ticket, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  }
  __syncthreads();
  if (!s_last) return;
  // as many threads four columns as there are
  const int parts = max(1, kThreads / items);
  Sum* const s_sum = reinterpret_cast<Sum*>(smem);
  for (int i0 = 0; i0 < items; i0 += kThreads) {
    const int part = parts > 1 ? quotient(tid, 1.0f / (float)items) : 0, item = i0 + tid - part * items;
    const int head = head0 + item / Q, quad = item % Q;
    Sum sum{-INFINITY, 0.f, make_float4(0.f, 0.f, 0.f, 0.f)};
    if (item < items && part < parts) {
      auto add = [&](int r, auto count) {
        constexpr int N = decltype(count)::value;
        float2 ml[N];
        float4 o[N];
#pragma unroll
        for (int n = 0; n < N; ++n) {
          const int at = (number - p.number + min(r + n * parts, p.pieces - 1)) * a.heads + head;
          ml[n] = all_ml.get2(at);
          o[n] = all_rows.get4(at * Q + quad);
        }
        float top = sum.m;
#pragma unroll
        for (int n = 0; n < N; ++n) {
          if (r + n * parts >= p.pieces) ml[n] = make_float2(-INFINITY, 0.f);
          top = fmaxf(top, ml[n].x);
        }
        const float ref = top == -INFINITY ? 0.f : top, keep = __builtin_amdgcn_exp2f(sum.m - ref);
        sum = Sum{top, sum.l * keep, make_float4(sum.o.x * keep, sum.o.y * keep, sum.o.z * keep, sum.o.w * keep)};
#pragma unroll
        for (int n = 0; n < N; ++n) {
          const float f = __builtin_amdgcn_exp2f(ml[n].x - ref);
          sum.l = fmaf(ml[n].y, f, sum.l);
          sum.o = make_float4(fmaf(o[n].x, f, sum.o.x), fmaf(o[n].y, f, sum.o.y), fmaf(o[n].z, f, sum.o.z), fmaf(o[n].w, f, sum.o.w));
        }
      };
      int r = part;
      for (; r + 4 * parts < p.pieces; r += 8 * parts) add(r, std::integral_constant<int, 8>{});
      if (r + parts < p.pieces) add(r, std::integral_constant<int, 4>{});
      else if (r < p.pieces) add(r, std::integral_constant<int, 1>{});
    }
    if (parts > 1) {
      s_sum[tid] = sum;
      __syncthreads();
      if (part == 0)
        for (int n = 1; n < parts; ++n) sum.add(s_sum[n * items + tid]);
    }
    if (item < items && part == 0) sum.store(static_cast<T*>(a.out) + (size_t)b * a.out_ld + head * DH + 4 * quad);
  }
}

template <typename Core, int DH, int NW>
hipError_t launch(MemoryAttentionArgs a, int cus, hipStream_t s) {
  const int G = a.heads / a.kv_heads, passes = (G + Core::kGroup - 1) / Core::kGroup;
  const int slabs = (a.kv_heads + Core::kSlabHeads - 1) / Core::kSlabHeads * passes;
  // Four slabs a workgroup, where their number can be cut so: it reads 512 bytes of a row together, and the streams' cut is made by a
  // quarter of the workgroups.  24 streams of 8,000 to 30,000, 768 / 12: 210 us, two 278, one 270; 1,024 of up to 100 46, 77, 143; 300 of up
  // to 900 53, 55, 70; only 64 of 2,000 94, 78, 74.  Eight, 1024 / 16 and / 8: 1,024 of up to 100 60 -> 40, 24 long ones 291 -> 269, but one of 50,001
  // 39.7 -> 42.2 and 26.6 -> 35.1, 64 of 2,000 97 -> 109, 300 of up to 900 77 -> 80.
  a.wave_slabs = slabs % 4 == 0 ? 4 : slabs % 2 == 0 ? 2 : 1;
  const int slab_groups = slabs / a.wave_slabs;
  // One workgroup a CU has enough asked for to keep memory busy; the CU's second place is for what streams leave over.  24 streams of
  // 8,000 to 64,000, a fifth masked: 47.6 us, 51.0 with pieces for both places; one of 200,003, width 768, 115.9 and 119.4.
  a.places = std::max(1, cus / slab_groups);
  hipLaunchKernelGGL((memory_attention_kernel<Core, DH, NW>), dim3(most_pieces(a.B, a.places) * slab_groups), dim3(64 * NW), 0, s, a);
  return hipGetLastError();
}

// Key heads of one query head go through lanes, those of several through matrix products, whose time is that of 16.  bf16, us:
// one query head, 256 wide in heads of 32: one stream of 1,600 tokens 10.1 by lanes, 11.9 by products; 1,024 of up to 100 18.4 and
// 21.5; heads of 64, width 768: 10.5 and 10.3, one stream of 200,003 116 and 116, and weights stay in 32 bits.  Two query
// heads: one stream of 1,600, 256 / 4 key heads, 12.3 and 11.4, 300 of up to 900 18.5 and 16.7.
template <int DH>
hipError_t launch(const MemoryAttentionArgs& a, bool use_bf16, int cus, hipStream_t s) {
  const int G = a.heads / a.kv_heads;
  if (use_bf16) {
    if (G == 1) return launch<CoreLanes<bf16_t, DH, 1>, DH, kWaves>(a, cus, s);
    return launch<Core16<DH>, DH, kWaves>(a, cus, s);
  }
  if (G == 1) return launch<CoreLanes<float, DH, 1>, DH, kWaves>(a, cus, s);
  return G == 2 ? launch<CoreLanes<float, DH, 2>, DH, kWaves>(a, cus, s) : launch<CoreLanes<float, DH, 4>, DH, kWaves>(a, cus, s);
}

}  // namespace

MemoryAttentionSpace memory_attention_space(int max_streams, int heads, int d_head, int cus) {
  // (places are CUs at most, and slabs as query heads)
  const uint64_t pieces = (uint64_t)most_pieces(max_streams, cus) * heads;
  return {pieces * sizeof(float2), pieces * d_head * sizeof(float), (uint64_t)max_streams * heads * sizeof(int32_t)};
}

hipError_t launch_memory_attention(const MemoryAttentionArgs& a, int d_head, bool use_bf16, int cus, hipStream_t s) {
  if (d_head == 64) return launch<64>(a, use_bf16, cus, s);
  if (d_head == 32) return launch<32>(a, use_bf16, cus, s);
  return hipErrorInvalidValue;
}

}  // namespace cfdetr
