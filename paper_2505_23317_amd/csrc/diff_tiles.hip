// Differential attention of many queries, bf16.
//
// A workgroup has 128 queries of one head and frame, a wavefront 32 of them, a query is a lane (S^T = K Q^T,
// O^T = V^T P^T, as in attention.hip).  Both maps of a head are worked out in one pass over the keys, because their
// values are the same: an operand of the values read from LDS feeds a product of each.  Units of 32 keys go
// from global memory straight into LDS, two stages ahead, one barrier a stage.
// Stage u: on the matrix unit the values of unit u - 1 under both maps (16 products at head width 64) and then the
// logits of unit u + 1 (8), between them the exponentials of unit u, in an order that the compiler is not to change.
//
// What it spends its time on: per stage and wavefront 24 products of 32 clocks' pipe and 2048 exponentials, sums and
// roundings, which two wavefronts overlap, and waits: the compiler does not count the loads into LDS and believes the
// query's operands, ordinary loads first used inside the loop, to be on their way there.  Without a list one of the
// loop's two stages hence waits for all loads (vmcnt 7 to 0) in front of its logits, those that it has itself just asked for
// among them; only the other has them two stages ahead.  With a list every entry is such a load with the wait behind it, two
// for the keys and two for the values of each stage at head width 64: 8 frames of 6400 tokens with a third masked take 740 us, without a
// mask 700, cut to the open keys 481.  Two logits and twice the values make 12 d_head operations a key, query and head: 8 frames of
// 6400 tokens, 3 heads of width 64, are 7.5e11 of them in 690 us, 1.09e15 a second, where a large product of matrices
// reaches 1.2e15.
//
// KG = 1: four wavefronts, two workgroups a CU.  KG = 2: eight, where those leave CUs with one workgroup: the even
// and the odd units of keys of the same queries, whose sums and rows (they have the same reference) are added at the end.
// us, KG 1 / 2, heads of width 64, frames of 6784 tokens, 159 tiles: 155 / 137; 228 tiles of 9728 tokens 230 / 213; 255 of 10,880 271 / 256;
// 270 (more than CUs) 404 / 471; 348 551 / 604; 4 frames, 252 tiles 80.7 / 75.4, 300 125 / 145; 12 frames of 300 queries over 3000, 216 tiles 89 / 82.
//
// Values lie in memory row by row.  The second product wants, for a lane's column, eight consecutive keys:
// the transposing LDS read gives four a lane, so no copy of the values by columns is made.
//
// Probabilities are powers of two relative to the reference 0 and not to a running maximum, rounded to bf16 (half
// a step of 2^-8 each, independent between keys and maps) and summed in 32 bits before that.  The rounding is relative to a
// map's product with the values: rows are off by 0.0022 of their size with independent maps, by 0.017 and 0.022 with
// lambda 0.9 and a second map of the first's queries and keys plus 7 and 2 % of noise (1600 keys, heads of width 64).  What
// the rounding leaves off, as a second operand, would be 8 d_head operations more.  A sum outside
// [2^-64, 2^100], or that is no number, and a row that is none, sends its query through a walk with a running
// maximum (redo_rows), and the rest of its tile with it: nothing is asked for ahead there, and 8 frames of 6400 tokens with
// one such query a tile, or nothing but those, take 1,790 to 1,920 us where they take 700, six frames of 400 to 1600 (width 256) 105 and 29.
#include "diff_attention.h"

namespace cfdetr {

namespace {

constexpr int kTileQ = 128;
constexpr int kAhead = 2;   // stages that a unit's loads have ahead of them
// LDS of a workgroup: the stages' keys and values.  Up to 64 KB it is declared with its size, and its addresses are
// constants: 1 % of the time with four wavefronts.
template <int DH, int KG>
constexpr int kStages = (2 * kAhead + 3) * KG * kUnitKeys * 4 * DH;
template <int DH, int KG>
constexpr bool kFixed = kStages<DH, KG> <= 63 * 1024;
constexpr float kSumLow = 0x1p-64f, kSumHigh = 0x1p+100f;

// A row of queries is finished: the difference of its maps, its norm, its type.  Lane l and l ^ 32 hold the columns
// 32 i + 8 r + 4 g on of a query; a swap between them makes runs of eight.  False: not written, asked for or because
// `finite` is and the row's squares are too large for 32 bits or no numbers.
template <int DH>
__device__ __forceinline__ bool finish_rows(const f32x16 (&acc)[2][DH / 16], const float (&l)[2], float lambda, const float* __restrict__ head_g,
                                            float eps, bf16_t* orow, int g, bool write, bool finite) {
  constexpr int W = 2 * DH, MO = W / 32;
  const float i0 = l[0] != 0.f ? 1.0f / l[0] : 0.f, i1 = l[1] != 0.f ? lambda / l[1] : 0.f;
  f32x16 o[MO];
  float sq = 0.f;
#pragma unroll
  for (int i = 0; i < MO; ++i)
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      // (lambda 0 leaves the first map alone, whatever the second holds)
      o[i][r] = acc[0][i][r] * i0;
      if (lambda != 0.f) o[i][r] = fmaf(-acc[1][i][r], i1, o[i][r]);
      sq = fmaf(o[i][r], o[i][r], sq);
    }
  sq = half_sum(sq);
  if (finite && !(sq < INFINITY)) write = false;
  if (head_g) {
    const float n = rsqrtf(sq * (1.0f / W) + eps);
#pragma unroll
    for (int i = 0; i < MO; ++i)
#pragma unroll
      for (int rq = 0; rq < 4; ++rq) {
        const float4 gain = *reinterpret_cast<const float4*>(head_g + 32 * i + 8 * rq + 4 * g);
        o[i][4 * rq] *= n * gain.x;
        o[i][4 * rq + 1] *= n * gain.y;
        o[i][4 * rq + 2] *= n * gain.z;
        o[i][4 * rq + 3] *= n * gain.w;
      }
  }
  typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
#pragma unroll
  for (int i = 0; i < MO; ++i)
#pragma unroll
    for (int rp = 0; rp < 2; ++rp) {
      // columns 8 (2 rp) + 4 g on and 8 (2 rp + 1) + 4 g on -> 8 (2 rp + g) on
      const u32x2 a = __builtin_amdgcn_permlane32_swap(pack_bf16x2(o[i][8 * rp], o[i][8 * rp + 1]), pack_bf16x2(o[i][8 * rp + 4], o[i][8 * rp + 5]), false, false);
      const u32x2 b = __builtin_amdgcn_permlane32_swap(pack_bf16x2(o[i][8 * rp + 2], o[i][8 * rp + 3]), pack_bf16x2(o[i][8 * rp + 6], o[i][8 * rp + 7]), false, false);
      if (write) *reinterpret_cast<uint4*>(orow + 32 * i + 16 * rp + 8 * g) = make_uint4(a[0], b[0], a[1], b[1]);
    }
  return write;
}

// The rare path: a workgroup's queries again, with a running maximum; only those with `again` are written.  A
// function of its own, so that the registers of the other path are not its business.
template <int DH, int THREADS>
__device__ __attribute__((noinline)) void redo_rows(const bf16_t* qrow, const bf16_t* kbase, int k_ld, const bf16_t* vbase, int v_ld,
                                                    const int32_t* list, int nk, float scale2, float lambda, const float* head_g, float eps,
                                                    bf16_t* orow, bool again, unsigned char* smem) {
  constexpr int W = 2 * DH, ROWB = 2 * W, CPR = ROWB / 16, KS = CPR / 4, MO = W / 32, UNIT = kUnitKeys * ROWB;
  const int tid = threadIdx.x, g = (tid & 63) >> 5;   // (wavefronts of the same queries do the same; `again` is set in one)
  unsigned char* const sK = smem;
  unsigned char* const sV = smem + UNIT;
  uint4 qf[2][KS];
#pragma unroll
  for (int m = 0; m < 2; ++m)
#pragma unroll
    for (int c = 0; c < KS; ++c) qf[m][c] = *reinterpret_cast<const uint4*>(qrow + m * DH + (2 * c + g) * 8);
  f32x16 acc[2][MO];
  float m_run[2] = {-INFINITY, -INFINITY}, l_run[2] = {0.f, 0.f};
#pragma unroll
  for (int m = 0; m < 2; ++m)
#pragma unroll
    for (int i = 0; i < MO; ++i)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[m][i][r] = 0.f;
#pragma nounroll
  for (int k0 = 0; k0 < nk; k0 += kUnitKeys) {
    __syncthreads();
    for (int p = tid; p < kUnitKeys * CPR; p += THREADS) {
      const int key = p / CPR, c = p % CPR, at = k0 + key, row = swap_bits_2_3(key);
      uint4 kk = make_uint4(0, 0, 0, 0), vv = kk;
      if (at < nk) {
        const size_t from = list ? list[at] : at;
        kk = *reinterpret_cast<const uint4*>(kbase + from * k_ld + c * 8);
        vv = *reinterpret_cast<const uint4*>(vbase + from * v_ld + c * 8);
      }
      *reinterpret_cast<uint4*>(sK + row * ROWB + key_chunk<bf16_t, ROWB>(row, c) * 16) = kk;
      *reinterpret_cast<uint4*>(sV + row * ROWB + value_piece<bf16_t, ROWB>(row, c) * 16) = vv;
    }
    __syncthreads();
    f32x16 s[2];
    unit_logits<bf16_t, DH>(sK, qf, s);
    unit_weights<bf16_t>(s, nk - k0, scale2, m_run, l_run, acc);
    unit_rows<bf16_t, DH>(sV, s, acc);
  }
  const float l[2] = {half_sum(l_run[0]), half_sum(l_run[1])};
  finish_rows<DH>(acc, l, lambda, head_g, eps, orow, g, again, false);
}

typedef __attribute__((ext_vector_type(4))) short s16x4;
typedef __attribute__((address_space(3))) s16x4* lds4;

// Which frame, head and tile workgroup w has.  w mod 8 is its XCD, with an L2 of its own: every XCD gets an eighth of
// every frame's items, in the order of heads, so that the workgroups of an XCD read the same keys, and the
// longest frames first, so that the last ones are short.
struct Item {
  int frame, head, tile;
};
__device__ __forceinline__ Item item_of(const Frames& fr, const int32_t* __restrict__ kv_len, int B, int heads) {
  const int lane = threadIdx.x & 63, xcd = blockIdx.x & 7;
  int at = blockIdx.x >> 3;
  int first[2], count[2], len[2], before[2] = {0, 0};
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int items = (fr.q[i + 1] - fr.q[i] + kTileQ - 1) / kTileQ * heads;
    xcd_share(items, xcd + 2 * lane + i, first[i], count[i]);
    len[i] = fr.k[i + 1] - fr.k[i];
    if (kv_len != nullptr && 2 * lane + i < B) len[i] = min(len[i], kv_len[2 * lane + i]);
  }
  for (int f = 0; f < B; ++f) {
    const int n0 = __builtin_amdgcn_readlane(len[0], f >> 1), n1 = __builtin_amdgcn_readlane(len[1], f >> 1);
    const int c0 = __builtin_amdgcn_readlane(count[0], f >> 1), c1 = __builtin_amdgcn_readlane(count[1], f >> 1);
    const int n = (f & 1) ? n1 : n0, c = (f & 1) ? c1 : c0;
#pragma unroll
    for (int i = 0; i < 2; ++i)
      if (n > len[i] || (n == len[i] && f < 2 * lane + i)) before[i] += c;
  }
  Item item{-1, 0, 0};
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const uint64_t in = __ballot(before[i] <= at && at < before[i] + count[i]);
    if (in != 0) {
      const int l = __ffsll((unsigned long long)in) - 1;
      const int n = __builtin_amdgcn_readlane(first[i] - before[i], l) + at;
      const int tiles = (__builtin_amdgcn_readlane(fr.q[i + 1] - fr.q[i], l) + kTileQ - 1) / kTileQ;
      item.frame = 2 * l + i;
      item.head = n / tiles;
      item.tile = n - item.head * tiles;
    }
  }
  return item;
}

// This lane's number, counted anew: the compiler cannot carry it, or what is made of it, through the loop, which has no
// registers for it.
__device__ __forceinline__ int lane_again() {
  int l;
  asm volatile("v_mbcnt_lo_u32_b32 %0, -1, 0\n\tv_mbcnt_hi_u32_b32 %0, -1, %0" : "=v"(l));
  return l;
}

template <int DH, bool LIST, bool SCALED, int KG>
__global__ __launch_bounds__(256 * KG, 2) void diff_tiles_kernel(DiffAttentionArgs a) {
  constexpr int W = 2 * DH, ROWB = 2 * W, CPR = ROWB / 16;
  constexpr int KS = DH / 16, MO = W / 32;
  constexpr int UNIT = kUnitKeys * ROWB, NI = UNIT / 4096, RPI = 1024 / ROWB;   // a wavefront's loads of a unit, rows of one
  constexpr int NOP = 2 * MO;                       // operands of the values of a unit
  constexpr int NPV = 2 * NOP, NQK = 2 * KS;        // products of a stage
  constexpr int AHEAD = kAhead, kKeySlots = AHEAD + 1, kValueSlots = AHEAD + 2;
  constexpr int STAGE = KG * kUnitKeys, BYTES = KG * UNIT;   // keys of a stage, and LDS of those (and of their values)
  extern __shared__ __attribute__((aligned(1024))) unsigned char sized[];
  __shared__ __attribute__((aligned(1024))) unsigned char fixed[kFixed<DH, KG> ? kStages<DH, KG> : 16];
  unsigned char* const smem = kFixed<DH, KG> ? fixed : sized;
  __shared__ float s_l[KG == 2 ? 2 : 1][4][32];

  const Frames fr = frames_of(a.cu_q, a.cu_k, a.B, a.n_q, a.n_k);
  if (fr.bad) {
    if (blockIdx.x == 0 && threadIdx.x == 0) *a.err_flag = 1;
    return;
  }
  const Item item = item_of(fr, a.kv_len, a.B, a.heads);
  if (item.frame < 0) return;
  const int tid = threadIdx.x, lane = tid & 63, l32 = lane & 31, g = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6) & 3, odd = KG == 2 ? __builtin_amdgcn_readfirstlane(tid >> 8) : 0;
  const int frame = __builtin_amdgcn_readfirstlane(item.frame), head = __builtin_amdgcn_readfirstlane(item.head);
  const int q0 = of_frame(fr.q, frame), nq = behind_frame(fr.q, frame) - q0;
  const int k0 = of_frame(fr.k, frame), nk_all = behind_frame(fr.k, frame) - k0;
  const int nk = a.kv_len ? min(nk_all, a.kv_len[frame]) : nk_all;
  const int q_first = __builtin_amdgcn_readfirstlane(item.tile) * kTileQ + wave * 32, q_local = q_first + l32;
  const bf16_t* qrow = static_cast<const bf16_t*>(a.q) + (size_t)(q0 + min(q_local, nq - 1)) * a.q_ld + head * W;
  const bf16_t* const kbase = static_cast<const bf16_t*>(a.k) + (size_t)k0 * a.k_ld + head * W;
  const bf16_t* const vbase = static_cast<const bf16_t*>(a.v) + (size_t)k0 * a.v_ld + head * W;
  const int32_t* const list = LIST ? a.key_list + k0 : nullptr;
  const float lambda = a.lambda[head];
  const int n = (nk + STAGE - 1) / STAGE;   // stages
  if (n == 0) {
    bf16_t* const orow = static_cast<bf16_t*>(a.out) + (size_t)(q0 + q_local) * a.out_ld + head * W;
    if (q_local < nq)
      for (int c = 2 * odd + g; c < CPR; c += 2 * KG) *reinterpret_cast<uint4*>(orow + 8 * c) = make_uint4(0, 0, 0, 0);
    return;
  }
  const int ragged = nk & (STAGE - 1);   // keys of a last stage that is not full

  bf16x8 qf[2][KS];
#pragma unroll
  for (int m = 0; m < 2; ++m)
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) qf[m][ks] = *reinterpret_cast<const bf16x8*>(qrow + m * DH + ks * 16 + g * 8);

  // Loads: piece `lane` of load j lies in LDS row (wave NI + j) RPI + lane / CPR; which key and chunk that is, is the order of
  // the rows and chunks in LDS.  Two loads of a wavefront are four rows apart: eight keys, with the same chunks of
  // the values.  The offsets of full units are kept, what else is asked for is worked out where it is.
  const uint32_t lds0 = (uint32_t)(uintptr_t)smem;
  auto row_of = [&](int l, int j) { return (wave * NI + j) * RPI + l / CPR; };
  auto column = [&](int l, int j, auto values) {
    const int rho = row_of(l, j), c = l % CPR;
    return (uint32_t)(decltype(values)::value ? value_piece<bf16_t, ROWB>(rho, c) : key_piece<bf16_t, ROWB>(rho, c)) * 16;
  };
  const auto of_keys = std::integral_constant<bool, false>{};
  const auto of_values = std::integral_constant<bool, true>{};
  static_assert(NI == 1 || (NI == 2 && RPI == 4), "the second load's keys are eight behind the first's");
  const uint32_t k_off = (uint32_t)swap_bits_2_3(row_of(lane, 0)) * (uint32_t)(a.k_ld * 2) + column(lane, 0, of_keys);
  const uint32_t v_off = (uint32_t)swap_bits_2_3(row_of(lane, 0)) * (uint32_t)(a.v_ld * 2) + column(lane, 0, of_values);
  auto load = [&](const bf16_t* base, int ld, auto values, int stage, uint32_t to) {
    to += odd * UNIT + wave * (NI * 1024);
    const int first = (KG * stage + odd) * kUnitKeys;
    if (!LIST && first + kUnitKeys <= nk) {
      const bf16_t* const from = base + (size_t)first * ld;
      dma16(from, decltype(values)::value ? v_off : k_off, to);
      if constexpr (NI == 2) {
        // eight keys on; the keys' chunks of rows four on: bit 2 of their number turned.  Four wavefronts have the registers to
        // keep that, 1.5 % of their time.
        const uint32_t off = decltype(values)::value ? v_off : k_off + 64 - (uint32_t)(((KG == 1 ? lane : lane_again()) & 4) << 5);
        if constexpr (KG == 1) dma16(from, off + (uint32_t)(16 * ld), to + 1024);
        else dma16(from + (size_t)8 * ld, off, to + 1024);
      }
    } else {
      // rows behind the last key are the last key's, and are not used
      const int l = lane_again();
#pragma unroll
      for (int j = 0; j < NI; ++j) {
        const int at = min(first + swap_bits_2_3(row_of(l, j)), nk - 1);
        const size_t row = LIST ? list[at] : at;
        dma16(reinterpret_cast<const char*>(base) + row * (size_t)ld * 2 + column(l, j, values), to + j * 1024);
      }
    }
  };
  auto slot = [](int u, int slots) { return (uint32_t)(u % slots) * BYTES; };
  constexpr uint32_t VALUES = kKeySlots * BYTES;
  auto load_k = [&](int u, uint32_t at) { load(kbase, a.k_ld, of_keys, u, lds0 + at); };
  auto load_v = [&](int u, uint32_t at) { load(vbase, a.v_ld, of_values, u, lds0 + VALUES + at); };

  // Operands: row l32 of the keys, chunk 2 ks + g of a map; for the values the transposing read's pieces.
  const uint32_t k_at = odd * UNIT + l32 * ROWB + key_chunk<bf16_t, ROWB>(l32, g) * 16;
  const int v_row = 4 * g + ((lane & 15) >> 2);   // of keys 8 g on; those of 8 g + 4 on are 8 rows behind
  const uint32_t v_at = VALUES + odd * UNIT + v_row * ROWB + value_block<bf16_t, ROWB>(v_row, 0) * 64 + ((lane >> 4) & 1) * 32 + (lane & 3) * 8;
  auto read_k = [&](uint32_t at, int kk) {   // operand kk = KS map + ks (chunks and blocks are moved by bits: an exclusive or)
    return *reinterpret_cast<const bf16x8*>(smem + ((at + k_at) ^ (uint32_t)(2 * kk * 16)));
  };
  auto read_v = [&](uint32_t at, int p) {   // operand p = 2 block + half of the unit's keys
    union {
      s16x4 half[2];
      bf16x8 whole;
    } v;
    const uint32_t from = ((at + v_at) ^ (uint32_t)((p >> 1) * 64)) + (p & 1) * 16 * ROWB;
    v.half[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)(smem + from));
    v.half[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)(smem + from + 8 * ROWB));
    return v.whole;
  };

  f32x16 acc[2][MO];
  float l_run[2] = {0.f, 0.f};
#pragma unroll
  for (int m = 0; m < 2; ++m)
#pragma unroll
    for (int i = 0; i < MO; ++i)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[m][i][r] = 0.f;
  f32x16 sA[2], sB[2];
  bf16x8 pA[2][2], pB[2][2];
  bf16x8 vb[3], kb[3];

  auto qk = [&](f32x16(&s)[2], const bf16x8& k, int kk) {
    const int m = kk / KS, ks = kk % KS;
    if (ks == 0) {
      f32x16 z;
#pragma unroll
      for (int r = 0; r < 16; ++r) z[r] = 0.f;
      s[m] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k, qf[m][ks], z, 0, 0, 0);
    } else {
      s[m] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k, qf[m][ks], s[m], 0, 0, 0);
    }
  };
  auto mask = [&](f32x16(&s)[2]) {
    const int g = lane_again() >> 5, left = ragged - odd * kUnitKeys;   // (an odd unit may have none)
#pragma unroll
    for (int m = 0; m < 2; ++m)
#pragma unroll
      for (int r = 0; r < 16; ++r)
        if (16 * (r >> 3) + 8 * g + (r & 7) >= left) s[m][r] = -INFINITY;
  };
  // In front of stage u: the keys of unit u + 1 and the values of unit u, asked for AHEAD stages before, are in LDS, everyone is
  // past stage u - 1, and the slots that that has left are filled.  What may still be on its way is what the
  // stages between have asked for, in the last ones less.
  auto begin = [&](int u) {
    const int left = n - (u + AHEAD);
    auto wait = [](auto units) {
      constexpr int kUnits = decltype(units)::value > 0 ? decltype(units)::value : 0;
      asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" : : "n"(kUnits * NI) : "memory");
    };
    constexpr int FULL = 2 * (AHEAD - 1);
    if (left > 0) wait(std::integral_constant<int, FULL>{});
    else if (left == 0) wait(std::integral_constant<int, FULL - 1>{});
    else if (left == -1) wait(std::integral_constant<int, FULL - 3>{});
    else if (left == -2) wait(std::integral_constant<int, FULL - 5>{});
    else if (left == -3) wait(std::integral_constant<int, FULL - 7>{});
    else wait(std::integral_constant<int, 0>{});
    if (u + AHEAD + 1 < n) load_k(u + AHEAD + 1, slot(u, kKeySlots));
    if (u + AHEAD < n) load_v(u + AHEAD, slot(u + AHEAD, kValueSlots));
  };
  auto stage = [&](f32x16(&s)[2], f32x16(&sn)[2], bf16x8(&pc)[2][2], bf16x8(&pp)[2][2], int u, auto more_tag) {
    constexpr bool kMore = decltype(more_tag)::value;   // there is a unit u + 1
    constexpr int NM = NPV + (kMore ? NQK : 0), PAIRS = 16;
    const uint32_t v_prev = slot(u + kValueSlots - 1, kValueSlots), v_this = slot(u, kValueSlots), k_next = slot(u + 1, kKeySlots);
    uint32_t w[2][8];
    float e0 = 0.f, e1 = 0.f, sum[2] = {0.f, 0.f};
#pragma unroll
    for (int m = 0; m < NM; ++m) {
      if (m < NPV) {
        const int p = m / 2, i = p >> 1, t = p & 1;
        if (m % 2 == 0) {
          if (p + 2 < NOP) vb[(p + 2) % 3] = read_v(v_prev, p + 2);
          else if (kMore) kb[p + 2 - NOP] = read_k(k_next, p + 2 - NOP);
        }
        acc[m & 1][i] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vb[p % 3], pp[m & 1][t], acc[m & 1][i], 0, 0, 0);
      } else {
        const int kk = m - NPV;
        if (kk + 2 < NQK) kb[(kk + 2) % 3] = read_k(k_next, kk + 2);
        else vb[kk + 2 - NQK] = read_v(v_this, kk + 2 - NQK);
        qk(sn, kb[kk % 3], kk);
      }
#pragma unroll
      for (int x = m * PAIRS / NM; x < (m + 1) * PAIRS / NM; ++x) {
        const int xm = x / 8, e = x % 8;
        // sum and rounding of the pair before: its exponentials have left the transcendental pipe by now
        if (x > 0) {
          const int ym = (x - 1) / 8, ye = (x - 1) % 8;
          sum[ym] = ye == 0 ? e0 + e1 : sum[ym] + (e0 + e1);
          w[ym][ye] = pack_bf16x2(e0, e1);
          asm volatile("" : "+v"(w[ym][ye]), "+v"(sum[ym]));
        }
        e0 = __builtin_amdgcn_exp2f(SCALED ? s[xm][2 * e] * a.scale2 : s[xm][2 * e]);
        e1 = __builtin_amdgcn_exp2f(SCALED ? s[xm][2 * e + 1] * a.scale2 : s[xm][2 * e + 1]);
        asm volatile("" : "+v"(e0), "+v"(e1));
      }
      __builtin_amdgcn_sched_barrier(0);
    }
    if constexpr (!kMore) {
      vb[0] = read_v(v_this, 0);
      vb[1] = read_v(v_this, 1);
    }
    sum[1] += e0 + e1;
    w[1][7] = pack_bf16x2(e0, e1);
#pragma unroll
    for (int m = 0; m < 2; ++m) {
      l_run[m] += sum[m];
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        uint4 packed = make_uint4(w[m][4 * t], w[m][4 * t + 1], w[m][4 * t + 2], w[m][4 * t + 3]);
        pc[m][t] = *reinterpret_cast<bf16x8*>(&packed);
      }
    }
  };
  const auto yes = std::integral_constant<bool, true>{};
  const auto no = std::integral_constant<bool, false>{};

  // in the order in which they are waited for
  load_k(0, slot(0, kKeySlots));
#pragma nounroll
  for (int u = 0; u < AHEAD && u < n; ++u) {
    if (u + 1 < n) load_k(u + 1, slot(u + 1, kKeySlots));
    load_v(u, slot(u, kValueSlots));
  }
  // In front of the first unit: values of a unit before it, all 0, met with probabilities 0.
  for (int p = tid; p < BYTES / 16; p += 256 * KG) *reinterpret_cast<uint4*>(smem + VALUES + slot(kValueSlots - 1, kValueSlots) + p * 16) = make_uint4(0, 0, 0, 0);
#pragma unroll
  for (int e = 0; e < 8; ++e) vb[0][e] = vb[1][e] = pA[0][0][e] = pA[0][1][e] = pA[1][0][e] = pA[1][1][e] = (__bf16)0.f;
  if (n >= AHEAD) asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" : : "n"((2 * AHEAD - 1) * NI) : "memory");
  else asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" : : : "memory");
  // The last unit: keys behind the frame's have no weight, and their values are cleared (0 times what they are copies of
  // may be no number).
  auto last = [&](f32x16(&s)[2]) {
    if (ragged == 0) return;
    mask(s);
    const uint32_t at = VALUES + slot(n - 1, kValueSlots);
    for (int p = (4 * odd + wave) * 64 + lane_again(); p < (STAGE - ragged) * CPR; p += 256 * KG) {
      const int key = ragged + p / CPR;
      *reinterpret_cast<uint4*>(smem + at + (key & kUnitKeys) / kUnitKeys * UNIT + swap_bits_2_3(key & (kUnitKeys - 1)) * ROWB + p % CPR * 16) = make_uint4(0, 0, 0, 0);
    }
    __syncthreads();
  };
  auto final_pv = [&](bf16x8(&p)[2][2]) {
    const uint32_t v_last = slot(n - 1, kValueSlots);
#pragma unroll
    for (int m = 0; m < NPV; ++m) {
      const int q = m / 2, i = q >> 1, t = q & 1;
      if (m % 2 == 0 && q + 2 < NOP) vb[(q + 2) % 3] = read_v(v_last, q + 2);
      acc[m & 1][i] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vb[q % 3], p[m & 1][t], acc[m & 1][i], 0, 0, 0);
    }
  };
  // An even number of units has one in front of the pairs, so that the last one is always where the loop leaves it.
  int u = 0;
  if (n & 1) {
#pragma unroll
    for (int kk = 0; kk < NQK; ++kk) qk(sA, read_k(slot(0, kKeySlots), kk), kk);
#pragma unroll
    for (int m = 0; m < 2; ++m)
#pragma unroll
      for (int t = 0; t < 2; ++t) pB[m][t] = pA[m][t];
  } else {
#pragma unroll
    for (int kk = 0; kk < NQK; ++kk) qk(sB, read_k(slot(0, kKeySlots), kk), kk);
    begin(0);
    stage(sB, sA, pB, pA, 0, yes);
    u = 1;
  }
  for (; u + 1 < n; u += 2) {
    begin(u);
    stage(sA, sB, pA, pB, u, yes);
    begin(u + 1);
    stage(sB, sA, pB, pA, u + 1, yes);
  }
  begin(u);
  last(sA);
  stage(sA, sB, pA, pB, u, no);
  final_pv(pA);

  // The odd units' sums and rows to the wavefront with the even ones, one map after the other; that one finishes its queries' rows
  // (where they lie is worked out again: the loop has no registers for it).
  const int lane_end = lane_again();
  float l[2] = {half_sum(l_run[0]), half_sum(l_run[1])};
  if constexpr (KG == 2) {
    if (odd && lane_end < 32) {
      s_l[0][wave][lane_end] = l[0];
      s_l[1][wave][lane_end] = l[1];
    }
    float4* const rows = reinterpret_cast<float4*>(smem) + wave * (MO * 4 * 64) + lane_end;
#pragma unroll
    for (int m = 0; m < 2; ++m) {
      __syncthreads();
      if (odd) {
#pragma unroll
        for (int i = 0; i < MO; ++i)
#pragma unroll
          for (int rq = 0; rq < 4; ++rq)
            rows[(4 * i + rq) * 64] = make_float4(acc[m][i][4 * rq], acc[m][i][4 * rq + 1], acc[m][i][4 * rq + 2], acc[m][i][4 * rq + 3]);
      }
      __syncthreads();
      if (!odd) {
#pragma unroll
        for (int i = 0; i < MO; ++i)
#pragma unroll
          for (int rq = 0; rq < 4; ++rq) {
            const float4 v = rows[(4 * i + rq) * 64];
            acc[m][i][4 * rq] += v.x;
            acc[m][i][4 * rq + 1] += v.y;
            acc[m][i][4 * rq + 2] += v.z;
            acc[m][i][4 * rq + 3] += v.w;
          }
        l[m] += s_l[m][wave][lane_end & 31];
      }
    }
  }
  const int q_again = q_first + (lane_end & 31);
  const bool mine = !odd && q_again < nq;
  const size_t q_row = (size_t)(q0 + min(q_again, nq - 1));
  qrow = static_cast<const bf16_t*>(a.q) + q_row * a.q_ld + head * W;
  bf16_t* const orow = static_cast<bf16_t*>(a.out) + q_row * a.out_ld + head * W;
  const bool in_range = l[0] >= kSumLow && l[0] <= kSumHigh && l[1] >= kSumLow && l[1] <= kSumHigh;
  bool again = false;
  if (!odd) again = !finish_rows<DH>(acc, l, lambda, a.head_g, a.eps, orow, lane_end >> 5, mine && in_range, true) && mine;
  if (__syncthreads_or(again))
    redo_rows<DH, 256 * KG>(qrow, kbase, a.k_ld, vbase, a.v_ld, list, nk, a.scale2, lambda, a.head_g, a.eps, orow, again, smem);
}

template <int DH, bool LIST, bool SCALED, int KG>
hipError_t go(const DiffAttentionArgs& a, hipStream_t s) {
  constexpr int LDS = kFixed<DH, KG> ? 0 : kStages<DH, KG>;
  static_assert(KG == 1 || kStages<DH, KG> >= 4 * 32 * 2 * DH * 4, "the odd units' rows of a map");
  static DeviceOnce once;
  if (LDS > 0)
    if (hipError_t e = allow_lds(diff_tiles_kernel<DH, LIST, SCALED, KG>, LDS, &once); e != hipSuccess) return e;
  const int64_t items = ((int64_t)a.n_q / kTileQ + a.B) * a.heads;
  hipLaunchKernelGGL((diff_tiles_kernel<DH, LIST, SCALED, KG>), dim3((unsigned)(8 * (items / 8 + a.B + 1))), dim3(256 * KG), LDS, s, a);
  return hipGetLastError();
}
template <int DH, int KG>
hipError_t go(const DiffAttentionArgs& a, hipStream_t s) {
  const bool scaled = a.scale2 != 1.0f;
  if (a.key_list) return scaled ? go<DH, true, true, KG>(a, s) : go<DH, true, false, KG>(a, s);
  return scaled ? go<DH, false, true, KG>(a, s) : go<DH, false, false, KG>(a, s);
}

}  // namespace

hipError_t launch_diff_tiles(const DiffAttentionArgs& a, int d_head, hipStream_t s) {
  if (d_head == 64) return a.wide ? go<64, 2>(a, s) : go<64, 1>(a, s);
  if (d_head == 32) return a.wide ? go<32, 2>(a, s) : go<32, 1>(a, s);
  return hipErrorInvalidValue;
}

}  // namespace cfdetr
