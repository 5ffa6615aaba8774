// Differential attention of many queries, bf16.
//
// A workgroup has 128 queries of one head and frame, a wavefront 32 of them, a query is a lane (S^T = K Q^T,
// O^T = V^T P^T, as in attention.hip).  Both maps of a head are worked out in one pass over the keys, because their
// values are the same: an operand of the values read from LDS feeds a product of each.  Units of 32 keys go
// from global memory straight into LDS, keys two stages and values one stage ahead of their use, one barrier a stage.
// Stage u: on the matrix unit the values of unit u - 1 under both maps (16 products at head width 64) and then the
// logits of unit u + 1 (8), between them the exponentials of unit u, in an order that the compiler is not to change.
//
// Values lie in memory row by row.  The second product wants, for a lane's column, eight consecutive keys:
// the transposing LDS read gives four a lane, so no copy of the values by columns is made.
//
// Probabilities are powers of two relative to the reference 0 and not to a running maximum, rounded to bf16 (half
// a step of 2^-8 each, independent between keys) and summed in 32 bits before that.  A sum outside
// [2^-64, 2^100], or that is no number, sends its query through a walk with a running maximum (redo_rows).
#include "diff_attention.h"

namespace cfdetr {

namespace {

constexpr int kTileQ = 128;
constexpr int kKeySlots = 3, kValueSlots = 4;
constexpr float kSumLow = 0x1p-64f, kSumHigh = 0x1p+100f;

// A row of queries is finished: the difference of its maps, its norm, its type.  Lane l and l ^ 32 hold the columns
// 32 i + 8 r + 4 g on of a query; a swap between them makes runs of eight.
template <int DH>
__device__ __forceinline__ void finish_rows(const f32x16 (&acc)[2][DH / 16], const float (&l)[2], float lambda, const float* __restrict__ head_g,
                                            float eps, bf16_t* orow, bool write) {
  constexpr int W = 2 * DH, MO = W / 32;
  const int g = (threadIdx.x & 63) >> 5;
  const float i0 = l[0] != 0.f ? 1.0f / l[0] : 0.f, i1 = l[1] != 0.f ? lambda / l[1] : 0.f;
  f32x16 o[MO];
  float sq = 0.f;
#pragma unroll
  for (int i = 0; i < MO; ++i)
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      // (lambda 0 leaves the first map alone, also where a value is infinite)
      o[i][r] = acc[0][i][r] * i0;
      if (lambda != 0.f) o[i][r] = fmaf(-acc[1][i][r], i1, o[i][r]);
      sq = fmaf(o[i][r], o[i][r], sq);
    }
  if (head_g) {
    const float n = rsqrtf(half_sum(sq) * (1.0f / W) + eps);
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
}

// The rare path: a workgroup's queries again, with a running maximum; only those with `again` are written.  A
// function of its own, so that the registers of the other path are not its business.
template <int DH>
__device__ __attribute__((noinline)) void redo_rows(const bf16_t* qrow, const bf16_t* kbase, int k_ld, const bf16_t* vbase, int v_ld,
                                                    const int32_t* list, int nk, float scale2, float lambda, const float* head_g, float eps,
                                                    bf16_t* orow, bool again, unsigned char* smem) {
  constexpr int W = 2 * DH, ROWB = 2 * W, CPR = ROWB / 16, KS = CPR / 4, MO = W / 32, UNIT = kUnitKeys * ROWB;
  const int tid = threadIdx.x, g = (tid & 63) >> 5;
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
    for (int p = tid; p < kUnitKeys * CPR; p += kThreads) {
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
  finish_rows<DH>(acc, l, lambda, head_g, eps, orow, again);
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
    first[i] = (int)((int64_t)items * xcd / 8);
    count[i] = (int)((int64_t)items * (xcd + 1) / 8) - first[i];
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

template <int DH, bool LIST, bool SCALED>
__global__ __launch_bounds__(kThreads, 2) void diff_tiles_kernel(DiffAttentionArgs a) {
  constexpr int W = 2 * DH, ROWB = 2 * W, CPR = ROWB / 16;
  constexpr int KS = DH / 16, MO = W / 32;
  constexpr int UNIT = kUnitKeys * ROWB, NI = UNIT / 4096, RPI = 1024 / ROWB;   // a wavefront's loads of a unit, rows of one
  constexpr int NOP = 2 * MO;                       // operands of the values of a unit
  constexpr int NPV = 2 * NOP, NQK = 2 * KS;        // products of a stage
  __shared__ __attribute__((aligned(1024))) unsigned char smem[(kKeySlots + kValueSlots) * UNIT];

  const Frames fr = frames_of(a.cu_q, a.cu_k, a.B, a.n_q, a.n_k);
  if (fr.bad) {
    if (blockIdx.x == 0 && threadIdx.x == 0) *a.err_flag = 1;
    return;
  }
  const Item item = item_of(fr, a.kv_len, a.B, a.heads);
  if (item.frame < 0) return;
  const int tid = threadIdx.x, lane = tid & 63, l32 = lane & 31, g = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int frame = __builtin_amdgcn_readfirstlane(item.frame), head = __builtin_amdgcn_readfirstlane(item.head);
  const int q0 = of_frame(fr.q, frame), nq = behind_frame(fr.q, frame) - q0;
  const int k0 = of_frame(fr.k, frame), nk_all = behind_frame(fr.k, frame) - k0;
  const int nk = a.kv_len ? min(nk_all, a.kv_len[frame]) : nk_all;
  const int q_local = __builtin_amdgcn_readfirstlane(item.tile) * kTileQ + wave * 32 + l32;
  const bool mine = q_local < nq;
  const size_t q_row = (size_t)(q0 + min(q_local, nq - 1));
  const bf16_t* const qrow = static_cast<const bf16_t*>(a.q) + q_row * a.q_ld + head * W;
  bf16_t* const orow = static_cast<bf16_t*>(a.out) + q_row * a.out_ld + head * W;
  const bf16_t* const kbase = static_cast<const bf16_t*>(a.k) + (size_t)k0 * a.k_ld + head * W;
  const bf16_t* const vbase = static_cast<const bf16_t*>(a.v) + (size_t)k0 * a.v_ld + head * W;
  const int32_t* const list = LIST ? a.key_list + k0 : nullptr;
  const float lambda = a.lambda[head];
  const int n = (nk + kUnitKeys - 1) / kUnitKeys;
  if (n == 0) {
    if (mine)
      for (int c = g; c < CPR; c += 2) *reinterpret_cast<uint4*>(orow + 8 * c) = make_uint4(0, 0, 0, 0);
    return;
  }
  const int ragged = nk & (kUnitKeys - 1);   // keys of a last unit that is not full

  bf16x8 qf[2][KS];
#pragma unroll
  for (int m = 0; m < 2; ++m)
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) qf[m][ks] = *reinterpret_cast<const bf16x8*>(qrow + m * DH + ks * 16 + g * 8);

  // Loads: piece `lane` of instruction j of this wavefront lies in LDS row (wave NI + j) RPI + lane / CPR; which key and
  // chunk that is, is the order of the rows and chunks in LDS.
  const uint32_t lds0 = (uint32_t)(uintptr_t)smem;
  int key[NI];
  uint32_t k_col[NI], v_col[NI];
#pragma unroll
  for (int j = 0; j < NI; ++j) {
    const int rho = (wave * NI + j) * RPI + lane / CPR, c = lane % CPR;
    key[j] = swap_bits_2_3(rho);
    k_col[j] = key_piece<bf16_t, ROWB>(rho, c) * 16;
    v_col[j] = value_piece<bf16_t, ROWB>(rho, c) * 16;
  }
  auto load = [&](const bf16_t* base, int ld, const uint32_t(&col)[NI], int u, uint32_t to) {
    to += wave * (NI * 1024);
    if constexpr (LIST) {
#pragma unroll
      for (int j = 0; j < NI; ++j) {
        const size_t row = list[min(u * kUnitKeys + key[j], nk - 1)];
        dma16(reinterpret_cast<const char*>(base) + row * (size_t)ld * 2 + col[j], to + j * 1024);
      }
    } else {
      const bf16_t* const from = base + (size_t)(u * kUnitKeys) * ld;
      const int last = nk - 1 - u * kUnitKeys;   // (rows behind the last key are the last key's, and are not used)
      if (last >= kUnitKeys - 1) {
#pragma unroll
        for (int j = 0; j < NI; ++j) dma16(from, (uint32_t)key[j] * (uint32_t)(ld * 2) + col[j], to + j * 1024);
      } else {
#pragma unroll
        for (int j = 0; j < NI; ++j) dma16(from, (uint32_t)min(key[j], last) * (uint32_t)(ld * 2) + col[j], to + j * 1024);
      }
    }
  };
  auto slot = [](int u, int slots) { return (uint32_t)(u % slots) * UNIT; };
  constexpr uint32_t VALUES = kKeySlots * UNIT;
  auto load_k = [&](int u, uint32_t at) { load(kbase, a.k_ld, k_col, u, lds0 + at); };
  auto load_v = [&](int u, uint32_t at) { load(vbase, a.v_ld, v_col, u, lds0 + VALUES + at); };

  // Operands: row l32 of the keys, chunk 2 ks + g of a map; for the values the transposing read's pieces.
  const uint32_t k_at = l32 * ROWB + key_chunk<bf16_t, ROWB>(l32, g) * 16;
  const int v_row = 4 * g + ((lane & 15) >> 2);   // of keys 8 g on; those of 8 g + 4 on are 8 rows behind
  const uint32_t v_at = VALUES + v_row * ROWB + value_block<bf16_t, ROWB>(v_row, 0) * 64 + ((lane >> 4) & 1) * 32 + (lane & 3) * 8;
  auto read_k = [&](uint32_t at, int kk) {   // operand kk = 2 ks + map (chunks and blocks are moved by bits: an exclusive or)
    return *reinterpret_cast<const bf16x8*>(smem + ((at + k_at) ^ (uint32_t)(((kk & 1) * 2 * KS + 2 * (kk >> 1)) * 16)));
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
    const int m = kk & 1, ks = kk >> 1;
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
#pragma unroll
    for (int m = 0; m < 2; ++m)
#pragma unroll
      for (int r = 0; r < 16; ++r)
        if (16 * (r >> 3) + 8 * g + (r & 7) >= ragged) s[m][r] = -INFINITY;
  };
  // In front of stage u: its keys' successors and its values are in LDS, everyone is past stage u - 1, and
  // the slots that that has left are filled.
  auto begin = [&](int u) {
    if (u + 2 < n) asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" : : "n"(2 * NI) : "memory");
    else asm volatile("s_waitcnt vmcnt(0)\n\ts_barrier" : : : "memory");
    if (u + 3 < n) load_k(u + 3, slot(u, kKeySlots));
    if (u + 2 < n) load_v(u + 2, slot(u + 2, kValueSlots));
  };
  auto stage = [&](f32x16(&s)[2], f32x16(&sn)[2], bf16x8(&pc)[2][2], bf16x8(&pp)[2][2], int u, auto more_tag) {
    constexpr bool kMore = decltype(more_tag)::value;   // there is a unit u + 1
    constexpr int NM = NPV + (kMore ? NQK : 0), PAIRS = 16;
    const uint32_t v_prev = slot(u - 1 + kValueSlots, kValueSlots), v_this = slot(u, kValueSlots), k_next = slot(u + 1, kKeySlots);
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

  load_k(0, slot(0, kKeySlots));
  load_v(0, slot(0, kValueSlots));
  if (n > 1) {
    load_k(1, slot(1, kKeySlots));
    load_v(1, slot(1, kValueSlots));
  }
  if (n > 2) load_k(2, slot(2, kKeySlots));
  // In front of the first unit: values of a unit before it, all 0, met with probabilities 0.
  for (int p = tid; p < UNIT / 16; p += kThreads) *reinterpret_cast<uint4*>(smem + VALUES + slot(kValueSlots - 1, kValueSlots) + p * 16) = make_uint4(0, 0, 0, 0);
#pragma unroll
  for (int e = 0; e < 8; ++e) vb[0][e] = vb[1][e] = pA[0][0][e] = pA[0][1][e] = pA[1][0][e] = pA[1][1][e] = (__bf16)0.f;
  asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" : : : "memory");
  // The last unit: keys behind the frame's have no weight, and their values are cleared (0 times what they are copies of
  // may be no number).
  auto last = [&](f32x16(&s)[2]) {
    if (ragged == 0) return;
    mask(s);
    const uint32_t at = VALUES + slot(n - 1, kValueSlots);
    for (int p = tid; p < (kUnitKeys - ragged) * CPR; p += kThreads)
      *reinterpret_cast<uint4*>(smem + at + swap_bits_2_3(ragged + p / CPR) * ROWB + p % CPR * 16) = make_uint4(0, 0, 0, 0);
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

  const float l[2] = {half_sum(l_run[0]), half_sum(l_run[1])};
  const bool again = !(l[0] >= kSumLow && l[0] <= kSumHigh && l[1] >= kSumLow && l[1] <= kSumHigh);
  finish_rows<DH>(acc, l, lambda, a.head_g, a.eps, orow, mine && !again);
  if (__syncthreads_or(mine && again))
    redo_rows<DH>(qrow, kbase, a.k_ld, vbase, a.v_ld, list, nk, a.scale2, lambda, a.head_g, a.eps, orow, mine && again, smem);
}

template <int DH>
hipError_t go(const DiffAttentionArgs& a, hipStream_t s) {
  const int64_t items = ((int64_t)a.n_q / kTileQ + a.B) * a.heads;
  const dim3 grid((unsigned)(8 * (items / 8 + a.B + 1)));
  const bool scaled = a.scale2 != 1.0f;
  if (a.key_list && scaled) hipLaunchKernelGGL((diff_tiles_kernel<DH, true, true>), grid, dim3(kThreads), 0, s, a);
  else if (a.key_list) hipLaunchKernelGGL((diff_tiles_kernel<DH, true, false>), grid, dim3(kThreads), 0, s, a);
  else if (scaled) hipLaunchKernelGGL((diff_tiles_kernel<DH, false, true>), grid, dim3(kThreads), 0, s, a);
  else hipLaunchKernelGGL((diff_tiles_kernel<DH, false, false>), grid, dim3(kThreads), 0, s, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_diff_tiles(const DiffAttentionArgs& a, int d_head, hipStream_t s) {
  if (d_head == 64) return go<64>(a, s);
  if (d_head == 32) return go<32>(a, s);
  return hipErrorInvalidValue;
}

}  // namespace cfdetr
