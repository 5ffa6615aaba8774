// Differential attention (operator of a differential encoder layer) over variable-length sequences.
//
// Head h has two query / key heads of width dh (2h and 2h + 1 of the rows) and values of width 2 dh:
//   A_m = softmax over the frame's keys of scale q_m k_m^T, m = 1, 2;   o = (A_1 - lambda_h A_2) v
// and, with a gain, o <- o / sqrt(mean(o^2) + eps) * gain.  A frame without keys gives rows of zeros.
#include <algorithm>
#include <type_traits>

#include "diff_attention.h"

namespace cfdetr {

namespace {

constexpr int kTileQ = 32;      // queries of a workgroup (a lane each)
constexpr int kMostSplits = 128;

// ---- few queries, or fp32 ----------------------------------------------------------------
// A workgroup has 32 queries of one head and frame and one run of its keys.  Its NW wavefronts take
// units of 32 keys in turn, each with a running maximum and sum of both maps, through LDS of its own, so that
// there is no barrier before the end: a unit's keys are asked for as soon as the logits of the unit before have been
// taken, its values behind that unit's.  (The compiler does not count the loads into LDS and believes the query's operands,
// ordinary loads first used inside the loop, to be on their way there: the last product of a unit's logits waits for all
// loads, the unit's values among them, before a weight is worked out.)  At the end the wavefronts' results are brought to one maximum and
// added up in LDS, one map after the other.
//
// Where the queries alone do not fill the chip, a frame's keys are cut into runs: one frame's into `splits`, several frames' into runs
// of about one length, as many workgroups in all as there are places (run_cut: lengths and masks are known on the device
// only).  A row of more than one run leaves the maxima, sums and unscaled rows of each in `partial`, which diff_join_kernel adds
// up in a fixed order.  4 frames of 300 queries over 1600, 3200, 4800 and 6400 keys: 39.2 us with as many runs for every frame,
// 35.9 with runs of one length (a third of the keys masked and one frame without any 38.5, 35.5); frames that are equally long pay 0.2 to
// 0.9 us for it.
__device__ __forceinline__ int runs_of(int units, float run_inv, int most) {
  return units == 0 ? 0 : min(most, max(1, (int)ceilf(fmaf((float)units, run_inv, -1e-3f))));
}
// Runs of this lane's two frames (0: no keys): every lane tries a length, from a unit a wavefront on each a ninth longer, 5,600 units at last,
// and the shortest is taken whose workgroups have places at once (one more would take as long again); one run each if none has.
__device__ __forceinline__ void run_cut(const Frames& fr, const int (&tiles)[2], const DiffAttentionArgs& a, int waves, int (&runs)[2]) {
  const int lane = threadIdx.x & 63;
  int units[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    int keys = fr.k[i + 1] - fr.k[i];
    if (a.kv_len != nullptr && 2 * lane + i < a.B) keys = min(keys, a.kv_len[2 * lane + i]);
    units[i] = (keys + kUnitKeys - 1) / kUnitKeys;
  }
  const float inv = __builtin_amdgcn_exp2f(-0.15f * (float)lane) * (1.0f / (float)waves);
  int n = 0;
  for (int f = 0; f < a.B; ++f) n += of_lane_pair(tiles, f) * runs_of(of_lane_pair(units, f), inv, a.splits);
  const uint64_t fit = __ballot(n * a.heads <= a.places);
  const float chosen = fit == 0 ? 0.f : __int_as_float(__builtin_amdgcn_readlane(__float_as_int(inv), __ffsll((unsigned long long)fit) - 1));
#pragma unroll
  for (int i = 0; i < 2; ++i) runs[i] = runs_of(units[i], chosen, a.splits);
}
template <typename T, int DH>
struct Few {
  static constexpr int W = 2 * DH;                     // columns of both keys of a head, and of its values
  static constexpr int ROWB = W * (int)sizeof(T);      // bytes of such a row
  static constexpr int UNIT = kUnitKeys * ROWB;
  static constexpr int ROW = 2 * W + 4;                // of partial results: maxima and sums of both maps, the two rows
  static constexpr int WAVE = 2 * UNIT > 32 * W * 4 ? 2 * UNIT : 32 * W * 4;   // LDS of a wavefront: keys and values, then the rows of a map
};
// Where places > 0: a row's and head's number of runs, behind the partial results.
template <typename T, int DH>
__device__ __forceinline__ int* runs_of_items(const DiffAttentionArgs& a) {
  return reinterpret_cast<int*>(a.partial + (size_t)a.n_q * a.heads * a.splits * Few<T, DH>::ROW);
}
template <typename T, int DH, bool LIST, int NW>
__global__ __launch_bounds__(64 * NW, sizeof(T) == 2 ? 2 : 1) void diff_few_kernel(DiffAttentionArgs a) {
  constexpr int W = Few<T, DH>::W, ROWB = Few<T, DH>::ROWB, UNIT = Few<T, DH>::UNIT, WAVE = Few<T, DH>::WAVE;
  constexpr int CPR = ROWB / 16;                    // chunks of a row
  constexpr int KS = CPR / 4;                       // chunk pairs of one map
  constexpr int MO = W / 32;                        // blocks of 32 output columns
  constexpr int NI = UNIT / 1024, RPI = 1024 / ROWB;   // loads of a unit's keys, rows of one
  extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];
  __shared__ float s_m[NW][2][32], s_l[NW][2][32];

  const Frames fr = frames_of(a.cu_q, a.cu_k, a.B, a.n_q, a.n_k);
  if (fr.bad) {
    if (blockIdx.x == 0 && threadIdx.x == 0) *a.err_flag = 1;
    return;
  }
  const int tid = threadIdx.x, lane = tid & 63, l32 = lane & 31, g = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  // The tiles of a head and run of keys, which read the same rows, next to each other, and every XCD (workgroup mod 8), with an L2 of
  // its own, an eighth of every frame's in that order: 8 frames of 300 queries over 1600 tokens, 29.5 us with the tiles over all XCDs, 24.1 so.
  const int tiles[2] = {(fr.q[1] - fr.q[0] + kTileQ - 1) / kTileQ, (fr.q[2] - fr.q[1] + kTileQ - 1) / kTileQ};
  const int xcd = blockIdx.x & 7;
  int runs_in[2] = {a.splits, a.splits};
  if (a.places > 0) run_cut(fr, tiles, a, NW, runs_in);
  int before[2], count[2];   // of a frame's workgroups: this XCD's first, and how many
#pragma unroll
  for (int i = 0; i < 2; ++i) xcd_share(tiles[i] * a.heads * runs_in[i], xcd + 2 * lane + i, before[i], count[i]);
  int piece = blockIdx.x >> 3;
  const int upto = sum_upto(count[0] + count[1]);
  int frame = frame_of_piece(count, upto, piece);
  if (frame >= 0) {
    piece += of_lane_pair(before, frame);
  } else {
    // behind them the tiles of frames that have no run (zeros), whichever XCD
    if (a.places == 0) return;
    const int empty[2] = {runs_in[0] == 0 ? tiles[0] * a.heads : 0, runs_in[1] == 0 ? tiles[1] * a.heads : 0};
    piece = 8 * (piece - __builtin_amdgcn_readlane(upto, 63)) + xcd;
    frame = frame_of_piece(empty, sum_upto(empty[0] + empty[1]), piece);
    if (frame < 0) return;
  }
  const int frame_tiles = of_lane_pair(tiles, frame), runs = max(1, of_lane_pair(runs_in, frame));
  const int group = piece / frame_tiles, tile = piece - group * frame_tiles;
  const int split = group / a.heads, head = group - split * a.heads;
  const int q0 = of_frame(fr.q, frame), nq = behind_frame(fr.q, frame) - q0;
  const int k0 = of_frame(fr.k, frame), nk_all = behind_frame(fr.k, frame) - k0;
  const int nk = a.kv_len ? min(nk_all, a.kv_len[frame]) : nk_all;
  const int units = (nk + kUnitKeys - 1) / kUnitKeys, share = (units + runs - 1) / runs;
  const int u_end = min(units, (split + 1) * share);
  if (units == 0 && runs == 1) {
    for (int p = tid; p < kTileQ * CPR; p += 64 * NW) {
      const int q = tile * kTileQ + p / CPR;
      if (q >= nq) return;
      T* const to = static_cast<T*>(a.out) + (size_t)(q0 + q) * a.out_ld + head * W;
      *reinterpret_cast<uint4*>(to + p % CPR * Elem<T>::kChunk) = make_uint4(0, 0, 0, 0);
      if (a.places > 0 && p % CPR == 0) runs_of_items<T, DH>(a)[(size_t)(q0 + q) * a.heads + head] = 1;
    }
    return;
  }

  const T* const kbase = static_cast<const T*>(a.k) + (size_t)k0 * a.k_ld + head * W;
  const T* const vbase = static_cast<const T*>(a.v) + (size_t)k0 * a.v_ld + head * W;
  const int32_t* const list = LIST ? a.key_list + k0 : nullptr;
  unsigned char* const sK = smem + wave * WAVE;
  unsigned char* const sV = sK + UNIT;
  const uint32_t ldsK = (uint32_t)(uintptr_t)sK, ldsV = ldsK + UNIT;

  uint4 qf[2][KS];
  {
    const int row = min(tile * kTileQ + l32, nq - 1);
    const T* const qrow = static_cast<const T*>(a.q) + (size_t)(q0 + row) * a.q_ld + head * W;
#pragma unroll
    for (int m = 0; m < 2; ++m)
#pragma unroll
      for (int c = 0; c < KS; ++c) qf[m][c] = *reinterpret_cast<const uint4*>(qrow + m * DH + (2 * c + g) * Elem<T>::kChunk);
  }
  // A unit's loads: piece `lane` of load j lies in LDS row RPI j + lane / CPR.  The key of that row is key_at(RPI j) + key_at(lane / CPR)
  // (row_of_key moves bits and is its own inverse), so that a full unit of consecutive keys needs an offset a
  // lane and its places in the row.  Rows behind the last key are the last key's again.  With a list lane l has the row of key l mod
  // 32, asked for two units ahead, and the others fetch it from there.
  auto key_at = [](int row) { return Elem<T>::row_of_key(row); };
  const int within = key_at(lane / CPR), place = lane % CPR;
  int listed = 0;
  auto ask = [&](int u) {
    if constexpr (LIST) listed = list[min(u * kUnitKeys + l32, nk - 1)];
  };
  auto load = [&](const T* base, int ld, auto values, int u, int rows, uint32_t to) {
    const int last = nk - 1 - u * kUnitKeys;
    const T* const from = base + (size_t)(u * kUnitKeys) * ld;
    const uint32_t step = (uint32_t)ld * (uint32_t)sizeof(T);
#pragma unroll
    for (int j = 0; j < NI; ++j) {
      const int row = RPI * j + lane / CPR;
      const uint32_t col = (uint32_t)(decltype(values)::value ? value_piece<T, ROWB>(row, place) : key_piece<T, ROWB>(row, place)) * 16;
      if constexpr (LIST)
        dma16(reinterpret_cast<const char*>(base) + (size_t)__shfl(rows, key_at(RPI * j) + within) * step + col, to + j * 1024);
      else if (last >= kUnitKeys - 1)
        dma16(from + (size_t)key_at(RPI * j) * ld, within * step + col, to + j * 1024);
      else
        dma16(from, (uint32_t)min(key_at(RPI * j) + within, last) * step + col, to + j * 1024);
    }
  };
  const auto of_keys = std::integral_constant<bool, false>{};
  const auto of_values = std::integral_constant<bool, true>{};
  f32x16 acc[2][MO];
  float m_run[2] = {-INFINITY, -INFINITY}, l_run[2] = {0.f, 0.f};
#pragma unroll
  for (int m = 0; m < 2; ++m)
#pragma unroll
    for (int i = 0; i < MO; ++i)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[m][i][r] = 0.f;

  int u = split * share + wave;
  if (u < u_end) {
    ask(u);
    load(kbase, a.k_ld, of_keys, u, listed, ldsK);
    load(vbase, a.v_ld, of_values, u, listed, ldsV);
    if (u + NW < u_end) ask(u + NW);
  }
#pragma nounroll
  for (; u < u_end; u += NW) {
    const bool more = u + NW < u_end;
    const int left = nk - u * kUnitKeys, rows = listed;
    // (the keys; their values, asked for behind them, need not be there yet)
    asm volatile("s_waitcnt vmcnt(%0)" : : "n"(NI) : "memory");
    f32x16 s[2];
    unit_logits<T, DH>(sK, qf, s);
    asm volatile("s_waitcnt lgkmcnt(0)" : : : "memory");
    if (more) load(kbase, a.k_ld, of_keys, u + NW, rows, ldsK);
    unit_weights<T>(s, left, a.scale2, m_run, l_run, acc);
    if (more) asm volatile("s_waitcnt vmcnt(%0)" : : "n"(NI) : "memory");
    else asm volatile("s_waitcnt vmcnt(0)" : : : "memory");
    if (left < kUnitKeys) {
      // weight 0 times what the last key's values are may be no number
      for (int p = lane; p < (kUnitKeys - left) * CPR; p += 64)
        *reinterpret_cast<uint4*>(sV + Elem<T>::row_of_key(left + p / CPR) * ROWB + p % CPR * 16) = make_uint4(0, 0, 0, 0);
      wave_fence();
    }
    unit_rows<T, DH>(sV, s, acc);
    asm volatile("s_waitcnt lgkmcnt(0)" : : : "memory");
    if (more) load(vbase, a.v_ld, of_values, u + NW, rows, ldsV);
    if (u + 2 * NW < u_end) ask(u + 2 * NW);
  }

  // The wavefronts' results to one maximum, and map by map into LDS: row of a query, its quads of columns moved by the
  // query.  Thread: query tid / (2 NW), one part of its columns.
#pragma unroll
  for (int m = 0; m < 2; ++m) {
    l_run[m] = half_sum(l_run[m]);
    if (g == 0) {
      s_m[wave][m][l32] = m_run[m];
      s_l[wave][m][l32] = l_run[m];
    }
  }
  __syncthreads();
  constexpr int PARTS = 2 * NW, CE = W / PARTS;
  const int qi = tid / PARTS, part = tid % PARTS;
  const int q_local = tile * kTileQ + qi;
  auto highest = [&](int m, int q) {
    float top = s_m[0][m][q];
#pragma unroll
    for (int w = 1; w < NW; ++w) top = fmaxf(top, s_m[w][m][q]);
    return top;
  };
  float o[2][CE], l_all[2], m_all[2];
#pragma unroll
  for (int m = 0; m < 2; ++m) {
    const float top = highest(m, l32);
    const float f = __builtin_amdgcn_exp2f(m_run[m] - (top == -INFINITY ? 0.f : top));
    float* const rows = reinterpret_cast<float*>(sK) + l32 * W;
#pragma unroll
    for (int i = 0; i < MO; ++i)
#pragma unroll
      for (int rq = 0; rq < 4; ++rq) {
        const int quad = 8 * i + 2 * rq + g;   // columns 32 i + 8 rq + 4 g on
        *reinterpret_cast<float4*>(rows + 4 * (quad ^ (l32 & (W / 4 - 1)))) =
            make_float4(acc[m][i][4 * rq] * f, acc[m][i][4 * rq + 1] * f, acc[m][i][4 * rq + 2] * f, acc[m][i][4 * rq + 3] * f);
      }
    __syncthreads();
    m_all[m] = highest(m, qi);
    l_all[m] = 0.f;
#pragma unroll
    for (int e = 0; e < CE; ++e) o[m][e] = 0.f;
#pragma unroll
    for (int w = 0; w < NW; ++w) {
      l_all[m] += s_l[w][m][qi] * __builtin_amdgcn_exp2f(s_m[w][m][qi] - (m_all[m] == -INFINITY ? 0.f : m_all[m]));
      const float* const from = reinterpret_cast<const float*>(smem + w * WAVE) + qi * W;
#pragma unroll
      for (int e = 0; e < CE / 4; ++e) {
        const float4 v = *reinterpret_cast<const float4*>(from + 4 * ((part * (CE / 4) + e) ^ (qi & (W / 4 - 1))));
        o[m][4 * e] += v.x;
        o[m][4 * e + 1] += v.y;
        o[m][4 * e + 2] += v.z;
        o[m][4 * e + 3] += v.w;
      }
    }
    if (m == 0) __syncthreads();
  }
  const size_t item = (size_t)(q0 + q_local) * a.heads + head;
  if (a.places > 0 && split == 0 && part == 0 && q_local < nq) runs_of_items<T, DH>(a)[item] = runs;
  if (runs > 1) {
    if (q_local < nq) {
      float* const to = a.partial + (item * a.splits + split) * Few<T, DH>::ROW;
      if (part == 0) *reinterpret_cast<float4*>(to) = make_float4(m_all[0], m_all[1], l_all[0], l_all[1]);
#pragma unroll
      for (int m = 0; m < 2; ++m)
#pragma unroll
        for (int e = 0; e < CE / 4; ++e)
          *reinterpret_cast<float4*>(to + 4 + m * W + part * CE + 4 * e) = make_float4(o[m][4 * e], o[m][4 * e + 1], o[m][4 * e + 2], o[m][4 * e + 3]);
    }
    return;
  }
  const float lambda = a.lambda[head];
  const float i0 = l_all[0] != 0.f ? 1.0f / l_all[0] : 0.f, i1 = l_all[1] != 0.f ? lambda / l_all[1] : 0.f;
  float x[CE], sq = 0.f;
#pragma unroll
  for (int e = 0; e < CE; ++e) {
    x[e] = o[0][e] * i0;
    if (lambda != 0.f) x[e] = fmaf(-o[1][e], i1, x[e]);   // (lambda 0 leaves the first map alone, whatever the second holds)
    sq = fmaf(x[e], x[e], sq);
  }
  if (a.head_g) {
#pragma unroll
    for (int s = 1; s < PARTS; s <<= 1) sq += __shfl_xor(sq, s);
    const float r = rsqrtf(sq * (1.0f / W) + a.eps);
#pragma unroll
    for (int e = 0; e < CE; ++e) x[e] *= r * a.head_g[part * CE + e];
  }
  if (q_local < nq) {
    store_columns<T, CE>(static_cast<T*>(a.out) + (size_t)(q0 + q_local) * a.out_ld + head * W + part * CE, x);
  }
}

// The runs' results of a row and head, by one workgroup: wavefront w adds up runs w, w + NW, .. in that order, lane l
// a quad of columns of map l / 32, and the wavefronts' sums are added in order.
template <typename T, int DH, int NW>
__global__ __launch_bounds__(64 * NW) void diff_join_kernel(DiffAttentionArgs a) {
  constexpr int W = 2 * DH, Q = W / 4;   // quads of a map: 32 or 16 lanes of its 32
  constexpr int ROW = Few<T, DH>::ROW;
  __shared__ float4 s_o[NW][64];
  __shared__ float s_l[NW][64];
  const int lane = threadIdx.x & 63, map = lane >> 5, quad = lane & 31;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int item = blockIdx.x, row = item / a.heads, head = item - row * a.heads;
  const float* const from = a.partial + (size_t)item * a.splits * ROW;
  // (of a row behind the last frame, or after bad offsets, nothing is known: what is read here is then not used)
  const int cut = a.places > 0 ? runs_of_items<T, DH>(a)[item] : a.splits;
  float top[kMostSplits / 32];
#pragma unroll
  for (int i = 0; i < kMostSplits / 32; ++i) top[i] = quad + 32 * i < a.splits ? from[(size_t)(quad + 32 * i) * ROW + map] : -INFINITY;
  if (frames_of(a.cu_q, a.cu_k, a.B, a.n_q, a.n_k).bad || row >= a.cu_q[a.B]) return;
  const int runs = __builtin_amdgcn_readfirstlane(cut);
  if (runs == 1) return;   // the row is finished
  float m = -INFINITY;
#pragma unroll
  for (int i = 0; i < kMostSplits / 32; ++i) m = quad + 32 * i < runs ? fmaxf(m, top[i]) : m;
#pragma unroll
  for (int s = 1; s < 32; s <<= 1) m = fmaxf(m, __shfl_xor(m, s));
  const float m_ref = m == -INFINITY ? 0.f : m;
  float l = 0.f;
  float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 8
  for (int s = wave; s < runs; s += NW) {
    const float* const p = from + (size_t)s * ROW;
    const float f = __builtin_amdgcn_exp2f(p[map] - m_ref);
    l = fmaf(p[2 + map], f, l);
    if (quad < Q) {
      const float4 v = *reinterpret_cast<const float4*>(p + 4 + map * W + 4 * quad);
      o = make_float4(fmaf(v.x, f, o.x), fmaf(v.y, f, o.y), fmaf(v.z, f, o.z), fmaf(v.w, f, o.w));
    }
  }
  s_o[wave][lane] = o;
  s_l[wave][lane] = l;
  __syncthreads();
  if (wave > 0) return;
#pragma unroll
  for (int w = 1; w < NW; ++w) {
    const float4 v = s_o[w][lane];
    o = make_float4(o.x + v.x, o.y + v.y, o.z + v.z, o.w + v.w);
    l += s_l[w][lane];
  }
  const float weight = map ? -a.lambda[head] : 1.0f, i = l != 0.f ? weight / l : 0.f;
  o = weight != 0.f ? make_float4(o.x * i, o.y * i, o.z * i, o.w * i) : make_float4(0.f, 0.f, 0.f, 0.f);
  o = make_float4(half_sum(o.x), half_sum(o.y), half_sum(o.z), half_sum(o.w));
  if (a.head_g) {
    float sq = fmaf(o.x, o.x, o.y * o.y) + fmaf(o.z, o.z, o.w * o.w);
#pragma unroll
    for (int s = 1; s < 32; s <<= 1) sq += __shfl_xor(sq, s);
    const float r = rsqrtf(sq * (1.0f / W) + a.eps);
    if (quad < Q) {
      const float4 gq = *reinterpret_cast<const float4*>(a.head_g + 4 * quad);
      o = make_float4(o.x * r * gq.x, o.y * r * gq.y, o.z * r * gq.z, o.w * r * gq.w);
    }
  }
  if (map == 0 && quad < Q) {
    T* const to = static_cast<T*>(a.out) + (size_t)row * a.out_ld + head * W + 4 * quad;
    const float x[4] = {o.x, o.y, o.z, o.w};
    store_columns<T, 4>(to, x);
  }
}

// ---- masked keys ---------------------------------------------------------------------------
// The keys of every frame that its mask leaves, in order, as row numbers within the frame, and their count: masked
// rows are then never read.  A workgroup lists kListKeys keys of one frame, after it has counted those before, byte by
// byte: the last one of a frame of 50,001 keys counts 48,000 (one query over them, 12 heads of width 64: 33.9 us without a mask, 43.5
// with a tenth masked).
constexpr int kListKeys = 2048;
__global__ __launch_bounds__(kThreads) void key_list_kernel(const uint8_t* __restrict__ mask, const int32_t* __restrict__ cu_k,
                                                            int B, int n_k, int32_t* __restrict__ list, int32_t* __restrict__ kv_len) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const Frames fr = frames_of(cu_k, cu_k, B, n_k, n_k);
  if (fr.bad) return;   // refused by the attention
  const int parts[2] = {lane * 2 < B ? max(1, (fr.k[1] - fr.k[0] + kListKeys - 1) / kListKeys) : 0,
                        lane * 2 + 1 < B ? max(1, (fr.k[2] - fr.k[1] + kListKeys - 1) / kListKeys) : 0};
  int part = blockIdx.x;
  const int f = frame_of_piece(parts, sum_upto(parts[0] + parts[1]), part);
  if (f < 0) return;
  const int k0 = of_frame(fr.k, f), nk = behind_frame(fr.k, f) - k0;
  const int first = part * kListKeys, end = min(nk, first + kListKeys);
  const uint8_t* const m = mask + k0;
  __shared__ int s_count[4];
  int before = 0;
#pragma unroll 8
  for (int i = tid; i < first; i += kThreads) before += m[i] != 0;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) before += __shfl_xor(before, o);
  if (lane == 0) s_count[wave] = before;
  __syncthreads();
  int at = s_count[0] + s_count[1] + s_count[2] + s_count[3];
  // this part: a wavefront's keys are consecutive, 64 a step
  constexpr int STEPS = kListKeys / kThreads;
  uint64_t bits[STEPS];
  int mine = 0;
#pragma unroll
  for (int s = 0; s < STEPS; ++s) {
    const int i = first + (wave * STEPS + s) * 64 + lane;
    bits[s] = __ballot(i < end && m[i] != 0);
    mine += __popcll(bits[s]);
  }
  __syncthreads();
  if (lane == 0) s_count[wave] = mine;
  __syncthreads();
  for (int w = 0; w < wave; ++w) at += s_count[w];
#pragma unroll
  for (int s = 0; s < STEPS; ++s) {
    if (bits[s] >> lane & 1) list[k0 + at + __popcll(bits[s] & ((uint64_t(1) << lane) - 1))] = first + (wave * STEPS + s) * 64 + lane;
    at += __popcll(bits[s]);
  }
  if (end == nk && wave == 3 && lane == 0) kv_len[f] = at;
}

template <typename T, int DH, bool LIST, int NW>
hipError_t few(const DiffAttentionArgs& a, hipStream_t s) {
  constexpr int LDS = NW * Few<T, DH>::WAVE;
  static DeviceOnce once;
  if (hipError_t e = allow_lds(diff_few_kernel<T, DH, LIST, NW>, LDS, &once); e != hipSuccess) return e;
  // (an eighth of a frame's workgroups, rounded up, for an XCD; run_cut leaves the tiles or no more runs than there are places, and
  // the tiles of frames without keys)
  const int64_t tiles = ((int64_t)a.n_q / kTileQ + a.B) * a.heads, rows = (int64_t)a.n_q * a.heads;
  const int64_t grid = 8 * ((a.places > 0 ? tiles + a.places : tiles * a.splits) / 8 + a.B + 2);
  if (grid > 0x7FFFFFFF || rows > 0x7FFFFFFF) return hipErrorInvalidValue;
  hipLaunchKernelGGL((diff_few_kernel<T, DH, LIST, NW>), dim3((unsigned)grid), dim3(64 * NW), LDS, s, a);
  if (a.splits > 16)
    hipLaunchKernelGGL((diff_join_kernel<T, DH, 16>), dim3((unsigned)rows), dim3(1024), 0, s, a);
  else if (a.splits > 1)
    hipLaunchKernelGGL((diff_join_kernel<T, DH, 2>), dim3((unsigned)rows), dim3(128), 0, s, a);
  return hipGetLastError();
}
template <typename T, int DH>
hipError_t few(const DiffAttentionArgs& a, hipStream_t s) {
  // fp32 has LDS for four wavefronts
  if constexpr (sizeof(T) == 2)
    if (a.wide) return a.key_list ? few<T, DH, true, 8>(a, s) : few<T, DH, false, 8>(a, s);
  return a.key_list ? few<T, DH, true, 4>(a, s) : few<T, DH, false, 4>(a, s);
}
template <typename T>
hipError_t few(const DiffAttentionArgs& a, int d_head, hipStream_t s) {
  if (d_head == 64) return few<T, 64>(a, s);
  if (d_head == 32) return few<T, 32>(a, s);
  return hipErrorInvalidValue;
}

}  // namespace

hipError_t launch_key_list(const uint8_t* mask, const int32_t* cu_k, int B, int n_k, int32_t* list, int32_t* kv_len, hipStream_t s) {
  hipLaunchKernelGGL(key_list_kernel, dim3(n_k / kListKeys + B), dim3(kThreads), 0, s, mask, cu_k, B, n_k, list, kv_len);
  return hipGetLastError();
}

// Which kernel, how many wavefronts, how many runs (us on 256 CUs, bf16; heads are pairs of heads):
// - 128 queries a workgroup from half a tile a CU on.  19,200 rows and heads of width 64 over 1600 keys 42 (32 a workgroup 58), 24,000
//   over 700 to 1300 39 (49); below, 9,600 over 1600 34 (39), 12,000 over 1000 26 (30), 9,000 in ten frames over 1200 30 (34).
//   The rule counts rows and not workgroups, and is wrong where frames fill little of a tile of 128: 64 frames of 42 queries
//   (6 heads of width 64, 16,128 rows) over themselves 16.8 by 32, of 43 (16,512) 30.9 by 128; over 300 keys 28.7 and 39.1.
// - 32 queries, eight wavefronts where such workgroups leave no CU two.  One frame of 700, 1000, 1600 keys, 4 heads of width 32: 10.4,
//   12.0, 15.0 (four wavefronts 11.4, 13.8, 19.0); from 16 units of keys on, two a wavefront: below they change nothing.  More workgroups than
//   CUs: 300 of 1600 keys 42 (34), 312 of 400 keys 17.0 (11.6).  The LDS of fp32 rows is too large for eight.
// - Runs where there are places for two a row and more than three units a wavefront.  One query over 600 keys 12.0 (in runs
//   13.4), over 900 13.7 (in one 15.3), over 1200 13.2 (17.1), over 2000 14.3 (22.3).  The mean of the frames decides: 12 queries of
//   as many frames, 11 of 100 keys and one of 6,000, are not cut and take 49; with 600 keys each 12.8, the long one alone 14.6.
void plan_diff_attention(DiffAttentionArgs& a, int rows_q, int rows_k, int d_head, bool use_bf16, uint64_t partial_bytes, int cus) {
  const int64_t per_frame = (rows_q + a.B - 1) / a.B;
  auto workgroups = [&](int queries) { return a.B * ((per_frame + queries - 1) / queries) * a.heads; };
  a.splits = 1;
  a.places = 0;
  a.tiles = use_bf16 && (int64_t)rows_q * a.heads >= (int64_t)64 * cus;
  if (a.tiles) {
    a.wide = workgroups(128) <= cus;   // (see the kernel)
    return;
  }
  const int64_t groups = workgroups(kTileQ), units = (rows_k / a.B + kUnitKeys - 1) / kUnitKeys;
  a.wide = use_bf16 && groups <= cus && units >= 16;
  const int waves = a.wide ? 8 : 4, places = use_bf16 && !a.wide ? 2 * cus : cus;
  if (units <= 3 * waves || 2 * groups > places) return;
  // (a row's and head's number of runs, and its runs' results)
  const int64_t room = (int64_t)partial_bytes / std::max<int64_t>(1, (int64_t)a.n_q * a.heads) - 4;
  int64_t splits = std::min<int64_t>(room / ((4 * d_head + 4) * 4), kMostSplits);
  if (a.B == 1) splits = std::min({splits, places / std::max<int64_t>(1, groups), units / waves});
  a.splits = (int)std::max<int64_t>(1, splits);
  if (a.B > 1 && a.splits > 1) a.places = places;
}

hipError_t launch_diff_attention(const DiffAttentionArgs& a, int d_head, bool use_bf16, hipStream_t s) {
  if (use_bf16 && a.tiles) return launch_diff_tiles(a, d_head, s);
  return use_bf16 ? few<bf16_t>(a, d_head, s) : few<float>(a, d_head, s);
}

}  // namespace cfdetr
