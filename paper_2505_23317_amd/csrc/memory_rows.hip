// Rows on their way into a paged stream memory: queries and keys turned by positions of several axes, and keys and values
// written into their slots (keys turned on the way, so that they are read and written once).
//
// Pair i of a head, i < n = rot_dim / 2, is turned by the angle pos[axis[i]] freq[i] as in rotary.hip; which axis a pair belongs
// to comes from a table, since time, row and column have numbers of pairs of their own, in blocks or in turn.
//
// Bound by memory, as there: a workgroup takes some rows, works their sines and cosines out once into LDS (product and
// whole turns in 64 bits: a far position is thousands of turns) while its features are on their way, and turns them.
// What is left of a turn goes through the 32-bit functions in bf16 (as in rotary.hip, the same bits; off by some 2^-23 where the
// result is rounded to 2^-8) and through the 64-bit ones in fp32, the check mode: sine and cosine are then rounded once, features
// off by what their own operations lose.  16,063 rows of 2 x 768 columns: 30.2 -> 30.5 us for it, 93,750 of 32 into a memory 10.8 -> 11.6.
#include <algorithm>
#include <type_traits>

#include "rotary.h"

namespace cfdetr {

namespace {

constexpr int kThreads = 256;

// Units (two runs of 16 bytes of one head) of a row: those of the first part's heads, then those of the second's.
template <typename T, bool INTERLEAVED, bool APPEND>
__global__ __launch_bounds__(kThreads) void turn_rows_kernel(TurnRowsArgs a, int rows_wg, int units_row, int units_first) {
  constexpr int RUN = Runs<T>::kRun;
  typedef typename Runs<T>::Piece Piece;
  extern __shared__ float2 turns[];   // [rows_wg][n] cosine and sine
  const int row0 = blockIdx.x * rows_wg, rows = min(rows_wg, a.M - row0);
  const int tid = threadIdx.x, per_head = a.d_head / (2 * RUN);
  const int r = tid / units_row, u = tid - r * units_row;
  const bool is_first = u < units_first;
  const int n = APPEND && !is_first ? 0 : a.rot_dim / 2;   // pairs of a head of this part
  const int head_run = is_first ? u : u - units_first;
  const int head = head_run / per_head, j = RUN * (head_run - head * per_head);
  const bool rotated = j < n;
  const int at = head * a.d_head + (rotated ? j : n + j);   // where the first run starts in the row
  const int apart = rotated ? n : a.d_head / 2 - n;         // and the second behind it
  const TurnRowsPart p = is_first ? a.first : a.second;
  size_t to = row0 + r;
  bool mine = r < rows;
  if (APPEND && mine) {
    const int slot = a.slots[to];
    mine = slot >= 0 && slot < a.n_slots;
    if (slot >= a.n_slots) *a.err_flag = 1;
    to = (size_t)slot;
  }
  Runs<T> f;
  if (mine) {
    const T* const src = static_cast<const T*>(p.in) + (size_t)(row0 + r) * p.in_ld + at;
    f.v[0] = *reinterpret_cast<const Piece*>(src);
    f.v[1] = *reinterpret_cast<const Piece*>(src + apart);
  }
  const int pairs = a.rot_dim / 2;
  for (int i = tid; i < rows * pairs; i += kThreads) {
    const int row = i / pairs, pair = i - row * pairs;
    const int axis = min((int)a.axis[pair], a.n_axes - 1);
    double t = (double)a.pos[(size_t)(row0 + row) * a.n_axes + axis] * a.freq[pair] * 0.15915494309189533577;
    t -= rint(t);
    if constexpr (std::is_same_v<T, float>) {
      double s, c;
      sincospi(2.0 * t, &s, &c);
      turns[i] = make_float2((float)c, (float)s);
    } else {
      float s, c;
      sincospif(2.0f * (float)t, &s, &c);
      turns[i] = make_float2(c, s);
    }
  }
  __syncthreads();
  if (!mine) return;
  float x[2][RUN];
  f.get(x);
  if (rotated) {
    const float2* const t0 = turns + r * n + (INTERLEAVED ? j / 2 : j);
#pragma unroll
    for (int q = 0; q < RUN; ++q) {
      // pair q of the unit: the runs' elements q, or two neighbours, the second half of the pairs in the second run
      const int h = 2 * q / RUN, e = 2 * q % RUN;
      float& x0 = INTERLEAVED ? x[h][e] : x[0][q];
      float& x1 = INTERLEAVED ? x[h][e + 1] : x[1][q];
      const float2 t = t0[INTERLEAVED ? (h ? n / 2 : 0) + e / 2 : q];
      const float y0 = fmaf(x0, t.x, -(x1 * t.y)), y1 = fmaf(x0, t.y, x1 * t.x);
      x0 = y0;
      x1 = y1;
    }
  }
  if (!APPEND && is_first) {
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int q = 0; q < RUN; ++q) x[h][q] *= a.scale;
  }
  // (what is neither turned nor scaled is written as it was read, whatever it holds)
  if (rotated || (!APPEND && is_first)) f.put(x);
  T* const dst = static_cast<T*>(p.out) + to * p.out_ld + at;
  *reinterpret_cast<Piece*>(dst) = f.v[0];
  *reinterpret_cast<Piece*>(dst + apart) = f.v[1];
}

template <typename T, bool INTERLEAVED, bool APPEND>
hipError_t launch(TurnRowsArgs a, hipStream_t s) {
  const int units_first = a.first.heads * a.d_head / (2 * Runs<T>::kRun);
  const int units_row = units_first + a.second.heads * a.d_head / (2 * Runs<T>::kRun);
  if (units_row > kThreads) return hipErrorInvalidValue;
  const int rows_wg = kThreads / units_row;
  // a launch has 2^32 threads at most: more rows go in several
  constexpr int kSlice = 1 << 23;
  const int M = a.M;
  for (int64_t done = 0; done < M; done += kSlice) {
    a.M = (int)std::min<int64_t>(kSlice, M - done);
    hipLaunchKernelGGL((turn_rows_kernel<T, INTERLEAVED, APPEND>), dim3((a.M + rows_wg - 1) / rows_wg), dim3(kThreads),
                       (size_t)rows_wg * (a.rot_dim / 2) * sizeof(float2), s, a, rows_wg, units_row, units_first);
    if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    for (TurnRowsPart* p : {&a.first, &a.second}) {
      if (!p->in) continue;
      p->in = static_cast<const T*>(p->in) + (size_t)kSlice * p->in_ld;
      if (!APPEND) p->out = static_cast<T*>(p->out) + (size_t)kSlice * p->out_ld;
    }
    a.pos += (size_t)kSlice * a.n_axes;
    if (APPEND) a.slots += kSlice;
  }
  return hipSuccess;
}

}  // namespace

hipError_t launch_turn_rows(const TurnRowsArgs& a, bool use_bf16, hipStream_t s) {
  if (a.rot_dim % 16 != 0 || a.d_head % 32 != 0) return hipErrorInvalidValue;   // whole runs in either half
  if (a.slots) {
    if (use_bf16) return a.interleaved ? launch<bf16_t, true, true>(a, s) : launch<bf16_t, false, true>(a, s);
    return a.interleaved ? launch<float, true, true>(a, s) : launch<float, false, true>(a, s);
  }
  if (use_bf16) return a.interleaved ? launch<bf16_t, true, false>(a, s) : launch<bf16_t, false, false>(a, s);
  return a.interleaved ? launch<float, true, false>(a, s) : launch<float, false, false>(a, s);
}

}  // namespace cfdetr
