// One step of a paged stream memory: tokens forgotten in front of every stream, pages given back and taken, slots of
// the new tokens (the arithmetic of a stream: stream_memory.h).
//
// Page numbers are taken from the front of a ring of free ones and given back at its end, so that what is taken and what is
// given back in one step are different places of the ring whatever the order of the threads.  Which place is whose: exclusive
// sums over the streams of the numbers taken and given back.  Every workgroup works them out for itself from all streams'
// spans, then takes its share of the slots and page numbers, so that a step is one launch.  A few microseconds
// of latency bound it: one round of loads for the spans, the sums, one for the page numbers.
#include "kernels.h"
#include "stream_memory.h"

namespace cfdetr {

namespace {

constexpr int kThreads = 256;

struct Sums {
  int taken, given, work;
};

// Exclusive sums of the threads' numbers over the workgroup, in order; the totals come back in `all`.
__device__ __forceinline__ Sums sums_before(const Sums& mine, Sums& all, int (*s_wave)[kThreads / 64]) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const Sums upto{sum_upto(mine.taken), sum_upto(mine.given), sum_upto(mine.work)};
  if (lane == 63) {
    s_wave[0][wave] = upto.taken;
    s_wave[1][wave] = upto.given;
    s_wave[2][wave] = upto.work;
  }
  __syncthreads();
  Sums base{};
  all = Sums{};
#pragma unroll
  for (int w = 0; w < kThreads / 64; ++w) {
    const Sums s{s_wave[0][w], s_wave[1][w], s_wave[2][w]};
    if (w < wave) base = Sums{base.taken + s.taken, base.given + s.given, base.work + s.work};
    all = Sums{all.taken + s.taken, all.given + s.given, all.work + s.work};
  }
  return Sums{base.taken + upto.taken - mine.taken, base.given + upto.given - mine.given, base.work + upto.work - mine.work};
}

__global__ __launch_bounds__(kThreads) void memory_advance_kernel(MemoryAdvanceArgs a) {
  extern __shared__ int lds[];
  __shared__ int s_wave[3][kThreads / 64], s_bad, s_last;
  const int B = a.B, cols = a.cols, tid = threadIdx.x;
  int* const s_cu = lds;                     // [B + 1]
  int* const s_taken = s_cu + B + 1;         // exclusive sums over the streams
  int* const s_given = s_taken + B;
  int* const s_work = s_given + B;
  const bool moved = a.table_out != a.table;
  const int head = a.pool[0], n_free = a.pool[1];
  auto step_of = [&](int b, int fresh) {
    const int2 span = a.span[b];
    return stream_step(span.x, span.y, a.drop ? a.drop[b] : 0, fresh, a.page_bits, cols);
  };

  if (tid == 0) s_bad = 0;
  __syncthreads();
  const int per = (B + kThreads - 1) / kThreads, b0 = tid * per, b1 = min(B, b0 + per);
  bool bad = false;
  Sums mine{};
  for (int b = b0; b < b1; ++b) {
    const int c0 = a.cu[b], c1 = a.cu[b + 1];
    s_cu[b] = c0;
    if (b == B - 1) s_cu[B] = c1;
    const bool wrong = c0 < 0 || c1 < c0 || c1 > a.n_new || (b == 0 && c0 != 0);
    const StreamStep s = step_of(b, wrong ? -1 : c1 - c0);
    s_taken[b] = mine.taken;
    s_given[b] = mine.given;
    s_work[b] = mine.work;
    if (s.bad) {
      bad = true;
      continue;
    }
    mine.taken += s.taken;
    mine.given += s.given;
    mine.work += s.given + s.taken + (moved ? s.kept : 0);
  }
  if (bad) s_bad = 1;
  Sums all;
  const Sums base = sums_before(mine, all, s_wave);
  for (int b = b0; b < b1; ++b) {
    s_taken[b] += base.taken;
    s_given[b] += base.given;
    s_work[b] += base.work;
  }
  __syncthreads();
  const bool refused = s_bad != 0 || head < 0 || head >= a.n_pages || n_free < 0 || n_free > a.n_pages || all.taken > n_free ||
                       all.given > a.n_pages - n_free;
  const int at = blockIdx.x * kThreads + tid, step = gridDim.x * kThreads;
  if (refused) {
    for (int m = at; m < a.n_new; m += step) a.slots[m] = -1;
    if (moved)
      for (size_t i = at; i < (size_t)B * cols; i += step) a.table_out[i] = a.table[i];
    if (at == 0) *a.err_flag = 1;
  } else {
    auto place = [&](int i) { return i >= a.n_pages ? i - a.n_pages : i; };
    for (int m = at; m < a.n_new; m += step) {
      int slot = -1;
      if (m < s_cu[B]) {
        const int b = stream_of(s_cu, B, m);
        const StreamStep s = step_of(b, s_cu[b + 1] - s_cu[b]);
        const int p = s.first + s.held + m - s_cu[b], page = p >> a.page_bits;
        const int id = page < s.have ? a.table[(size_t)b * cols + ring_column(page, cols)] : a.free[place(head + s_taken[b] + page - s.have)];
        if ((unsigned)id < (unsigned)a.n_pages) slot = (id << a.page_bits) | (p & ((1 << a.page_bits) - 1));
        else *a.err_flag = 1;   // (a table or a list that no step has left)
      }
      a.slots[m] = slot;
    }
    for (int i = at; i < all.work; i += step) {
      const int b = stream_of(s_work, B, i);
      const StreamStep s = step_of(b, s_cu[b + 1] - s_cu[b]);
      const PageWork w = page_work(s, i - s_work[b], cols);
      const size_t entry = (size_t)b * cols + w.column;
      if (w.given >= 0) a.free[place(head + n_free + s_given[b] + w.given)] = a.table[entry];
      if (w.taken >= 0) a.table_out[entry] = a.free[place(head + s_taken[b] + w.taken)];
      if (w.kept) a.table_out[entry] = a.table[entry];
    }
  }
  // The new spans may lie over the old ones: they are written by the workgroup that is done last, when nobody reads the
  // old ones any more.
  if (gridDim.x > 1) {
    __syncthreads();
    if (tid == 0) {
      s_last = __hip_atomic_fetch_add(a.arrived, 1, __ATOMIC_ACQ_REL, __HIP_MEMORY_SCOPE_AGENT) == (int)gridDim.x - 1;
      if (s_last) __hip_atomic_store(a.arrived, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    __syncthreads();
    if (!s_last) return;
  } else {
    __syncthreads();
  }
  for (int b = tid; b < B; b += kThreads) {
    int2 to = a.span[b];
    if (!refused) {
      const int fresh = s_cu[b + 1] - s_cu[b];
      const StreamStep s = step_of(b, fresh);
      to = make_int2(s.first, s.held + fresh);
    }
    a.span_out[b] = to;
  }
  if (tid == 0) {
    a.pool_out[0] = refused ? head : head + all.taken - (head + all.taken >= a.n_pages ? a.n_pages : 0);
    a.pool_out[1] = refused ? n_free : n_free - all.taken + all.given;
  }
}

}  // namespace

hipError_t launch_memory_advance(const MemoryAdvanceArgs& a, int cus, hipStream_t s) {
  // a few slots or page numbers a thread, a workgroup a CU at most; a single workgroup needs no counting at the end
  const int64_t work = ((int64_t)a.n_new + 1023) / 1024 + (a.table_out != a.table ? ((int64_t)a.B * a.cols + 4095) / 4096 : 0);
  const int grid = (int)(work < 1 ? 1 : work > cus ? cus : work);
  const size_t lds = (size_t)(4 * a.B + 1) * sizeof(int);
  static DeviceOnce once;
  if (hipError_t e = allow_lds(memory_advance_kernel, (4 * kMemoryMaxStreams + 1) * (int)sizeof(int), &once); e != hipSuccess) return e;
  hipLaunchKernelGGL(memory_advance_kernel, dim3(grid), dim3(kThreads), lds, s, a);
  return hipGetLastError();
}

}  // namespace cfdetr
