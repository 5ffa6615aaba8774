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

constexpr int kThreads = kAdvanceThreads, kWaves = kThreads / 64;

struct Sums {
  int taken, given, work;
};

// Exclusive sums of the threads' numbers over the workgroup, in order; the totals come back in `all`, and in `bad` whether any
// thread's was.
__device__ __forceinline__ Sums sums_before(const Sums& mine, Sums& all, bool& bad, int (*s_wave)[kWaves]) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const Sums upto{sum_upto(mine.taken), sum_upto(mine.given), sum_upto(mine.work)};
  const int any = __any(bad);
  if (lane == 63) {
    s_wave[0][wave] = upto.taken;
    s_wave[1][wave] = upto.given;
    s_wave[2][wave] = upto.work;
    s_wave[3][wave] = any;
  }
  __syncthreads();
  Sums base{};
  all = Sums{};
  bad = false;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    const Sums s{s_wave[0][w], s_wave[1][w], s_wave[2][w]};
    if (w < wave) base = Sums{base.taken + s.taken, base.given + s.given, base.work + s.work};
    all = Sums{all.taken + s.taken, all.given + s.given, all.work + s.work};
    bad |= s_wave[3][w] != 0;
  }
  return Sums{base.taken + upto.taken - mine.taken, base.given + upto.given - mine.given, base.work + upto.work - mine.work};
}

// What the slots of a stream's new tokens come from, and its new span, in LDS.
constexpr int kStreamWords = 7;

// A thread has CHUNK consecutive slots: one search for their stream, and few numbers of pages.
template <int CHUNK>
__global__ __launch_bounds__(kThreads) void memory_advance_kernel(MemoryAdvanceArgs a) {
  extern __shared__ int lds[];
  __shared__ int s_wave[4][kWaves], s_last;
  const int B = a.B, cols = a.cols, tid = threadIdx.x;
  int* const s_cu = lds;                     // [B + 1]
  int* const s_take = s_cu + B + 1;          // page p >= have is number s_take + p of the free ones
  int* const s_given = s_take + B;           // exclusive sums over the streams
  int* const s_work = s_given + B;
  int* const s_first = s_work + B;           // after forgetting
  int* const s_behind = s_first + B;         // position of the first new token
  int* const s_have = s_behind + B;
  const bool moved = a.table_out != a.table;
  const int head = a.pool[0], n_free = a.pool[1];
  auto step_of = [&](int b, int fresh) {
    const int2 span = a.span[b];
    return stream_step(span.x, span.y, a.drop ? a.drop[b] : 0, fresh, a.page_bits, cols);
  };

  const int per = (B + kThreads - 1) / kThreads, b0 = tid * per, b1 = min(B, b0 + per);
  bool bad = false;
  Sums mine{};
  for (int b = b0; b < b1; ++b) {
    const int c0 = a.cu[b], c1 = a.cu[b + 1];
    s_cu[b] = c0;
    if (b == B - 1) s_cu[B] = c1;
    const bool wrong = c0 < 0 || c1 < c0 || c1 > a.n_new || (b == 0 && c0 != 0);
    const StreamStep s = step_of(b, wrong ? -1 : c1 - c0);
    s_take[b] = mine.taken - s.have;
    s_given[b] = mine.given;
    s_work[b] = mine.work;
    s_first[b] = s.first;
    s_behind[b] = s.first + s.held;
    s_have[b] = s.have;
    if (s.bad) {
      bad = true;
      continue;
    }
    mine.taken += s.taken;
    mine.given += s.given;
    mine.work += s.given + s.taken + (moved ? s.kept : 0);
  }
  Sums all;
  const Sums base = sums_before(mine, all, bad, s_wave);
  for (int b = b0; b < b1; ++b) {
    s_take[b] += base.taken;
    s_given[b] += base.given;
    s_work[b] += base.work;
  }
  __syncthreads();
  const bool refused = bad || head < 0 || head >= a.n_pages || n_free < 0 || n_free > a.n_pages || all.taken > n_free ||
                       all.given > a.n_pages - n_free;
  const int at = blockIdx.x * kThreads + tid, step = gridDim.x * kThreads;
  if (refused) {
    for (int m = at; m < a.n_new; m += step) a.slots[m] = -1;
    if (moved)
      for (size_t i = at; i < (size_t)B * cols; i += step) a.table_out[i] = a.table[i];
    if (at == 0) *a.err_flag = 1;
  } else {
    auto place = [&](int i) { return i >= a.n_pages ? i - a.n_pages : i; };
    // page numbers: what is read for the first one is on its way while the slots are worked out
    struct Page {
      PageWork w;
      size_t entry;
      int old, fresh, back;
    };
    auto ask = [&](int i) {
      const int b = stream_of(s_work, B, i);
      const StreamStep s = step_of(b, s_cu[b + 1] - s_cu[b]);
      Page p{};
      p.w = page_work(s, i - s_work[b], cols);
      p.entry = (size_t)b * cols + p.w.column;
      p.back = place(head + n_free + s_given[b] + p.w.given);
      if (p.w.given >= 0 || p.w.kept) p.old = a.table[p.entry];
      if (p.w.taken >= 0) p.fresh = a.free[place(head + s_take[b] + s.have + p.w.taken)];
      return p;
    };
    auto put = [&](const Page& p) {
      if (p.w.given >= 0) a.free[p.back] = p.old;
      if (p.w.taken >= 0) a.table_out[p.entry] = p.fresh;
      if (p.w.kept) a.table_out[p.entry] = p.old;
    };
    Page first{};
    if (at < all.work) first = ask(at);
    const int n = s_cu[B], page_mask = (1 << a.page_bits) - 1;
    for (int m0 = at * CHUNK; m0 < a.n_new; m0 += step * CHUNK) {
      int slot[CHUNK], b = 0, end = -1, from = 0, seen = -1, id = 0;
#pragma unroll
      for (int c = 0; c < CHUNK; ++c) {
        const int m = m0 + c;
        slot[c] = -1;
        if (m >= n) continue;
        if (m >= end) {
          // (the first of them looks for its stream; behind its end the next that has tokens)
          if (c == 0) b = stream_of(s_cu, B, m);
          else
            while (s_cu[b + 1] <= m) ++b;
          end = s_cu[b + 1];
          from = s_behind[b] - s_cu[b];
          seen = -1;
        }
        const int p = from + m, page = p >> a.page_bits;
        if (page != seen) {
          id = page < s_have[b] ? a.table[(size_t)b * cols + ring_column(page, cols)] : a.free[place(head + s_take[b] + page)];
          if ((unsigned)id >= (unsigned)a.n_pages) *a.err_flag = 1;   // (a table or a list that no step has left)
          seen = page;
        }
        if ((unsigned)id < (unsigned)a.n_pages) slot[c] = (id << a.page_bits) | (p & page_mask);
      }
#pragma unroll
      for (int c = 0; c < CHUNK; ++c)
        if (m0 + c < a.n_new) a.slots[m0 + c] = slot[c];
    }
    if (at < all.work) put(first);
    for (int i = at + step; i < all.work; i += step) put(ask(i));
  }
  // The new spans may lie over the old ones: then they are written by the workgroup that is done last, when nobody reads the
  // old ones any more.
  const bool over = a.span_out == a.span || a.pool_out == a.pool;
  __syncthreads();
  if (gridDim.x > 1 && over) {
    if (tid == 0) {
      s_last = __hip_atomic_fetch_add(a.arrived, 1, __ATOMIC_ACQ_REL, __HIP_MEMORY_SCOPE_AGENT) == (int)gridDim.x - 1;
      if (s_last) __hip_atomic_store(a.arrived, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    __syncthreads();
    if (!s_last) return;
  } else if (blockIdx.x > 0) {
    return;
  }
  for (int b = b0; b < b1; ++b)
    a.span_out[b] = refused ? a.span[b] : make_int2(s_first[b], s_behind[b] - s_first[b] + s_cu[b + 1] - s_cu[b]);
  if (tid == 0) {
    a.pool_out[0] = refused ? head : head + all.taken - (head + all.taken >= a.n_pages ? a.n_pages : 0);
    a.pool_out[1] = refused ? n_free : n_free - all.taken + all.given;
  }
}

template <int CHUNK>
hipError_t launch(const MemoryAdvanceArgs& a, int grid, hipStream_t s) {
  static DeviceOnce once;
  if (hipError_t e = allow_lds(memory_advance_kernel<CHUNK>, (kStreamWords * kMemoryMaxStreams + 1) * sizeof(int), &once); e != hipSuccess) return e;
  hipLaunchKernelGGL(memory_advance_kernel<CHUNK>, dim3(grid), dim3(kThreads), (size_t)(kStreamWords * a.B + 1) * sizeof(int), s, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_memory_advance(const MemoryAdvanceArgs& a, int cus, hipStream_t s) {
  const AdvanceLaunch l = advance_launch(a.n_new, a.B, a.cols, a.n_pages, a.drop != nullptr, a.table_out != a.table, cus);
  return l.chunk == 4 ? launch<4>(a, l.grid, s) : launch<1>(a, l.grid, s);
}

}  // namespace cfdetr
