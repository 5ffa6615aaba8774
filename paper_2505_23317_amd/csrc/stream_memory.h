// Arithmetic of a paged stream memory, the same on the host and the GPU (no HIP here: the tests build it for the host).
//
// A stream holds `held` tokens from position `first` on; the token at position p lies in page table[(p >> page_bits) mod cols]
// at place p mod page.  Page numbers go round in the table's columns, so that tokens can be forgotten in front while
// others come behind: first < cols pages, and what is held and added spans cols pages at most, so that a position stays below
// 2 cols pages.  cols pages are 2^29 tokens at most: sums of three such numbers fit 32 bits.
#pragma once
#include <cstdint>

namespace cfdetr {

constexpr int kMemoryMaxStreams = 4096;
constexpr int kMemoryMaxRing = 1 << 29;     // tokens of a table's columns
constexpr int kMemoryMaxTable = 1 << 28;    // page numbers of a table

constexpr int ring_column(int page, int cols) { return page >= cols ? page - cols : page; }

// Where a stream's tokens lie, or `bad`: a span that no step leaves.
constexpr bool span_is_bad(int first, int held, int page_bits, int cols) {
  const int ring = cols << page_bits;
  if (first < 0 || first >= ring || held < 0 || held > ring) return true;
  return held > 0 && ((first + held - 1) >> page_bits) - (first >> page_bits) >= cols;
}

// One step of a stream: `drop` tokens forgotten in front (all, if it is that many or more), `fresh` added behind.
struct StreamStep {
  int first, held;       // after forgetting
  int lo, given;         // pages given back: the `given` from page lo on (in the old positions)
  int from, kept;        // pages kept: `kept` from page `from` on (in the new positions, as below)
  int have, taken;       // pages taken: `taken` from page `have` on
  bool bad;
};
constexpr StreamStep stream_step(int first, int held, int drop, int fresh, int page_bits, int cols) {
  StreamStep s{};
  const int ring = cols << page_bits, round = (1 << page_bits) - 1;
  s.bad = span_is_bad(first, held, page_bits, cols) || drop < 0 || fresh < 0 || fresh > ring;
  if (s.bad) return s;
  s.lo = first >> page_bits;
  if (drop >= held) {
    s.given = held > 0 ? ((first + held + round) >> page_bits) - s.lo : 0;
  } else {
    s.first = first + drop;
    s.held = held - drop;
    s.given = (s.first >> page_bits) - s.lo;
    if (s.first >= ring) s.first -= ring;
    s.from = s.first >> page_bits;
    s.have = (s.first + s.held + round) >> page_bits;
    s.kept = s.have - s.from;
  }
  s.taken = ((s.first + s.held + fresh + round) >> page_bits) - s.have;
  s.bad = s.have + s.taken - s.from > cols;
  return s;
}

// Work on a stream's page numbers, one number at a time: the given ones, then the taken ones, then (where the new table is
// another) the kept ones.  A column whose page is given back may get a taken one at once: the same thread then does both,
// so that the old number is read before the new one is written over it.
struct PageWork {
  int column;
  int given, taken;   // which of the given and taken ones it is, or -1
  bool kept;
};
constexpr PageWork page_work(const StreamStep& s, int i, int cols) {
  PageWork w{-1, -1, -1, false};
  if (i < s.given) {
    w.given = i;
    w.column = ring_column(s.lo + i, cols);
    int t = w.column - ring_column(s.have, cols);
    if (t < 0) t += cols;
    if (t < s.taken) w.taken = t;
    return w;
  }
  i -= s.given;
  if (i < s.taken) {
    w.column = ring_column(s.have + i, cols);
    int g = w.column - ring_column(s.lo, cols);
    if (g < 0) g += cols;
    if (g >= s.given) w.taken = i;   // (else with the given one)
    return w;
  }
  w.kept = true;
  w.column = ring_column(s.from + i - s.taken, cols);
  return w;
}

// Last i < n with offsets[i] <= at (offsets[0] = 0, ascending): the stream that a token belongs to.
template <typename Offsets>
constexpr int stream_of(const Offsets& offsets, int n, int at) {
  int lo = 0, hi = n - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (offsets[mid] <= at) lo = mid;
    else hi = mid - 1;
  }
  return lo;
}

// ---- attention: streams cut into pieces ---------------------------------------------
// A stream's tokens are units of 32 positions that lie on multiples of 32: at most 2^24 and one.
constexpr int kMemoryUnit = 32;
constexpr int units_of(int first, int held) { return held > 0 ? (first + held - 1) / kMemoryUnit - first / kMemoryUnit + 1 : 0; }

// Units of all pieces but a stream's last, which is shorter: at most as many pieces as the length would make of one stream,
// and one more a stream.  Few streams: no more pieces than places.  The launch and the pieces' room count on `most_pieces`.
constexpr int cut_length(int units, int streams, int places, int least) {
  const int room = 2 * streams <= places ? places - streams : places;
  const int even = (units + room - 1) / room;
  return even > least ? even : least;
}
constexpr int most_pieces(int streams, int places) { return places + streams; }

// Pieces of a stream of n units: one up to `whole`, then ceil(n / length) by a product with 1 / length that may be one off.
constexpr int pieces_of(int n, int length, float per_length, int whole) {
  if (n <= whole) return n > 0 ? 1 : 0;
  int q = (int)((float)n * per_length);
  q += q * length < n ? 1 : 0;
  q += q * length < n ? 1 : 0;
  return q - ((q - 1) * length >= n ? 1 : 0);
}

// ---- steps: workgroups --------------------------------------------------------------
// Workgroups of a step, one a CU at most, and consecutive slots of a thread.  What the step has to do is known on the device only: a
// slot for every new token, and of page numbers those that may go or move, all entries of a table that lies apart, and of
// one in place, if tokens are forgotten, as many as there are pages at most.  Two rounds of numbers a workgroup, us: 300 streams of 700 tokens, page 16, in
// place, all lost 10.7 (one workgroup 46, eight rounds 18, one 9.4), a quarter of 1,024 of 3,000, page 32, 11.1 (46, 12.2, 12.0), one of 200,000,
// page 8, 8.9 (40.5, 12.2, 8.3); where they only slide by a token several workgroups take longer, 300 streams 8.1 (one 7.1).  Apart, 300 streams
// that slide 9.9 (eight rounds 14.5, one 8.5).
constexpr int kAdvanceThreads = 512;
struct AdvanceLaunch {
  int chunk, grid;
};
constexpr AdvanceLaunch advance_launch(int n_new, int streams, int cols, int n_pages, bool forgets, bool apart, int cus) {
  constexpr int64_t T = kAdvanceThreads;
  const int64_t entries = (int64_t)streams * cols;
  const int64_t numbers = apart ? entries : !forgets ? 0 : entries < n_pages ? entries : n_pages;
  const int chunk = n_new > T * cus ? 4 : 1;
  const int64_t slots = (n_new + chunk * T - 1) / (chunk * T), pages = (numbers + 2 * T - 1) / (2 * T);
  const int64_t most = slots > pages ? slots : pages;
  return {chunk, (int)(most < 1 ? 1 : most < cus ? most : cus)};
}

// Why a memory's sizes are refused; null: they are not.
constexpr const char* check_memory_sizes(int page_size, int n_pages, int max_pages, int max_streams, int kv_heads, int heads) {
  if (page_size < 8 || page_size > 1024 || (page_size & (page_size - 1)) != 0) return "page_size must be a power of two from 8 to 1024";
  if (n_pages < 1 || (int64_t)n_pages * page_size > 0x7FFFFFFF) return "n_pages must be at least 1, and slots are counted with 31 bits";
  if (max_pages < 1 || (int64_t)max_pages * page_size > kMemoryMaxRing) return "max_pages must be at least 1 and hold 2^29 tokens at most";
  if (max_streams < 1 || max_streams > kMemoryMaxStreams) return "max_streams must be 1..4096";
  if ((int64_t)max_streams * max_pages > kMemoryMaxTable) return "a table has at most 2^28 page numbers";
  if (kv_heads < 1 || kv_heads > heads || heads % kv_heads != 0) return "n_kv_heads must divide n_heads";
  return nullptr;
}

}  // namespace cfdetr
