// libqkn, part 6: the book of a paged cache's pages, and copies of pages (AMD MI355X, gfx950).
//
// The book's calls are integer work on small arrays, each a chain of latencies: taking pages is one workgroup, so that
// ranks among the free pages and among the rows' needs need no second launch; the rest has a workgroup for a row or for
// 4096 pages. 8 rows that are emptied and grown again by up to 2048 tokens each, in a book of 8192 pages: 11.7 us; 64 rows
// emptied and forked from 16, with the copies of four layers: 18.9. (Of a profiler's dispatches, which are longer than the
// same launches in a row without it: 2.7 emptying, 4.7 taking, 4.9 the slots; 2.6, 5.9 taking, 2.6 sharing, 8.1 the copy.)
// Sums over lanes go by DPP (through LDS, in 64 bits, the 8 rows took 15.3 us for 12.7), the slots of many tokens are a launch
// of their own (in the one workgroup 17.8), and a free page's row is looked for by a thread for each page in order, behind
// barriers that wait for LDS alone (by the thread that read the page's count, four one after the other, taking took 5.6 and
// 8.0 us in the profiler). Free pages are looked for 16384 pages a pass, each pass a trip to memory behind the one before,
// and lowest-first packs the pages in use at the front: 64 rows that need a page each behind 7360 used pages of 8192 take 5.1
// us, behind 58944 of 65536 8.6, behind 471808 of 524288 38.9; rows that need none 3.0 whatever the pool. The moves of 4096
// pages: 4.7 and 4.6 in two launches (4.6, 7.1 and 4.6 with the counts in a launch of their own; in the profiler). Copies are
// bound by bytes.

#include <string.h>

#include "qkn_block.h"
#include "qkn_pages.h"

namespace {

using namespace qkn_block;
using qkn_host::Span;
using qkn_host::spans_overlap;

typedef int i32x4 __attribute__((ext_vector_type(4)));

// ------------------------------------------------------------------ sums over a workgroup

// x plus what lanes further back have (DPP: through no memory).
template <int CTRL, int ROWS>
__device__ __forceinline__ uint32_t add_from(uint32_t x) {
  return x + static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(x), CTRL, ROWS, 0xf, false));
}
__device__ __forceinline__ uint32_t wave_sums(uint32_t x) {  // inclusive
  x = add_from<0x111, 0xf>(x);  // 1, 2, 4, 8 lanes back in the row of 16
  x = add_from<0x112, 0xf>(x);
  x = add_from<0x114, 0xf>(x);
  x = add_from<0x118, 0xf>(x);
  x = add_from<0x142, 0xa>(x);     // the end of row 0 (2) into row 1 (3)
  return add_from<0x143, 0xc>(x);  // the end of row 1 into rows 2 and 3
}

// Barrier for what is in LDS: loads and stores of global memory stay under way across it.
__device__ __forceinline__ void lds_barrier() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(0xC07F);  // lgkmcnt(0)
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// Two 32-bit numbers that are summed side by side.
struct Pair {
  uint32_t a, b;
};
__device__ __forceinline__ Pair operator+(Pair x, Pair y) { return Pair{x.a + y.a, x.b + y.b}; }
__device__ __forceinline__ Pair operator-(Pair x, Pair y) { return Pair{x.a - y.a, x.b - y.b}; }
// Sums of up to 1024 numbers below 2^31, whose 20 lower bits and the rest are summed apart.
__device__ __forceinline__ Pair apart(int64_t x) {
  return Pair{static_cast<uint32_t>(x) & 0xfffffu, static_cast<uint32_t>(x >> 20)};
}
__device__ __forceinline__ int64_t together(Pair x) { return (static_cast<int64_t>(x.b) << 20) + x.a; }

// Inclusive sums over the threads, and the sum of all. `room`: one value a wavefront; free again behind the next barrier.
template <int WAVES>
__device__ __forceinline__ Pair group_sums(Pair x, Pair (&room)[WAVES], Pair& all) {
  const int wave = __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x) >> 6), lane = static_cast<int>(threadIdx.x) & 63;
  const Pair s = {wave_sums(x.a), wave_sums(x.b)};
  if (lane == 63) room[wave] = s;
  lds_barrier();
  const Pair w = lane < WAVES ? room[lane] : Pair{0, 0};
  const Pair upto = {wave_sums(w.a), wave_sums(w.b)};  // those up to each wavefront
  const auto at = [&](int l) {
    return Pair{static_cast<uint32_t>(__builtin_amdgcn_readlane(static_cast<int>(upto.a), l)),
                static_cast<uint32_t>(__builtin_amdgcn_readlane(static_cast<int>(upto.b), l))};
  };
  all = at(WAVES - 1);
  return wave ? s + at(wave - 1) : s;
}

// ------------------------------------------------------------------ taking pages

constexpr int kMost = QKN_PAGES_MOST, kTakeWaves = kMost / 64;

struct Book {
  int32_t* refs;
  int32_t* table;
  int32_t* kv_len;
  int64_t num_pages, ld_table;
  int32_t rows, page_shift;
};

struct TakeParams {
  Book b;
  const int32_t* which;   // grow: rows, or NULL; fork: `to`
  const int32_t* from;    // fork
  const int32_t* count;   // grow
  int32_t n;
  int64_t T;
  int64_t* slots;
  int32_t* pos;
  int32_t *src, *dst, *done;
};

// refs[at .. at + 3]; past the end `past`. at is a multiple of 4, refs of 4 bytes' alignment at least.
__device__ __forceinline__ i32x4 refs_at(const int32_t* refs, int64_t at, int64_t num_pages, int32_t past) {
  typedef int i32x4_any __attribute__((ext_vector_type(4), aligned(4)));
  if (at + 4 <= num_pages) return *reinterpret_cast<const i32x4_any*>(refs + at);
  i32x4 r;
#pragma unroll
  for (int e = 0; e < 4; ++e) r[e] = at + e < num_pages ? refs[at + e] : past;
  return r;
}

__device__ __forceinline__ int64_t pages_for(int64_t tokens, int shift) { return (tokens + (int64_t{1} << shift) - 1) >> shift; }

// The first i with upto[i] > r: upto ascending, r below the last.
__device__ __forceinline__ int holder(const int32_t* upto, int n, int32_t r) {
  int lo = 0, hi = n - 1;
  while (lo < hi) {
    const int mid = (lo + hi) / 2;
    if (upto[mid] > r) hi = mid;
    else lo = mid + 1;
  }
  return lo;
}

// Slots and positions of the four tokens t0, t0 + THREADS, .. (of all tokens where pages are taken, T up to 4 * kMost). A
// token's table entry is a trip to memory, so the four go out together.
template <int THREADS>
__device__ __forceinline__ void list_tokens(const TakeParams& p, const int32_t* rows, const int32_t* length, const int32_t* first,
                                            const int32_t* tokens, int64_t all, int64_t t0) {
  const int shift = p.b.page_shift;
  int32_t pos[4], page[4];
#pragma unroll
  for (int x = 0; x < 4; ++x) {
    const int64_t t = t0 + x * THREADS;
    pos[x] = 0;
    page[x] = -1;
    if (t >= p.T || t >= all) continue;
    const int at = holder(tokens, p.n, static_cast<int32_t>(t));
    if (first[at] < 0) continue;  // refused
    pos[x] = length[at] + static_cast<int32_t>(t - (at ? tokens[at - 1] : 0));
    page[x] = p.b.table[rows[at] * p.b.ld_table + (pos[x] >> shift)];
  }
#pragma unroll
  for (int x = 0; x < 4; ++x) {
    const int64_t t = t0 + x * THREADS;
    if (t >= p.T) break;
    if (p.slots) p.slots[t] = page[x] < 0 ? -1 : (static_cast<int64_t>(page[x]) << shift) + (pos[x] & ((1 << shift) - 1));
    if (p.pos) p.pos[t] = pos[x];
  }
}

// One workgroup, thread i for entry i of the list. Sums that pass 2^31 are cut: no pool has as many pages, no list that
// is written as many tokens.
template <bool FORK>
__global__ __launch_bounds__(kMost) void qkn_pages_take(const TakeParams p) {
  __shared__ Pair room[2][kTakeWaves];
  __shared__ __align__(16) int32_t rows[kMost];
  __shared__ int32_t upto[kMost], first[kMost], tokens[kMost], length[kMost];
  __shared__ int32_t got[4 * kMost];  // free pages in order
  __shared__ struct { int64_t entry; int32_t count; } partly;  // the table's entries of a row that did not get all its pages
  const int i = static_cast<int>(threadIdx.x), shift = p.b.page_shift;
  const int64_t most = p.b.ld_table << shift;
  // the first pages' counts are asked for before they are needed
  i32x4 r[4];
  const auto ask = [&](int64_t base) {
#pragma unroll
    for (int k = 0; k < 4; ++k) r[k] = refs_at(p.b.refs, base + (k * kMost + i) * 4, p.b.num_pages, 1);
  };
  ask(0);
  const auto cut = [](int64_t x) { return static_cast<int32_t>(x < 0x7fffffff ? x : 0x7fffffff); };

  const int32_t row = i >= p.n ? -1 : p.which ? p.which[i] : i;
  const int32_t from = i < p.n && FORK ? p.from[i] : row;
  int64_t more = i < p.n && !FORK ? p.count[i] : 0;
  rows[i] = row;
  if (i == 0) partly = {0, 0};
  bool fine = row >= 0 && row < p.b.rows && from >= 0 && from < p.b.rows;
  const int64_t len = fine ? p.b.kv_len[from] : 0;
  const int32_t old = FORK && fine ? p.b.kv_len[row] : 0;
  lds_barrier();
  if (p.which) {  // listed before
    for (int j = 0; j < i && fine; j += 4) {
      const i32x4 r = *reinterpret_cast<const i32x4*>(&rows[j]);
#pragma unroll
      for (int e = 0; e < 4; ++e) fine = fine && !(j + e < i && r[e] == row);
    }
  }
  fine = fine && old == 0 && more >= 0 && len >= 0 && len + more <= most;
  if (more < 0) more = 0;
  const int64_t have = FORK ? len >> shift : pages_for(len, shift);
  const int64_t need = fine ? pages_for(len + more, shift) - have : 0;
  // no call's row is both: `from` has tokens here, and `to` none
  const int32_t last = FORK && need ? p.b.table[from * p.b.ld_table + have] : -1;
  Pair all_needs, all_more = {0, 0};
  const int64_t ends = together(group_sums<kTakeWaves>(apart(need), room[0], all_needs)), total = together(all_needs);
  const int64_t token_end = FORK ? 0 : together(group_sums<kTakeWaves>(apart(more), room[1], all_more));
  const int64_t all_tokens = together(all_more);
  upto[i] = cut(ends);
  first[i] = static_cast<int32_t>(have);
  length[i] = static_cast<int32_t>(len);
  if (!FORK) tokens[i] = cut(token_end);
  lds_barrier();

  // free pages, lowest first, to the needs in order
  int64_t found = 0;
  for (int64_t base = 0; base < p.b.num_pages && found < total; base += 16 * kMost) {
    if (base) ask(base);
    uint32_t c[4];  // free pages of this thread, of each k
#pragma unroll
    for (int k = 0; k < 4; ++k) c[k] = (r[k][0] == 0) + (r[k][1] == 0) + (r[k][2] == 0) + (r[k][3] == 0);
    const Pair counts = {c[0] | c[1] << 16, c[2] | c[3] << 16};  // up to 4096 each in 16 bits
    Pair all;
    const Pair before = group_sums<kTakeWaves>(counts, room[0], all) - counts;
    int64_t start = found;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int half = 16 * (k % 2), here = ((k < 2 ? all.a : all.b) >> half) & 0xffff;
      if (here == 0 || start >= total) continue;
      int at = ((k < 2 ? before.a : before.b) >> half) & 0xffff;
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (r[k][e] == 0) got[at++] = static_cast<int32_t>(base + (k * kMost + i) * 4 + e);
      lds_barrier();
      for (int x = i; x < here && start + x < total; x += kMost) {
        const int32_t page = got[x], rank = static_cast<int32_t>(start + x);
        const int to = holder(upto, p.n, rank);
        p.b.table[rows[to] * p.b.ld_table + first[to] + (rank - (to ? upto[to - 1] : 0))] = page;
        p.b.refs[page] = 1;
        if (FORK) p.dst[to] = page;
      }
      lds_barrier();
      start += here;
    }
    found = start;
    lds_barrier();  // room
  }
  if (!FORK || found < total) __syncthreads();  // the table's entries are there

  const bool served = fine && (need == 0 || ends <= found);
  if (found < total) {
    // The first row that did not get all of its pages gives back what it got: all threads do, four entries each at a time.
    // A row refused in a pool of 65536 pages takes 39.6 us, a served one 34.3 (by that row's thread, each entry behind the one
    // before, 7.4 ms).
    if (need > 0 && !served && ends - need < found) {
      partly.entry = row * p.b.ld_table + have;
      partly.count = static_cast<int32_t>(found - (ends - need));
    }
    lds_barrier();
    const int32_t* entries = p.b.table + partly.entry;
    for (int32_t x0 = i; x0 < partly.count; x0 += 4 * kMost) {
      int32_t page[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) page[k] = x0 + k * kMost < partly.count ? entries[x0 + k * kMost] : -1;
#pragma unroll
      for (int k = 0; k < 4; ++k)
        if (page[k] >= 0) p.b.refs[page[k]] = 0;
    }
  }
  if (i < p.n) {
    p.done[i] = served ? static_cast<int32_t>(len + more) : -1;
    if (served) p.b.kv_len[row] = static_cast<int32_t>(len + more);
    if (FORK) {
      p.src[i] = served && need ? last : -1;
      if (!(served && need)) p.dst[i] = -1;
    }
  }
  if constexpr (!FORK) {
    if ((!p.slots && !p.pos) || p.T > 4 * kMost) return;  // qkn_pages_slots
    if (!served) first[i] = -1;
    lds_barrier();
    list_tokens<kMost>(p, rows, length, first, tokens, all_tokens, i);
  }
}

// The slots of many new tokens, kMany a workgroup: what the workgroup above knows of the rows is found again.
constexpr int kManyThreads = 256, kMany = 4 * kManyThreads;
__global__ __launch_bounds__(kManyThreads) void qkn_pages_slots(const TakeParams p) {
  __shared__ Pair room[kManyThreads / 64];
  __shared__ int32_t rows[kMost], first[kMost], tokens[kMost], length[kMost];
  const int i0 = 4 * static_cast<int>(threadIdx.x);
  int64_t count[4], sum = 0;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const int i = i0 + e;
    const int32_t c = i < p.n ? p.count[i] : 0, done = i < p.n ? p.done[i] : -1;
    count[e] = c < 0 ? 0 : c;
    sum += count[e];
    rows[i] = i >= p.n ? -1 : p.which ? p.which[i] : i;
    first[i] = done < 0 ? -1 : 0;
    length[i] = static_cast<int32_t>(done - count[e]);
  }
  // up to four numbers below 2^31 a thread: the lower parts' sums stay below 2^32
  Pair all_more;
  int64_t end = together(group_sums<kManyThreads / 64>(apart(sum), room, all_more)) - sum;
  const int64_t all = together(all_more);
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    end += count[e];
    tokens[i0 + e] = static_cast<int32_t>(end < 0x7fffffff ? end : 0x7fffffff);
  }
  lds_barrier();
  list_tokens<kManyThreads>(p, rows, length, first, tokens, all, static_cast<int64_t>(blockIdx.x) * kMany + threadIdx.x);
}

// The whole pages of forked rows: 1024 entries of a row a workgroup.
constexpr int kShare = 1024, kRowThreads = 256;
__global__ __launch_bounds__(kRowThreads) void qkn_pages_share(const TakeParams p) {
  const int i = static_cast<int>(blockIdx.x);
  const int64_t whole = p.done[i] >> p.b.page_shift;  // -1 (refused): -1
  const int64_t e0 = static_cast<int64_t>(blockIdx.y) * kShare;
  if (e0 >= whole) return;
  const int32_t* from = p.b.table + p.from[i] * p.b.ld_table;
  int32_t* to = p.b.table + p.which[i] * p.b.ld_table;
  for (int64_t e = e0 + threadIdx.x; e < whole && e < e0 + kShare; e += kRowThreads) {
    const int32_t page = from[e];
    to[e] = page;
    if (page >= 0 && page < p.b.num_pages) atomicAdd(&p.b.refs[page], 1);  // integers: in any order the same
  }
}

__global__ __launch_bounds__(kRowThreads) void qkn_pages_drop(const TakeParams p) {
  __shared__ int32_t length;
  const int32_t row = p.which ? p.which[blockIdx.x] : static_cast<int32_t>(blockIdx.x);
  if (row < 0 || row >= p.b.rows) return;
  if (threadIdx.x == 0) length = atomicExch(&p.b.kv_len[row], 0);  // a row listed again finds 0
  __syncthreads();
  const int64_t most = p.b.ld_table << p.b.page_shift, len = length < 0 ? 0 : length < most ? length : most;
  const int64_t pages = pages_for(len, p.b.page_shift);
  for (int64_t e = threadIdx.x; e < pages; e += kRowThreads) {
    const int32_t page = p.b.table[row * p.b.ld_table + e];
    if (page >= 0 && page < p.b.num_pages) atomicSub(&p.b.refs[page], 1);
  }
}

// ------------------------------------------------------------------ moving pages to the front

// Of U pages in use, the k-th last, p, moves to the k-th first free one if that is before p, which is to say if more
// than k free pages are before p; likewise for free pages. So every page finds its part of a move from the number of
// pages in use before it.
constexpr int kScan = 4096, kScanThreads = 1024, kScanWaves = kScanThreads / 64;

struct MoveParams {
  Book b, out;
  int32_t *src, *dst;
  int32_t n;
  int32_t* counts;   // pages in use of each kScan pages (more than kFewBlocks of them); the last one: moves
  int32_t* moved;    // [num_pages]: its move, -1: stays, -2: a move's end
  int32_t blocks;
};

__device__ __forceinline__ int used_of(const MoveParams& p, int block, bool (&used)[4], int64_t& at) {
  at = static_cast<int64_t>(block) * kScan + 4 * threadIdx.x;
  const i32x4 r = refs_at(p.b.refs, at, p.b.num_pages, 0);
#pragma unroll
  for (int e = 0; e < 4; ++e) used[e] = r[e] != 0;
  return used[0] + used[1] + used[2] + used[3];
}
// Up to so many blocks of pages, each workgroup counts all of them itself: a launch less.
constexpr int kFewBlocks = 16;

__global__ __launch_bounds__(kScanThreads) void qkn_pages_count(const MoveParams p) {
  __shared__ Pair room[kScanWaves];
  bool used[4];
  int64_t at;
  Pair all;
  const int c = used_of(p, static_cast<int>(blockIdx.x), used, at);
  group_sums<kScanWaves>(Pair{static_cast<uint32_t>(c), 0}, room, all);
  if (threadIdx.x == 0) p.counts[blockIdx.x] = static_cast<int32_t>(all.a);
}

__global__ __launch_bounds__(kScanThreads) void qkn_pages_moves(const MoveParams p) {
  __shared__ Pair room[2][kScanWaves];
  bool used[4];
  int64_t at;
  const int64_t c = used_of(p, static_cast<int>(blockIdx.x), used, at);
  uint32_t mine = 0, others = 0;  // pages in use in earlier blocks, in all
  if (p.blocks <= kFewBlocks) {
    for (int b = 0; b < p.blocks; ++b) {
      bool u[4];
      int64_t a;
      const int n = b == static_cast<int>(blockIdx.x) ? static_cast<int>(c) : used_of(p, b, u, a);
      others += n;
      mine += b < static_cast<int>(blockIdx.x) ? n : 0;
    }
  } else {
    for (int b = static_cast<int>(threadIdx.x); b < p.blocks; b += kScanThreads) {
      others += p.counts[b];
      mine += b < static_cast<int>(blockIdx.x) ? p.counts[b] : 0;
    }
  }
  Pair sums, here;
  group_sums<kScanWaves>(Pair{mine, others}, room[0], sums);
  const int64_t U = sums.b;
  const Pair own = {static_cast<uint32_t>(c), 0};
  int64_t used_before = sums.a + static_cast<int64_t>((group_sums<kScanWaves>(own, room[1], here) - own).a);
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    // the free pages before page U are as many as the moves
    if (at + e == U) p.counts[p.blocks] = static_cast<int32_t>(U - used_before);
    if (at + e >= p.b.num_pages) break;
    const int64_t free_before = at + e - used_before;
    const int64_t k = used[e] ? U - 1 - used_before : free_before;
    const bool moves = k < p.n && k < (used[e] ? free_before : U - used_before);
    if (moves) (used[e] ? p.src : p.dst)[k] = static_cast<int32_t>(at + e);
    p.moved[at + e] = !moves ? -1 : used[e] ? static_cast<int32_t>(k) : -2;
    used_before += used[e];
  }
  if (U == static_cast<int64_t>(p.blocks) * kScan && blockIdx.x == 0 && threadIdx.x == 0) p.counts[p.blocks] = 0;  // all in use
}

__global__ __launch_bounds__(kRowThreads) void qkn_pages_apply(const MoveParams p) {
  const int64_t i = static_cast<int64_t>(blockIdx.x) * kRowThreads + threadIdx.x;
  for (int64_t k = i; k < p.n; k += static_cast<int64_t>(gridDim.x) * kRowThreads)
    if (k >= p.counts[p.blocks]) p.src[k] = p.dst[k] = -1;
  if (i < p.b.num_pages) {
    const int32_t k = p.moved[i];
    if (k != -2) {  // else the page that moves here writes it
      const int32_t r = p.b.refs[i];
      if (k >= 0) p.out.refs[p.dst[k]] = r;
      p.out.refs[i] = k >= 0 ? 0 : r;
    }
    return;
  }
  const int64_t x = i - p.b.num_pages;
  if (x >= p.b.rows * p.b.ld_table) return;
  const int64_t row = x / p.b.ld_table, e = x - row * p.b.ld_table;
  int32_t page = p.b.table[x];
  if ((e << p.b.page_shift) < p.b.kv_len[row] && page >= 0 && page < p.b.num_pages) {
    const int32_t k = p.moved[page];
    if (k >= 0) page = p.dst[k];
  }
  p.out.table[x] = page;
}

// ------------------------------------------------------------------ copies

// A page of a pool: `outer` times `inner` runs of bytes; where runs touch they are one.
struct CopyPool {
  unsigned char* base;
  int64_t page, outer, inner;  // strides
  int32_t units;               // vectors of a page
  FastDiv of_outer, of_inner;  // vectors of an outer, of an inner run
};
constexpr int kCopyThreads = 256, kCopyPools = 40;
struct CopyParams {
  CopyPool pool[kCopyPools];
  const int32_t *src, *dst;
  int32_t n, each;             // pairs; pairs of a workgroup
  int64_t num_pages;
  int32_t chunks;
};

// EACH: vectors of a thread. Pages are read as they are (forks read the same one several times: 64 of 16 pages 9.6 us,
// 13.8 with loads past the caches) and written past the caches (980 of 2048 pages of 32 KiB in four layers, 258 MB, with the
// list's launches 59.4 us, 66.3 with stores into them). A workgroup for each pair: 51.7 of those 59.4, 5.7 TB/s the copy.
// 4-bit pages, half of whose pools are exponents, a sixteenth of the codes: 980 of 8 heads of 128 in four layers, 137 MB, 22.1
// us, 6.2 TB/s; 64, 9 MB, 3.2.
template <class U, int EACH>
__global__ __launch_bounds__(kCopyThreads) void qkn_pages_copy_kernel(const CopyParams p) {
  const CopyPool& c = p.pool[blockIdx.y];
  const int chunk = static_cast<int>(blockIdx.x % p.chunks), first = static_cast<int>(blockIdx.x / p.chunks) * p.each;
  const uint32_t u0 = static_cast<uint32_t>(chunk) * (kCopyThreads * EACH) + threadIdx.x;
  if (chunk * (kCopyThreads * EACH) >= c.units) return;
  int64_t off[EACH];
#pragma unroll
  for (int x = 0; x < EACH; ++x) {
    const uint32_t u = u0 + x * kCopyThreads, o = div(u, c.of_outer), in_outer = u - o * c.of_outer.d;
    const uint32_t r = div(in_outer, c.of_inner);
    off[x] = o * c.outer + r * c.inner + static_cast<int64_t>(in_outer - r * c.of_inner.d) * sizeof(U);
  }
  for (int i = first; i < first + p.each && i < p.n; ++i) {
    const int64_t s = p.src[i], d = p.dst[i];
    if (s == d || s < 0 || d < 0 || s >= p.num_pages || d >= p.num_pages) continue;
    const unsigned char* from = c.base + s * c.page;
    unsigned char* to = c.base + d * c.page;
    U v[EACH];
#pragma unroll
    for (int x = 0; x < EACH; ++x)
      if (u0 + x * kCopyThreads < static_cast<uint32_t>(c.units)) v[x] = *reinterpret_cast<const U*>(from + off[x]);
#pragma unroll
    for (int x = 0; x < EACH; ++x)
      if (u0 + x * kCopyThreads < static_cast<uint32_t>(c.units)) __builtin_nontemporal_store(v[x], reinterpret_cast<U*>(to + off[x]));
  }
}

// ------------------------------------------------------------------ host side

bool book_ok(const qkn_pages* b) {
  return b && b->num_pages >= 0 && b->num_pages <= 1 << 24 && b->rows >= 0 && b->ld_table >= 0 && b->page_size >= 1 &&
         b->page_size <= 65536 && !(b->page_size & (b->page_size - 1)) &&
         b->ld_table < (int64_t{1} << 31) / b->page_size;
}
bool book_given(const qkn_pages& b) {
  return (b.refs || !b.num_pages) && (b.table || !(b.rows * b.ld_table)) && (b.kv_len || !b.rows);
}
Book book_of(const qkn_pages& b) {
  return Book{b.refs, b.table, b.kv_len, b.num_pages, b.ld_table, b.rows, log2_of(b.page_size)};
}

// Arrays of a call: outputs overlap nothing.
struct Arrays {
  Span item[12];
  bool out[12];
  int n = 0;
  void add(const void* at, int64_t count, int64_t esz, bool is_out) {
    item[n] = array_span(at, count, esz);
    out[n++] = is_out;
  }
  void book(const qkn_pages& b) {
    add(b.refs, b.num_pages, 4, true);
    add(b.table, b.rows * b.ld_table, 4, true);
    add(b.kv_len, b.rows, 4, true);
  }
  bool overlap() const {
    for (int a = 0; a < n; ++a)
      for (int b = a + 1; b < n; ++b)
        if ((out[a] || out[b]) && spans_overlap(item[a], item[b])) return true;
    return false;
  }
};

bool launch(const void* fn, int64_t x, int64_t y, int threads, const void* params, void* stream) {
  void* args[] = {const_cast<void*>(params)};
  return hipLaunchKernel(fn, dim3(static_cast<unsigned>(x), static_cast<unsigned>(y)), dim3(threads), args, 0,
                         static_cast<hipStream_t>(stream)) == hipSuccess;
}
int dry(const char* name) {
  qkn_host::record_launch(qkn_launch_info{name, 0, 0, 0, 0});
  return QKN_EDRYRUN;
}
int launched(const char* name, int64_t blocks, int threads) {
  qkn_host::record_launch(qkn_launch_info{name, blocks, threads, blocks * (threads / 64), 0});
  return QKN_OK;
}

CopyPool copy_pool(void* base, int64_t page, int64_t head, int64_t token, int64_t row, int64_t heads, int64_t tokens) {
  // the dimension whose elements are further apart outside
  int64_t outer = head, n_outer = heads, inner = token, n_inner = tokens;
  if (n_outer == 1 || (n_inner > 1 && token > head)) {
    outer = token;
    n_outer = tokens;
    inner = head;
    n_inner = heads;
  }
  int64_t run = row;
  if (n_inner == 1 || inner == run) {
    run *= n_inner;
    n_inner = 1;
    inner = run;
  }
  if (n_inner == 1 && (n_outer == 1 || outer == run)) {
    run *= n_outer;
    n_outer = 1;
    outer = inner = run;
  }
  CopyPool c{};
  c.base = static_cast<unsigned char*>(base);
  c.page = page;
  c.outer = outer;
  c.inner = inner;
  c.of_inner.d = static_cast<uint32_t>(run);  // bytes, until the vectors are chosen
  c.of_outer.d = static_cast<uint32_t>(run * n_inner);
  c.units = static_cast<int32_t>(run * n_inner * n_outer);
  return c;
}

// The pools in launches of up to kCopyPools; caches of one size of pool.
int copy_impl(CopyPool* pools, int64_t count, int64_t num_pages, const int32_t* src, const int32_t* dst, int32_t n,
              void* stream) {
  int64_t unit = 16;
  int32_t bytes = 0;
  for (int64_t i = 0; i < count; ++i) {
    const CopyPool& c = pools[i];
    while (unit > 1 && ((reinterpret_cast<uintptr_t>(c.base) | c.page | c.outer | c.inner | c.of_inner.d) & (unit - 1)))
      unit = unit == 16 ? 4 : unit == 4 ? 2 : 1;
    bytes = c.units > bytes ? c.units : bytes;
  }
  CopyParams p;
  memset(&p, 0, sizeof(p));
  for (int64_t i = 0; i < count; ++i) {
    CopyPool c = pools[i];
    c.units /= static_cast<int32_t>(unit);
    c.of_inner = fast_div(static_cast<uint32_t>(c.of_inner.d / unit));
    c.of_outer = fast_div(static_cast<uint32_t>(c.of_outer.d / unit));
    p.pool[i] = c;
  }
  p.src = src;
  p.dst = dst;
  p.n = n;
  p.num_pages = num_pages;
  // 16 KiB a workgroup; 8 where these are few (64 forks: 20.7 and 22.6 us; the 2048 moves above 55.4 and 51.7)
  const auto chunks = [&](int each) { return (bytes / unit + kCopyThreads * each - 1) / (kCopyThreads * each); };
  const int each = unit == 16 && n * count * chunks(4) < 8192 ? 2 : 4;
  p.chunks = static_cast<int32_t>(chunks(each));
  // long lists have few pairs at their front: a workgroup takes several, so that there are not too many of them
  const int64_t all = n * count * p.chunks;
  p.each = static_cast<int32_t>(all / 65536 + 1);
  const int64_t grid = (n + p.each - 1) / p.each * p.chunks;
  if (grid >= int64_t{1} << 31) return QKN_ENOTSUP;
  const char* name = unit == 16 ? "pages_copy<16>" : unit == 4 ? "pages_copy<4>" : unit == 2 ? "pages_copy<2>" : "pages_copy<1>";
  if (qkn_host::validate_only()) return dry(name);
  const void* fn = unit == 16  ? (each == 2 ? reinterpret_cast<const void*>(qkn_pages_copy_kernel<u32x4, 2>)
                                            : reinterpret_cast<const void*>(qkn_pages_copy_kernel<u32x4, 4>))
                   : unit == 4 ? reinterpret_cast<const void*>(qkn_pages_copy_kernel<uint32_t, 4>)
                   : unit == 2 ? reinterpret_cast<const void*>(qkn_pages_copy_kernel<uint16_t, 4>)
                               : reinterpret_cast<const void*>(qkn_pages_copy_kernel<uint8_t, 4>);
  if (!launch(fn, grid, count, kCopyThreads, &p, stream)) return QKN_EHIP;
  return launched(name, grid * count, kCopyThreads);
}

int pools_of(const qkn_cache& c, CopyPool (&to)[4], Span (&spans)[4]) {
  const int64_t esz = c.fp8 ? 1 : 2;
  to[0] = copy_pool(c.k, c.k_page * esz, c.k_head * esz, c.k_token * esz, c.head_dim * esz, c.n_kv, c.page_size);
  to[1] = copy_pool(c.v, c.v_page * esz, c.v_head * esz, c.v_token * esz, c.head_dim * esz, c.n_kv, c.page_size);
  spans[0] = pool_span(c, c.k, c.k_page, c.k_head, c.k_token);
  spans[1] = pool_span(c, c.v, c.v_page, c.v_head, c.v_token);
  return 2;
}
int pools_of(const qkn_cache4& c, CopyPool (&to)[4], Span (&spans)[4]) {
  for (int i = 0; i < 4; ++i) {
    const Pool4 x = pool4(c, i);
    to[i] = copy_pool(x.base, x.page, x.head, x.token, x.row, c.n_kv, c.page_size);
    spans[i] = pool4_span(c, i);
  }
  return 4;
}
bool cache_fine(const qkn_cache& c) { return cache_ok(c); }
bool cache_fine(const qkn_cache4& c) { return cache4_ok(c); }

template <class C>
int copy_caches(const C* caches, int32_t count, const int32_t* src, const int32_t* dst, int32_t n, void* stream) {
  if (count < 0 || n < 0 || (count && !caches)) return QKN_EINVAL;
  for (int32_t i = 0; i < count; ++i) {
    const C& c = caches[i];
    if (!cache_fine(c)) return QKN_EINVAL;
    if (int64_t{2} * c.n_kv * c.page_size * c.head_dim >= int64_t{1} << 31) return QKN_ENOTSUP;
  }
  if (n > 1 << 24) return QKN_ENOTSUP;
  if (n == 0 || count == 0) return QKN_OK;
  if (!src || !dst) return QKN_EINVAL;
  CopyPool pools[4];
  Span spans[4];
  for (int32_t i = 0; i < count; ++i) {
    const int per = pools_of(caches[i], pools, spans);
    for (int k = 0; k < per; ++k) {
      if (caches[i].num_pages && !pools[k].base) return QKN_EINVAL;
      if (spans_overlap(spans[k], array_span(src, n, 4)) || spans_overlap(spans[k], array_span(dst, n, 4))) return QKN_EOVERLAP;
    }
  }
  // caches of the same number of pages follow each other in one launch
  CopyPool batch[kCopyPools];
  int in_batch = 0, rc = QKN_OK;
  for (int32_t i = 0; i < count; ++i) {
    const int per = pools_of(caches[i], pools, spans);
    for (int k = 0; k < per; ++k) batch[in_batch++] = pools[k];
    const bool end = i + 1 == count || in_batch + per > kCopyPools || caches[i + 1].num_pages != caches[i].num_pages;
    if (!end) continue;
    if (caches[i].num_pages) rc = copy_impl(batch, in_batch, caches[i].num_pages, src, dst, n, stream);
    if (rc != QKN_OK && rc != QKN_EDRYRUN) return rc;
    in_batch = 0;
  }
  return rc;
}

}  // namespace

extern "C" {

int qkn_pages_grow(const qkn_pages* book, const int32_t* which, const int32_t* count, int32_t n, int64_t T,
                   int64_t* slots, int32_t* pos, int32_t* done, void* stream) {
  if (!book_ok(book) || n < 0 || T < 0) return QKN_EINVAL;
  if (n > kMost || T >= int64_t{1} << 31) return QKN_ENOTSUP;
  if (n == 0 && (T == 0 || (!slots && !pos))) return QKN_OK;
  if (!book_given(*book) || (n && (!count || !done))) return QKN_EINVAL;
  Arrays a;
  a.book(*book);
  a.add(which, n, 4, false);
  a.add(count, n, 4, false);
  a.add(slots, T, 8, true);
  a.add(pos, T, 4, true);
  a.add(done, n, 4, true);
  if (a.overlap()) return QKN_EOVERLAP;
  if (qkn_host::validate_only()) return dry("pages_grow");
  TakeParams p;
  memset(&p, 0, sizeof(p));
  p.b = book_of(*book);
  p.which = which;
  p.count = count;
  p.n = n;
  p.T = T;
  p.slots = slots;
  p.pos = pos;
  p.done = done;
  if (!launch(reinterpret_cast<const void*>(qkn_pages_take<false>), 1, 1, kMost, &p, stream)) return QKN_EHIP;
  if (T > 4 * kMost && (slots || pos) &&
      !launch(reinterpret_cast<const void*>(qkn_pages_slots), (T + kMany - 1) / kMany, 1, kManyThreads, &p, stream))
    return QKN_EHIP;
  return launched("pages_grow", 1, kMost);
}

int qkn_pages_fork(const qkn_pages* book, const int32_t* from, const int32_t* to, int32_t n, int32_t* src,
                   int32_t* dst, int32_t* done, void* stream) {
  if (!book_ok(book) || n < 0) return QKN_EINVAL;
  if (n > kMost) return QKN_ENOTSUP;
  if (n == 0) return QKN_OK;
  if (!book_given(*book) || !from || !to || !src || !dst || !done) return QKN_EINVAL;
  Arrays a;
  a.book(*book);
  a.add(from, n, 4, false);
  a.add(to, n, 4, false);
  a.add(src, n, 4, true);
  a.add(dst, n, 4, true);
  a.add(done, n, 4, true);
  if (a.overlap()) return QKN_EOVERLAP;
  const int64_t parts = (book->ld_table + kShare - 1) / kShare;
  if (parts > 65535) return QKN_ENOTSUP;
  if (qkn_host::validate_only()) return dry("pages_fork");
  TakeParams p;
  memset(&p, 0, sizeof(p));
  p.b = book_of(*book);
  p.which = to;
  p.from = from;
  p.n = n;
  p.src = src;
  p.dst = dst;
  p.done = done;
  if (!launch(reinterpret_cast<const void*>(qkn_pages_take<true>), 1, 1, kMost, &p, stream) ||
      (parts && !launch(reinterpret_cast<const void*>(qkn_pages_share), n, parts, kRowThreads, &p, stream)))
    return QKN_EHIP;
  return launched("pages_fork", n * parts, kRowThreads);
}

int qkn_pages_free(const qkn_pages* book, const int32_t* which, int32_t n, void* stream) {
  if (!book_ok(book) || n < 0) return QKN_EINVAL;
  if (n > kMost) return QKN_ENOTSUP;
  if (n == 0) return QKN_OK;
  if (!book_given(*book)) return QKN_EINVAL;
  Arrays a;
  a.book(*book);
  a.add(which, n, 4, false);
  if (a.overlap()) return QKN_EOVERLAP;
  if (qkn_host::validate_only()) return dry("pages_free");
  TakeParams p;
  memset(&p, 0, sizeof(p));
  p.b = book_of(*book);
  p.which = which;
  p.n = n;
  if (!launch(reinterpret_cast<const void*>(qkn_pages_drop), n, 1, kRowThreads, &p, stream)) return QKN_EHIP;
  return launched("pages_free", n, kRowThreads);
}

int64_t qkn_pages_compact_workspace_bytes(const qkn_pages* book) {
  if (!book_ok(book)) return QKN_EINVAL;
  const int64_t blocks = (book->num_pages + kScan - 1) / kScan;
  return 4 * ((blocks ? blocks : 1) + 1 + book->num_pages);
}

int qkn_pages_compact(const qkn_pages* book, const qkn_pages* out, int32_t* src, int32_t* dst, int32_t n,
                      void* workspace, int64_t workspace_bytes, void* stream) {
  if (!out) out = book;
  if (!book_ok(book) || !book_ok(out) || n < 0 || out->num_pages != book->num_pages || out->rows != book->rows ||
      out->ld_table != book->ld_table || out->page_size != book->page_size)
    return QKN_EINVAL;
  if (n > 1 << 24) return QKN_ENOTSUP;
  const int64_t need = qkn_pages_compact_workspace_bytes(book), entries = book->rows * book->ld_table;
  if (book->num_pages == 0 && entries == 0 && n == 0) return QKN_OK;
  if (!book_given(*book) || (out->num_pages && !out->refs) || (entries && !out->table) || (n && (!src || !dst)) ||
      !workspace || workspace_bytes < need)
    return QKN_EINVAL;
  if (!aligned(workspace, 16)) return QKN_ENOTSUP;
  int64_t work = (book->num_pages + entries + kRowThreads - 1) / kRowThreads;
  if (work == 0) work = 1;  // the lists alone
  if (!qkn_host::launchable(work, kRowThreads)) return QKN_ENOTSUP;  // before the list of moves is written
  Arrays a;
  a.book(*book);
  if (out->refs != book->refs) a.add(out->refs, out->num_pages, 4, true);
  if (out->table != book->table) a.add(out->table, entries, 4, true);
  a.add(src, n, 4, true);
  a.add(dst, n, 4, true);
  a.add(workspace, need, 1, true);
  if (a.overlap()) return QKN_EOVERLAP;
  if (qkn_host::validate_only()) return dry("pages_compact");
  MoveParams p;
  memset(&p, 0, sizeof(p));
  p.b = book_of(*book);
  p.out = book_of(*out);
  p.src = src;
  p.dst = dst;
  p.n = n;
  const int64_t blocks = book->num_pages ? (book->num_pages + kScan - 1) / kScan : 1;
  p.blocks = static_cast<int32_t>(blocks);
  p.moved = static_cast<int32_t*>(workspace);
  p.counts = p.moved + book->num_pages;
  if ((blocks > kFewBlocks && !launch(reinterpret_cast<const void*>(qkn_pages_count), blocks, 1, kScanThreads, &p, stream)) ||
      !launch(reinterpret_cast<const void*>(qkn_pages_moves), blocks, 1, kScanThreads, &p, stream) ||
      !launch(reinterpret_cast<const void*>(qkn_pages_apply), work, 1, kRowThreads, &p, stream))
    return QKN_EHIP;
  return launched("pages_compact", work, kRowThreads);
}

int qkn_pages_copy(const qkn_cache* caches, int32_t count, const int32_t* src, const int32_t* dst, int32_t n,
                   void* stream) {
  return copy_caches(caches, count, src, dst, n, stream);
}

int qkn_pages_copy4(const qkn_cache4* caches, int32_t count, const int32_t* src, const int32_t* dst, int32_t n,
                    void* stream) {
  return copy_caches(caches, count, src, dst, n, stream);
}

}  // extern "C"
