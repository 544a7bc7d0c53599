// The pages of a cache: rows of a block table that continue others, with copies of pages that two would write, room for the next tokens and counts of who
// holds what; and the move of the pages in use to the lowest numbers.
//
// What has to be counted over rows or pages in order (who copies, who gets which free page) is done by one workgroup with running sums; what is left is copying, for which
// waves take pieces of 4 KB in turn, however many there turn out to be.
#include <hip/hip_runtime.h>

#include "fi_device.h"
#include "fi_ops.h"

namespace fi {
namespace {

constexpr int THREADS = 1024, PIECE = 4096;
// What one workgroup takes with all counts in LDS: rows, old and new, pages, entries of the old table.
constexpr int SMALL_ROWS = 1024, SMALL_PAGES = 24576;
constexpr int64_t SMALL_TABLE = 1 << 17;

// The caches of a call (kernel arguments are 4 KB at most, so a launch takes MOST of them).  start: where a cache's pieces of a page begin, last: of all.
struct Copies {
  static constexpr int MOST = 64;
  int n;
  int start[MOST + 1];
  uint8_t* base[MOST];
  int64_t stride[MOST], bytes[MOST];
};

// Sum over the threads before this one; total: over all.
__device__ __forceinline__ int before(int x, int* lds, int& total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int upto = x;
  for (int o = 1; o < 64; o <<= 1) {
    const int up = __shfl_up(upto, o);
    if (lane >= o) upto += up;
  }
  __syncthreads();
  if (lane == 63) lds[wave] = upto;
  __syncthreads();
  int first = 0;
  total = 0;
  for (int w = 0; w < THREADS / 64; ++w) {
    first += w < wave ? lds[w] : 0;
    total += lds[w];
  }
  return first + upto - x;
}

// Copies page from to page to of every cache: workgroup `group` of `groups` (of 256 threads).
template <typename Pair>
__device__ __forceinline__ void copy_pages(const Copies& c, int group, int groups, int pairs, Pair pair) {
  const int per = c.start[c.n], lane = threadIdx.x & 63;
  for (int64_t at = (int64_t)group * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); at < (int64_t)pairs * per; at += (int64_t)groups * 4) {
    const int i = (int)(at / per), piece = (int)(at - (int64_t)i * per);
    int k = 0;
    while (k + 1 < c.n && c.start[k + 1] <= piece) ++k;
    int from, to;
    pair(i, from, to);
    const int64_t off = (int64_t)(piece - c.start[k]) * PIECE, n = c.bytes[k] - off < PIECE ? c.bytes[k] - off : PIECE;
    const uint8_t* const x = c.base[k] + from * c.stride[k] + off;
    uint8_t* const y = c.base[k] + to * c.stride[k] + off;
    if (((reinterpret_cast<uintptr_t>(x) | reinterpret_cast<uintptr_t>(y) | (uintptr_t)n) & 15) == 0) {
      u32x4 w[4];
#pragma unroll
      for (int u = 0; u < 4; ++u)
        if ((u * 64 + lane) * 16 < n) w[u] = reinterpret_cast<const u32x4*>(x)[u * 64 + lane];
#pragma unroll
      for (int u = 0; u < 4; ++u)
        if ((u * 64 + lane) * 16 < n) reinterpret_cast<u32x4*>(y)[u * 64 + lane] = w[u];
    } else if (((reinterpret_cast<uintptr_t>(x) | reinterpret_cast<uintptr_t>(y) | (uintptr_t)n) & 3) == 0) {
      for (int b = lane * 4; b < n; b += 256) *reinterpret_cast<uint32_t*>(y + b) = *reinterpret_cast<const uint32_t*>(x + b);
    } else {
      for (int b = lane; b < n; b += 64) y[b] = x[b];
    }
  }
}

// ---- forks ----------------------------------------------------------------------------------------
// The workspace: [0] pages that could be given, [1] copies; then for every new row its last page (-1: none that it writes), what it needs and where that
// begins among all needs, and where its copy stands; for every old row how many continue it; the pages given; the copies' sources and targets.
struct ForkSpace {
  int *head, *last, *need, *first, *copy, *children, *given, *source, *target;
  __host__ __device__ ForkSpace(void* p, int rows, int new_rows, int n_pages) {
    head = static_cast<int*>(p);
    last = head + 4;
    need = last + new_rows;
    first = need + new_rows;
    copy = first + new_rows;
    source = copy + new_rows;
    target = source + new_rows;
    children = target + new_rows;
    given = children + rows;
    end = given + n_pages;
  }
  int* end;
};

struct ForkRow {
  int parent, length, before, after;   // pages of the committed tokens, pages with the room
  bool fits;
};
__device__ __forceinline__ int pages_of(uint32_t tokens, int page) {   // (below 2^32)
  const uint32_t q = tokens / (uint32_t)page;
  return (int)(q + (q * (uint32_t)page != tokens));
}
__device__ __forceinline__ int held_pages(const fi_fork_pages_args& a, const int32_t* tokens, int row) {
  const int n = tokens[row], most = a.columns * a.page_size;
  return pages_of(n < 0 ? 0 : n > most ? most : n, a.page_size);
}
__device__ __forceinline__ ForkRow fork_row(const fi_fork_pages_args& a, int i) {
  ForkRow r;
  r.parent = a.parents ? a.parents[i] : i;
  if (r.parent < 0 || r.parent >= a.rows) r.parent = -1;
  const int most = a.columns * a.page_size, n = r.parent < 0 ? 0 : a.lengths[r.parent];
  r.length = n < 0 ? 0 : n > most ? most : n;
  r.before = pages_of(r.length, a.page_size);
  const int after = pages_of((uint32_t)r.length + (uint32_t)a.room, a.page_size);
  r.fits = r.parent >= 0 && after <= a.columns;
  r.after = r.fits ? after : r.before;
  return r;
}
__device__ __forceinline__ bool is_page(const fi_fork_pages_args& a, int p) { return p >= 0 && p < a.n_pages; }

// The page that a new row would write next to tokens that it has, or -1.
__device__ __forceinline__ int fork_last(const fi_fork_pages_args& a, const ForkRow& r) {
  if (!r.fits || a.room == 0) return -1;
  const uint32_t at = (uint32_t)r.length / (uint32_t)a.page_size;
  if (at * (uint32_t)a.page_size == (uint32_t)r.length) return -1;
  const int p = a.block_table[r.parent * a.table_stride + at];
  return is_page(a, p) ? p : -1;
}
// An old row's entry: children share it where it holds committed tokens; the row itself lets go.
__device__ __forceinline__ void fork_count(const fi_fork_pages_args& a, int row, int column, int children, int committed, int held) {
  const int change = (column < committed ? children : 0) - (column < held ? 1 : 0);
  if (!change) return;
  const int p = a.block_table[row * a.table_stride + column];
  if (is_page(a, p)) atomicAdd(a.refs_out + p, change);
}

// Whether the pages that are there suffice for a row, of which rows before it need the `first` first ones.
__device__ __forceinline__ bool suffices(int first, int need, int there) { return first <= there - need; }

// What every row needs, in order, and the free pages for it: by one workgroup.
__device__ __forceinline__ void fork_deal(const fi_fork_pages_args& a, const ForkSpace& w, int* lds) {
  int64_t wanted = 0;   // (needs of all rows may pass 32 bits; more than there are pages is as good as one more)
  int copies = 0;
  for (int i0 = 0; i0 < a.new_rows; i0 += THREADS) {
    const int i = i0 + threadIdx.x;
    int need = i < a.new_rows ? w.need[i] : 0, copy = i < a.new_rows ? w.copy[i] : 0;
    int all, all_copies;
    const int first = before(need, lds, all), at = before(copy, lds, all_copies);
    if (i < a.new_rows) {
      const int64_t f = wanted + first;
      w.first[i] = f < a.n_pages + 1 ? (int)f : a.n_pages + 1;
      w.copy[i] = copy ? copies + at : -1;
    }
    wanted += all;
    if (wanted > a.n_pages + 1) wanted = a.n_pages + 1;
    copies += all_copies;
  }
  int found = 0;
  for (int64_t begin = 0; begin < a.n_pages && found < wanted; begin += THREADS * 4) {   // (n_pages and a round of the loop may pass 2^31)
    const int p0 = (int)begin;
    int free[4], n = 0;
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int p = p0 + threadIdx.x * 4 + u;
      free[u] = p < a.n_pages && a.refs_out[p] == 0;
      n += free[u];
    }
    int all;
    int at = found + before(n, lds, all);
#pragma unroll
    for (int u = 0; u < 4; ++u)
      if (free[u]) {
        if (at < wanted) w.given[at] = p0 + threadIdx.x * 4 + u;
        ++at;
      }
    found += all;
  }
  if (threadIdx.x == 0) {
    w.head[0] = found < wanted ? found : (int)wanted;
    w.head[1] = 0;
  }
  __syncthreads();
  // the rows that get what they need are those before the pages run out, so their copies come first
  int made = 0;
  const int there = w.head[0];
  for (int i = threadIdx.x; i < a.new_rows; i += THREADS)
    if (w.copy[i] >= 0 && suffices(w.first[i], w.need[i], there)) ++made;
  if (made) atomicAdd(w.head + 1, made);
}

// What a new row gets is held (count(page, change)); its copy is noted.
template <typename Count>
__device__ __forceinline__ void fork_take(const ForkSpace& w, int need, int first, int copy, int last, const int* given, Count count) {
  for (int n = 0; n < need; ++n) count(given[first + n], 1);
  if (copy < 0) return;
  w.source[copy] = last;
  w.target[copy] = given[first];
}
// A new row's entries, by a wave.
__device__ __forceinline__ void fork_write(const fi_fork_pages_args& a, const ForkSpace& w, int i) {
  const int lane = threadIdx.x & 63;
  const int need = w.need[i], first = w.first[i], there = w.head[0], asked = w.copy[i];
  const ForkRow r = fork_row(a, i);
  bool made = r.fits && (need == 0 || suffices(first, need, there));
  const bool copy = made && asked >= 0;
  if (made && need == 0 && !suffices(w.first[a.new_rows - 1], w.need[a.new_rows - 1], there)) {   // rows before this one may hold more of the page that it would write, and have got no copy
    const int mine = fork_last(a, r);
    if (mine >= 0)
      for (int j0 = 0; j0 < i && made; j0 += 64) {
        const int j = j0 + lane;
        bool over = false;
        if (j < i && w.copy[j] >= 0 && !suffices(w.first[j], w.need[j], there)) {
          const ForkRow other = fork_row(a, j);
          over = other.length > r.length && fork_last(a, other) == mine;
        }
        made = !__any(over);
      }
  }
  const int at = r.length / a.page_size;
  auto entry = [&](int j) {
    if (copy && j == at) return w.given[first];
    if (j < r.before) return a.block_table[r.parent * a.table_stride + j];
    return made && j < r.after ? w.given[first + (copy ? 1 : 0) + j - r.before] : -1;
  };
  for (int j = lane; j < a.columns; j += 64) a.table_out[i * a.table_out_stride + j] = entry(j);
  for (int t = lane; t < a.room; t += 64) {
    const int place = r.length + t, p = made ? entry(place / a.page_size) : -1;
    a.slots_out[(int64_t)i * a.room + t] = is_page(a, p) ? (int64_t)p * a.page_size + place % a.page_size : -1;
  }
  if (lane == 0) {
    a.lengths_out[i] = r.length;
    a.held_out[i] = made ? r.length + a.room : r.length;
  }
}

// Few rows: all that is counted by one workgroup, in LDS.  512 rows of up to 63 pages: 16.0 us; with the counts in memory (atomics, and loads past the
// caches) 122, 4 rows 22 -> 6.  The rest is latency: 2 us until the rows are known, 8.5 for the old table, a few for running sums and what is written.
__global__ void __launch_bounds__(THREADS) fork_small_kernel(fi_fork_pages_args a) {
  __shared__ int refs[SMALL_PAGES], children[SMALL_ROWS], committed[SMALL_ROWS], held[SMALL_ROWS], sums[THREADS / 64];
  if (blockIdx.x) {   // large tables: the one on the first one's XCD brings what that will read to their cache (512 rows of 64 entries: 17.6 us, so 16.0)
    if (blockIdx.x % NXCD) return;
    constexpr int LINE = 32;   // entries
    int x = 0;
    for (int i = threadIdx.x * LINE; i < a.rows * a.columns; i += THREADS * LINE) {   // (at most 2^17)
      const int r = i / a.columns;
      x ^= a.block_table[r * a.table_stride + i - r * a.columns];
    }
    for (int p = threadIdx.x * LINE; p < a.n_pages; p += THREADS * LINE) x ^= a.refs[p];
    asm volatile("" ::"v"(x));
    return;
  }
  const ForkSpace w(a.workspace, a.rows, a.new_rows, a.n_pages);
  const int me = threadIdx.x, lane = me & 63, wave = __builtin_amdgcn_readfirstlane(me >> 6);
  ForkRow row{-1, 0, 0, 0, false};
  if (me < a.new_rows) row = fork_row(a, me);
  const int mine = me < a.new_rows ? fork_last(a, row) : -1;
  children[me] = 0;
  if (me < a.rows) {
    committed[me] = held_pages(a, a.lengths, me);
    held[me] = a.held ? held_pages(a, a.held, me) : committed[me];
  }
  for (int p = me; p < a.n_pages; p += THREADS) refs[p] = a.refs[p];
  __syncthreads();
  if (row.parent >= 0) atomicAdd(&children[row.parent], 1);
  __syncthreads();
  // Entries that change: children share them where they are committed, the row itself lets go.  Lane l of wave x has row 16 l + x; rows and pieces of 64 of their entries
  // are gone through by scalar registers (with vector ones, 512 rows of 64 entries take 12 us, so 8.5, which is what one unit has of lines on their way: 2, 8 or 32 loads
  // at a time do not change it).
  {
    constexpr int WAVES = THREADS / 64, AT_ONCE = 4;
    const int r = lane * WAVES + wave, c = r < a.rows ? children[r] : 0, kept = r < a.rows ? committed[r] : 0, all = r < a.rows ? held[r] : 0;
    uint64_t left = __ballot(c == 1 ? kept != all : kept > 0 || all > 0);
    int j0 = 0;
    while (left) {
      int p[AT_ONCE], change[AT_ONCE];
#pragma unroll
      for (int u = 0; u < AT_ONCE; ++u) {
        p[u] = -1;
        change[u] = 0;
        if (!left) continue;
        const int l = __ffsll((long long)left) - 1, times = __builtin_amdgcn_readlane(c, l), some = __builtin_amdgcn_readlane(kept, l), most = __builtin_amdgcn_readlane(all, l);
        const int j = j0 + lane;
        change[u] = (j < some ? times : 0) - (j < most ? 1 : 0);
        if (change[u]) p[u] = a.block_table[(int64_t)(l * WAVES + wave) * a.table_stride + j];
        j0 += 64;
        if (j0 >= some && j0 >= most) {
          j0 = 0;
          left &= left - 1;
        }
      }
#pragma unroll
      for (int u = 0; u < AT_ONCE; ++u)
        if (is_page(a, p[u])) atomicAdd(&refs[p[u]], change[u]);
    }
  }
  // Rows of a wave that write one page, those before this one; then the waves in order take their copies off the counts.
  int sharers = 0;
  for (uint64_t left = __ballot(mine >= 0); left;) {
    const int page = __builtin_amdgcn_readlane(mine, __ffsll((long long)left) - 1);
    const uint64_t same = __ballot(mine == page);
    if (mine == page) sharers = __popcll(same & ((1ull << lane) - 1));
    left &= ~same;
  }
  bool copy = false;
  for (int x = 0; x < (a.new_rows + 63) / 64; ++x) {
    __syncthreads();
    if (x == wave && mine >= 0) {
      copy = refs[mine] - sharers > 1;
      if (copy) atomicAdd(&refs[mine], -1);   // (after all lanes have read: a wave's accesses to LDS keep their order)
    }
  }
  const int need = row.fits ? (copy ? 1 : 0) + row.after - row.before : 0;
  int wanted, copies;
  const int first = before(need, sums, wanted), at = before(copy ? 1 : 0, sums, copies);   // (at most 1024 rows of 2^16 + 1)
  int found = 0;
  for (int p0 = 0; p0 < a.n_pages && found < wanted; p0 += THREADS * 4) {
    const int p = p0 + me * 4;
    int free = 0;
#pragma unroll
    for (int u = 0; u < 4; ++u) free |= (p + u < a.n_pages && refs[p + u] == 0) << u;
    int all, to = found + before(__popc(free), sums, all);
#pragma unroll
    for (int u = 0; u < 4; ++u)
      if (free >> u & 1) {
        if (to < wanted) w.given[to] = p + u;
        ++to;
      }
    found += all;
  }
  const int there = found < wanted ? found : wanted;
  const bool made = row.fits && suffices(first, need, there);
  before(copy && made ? 1 : 0, sums, copies);   // (and what is given has been written)
  if (me < a.new_rows) {
    w.need[me] = need;
    w.first[me] = first;
    w.copy[me] = copy ? at : -1;
    if (made) fork_take(w, need, first, copy ? at : -1, mine, w.given, [&](int p, int change) { atomicAdd(&refs[p], change); });
    else if (copy) atomicAdd(&refs[mine], 1);
  }
  if (me == 0) {
    w.head[0] = there;
    w.head[1] = copies;
  }
  __syncthreads();
  for (int p = me; p < a.n_pages; p += THREADS) a.refs_out[p] = refs[p];
}

// Many rows: the same steps, a launch each.
__global__ void __launch_bounds__(256) fork_begin_kernel(fi_fork_pages_args a) {
  const ForkSpace w(a.workspace, a.rows, a.new_rows, a.n_pages);
  const int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x, step = (int64_t)gridDim.x * 256;
  for (int64_t p = at; p < a.n_pages; p += step) a.refs_out[p] = a.refs[p];
  for (int64_t r = at; r < a.rows; r += step) w.children[r] = 0;
  for (int64_t i = at; i < a.new_rows; i += step) w.last[i] = fork_last(a, fork_row(a, (int)i));
}
__global__ void __launch_bounds__(256) fork_children_kernel(fi_fork_pages_args a) {
  const ForkSpace w(a.workspace, a.rows, a.new_rows, a.n_pages);
  const int i = blockIdx.x * 256 + threadIdx.x;
  if (i >= a.new_rows) return;
  const ForkRow r = fork_row(a, i);
  if (r.parent >= 0) atomicAdd(w.children + r.parent, 1);
}
__global__ void __launch_bounds__(256) fork_count_kernel(fi_fork_pages_args a) {
  const ForkSpace w(a.workspace, a.rows, a.new_rows, a.n_pages);
  for (int r = blockIdx.x; r < a.rows; r += gridDim.x) {
    const int committed = held_pages(a, a.lengths, r), held = a.held ? held_pages(a, a.held, r) : committed, children = w.children[r];
    for (int j = threadIdx.x; j < a.columns; j += 256) fork_count(a, r, j, children, committed, held);
  }
}
__global__ void __launch_bounds__(256) fork_need_kernel(fi_fork_pages_args a) {
  const ForkSpace w(a.workspace, a.rows, a.new_rows, a.n_pages);
  const int lane = threadIdx.x & 63, i = blockIdx.x * 4 + (threadIdx.x >> 6);
  if (i >= a.new_rows) return;
  const ForkRow r = fork_row(a, i);
  const int mine = w.last[i];
  int sharers = 0;
  if (mine >= 0)
    for (int j = lane; j < i; j += 64) sharers += w.last[j] == mine;
  for (int o = 32; o; o >>= 1) sharers += __shfl_xor(sharers, o);
  if (lane) return;
  const bool copy = mine >= 0 && a.refs_out[mine] - sharers > 1;
  w.copy[i] = copy;
  w.need[i] = r.fits ? (copy ? 1 : 0) + r.after - r.before : 0;
}
__global__ void __launch_bounds__(THREADS) fork_deal_kernel(fi_fork_pages_args a) {
  __shared__ int sums[THREADS / 64];
  fork_deal(a, ForkSpace(a.workspace, a.rows, a.new_rows, a.n_pages), sums);
}
__global__ void __launch_bounds__(256) fork_take_kernel(fi_fork_pages_args a) {
  const ForkSpace w(a.workspace, a.rows, a.new_rows, a.n_pages);
  const int i = blockIdx.x * 256 + threadIdx.x;
  if (i >= a.new_rows || w.need[i] == 0 || !suffices(w.first[i], w.need[i], w.head[0])) return;
  if (w.copy[i] >= 0) atomicAdd(a.refs_out + w.last[i], -1);
  fork_take(w, w.need[i], w.first[i], w.copy[i], w.last[i], w.given, [&](int p, int change) { atomicAdd(a.refs_out + p, change); });
}
// The rows, by the first `row_groups` workgroups, and the copies by the others.
__global__ void __launch_bounds__(256) fork_write_kernel(fi_fork_pages_args a, Copies c, int row_groups) {
  const ForkSpace w(a.workspace, a.rows, a.new_rows, a.n_pages);
  if ((int)blockIdx.x < row_groups) {
    const int i = blockIdx.x * 4 + (threadIdx.x >> 6);
    if (i < a.new_rows) fork_write(a, w, i);
    return;
  }
  copy_pages(c, blockIdx.x - row_groups, gridDim.x - row_groups, w.head[1], [&](int i, int& from, int& to) {
    from = w.source[i];
    to = w.target[i];
  });
}

// ---- compaction -----------------------------------------------------------------------------------
// The workspace: [0] pages in use, [1] moves; the moves' sources and targets.
struct CompactSpace {
  int *head, *source, *target;
  __host__ __device__ CompactSpace(void* p, int n_pages) : head(static_cast<int*>(p)), source(head + 4), target(source + n_pages / 2 + 1), end(target + n_pages / 2 + 1) {}
  int* end;
};
// One workgroup, four pages a thread, holes and movers in one running sum: 4096 pages 7.4 us (a page a thread and two sums: 11.8), 512 pages 3.4.
__global__ void __launch_bounds__(THREADS) compact_plan_kernel(fi_compact_pages_args a) {
  __shared__ int sums[THREADS / 64];
  const CompactSpace w(a.workspace, a.n_pages);
  constexpr int EACH = 4;   // pages of a thread, one after the other
  auto counts = [&](int p0, int (&n)[EACH]) {
#pragma unroll
    for (int e = 0; e < EACH; ++e) n[e] = 0;
#pragma unroll
    for (int e = 0; e < EACH; ++e)
      if (p0 + e < a.n_pages) n[e] = a.refs[p0 + e];
  };
  int live = 0, first[EACH], n[EACH];
  counts(threadIdx.x * EACH, first);
  for (int64_t p0 = threadIdx.x * EACH; p0 < a.n_pages; p0 += THREADS * EACH) {
    if (p0 >= THREADS * EACH) counts((int)p0, n);
#pragma unroll
    for (int e = 0; e < EACH; ++e) live += (p0 < THREADS * EACH ? first[e] : n[e]) > 0;
  }
  int total;
  before(live, sums, total);
  live = total;
  int holes = 0, movers = 0;
  for (int64_t at = 0; at < a.n_pages; at += THREADS * EACH) {
    const int p0 = (int)at + (int)threadIdx.x * EACH;   // (n_pages + a round of the loop stays below 2^31)
    if (at) counts(p0, n);
    else
#pragma unroll
      for (int e = 0; e < EACH; ++e) n[e] = first[e];
    int mine = 0;   // holes in the low half, movers in the high one
#pragma unroll
    for (int e = 0; e < EACH; ++e)
      if (p0 + e < a.n_pages) mine += p0 + e < live ? n[e] <= 0 : n[e] > 0 ? 1 << 16 : 0;
    const int ahead = before(mine, sums, total);
    int h = holes + (ahead & 0xffff), m = movers + (ahead >> 16);
#pragma unroll
    for (int e = 0; e < EACH; ++e) {
      const int p = p0 + e;
      if (p >= a.n_pages) break;
      const bool hole = p < live && n[e] <= 0, mover = p >= live && n[e] > 0;
      if (hole) w.target[h++] = p;
      if (mover) w.source[m++] = p;
      else a.moved_out[p] = n[e] > 0 ? p : -1;
      if (!hole) a.refs_out[p] = p < live ? n[e] : 0;
    }
    holes += total & 0xffff;
    movers += total >> 16;
  }
  __syncthreads();
  for (int i = threadIdx.x; i < movers; i += THREADS) {
    a.moved_out[w.source[i]] = w.target[i];
    a.refs_out[w.target[i]] = a.refs[w.source[i]];
  }
  if (threadIdx.x == 0) {
    *a.live_out = live;
    w.head[0] = live;
    w.head[1] = movers;
  }
}
// Bound by memory: 1.0 GB read and written in 211 us, 4.8 TB/s, a large copy's rate is 4.96.  Pieces of a workgroup's, 16 KB, took 215; 4715 pages of 20 KB in 6 caches 52.9 us, so 46.0;
// 6730 of 288 bytes 20.5 and 15.3.
__global__ void __launch_bounds__(256) compact_move_kernel(fi_compact_pages_args a, Copies c, int table_groups) {
  const CompactSpace w(a.workspace, a.n_pages);
  if ((int)blockIdx.x < table_groups) {
    for (int r = blockIdx.x; r < a.rows; r += table_groups)
      for (int j = threadIdx.x; j < a.columns; j += 256) {
        const int p = a.block_table[r * a.table_stride + j], to = p >= 0 && p < a.n_pages ? a.moved_out[p] : -1;
        a.table_out[r * a.table_out_stride + j] = to >= 0 ? to : p;
      }
    return;
  }
  copy_pages(c, blockIdx.x - table_groups, gridDim.x - table_groups, w.head[1], [&](int i, int& from, int& to) {
    from = w.source[i];
    to = w.target[i];
  });
}

// Caches [at, at + MOST) of a call.
Copies copies_of(const fi_page_cache* caches, int n, int at) {
  Copies c = {};
  for (int i = at; i < n && c.n < Copies::MOST; ++i) {
    if (caches[i].page_bytes == 0) continue;
    c.base[c.n] = static_cast<uint8_t*>(caches[i].base);
    c.stride[c.n] = caches[i].page_stride;
    c.bytes[c.n] = caches[i].page_bytes;
    c.start[c.n + 1] = c.start[c.n] + (int)((caches[i].page_bytes + PIECE - 1) / PIECE);
    ++c.n;
  }
  return c;
}
// Workgroups for at most `pairs` pages: what fills the chip (eight on a unit), or what there can be to do.
uint32_t copy_groups(const Copies& c, int64_t pairs) {
  const int64_t groups = (pairs * c.start[c.n] + 3) / 4;
  return (uint32_t)(groups < 2048 ? groups : 2048);
}

}  // namespace

uint64_t fork_workspace(const fi_fork_pages_args& a) {
  const ForkSpace w(nullptr, a.rows, a.new_rows, a.n_pages);
  return (uint64_t)reinterpret_cast<uintptr_t>(w.end);
}

int launch_fork_pages(const fi_fork_pages_args& a, void* stream) {
  const hipStream_t s = static_cast<hipStream_t>(stream);
  if (a.rows <= SMALL_ROWS && a.new_rows <= SMALL_ROWS && a.n_pages <= SMALL_PAGES && (int64_t)a.rows * a.columns <= SMALL_TABLE) {
    fork_small_kernel<<<dim3((int64_t)a.rows * a.columns > 8192 ? 1 + NXCD : 1), THREADS, 0, s>>>(a);
  } else {
    const int64_t widest = a.n_pages > a.new_rows ? a.n_pages : a.new_rows, begin = (widest + 255) / 256;
    fork_begin_kernel<<<dim3((uint32_t)(begin < 1 ? 1 : begin < 2048 ? begin : 2048)), 256, 0, s>>>(a);
    if (a.new_rows) fork_children_kernel<<<dim3((a.new_rows + 255) / 256), 256, 0, s>>>(a);
    if (a.rows) fork_count_kernel<<<dim3(a.rows < 4096 ? a.rows : 4096), 256, 0, s>>>(a);
    if (a.new_rows) fork_need_kernel<<<dim3((a.new_rows + 3) / 4), 256, 0, s>>>(a);
    fork_deal_kernel<<<dim3(1), THREADS, 0, s>>>(a);
    if (a.new_rows) fork_take_kernel<<<dim3((a.new_rows + 255) / 256), 256, 0, s>>>(a);
  }
  if (!a.new_rows) return (int)hipGetLastError();
  const bool copies = a.room > 0 && a.n_pages > 0;
  int rows = (a.new_rows + 3) / 4;
  for (int at = 0; at == 0 || (copies && at < a.n_caches); at += Copies::MOST) {
    const Copies c = copies_of(a.caches, copies ? a.n_caches : 0, at);
    const uint32_t groups = (uint32_t)rows + copy_groups(c, a.new_rows);
    if (groups) fork_write_kernel<<<dim3(groups), 256, 0, s>>>(a, c, rows);
    rows = 0;
  }
  return (int)hipGetLastError();
}

uint64_t compact_workspace(const fi_compact_pages_args& a) {
  const CompactSpace w(nullptr, a.n_pages);
  return (uint64_t)reinterpret_cast<uintptr_t>(w.end);
}

int launch_compact_pages(const fi_compact_pages_args& a, void* stream) {
  const hipStream_t s = static_cast<hipStream_t>(stream);
  compact_plan_kernel<<<dim3(1), THREADS, 0, s>>>(a);
  int table = a.columns ? (a.rows < 1024 ? a.rows : 1024) : 0;
  for (int at = 0; at == 0 || at < a.n_caches; at += Copies::MOST) {
    const Copies c = copies_of(a.caches, a.n_caches, at);
    const uint32_t groups = (uint32_t)table + copy_groups(c, a.n_pages / 2);
    if (groups) compact_move_kernel<<<dim3(groups), 256, 0, s>>>(a, c, table);
    table = 0;
  }
  return (int)hipGetLastError();
}

}  // namespace fi
