// The pages of a cache: rows of a block table that continue others, with copies of pages that two would write, room for the next tokens and counts of who
// holds what; and the move of the pages in use to the lowest numbers.
//
// What has to be counted over rows or pages in order (who copies, who gets which free page) is done by one workgroup with running sums; what is left is copying, for which
// workgroups take pieces of 16 KB in turn, however many there turn out to be.
#include <hip/hip_runtime.h>

#include "fi_device.h"
#include "fi_ops.h"

namespace fi {
namespace {

constexpr int THREADS = 1024, PIECE = 16384;
constexpr int SMALL_ROWS = 1024;           // rows, old and new, that one workgroup takes with its lists in LDS
constexpr int64_t SMALL_TABLE = 1 << 16;   // and entries of their tables

// The caches of a call (kernel arguments are 4 KB at most, so a launch takes MOST of them).  start: where a cache's pieces of a page begin, last: of all.
struct Copies {
  static constexpr int MOST = 64;
  int n;
  int start[MOST + 1];
  uint8_t* base[MOST];
  int64_t stride[MOST], bytes[MOST];
};

__device__ __forceinline__ int agent_load(const int* p) { return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }   // (counts change by atomics)

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

// Copies page from to page to of every cache, pieces `first`, first + step, ... of pairs x pieces of a page.
template <typename Pair>
__device__ __forceinline__ void copy_pages(const Copies& c, int64_t first, int64_t step, int pairs, Pair pair) {
  const int per = c.start[c.n];
  for (int64_t at = first; at < (int64_t)pairs * per; at += step) {
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
        if ((u * 256 + threadIdx.x) * 16 < n) w[u] = reinterpret_cast<const u32x4*>(x)[u * 256 + threadIdx.x];
#pragma unroll
      for (int u = 0; u < 4; ++u)
        if ((u * 256 + threadIdx.x) * 16 < n) reinterpret_cast<u32x4*>(y)[u * 256 + threadIdx.x] = w[u];
    } else if (((reinterpret_cast<uintptr_t>(x) | reinterpret_cast<uintptr_t>(y) | (uintptr_t)n) & 3) == 0) {
      for (int b = threadIdx.x * 4; b < n; b += 1024) *reinterpret_cast<uint32_t*>(y + b) = *reinterpret_cast<const uint32_t*>(x + b);
    } else {
      for (int b = threadIdx.x; b < n; b += 256) y[b] = x[b];
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
__device__ __forceinline__ int pages_of(int tokens, int page) { return (int)(((int64_t)tokens + page - 1) / page); }
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
  const int64_t after = ((int64_t)r.length + a.room + a.page_size - 1) / a.page_size;
  r.fits = r.parent >= 0 && after <= a.columns;
  r.after = r.fits ? (int)after : r.before;
  return r;
}
__device__ __forceinline__ bool is_page(const fi_fork_pages_args& a, int p) { return p >= 0 && p < a.n_pages; }

// The page that a new row would write next to tokens that it has, or -1.
__device__ __forceinline__ int fork_last(const fi_fork_pages_args& a, const ForkRow& r) {
  if (!r.fits || a.room == 0 || r.length % a.page_size == 0) return -1;
  const int p = a.block_table[r.parent * a.table_stride + r.length / a.page_size];
  return is_page(a, p) ? p : -1;
}
// An old row's entry: children share it where it holds committed tokens; the row itself lets go.
__device__ __forceinline__ void fork_count(const fi_fork_pages_args& a, int row, int column, int children, int committed, int held) {
  const int change = (column < committed ? children : 0) - (column < held ? 1 : 0);
  if (!change) return;
  const int p = a.block_table[row * a.table_stride + column];
  if (is_page(a, p)) atomicAdd(a.refs_out + p, change);
}

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
  for (int p0 = 0; p0 < a.n_pages && found < wanted; p0 += THREADS * 4) {
    int free[4], n = 0;
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int p = p0 + threadIdx.x * 4 + u;
      free[u] = p < a.n_pages && agent_load(a.refs_out + p) == 0;
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
    if (w.copy[i] >= 0 && w.first[i] + w.need[i] <= there) ++made;
  if (made) atomicAdd(w.head + 1, made);
}

// A new row's entries, by `lanes` threads.
__device__ __forceinline__ void fork_write(const fi_fork_pages_args& a, const ForkSpace& w, int i, int lane, int lanes) {
  const ForkRow r = fork_row(a, i);
  const int need = w.need[i], first = w.first[i], there = agent_load(w.head);
  const bool made = r.fits && (need == 0 || first + need <= there);
  const bool copy = made && w.copy[i] >= 0;
  const int at = r.length / a.page_size;
  auto entry = [&](int j) {
    if (copy && j == at) return w.given[first];
    if (j < r.before) return a.block_table[r.parent * a.table_stride + j];
    return made && j < r.after ? w.given[first + (copy ? 1 : 0) + j - r.before] : -1;
  };
  for (int j = lane; j < a.columns; j += lanes) a.table_out[i * a.table_out_stride + j] = entry(j);
  for (int t = lane; t < a.room; t += lanes) {
    const int place = r.length + t, p = made ? entry(place / a.page_size) : -1;
    a.slots_out[(int64_t)i * a.room + t] = is_page(a, p) ? (int64_t)p * a.page_size + place % a.page_size : -1;
  }
  if (made)
    for (int n = lane; n < need; n += lanes) atomicAdd(a.refs_out + w.given[first + n], 1);
  if (lane == 0) {
    a.lengths_out[i] = r.length;
    a.held_out[i] = made ? r.length + a.room : r.length;
    if (copy) {
      atomicAdd(a.refs_out + w.last[i], -1);
      w.source[w.copy[i]] = w.last[i];
      w.target[w.copy[i]] = w.given[first];
    }
  }
}

// Few rows: all of it by one workgroup.
__global__ void __launch_bounds__(THREADS) fork_small_kernel(fi_fork_pages_args a) {
  __shared__ int children[SMALL_ROWS], committed[SMALL_ROWS], held[SMALL_ROWS], sums[THREADS / 64];
  __shared__ __attribute__((aligned(16))) int last[SMALL_ROWS];
  const ForkSpace w(a.workspace, a.rows, a.new_rows, a.n_pages);
  for (int p = threadIdx.x; p < a.n_pages; p += THREADS) a.refs_out[p] = a.refs[p];
  for (int r = threadIdx.x; r < a.rows; r += THREADS) {
    children[r] = 0;
    committed[r] = held_pages(a, a.lengths, r);
    held[r] = a.held ? held_pages(a, a.held, r) : committed[r];
  }
  for (int i = threadIdx.x; i < SMALL_ROWS; i += THREADS) last[i] = -1;
  __threadfence();
  __syncthreads();
  ForkRow row{-1, 0, 0, 0, false};
  if ((int)threadIdx.x < a.new_rows) {
    row = fork_row(a, threadIdx.x);
    if (row.parent >= 0) atomicAdd(&children[row.parent], 1);
    last[threadIdx.x] = fork_last(a, row);
  }
  __syncthreads();
  for (int i = threadIdx.x; i < a.rows * a.columns; i += THREADS) {
    const int r = i / a.columns;
    fork_count(a, r, i - r * a.columns, children[r], committed[r], held[r]);
  }
  __threadfence();
  __syncthreads();
  if ((int)threadIdx.x < a.new_rows) {
    const int mine = last[threadIdx.x];
    bool copy = false;
    if (mine >= 0) {
      int sharers = 0;   // rows before this one that write the same page
      for (int j = 0; j < (int)threadIdx.x; j += 4) {
        const int4 o = *reinterpret_cast<const int4*>(last + j);
        sharers += (o.x == mine) + (o.y == mine && j + 1 < (int)threadIdx.x) + (o.z == mine && j + 2 < (int)threadIdx.x) + (o.w == mine && j + 3 < (int)threadIdx.x);
      }
      copy = agent_load(a.refs_out + mine) - sharers > 1;
    }
    w.last[threadIdx.x] = mine;
    w.copy[threadIdx.x] = copy;
    w.need[threadIdx.x] = row.fits ? (copy ? 1 : 0) + row.after - row.before : 0;
  }
  __threadfence();
  __syncthreads();
  fork_deal(a, w, sums);
  __threadfence();
  __syncthreads();
  for (int i = threadIdx.x / 64; i < a.new_rows; i += THREADS / 64) fork_write(a, w, i, threadIdx.x & 63, 64);
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
__global__ void __launch_bounds__(256) fork_write_kernel(fi_fork_pages_args a) {
  const ForkSpace w(a.workspace, a.rows, a.new_rows, a.n_pages);
  const int i = blockIdx.x * 4 + (threadIdx.x >> 6);
  if (i < a.new_rows) fork_write(a, w, i, threadIdx.x & 63, 64);
}
__global__ void __launch_bounds__(256) fork_copy_kernel(const int* head, const int* source, const int* target, Copies c) {
  copy_pages(c, blockIdx.x, gridDim.x, head[1], [&](int i, int& from, int& to) {
    from = source[i];
    to = target[i];
  });
}

// ---- compaction -----------------------------------------------------------------------------------
// The workspace: [0] pages in use, [1] moves; the moves' sources and targets.
struct CompactSpace {
  int *head, *source, *target;
  __host__ __device__ CompactSpace(void* p, int n_pages) : head(static_cast<int*>(p)), source(head + 4), target(source + n_pages / 2 + 1), end(target + n_pages / 2 + 1) {}
  int* end;
};
__global__ void __launch_bounds__(THREADS) compact_plan_kernel(fi_compact_pages_args a) {
  __shared__ int sums[THREADS / 64];
  const CompactSpace w(a.workspace, a.n_pages);
  int live = 0;
  for (int p = threadIdx.x; p < a.n_pages; p += THREADS) live += a.refs[p] > 0;
  int total;
  before(live, sums, total);
  live = total;
  int holes = 0, movers = 0;
  for (int p0 = 0; p0 < a.n_pages; p0 += THREADS) {
    const int p = p0 + threadIdx.x, n = p < a.n_pages ? a.refs[p] : 0;
    const int hole = p < live && n <= 0, mover = p >= live && n > 0;
    int all_holes, all_movers;
    const int h = before(hole, sums, all_holes), m = before(mover, sums, all_movers);
    if (hole) w.target[holes + h] = p;
    if (mover) w.source[movers + m] = p;
    if (p < a.n_pages) {
      if (!mover) a.moved_out[p] = n > 0 ? p : -1;
      if (!hole) a.refs_out[p] = p < live ? n : 0;
    }
    holes += all_holes;
    movers += all_movers;
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
  const int64_t pieces = pairs * c.start[c.n];
  return (uint32_t)(pieces < 2048 ? pieces : 2048);
}

}  // namespace

uint64_t fork_workspace(const fi_fork_pages_args& a) {
  const ForkSpace w(nullptr, a.rows, a.new_rows, a.n_pages);
  return (uint64_t)reinterpret_cast<uintptr_t>(w.end);
}

int launch_fork_pages(const fi_fork_pages_args& a, void* stream) {
  const hipStream_t s = static_cast<hipStream_t>(stream);
  if (a.rows <= SMALL_ROWS && a.new_rows <= SMALL_ROWS && (int64_t)a.rows * a.columns <= SMALL_TABLE && (int64_t)a.new_rows * a.columns <= SMALL_TABLE) {
    fork_small_kernel<<<dim3(1), THREADS, 0, s>>>(a);
  } else {
    const int64_t widest = a.n_pages > a.new_rows ? a.n_pages : a.new_rows, begin = (widest + 255) / 256;
    fork_begin_kernel<<<dim3((uint32_t)(begin < 1 ? 1 : begin < 2048 ? begin : 2048)), 256, 0, s>>>(a);
    if (a.new_rows) fork_children_kernel<<<dim3((a.new_rows + 255) / 256), 256, 0, s>>>(a);
    if (a.rows) fork_count_kernel<<<dim3(a.rows < 4096 ? a.rows : 4096), 256, 0, s>>>(a);
    if (a.new_rows) fork_need_kernel<<<dim3((a.new_rows + 3) / 4), 256, 0, s>>>(a);
    fork_deal_kernel<<<dim3(1), THREADS, 0, s>>>(a);
    if (a.new_rows) fork_write_kernel<<<dim3((a.new_rows + 3) / 4), 256, 0, s>>>(a);
  }
  if (a.room == 0 || a.new_rows == 0 || a.n_pages == 0) return (int)hipGetLastError();
  const ForkSpace w(a.workspace, a.rows, a.new_rows, a.n_pages);
  for (int at = 0; at < a.n_caches; at += Copies::MOST) {
    const Copies c = copies_of(a.caches, a.n_caches, at);
    if (c.n) fork_copy_kernel<<<dim3(copy_groups(c, a.new_rows)), 256, 0, s>>>(w.head, w.source, w.target, c);
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
