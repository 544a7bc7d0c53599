// What the attention kernels over a paged cache share, whatever the cache holds: which rows and keys a workgroup takes, what a node sees, and the parts of a row
// that a second launch joins.  A is the operator's argument struct; its fields of these names mean the same in all of them.
#pragma once

#include "fi_ops_device.h"

namespace fi {
namespace {

__device__ __forceinline__ int clamp_int(int v, int lo, int hi) { return v < lo ? lo : v > hi ? hi : v; }

__device__ __forceinline__ float wave_max(float v) {
  for (int o = 32; o; o >>= 1) v = fmaxf(v, __shfl_xor(v, o));
  return v;
}
__device__ __forceinline__ float wave_sum(float v) {
  for (int o = 32; o; o >>= 1) v += __shfl_xor(v, o);
  return v;
}

// The sequence that a packed row belongs to: the last one whose offset is not past it (offsets ascend; empty sequences have none).
__device__ __forceinline__ int find_seq(const int32_t* cu, int n, int row) {
  int lo = 0, hi = n - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (cu[mid] <= row) lo = mid;
    else hi = mid - 1;
  }
  return lo;
}

__device__ __forceinline__ uint32_t low_bits(int n) { return n <= 0 ? 0u : n >= 32 ? ~0u : (1u << n) - 1u; }

// What a workgroup of the tree kernels works on: a block of rows (node, head) of one key head of one sequence, and of its keys the tiles [t0, t1).
struct TreeWork {
  int b, hk, cached, keys, n0, nodes, block, split, splits, t0, t1;
};
// How a call is shared out (on the host): parts that a row can have, least tiles of a part, keys of a tile, what a stream costs beside its tiles, in tiles,
// rows of a block, blocks of a sequence at most, floats before the parts in the workspace.
struct TreeSplit { int splits, least, unit, over, rows, blocks, header; };

// A sequence as the kernels see it: its offsets and lengths clamped to the tensors.
template <typename A>
__device__ __forceinline__ void tree_sequence(const A& a, int b, TreeWork& w) {
  const int total = (int)a.nodes, places = a.n_pages ? a.page_size * a.table_columns : 0;
  w.b = b;
  w.n0 = clamp_int(a.cu_nodes[b], 0, total);
  w.nodes = clamp_int(a.cu_nodes[b + 1], w.n0, total) - w.n0;
  if (w.nodes > a.max_nodes) w.nodes = a.max_nodes;
  w.cached = clamp_int(a.cached[b], 0, places);
  w.keys = w.nodes < places - w.cached ? w.cached + w.nodes : places;
}
// The work of a call goes to the workgroups in one of two ways.
//  Direct: a workgroup for every part that a sequence can have, of equal size; parts that a shorter one has not end at once, but wait for a compute unit first.
//  Counted: as many workgroups as run at a time.  The first wave of each lines up the tiles of all streams (sequence, block, key head; a stream's beginning
//  counts for `over` tiles) and every workgroup takes its stretch of the line, wherever that begins and ends in a stream.
//  Lengths up to 8000, spread over their logarithm: 16 sequences of 32 key heads direct 253 us, counted 90; 64 of 8 key heads and ten nodes 344, 114; the last
//  with 8000 keys each 428, 479; 2 of 1000 keys 12, 19.
constexpr int SEQS = 256;   // most sequences that are counted
struct TreeLine {
  int start[SEQS];   // where a sequence begins
  int n0[SEQS], nodes[SEQS], cached[SEQS], keys[SEQS];
  int quota, total;
};
__device__ __forceinline__ int tiles_of(int keys, int unit) { return keys > unit ? (keys + unit - 1) / unit : 1; }
template <typename A>
__device__ __forceinline__ int streams_of(const A& a, const TreeSplit& p, int nodes) {
  return (nodes * (a.q_heads / a.kv_heads) + p.rows - 1) / p.rows * a.kv_heads;
}
template <typename A>
__device__ __forceinline__ void line_up(const A& a, const TreeSplit& p, TreeLine& line) {
  const int n = a.n_seqs, lane = threadIdx.x;
  if (threadIdx.x < 64) {
    int total = 0, longest = 1;
    for (int c = 0; c < n; c += 64) {
      const int b = c + lane;
      int upto = 0;
      if (b < n) {
        TreeWork w;
        tree_sequence(a, b, w);
        line.n0[b] = w.n0;
        line.nodes[b] = w.nodes;
        line.cached[b] = w.cached;
        line.keys[b] = w.keys;
        const int tiles = tiles_of(w.keys, p.unit);
        upto = streams_of(a, p, w.nodes) * (tiles + p.over);
        if (tiles > longest) longest = tiles;
      }
      const int mine = upto;
      for (int o = 1; o < 64; o <<= 1) {
        const int up = __shfl_up(upto, o);
        if (lane >= o) upto += up;
      }
      if (b < n) {
        line.start[b] = total + upto - mine;
        if (blockIdx.x == 0) static_cast<int*>(a.workspace)[4 + b] = total + upto - mine;   // (for the join)
      }
      total += __shfl(upto, 63);
    }
    for (int o = 32; o; o >>= 1) {
      const int other = __shfl_xor(longest, o);
      if (other > longest) longest = other;
    }
    if (lane == 0) {
      int quota = (total + (int)gridDim.x - 1) / (int)gridDim.x;
      if (quota < p.least) quota = p.least;
      const int fits = (longest + p.splits - 2) / (p.splits - 1);   // (a stretch may begin inside a tile's share: one part more)
      if (quota < fits) quota = fits;
      line.quota = quota;
      line.total = total;
      if (blockIdx.x == 0) *static_cast<int*>(a.workspace) = quota;
    }
  }
  __syncthreads();
}
// Parts of the stream that begins at `base` with `tiles` tiles: the workgroups whose stretches its tiles lie in.
__device__ __forceinline__ void parts_of(const TreeSplit& p, int base, int tiles, int quota, int& first, int& count) {
  first = (base + p.over) / quota;
  count = (base + p.over + tiles - 1) / quota - first + 1;
}
// Every piece of this workgroup's stretch.
template <typename A, typename Work>
__device__ __forceinline__ void along_the_line(const A& a, const TreeSplit& p, const TreeLine& line, Work work) {
  auto same = [](int v) { return __builtin_amdgcn_readfirstlane(v); };
  const int n = a.n_seqs, quota = same(line.quota), total = same(line.total);
  if ((int64_t)blockIdx.x * quota >= total) return;
  int pos = blockIdx.x * quota, b = 0;
  const int end = total - pos < quota ? total : pos + quota;
  for (int hi = n - 1; b < hi;) {   // the last sequence that begins here or before
    const int mid = (b + hi + 1) >> 1;
    if (same(line.start[mid]) <= pos) b = mid;
    else hi = mid - 1;
  }
  while (pos < end) {
    while (b + 1 < n && same(line.start[b + 1]) <= pos) ++b;
    TreeWork w;
    w.b = b;
    w.n0 = same(line.n0[b]);
    w.nodes = same(line.nodes[b]);
    w.cached = same(line.cached[b]);
    w.keys = same(line.keys[b]);
    const int tiles = tiles_of(w.keys, p.unit), per = tiles + p.over, start = same(line.start[b]), stream = (pos - start) / per, base = start + stream * per;
    w.hk = stream % a.kv_heads;
    w.block = stream / a.kv_heads;
    w.t0 = pos - base > p.over ? pos - base - p.over : 0;
    w.t1 = end - base - p.over < tiles ? end - base - p.over : tiles;
    if (w.t0 < w.t1) {
      int first;
      parts_of(p, base, tiles, quota, first, w.splits);
      w.split = (int)blockIdx.x - first;
      if (w.keys == 0) w.t1 = 0;
      work(w);
    }
    pos = base + per;
  }
}
// Shares of a sequence's keys in direct calls: `splits` at most, of `least` tiles or more.
__device__ __forceinline__ int shares(const TreeSplit& p, int keys) { return clamp_int((tiles_of(keys, p.unit) + p.least - 1) / p.least, 1, p.splits); }
// Direct: the grid is sequences and blocks, key heads, parts.  Every sequence has `blocks` blocks, or (packed, blocks 0) sequence b those from its first row over the
// rows of a block, plus b, on: enough for its rows wherever they start, and no more than one for each sequence than rows fill.
template <typename A>
__device__ __forceinline__ bool tree_direct(const A& a, const TreeSplit& p, TreeWork& w) {
  int b;
  if (p.blocks > 0) {
    b = p.blocks == 1 ? blockIdx.x : blockIdx.x / p.blocks;
    w.block = blockIdx.x - b * p.blocks;
  } else {
    const int group = a.q_heads / a.kv_heads, id = blockIdx.x, total = (int)a.nodes;
    auto begins = [&](int s) { return clamp_int(a.cu_nodes[s], 0, total) * group / p.rows + s; };
    b = 0;
    for (int hi = a.n_seqs - 1; b < hi;) {
      const int mid = (b + hi + 1) >> 1;
      if (begins(mid) <= id) b = mid;
      else hi = mid - 1;
    }
    w.block = id - begins(b);
    if (w.block < 0) return false;   // (offsets that do not ascend)
  }
  tree_sequence(a, b, w);
  w.hk = blockIdx.y;
  w.split = blockIdx.z;
  w.splits = shares(p, w.keys);
  const int tiles = w.keys ? tiles_of(w.keys, p.unit) : 0;
  w.t0 = (int)((int64_t)tiles * w.split / w.splits);
  w.t1 = (int)((int64_t)tiles * (w.split + 1) / w.splits);
  return w.split < w.splits && (int64_t)w.block * p.rows < w.nodes * (a.q_heads / a.kv_heads);
}

// Which of the 32 keys from `key` on a node (place `node` in its tree, mask row `words`) sees.
template <typename A>
__device__ __forceinline__ uint32_t tree_visible(const A& a, const TreeWork& w, int node, const uint64_t* words, int key) {
  const int base = key - w.cached;   // the tree's node that the first key is; below zero: committed
  uint32_t bits;
  if (!a.mask) bits = low_bits(node + 1 - base);
  else if (base < 0) bits = base <= -32 ? ~0u : low_bits(-base) | (uint32_t)words[0] << -base;
  else {
    const int at = base >> 6, sh = base & 63;
    uint64_t x = at < a.mask_words ? words[at] >> sh : 0;
    if (sh > 32 && at + 1 < a.mask_words) x |= words[at + 1] << (64 - sh);
    bits = (uint32_t)x;
  }
  return bits & low_bits(w.keys - key);
}

// The workspace: the line of a counted call (16 bytes with its quota, then where each sequence begins), then parts of a row (node, head): `splits` times
// head_dim sums, then for all rows the maximum and the weights' sum of each.
template <typename A>
__device__ __forceinline__ float* part_sums(const A& a, const TreeSplit& p, int64_t row, int split) {
  return static_cast<float*>(a.workspace) + p.header + (row * p.splits + split) * a.head_dim;
}
template <typename A>
__device__ __forceinline__ float* part_stats(const A& a, const TreeSplit& p, int64_t row, int split) {
  return static_cast<float*>(a.workspace) + p.header + a.nodes * a.q_heads * p.splits * a.head_dim + (row * p.splits + split) * 2;
}

// Joins the parts of a row (node, head), in their order and 16 in flight at once (they come from other dies: a load takes microseconds).  A wave per row: with
// thousands of them its instructions count, so everything that the row's lanes share is scalar and a lane has PER values next to each other.  WIDE (more
// parts of few rows): a workgroup per row, its waves add a quarter of the parts each, then the waves' sums are added.
template <typename A, typename T, int PER, bool WIDE>
__global__ void __launch_bounds__(256) tree_join_kernel(A a, TreeSplit p, bool counted) {
  typedef float vec __attribute__((ext_vector_type(PER)));
  __shared__ vec sums[3][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), D = a.head_dim;
  const int row = WIDE ? (int)blockIdx.x : (int)blockIdx.x * 4 + wave;   // (rows are below 2^31)
  if (row >= (int)a.nodes * a.q_heads) return;
  const int node = row / a.q_heads, head = row - node * a.q_heads;
  const int b = find_seq(a.cu_nodes, a.n_seqs, node);
  TreeWork w;
  tree_sequence(a, b, w);
  if (node < w.n0 || node - w.n0 >= w.nodes) return;
  if (counted) {
    const int* const line = static_cast<const int*>(a.workspace);
    const int group = a.q_heads / a.kv_heads, hk = head / group, block = ((node - w.n0) * group + head - hk * group) / p.rows, tiles = tiles_of(w.keys, p.unit);
    int first;
    parts_of(p, line[4 + b] + (block * a.kv_heads + hk) * (tiles + p.over), tiles, line[0], first, w.splits);
  } else {
    w.splits = shares(p, w.keys);
  }
  if (w.splits == 1) return;
  const float c = a.scale * 1.44269504f;
  const bool inside = lane * PER < D;   // (D is a multiple of four)
  const float* const parts = part_sums(a, p, row, 0) + (inside ? lane * PER : 0);
  // lane s has part s (64 at most): the weights of all parts at once
  const float2 mine = lane < w.splits ? *reinterpret_cast<const float2*>(part_stats(a, p, row, lane)) : make_float2(-INFINITY, 0.0f);
  const int each = WIDE ? (w.splits + 3) / 4 : w.splits, s0 = WIDE ? wave * each : 0, s1 = s0 + each < w.splits ? s0 + each : w.splits;
  vec acc = 0.0f, x[16];
  auto ask = [&](int from) {
#pragma unroll
    for (int s = 0; s < 16; ++s)
      if (from + s < s1) x[s] = *reinterpret_cast<const vec*>(parts + (int64_t)(from + s) * D);
  };
  ask(s0);
  const float top = wave_max(mine.x), base = top == -INFINITY ? 0.0f : top;
  const float weight = lane < w.splits ? __builtin_amdgcn_exp2f((mine.x - base) * c) : 0.0f, total = wave_sum(lane < w.splits ? mine.y * weight : 0.0f);
  for (int from = s0; from < s1; from += 16) {
    if (from > s0) ask(from);
#pragma unroll
    for (int s = 0; s < 16; ++s)
      if (from + s < s1) acc += x[s] * __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(weight), from + s));
  }
  if constexpr (WIDE) {
    if (wave) sums[wave - 1][lane] = acc;
    __syncthreads();
    if (wave) return;
    acc = acc + sums[0][lane] + sums[1][lane] + sums[2][lane];
  }
  const float inv = total == 0.0f ? 0.0f : 1.0f / total;
  T* const out = static_cast<T*>(a.out) + node * a.out_strides[0] + head * a.out_strides[1] + lane * PER;
  if (!inside) return;
#pragma unroll
  for (int i = 0; i < PER; ++i) st(out + i, acc[i] * inv);
}

}  // namespace
}  // namespace fi
