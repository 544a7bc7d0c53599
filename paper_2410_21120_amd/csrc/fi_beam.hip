// Beam search's selection: the best continuations of every sequence over its beams and the vocabulary.
//
// Two launches.  The first reads the logits once: a wave holds a stretch of a row in registers, all of its loads on their way at once, and goes over it three times: the lanes'
// maxima, which give a border that hardly more than `keep` of the workgroup's values reach; the softmax's sum; the values that reach the border, which are
// sorted over the lanes of one wave.  The second has a workgroup a sequence: it joins the waves' sums and lists row by row, and finds a candidate's place among all rows' by
// looking it up in each of their sorted lists.
// Scores of different beams lie close, so sums of waves are joined and scores made in 64 bits; terms, and the sums of at most 64 of them by a lane, are fp32.  A log-sum is off by less than 1e-5 by
// that (scores by 2.6e-8 of their size as measured), and beams that lie closer may change places.
#include <hip/hip_runtime.h>

#include "fi_device.h"
#include "fi_ops.h"

namespace fi {
namespace {

constexpr int WAVES = 4, LIST = 64;   // waves of a workgroup of the first launch
// A logit and its token as a number that orders them: larger logits first, then smaller tokens.  0: none.
__device__ __forceinline__ uint64_t key_of(float x, uint32_t token) {
  const uint32_t b = __float_as_uint(x + 0.0f);   // (-0 is 0)
  return (uint64_t)(b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u)) << 32 | (uint32_t)~token;
}
__device__ __forceinline__ float logit_of(uint64_t key) {
  const uint32_t b = (uint32_t)(key >> 32);
  return __uint_as_float(b & 0x80000000u ? b ^ 0x80000000u : ~b);
}
__device__ __forceinline__ uint32_t token_of(uint64_t key) { return ~(uint32_t)key; }

// The value of lane ^ D by vector instructions alone (through LDS, as shuffles go, a sort takes twice as long).
template <int D>
__device__ __forceinline__ uint32_t lane_xor(uint32_t x) {
  if constexpr (D == 1) return __builtin_amdgcn_update_dpp(0, x, 0xB1, 0xF, 0xF, true);        // quad_perm [1, 0, 3, 2]
  else if constexpr (D == 2) return __builtin_amdgcn_update_dpp(0, x, 0x4E, 0xF, 0xF, true);   // quad_perm [2, 3, 0, 1]
  else if constexpr (D == 4) return lane_xor<1>(lane_xor<2>(__builtin_amdgcn_update_dpp(0, x, 0x141, 0xF, 0xF, true)));   // halves of a row mirrored: ^ 7
  else if constexpr (D == 8) return __builtin_amdgcn_update_dpp(0, x, 0x128, 0xF, 0xF, true);  // a row rotated by 8
  else {
    const auto r = [&] {
      if constexpr (D == 16) return __builtin_amdgcn_permlane16_swap(x, x, false, false);
      else return __builtin_amdgcn_permlane32_swap(x, x, false, false);
    }();
    return threadIdx.x & D ? r[0] : r[1];
  }
}
template <int D>
__device__ __forceinline__ uint64_t swapped(uint64_t x) { return (uint64_t)lane_xor<D>((uint32_t)(x >> 32)) << 32 | lane_xor<D>((uint32_t)x); }
__device__ __forceinline__ uint64_t from_lane(uint64_t x, int lane) {   // lane: the same for the wave
  return (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(x >> 32), lane) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)x, lane);
}
// Lanes sorted, the largest first; bitonic.  merge: of a sequence that rises and falls at most once.
template <int D>
__device__ __forceinline__ uint64_t exchange(uint64_t x, bool first) {   // first: this lane gets the larger one
  const uint64_t y = swapped<D>(x);
  return first == (x > y) ? x : y;
}
__device__ __forceinline__ uint64_t merge64(uint64_t x) {
  const int lane = threadIdx.x & 63;
  x = exchange<32>(x, !(lane & 32));
  x = exchange<16>(x, !(lane & 16));
  x = exchange<8>(x, !(lane & 8));
  x = exchange<4>(x, !(lane & 4));
  x = exchange<2>(x, !(lane & 2));
  return exchange<1>(x, !(lane & 1));
}
__device__ __noinline__ uint64_t sort64(uint64_t x) {   // (a call: where it is needed is rarely reached, and its instructions would be fetched with those around)
  const int lane = threadIdx.x & 63;
  auto up = [&](int n, int d) { return !(lane & n) == !(lane & d); };
  x = exchange<1>(x, up(2, 1));
  x = exchange<2>(x, up(4, 2));
  x = exchange<1>(x, up(4, 1));
  x = exchange<4>(x, up(8, 4));
  x = exchange<2>(x, up(8, 2));
  x = exchange<1>(x, up(8, 1));
  x = exchange<8>(x, up(16, 8));
  x = exchange<4>(x, up(16, 4));
  x = exchange<2>(x, up(16, 2));
  x = exchange<1>(x, up(16, 1));
  x = exchange<16>(x, up(32, 16));
  x = exchange<8>(x, up(32, 8));
  x = exchange<4>(x, up(32, 4));
  x = exchange<2>(x, up(32, 2));
  x = exchange<1>(x, up(32, 1));
  return merge64(x);
}
// The n-th and the m-th largest (from 0) of the lanes' values.
template <int D>
__device__ __forceinline__ float exchange(float x, bool first) {
  const float y = __uint_as_float(lane_xor<D>(__float_as_uint(x)));
  return first ? fmaxf(x, y) : fminf(x, y);
}
__device__ __forceinline__ void nth64(float x, int n, int m, float& nth, float& mth) {
  const int lane = threadIdx.x & 63;
  auto up = [&](int n, int d) { return !(lane & n) == !(lane & d); };
  x = exchange<1>(x, up(2, 1));
  x = exchange<2>(x, up(4, 2));
  x = exchange<1>(x, up(4, 1));
  x = exchange<4>(x, up(8, 4));
  x = exchange<2>(x, up(8, 2));
  x = exchange<1>(x, up(8, 1));
  x = exchange<8>(x, up(16, 8));
  x = exchange<4>(x, up(16, 4));
  x = exchange<2>(x, up(16, 2));
  x = exchange<1>(x, up(16, 1));
  x = exchange<16>(x, up(32, 16));
  x = exchange<8>(x, up(32, 8));
  x = exchange<4>(x, up(32, 4));
  x = exchange<2>(x, up(32, 2));
  x = exchange<1>(x, up(32, 1));
  x = exchange<32>(x, up(64, 32));
  x = exchange<16>(x, up(64, 16));
  x = exchange<8>(x, up(64, 8));
  x = exchange<4>(x, up(64, 4));
  x = exchange<2>(x, up(64, 2));
  x = exchange<1>(x, up(64, 1));
  nth = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(x), n));
  mth = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(x), m));
}
// Over all lanes, in an order that is the same for every lane.
__device__ __forceinline__ float max64(float x) {
  x = fmaxf(x, __uint_as_float(lane_xor<1>(__float_as_uint(x))));
  x = fmaxf(x, __uint_as_float(lane_xor<2>(__float_as_uint(x))));
  x = fmaxf(x, __uint_as_float(lane_xor<4>(__float_as_uint(x))));
  x = fmaxf(x, __uint_as_float(lane_xor<8>(__float_as_uint(x))));
  x = fmaxf(x, __uint_as_float(lane_xor<16>(__float_as_uint(x))));
  return fmaxf(x, __uint_as_float(lane_xor<32>(__float_as_uint(x))));
}
template <int D>
__device__ __forceinline__ double lane_xor(double x) { return __builtin_bit_cast(double, swapped<D>(__builtin_bit_cast(uint64_t, x))); }
__device__ __forceinline__ double sum64(double x) {
  x += lane_xor<1>(x);
  x += lane_xor<2>(x);
  x += lane_xor<4>(x);
  x += lane_xor<8>(x);
  x += lane_xor<16>(x);
  return x + lane_xor<32>(x);
}
// The 64 largest of two sorted sets of lanes, sorted.
__device__ __noinline__ uint64_t best64(uint64_t a, uint64_t b) {
  b = swapped<32>(swapped<16>(swapped<8>(swapped<4>(swapped<2>(swapped<1>(b))))));   // backwards
  return merge64(a > b ? a : b);
}

// The 64 best keys that a wave has seen, sorted over its lanes, and a list in LDS of those that came since.
struct Best {
  uint64_t mine, border;   // border: the keep-th best, the same for the wave; what does not beat it is of no interest
  uint64_t* list;
  int count, keep;
  bool some;
  __device__ __forceinline__ Best(uint64_t* l, int k) : mine(0), border(0), list(l), count(0), keep(k), some(false) {}
  __device__ __forceinline__ void flush() {
    if (!count) return;
    const int lane = threadIdx.x & 63;
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    const uint64_t x = lane < count ? *(volatile uint64_t*)(list + lane) : 0;
    mine = some ? best64(mine, sort64(x)) : sort64(x);
    some = true;
    raise(from_lane(mine, keep - 1));
    count = 0;
  }
  __device__ __forceinline__ void begin(uint64_t ranked) {   // with a sorted set
    mine = ranked;
    some = true;
    raise(from_lane(mine, keep - 1));
  }
  __device__ __forceinline__ void raise(uint64_t to) { border = to > border ? to : border; }
  __device__ __forceinline__ void offer(uint64_t key) {
    if (count + __popcll(__ballot(key > border)) > LIST) flush();
    append(key);
  }
  // There is room for them: logits and tokens of the lanes of `in`.
  __device__ __forceinline__ void append(uint64_t in, float logit, uint32_t token) {
    if (in >> (threadIdx.x & 63) & 1) ((volatile uint64_t*)list)[count + __builtin_amdgcn_mbcnt_hi((uint32_t)(in >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)in, 0))] = logit > -INFINITY ? key_of(logit, token) : 0;
    count += __popcll(in);
  }
  __device__ __forceinline__ void append(uint64_t key) {
    const uint64_t in = __ballot(key > border);
    if (key > border) ((volatile uint64_t*)list)[count + __popcll(in & ((1ull << (threadIdx.x & 63)) - 1))] = key;
    count += __popcll(in);
  }
};

// What a wave leaves of its stretch: sum of 2^(x log2 e - base), and the best keys.
struct Part {
  double sum;
  float base, reserved;
};
constexpr float LOG2E = 1.44269504f, LOG2E_REST = 1.92596303e-8f;   // (log2 e - LOG2E)
constexpr float LARGEST = 3.40282347e38f;

// sum 2^(base - to), to >= base: whole numbers both.
__device__ __forceinline__ double scaled(double sum, float base, float to) { return ldexp(sum, (int)fmaxf(base - to, -4096.0f)); }

// How a call is shared out: stretches of `stretch` logits, four to a workgroup; `strips` workgroups a row.
struct BeamSplit { int strips, stretch; };

__device__ __forceinline__ bool beam_counts(const fi_beam_select_args& a, int row) {   // whether the row's logits are looked at
  const float s = a.scores[row];
  return !(a.ended && a.ended[row]) && s > -INFINITY;   // (a NaN does not)
}

// Eight logits of a lane: values i of piece `at`, which the row's end may have moved forward (clamped); those before `first` are another lane's.
template <typename T>
struct Eight {
  static constexpr int N = 16 / sizeof(T), PIECES = 8 / N;
  typedef uint32_t piece __attribute__((ext_vector_type(4), aligned(2)));
  piece w[PIECES];
  __device__ __forceinline__ void load(const T* p) {
#pragma unroll
    for (int i = 0; i < PIECES; ++i) w[i] = reinterpret_cast<const piece*>(p)[i];
  }
  __device__ __forceinline__ float at(int i) const {
    if constexpr (N == 4) return __uint_as_float(w[i >> 2][i & 3]);
    else return __uint_as_float(i & 1 ? w[0][i >> 1] & 0xFFFF0000u : w[0][i >> 1] << 16);
  }
  __device__ __forceinline__ void hide(int i) {   // to minus infinity
    if constexpr (N == 4) w[i >> 2][i & 3] = 0xFF800000u;
    else w[0][i >> 1] = i & 1 ? (w[0][i >> 1] & 0xFFFFu) | 0xFF800000u : (w[0][i >> 1] & 0xFFFF0000u) | 0xFF80u;
  }
};

// Which lane has which values goes by their place in the row alone, not by where the row starts in memory: rows that are alike get sums that are alike to the last bit, and tie.
// 512 rows of 131072 fp32 logits, sixteen kept: 43 us, HBM at 6.2 TB/s (vector unit busy for 20 of them).  4096 logits a wave: with 8192 (two waves on a unit instead of four) 47.
// What made the difference is how few values reach the border: with the keep-th largest of each wave's maxima as its own border, a list, a sort and a merge a wave, 50 to 59; with a
// running maximum and list, values a step ahead in registers, 48 to 73.  4 rows of 32000: 4.5 us, of which the launch is most.
template <typename T, int STEPS>
__global__ void __launch_bounds__(64 * WAVES) beam_scan_kernel(fi_beam_select_args a, BeamSplit p) {
  __shared__ uint64_t lists[WAVES][LIST], sorted[WAVES][LIST];
  __shared__ float4 hint[WAVES];
  __shared__ double sums[WAVES];
  __shared__ int counts[WAVES];
  static_assert(WAVES == 4, "");
  const int row = blockIdx.x / p.strips, strip = blockIdx.x - row * p.strips, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int64_t begin = ((int64_t)strip * WAVES + wave) * (STEPS * 512);
  // A lane's places count from the stretch's beginning: sums of a place in the row and a stretch may pass 2^31.
  const int from = (int)(begin < a.vocab ? begin : a.vocab), size = a.vocab - from < STEPS * 512 ? a.vocab - from : STEPS * 512;
  const T* const logits = static_cast<const T*>(a.logits) + row * a.logits_stride;
  Eight<T> x[STEPS];
  const bool whole = size == STEPS * 512;
  auto place = [&](int u) {   // where piece u of this lane lies: before the stretch, where that is shorter than a piece
    const int at = u * 512 + lane * 8;
    return from + (at + 8 <= size ? at : size - 8);
  };
  if (a.vocab >= 8) {
#pragma unroll
    for (int u = 0; u < STEPS; ++u)
      if (u * 512 < size) x[u].load(logits + place(u));
  }
  if (!beam_counts(a, row)) return;
  if (!whole) {
#pragma unroll
    for (int u = 0; u < STEPS; ++u) {
      const int at = u * 512 + lane * 8;
      if (u * 512 + 512 <= size) continue;
      if (a.vocab >= 8) {
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (u * 512 >= size || place(u) - from + i < at) x[u].hide(i);
      } else {   // (a row shorter than a piece)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float y = u == 0 && at + i < size ? ld(logits + from + at + i) : -INFINITY;
          if constexpr (sizeof(T) == 4) x[u].w[i >> 2][i & 3] = __float_as_uint(y);
          else x[u].w[0][i >> 1] = i & 1 ? (x[u].w[0][i >> 1] & 0xFFFFu) | (__float_as_uint(y) & 0xFFFF0000u) : __float_as_uint(y) >> 16;
        }
      }
    }
  }
  float tops[STEPS], top = -INFINITY;
#pragma unroll
  for (int u = 0; u < STEPS; ++u) {
    tops[u] = x[u].at(0);
#pragma unroll
    for (int i = 1; i < 8; ++i) tops[u] = fmaxf(tops[u], x[u].at(i));
    top = fmaxf(top, tops[u]);
  }
  // The border: `keep` values at least reach the keep-th largest of a wave's maxima, and the least of what a quarter of `keep` reach in every wave.
  const int quarter = (a.keep + WAVES - 1) / WAVES;
  float many_th, few_th;
  nth64(top, a.keep - 1, quarter - 1, many_th, few_th);
  const float highest_here = max64(top);
  if (lane == 0) hint[wave] = make_float4(highest_here, many_th, few_th, 0.0f);
  __syncthreads();
  float highest = hint[0].x, border = hint[0].y, all_reach = hint[0].z;
#pragma unroll
  for (int w = 1; w < WAVES; ++w) {
    highest = fmaxf(highest, hint[w].x);
    border = fmaxf(border, hint[w].y);
    all_reach = fminf(all_reach, hint[w].z);
  }
  border = fmaxf(border, all_reach);
  // base is a whole number, so that sums of other bases are added exactly, and x log2 e - base is rounded once
  const float base = fminf(fmaxf(ceilf(highest * LOG2E), -LARGEST), LARGEST);
  float sum = 0.0f;
#pragma unroll
  for (int u = 0; u < STEPS; ++u)
#pragma unroll
    for (int i = 0; i < 8; ++i) sum += __builtin_amdgcn_exp2f(__builtin_fmaf(x[u].at(i), LOG2E_REST, __builtin_fmaf(x[u].at(i), LOG2E, -base)));
  Best best(lists[wave], a.keep);
#pragma unroll
  for (int u = 0; u < STEPS; ++u) {
    if (!__any(tops[u] >= border)) continue;
    uint64_t in[8];
    int many = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      in[i] = __ballot(x[u].at(i) >= border);
      many += __popcll(in[i]);
    }
    const uint32_t token = (uint32_t)((a.vocab >= 8 ? place(u) : from + lane * 8));
    if (many + best.count > LIST) best.flush();
    if (many <= LIST) {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (in[i]) best.append(in[i], x[u].at(i), token + i);
    } else {   // (ties, or nearly all asked for)
#pragma unroll 1
      for (int i = 0; i < 8; ++i) {
        float y = x[u].at(0);
#pragma unroll
        for (int k = 1; k < 8; ++k) y = i == k ? x[u].at(k) : y;
        best.offer(y > -INFINITY ? key_of(y, token + i) : 0);
      }
    }
  }
  // the workgroup's list and sum, by its first wave: what the waves found together is mostly 64 values at most, and sorted once
  if (best.some) sorted[wave][lane] = best.mine;
  const double mine = sum64((double)sum);
  if (lane == 0) {
    sums[wave] = mine;
    counts[wave] = best.count | (best.some ? 256 : 0);
  }
  __syncthreads();
  if (wave) return;
  const int n0 = counts[0], n1 = counts[1], n2 = counts[2], n3 = counts[3], n = n0 + n1 + n2 + n3;   // (64 and 256 at most each)
  uint64_t found = 0;
  if (n <= LIST) {
    const int w = lane < n0 ? 0 : lane < n0 + n1 ? 1 : lane < n0 + n1 + n2 ? 2 : 3, at = lane - (w > 0 ? n0 : 0) - (w > 1 ? n1 : 0) - (w > 2 ? n2 : 0);
    found = sort64(lane < n ? lists[w][at] : 0);
  } else {
#pragma unroll 1
    for (int w = 0; w < WAVES; ++w) {
      const int c = counts[w] & 255;
      if (c) found = best64(found, sort64(lane < c ? lists[w][lane] : 0));
      if (counts[w] & 256) found = best64(found, sorted[w][lane]);
    }
  }
  const double total = sums[0] + sums[1] + sums[2] + sums[3];
  Part* const out = static_cast<Part*>(a.workspace) + (int64_t)row * p.strips + strip;
  uint64_t* const keys = reinterpret_cast<uint64_t*>(static_cast<Part*>(a.workspace) + (int64_t)a.n_seqs * a.beams * p.strips) + ((int64_t)row * p.strips + strip) * a.keep;
  if (lane == 0) *out = Part{total, base, 0.0f};
  if (lane < a.keep) keys[lane] = found;
}

// log of the sum of exp over a row, by its definition in 64 bits: for rows whose sum left the range of 32.
template <typename T, int JOIN_WAVES>
__device__ double log_sum(const T* row, int vocab, double* lds) {
  double top = -INFINITY, sum = 0.0;
  bool nan = false;
  for (int t = threadIdx.x; t < vocab; t += 64 * JOIN_WAVES) {
    const double x = ld(row + t);
    nan |= x != x;
    top = fmax(top, x);
  }
  auto all = [&](double x, bool add) {
    __syncthreads();
    lds[threadIdx.x] = x;
    __syncthreads();
    double r = lds[0];
    for (int i = 1; i < 64 * JOIN_WAVES; ++i) r = add ? r + lds[i] : fmax(r, lds[i]);
    return r;
  };
  top = all(nan ? INFINITY : top, false);
  if (!(fabs(top) < INFINITY)) return NAN;
  for (int t = threadIdx.x; t < vocab; t += 64 * JOIN_WAVES) sum += exp((double)ld(row + t) - top);
  return top + log(all(sum, true));
}

// A candidate's place: better scores first, then by beam, then by place in its row's list.
template <typename T, int JOIN_WAVES>
__global__ void __launch_bounds__(64 * JOIN_WAVES) beam_join_kernel(fi_beam_select_args a, BeamSplit p) {
  extern __shared__ double scores[];                                              // [beams][keep], of every row the best first
  uint64_t* const found = reinterpret_cast<uint64_t*>(scores);                    // (before its scores are known: a row's keys, in the same places)
  int* const tokens = reinterpret_cast<int*>(scores + a.beams * a.keep);          // [beams][keep]
  __shared__ uint64_t lists[JOIN_WAVES][LIST];
  __shared__ double sums[FI_MAX_BEAMS], lds[64 * JOIN_WAVES];
  __shared__ int counts[FI_MAX_BEAMS], odd;
  const int s = blockIdx.x, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const Part* const parts = static_cast<const Part*>(a.workspace);
  const uint64_t* const keys = reinterpret_cast<const uint64_t*>(parts + (int64_t)a.n_seqs * a.beams * p.strips);
  if (threadIdx.x == 0) odd = 0;
  __syncthreads();
  // A wave's rows: their sums and lists.
  constexpr double LN2 = 0.69314718055994530942;
  for (int b = wave; b < a.beams; b += JOIN_WAVES) {
    const int row = s * a.beams + b, n = p.strips * a.keep;
    const Part* const mine = parts + (int64_t)row * p.strips;
    const uint64_t* const list = keys + (int64_t)row * n;
    // (asked for before it is known whether they count: in rows that do not they are anything)
    uint64_t best = lane < n ? list[lane] : 0;
    const uint64_t second = lane + 64 < n ? list[lane + 64] : 0;
    Part first = {0.0, -LARGEST, 0.0f};
    if (lane < p.strips) first = mine[lane];
    const float score = a.scores[row];
    const bool over = a.ended && a.ended[row];
    int count = 0;
    if (over || !(score > -INFINITY)) {
      count = over && score > -INFINITY;
      if (lane == 0 && count) {
        scores[b * a.keep] = score;
        tokens[b * a.keep] = a.end;
      }
    } else {
      float top = first.base;
      double sum = first.sum;
      for (int i = lane + 64; i < p.strips; i += 64) {
        const Part x = mine[i];
        const float up = fmaxf(top, x.base);
        sum = scaled(sum, top, up) + scaled(x.sum, x.base, up);
        top = up;
      }
      const float highest = max64(top);
      sum = sum64(scaled(sum, top, highest));
      if (lane == 0) {
        sums[b] = ((double)highest + log2(sum)) * LN2;
        if (!(sum > 0.0 && sum < INFINITY && fabsf(highest) < 1e38f)) sums[b] = NAN, odd = 1;
      }
      if (p.strips > 1) best = sort64(best);   // (one stretch's list is sorted)
      if (n > 64) best = best64(best, sort64(second));
      if (n > 128) {
        Best all(lists[wave], a.keep);
        all.begin(best);
        for (int i = 128; i < n; i += 64) all.offer(i + lane < n ? list[i + lane] : 0);
        all.flush();
        best = all.mine;
      }
      if (lane < a.keep) found[b * a.keep + lane] = best;
      count = -1;
    }
    if (lane == 0) counts[b] = count;
  }
  __syncthreads();
  if (odd)
    for (int b = 0; b < a.beams; ++b) {
      if (counts[b] >= 0 || sums[b] == sums[b]) continue;   // (the same for the workgroup: sums are written below by all of it)
      const double exact = log_sum<T, JOIN_WAVES>(static_cast<const T*>(a.logits) + (int64_t)(s * a.beams + b) * a.logits_stride, a.vocab, lds);
      __syncthreads();
      if (threadIdx.x == 0) sums[b] = exact, counts[b] = -2;
      __syncthreads();
    }
  for (int b = wave; b < a.beams; b += JOIN_WAVES) {   // their scores
    if (counts[b] >= 0) continue;
    const uint64_t key = lane < a.keep ? found[b * a.keep + lane] : 0;
    const double value = (double)a.scores[s * a.beams + b] + ((double)logit_of(key) - sums[b]);
    const bool there = key != 0 && value > -INFINITY;
    if (there) {
      scores[b * a.keep + lane] = value;
      tokens[b * a.keep + lane] = (int)token_of(key);
    }
    const int count = __popcll(__ballot(there));   // (values fall from lane to lane)
    if (lane == 0) counts[b] = count;
  }
  __syncthreads();
  int total = 0;
  for (int b = 0; b < a.beams; ++b) total += counts[b];
  // `sharing` threads look a candidate up in some of the rows each, AT_ONCE rows at a time, until `keep` others are known to come first.  Those that are as far down their rows'
  // lists are looked up together: the further down, the sooner they are done.
  const int candidates = a.beams * a.keep, half = 1 << (31 - __clz(a.keep));
  int sharing = 1;
  while (sharing < 8 && sharing * 2 <= a.beams && sharing * 2 * candidates <= 64 * JOIN_WAVES) sharing *= 2;
  for (int i0 = 0; i0 < candidates; i0 += 64 * JOIN_WAVES / sharing) {
    constexpr int AT_ONCE = JOIN_WAVES == 8 ? 2 : 4;   // (up to 8 beams, 4 at once: 4.6 us for 4.3, what is not there is looked up, too)
    const int i = i0 + (int)threadIdx.x / sharing, part = (int)threadIdx.x & (sharing - 1);
    const int at = i < candidates ? i / a.beams : 0, b = i < candidates ? i - at * a.beams : 0;
    const bool there = i < candidates && at < counts[b];
    const double value = there ? scores[b * a.keep + at] : 0.0;
    int place = part == 0 ? at : 0;
    for (int o0 = part; o0 < a.beams && __any(there && place < a.keep); o0 += AT_ONCE * sharing) {
      int row[AT_ONCE], rows[AT_ONCE], most[AT_ONCE], first[AT_ONCE];   // first: how many of the row come first: those that are larger, or as large in a row before
#pragma unroll
      for (int u = 0; u < AT_ONCE; ++u) {
        row[u] = o0 + u * sharing;
        const bool other = row[u] < a.beams && row[u] != b;
        rows[u] = other ? row[u] * a.keep : 0;
        most[u] = other ? counts[row[u]] : 0;
        first[u] = 0;
      }
      for (int step = half; step; step >>= 1)
#pragma unroll
        for (int u = 0; u < AT_ONCE; ++u) {
          const int to = first[u] + step;
          const double other = scores[rows[u] + (to <= most[u] ? to : 1) - 1];
          if (to <= most[u] && (other > value || (other == value && row[u] < b))) first[u] = to;
        }
#pragma unroll
      for (int u = 0; u < AT_ONCE; ++u) place += first[u];
    }
    for (int o = 1; o < sharing; o <<= 1) place += __shfl_xor(place, o);
    if (!there || part || place >= a.keep) continue;
    const int row = s * a.beams + b, to = s * a.keep + place, token = tokens[b * a.keep + at];
    a.tokens_out[to] = token;
    a.parents_out[to] = row;
    a.scores_out[to] = (float)value;
    if (a.ended_out) a.ended_out[to] = token == a.end || (a.ended && a.ended[row]);
  }
  for (int place = total + threadIdx.x; place < a.keep; place += 64 * JOIN_WAVES) {
    const int to = s * a.keep + place;
    a.tokens_out[to] = -1;
    a.parents_out[to] = -1;
    a.scores_out[to] = -INFINITY;
    if (a.ended_out) a.ended_out[to] = 0;
  }
}

// Stretches as short as the chip has workgroups for and the join has registers for lists (3 sequences of 5 beams, 126434 tokens, 10 kept: 16.9 us by the first alone, so 14.8; one
// of 16 beams, 131072 tokens, 32 kept: 38.4 and 27.3).
BeamSplit plan_beams(const fi_beam_select_args& a) {
  const int64_t rows = (int64_t)a.n_seqs * a.beams;
  auto strips = [&](int64_t stretch) { return a.vocab ? (a.vocab + WAVES * stretch - 1) / (WAVES * stretch) : 1; };
  int stretch = 512;
  while (stretch < 4096 && a.vocab > WAVES * stretch && (rows * strips(stretch) > 1024 || strips(stretch) * a.keep > 128)) stretch *= stretch == 512 ? 4 : 2;
  return BeamSplit{(int)strips(stretch), stretch};
}
template <typename T>
void launch_beam_scan(const fi_beam_select_args& a, const BeamSplit& p, uint32_t groups, hipStream_t s) {
  if (p.stretch == 512) beam_scan_kernel<T, 1><<<dim3(groups), 64 * WAVES, 0, s>>>(a, p);
  else if (p.stretch == 2048) beam_scan_kernel<T, 4><<<dim3(groups), 64 * WAVES, 0, s>>>(a, p);
  else beam_scan_kernel<T, 8><<<dim3(groups), 64 * WAVES, 0, s>>>(a, p);
}
// A wave a row, up to 16 (6 sequences of 16 beams, 32 kept, 669 tokens, 8 waves / 16: 14.0 us / 9.8).
template <typename T>
void launch_beam_join(const fi_beam_select_args& a, const BeamSplit& p, hipStream_t s) {
  const uint32_t lds = (uint32_t)(a.beams * a.keep * 12);
  if (a.beams <= 8) beam_join_kernel<T, 8><<<dim3((uint32_t)a.n_seqs), 64 * 8, lds, s>>>(a, p);
  else beam_join_kernel<T, 16><<<dim3((uint32_t)a.n_seqs), 64 * 16, lds, s>>>(a, p);
}

}  // namespace

uint64_t beam_workspace(const fi_beam_select_args& a) {
  const BeamSplit p = plan_beams(a);
  return (uint64_t)a.n_seqs * a.beams * p.strips * (sizeof(Part) + 8ull * a.keep);
}

int launch_beam_select(const fi_beam_select_args& a, void* stream) {
  const hipStream_t s = static_cast<hipStream_t>(stream);
  const BeamSplit p = plan_beams(a);
  const int64_t groups = (int64_t)a.n_seqs * a.beams * p.strips;
  if (!one_launch(groups, 64 * WAVES) || !one_launch(a.n_seqs, 64 * 16)) return kTooLarge;
  if (a.dtype == FI_F32) {
    launch_beam_scan<float>(a, p, (uint32_t)groups, s);
    launch_beam_join<float>(a, p, s);
  } else {
    launch_beam_scan<bf16_t>(a, p, (uint32_t)groups, s);
    launch_beam_join<bf16_t>(a, p, s);
  }
  return (int)hipGetLastError();
}

}  // namespace fi
