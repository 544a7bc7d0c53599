// Beam search's selection: the best continuations of every sequence over its beams and the vocabulary.
//
// Two launches.  The first reads the logits once: a wave goes through a stretch of a row with the running maximum and sum of the softmax and the 64 best logits so far, sorted, one
// a lane; a value enters a list in LDS only if it beats the keep-th of them, which after the first few thousand values hardly one does, and every 64 of these are
// sorted and merged.  The second has a workgroup a sequence: it joins the waves' sums and lists row by row, and finds a candidate's place among all rows' by
// looking it up in each of their sorted lists.
// Scores of different beams lie close and their order must be right, so sums of waves are joined and scores made in 64 bits.
#include <hip/hip_runtime.h>

#include "fi_device.h"
#include "fi_ops.h"

namespace fi {
namespace {

constexpr int WAVES = 4, LIST = 64;
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

__device__ __forceinline__ uint64_t swapped(uint64_t x, int with) {
  const uint32_t lo = (uint32_t)__shfl_xor((int)(uint32_t)x, with), hi = (uint32_t)__shfl_xor((int)(uint32_t)(x >> 32), with);
  return (uint64_t)hi << 32 | lo;
}
__device__ __forceinline__ uint64_t from_lane(uint64_t x, int lane) {
  const uint32_t lo = (uint32_t)__shfl((int)(uint32_t)x, lane), hi = (uint32_t)__shfl((int)(uint32_t)(x >> 32), lane);
  return (uint64_t)hi << 32 | lo;
}
// Lanes sorted, the largest first; bitonic.  merge: of a sequence that rises and falls at most once.
__device__ __forceinline__ uint64_t merge64(uint64_t x) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int d = 32; d; d >>= 1) {
    const uint64_t y = swapped(x, d);
    x = ((lane & d) == 0) == (x > y) ? x : y;
  }
  return x;
}
__device__ __forceinline__ uint64_t sort64(uint64_t x) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int n = 2; n <= 64; n <<= 1)
#pragma unroll
    for (int d = n >> 1; d; d >>= 1) {
      const uint64_t y = swapped(x, d);
      x = (((lane & d) == 0) == ((lane & n) == 0 || n == 64)) == (x > y) ? x : y;
    }
  return x;
}
// The 64 largest of two sorted sets of lanes, sorted.
__device__ __forceinline__ uint64_t best64(uint64_t a, uint64_t b) {
  const uint64_t r = from_lane(b, 63 - (threadIdx.x & 63));
  return merge64(a > r ? a : r);
}

// The 64 best keys that a wave has seen, sorted over its lanes, and a list in LDS of those that came since.
struct Best {
  uint64_t mine, border;   // border: the keep-th best, the same for the wave; what does not beat it is of no interest
  uint64_t* list;
  int count, keep;
  __device__ __forceinline__ Best(uint64_t* l, int k) : mine(0), border(0), list(l), count(0), keep(k) {}
  __device__ __forceinline__ void flush() {
    if (!count) return;
    const int lane = threadIdx.x & 63;
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    const uint64_t x = lane < count ? *(volatile uint64_t*)(list + lane) : 0;
    mine = best64(mine, sort64(x));
    raise(from_lane(mine, keep - 1));
    count = 0;
  }
  __device__ __forceinline__ void raise(uint64_t to) { border = to > border ? to : border; }
  __device__ __forceinline__ void offer(uint64_t key) {
    uint64_t in = __ballot(key > border);
    if (!in) return;
    if (count + __popcll(in) > LIST) {
      flush();
      in = __ballot(key > border);
    }
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

// The running sum of a lane: base is a whole number, so that moving it is exact and x log2 e - base is rounded once.
struct Sum {
  float base, sum;
  __device__ __forceinline__ void add(float x) {
    sum += __builtin_amdgcn_exp2f(__builtin_fmaf(x, LOG2E_REST, __builtin_fmaf(x, LOG2E, -base)));
  }
  __device__ __forceinline__ void reach(float top) {   // top: the largest of what comes next
    const float up = fminf(fmaxf(ceilf(top * LOG2E), -LARGEST), LARGEST);
    if (up > base) {
      sum = sum == 0.0f ? 0.0f : sum * __builtin_amdgcn_exp2f(base - up);
      base = up;
    }
  }
};

// How a call is shared out: stretches of `stretch` logits (a multiple of 8), four to a workgroup; `strips` workgroups a row.
struct BeamSplit { int strips, stretch; };

template <typename T>
__device__ __forceinline__ bool beam_counts(const fi_beam_select_args& a, int row) {   // whether the row's logits are looked at
  const float s = a.scores[row];
  return !(a.ended && a.ended[row]) && s > -INFINITY;   // (a NaN does not)
}

// Calls some(values, first, n) for the wave's values in ascending order: of lane l n = 8 (as long as there are 512 and more) or 1 from token `first` on.  Which lane adds which
// values goes by their place in the row alone, not by where the row starts in memory: rows that are alike get sums that are alike to the last bit, and tie.
template <typename T, typename Some>
__device__ __forceinline__ void along(const T* row, int from, int to, Some some) {
  constexpr int N = 16 / sizeof(T), STEP = 64 * 8;
  typedef uint32_t piece __attribute__((ext_vector_type(4), aligned(2)));
  const int lane = threadIdx.x & 63;
  float x[8];
  piece w[8 / N], next[8 / N];
  auto load = [&](int p, piece (&r)[8 / N]) {
#pragma unroll
    for (int i = 0; i < 8 / N; ++i) r[i] = reinterpret_cast<const piece*>(row + p)[lane * (8 / N) + i];
  };
  int at = from;
  if (at + STEP <= to) load(at, next);
  for (; at + STEP <= to; at += STEP) {
#pragma unroll
    for (int i = 0; i < 8 / N; ++i) w[i] = next[i];
    if (at + 2 * STEP <= to) load(at + STEP, next);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if constexpr (N == 4) x[i] = __uint_as_float(w[i >> 2][i & 3]);
      else x[i] = __uint_as_float(i & 1 ? w[0][i >> 1] & 0xFFFF0000u : w[0][i >> 1] << 16);
    }
    some(x, at + lane * 8, 8);
  }
  for (; at < to; at += 64) {
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = -INFINITY;
    if (at + lane < to) x[0] = ld(row + at + lane);
    some(x, at + lane, 1);
  }
}

template <typename T>
__global__ void __launch_bounds__(64 * WAVES) beam_scan_kernel(fi_beam_select_args a, BeamSplit p) {
  __shared__ uint64_t lists[WAVES][LIST];
  const int row = blockIdx.x / p.strips, strip = blockIdx.x - row * p.strips, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  if (!beam_counts<T>(a, row)) return;
  const int64_t first = ((int64_t)strip * WAVES + wave) * p.stretch;
  const int from = (int)(first < a.vocab ? first : a.vocab), to = (int)(first + p.stretch < a.vocab ? first + p.stretch : a.vocab);
  Best best(lists[wave], a.keep);
  Sum sum{-LARGEST, 0.0f};
  bool begun = false;
  along<T>(static_cast<const T*>(a.logits) + row * a.logits_stride, from, to, [&](float (&x)[8], int token, int n) {
    float top = x[0];
#pragma unroll
    for (int i = 1; i < 8; ++i) top = fmaxf(top, x[i]);
    sum.reach(top);
    if (n == 8) {
#pragma unroll
      for (int i = 0; i < 8; ++i) sum.add(x[i]);
    } else if (x[0] > -INFINITY || !(x[0] == x[0])) {
      sum.add(x[0]);
    }
    if (n == 8 && !begun) {   // the keep-th largest of the lanes' best is a border that spares most of the first values
      begun = true;
      const float kth = logit_of(from_lane(sort64(key_of(top, 0)), a.keep - 1));
      if (kth > -INFINITY) best.raise(key_of(kth, 0xFFFFFFFFu) - 1);   // (what equals it passes, whatever its token)
    }
    const float least = best.border ? logit_of(best.border) : -INFINITY;
    if (!__any(top >= least)) return;
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < n) best.offer(x[i] > -INFINITY ? key_of(x[i], token + i) : 0);
  });
  best.flush();
  // the workgroup's list and sum
  lists[wave][lane] = best.mine;
  __shared__ Part parts[WAVES];
  float base = sum.base;
  for (int o = 32; o; o >>= 1) base = fmaxf(base, __shfl_xor(base, o));
  double total = sum.sum == 0.0f ? 0.0 : (double)sum.sum * exp2((double)sum.base - (double)base);
  for (int o = 32; o; o >>= 1) total += __shfl_xor(total, o);
  if (lane == 0) parts[wave] = Part{total, base, 0.0f};
  __syncthreads();
  if (wave) return;
  uint64_t mine = best.mine;
  float top = parts[0].base;
  for (int w = 1; w < WAVES; ++w) {
    mine = best64(mine, lists[w][lane]);
    top = fmaxf(top, parts[w].base);
  }
  total = 0.0;
  for (int w = 0; w < WAVES; ++w) total += parts[w].sum == 0.0 ? 0.0 : parts[w].sum * exp2((double)parts[w].base - (double)top);
  Part* const out = static_cast<Part*>(a.workspace) + (int64_t)row * p.strips + strip;
  uint64_t* const keys = reinterpret_cast<uint64_t*>(static_cast<Part*>(a.workspace) + (int64_t)a.n_seqs * a.beams * p.strips) + ((int64_t)row * p.strips + strip) * a.keep;
  if (lane == 0) *out = Part{total, top, 0.0f};
  if (lane < a.keep) keys[lane] = mine;
}

// log of the sum of exp over a row, by its definition in 64 bits: for rows whose sum left the range of 32.
template <typename T>
__device__ double log_sum(const T* row, int vocab, double* lds) {
  double top = -INFINITY, sum = 0.0;
  bool nan = false;
  for (int t = threadIdx.x; t < vocab; t += 64 * WAVES) {
    const double x = ld(row + t);
    nan |= x != x;
    top = fmax(top, x);
  }
  auto all = [&](double x, bool add) {
    __syncthreads();
    lds[threadIdx.x] = x;
    __syncthreads();
    double r = lds[0];
    for (int i = 1; i < 64 * WAVES; ++i) r = add ? r + lds[i] : fmax(r, lds[i]);
    return r;
  };
  top = all(nan ? INFINITY : top, false);
  if (!(fabs(top) < INFINITY)) return NAN;
  for (int t = threadIdx.x; t < vocab; t += 64 * WAVES) sum += exp((double)ld(row + t) - top);
  return top + log(all(sum, true));
}

// A candidate's place: better scores first, then by beam, then by place in its row's list.
template <typename T>
__global__ void __launch_bounds__(64 * WAVES) beam_join_kernel(fi_beam_select_args a, BeamSplit p) {
  extern __shared__ double scores[];                              // [beams][keep], of every row the best first
  int* const tokens = reinterpret_cast<int*>(scores + a.beams * a.keep);   // [beams][keep]
  __shared__ uint64_t lists[WAVES][LIST];
  __shared__ double sums[FI_MAX_BEAMS], lds[64 * WAVES];
  __shared__ int counts[FI_MAX_BEAMS], odd;
  const int s = blockIdx.x, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const Part* const parts = static_cast<const Part*>(a.workspace);
  const uint64_t* const keys = reinterpret_cast<const uint64_t*>(parts + (int64_t)a.n_seqs * a.beams * p.strips);
  if (threadIdx.x == 0) odd = 0;
  __syncthreads();
  for (int b = wave; b < a.beams; b += WAVES) {   // a wave's rows: their sums
    const int row = s * a.beams + b;
    if (!beam_counts<T>(a, row)) continue;
    const Part* const mine = parts + (int64_t)row * p.strips;
    double top = -INFINITY, total = 0.0;
    for (int i = lane; i < p.strips; i += 64) top = fmax(top, (double)mine[i].base);
    for (int o = 32; o; o >>= 1) top = fmax(top, __shfl_xor(top, o));
    for (int i = lane; i < p.strips; i += 64) total += mine[i].sum == 0.0 ? 0.0 : mine[i].sum * exp2((double)mine[i].base - top);
    for (int o = 32; o; o >>= 1) total += __shfl_xor(total, o);
    if (lane == 0) {
      sums[b] = (top + log2(total)) * 0.69314718055994530942;
      if (!(total > 0.0 && total < INFINITY && fabs(top) < 1e38)) odd = 1;
    }
  }
  __syncthreads();
  if (odd)
    for (int b = 0; b < a.beams; ++b) {
      const int row = s * a.beams + b;
      if (!beam_counts<T>(a, row) || fabs(sums[b]) < 1e37) continue;   // (the same for the workgroup: sums are written below only by all of it)
      const double exact = log_sum<T>(static_cast<const T*>(a.logits) + row * a.logits_stride, a.vocab, lds);
      __syncthreads();
      if (threadIdx.x == 0) sums[b] = exact;
      __syncthreads();
    }
  for (int b = wave; b < a.beams; b += WAVES) {   // their lists
    const int row = s * a.beams + b;
    const float score = a.scores[row];
    int count = 0;
    if (a.ended && a.ended[row]) {
      count = score > -INFINITY;
      if (lane == 0) {
        scores[b * a.keep] = score;
        tokens[b * a.keep] = a.end;
      }
    } else if (score > -INFINITY) {
      Best best(lists[wave], a.keep);
      const uint64_t* const mine = keys + (int64_t)row * p.strips * a.keep;
      const int n = p.strips * a.keep;
      for (int i = 0; i < n; i += 64) best.offer(i + lane < n ? mine[i + lane] : 0);
      best.flush();
      const double value = (double)score + ((double)logit_of(best.mine) - sums[b]);
      const bool there = lane < a.keep && best.mine != 0 && value > -INFINITY;
      count = __popcll(__ballot(there));   // (values fall from lane to lane)
      if (there) {
        scores[b * a.keep + lane] = value;
        tokens[b * a.keep + lane] = (int)token_of(best.mine);
      }
    }
    if (lane == 0) counts[b] = count;
  }
  __syncthreads();
  int total = 0;
  for (int b = 0; b < a.beams; ++b) total += counts[b];
  for (int i = threadIdx.x; i < a.beams * a.keep; i += 64 * WAVES) {
    const int b = i / a.keep, at = i - b * a.keep;
    if (at >= counts[b]) continue;
    const double value = scores[i];
    int place = at;
    for (int o = 0; o < a.beams && place < a.keep; ++o) {
      if (o == b) continue;
      int lo = 0, hi = counts[o];   // how many of row o come first: those that are larger, or as large in a row before
      while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        const double other = scores[o * a.keep + mid];
        if (other > value || (other == value && o < b)) lo = mid + 1;
        else hi = mid;
      }
      place += lo;
    }
    if (place >= a.keep) continue;
    const int row = s * a.beams + b, to = s * a.keep + place, token = tokens[i];
    a.tokens_out[to] = token;
    a.parents_out[to] = row;
    a.scores_out[to] = (float)value;
    if (a.ended_out) a.ended_out[to] = token == a.end || (a.ended && a.ended[row]);
  }
  for (int place = total + threadIdx.x; place < a.keep; place += 64 * WAVES) {
    const int to = s * a.keep + place;
    a.tokens_out[to] = -1;
    a.parents_out[to] = -1;
    a.scores_out[to] = -INFINITY;
    if (a.ended_out) a.ended_out[to] = 0;
  }
}

BeamSplit plan_beams(const fi_beam_select_args& a) {
  const int64_t rows = (int64_t)a.n_seqs * a.beams;
  int64_t stretch = 2048;
  while (stretch < 16384 && rows * ((a.vocab + WAVES * stretch - 1) / (WAVES * stretch)) > 2048) stretch *= 2;
  const int64_t strips = (a.vocab + WAVES * stretch - 1) / (WAVES * stretch);
  return BeamSplit{(int)(strips < 1 ? 1 : strips), (int)stretch};
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
  if (!one_launch(groups, 64 * WAVES) || !one_launch(a.n_seqs, 64 * WAVES)) return kTooLarge;
  const uint32_t lds = (uint32_t)(a.beams * a.keep * 12);
  if (a.dtype == FI_F32) {
    beam_scan_kernel<float><<<dim3((uint32_t)groups), 64 * WAVES, 0, s>>>(a, p);
    beam_join_kernel<float><<<dim3((uint32_t)a.n_seqs), 64 * WAVES, lds, s>>>(a, p);
  } else {
    beam_scan_kernel<bf16_t><<<dim3((uint32_t)groups), 64 * WAVES, 0, s>>>(a, p);
    beam_join_kernel<bf16_t><<<dim3((uint32_t)a.n_seqs), 64 * WAVES, lds, s>>>(a, p);
  }
  return (int)hipGetLastError();
}

}  // namespace fi
