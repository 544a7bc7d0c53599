// Attention over whole prompts (packed sequences) and of drafted trees over a paged cache.
#include <hip/hip_runtime.h>

#include <type_traits>

#include "fi_device.h"
#include "fi_ops.h"
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

constexpr int RUN = FI_MAX_HEAD_DIM / 64;   // values of a row per lane

// One query of one head by one wave, any type, strides and head size: a lane computes the score of one key of 64 and holds every 64th
// value of the output.  `keys` places are offered, seen(j) tells which the query sees and row(j) where they are (key and value rows).
template <typename T, typename Seen, typename KRow, typename VRow>
__device__ __forceinline__ void attend_row(const T* q, T* out, int D, int keys, float scale, float* lds, Seen seen, KRow krow, VRow vrow) {
  const int lane = threadIdx.x & 63;
  for (int d = lane; d < D; d += 64) lds[d] = ld(q + d);
  float acc[RUN] = {}, top = -INFINITY, total = 0.0f;
  for (int j0 = 0; j0 < keys; j0 += 64) {
    const int j = j0 + lane;
    const bool see = j < keys && seen(j);
    float score = -INFINITY;
    if (see) {
      const T* const k = krow(j);
      score = 0.0f;
      for (int d = 0; d < D; ++d) score += lds[d] * ld(k + d);
      score *= scale;
    }
    const float now = fmaxf(top, wave_max(score)), base = now == -INFINITY ? 0.0f : now;
    const float p = see ? expf(score - base) : 0.0f, shrink = expf(top - base);
    total = total * shrink + wave_sum(p);
    top = now;
#pragma unroll
    for (int i = 0; i < RUN; ++i) acc[i] *= shrink;
    for (uint64_t left = __ballot(see); left; left &= left - 1) {   // unseen values are not touched
      const int at = __ffsll((long long)left) - 1;
      const float w = __shfl(p, at);
      const T* const v = vrow(j0 + at);
#pragma unroll
      for (int i = 0; i < RUN; ++i)
        if (lane + 64 * i < D) acc[i] += w * ld(v + lane + 64 * i);
    }
  }
  const float inv = total == 0.0f ? 0.0f : 1.0f / total;
#pragma unroll
  for (int i = 0; i < RUN; ++i)
    if (lane + 64 * i < D) st(out + lane + 64 * i, total == 0.0f ? 0.0f : acc[i] * inv);
}

template <typename T>
__global__ void __launch_bounds__(64) prompt_row_kernel(fi_prompt_attention_args a) {
  __shared__ float lds[FI_MAX_HEAD_DIM];
  const int row = blockIdx.x, h = blockIdx.y, hk = h / (a.q_heads / a.kv_heads);
  const int b = find_seq(a.cu_q, a.n_seqs, row), nq = (int)a.q_tokens, nk = (int)a.k_tokens;
  const int q0 = clamp_int(a.cu_q[b], 0, nq), q1 = clamp_int(a.cu_q[b + 1], q0, nq);
  const int k0 = clamp_int(a.cu_k[b], 0, nk), k1 = clamp_int(a.cu_k[b + 1], k0, nk);
  int keys = k1 - k0;
  if (a.causal) keys = clamp_int(keys - (q1 - q0) + (row - q0) + 1, 0, keys);
  const T* const k = static_cast<const T*>(a.k) + k0 * a.k_strides[0] + hk * a.k_strides[1];
  const T* const v = static_cast<const T*>(a.v) + k0 * a.v_strides[0] + hk * a.v_strides[1];
  attend_row<T>(
      static_cast<const T*>(a.q) + row * a.q_strides[0] + h * a.q_strides[1], static_cast<T*>(a.out) + row * a.out_strides[0] + h * a.out_strides[1], a.head_dim, keys,
      a.scale, lds, [&](int) { return true; }, [&](int j) { return k + j * a.k_strides[0]; }, [&](int j) { return v + j * a.v_strides[0]; });
}

template <typename T>
__global__ void __launch_bounds__(64) tree_row_kernel(fi_tree_attention_args a) {
  __shared__ float lds[FI_MAX_HEAD_DIM];
  const int row = blockIdx.x, h = blockIdx.y, hk = h / (a.q_heads / a.kv_heads);
  const int b = find_seq(a.cu_nodes, a.n_seqs, row), total = (int)a.nodes;
  const int n0 = clamp_int(a.cu_nodes[b], 0, total), all = clamp_int(a.cu_nodes[b + 1], n0, total) - n0, nodes = all < a.max_nodes ? all : a.max_nodes;
  if (row - n0 >= a.max_nodes) return;
  const int places = a.n_pages ? a.page_size * a.table_columns : 0;
  const int cached = clamp_int(a.cached[b], 0, places), keys = nodes < places - cached ? cached + nodes : places;
  const int32_t* const table = a.block_table + b * a.table_stride;
  auto seen = [&](int j) {
    const int node = j - cached;
    if (node < 0) return true;
    if (!a.mask) return node <= row - n0;
    return node < 64 * a.mask_words && (a.mask[(int64_t)row * a.mask_words + node / 64] >> (node % 64) & 1) != 0;
  };
  auto at = [&](const void* cache, const int64_t* s, int j) {
    const int page = clamp_int(table[j / a.page_size], 0, a.n_pages - 1);
    return static_cast<const T*>(cache) + page * s[0] + (j % a.page_size) * s[1] + hk * s[2];
  };
  attend_row<T>(
      static_cast<const T*>(a.q) + row * a.q_strides[0] + h * a.q_strides[1], static_cast<T*>(a.out) + row * a.out_strides[0] + h * a.out_strides[1], a.head_dim, keys,
      a.scale, lds, seen, [&](int j) { return at(a.k_cache, a.k_strides, j); }, [&](int j) { return at(a.v_cache, a.v_strides, j); });
}

// ---------------------------------------------------------------------------------------------------
// Tiles on the matrix cores
// ---------------------------------------------------------------------------------------------------
// A wave has 32 queries as the columns of everything: scores S^T = K Q^T (keys x queries), outputs O^T = V^T P^T (values x queries).  A lane then
// holds scores of ONE query (lanes l and l + 32 share it), so the running maximum and sum of the softmax are sums inside a lane and one
// exchange, and the scores' registers are, rounded, the operand of the second product as they stand: its reduction runs over keys
// in the order that the first product leaves them in (key 8 g + 4 h + i is element 4 g + i of half h).
// Keys and values come into LDS by direct loads, 16-byte pieces permuted at the source so that operand reads meet no bank twice; values are read
// transposed (16 lanes get columns of 4 x 16 elements), fp32 ones column by column.
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef short v4i16 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) v4i16 lds_v4i16;

template <typename T, int DB_, int DQ = DB_ * 32>   // DB: blocks of 32 values of a head; DQ: values that its scores are summed over
struct Tile {
  static constexpr bool F32 = sizeof(T) == 4;
  static constexpr int DB = DB_, ES = sizeof(T), EP = 16 / ES;                          // bytes of an element, elements of a piece
  static constexpr int PB = (DB <= 2 ? 64 : DB <= 4 ? 128 : 256) * ES, NP = PB / 16;    // bytes and pieces of a row in LDS
  static constexpr int KS = DQ / (2 * EP);                                             // steps of two pieces in a score's sum
  static constexpr int RPI = 1024 / PB;                                                 // rows that one load instruction brings
  static constexpr int FV = F32 ? 2 : 4;                                                // values' addresses that differ by more than a constant

  struct Addr { uint32_t k[KS < 8 ? KS : 8], v[FV]; };   // of the lane's operands in a tile of keys / values
  static __device__ __forceinline__ int swizzle_k(int row) { return NP >= 16 ? row & 15 : (row >> 1) & 7; }
  static __device__ __forceinline__ int swizzle_v(int row) { return F32 ? ((row >> 2) & 1) << 3 : NP >= 16 ? (row & 3) << 2 : ((row >> 1) & 1) << 2; }

  static __device__ __forceinline__ void addresses(Addr& a) {
    const int lane = threadIdx.x & 63, r31 = lane & 31, half = lane >> 5;
#pragma unroll
    for (int kk = 0; kk < (KS < 8 ? KS : 8); ++kk) a.k[kk] = r31 * PB + (((2 * kk + half) ^ swizzle_k(r31)) << 4);
#pragma unroll
    for (int f = 0; f < FV; ++f) {
      if constexpr (F32) a.v[f] = 4 * half * PB + (((f * 8) ^ (half << 3)) << 4) + r31 * 4;
      else {
        const int i = lane & 15, row = 4 * half + (i >> 2);
        a.v[f] = row * PB + (((f * 4) ^ swizzle_v(row)) << 4) + ((lane >> 4) & 1) * 32 + (i & 3) * 8;
      }
    }
  }

  // The queries as operands: q[kk] = values (2 kk + half) * EP .. of this lane's query; zeros past D (a multiple of EP).
  static __device__ __forceinline__ void load_q(const T* row, int D, u32x4 (&q)[KS]) {
    const int half = (threadIdx.x & 63) >> 5;
#pragma unroll
    for (int kk = 0; kk < KS; ++kk) {
      const int at = (2 * kk + half) * EP;
      q[kk] = u32x4{0, 0, 0, 0};
      if (at < D) q[kk] = *reinterpret_cast<const u32x4*>(row + at);
    }
  }

  // Waits for the queries here: a wait that the compiler puts before their first use would stand in the loop over the tiles and hold up its loads.
  static __device__ __forceinline__ void have_q(u32x4 (&q)[KS]) {
#pragma unroll
    for (int kk = 0; kk < KS; ++kk) asm volatile("" : "+v"(q[kk]));
  }

  // Rows [0, 32 KB) of a tile, instruction by instruction: `waves` waves share them, this is number `wave`.  rows(r): where key r's row begins, in pieces.
  template <int KB, int WAVES, typename Rows>
  static __device__ __forceinline__ void load_tile(const T* k, const T* v, uint8_t* tile, int wave, int D, Rows rows) {
    const int lane = threadIdx.x & 63;
    constexpr int NI = KB * 32 / RPI;
#pragma unroll
    for (int u = 0; u < (NI + WAVES - 1) / WAVES; ++u) {
      const int i = u * WAVES + wave;
      if (NI % WAVES && i >= NI) break;
      const int row = i * RPI + lane / NP, pos = lane % NP;
      uint32_t ko, vo;
      rows(u, row, ko, vo);
      const int pk = pos ^ swizzle_k(row), pv = pos ^ swizzle_v(row);
      uint8_t* const at = tile + i * 1024;
      if (pk * EP < D) load_lds_from<16>(k + ((uint64_t)ko + pk) * EP, at);
      if (pv * EP < D) load_lds_from<16>(v + ((uint64_t)vo + pv) * EP, at + KB * 32 * PB);
    }
  }

  static __device__ __forceinline__ f32x16 product(const u32x4 a, const u32x4 b, f32x16 c) {
    if constexpr (F32) {
      const float4 x = __builtin_bit_cast(float4, a), y = __builtin_bit_cast(float4, b);
      c = __builtin_amdgcn_mfma_f32_32x32x2f32(x.x, y.x, c, 0, 0, 0);
      c = __builtin_amdgcn_mfma_f32_32x32x2f32(x.y, y.y, c, 0, 0, 0);
      c = __builtin_amdgcn_mfma_f32_32x32x2f32(x.z, y.z, c, 0, 0, 0);
      return __builtin_amdgcn_mfma_f32_32x32x2f32(x.w, y.w, c, 0, 0, 0);
    } else {
      return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
    }
  }

  struct State {
    f32x16 o[DB];
    float top, total;   // the maximum that the weights are taken against; the lane's share of their sum
  };
  static __device__ __forceinline__ void clear(State& s) {
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int e = 0; e < 16; ++e) s.o[db][e] = 0.0f;
    s.top = -INFINITY;
    s.total = 0.0f;
  }

  // An infinity or a NaN among the values times a weight that is zero would be NaN, for queries that do not see the key too.  In tiles where some query
  // does not see every key such values are taken out before the product, by all threads that share the tile (add_strange gives them to the queries that
  // see them).  Tells whether the thread found one.
  template <int KB>
  static __device__ __forceinline__ bool take_out(uint8_t* tile, int thread, int threads) {
    bool found = false;
    for (int i = thread * 16; i < KB * 32 * PB; i += threads * 16) {
      u32x4* const at = reinterpret_cast<u32x4*>(tile + KB * 32 * PB + i);
      u32x4 a = *at;
      uint32_t x = 0;
#pragma unroll
      for (int e = 0; e < 4; ++e) x |= F32 ? (a[e] & 0x7F800000u) + 0x00800000u : (a[e] & 0x7F807F80u) + 0x00800080u;   // an exponent of ones carries into the sign's place
      if (x & (F32 ? 0x80000000u : 0x80008000u)) {
        found = true;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          if (F32) a[e] = (a[e] & 0x7F800000u) == 0x7F800000u ? 0u : a[e];
          else a[e] = ((a[e] & 0x7F80u) == 0x7F80u ? 0u : a[e] & 0xFFFFu) | ((a[e] & 0x7F800000u) == 0x7F800000u ? 0u : a[e] & 0xFFFF0000u);
        }
        *at = a;
      }
    }
    return found;
  }
  // Adds the values of the keys [from, to) that are no finite numbers to the sums of the queries that see them.
  template <typename Row, typename Seen>
  static __device__ __forceinline__ void add_strange(State& st, int D, int from, int to, Row row, Seen seen) {
    const int half = (threadIdx.x & 63) >> 5;
#pragma unroll 1
    for (int key = from; key < to; ++key) {
      const T* const v = row(key);
      const bool see = seen(key);
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          const int d = db * 32 + 8 * g + 4 * half, at = d < D ? d : 0;   // (sums past D are not stored)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float f = ld(v + at + i);
            st.o[db][4 * g + i] += see && (__float_as_uint(f) & 0x7F800000u) == 0x7F800000u ? f : 0.0f;
          }
          __builtin_amdgcn_sched_barrier(0);   // (rare: not worth registers for a row in flight)
        }
    }
  }

  // ---- one tile of 32 KB keys, in five steps; c: scale * log2(e)
  template <int KB>
  static __device__ __forceinline__ void scores(f32x16 (&s)[KB], const u32x4 (&q)[KS], const uint8_t* tile, const Addr& at) {
#pragma unroll
    for (int kb = 0; kb < KB; ++kb) {
#pragma unroll
      for (int e = 0; e < 16; ++e) s[kb][e] = 0.0f;
#pragma unroll
      for (int kk = 0; kk < KS; ++kk)
        s[kb] = product(*reinterpret_cast<const u32x4*>(tile + at.k[kk & 7] + (kk >> 3) * 256 + kb * 32 * PB), q[kk], s[kb]);
    }
  }
  // Bit 8 g + 4 half + i of visible(kb) (half: this lane's) tells whether the lane's query sees key 32 kb + 8 g + 4 half + i.
  template <int KB, typename Visible>
  static __device__ __forceinline__ void hide(f32x16 (&s)[KB], Visible visible) {
    const int half = (threadIdx.x & 63) >> 5;
#pragma unroll
    for (int kb = 0; kb < KB; ++kb) {
      const uint32_t bits = visible(kb) >> (4 * half);
#pragma unroll
      for (int e = 0; e < 16; ++e) s[kb][e] = (bits >> (8 * (e >> 2) + (e & 3))) & 1 ? s[kb][e] : -INFINITY;
    }
  }
  template <int KB>
  static __device__ __forceinline__ float highest(const f32x16 (&s)[KB]) {
    float m = s[0][0];
#pragma unroll
    for (int kb = 0; kb < KB; ++kb)
#pragma unroll
      for (int e = 0; e < 16; ++e) m = fmaxf(m, s[kb][e]);
    const auto both = __builtin_amdgcn_permlane32_swap(__float_as_uint(m), __float_as_uint(m), false, false);
    return fmaxf(__uint_as_float(both[0]), __uint_as_float(both[1]));
  }
  // The weights may be taken against any number that keeps them in range: it moves only when the maximum has grown by a factor of 2^8 in weight.
  static __device__ __forceinline__ void follow(State& st, float m, float c) {
    if (__any((m - st.top) * c > 8.0f || (st.top == -INFINITY && m > -INFINITY))) {
      const float now = fmaxf(st.top, m), shrink = __builtin_amdgcn_exp2f((st.top - (now == -INFINITY ? 0.0f : now)) * c);
      st.total *= shrink;
      st.top = now;
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int e = 0; e < 16; ++e) st.o[db][e] *= shrink;
    }
  }
  template <int KB>
  static __device__ __forceinline__ void weigh(State& st, f32x16 (&s)[KB], float c) {
    const float base = st.top == -INFINITY ? 0.0f : st.top * c;
#pragma unroll
    for (int kb = 0; kb < KB; ++kb)
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        s[kb][e] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[kb][e], c, -base));
        st.total += s[kb][e];
      }
  }
  // The matrix cores take the weights in bf16 where the values are.  FINE: in two terms, what the first leaves out by itself (16 bits, so that what is rounded to bf16 is the result
  // alone); else rounded once (8 bits), their sum as it is.  Rounding halves the products, which counts where they bound the call: us in two terms / rounded, 8192 queries of 32 heads
  // of 128 716 / 533, 12 trees of up to 37 nodes over up to 5001 keys 39.8 / 35.8; 4 single tokens over 131071 keys each, which HBM bounds, 391 / 389, one over 1003 10.6 / 10.5.
  // So blocks of 32 rows over a cache (single tokens, small trees) take two terms, all others one.
  template <int KB, bool FINE>
  static __device__ __forceinline__ void add_values(State& st, const f32x16 (&s)[KB], const uint8_t* tile, const Addr& at) {
    const uint8_t* const values = tile + KB * 32 * PB;
#pragma unroll
    for (int kb = 0; kb < KB; ++kb) {
      if constexpr (F32) {
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          const u32x4 p = {__float_as_uint(s[kb][4 * g]), __float_as_uint(s[kb][4 * g + 1]), __float_as_uint(s[kb][4 * g + 2]), __float_as_uint(s[kb][4 * g + 3])};
#pragma unroll
          for (int db = 0; db < DB; ++db) {
            u32x4 a;
#pragma unroll
            for (int i = 0; i < 4; ++i) a[i] = *reinterpret_cast<const uint32_t*>(values + at.v[db & 1] + (db >> 1) * 256 + (kb * 32 + 8 * g + i) * PB);
            st.o[db] = product(a, p, st.o[db]);
          }
        }
      } else {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          u32x4 p;
#pragma unroll
          for (int i = 0; i < 4; ++i) p[i] = pack_bf16x2(s[kb][8 * h + 2 * i], s[kb][8 * h + 2 * i + 1]);
          u32x4 rest;
          if constexpr (FINE) {
#pragma unroll
            for (int i = 0; i < 4; ++i) rest[i] = pack_bf16x2(s[kb][8 * h + 2 * i] - __uint_as_float(p[i] << 16), s[kb][8 * h + 2 * i + 1] - __uint_as_float(p[i] & 0xFFFF0000u));
          }
#pragma unroll
          for (int db = 0; db < DB; ++db) {
            const uint8_t* const from = values + at.v[db & 3] + (db >> 2) * 256 + (kb * 32 + 16 * h) * PB;
            const u32x2 lo = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4i16*)from));
            const u32x2 hi = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4i16*)(from + 8 * PB)));
            const u32x4 v = {lo[0], lo[1], hi[0], hi[1]};
            st.o[db] = product(v, p, st.o[db]);
            if constexpr (FINE) st.o[db] = product(v, rest, st.o[db]);
          }
        }
      }
    }
  }
  // All five.  masked: the same for the wave.
  template <int KB, bool FINE, typename Visible>
  static __device__ __forceinline__ void attend(State& st, const u32x4 (&q)[KS], const uint8_t* tile, const Addr& at, float c, bool masked, Visible visible) {
    f32x16 s[KB];
    scores<KB>(s, q, tile, at);
    if (masked) hide<KB>(s, visible);
    follow(st, highest<KB>(s), c);
    weigh<KB>(st, s, c);
    add_values<KB, FINE>(st, s, tile, at);
  }

  // The lane's outputs, N blocks of values from block `from` on: o[b][4 g ..] are values 32 (from + b) + 8 g + 4 half .. of its query.
  template <int N>
  static __device__ __forceinline__ void store(const f32x16 (&o)[N], int from, T* row, int D, float inv) {
    const int half = (threadIdx.x & 63) >> 5;
#pragma unroll
    for (int b = 0; b < N; ++b)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const int d = (from + b) * 32 + 8 * g + 4 * half;
        if (d >= D) continue;
        if constexpr (F32) *reinterpret_cast<float4*>(row + d) = make_float4(o[b][4 * g] * inv, o[b][4 * g + 1] * inv, o[b][4 * g + 2] * inv, o[b][4 * g + 3] * inv);
        else *reinterpret_cast<uint2*>(row + d) = make_uint2(pack_bf16x2(o[b][4 * g] * inv, o[b][4 * g + 1] * inv), pack_bf16x2(o[b][4 * g + 2] * inv, o[b][4 * g + 3] * inv));
      }
  }
};

__device__ __forceinline__ float both_halves(float v) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
__device__ __forceinline__ uint32_t low_bits(int n) { return n <= 0 ? 0u : n >= 32 ? ~0u : (1u << n) - 1u; }
template <typename TL, int BYTES>
__device__ __forceinline__ void clear_pads(uint8_t* smem, int D, int threads) {   // pieces past D are never loaded: zeros
  if (D == TL::PB / TL::ES) return;
  for (int i = threadIdx.x * 16; i < BYTES; i += threads * 16) *reinterpret_cast<u32x4*>(smem + i) = u32x4{0, 0, 0, 0};
  __syncthreads();
}

// What a workgroup of the prompt kernels works on: ROWS queries of a head.
struct PromptWork {
  int h, hk, q0, k0, rows, keys, first;   // the sequence's first query and key, how many it has; the workgroup's first query among them
  bool causal;
  // the last key that query r of the sequence sees (-1: none); past the last query: as it
  __device__ __forceinline__ int last(int r) const { return causal ? clamp_int(keys - rows + (r < rows ? r : rows - 1), -1, keys - 1) : keys - 1; }
};
template <int ROWS>
__device__ __forceinline__ bool prompt_work(const fi_prompt_attention_args& a, PromptWork& w) {
  // heads of one key head on one die (workgroups go to the eight dies in turn), late rows first: they see most keys
  const int hq = a.q_heads, tile_id = (int)(gridDim.x / hq) - 1 - (int)(blockIdx.x / hq);
  w.h = blockIdx.x % hq;
  if (hq % NXCD == 0) w.h = w.h % NXCD * (hq / NXCD) + w.h / NXCD;
  w.hk = w.h / (hq / a.kv_heads);
  w.causal = a.causal != 0;
  // sequence b has the tiles from cu_q[b] / ROWS + b on: enough for its rows wherever they start
  int lo = 0, hi = a.n_seqs - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (a.cu_q[mid] / ROWS + mid <= tile_id) lo = mid;
    else hi = mid - 1;
  }
  const int nq = (int)a.q_tokens, nk = (int)a.k_tokens;
  w.q0 = clamp_int(a.cu_q[lo], 0, nq);
  w.rows = clamp_int(a.cu_q[lo + 1], w.q0, nq) - w.q0;
  w.k0 = clamp_int(a.cu_k[lo], 0, nk);
  w.keys = clamp_int(a.cu_k[lo + 1], w.k0, nk) - w.k0;
  w.first = (tile_id - (w.q0 / ROWS + lo)) * ROWS;
  return w.first >= 0 && w.first < w.rows;
}

// Few rows: every wave has the same 32 rows and keys of its own, 32 at a time, loaded by itself (no barriers); joined in LDS at the end.
// SMALL, for many short histories: one wave and one tile in LDS, so that several workgroups are on a compute unit.
template <typename T, int DB, bool SMALL = false>
struct Own {
  using TL = Tile<T, DB>;
  static constexpr int BYTES = 2 * 32 * TL::PB;   // a tile
  // 128 KB of tiles at most: waves before a second tile each, so that all four matrix units are at work (12 fp32 heads of 128, 7 prompts up to 301 tokens: two waves with two
  // tiles 34 us, four with one 25; 4 x 100000 keys of 8 bf16 heads of 256, one node: 172, 176)
  static constexpr int WAVES = SMALL ? 1 : TL::PB <= 512 ? 4 : 2;
  static constexpr int BUFS = SMALL || TL::PB >= 512 ? 1 : 2, LDS = BUFS * BYTES * WAVES + WAVES * 512;
};
// The tiles [first, end) of 32 keys.  query: the lane's; some query may not see all keys from `sure` on; find(t): where lane r's key of a tile is, asked for a
// tile ahead, and offsets(place, ko, vo); visible(t): which of them the lane's query sees; strange(t0, t1): TL::add_strange for a wave's tiles.
// A wave ends with the joined sums of some blocks of values.
template <typename TL, int WAVES>
struct Joined {
  static constexpr int N = (TL::DB + WAVES - 1) / WAVES;   // (blocks past the last are not stored)
  f32x16 o[N];
  int from;
  float top, total;
};
template <typename TL, typename T, int WAVES, int BUFS, bool FINE, typename Find, typename Offsets, typename Visible, typename Strange>
__device__ __forceinline__ void own_walk(Joined<TL, WAVES>& r, uint8_t* smem, const T* k, const T* v, const T* query, int D, float c, int first, int end, int sure, Find find,
                                         Offsets offsets, Visible visible, Strange add_strange) {
  constexpr int BYTES = 2 * 32 * TL::PB, DB = TL::DB;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  auto share = [&](int x) { return first + (int)((int64_t)(end - first) * x / WAVES); };
  const int t0 = share(wave), t1 = share(wave + 1);
  typename TL::State st;
  static_assert(WAVES == 1 || DB * 4096 <= BUFS * BYTES, "a wave's sums fit its tiles");
  uint8_t* const tiles = smem + wave * BUFS * BYTES;
  clear_pads<TL, BUFS * BYTES * WAVES>(smem, D, 64 * WAVES);
  u32x4 q[TL::KS];
  TL::load_q(query, D, q);
  typename TL::Addr at;
  TL::addresses(at);
  TL::clear(st);
  decltype(find(0)) place{};
  auto load = [&](int t) {
    uint32_t mk, mv;
    offsets(place, mk, mv);
    TL::template load_tile<1, 1>(k, v, tiles + (t & (BUFS - 1)) * BYTES, 0, D, [&](int, int r, uint32_t& ko, uint32_t& vo) {
      ko = __shfl(mk, r);
      vo = __shfl(mv, r);
    });
    if (t + 1 < t1) place = find(t + 1);
  };
  bool strange = false;
  if (t0 < t1) place = find(t0);
  TL::have_q(q);
  if (t0 < t1) load(t0);
  for (int t = t0; t < t1; ++t) {
    arrived();
    if (BUFS > 1 && t + 1 < t1) load(t + 1);
    uint8_t* const tile = tiles + (t & (BUFS - 1)) * BYTES;
    if ((t + 1) * 32 > sure) strange |= __any(TL::template take_out<1>(tile, lane, 64)) != 0;
    TL::template attend<1, FINE>(st, q, tile, at, c, (t + 1) * 32 > sure, [&](int) { return visible(t); });
    if (BUFS == 1 && t + 1 < t1) {
      arrived();   // (the tile has been read)
      load(t + 1);
    }
  }
  if (strange) add_strange(st, t0, t1);
  const float total = both_halves(st.total);
  if constexpr (WAVES == 1) {
#pragma unroll
    for (int db = 0; db < DB; ++db) r.o[db] = st.o[db];
    r.from = 0;
    r.top = st.top;
    r.total = total;
  } else {
    // the waves' sums against the largest maximum, added in the order of the waves, some blocks by each
    f32x4* const own = reinterpret_cast<f32x4*>(tiles) + lane;
    float2* const stats = reinterpret_cast<float2*>(smem + BUFS * BYTES * WAVES) + lane;
    arrived();
    if (t0 < t1) {
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int g = 0; g < 4; ++g) own[(db * 4 + g) * 64] = f32x4{st.o[db][4 * g], st.o[db][4 * g + 1], st.o[db][4 * g + 2], st.o[db][4 * g + 3]};
    }
    stats[wave * 64] = make_float2(st.top, total);
    __syncthreads();
    float factor[WAVES];
    r.top = stats[0].x;
#pragma unroll
    for (int x = 1; x < WAVES; ++x) r.top = fmaxf(r.top, stats[x * 64].x);
    const float base = r.top == -INFINITY ? 0.0f : r.top;
    r.total = 0.0f;
#pragma unroll
    for (int x = 0; x < WAVES; ++x) {
      factor[x] = __builtin_amdgcn_exp2f((stats[x * 64].x - base) * c);
      r.total += stats[x * 64].y * factor[x];
    }
    r.from = wave * r.N;
#pragma unroll
    for (int b = 0; b < r.N; ++b) {
#pragma unroll
      for (int e = 0; e < 16; ++e) r.o[b][e] = 0.0f;
      if (r.from + b >= DB) continue;
#pragma unroll
      for (int x = 0; x < WAVES; ++x) {
        if (share(x) >= share(x + 1)) continue;
        const f32x4* const other = reinterpret_cast<const f32x4*>(smem + x * BUFS * BYTES) + lane;
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          const f32x4 v4 = other[((r.from + b) * 4 + g) * 64];
#pragma unroll
          for (int i = 0; i < 4; ++i) r.o[b][4 * g + i] += v4[i] * factor[x];
        }
      }
    }
  }
}

// Short prompts: 32 queries a workgroup, whose waves have keys of their own: four times the workgroups, each with a quarter of the walk.
template <typename T, int DB, int DQ>
__global__ void __launch_bounds__((64 * Own<T, DB>::WAVES), 1) prompt_own_kernel(fi_prompt_attention_args a) {
  using TL = Tile<T, DB, DQ>;
  __shared__ __attribute__((aligned(1024))) uint8_t smem[Own<T, DB>::LDS];
  PromptWork w;
  if (!prompt_work<32>(a, w)) return;
  const int lane = threadIdx.x & 63, row = w.first + (lane & 31), mine = row < w.rows ? row : w.rows - 1, last = w.last(mine), least = w.last(w.first), most = w.last(w.first + 31);
  const int D = a.head_dim, keys = w.keys;
  const T* const k = static_cast<const T*>(a.k) + w.k0 * a.k_strides[0] + w.hk * a.k_strides[1];
  const T* const v = static_cast<const T*>(a.v) + w.k0 * a.v_strides[0] + w.hk * a.v_strides[1];
  const uint32_t ks = (uint32_t)(a.k_strides[0] / TL::EP), vs = (uint32_t)(a.v_strides[0] / TL::EP);
  Joined<TL, Own<T, DB>::WAVES> r;
  own_walk<TL, T, Own<T, DB>::WAVES, Own<T, DB>::BUFS, false>(
      r, smem, k, v, static_cast<const T*>(a.q) + (int64_t)(w.q0 + mine) * a.q_strides[0] + w.h * a.q_strides[1], D, a.scale * 1.44269504f, 0, (most + 32) / 32, least + 1,
      [&](int t) { return (uint32_t)(t * 32 + (lane & 31) < keys ? t * 32 + (lane & 31) : keys - 1); },
      [&](uint32_t key, uint32_t& ko, uint32_t& vo) {
        ko = key * ks;
        vo = key * vs;
      },
      [&](int t) { return low_bits(last + 1 - t * 32); },
      [&](typename TL::State& st, int t0, int t1) {
        const int masked = (least + 1) / 32 * 32;
        TL::add_strange(st, D, t0 * 32 > masked ? t0 * 32 : masked, t1 * 32 <= most ? t1 * 32 : most + 1, [&](int key) { return v + (uint64_t)((uint32_t)key * vs) * TL::EP; },
                        [&](int key) { return key <= last; });
      });
  if (row < w.rows) TL::store(r.o, r.from, static_cast<T*>(a.out) + (int64_t)(w.q0 + row) * a.out_strides[0] + w.h * a.out_strides[1], D, r.total == 0.0f ? 0.0f : 1.0f / r.total);
}

constexpr int PROMPT_WAVES = 4, PROMPT_ROWS = 32 * PROMPT_WAVES;

// A workgroup has 128 queries of a head and walks the keys they see, 64 (32) at a time, two tiles in LDS; two workgroups on a compute unit.  GROUPS 2, for calls that
// do not fill the chip: two groups of four waves have the same queries, one the even tiles, one the odd, joined in LDS at the end (bf16, causal, us with one / two:
// 512 tokens of 8 heads of 64 12.2 / 10.9, 2048 33 / 25; heads of 128: 512 16.4 / 16.4, 2048 47 / 43; fp32 is bound by its products, 91 / 94; of heads of 256 the registers of two
// groups do not fit, 124 / 298).  Heads of 256 in bf16 take all 256 registers so that two workgroups fit (12 heads, 6000 tokens: 462 us with one, 355).
template <typename T, int DB, int GROUPS, int DQ>
__global__ void __launch_bounds__(64 * PROMPT_WAVES * GROUPS, DB > 4 && sizeof(T) == 4 ? 1 : 2) prompt_tile_kernel(fi_prompt_attention_args a) {
  constexpr int WAVES = PROMPT_WAVES;
  using TL = Tile<T, DB, DQ>;
  constexpr int KB = TL::PB <= 256 ? 2 : 1, KEYS = 32 * KB, BYTES = 2 * KEYS * TL::PB;
  __shared__ __attribute__((aligned(1024))) uint8_t smem[GROUPS * 2 * BYTES + 16];
  int* const strange = reinterpret_cast<int*>(smem + GROUPS * 2 * BYTES);   // a masked tile held values that are no finite numbers
  if (threadIdx.x == 0) *strange = 0;
  PromptWork w;
  if (!prompt_work<PROMPT_ROWS>(a, w)) return;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) & (WAVES - 1), group = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) / WAVES;
  const int row = w.first + 32 * wave + (lane & 31), mine = row < w.rows ? row : w.rows - 1;
  const int last = w.last(mine), wave_least = w.last(w.first + 32 * wave), least = w.last(w.first), most = w.last(w.first + PROMPT_ROWS - 1);
  const int wave_most = w.first + 32 * wave < w.rows ? w.last(w.first + 32 * wave + 31) : -1;   // (a wave without queries does nothing)
  const int D = a.head_dim, keys = w.keys;
  const T* const k = static_cast<const T*>(a.k) + w.k0 * a.k_strides[0] + w.hk * a.k_strides[1];
  const T* const v = static_cast<const T*>(a.v) + w.k0 * a.v_strides[0] + w.hk * a.v_strides[1];
  const uint32_t ks = (uint32_t)(a.k_strides[0] / TL::EP), vs = (uint32_t)(a.v_strides[0] / TL::EP);
  clear_pads<TL, GROUPS * 2 * BYTES>(smem, D, 64 * WAVES * GROUPS);
  uint8_t* const tiles_at = smem + group * 2 * BYTES;
  u32x4 q[TL::KS];
  TL::load_q(static_cast<const T*>(a.q) + (int64_t)(w.q0 + mine) * a.q_strides[0] + w.h * a.q_strides[1], D, q);
  typename TL::Addr at;
  TL::addresses(at);
  typename TL::State st;
  TL::clear(st);
  const float c = a.scale * 1.44269504f;
  const int tiles = (most + KEYS) / KEYS, turns = (tiles + GROUPS - 1) / GROUPS;   // 0 where nobody sees a key
  auto load = [&](int turn) {
    const int t = turn * GROUPS + group;
    if (t >= tiles) return;
    TL::template load_tile<KB, WAVES>(k, v, tiles_at + (turn & 1) * BYTES, wave, D, [&](int, int r, uint32_t& ko, uint32_t& vo) {
      const uint32_t key = (uint32_t)(t * KEYS + r < keys ? t * KEYS + r : keys - 1);   // (rows past the end: the last key once more, unseen)
      ko = key * ks;
      vo = key * vs;
    });
  };
  TL::have_q(q);
  load(0);
  for (int turn = 0; turn < turns; ++turn) {
    meet();
    if (turn + 1 < turns) load(turn + 1);
    const int t = turn * GROUPS + group;
    uint8_t* const tile = tiles_at + (turn & 1) * BYTES;
    if ((turn + 1) * GROUPS * KEYS - 1 > least) {   // (of the groups' tiles at least one is masked)
      if (t < tiles && t * KEYS + KEYS - 1 > least && TL::template take_out<KB>(tile, threadIdx.x & (64 * WAVES - 1), 64 * WAVES)) *strange = 1;
      meet_lds();
    }
    if (t * KEYS <= wave_most)
      TL::template attend<KB, false>(st, q, tile, at, c, t * KEYS + KEYS - 1 > wave_least, [&](int kb) { return low_bits(last + 1 - t * KEYS - 32 * kb); });
  }
  float total = both_halves(st.total);
  if constexpr (GROUPS == 2) {
    static_assert(WAVES * DB * 4096 + WAVES * 512 <= 4 * BYTES, "the second group's sums fit the tiles");
    float* const sums = reinterpret_cast<float*>(smem + wave * DB * 4096) + lane;
    float2* const stats = reinterpret_cast<float2*>(smem + WAVES * DB * 4096 + wave * 512) + lane;
    meet();
    if (group == 1) {
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int e = 0; e < 16; ++e) sums[(db * 16 + e) * 64] = st.o[db][e];
      *stats = make_float2(st.top, total);
    }
    __syncthreads();
    if (group == 1) return;
    const float top = fmaxf(st.top, stats->x), base = top == -INFINITY ? 0.0f : top;
    const float f0 = __builtin_amdgcn_exp2f((st.top - base) * c), f1 = __builtin_amdgcn_exp2f((stats->x - base) * c);
    total = total * f0 + stats->y * f1;
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int e = 0; e < 16; ++e) st.o[db][e] = st.o[db][e] * f0 + sums[(db * 16 + e) * 64] * f1;
  }
  if (tiles > 0 && *strange)   // (written before the last barrier)
    TL::add_strange(st, D, (least + 1) / KEYS * KEYS, wave_most + 1, [&](int key) { return v + (uint64_t)((uint32_t)key * vs) * TL::EP; }, [&](int key) { return key <= last; });
  if (row < w.rows) TL::store(st.o, 0, static_cast<T*>(a.out) + (int64_t)(w.q0 + row) * a.out_strides[0] + w.h * a.out_strides[1], D, total == 0.0f ? 0.0f : 1.0f / total);
}

// Long prompts in bf16: 256 queries a workgroup, eight waves, four tiles in LDS of which three are on their way; the lanes' offsets of a whole tile stay in registers.
// 8192 queries of 32 heads of 128, causal: 529 to 548 us (1.0 PFLOP/s of the seen half, three quarters of what a large library product reaches; with four waves and two
// tiles 565).  What bounds it: the matrix unit is busy 47 % of the time and the vector unit, with the exponentials, 45 %, and they hardly overlap.
// Tried: the next block's scores among this one's exponentials in a wave 608; the two waves of a unit half a tile apart by barriers 594; wave priorities 543 to 552.
constexpr int LONG_ROWS = 256, LONG_GROUPS = 512;
template <int DB, int DQ>
__global__ void __launch_bounds__(512, 1) prompt_long_kernel(fi_prompt_attention_args a) {
  typedef bf16_t T;
  using TL = Tile<T, DB, DQ>;
  constexpr int KB = 2, KEYS = 64, BYTES = 2 * KEYS * TL::PB, NI = KEYS / TL::RPI, U = NI / 8, L = 2 * U;
  static_assert(NI % 8 == 0, "every wave issues U loads of keys and U of values");
  __shared__ __attribute__((aligned(1024))) uint8_t smem[4 * BYTES + 16];
  int* const strange = reinterpret_cast<int*>(smem + 4 * BYTES);
  if (threadIdx.x == 0) *strange = 0;
  PromptWork w;
  if (!prompt_work<LONG_ROWS>(a, w)) return;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int row = w.first + 32 * wave + (lane & 31), mine = row < w.rows ? row : w.rows - 1;
  const int last = w.last(mine), wave_least = w.last(w.first + 32 * wave), least = w.last(w.first), most = w.last(w.first + LONG_ROWS - 1);
  const int wave_most = w.first + 32 * wave < w.rows ? w.last(w.first + 32 * wave + 31) : -1;   // (a wave without queries does nothing)
  const int D = a.head_dim, keys = w.keys;
  const T* const k = static_cast<const T*>(a.k) + w.k0 * a.k_strides[0] + w.hk * a.k_strides[1];
  const T* const v = static_cast<const T*>(a.v) + w.k0 * a.v_strides[0] + w.hk * a.v_strides[1];
  const uint32_t ks = (uint32_t)(a.k_strides[0] / TL::EP), vs = (uint32_t)(a.v_strides[0] / TL::EP);
  clear_pads<TL, 4 * BYTES>(smem, D, 512);
  u32x4 q[TL::KS];
  TL::load_q(static_cast<const T*>(a.q) + (int64_t)(w.q0 + mine) * a.q_strides[0] + w.h * a.q_strides[1], D, q);
  typename TL::Addr at;
  TL::addresses(at);
  typename TL::State st;
  TL::clear(st);
  const float c = a.scale * 1.44269504f;
  const int tiles = (most + KEYS) / KEYS;
  uint32_t ko[U], vo[U];   // bytes from the tile's first row
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int r = (u * 8 + wave) * TL::RPI + lane / TL::NP, pos = lane % TL::NP;
    ko[u] = (r * ks + (pos ^ TL::swizzle_k(r))) * 16;
    vo[u] = (r * vs + (pos ^ TL::swizzle_v(r))) * 16;
  }
  auto load = [&](int t) {
    const T* const kt = k + (int64_t)t * KEYS * a.k_strides[0];
    const T* const vt = v + (int64_t)t * KEYS * a.v_strides[0];
    uint8_t* const tile = smem + (t & 3) * BYTES;
    const int left = keys - t * KEYS;   // rows past the end: the last key once more, unseen
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int r = (u * 8 + wave) * TL::RPI + lane / TL::NP, pos = lane % TL::NP, pk = pos ^ TL::swizzle_k(r), pv = pos ^ TL::swizzle_v(r);
      const uint32_t over = left < KEYS && r >= left ? (uint32_t)(r - left + 1) : 0u;
      uint8_t* const to = tile + (u * 8 + wave) * 1024;
      if (pk * TL::EP < D) load_lds_off<16>(kt, ko[u] - over * ks * 16, to);
      if (pv * TL::EP < D) load_lds_off<16>(vt, vo[u] - over * vs * 16, to + KEYS * TL::PB);
    }
  };
  TL::have_q(q);
#pragma unroll
  for (int u = 0; u < 3; ++u)
    if (u < tiles) load(u);
  for (int t = 0; t < tiles; ++t) {
    if (t + 2 < tiles) meet_but<2 * L>();
    else meet();
    if (t + 3 < tiles) load(t + 3);
    uint8_t* const tile = smem + (t & 3) * BYTES;
    if (t * KEYS + KEYS - 1 > least) {
      if (TL::template take_out<KB>(tile, threadIdx.x, 512)) *strange = 1;
      meet_lds();
    }
    if (t * KEYS <= wave_most)
      TL::template attend<KB, false>(st, q, tile, at, c, t * KEYS + KEYS - 1 > wave_least, [&](int kb) { return low_bits(last + 1 - t * KEYS - 32 * kb); });
  }
  if (tiles > 0 && *strange)   // (written before the last barrier)
    TL::add_strange(st, D, (least + 1) / KEYS * KEYS, wave_most + 1, [&](int key) { return v + (uint64_t)((uint32_t)key * vs) * TL::EP; }, [&](int key) { return key <= last; });
  const float total = both_halves(st.total);
  if (row < w.rows) TL::store(st.o, 0, static_cast<T*>(a.out) + (int64_t)(w.q0 + row) * a.out_strides[0] + w.h * a.out_strides[1], D, total == 0.0f ? 0.0f : 1.0f / total);
}

// What a workgroup of the tree kernels works on: a block of rows (node, head) of one key head of one sequence, and of its keys the tiles [t0, t1).
struct TreeWork {
  int b, hk, cached, keys, n0, nodes, block, split, splits, t0, t1;
};
// How a call is shared out (on the host): parts that a row can have, least tiles of a part, keys of a tile, what a stream costs beside its tiles, in tiles,
// rows of a block, blocks of a sequence at most, floats before the parts in the workspace.
struct TreeSplit { int splits, least, unit, over, rows, blocks, header; };

// A sequence as the kernels see it: its offsets and lengths clamped to the tensors.
__device__ __forceinline__ void tree_sequence(const fi_tree_attention_args& a, int b, TreeWork& w) {
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
// Counted: the least keys of a stretch, and what a stream's beginning counts for, in tiles (64 keys, of own waves 32; fp32 tiles take longer).  12 sequences, lengths spread
// over their logarithm, us: one node, least 128 keys 30.4, 256 26.5 up to 5001 keys; beginnings of 4, 8, 10, 20 tiles 63, 49, 49, 50 up to 20000; 37 nodes, of 1, 3, 5 tiles
// 114, 85, 84; 10 sequences of 32 heads of 72, fp32, up to 1302 keys, of 4, 8, 20 tiles 47, 57, 85.
struct Stretch { int least, over; };
constexpr Stretch stretch(bool own, bool f32) { return own ? (f32 ? Stretch{128, 4} : Stretch{256, 12}) : (f32 ? Stretch{128, 1} : Stretch{128, 4}); }
struct TreeLine {
  int start[SEQS];   // where a sequence begins
  int n0[SEQS], nodes[SEQS], cached[SEQS], keys[SEQS];
  int quota, total;
};
__device__ __forceinline__ int tiles_of(int keys, int unit) { return keys > unit ? (keys + unit - 1) / unit : 1; }
__device__ __forceinline__ int streams_of(const fi_tree_attention_args& a, const TreeSplit& p, int nodes) {
  return (nodes * (a.q_heads / a.kv_heads) + p.rows - 1) / p.rows * a.kv_heads;
}
__device__ __forceinline__ void line_up(const fi_tree_attention_args& a, const TreeSplit& p, TreeLine& line) {
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
template <typename Work>
__device__ __forceinline__ void along_the_line(const fi_tree_attention_args& a, const TreeSplit& p, const TreeLine& line, Work work) {
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
__device__ __forceinline__ bool tree_direct(const fi_tree_attention_args& a, const TreeSplit& p, TreeWork& w) {
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
__device__ __forceinline__ uint32_t tree_visible(const fi_tree_attention_args& a, const TreeWork& w, int node, const uint64_t* words, int key) {
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

// Where keys of a sequence are: page and place by a reciprocal of the page size (floor(2^32 / size): the quotient is right or one too small), offsets in
// pieces of 16 bytes from the key head's part of the caches (below 2^32: checked on the host).
struct Pages {
  const int32_t* table;
  uint32_t size, inv, most, kp, kt, vp, vt;
  __device__ __forceinline__ Pages(const fi_tree_attention_args& a, int b, int ep)
      : table(a.block_table + b * a.table_stride), size(a.page_size), inv(a.page_size == 1 ? ~0u : (uint32_t)((1ull << 32) / (uint32_t)a.page_size)), most(a.n_pages - 1),
        kp((uint32_t)(a.k_strides[0] / ep)), kt((uint32_t)(a.k_strides[1] / ep)), vp((uint32_t)(a.v_strides[0] / ep)), vt((uint32_t)(a.v_strides[1] / ep)) {}
  __device__ __forceinline__ uint32_t column(int key, uint32_t& row) const {
    uint32_t c = __umulhi((uint32_t)key, inv);
    row = (uint32_t)key - c * size;
    if (row >= size) { ++c; row -= size; }
    return c;
  }
  struct Place { int32_t page; uint32_t row; };
  __device__ __forceinline__ Place find(int key) const {   // issues the table's load
    uint32_t row;
    const uint32_t c = column(key, row);
    return Place{table[c], row};
  }
  __device__ __forceinline__ void offsets(const Place& p, uint32_t& ko, uint32_t& vo) const {
    const uint32_t page = p.page < 0 ? 0u : (uint32_t)p.page > most ? most : (uint32_t)p.page;
    ko = page * kp + p.row * kt;
    vo = page * vp + p.row * vt;
  }
};

// The workspace: the line of a counted call (16 bytes with its quota, then where each sequence begins), then parts of a row (node, head): `splits` times
// head_dim sums, then for all rows the maximum and the weights' sum of each.
__device__ __forceinline__ float* part_sums(const fi_tree_attention_args& a, const TreeSplit& p, int64_t row, int split) {
  return static_cast<float*>(a.workspace) + p.header + (row * p.splits + split) * a.head_dim;
}
__device__ __forceinline__ float* part_stats(const fi_tree_attention_args& a, const TreeSplit& p, int64_t row, int split) {
  return static_cast<float*>(a.workspace) + p.header + a.nodes * a.q_heads * p.splits * a.head_dim + (row * p.splits + split) * 2;
}

// TL::add_strange for the keys [from, to) of a tree: of those only the tiles that were masked.
template <typename TL, typename T>
__device__ __forceinline__ void tree_strange(const fi_tree_attention_args& a, const TreeWork& w, typename TL::State& st, const T* v, const Pages& pages, const uint64_t* words,
                                             int node, int from, int to, int tile) {
  const int masked = w.cached / tile * tile;
  TL::add_strange(st, a.head_dim, from > masked ? from : masked, to < w.keys ? to : w.keys,
                  [&](int key) {
                    uint32_t ko, vo;
                    pages.offsets(pages.find(key), ko, vo);
                    return v + (uint64_t)vo * TL::EP;
                  },
                  [&](int key) { return (tree_visible(a, w, node, words, key) & 1) != 0; });
}

// Writes N blocks of values from block `from` on: results, or sums of a part.
template <typename TL, typename T, int N>
__device__ __forceinline__ void finish(const fi_tree_attention_args& a, const TreeWork& w, const TreeSplit& p, const f32x16 (&o)[N], int from, float top, float total, bool there, int node, int head) {
  if (!there) return;
  if (w.splits == 1) {
    TL::store(o, from, static_cast<T*>(a.out) + (int64_t)(w.n0 + node) * a.out_strides[0] + head * a.out_strides[1], a.head_dim, total == 0.0f ? 0.0f : 1.0f / total);
    return;
  }
  const int64_t row = (int64_t)(w.n0 + node) * a.q_heads + head;
  float* const sums = part_sums(a, p, row, w.split);
  const int half = (threadIdx.x & 63) >> 5;
#pragma unroll
  for (int b = 0; b < N; ++b)
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const int d = (from + b) * 32 + 8 * g + 4 * half;
      if (d < a.head_dim) *reinterpret_cast<float4*>(sums + d) = make_float4(o[b][4 * g], o[b][4 * g + 1], o[b][4 * g + 2], o[b][4 * g + 3]);
    }
  if (half == 0 && from == 0) *reinterpret_cast<float2*>(part_stats(a, p, row, w.split)) = make_float2(top, total);
}

// Many rows: the waves have 32 rows each and share the tiles, as for a prompt, but few workgroups are there to hide each other's waiting: three tiles
// are on their way while one is multiplied, and the pages are asked for (into a ring in LDS, by the same kind of load) three tiles earlier still.
// A wave's loads come back in order, so its waits count them: L loads a tile and one page request, which comes first.
template <typename T, int DB, int WAVES>
struct Shared {
  using TL = Tile<T, DB>;
  static constexpr int KB = TL::PB <= 256 ? 2 : 1, KEYS = 32 * KB, BYTES = 2 * KEYS * TL::PB;
  static constexpr int AHEAD = BYTES <= 32768 ? 3 : 1, BUFS = AHEAD + 1, L = 2 * (KEYS / TL::RPI) / WAVES, RING = 8, LDS = BUFS * BYTES + WAVES * RING * 256 + 16;
  static_assert(KEYS / TL::RPI % WAVES == 0 && 2 * AHEAD + 2 <= RING, "every wave issues L loads a tile; a ring slot is free again");
};
template <typename T, int DB, int WAVES>
__device__ __forceinline__ void tree_tile_work(const fi_tree_attention_args& a, const TreeWork& w, const TreeSplit& p, uint8_t* smem) {
  using TL = Tile<T, DB>;
  using SH = Shared<T, DB, WAVES>;
  constexpr int KB = SH::KB, KEYS = SH::KEYS, BYTES = SH::BYTES, AHEAD = SH::AHEAD, BUFS = SH::BUFS, L = SH::L, RING = SH::RING;
  int* const strange = reinterpret_cast<int*>(smem + BUFS * BYTES + WAVES * RING * 256);
  if (threadIdx.x == 0) *strange = 0;
  const int D = a.head_dim, group = a.q_heads / a.kv_heads;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int rows = w.nodes * group, first = w.block * 32 * WAVES;
  if (first >= rows) return;
  const int row = first + 32 * wave + (lane & 31), mine = row < rows ? row : rows - 1, node = mine / group, head = w.hk * group + mine % group;
  const int t0 = w.t0, t1 = w.t1;
  const T* const k = static_cast<const T*>(a.k_cache) + w.hk * a.k_strides[2];
  const T* const v = static_cast<const T*>(a.v_cache) + w.hk * a.v_strides[2];
  const Pages pages(a, w.b, TL::EP);
  const uint64_t* const words = a.mask ? a.mask + (int64_t)(w.n0 + node) * a.mask_words : nullptr;
  uint8_t* const ring = smem + BUFS * BYTES + wave * RING * 256;
  // lane r is asked where row r of a tile is
  auto key_of = [&](int t) { return t * KEYS + (lane & (KEYS - 1)) < w.keys ? t * KEYS + (lane & (KEYS - 1)) : w.keys - 1; };
  auto ask = [&](int t) {
    uint32_t at_row;
    const int32_t* const entry = pages.table + pages.column(key_of(t < t1 ? t : t1 - 1), at_row);
    load_lds_from<4>(entry, ring + (t & (RING - 1)) * 256);
  };
  auto load = [&](int t) {
    uint32_t mk, mv;
    typename Pages::Place place;
    pages.column(key_of(t), place.row);
    place.page = *reinterpret_cast<const int32_t*>(ring + (t & (RING - 1)) * 256 + lane * 4);
    pages.offsets(place, mk, mv);
    TL::template load_tile<KB, WAVES>(k, v, smem + (t & (BUFS - 1)) * BYTES, wave, D, [&](int, int r, uint32_t& ko, uint32_t& vo) {
      ko = __shfl(mk, r);
      vo = __shfl(mv, r);
    });
  };
  if (t0 < t1) {
#pragma unroll
    for (int u = 0; u <= 2 * AHEAD; ++u) ask(t0 + u);
  }
  clear_pads<TL, BUFS * BYTES>(smem, D, 64 * WAVES);
  u32x4 q[TL::KS];
  TL::load_q(static_cast<const T*>(a.q) + (int64_t)(w.n0 + node) * a.q_strides[0] + head * a.q_strides[1], D, q);
  typename TL::Addr at;
  TL::addresses(at);
  typename TL::State st;
  TL::clear(st);
  const float c = a.scale * 1.44269504f;
  arrived();
  TL::have_q(q);
#pragma unroll
  for (int u = 0; u < AHEAD; ++u)
    if (t0 + u < t1) load(t0 + u);
  for (int t = t0; t < t1; ++t) {
    ask(t + 2 * AHEAD + 1);
    // behind tile t: the loads of up to AHEAD - 1 tiles and at least this page request
    if (AHEAD > 1 && t + 2 < t1) meet_but<(AHEAD - 1) * L + 1>();
    else if (AHEAD > 1 && t + 1 < t1) meet_but<L + 1>();
    else meet_but<1>();
    if (t + AHEAD < t1) load(t + AHEAD);
    uint8_t* const tile = smem + (t & (BUFS - 1)) * BYTES;
    if ((t + 1) * KEYS > w.cached) {
      if (TL::template take_out<KB>(tile, threadIdx.x, 64 * WAVES)) *strange = 1;
      meet_lds();
    }
    if (first + 32 * wave >= rows) continue;
    TL::template attend<KB, false>(st, q, tile, at, c, (t + 1) * KEYS > w.cached, [&](int kb) { return tree_visible(a, w, node, words, t * KEYS + 32 * kb); });
  }
  arrived();   // (page requests past the end)
  if (t0 < t1 && *strange) tree_strange<TL, T>(a, w, st, v, pages, words, node, t0 * KEYS, t1 * KEYS, KEYS);
  finish<TL, T>(a, w, p, st.o, 0, st.top, both_halves(st.total), row < rows, node, head);
}
template <typename T, int DB, int WAVES, bool COUNTED>
__global__ void __launch_bounds__(64 * WAVES, 1) tree_tile_kernel(fi_tree_attention_args a, TreeSplit p) {
  __shared__ __attribute__((aligned(1024))) uint8_t smem[Shared<T, DB, WAVES>::LDS];
  if constexpr (COUNTED) {
    __shared__ TreeLine line;
    line_up(a, p, line);
    along_the_line(a, p, line, [&](const TreeWork& w) {
      meet();   // (the piece before has been read to the end)
      tree_tile_work<T, DB, WAVES>(a, w, p, smem);
    });
  } else {
    TreeWork w;
    if (tree_direct(a, p, w)) tree_tile_work<T, DB, WAVES>(a, w, p, smem);
  }
}

template <typename T, int DB, bool SMALL>
__device__ __forceinline__ void tree_own_work(const fi_tree_attention_args& a, const TreeWork& w, const TreeSplit& p, uint8_t* smem) {
  using TL = Tile<T, DB>;
  const int D = a.head_dim, group = a.q_heads / a.kv_heads;
  const int lane = threadIdx.x & 63;
  const int rows = w.nodes * group, first = w.block * 32;
  if (first >= rows) return;
  const int row = first + (lane & 31), mine = row < rows ? row : rows - 1, node = mine / group, head = w.hk * group + mine % group;
  const T* const k = static_cast<const T*>(a.k_cache) + w.hk * a.k_strides[2];
  const T* const v = static_cast<const T*>(a.v_cache) + w.hk * a.v_strides[2];
  const Pages pages(a, w.b, TL::EP);
  const uint64_t* const words = a.mask ? a.mask + (int64_t)(w.n0 + node) * a.mask_words : nullptr;
  using O = Own<T, DB, SMALL>;
  Joined<TL, O::WAVES> r;
  own_walk<TL, T, O::WAVES, O::BUFS, true>(
      r, smem, k, v, static_cast<const T*>(a.q) + (int64_t)(w.n0 + node) * a.q_strides[0] + head * a.q_strides[1], D, a.scale * 1.44269504f, w.t0, w.t1, w.cached,
      [&](int t) { return pages.find(t * 32 + (lane & 31) < w.keys ? t * 32 + (lane & 31) : w.keys - 1); },
      [&](const Pages::Place& place, uint32_t& ko, uint32_t& vo) { pages.offsets(place, ko, vo); }, [&](int t) { return tree_visible(a, w, node, words, t * 32); },
      [&](typename TL::State& st, int t0, int t1) { tree_strange<TL, T>(a, w, st, v, pages, words, node, t0 * 32, t1 * 32, 32); });
  finish<TL, T>(a, w, p, r.o, r.from, r.top, r.total, row < rows, node, head);
}
template <typename T, int DB, bool COUNTED, bool SMALL>
__global__ void __launch_bounds__((64 * Own<T, DB, SMALL>::WAVES), 1) tree_own_kernel(fi_tree_attention_args a, TreeSplit p) {
  __shared__ __attribute__((aligned(1024))) uint8_t smem[Own<T, DB, SMALL>::LDS];
  if constexpr (COUNTED) {
    __shared__ TreeLine line;
    line_up(a, p, line);
    along_the_line(a, p, line, [&](const TreeWork& w) {
      __syncthreads();   // (the piece before has been read to the end)
      tree_own_work<T, DB, SMALL>(a, w, p, smem);
    });
  } else {
    TreeWork w;
    if (tree_direct(a, p, w)) tree_own_work<T, DB, SMALL>(a, w, p, smem);
  }
}

// Joins the parts of a row (node, head), in their order and 16 in flight at once (they come from other dies: a load takes microseconds).  A wave per row: with
// thousands of them its instructions count, so everything that the row's lanes share is scalar and a lane has PER values next to each other.  WIDE (more
// parts of few rows): a workgroup per row, its waves add a quarter of the parts each, then the waves' sums are added.
template <typename T, int PER, bool WIDE>
__global__ void __launch_bounds__(256) tree_join_kernel(fi_tree_attention_args a, TreeSplit p, bool counted) {
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

// Whether every row of a tensor starts on 16 bytes and its last one, counted in 16-byte pieces, has a 32-bit offset.
bool pieces(const void* p, const int64_t* strides, const int64_t* counts, int n, int es) {
  if (reinterpret_cast<uintptr_t>(p) % 16) return false;
  double reach = 0;
  for (int i = 0; i < n; ++i) {
    if (strides[i] * es % 16) return false;
    reach += (double)strides[i] * es / 16 * (counts[i] > 0 ? counts[i] - 1 : 0);
  }
  return reach + 64 < 4294967296.0;
}
bool starts(const void* p, const int64_t* strides, int n, int es, int bytes) {
  if (reinterpret_cast<uintptr_t>(p) % bytes) return false;
  for (int i = 0; i < n; ++i)
    if (strides[i] * es % bytes) return false;
  return true;
}
int blocks_of(int head_dim) { return head_dim <= 64 ? 2 : head_dim <= 96 ? 3 : head_dim <= 128 ? 4 : 8; }

bool prompt_on_tiles(const fi_prompt_attention_args& a) {
  const int es = elem_size(a.dtype);
  const int64_t n[2] = {a.k_tokens, a.kv_heads};
  return a.head_dim * es % 16 == 0 && starts(a.q, a.q_strides, 2, es, 16) && starts(a.out, a.out_strides, 2, es, 4 * es) && pieces(a.k, a.k_strides, n, 2, es) &&
         pieces(a.v, a.v_strides, n, 2, es);
}
// The kernel of eight waves wants enough workgroups of 256 queries to fill the chip more than once, and offsets inside a tile below 2^32 bytes.
bool prompt_is_long(const fi_prompt_attention_args& a) {
  return a.dtype == FI_BF16 && a.head_dim <= 128 && (a.q_tokens / LONG_ROWS) * a.q_heads >= LONG_GROUPS && a.k_strides[0] < 1 << 24 && a.v_strides[0] < 1 << 24;
}
// Workgroups of 32 queries up to which they are taken (us, 128 queries / 32; 12 heads, sequences spread over their logarithm, causal).  bf16, heads of 64, two on a compute unit:
// 7 up to 301 tokens, 276 workgroups, 8.8 / 7.1; up to 1000, 684: 16.1 / 14.6; up to 2000, 1200: 25.8 / 30.6.  Of 128, one on a unit: 256 tokens, 108: 12.2 / 8.7; 7 up to 301: 11.5 / 12.8.
// Of 256: 7 up to 100 17.3 / 12.8; one of 2000, 756: 123 / 106.  fp32, bound by its products: heads of 128, 7 up to 301 48 / 25; one of 3000, 1128: 439 / 336; of 256, 7 up to 1000
// 284 / 214.  Without a causal mask all walks of a sequence are as long and sharing them counts for more: 4 images of up to 729 fp32 patches, 16 heads of 72, 960: 82 / 120;
// one of 729, 368: 78 / 65; of 256 in bf16, 336: 28 / 33.
template <typename T, int DB>
int64_t own_most(bool causal) {
  constexpr bool SLOW = sizeof(T) == 4 || DB > 4;
  return SLOW ? (DB <= 4 ? (causal ? 1200 : 384) : (causal ? 768 : 256)) : DB == 2 ? 768 : 256;
}
template <typename T, int DB, int DQ>
void prompt_waves(const fi_prompt_attention_args& a, dim3 grid, bool two, hipStream_t s) {
  const int64_t small = (a.q_tokens / 32 + a.n_seqs) * a.q_heads;
  if (small <= own_most<T, DB>(a.causal != 0)) return (void)(prompt_own_kernel<T, DB, DQ><<<dim3((uint32_t)small), 64 * Own<T, DB>::WAVES, 0, s>>>(a));
  if constexpr (sizeof(T) == 2 && DB <= 4) {
    if (two) return (void)(prompt_tile_kernel<T, DB, 2, DQ><<<grid, 128 * PROMPT_WAVES, 0, s>>>(a));
  }
  prompt_tile_kernel<T, DB, 1, DQ><<<grid, 64 * PROMPT_WAVES, 0, s>>>(a);
}
// (heads of 65 to 80 values: scores without the steps that heads of 96 take; 4 images of up to 729 fp32 queries, 16 heads of 72: 91 us, 82)
template <typename T>
int launch_prompt_tiles(const fi_prompt_attention_args& a, hipStream_t s) {
  const int db = blocks_of(a.head_dim);
  if constexpr (sizeof(T) == 2) {
    if (prompt_is_long(a)) {
      if (!one_launch((a.q_tokens / LONG_ROWS + a.n_seqs) * a.q_heads, 512)) return kTooLarge;
      const dim3 grid((uint32_t)((a.q_tokens / LONG_ROWS + a.n_seqs) * a.q_heads));
      if (db == 2) prompt_long_kernel<2, 64><<<grid, 512, 0, s>>>(a);
      else if (db == 3 && a.head_dim <= 80) prompt_long_kernel<3, 80><<<grid, 512, 0, s>>>(a);
      else if (db == 3) prompt_long_kernel<3, 96><<<grid, 512, 0, s>>>(a);
      else prompt_long_kernel<4, 128><<<grid, 512, 0, s>>>(a);
      return (int)hipGetLastError();
    }
  }
  // two groups where there is a workgroup or so per compute unit, and a walk is long (12 heads, 7 sequences up to 1000 tokens, spread over their logarithm: heads of 64 19.8 us
  // with one group, 16.4; of 128 27.1, 25.7; up to 301: 8.7, 8.4; 11.5, 12.7)
  if (!one_launch((a.q_tokens / PROMPT_ROWS + a.n_seqs) * a.q_heads, 64 * PROMPT_WAVES)) return kTooLarge;   // (two groups: 511 workgroups at most)
  const dim3 grid((uint32_t)((a.q_tokens / PROMPT_ROWS + a.n_seqs) * a.q_heads));
  const bool two = (int64_t)grid.x < 512 && a.k_tokens >= (db == 2 ? 128 : 256) * (int64_t)a.n_seqs;
  if (db == 2) prompt_waves<T, 2, 64>(a, grid, two, s);
  else if (db == 3 && a.head_dim <= 80) prompt_waves<T, 3, 80>(a, grid, two, s);
  else if (db == 3) prompt_waves<T, 3, 96>(a, grid, two, s);
  else if (db == 4) prompt_waves<T, 4, 128>(a, grid, two, s);
  else prompt_waves<T, 8, 256>(a, grid, two, s);
  return (int)hipGetLastError();
}

bool tree_on_tiles(const fi_tree_attention_args& a) {
  const int es = elem_size(a.dtype);
  const int64_t n[3] = {a.n_pages, a.page_size, a.kv_heads};
  return a.n_pages > 0 && a.table_columns > 0 && a.head_dim * es % 16 == 0 && starts(a.q, a.q_strides, 2, es, 16) && starts(a.out, a.out_strides, 2, es, 4 * es) &&
         pieces(a.k_cache, a.k_strides, n, 3, es) && pieces(a.v_cache, a.v_strides, n, 3, es);
}

// How a tree call is shared out, from its sizes alone (the workspace goes by it): rows of 32 whose waves have keys of their own, or of 128 or 256 that
// share them; parts of every sequence's keys, and the least keys of a part.
struct TreePlan { bool own, small, counted; int waves, blocks, splits, least, header; int64_t packed; };   // packed: blocks of all sequences together, if so dealt out
TreePlan plan_tree(const fi_tree_attention_args& a) {
  TreePlan p;
  const int64_t nodes = a.max_nodes < a.nodes ? a.max_nodes : a.nodes, rows = nodes * (a.q_heads / a.kv_heads);
  p.waves = rows <= 128 || a.head_dim > 128 ? 4 : 8;
  // Blocks of 32 rows with keys of their own, too, where the workgroups are few (us, shared / own; 64 nodes of one sequence of 100 keys, 8 heads 17.3 / 12.6), or keys are and
  // the workgroups many (about 10 keys, 40 nodes: 61 sequences of 32 heads 53 / 25, 16 nodes of 8 heads 15.8 / 10.9; 12 sequences, 60 keys 12.0 / 13.8).
  const int64_t streams = (int64_t)a.n_seqs * a.kv_heads;
  auto some = [](int64_t n) { return n < 1 << 20 ? n : 1 << 20; };   // (products of two stay in 64 bits)
  p.own = rows <= 32 || some(streams * ((rows + 31) / 32)) * (((int64_t)a.max_length + 127) / 128) <= 256 ||
          (a.max_length <= 256 && streams * ((rows + 32 * p.waves - 1) / (32 * p.waves)) > 256);
  const int64_t per_block = p.own ? 32 : 32 * p.waves;
  p.blocks = (int)((rows + per_block - 1) / per_block);
  const int64_t units = streams * p.blocks;
  auto parts = [&](int least) { return ((int64_t)a.max_length + least - 1) / least; };
  p.least = p.own ? 128 : 512;
  const double line = (double)units * ((double)a.page_size * a.table_columns / 32 + 64);   // (tiles, beginnings)
  p.counted = a.n_seqs > 1 && a.n_seqs <= SEQS && parts(p.least) > 1 && some(units) * parts(p.least) > 256 && line < 2147483648.0;
  // One wave, several workgroups on a compute unit (us, else / so; one node of 14 sequences of 32 heads: 7 keys 12.7 / 7.4, 100 keys 15.9 / 13.4; 64 of 32: 120 keys 64 / 32,
  // 240 85 / 56; 64 of 8: 240 keys 21.2 / 21.4; 12 nodes of 61 sequences of 32 heads, no history 46 / 10).
  p.small = p.own && (a.max_length <= 32 || (a.max_length <= 128 && units > 256) || (a.max_length <= 256 && units > 1024));
  int64_t splits;
  if (p.counted) {   // one sequence may have most of the keys
    p.least = stretch(p.own, a.dtype == FI_F32).least;
    splits = (255 + (int64_t)a.kv_heads * p.blocks) / ((int64_t)a.kv_heads * p.blocks);
  } else {
    // Four rounds of workgroups (4 x 131072 keys: one round 398 us, four 383: the hardware hands them out as units come free); parts of fewer keys where that
    // does not even make one (2 sequences of 1000 keys, 20 nodes: 22.7 us, 15.2).
    if (!p.own && some(units) * parts(512) <= 256)
      while (p.least > 128 && some(units) * parts(p.least - 128) <= 256) p.least -= 128;
    splits = units > 0 ? (1023 + units) / units : 1;
  }
  if (splits > parts(p.least)) splits = parts(p.least);
  // the workspace stays below 64 MB as far as the chip is full
  const int64_t room = (64ll << 20) / ((int64_t)a.nodes * a.q_heads * (a.head_dim + 2) * 4 + 1);
  if (splits > room && splits * some(units) > 512) splits = room * some(units) > 512 ? room : (512 + units - 1) / units;
  p.splits = splits < 1 ? 1 : splits > 63 ? 63 : (int)splits;
  if (p.splits == 1) p.counted = false;
  if (p.counted) ++p.splits;   // (a stretch may begin and end inside a part)
  if (p.small) p.counted = false, p.splits = 1;
  p.header = p.counted ? 4 + (a.n_seqs + 3) / 4 * 4 : 0;
  // Blocks for the most nodes of every sequence grow with sequences times nodes where one may have them all (max_nodes left out): past what a launch takes, and mostly without rows.
  // Packed ones cost a search for the sequence (us, single tokens of 32 heads of 128 with nothing said about them, direct / packed, and direct with max_nodes 1: 64 of 40 keys
  // 21.8 / 9.5, 8.5; 512 of 500 1895 / 285, 235; 2048 of 40 3436 / 100, 94).
  const int64_t packed = a.nodes * (a.q_heads / a.kv_heads) / per_block + a.n_seqs;
  p.packed = !p.counted && (int64_t)a.n_seqs * p.blocks > 4 * packed ? packed : 0;
  return p;
}
template <typename T, int DB>
int launch_tree_db(const fi_tree_attention_args& a, const TreePlan& p, hipStream_t s) {
  using TL = Tile<T, DB>;
  const int unit = p.own ? 32 : Shared<T, DB, 4>::KEYS;
  const TreeSplit t = {p.splits, p.least / unit, unit, stretch(p.own, TL::F32).over, p.own ? 32 : 32 * p.waves, p.packed ? 0 : p.blocks, p.header};
  const int64_t direct = p.packed ? p.packed : (int64_t)a.n_seqs * p.blocks, all_rows = a.nodes * a.q_heads;
  if (!p.counted && !one_launch(direct, p.small ? 64 : p.own ? 64 * Own<T, DB>::WAVES : 64 * p.waves)) return kTooLarge;
  if (p.splits > 1 && !one_launch((all_rows + 3) / 4, 256)) return kTooLarge;
  if (p.counted) {   // as many workgroups as run at a time: by LDS one on a compute unit, of the smallest heads two
    const dim3 grid(TL::PB == 128 && (p.own || p.waves == 4) ? 512 : 256);
    if (p.own) tree_own_kernel<T, DB, true, false><<<grid, 64 * Own<T, DB>::WAVES, 0, s>>>(a, t);
    else if (p.waves == 4) tree_tile_kernel<T, DB, 4, true><<<grid, 256, 0, s>>>(a, t);
    else if constexpr (DB <= 4) tree_tile_kernel<T, DB, 8, true><<<grid, 512, 0, s>>>(a, t);
  } else {
    const dim3 grid((uint32_t)direct, (uint32_t)a.kv_heads, (uint32_t)p.splits);
    if (p.own && p.small) tree_own_kernel<T, DB, false, true><<<grid, 64, 0, s>>>(a, t);
    else if (p.own) tree_own_kernel<T, DB, false, false><<<grid, 64 * Own<T, DB>::WAVES, 0, s>>>(a, t);
    else if (p.waves == 4) tree_tile_kernel<T, DB, 4, false><<<grid, 256, 0, s>>>(a, t);
    else if constexpr (DB <= 4) tree_tile_kernel<T, DB, 8, false><<<grid, 512, 0, s>>>(a, t);
  }
  constexpr int PER = DB <= 2 ? 1 : DB <= 4 ? 2 : 4;
  if (p.splits > 16 && all_rows <= 1024) tree_join_kernel<T, PER, true><<<dim3((uint32_t)all_rows), 256, 0, s>>>(a, t, p.counted);
  else if (p.splits > 1) tree_join_kernel<T, PER, false><<<dim3((uint32_t)((all_rows + 3) / 4)), 256, 0, s>>>(a, t, p.counted);
  return (int)hipGetLastError();
}
template <typename T>
int launch_tree_tiles(const fi_tree_attention_args& a, hipStream_t s) {
  const TreePlan p = plan_tree(a);
  switch (blocks_of(a.head_dim)) {
    case 2: return launch_tree_db<T, 2>(a, p, s);
    case 3: return launch_tree_db<T, 3>(a, p, s);
    case 4: return launch_tree_db<T, 4>(a, p, s);
    default: return launch_tree_db<T, 8>(a, p, s);
  }
}

}  // namespace

int launch_prompt_attention(const fi_prompt_attention_args& a, void* stream) {
  const hipStream_t s = static_cast<hipStream_t>(stream);
  if (prompt_on_tiles(a)) return a.dtype == FI_F32 ? launch_prompt_tiles<float>(a, s) : launch_prompt_tiles<bf16_t>(a, s);
  if (!one_launch(a.q_tokens, 64)) return kTooLarge;
  const dim3 grid((uint32_t)a.q_tokens, (uint32_t)a.q_heads);
  if (a.dtype == FI_F32) prompt_row_kernel<float><<<grid, 64, 0, s>>>(a);
  else prompt_row_kernel<bf16_t><<<grid, 64, 0, s>>>(a);
  return (int)hipGetLastError();
}

uint64_t tree_workspace(const fi_tree_attention_args& a) {
  const TreePlan p = plan_tree(a);
  return p.splits > 1 ? ((uint64_t)a.nodes * a.q_heads * p.splits * (a.head_dim + 2) + p.header) * 4 : 0;
}

int launch_tree_attention(const fi_tree_attention_args& a, void* stream) {
  const hipStream_t s = static_cast<hipStream_t>(stream);
  if (tree_on_tiles(a)) return a.dtype == FI_F32 ? launch_tree_tiles<float>(a, s) : launch_tree_tiles<bf16_t>(a, s);
  if (!one_launch(a.nodes, 64)) return kTooLarge;
  const dim3 grid((uint32_t)a.nodes, (uint32_t)a.q_heads);
  if (a.dtype == FI_F32) tree_row_kernel<float><<<grid, 64, 0, s>>>(a);
  else tree_row_kernel<bf16_t><<<grid, 64, 0, s>>>(a);
  return (int)hipGetLastError();
}

}  // namespace fi
