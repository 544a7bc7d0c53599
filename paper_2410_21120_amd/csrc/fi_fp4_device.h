// Attention of drafted trees, or single tokens, over a paged cache of 4-bit values: the kernels and their launch, for one type of queries each (fi_fp4.hip, fi_fp4_f32.hip).
//
// A value is an E2M1 code times its block's power of two.  CDNA4 converts two codes with their scale to two bf16 in one instruction, exactly (two significant
// bits), so keys and values enter the bf16 matrix instructions as they are held: nothing is left to apply to sums, whatever blocks a head has.
#pragma once

#include "fi_ops.h"
#include "fi_tree_device.h"

namespace fi {

// How a call is shared out, from its sizes alone (the workspace goes by it): dwords of codes of a key that a lane has, columns of 16 queries a wave has, blocks of
// rows of a sequence, parts of its keys and the least keys of one, floats before the parts in the workspace, blocks of all sequences together where they are so dealt out.
struct Fp4Plan { int kd, nb, blocks, splits, least, header; bool counted; int64_t packed; };
Fp4Plan plan_fp4(const fi_fp4_tree_attention_args& a);
int launch_fp4_tree_f32(const fi_fp4_tree_attention_args& a, void* stream);

namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
constexpr int BLOCK = FI_FP4_BLOCK, NAN_SCALE = 255, MOST_SCALE = 252;

// Eight values of a head as fp32, from any start (VEC: rows start on 16 bytes).
template <bool VEC>
__device__ __forceinline__ void load8(const bf16_t* p, float (&x)[8]) {
  if constexpr (VEC) {
    const u32x4 a = *reinterpret_cast<const u32x4*>(p);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[2 * i] = __uint_as_float(a[i] << 16);
      x[2 * i + 1] = __uint_as_float(a[i] & 0xFFFF0000u);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = bf2f(p[i]);
  }
}
template <bool VEC>
__device__ __forceinline__ void load8(const float* p, float (&x)[8]) {
  if constexpr (VEC) {
    const float4 a = reinterpret_cast<const float4*>(p)[0], b = reinterpret_cast<const float4*>(p)[1];
    x[0] = a.x, x[1] = a.y, x[2] = a.z, x[3] = a.w, x[4] = b.x, x[5] = b.y, x[6] = b.z, x[7] = b.w;
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = p[i];
  }
}
// Byte B of a dword of codes: two values as bf16, the low half's in the low half.
template <int B>
__device__ __forceinline__ uint32_t decode2(uint32_t codes, float scale) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, B));
}
__device__ __forceinline__ float scale_of(uint32_t b) { return __uint_as_float(b << 23); }   // (255: an exponent of ones, of which the conversion makes NaN)

// A wave has 16 NB queries (rows: node and head) as columns and keys of its own, 32 at a time: scores S^T = K Q^T, outputs O^T = V^T P^T, by 16 x 16 x 32 products.
// Lane l holds scores of query l & 15, of the keys 4 (l >> 4) + i and 16 + 4 (l >> 4) + i, i < 4, of a tile, and these registers are the operand of the second product
// as they stand: its lane l has to bring values of just these eight keys.  The reduction over a head's values may run in any order, so lane l brings the KD dwords
// of codes from KD (l >> 4) on, of key l & 15.  Values: DT of a head's, from DT (l & 15) on, of each of the eight keys; two keys' are paired by a byte permute.
// All loads go to registers, a tile ahead: lanes of a key read 64 bytes and more that follow each other.
// MODE: how the lanes find their keys.  WHOLE pages hold a multiple of 16 keys, so the 16 keys of half a tile lie in one page, whose number and address are the wave's (scalar registers), and
// a lane's offsets are the same in every tile; FULL heads beside that have 32 KD values, so a lane's codes of a key are one load.  Else every lane looks up its own ten keys.
enum Fp4Mode { ANY, WHOLE, FULL };
template <typename T, int KD_, int NB_, Fp4Mode MODE_>
struct Fp4 {
  static constexpr int KD = KD_, NB = NB_;                                             // dwords of codes of a key per lane; columns of queries
  static constexpr Fp4Mode MODE = MODE_;
  static constexpr bool F32 = sizeof(T) == 4;
  static constexpr int QT = F32 ? 3 : 1, PT = F32 ? 3 : NB <= 2 ? 2 : 1;               // bf16 terms of a query's value, of a weight
  static constexpr int VW = KD == 8 ? 2 : 1, DT = KD == 2 ? 4 : 8 * VW;                // words of codes of a value row per lane; values in them
  static constexpr int KS = KD == 8 ? 2 : KD == 3 ? 3 : 1;                             // scales of a key per lane
  static constexpr int WAVES = 4;
  static constexpr int LDS = WAVES * (NB * DT * 1024 + NB * 512);
};
template <typename F>
struct Fp4Tile {
  uint32_t k[2][F::KD], ks[2][F::KS], v[8][F::VW], vs[8][F::VW];
};

// A lane's bytes in rows of codes and scales.
template <typename F>
struct Fp4Lane {
  uint32_t k[F::KD], ks[F::KS], v[F::VW], vs[F::VW];
  __device__ __forceinline__ explicit Fp4Lane(int D) {
    const int lane = threadIdx.x & 63, kq = lane >> 4, m = lane & 15, words = D / 8, blocks = (D + BLOCK - 1) / BLOCK;
    auto most = [](int x, int n) { return (uint32_t)(x < n ? x : n - 1); };
#pragma unroll
    for (int c = 0; c < F::KD; ++c) k[c] = 4 * most(kq * F::KD + c, words);   // past the head's end: its last dword, against queries' zeros
#pragma unroll
    for (int c = 0; c < F::KS; ++c) ks[c] = most(F::KD == 3 ? (kq * 3 + c) >> 2 : F::KD == 2 ? kq >> 1 : F::KD == 4 ? kq : 2 * kq + c, blocks);
#pragma unroll
    for (int c = 0; c < F::VW; ++c) {
      v[c] = F::DT == 4 ? 2 * most(m, 2 * words) : 4 * most(16 * c + m, words);   // (rows of outputs past the head's end are not stored)
      vs[c] = most(F::DT == 4 ? m >> 3 : 4 * c + (m >> 2), blocks);
    }
  }
  __device__ __forceinline__ void ahead(uint32_t codes, uint32_t scales, uint32_t value_codes, uint32_t value_scales) {
#pragma unroll
    for (int c = 0; c < F::KD; ++c) k[c] += codes;
#pragma unroll
    for (int c = 0; c < F::KS; ++c) ks[c] += scales;
#pragma unroll
    for (int c = 0; c < F::VW; ++c) v[c] += value_codes, vs[c] += value_scales;
  }
};
// A lane's address: `base` is the wave's (in WHOLE and FULL), so that a load takes it from scalar registers with the lane's offset as it stands.  (The empty asm keeps the
// compiler from adding the two ahead of the loop, which leaves an addition of 64 bits and two registers for every load in it.)
__device__ __forceinline__ const uint8_t* lane_at(const uint8_t* base, uint32_t off) {
  asm("" : "+v"(off));
  return base + off;
}
template <typename F>
__device__ __forceinline__ void fp4_load_key(Fp4Tile<F>& t, int h, const Fp4Lane<F>& at, const uint8_t* codes, const uint8_t* scales) {
  if constexpr (F::MODE == FULL) {
    const uint8_t* const p = lane_at(codes, at.k[0]);
#pragma unroll
    for (int c = 0; c < F::KD; c += 4) {
      constexpr int N = F::KD < 4 ? F::KD : 4;
      typedef uint32_t vec __attribute__((ext_vector_type(N), aligned(4)));
      const vec x = *reinterpret_cast<const vec*>(p + 4 * c);
#pragma unroll
      for (int i = 0; i < N; ++i) t.k[h][c + i] = x[i];
    }
  } else {
#pragma unroll
    for (int c = 0; c < F::KD; ++c) t.k[h][c] = *reinterpret_cast<const uint32_t*>(lane_at(codes, at.k[c]));
  }
#pragma unroll
  for (int c = 0; c < F::KS; ++c) t.ks[h][c] = *lane_at(scales, at.ks[c]);
}
template <typename F>
__device__ __forceinline__ void fp4_load_value(Fp4Tile<F>& t, int j, const Fp4Lane<F>& at, const uint8_t* codes, const uint8_t* scales) {
#pragma unroll
  for (int c = 0; c < F::VW; ++c) {
    const uint8_t* const p = lane_at(codes, at.v[c]);
    t.v[j][c] = F::DT == 4 ? (uint32_t)*reinterpret_cast<const uint16_t*>(p) : *reinterpret_cast<const uint32_t*>(p);
    t.vs[j][c] = *lane_at(scales, at.vs[c]);
  }
}

// Eight values of a row in bf16 terms: what each leaves out by itself is the next.
template <int TERMS>
__device__ __forceinline__ void terms8(float (&x)[8], u32x4 (&w)[TERMS]) {
#pragma unroll
  for (int t = 0; t < TERMS; ++t)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      w[t][i] = pack_bf16x2(x[2 * i], x[2 * i + 1]);
      if (t + 1 < TERMS) {
        x[2 * i] -= __uint_as_float(w[t][i] << 16);
        x[2 * i + 1] -= __uint_as_float(w[t][i] & 0xFFFF0000u);
      }
    }
}

template <typename F>
struct Fp4State {
  f32x4 o[F::NB][F::DT];
  float top[F::NB], total[F::NB];
};

__device__ __forceinline__ f32x4 product16(const u32x4 a, const u32x4 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}
__device__ __forceinline__ float over_keys_max(float m) {   // over the four lanes of a query
  const auto x = __builtin_amdgcn_permlane16_swap(__float_as_uint(m), __float_as_uint(m), false, false);
  m = fmaxf(__uint_as_float(x[0]), __uint_as_float(x[1]));
  const auto y = __builtin_amdgcn_permlane32_swap(__float_as_uint(m), __float_as_uint(m), false, false);
  return fmaxf(__uint_as_float(y[0]), __uint_as_float(y[1]));
}
__device__ __forceinline__ float over_keys_sum(float m) {
  const auto x = __builtin_amdgcn_permlane16_swap(__float_as_uint(m), __float_as_uint(m), false, false);
  m = __uint_as_float(x[0]) + __uint_as_float(x[1]);
  const auto y = __builtin_amdgcn_permlane32_swap(__float_as_uint(m), __float_as_uint(m), false, false);
  return __uint_as_float(y[0]) + __uint_as_float(y[1]);
}

// Pair u of a word of codes, values 2 u and 2 u + 1.
__device__ __forceinline__ uint32_t decode_pair(int u, uint32_t codes, float scale) {
  return u == 0 ? decode2<0>(codes, scale) : u == 1 ? decode2<1>(codes, scale) : u == 2 ? decode2<2>(codes, scale) : decode2<3>(codes, scale);
}

// One tile.  masked: some query does not see some key; visible(nb): bit k tells whether the lane's query of column nb sees key k of the tile.  Returns whether a value's
// scale was put aside (masked tiles: NaN times a weight of zero would be NaN for queries that do not see the key).
template <typename F, typename Visible>
__device__ __forceinline__ bool fp4_attend(Fp4State<F>& st, const u32x4 (&q)[F::NB][F::QT][F::KD], Fp4Tile<F>& t, float c, bool masked, Visible visible) {
  const int kq = (threadIdx.x & 63) >> 4;
  f32x4 s[F::NB][2];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
#pragma unroll
    for (int nb = 0; nb < F::NB; ++nb) s[nb][h] = f32x4{0, 0, 0, 0};
#pragma unroll
    for (int w = 0; w < F::KD; ++w) {
      const float scale = scale_of(t.ks[h][F::KD == 8 ? w >> 2 : F::KD == 3 ? w : 0]);
      const uint32_t x = t.k[h][w];
      const u32x4 key = {decode2<0>(x, scale), decode2<1>(x, scale), decode2<2>(x, scale), decode2<3>(x, scale)};
#pragma unroll
      for (int nb = 0; nb < F::NB; ++nb)
#pragma unroll
        for (int term = F::QT - 1; term >= 0; --term) s[nb][h] = product16(key, q[nb][term][w], s[nb][h]);
    }
  }
  bool strange = false;
  if (masked) {
#pragma unroll
    for (int nb = 0; nb < F::NB; ++nb) {
      const uint32_t bits = visible(nb) >> (4 * kq);
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int i = 0; i < 4; ++i) s[nb][h][i] = (bits >> (16 * h + i)) & 1 ? s[nb][h][i] : -INFINITY;
    }
#pragma unroll
    for (int j = 0; j < 8; ++j)
#pragma unroll
      for (int w = 0; w < F::VW; ++w) {
        const bool odd = t.vs[j][w] > MOST_SCALE;
        strange |= odd;
        t.vs[j][w] = odd ? 127 : t.vs[j][w];
      }
  }
  u32x4 p[F::NB][F::PT];
#pragma unroll
  for (int nb = 0; nb < F::NB; ++nb) {
    float m = s[nb][0][0];
#pragma unroll
    for (int i = 1; i < 8; ++i) m = fmaxf(m, s[nb][i >> 2][i & 3]);
    m = over_keys_max(m);
    // the weights may be taken against any number that keeps them in range: it moves only when the maximum has grown by a factor of 2^8 in weight
    if (__any((m - st.top[nb]) * c > 8.0f || (st.top[nb] == -INFINITY && m > -INFINITY))) {
      const float now = fmaxf(st.top[nb], m), shrink = __builtin_amdgcn_exp2f((st.top[nb] - (now == -INFINITY ? 0.0f : now)) * c);
      st.total[nb] *= shrink;
      st.top[nb] = now;
#pragma unroll
      for (int d = 0; d < F::DT; ++d)
#pragma unroll
        for (int i = 0; i < 4; ++i) st.o[nb][d][i] *= shrink;
    }
    const float base = st.top[nb] == -INFINITY ? 0.0f : st.top[nb] * c;
    float x[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      x[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[nb][i >> 2][i & 3], c, -base));
      st.total[nb] += x[i];
    }
    terms8<F::PT>(x, p[nb]);
  }
#pragma unroll
  for (int w = 0; w < F::VW; ++w)
#pragma unroll
    for (int u = 0; u < (F::DT == 4 ? 2 : 4); ++u) {
      uint32_t x[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) x[j] = decode_pair(u, t.v[j][w], scale_of(t.vs[j][w]));
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        u32x4 v;
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = __builtin_amdgcn_perm(x[2 * j + 1], x[2 * j], half ? 0x07060302u : 0x05040100u);
#pragma unroll
        for (int nb = 0; nb < F::NB; ++nb)
#pragma unroll
          for (int term = F::PT - 1; term >= 0; --term) {
            f32x4& o = st.o[nb][8 * w + 2 * u + half];
            o = product16(v, p[nb][term], o);
          }
      }
    }
  return strange;
}

// A sequence's tiles in the cache.  Keys past the last one read the place that they would have (there is one in its page) or, from pages past the last, that page's.
template <typename F>
struct Fp4Walk {
  const fi_fp4_tree_attention_args& a;
  const int32_t* table;
  const uint8_t *k, *ks, *v, *vs;   // the key head's part
  Fp4Lane<F> at;
  uint32_t inv;                     // floor(2^32 / page size): a quotient by it is right or one too small
  int keys, last_column, page[2];   // page: of the tile that is loaded next
  // where a row of a page begins: in WHOLE and FULL by two scalar products of 32 bits (strides are below 2^31 there: checked on the host)
  static __device__ __forceinline__ uint64_t row_at(const int64_t* strides, int p, int row) {
    if constexpr (F::MODE != ANY) return (uint64_t)(uint32_t)p * (uint32_t)strides[0] + (uint64_t)(uint32_t)row * (uint32_t)strides[1];
    else return (uint64_t)((int64_t)p * strides[0] + (int64_t)row * strides[1]);
  }
  __device__ __forceinline__ Fp4Walk(const fi_fp4_tree_attention_args& args, const TreeWork& w)
      : a(args), table(args.block_table + w.b * args.table_stride), k(args.k_codes + w.hk * args.k_codes_strides[2]), ks(args.k_scales + w.hk * args.k_scales_strides[2]),
        v(args.v_codes + w.hk * args.v_codes_strides[2]), vs(args.v_scales + w.hk * args.v_scales_strides[2]), at(args.head_dim),
        inv(args.page_size == 1 ? ~0u : (uint32_t)((1ull << 32) / (uint32_t)args.page_size)), keys(w.keys) {
    int row;
    last_column = place(keys - 1, row);
    if constexpr (F::MODE != ANY) {   // (offsets of 16 rows are below 2^31: checked on the host)
      const int lane = threadIdx.x & 63, r = lane & 15, first = 4 * (lane >> 4);
      at.ahead((uint32_t)(r * a.k_codes_strides[1]), (uint32_t)(r * a.k_scales_strides[1]), (uint32_t)(first * a.v_codes_strides[1]), (uint32_t)(first * a.v_scales_strides[1]));
    }
  }
  __device__ __forceinline__ int place(int key, int& row) const {
    uint32_t c = __umulhi((uint32_t)key, inv), r = (uint32_t)key - c * (uint32_t)a.page_size;
    if (r >= (uint32_t)a.page_size) ++c, r -= (uint32_t)a.page_size;
    row = (int)r;
    return (int)c;
  }
  __device__ __forceinline__ int page_at(int column) const { return clamp_int(table[column], 0, a.n_pages - 1); }
  __device__ __forceinline__ void ask(int tile) {
    if constexpr (F::MODE != ANY) {
      typedef const int32_t __attribute__((address_space(4))) entry;   // (the table does not change meanwhile: scalar loads)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        int row;
        const int column = place(tile * 32 + 16 * h, row);
        page[h] = ((entry*)(uintptr_t)table)[column < last_column ? column : last_column];
      }
    }
  }
  __device__ __forceinline__ void load(Fp4Tile<F>& t, int tile) {
    const int lane = threadIdx.x & 63, kq = lane >> 4, r = lane & 15;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int first = tile * 32 + 16 * h;
      if constexpr (F::MODE != ANY) {
        int row;
        place(first, row);
        const int p = clamp_int(page[h], 0, a.n_pages - 1);
        fp4_load_key<F>(t, h, at, k + row_at(a.k_codes_strides, p, row), ks + row_at(a.k_scales_strides, p, row));
        const uint8_t *from = v + row_at(a.v_codes_strides, p, row), *scales = vs + row_at(a.v_scales_strides, p, row);
#pragma unroll
        for (int i = 0; i < 4; ++i) fp4_load_value<F>(t, 4 * h + i, at, from + i * (uint32_t)a.v_codes_strides[1], scales + i * (uint32_t)a.v_scales_strides[1]);
      } else {
        auto find = [&](int key, int& p, int& row) { p = page_at(place(key < keys ? key : keys - 1, row)); };
        int p, row;
        find(first + r, p, row);
        fp4_load_key<F>(t, h, at, k + row_at(a.k_codes_strides, p, row), ks + row_at(a.k_scales_strides, p, row));
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          find(first + 4 * kq + i, p, row);
          fp4_load_value<F>(t, 4 * h + i, at, v + row_at(a.v_codes_strides, p, row), vs + row_at(a.v_scales_strides, p, row));
        }
      }
    }
  }
  __device__ __forceinline__ const uint8_t* value_scales(int key) const {
    int row;
    const int p = page_at(place(key, row));
    return vs + row_at(a.v_scales_strides, p, row);
  }
};

template <typename T, typename F>
__device__ __forceinline__ void fp4_work(const fi_fp4_tree_attention_args& a, const TreeWork& w, const TreeSplit& p, uint8_t* smem) {
  constexpr int NB = F::NB, DT = F::DT, WAVES = F::WAVES;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), kq = lane >> 4;
  const int D = a.head_dim, group = a.q_heads / a.kv_heads, rows = w.nodes * group, first = w.block * 16 * NB;
  if (first >= rows) return;
  auto share = [&](int x) { return __builtin_amdgcn_readfirstlane(w.t0 + (int)((int64_t)(w.t1 - w.t0) * x / WAVES)); };
  const int t0 = share(wave), t1 = share(wave + 1);
  auto row_of = [&](int nb) { return first + 16 * nb + (lane & 15); };
  auto mine = [&](int nb) { return row_of(nb) < rows ? row_of(nb) : rows - 1; };
  // the queries: values 8 (KD kq + c) .. of the lane's row of every column, as they are or in three terms; zeros past the head's end
  u32x4 q[NB][F::QT][F::KD];
#pragma unroll
  for (int nb = 0; nb < NB; ++nb) {
    const int node = mine(nb) / group, head = w.hk * group + mine(nb) % group;
    const T* const from = static_cast<const T*>(a.q) + (int64_t)(w.n0 + node) * a.q_strides[0] + head * a.q_strides[1];
#pragma unroll
    for (int c = 0; c < F::KD; ++c) {
      const int d = 8 * (F::KD * kq + c);
      float x[8] = {};
      if (d < D) load8<false>(from + d, x);
      u32x4 terms[F::QT];
      terms8<F::QT>(x, terms);
#pragma unroll
      for (int term = 0; term < F::QT; ++term) q[nb][term][c] = terms[term];
    }
  }
  Fp4State<F> st;
#pragma unroll
  for (int nb = 0; nb < NB; ++nb) {
    st.top[nb] = -INFINITY;
    st.total[nb] = 0.0f;
#pragma unroll
    for (int d = 0; d < DT; ++d) st.o[nb][d] = f32x4{0, 0, 0, 0};
  }
  const float c = a.scale * 1.44269504f;
  auto visible = [&](int nb, int key) {
    const int node = mine(nb) / group;
    return tree_visible(a, w, node, a.mask ? a.mask + (int64_t)(w.n0 + node) * a.mask_words : nullptr, key);
  };
  if (t0 < t1) {
    Fp4Walk<F> walk(a, w);
    Fp4Tile<F> x, y;
    bool strange = false;
    auto load = [&](Fp4Tile<F>& tile, int t) {
      walk.load(tile, t);
      if (t + 1 < t1) walk.ask(t + 1);
      __builtin_amdgcn_sched_barrier(0);   // (they are on their way before the tile at hand is worked on)
    };
    auto attend = [&](Fp4Tile<F>& tile, int t) {
      strange |= fp4_attend<F>(st, q, tile, c, (t + 1) * 32 > w.cached, [&](int nb) { return visible(nb, t * 32); });
    };
    walk.ask(t0);
    load(x, t0);
    for (int t = t0; t < t1; t += 2) {
      if (t + 1 < t1) load(y, t + 1);
      attend(x, t);
      if (t + 1 >= t1) break;
      if (t + 2 < t1) load(x, t + 2);
      attend(y, t + 1);
    }
    if (__any(strange)) {   // blocks of NaN in masked tiles: for the queries that see the key
      const int masked = w.cached / 32 * 32, blocks = (D + BLOCK - 1) / BLOCK;
      for (int key = t0 * 32 > masked ? t0 * 32 : masked; key < t1 * 32 && key < w.keys; ++key) {
        const uint8_t* const scales = walk.value_scales(key);
#pragma unroll
        for (int half = 0; half < F::VW; ++half) {
          const int block = F::DT == 4 ? kq >> 1 : 4 * half + kq;   // of the lane's values DT (4 kq + i) + ...
          if (block >= blocks || scales[block] <= MOST_SCALE) continue;
#pragma unroll
          for (int nb = 0; nb < NB; ++nb)
            if (visible(nb, key) & 1)
#pragma unroll
              for (int d = 0; d < DT / F::VW; ++d) st.o[nb][half * 8 + d] += __uint_as_float(0x7FC00000u);
        }
      }
    }
  }
  // the waves' sums against the largest maximum, added in the order of the waves: wave x adds the values d with d % WAVES == x
  f32x4* const sums = reinterpret_cast<f32x4*>(smem) + lane;
  float2* const stats = reinterpret_cast<float2*>(smem + WAVES * NB * DT * 1024) + lane;
#pragma unroll
  for (int nb = 0; nb < NB; ++nb) {
#pragma unroll
    for (int d = 0; d < DT; ++d) sums[((wave * NB + nb) * DT + d) * 64] = st.o[nb][d];
    stats[(wave * NB + nb) * 64] = make_float2(st.top[nb], over_keys_sum(st.total[nb]));
  }
  __syncthreads();
#pragma unroll
  for (int nb = 0; nb < NB; ++nb) {
    float top = stats[nb * 64].x, total = 0.0f, factor[WAVES];
#pragma unroll
    for (int x = 1; x < WAVES; ++x) top = fmaxf(top, stats[(x * NB + nb) * 64].x);
    const float base = top == -INFINITY ? 0.0f : top;
#pragma unroll
    for (int x = 0; x < WAVES; ++x) {
      const float2 other = stats[(x * NB + nb) * 64];
      factor[x] = __builtin_amdgcn_exp2f((other.x - base) * c);
      total += other.y * factor[x];
    }
    const float inv = w.splits > 1 ? 1.0f : total == 0.0f ? 0.0f : 1.0f / total;
    const bool there = row_of(nb) < rows;
    const int node = mine(nb) / group, head = w.hk * group + mine(nb) % group;
    const int64_t row = (int64_t)(w.n0 + node) * a.q_heads + head;
    T* const out = static_cast<T*>(a.out) + (int64_t)(w.n0 + node) * a.out_strides[0] + head * a.out_strides[1];
    float* const part = part_sums(a, p, row, w.split);
    // DT values from DT (4 kq + i) on (of KD 8: 8 of each half) are the lane's; a wave takes DT / WAVES that follow each other
    constexpr int N = DT / WAVES;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float v[N];
#pragma unroll
      for (int n = 0; n < N; ++n) v[n] = 0.0f;
#pragma unroll
      for (int n = 0; n < N; ++n)
#pragma unroll
        for (int x = 0; x < WAVES; ++x) v[n] += reinterpret_cast<const float*>(&sums[((x * NB + nb) * DT + wave * N + n) * 64])[i] * factor[x];
      const int e = wave * N, d = F::VW == 2 ? (e >> 3) * 128 + 8 * (4 * kq + i) + (e & 7) : DT * (4 * kq + i) + e;
      if (!there || d >= D) continue;
#pragma unroll
      for (int n = 0; n < N; ++n) {
        if (w.splits > 1) part[d + n] = v[n];
        else fi::st(out + d + n, v[n] * inv);
      }
    }
    if (w.splits > 1 && there && wave == 0 && kq == 0) *reinterpret_cast<float2*>(part_stats(a, p, row, w.split)) = make_float2(top, total);
  }
}

template <typename T, int KD, int NB, Fp4Mode MODE, bool COUNTED>
__global__ void __launch_bounds__(256, (KD <= 4 && sizeof(T) == 2 ? (NB == 1 ? 3 : NB == 2 ? 2 : 1) : 1)) fp4_tree_kernel(fi_fp4_tree_attention_args a, TreeSplit p) {
  using F = Fp4<T, KD, NB, MODE>;
  __shared__ __attribute__((aligned(16))) uint8_t smem[F::LDS];
  if constexpr (COUNTED) {
    __shared__ TreeLine line;
    line_up(a, p, line);
    along_the_line(a, p, line, [&](const TreeWork& w) {
      __syncthreads();   // (the piece before has been joined)
      fp4_work<T, F>(a, w, p, smem);
    });
  } else {
    TreeWork w;
    if (tree_direct(a, p, w)) fp4_work<T, F>(a, w, p, smem);
  }
}

template <typename T, int KD, int NB, Fp4Mode MODE>
int launch_fp4_tree(const fi_fp4_tree_attention_args& a, const Fp4Plan& p, hipStream_t s) {
  const TreeSplit t = {p.splits, p.least / 32, 32, 8, 16 * NB, p.packed ? 0 : p.blocks, p.header};
  const int64_t direct = p.packed ? p.packed : (int64_t)a.n_seqs * p.blocks, all_rows = a.nodes * a.q_heads;
  if (!p.counted && !one_launch(direct, 256)) return kTooLarge;
  if (p.splits > 1 && !one_launch((all_rows + 3) / 4, 256)) return kTooLarge;
  if (p.counted) fp4_tree_kernel<T, KD, NB, MODE, true><<<dim3(KD <= 4 && NB == 1 && sizeof(T) == 2 ? 768 : 512), 256, 0, s>>>(a, t);
  else fp4_tree_kernel<T, KD, NB, MODE, false><<<dim3((uint32_t)direct, (uint32_t)a.kv_heads, (uint32_t)p.splits), 256, 0, s>>>(a, t);
  constexpr int PER = KD <= 2 ? 1 : KD <= 4 ? 2 : 4;
  if (p.splits > 16 && all_rows <= 1024) tree_join_kernel<fi_fp4_tree_attention_args, T, PER, true><<<dim3((uint32_t)all_rows), 256, 0, s>>>(a, t, p.counted);
  else if (p.splits > 1) tree_join_kernel<fi_fp4_tree_attention_args, T, PER, false><<<dim3((uint32_t)((all_rows + 3) / 4)), 256, 0, s>>>(a, t, p.counted);
  return (int)hipGetLastError();
}
template <typename T, int KD, int NB>
int launch_fp4_mode(const fi_fp4_tree_attention_args& a, const Fp4Plan& p, hipStream_t s) {
  const int64_t far = (1ll << 31) / 16 - 1024;
  bool whole = a.page_size % 16 == 0;
  for (const int64_t* strides : {a.k_codes_strides, a.k_scales_strides, a.v_codes_strides, a.v_scales_strides}) whole = whole && strides[0] < 1ll << 31 && strides[1] < far;
  return !whole ? launch_fp4_tree<T, KD, NB, ANY>(a, p, s) : a.head_dim == 32 * KD ? launch_fp4_tree<T, KD, NB, FULL>(a, p, s) : launch_fp4_tree<T, KD, NB, WHOLE>(a, p, s);
}
template <typename T, int KD>
int launch_fp4_columns(const fi_fp4_tree_attention_args& a, const Fp4Plan& p, hipStream_t s) {
  if (p.nb == 1) return launch_fp4_mode<T, KD, 1>(a, p, s);
  if constexpr (sizeof(T) == 2 || KD < 8)
    if (p.nb == 2) return launch_fp4_mode<T, KD, 2>(a, p, s);
  if constexpr (sizeof(T) == 2 && KD < 8)
    if (p.nb == 4) return launch_fp4_mode<T, KD, 4>(a, p, s);
  return (int)hipErrorInvalidValue;   // (plan_fp4 makes no other)
}
template <typename T>
int launch_fp4_type(const fi_fp4_tree_attention_args& a, hipStream_t s) {
  const Fp4Plan p = plan_fp4(a);
  switch (p.kd) {
    case 2: return launch_fp4_columns<T, 2>(a, p, s);
    case 3: return launch_fp4_columns<T, 3>(a, p, s);
    case 4: return launch_fp4_columns<T, 4>(a, p, s);
    default: return launch_fp4_columns<T, 8>(a, p, s);
  }
}

}  // namespace
}  // namespace fi
