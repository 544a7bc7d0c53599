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
struct Fp4Plan { int kd, nb, on_unit, blocks, splits, least, header; bool counted, small; int64_t packed; };   // small: a wave a workgroup, and parts are none
Fp4Plan plan_fp4(const fi_fp4_tree_attention_args& a);
int launch_fp4_tree_f32(const fi_fp4_tree_attention_args& a, void* stream);

namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
constexpr int BLOCK = FI_FP4_BLOCK, NAN_SCALE = 255, MOST_SCALE = 252;

// Eight values of a head as fp32, from any start (the hardware takes loads that are aligned to two bytes).
__device__ __forceinline__ void load8(const bf16_t* p, float (&x)[8]) {
  typedef uint32_t piece __attribute__((ext_vector_type(4), aligned(2)));
  const piece a = *reinterpret_cast<const piece*>(p);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = __uint_as_float(a[i] << 16);
    x[2 * i + 1] = __uint_as_float(a[i] & 0xFFFF0000u);
  }
}
__device__ __forceinline__ void load8(const float* p, float (&x)[8]) {
  typedef float piece __attribute__((ext_vector_type(4), aligned(4)));
  const piece a = reinterpret_cast<const piece*>(p)[0], b = reinterpret_cast<const piece*>(p)[1];
#pragma unroll
  for (int i = 0; i < 4; ++i) x[i] = a[i], x[4 + i] = b[i];
}
// Four results, to any start.
__device__ __forceinline__ void store4(float* p, float a, float b, float c, float d) {
  typedef float piece __attribute__((ext_vector_type(4), aligned(4)));
  *reinterpret_cast<piece*>(p) = piece{a, b, c, d};
}
__device__ __forceinline__ void store4(bf16_t* p, float a, float b, float c, float d) {
  typedef uint32_t piece __attribute__((ext_vector_type(2), aligned(2)));
  *reinterpret_cast<piece*>(p) = piece{pack_bf16x2(a, b), pack_bf16x2(c, d)};
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
// MODE: how keys come to the lanes.  In pages that hold a multiple of 16 keys, the 16 keys of half a tile lie in one page, whose number and address are the wave's (scalar registers), and a
// lane's offsets are the same in every tile: direct loads bring a tile to LDS, a wave's own, while the one before it is worked on.  RING: heads of 64, 128 and 256, by 16
// bytes; WORDS: others, by 4.  ANY: other pages, or strides that the offsets do not hold; every lane looks up its own ten keys and loads to registers, a tile ahead.
// 4 tokens over 131071 keys: 119 us with 16 waves on a unit, of which the loads alone take 108 (5.5 TB/s) and all that is computed alone 78; loaded to registers, which leaves room for 12
// waves, 128, and 196 with addresses by vector instructions.  Three tiles on their way, and half the waves, are no faster.
enum Fp4Mode { ANY, WORDS, RING };
// Workgroups of four waves that run on a unit at a time, by the registers of a wave.  (ANY: two tiles are in registers.)
constexpr int on_unit(bool f32, int kd, int nb, Fp4Mode mode) {
  if (mode == ANY) return kd == 2 ? (nb == 1 && !f32 ? 3 : nb <= 2 ? 2 : 1) : kd < 8 && nb == 1 && !f32 ? 2 : 1;
  if (kd == 8) return mode == RING && !f32 ? 2 : 1;
  return nb > 1 ? 2 : f32 || (mode == WORDS && kd == 4) ? 3 : 4;
}
template <typename T, int KD_, int NB_, Fp4Mode MODE_, int WAVES_>
struct Fp4 {
  static constexpr int KD = KD_, NB = NB_;                                             // dwords of codes of a key per lane; columns of queries
  static constexpr Fp4Mode MODE = MODE_;
  static constexpr bool F32 = sizeof(T) == 4;
  // bf16 terms of a query's value, of a weight (the weights' sum takes them as they are, in fp32).  With a second term of the weights the error is that of rounding the result: heads of 128,
  // 1000 keys 2.0e-3 to 2.1e-3 with one, 1.65e-3 with two and for the exact result rounded.  It costs 1 to 9 % in up to two columns (one / two: a node each, 16 histories of 8000 keys 38.0 us / 38.6;
  // 8 nodes, 12 of 8000 42.7 / 46.6); in four, which its products bound, up to 15 (37 nodes, 12 of 8000 133.5 / 153.5, 100 of 500 100 / 113), and one is left there as in fi_tree_attention.
  static constexpr int QT = F32 ? 3 : 1, PT = F32 ? 3 : NB <= 2 ? 2 : 1;
  static constexpr int VW = KD == 8 ? 2 : 1, DT = KD == 2 ? 4 : 8 * VW;                // words of codes of a value row per lane; values in them
  static constexpr int KS = KD == 8 ? 2 : KD == 3 ? 3 : 1;                             // scales of a key per lane
  static constexpr int WAVES = WAVES_;
  // a tile in LDS: codes of keys, codes of values, scales of either (SB bytes a key; WORDS: four bytes a scale, PS times 64 of them a half); what a wave issues for it
  static constexpr int PS = KD == 8 ? 2 : 1, SB = KD == 8 ? 8 : 4, CODES = 512 * KD, SCALES = MODE == RING ? 32 * SB : 512 * PS, TILE = 2 * CODES + 2 * SCALES;
  static constexpr int LOADS = MODE == RING ? (KD == 8 ? 12 : 8) : 4 * (KD + PS), DEPTH = 2;
  // Queries of many columns are read from LDS, where all waves of a workgroup share them, and sums are joined by one column at a time: two workgroups find room on a unit then, and
  // with 256 registers the matrix instructions' sums stay where the vector unit reads them (one workgroup with 460 moved them back and forth, 290 of 960 instructions a tile; 100 trees of
  // 37 nodes, 32 heads on 8 of 128, over 500 keys 217 us, so 101; 12 over 8000 207 and 134; fp32, 16 on 4 of 72, 100 over 1000 201 and 108).  bf16 heads of 72 to 128 do not quite fit: 8 to 16 words a lane
  // go to scratch memory, of which tiles by words load 3 to 12 again each (heads of 72, 12 over 8000: 132, with one workgroup and nothing put aside 236; of 112 138 and 256).
  static constexpr bool SHARED = WAVES > 1 && KD <= 4 && NB == (F32 ? 2 : 4);
  static constexpr int COLUMNS = SHARED ? 1 : NB;                             // joined at a time
  static constexpr int JOIN = WAVES == 1 ? 16 : COLUMNS * (DT * 1024 + 512);   // a wave's sums
  static constexpr int TILES = WAVES * (MODE != ANY && DEPTH * TILE > JOIN ? DEPTH * TILE : JOIN), LDS = TILES + (SHARED ? NB * QT * KD * 1024 : 0);
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
};
template <typename F>
__device__ __forceinline__ void fp4_load_key(Fp4Tile<F>& t, int h, const Fp4Lane<F>& at, const uint8_t* codes, const uint8_t* scales) {
#pragma unroll
  for (int c = 0; c < F::KD; ++c) t.k[h][c] = *reinterpret_cast<const uint32_t*>(codes + at.k[c]);
#pragma unroll
  for (int c = 0; c < F::KS; ++c) t.ks[h][c] = scales[at.ks[c]];
}
template <typename F>
__device__ __forceinline__ void fp4_load_value(Fp4Tile<F>& t, int j, const Fp4Lane<F>& at, const uint8_t* codes, const uint8_t* scales) {
#pragma unroll
  for (int c = 0; c < F::VW; ++c) {
    const uint8_t* const p = codes + at.v[c];
    t.v[j][c] = F::DT == 4 ? (uint32_t)*reinterpret_cast<const uint16_t*>(p) : *reinterpret_cast<const uint32_t*>(p);
    t.vs[j][c] = scales[at.vs[c]];
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

// The same for fp32 queries, cut off where rounding would make an infinity of the largest numbers: fp32's 24 bits are three times eight, so the terms' sum is exact and none is
// larger than the value.
__device__ __forceinline__ void cut8(float (&x)[8], u32x4 (&w)[3]) {
#pragma unroll
  for (int t = 0; t < 3; ++t)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      w[t][i] = __builtin_amdgcn_perm(__float_as_uint(x[2 * i + 1]), __float_as_uint(x[2 * i]), 0x07060302u);
      x[2 * i] -= __uint_as_float(w[t][i] << 16);
      x[2 * i + 1] -= __uint_as_float(w[t][i] & 0xFFFF0000u);
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
template <typename F, typename Query, typename Visible>
__device__ __forceinline__ bool fp4_attend(Fp4State<F>& st, Query query, Fp4Tile<F>& t, float c, bool masked, Visible visible) {
  const int kq = (threadIdx.x & 63) >> 4;
  f32x4 s[F::NB][2];
  auto key_of = [&](int h, int w) {
    const float scale = scale_of(t.ks[h][F::KD == 8 ? w >> 2 : F::KD == 3 ? w : 0]);
    const uint32_t x = t.k[h][w];
    return u32x4{decode2<0>(x, scale), decode2<1>(x, scale), decode2<2>(x, scale), decode2<3>(x, scale)};
  };
#pragma unroll
  for (int nb = 0; nb < F::NB; ++nb) s[nb][0] = s[nb][1] = f32x4{0, 0, 0, 0};
  if constexpr (F::SHARED) {   // (a query's words are read once for both halves)
#pragma unroll
    for (int w = 0; w < F::KD; ++w) {
      const u32x4 key[2] = {key_of(0, w), key_of(1, w)};
#pragma unroll
      for (int nb = 0; nb < F::NB; ++nb)
#pragma unroll
        for (int term = F::QT - 1; term >= 0; --term) {
          const u32x4 q = query(nb, term, w);
          s[nb][0] = product16(key[0], q, s[nb][0]);
          s[nb][1] = product16(key[1], q, s[nb][1]);
        }
    }
  } else {
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int w = 0; w < F::KD; ++w) {
        const u32x4 key = key_of(h, w);
#pragma unroll
        for (int nb = 0; nb < F::NB; ++nb)
#pragma unroll
          for (int term = F::QT - 1; term >= 0; --term) s[nb][h] = product16(key, query(nb, term, w), s[nb][h]);
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
  // where a row of a page begins: in WHOLE pages by two scalar products of 32 bits (strides are below 2^31 there: checked on the host)
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
  // For both halves of a tile in whole pages: where their rows of codes and scales begin.
  template <typename Half>
  __device__ __forceinline__ void halves(int tile, Half half) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      int row;
      place(tile * 32 + 16 * h, row);
      const int p = clamp_int(page[h], 0, a.n_pages - 1);
      half(h, k + row_at(a.k_codes_strides, p, row), ks + row_at(a.k_scales_strides, p, row), v + row_at(a.v_codes_strides, p, row), vs + row_at(a.v_scales_strides, p, row));
    }
  }
  __device__ __forceinline__ void load(Fp4Tile<F>& t, int tile) {
    const int lane = threadIdx.x & 63, kq = lane >> 4, r = lane & 15;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int first = tile * 32 + 16 * h;
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
  __device__ __forceinline__ const uint8_t* value_scales(int key) const {
    int row;
    const int p = page_at(place(key, row));
    return vs + row_at(a.v_scales_strides, p, row);
  }
};

// A wave's ring.  RING: rows of a head are KD pieces of 16 bytes; keys lie in their order, values so that the four rows that lanes read at a time follow each other (row
// 4 k + i of a half at place 4 i + k): reads of 64 and 128 values meet no bank twice; of 256 pieces change places with the row, which leaves two at most.  WORDS: rows of codes, and of
// scales as words, one behind the other; lanes past the half's end bring its last words again, so that every tile is as many loads.
template <typename F>
struct Fp4Ring {
  static constexpr int KD = F::KD, PARTS = F::MODE == WORDS ? KD : KD == 8 ? 2 : 1;   // load instructions of half a tile's codes
  uint8_t* const base;
  uint32_t k[PARTS], v[PARTS], ks[F::PS], vs[F::PS];   // a lane's bytes from half a tile's first row: its pieces, its scales
  uint32_t key_at, value_at, key_scale, value_scale;   // where the lane reads
  uint32_t row_bytes, row_scales;                      // (WORDS) of a row in LDS
  static __device__ __forceinline__ int turn_k(int row) { return KD == 8 ? row & 7 : 0; }
  static __device__ __forceinline__ int turn_v(int place) { return KD == 8 ? (place >> 1 & 1) << 2 : 0; }
  __device__ __forceinline__ Fp4Ring(uint8_t* b, const fi_fp4_tree_attention_args& a) : base(b) {
    const int lane = threadIdx.x & 63, kq = lane >> 4, r = lane & 15;
    const uint32_t kt = (uint32_t)a.k_codes_strides[1], vt = (uint32_t)a.v_codes_strides[1], kst = (uint32_t)a.k_scales_strides[1], vst = (uint32_t)a.v_scales_strides[1];
    if constexpr (F::MODE == WORDS) {
      const int words = a.head_dim / 8, blocks = (a.head_dim + BLOCK - 1) / BLOCK;
      auto most = [](int x, int n) { return (uint32_t)(x < n ? x : n - 1); };
#pragma unroll
      for (int j = 0; j < PARTS; ++j) {
        const int piece = j * 64 + lane;
        const uint32_t row = most(piece / words, 16), c = 4 * most(piece - (int)row * words, words);
        k[j] = row * kt + c;
        v[j] = row * vt + c;
      }
#pragma unroll
      for (int j = 0; j < F::PS; ++j) {
        const int piece = j * 64 + lane;
        const uint32_t row = most(piece / blocks, 16), c = most(piece - (int)row * blocks, blocks);
        ks[j] = row * kst + c;
        vs[j] = row * vst + c;
      }
      row_bytes = 4 * words;
      row_scales = 4 * blocks;
      key_at = r * row_bytes;
      value_at = F::CODES + 4 * kq * row_bytes;
      key_scale = 2 * F::CODES + r * row_scales;
      value_scale = 2 * F::CODES + F::SCALES + 4 * kq * row_scales;
    } else {
#pragma unroll
      for (int j = 0; j < PARTS; ++j) {
        const int piece = j * 64 + lane, place = piece / KD & 15, c = piece % KD, row = 4 * (place & 3) + (place >> 2);
        k[j] = (uint32_t)place * kt + 16 * (c ^ turn_k(place));
        v[j] = (uint32_t)row * vt + 16 * (c ^ turn_v(place));
      }
      const int key = KD == 8 ? lane >> 1 & 15 : r, part = KD == 8 ? 4 * (lane & 1) : 0;
      ks[0] = (uint32_t)key * kst + part;
      vs[0] = (uint32_t)key * vst + part;
      key_at = KD == 8 ? r * 128 : r * 16 * KD + kq * 4 * KD;
      value_at = F::CODES + 16 * KD * kq;   // of place kq, the first of four
      key_scale = 2 * F::CODES + r * F::SB + (KD == 2 ? kq >> 1 : KD == 4 ? kq : 2 * kq);
      value_scale = 2 * F::CODES + 32 * F::SB + 4 * kq * F::SB;
    }
  }
  // Half h of tile number `slot` of the ring: rows from these addresses on.
  __device__ __forceinline__ void load(int slot, int h, const uint8_t* kc, const uint8_t* kss, const uint8_t* vc, const uint8_t* vss) const {
    const int lane = threadIdx.x & 63;
    uint8_t* const tile = base + slot * F::TILE;
    uint8_t *const codes = tile + h * (F::CODES / 2), *const scales = tile + 2 * F::CODES + h * (F::SCALES / 2);
    if constexpr (F::MODE == WORDS) {
#pragma unroll
      for (int j = 0; j < PARTS; ++j) {
        load_lds_off<4>(kc, k[j], codes + j * 256);
        load_lds_off<4>(vc, v[j], codes + F::CODES + j * 256);
      }
#pragma unroll
      for (int j = 0; j < F::PS; ++j) {
        load_lds_off<1>(kss, ks[j], scales + j * 256);
        load_lds_off<1>(vss, vs[j], scales + F::SCALES + j * 256);
      }
    } else {
      if (KD != 2 || lane < 32) {
#pragma unroll
        for (int j = 0; j < PARTS; ++j) {
          load_lds_off<16>(kc, k[j], codes + j * 1024);
          load_lds_off<16>(vc, v[j], codes + F::CODES + j * 1024);
        }
      }
      if (lane < (KD == 8 ? 32 : 16)) {
        load_lds_off<(KD == 2 ? 2 : 4)>(kss, ks[0], scales);
        load_lds_off<(KD == 2 ? 2 : 4)>(vss, vs[0], scales + F::SCALES);
      }
    }
  }
  __device__ __forceinline__ void read(Fp4Tile<F>& t, int slot, const Fp4Lane<F>& at) const {
    const int lane = threadIdx.x & 63, kq = lane >> 4, m = lane & 15, r = lane & 15;
    const uint8_t* const tile = base + slot * F::TILE;
    if constexpr (F::MODE == WORDS) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const uint8_t *const codes = tile + h * (F::CODES / 2), *const scales = tile + h * (F::SCALES / 2);
#pragma unroll
        for (int c = 0; c < KD; ++c) t.k[h][c] = *reinterpret_cast<const uint32_t*>(codes + key_at + at.k[c]);
#pragma unroll
        for (int c = 0; c < F::KS; ++c) t.ks[h][c] = scales[key_scale + 4 * at.ks[c]];
      }
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const uint8_t *const codes = tile + h * (F::CODES / 2), *const scales = tile + h * (F::SCALES / 2);
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int w = 0; w < F::VW; ++w) {
            const uint8_t* const row = codes + value_at + i * row_bytes + at.v[w];
            t.v[4 * h + i][w] = F::DT == 4 ? (uint32_t)*reinterpret_cast<const uint16_t*>(row) : *reinterpret_cast<const uint32_t*>(row);
            t.vs[4 * h + i][w] = scales[value_scale + i * row_scales + 4 * at.vs[w]];
          }
      }
    } else {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const uint8_t* const row = tile + h * (F::CODES / 2) + key_at;
        if constexpr (KD == 2) {
          const uint2 x = *reinterpret_cast<const uint2*>(row);
          t.k[h][0] = x.x, t.k[h][1] = x.y;
        } else {
#pragma unroll
          for (int c = 0; c < KD / 4; ++c) {
            const u32x4 x = *reinterpret_cast<const u32x4*>(KD == 8 ? row + 16 * ((2 * kq + c) ^ turn_k(r)) : row);
#pragma unroll
            for (int i = 0; i < 4; ++i) t.k[h][4 * c + i] = x[i];
          }
        }
        const uint8_t* const scales = tile + h * 16 * F::SB + key_scale;
        if constexpr (KD == 8) {
          const uint32_t x = *reinterpret_cast<const uint16_t*>(scales);
          t.ks[h][0] = x & 255, t.ks[h][1] = x >> 8;
        } else {
          t.ks[h][0] = *scales;
        }
      }
#pragma unroll
      for (int h = 0; h < 2; ++h) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const uint8_t* const row = tile + h * (F::CODES / 2) + value_at + i * 4 * 16 * KD;   // place 4 i + kq
#pragma unroll
          for (int w = 0; w < F::VW; ++w) {
            const int c = 4 * w + (m >> 2);
            if constexpr (KD == 2) t.v[4 * h + i][w] = *reinterpret_cast<const uint16_t*>(row + 2 * m);
            else t.v[4 * h + i][w] = *reinterpret_cast<const uint32_t*>(row + 16 * (c ^ turn_v(kq)) + 4 * (m & 3));
          }
        }
        u32x4 x[F::SB / 4];
#pragma unroll
        for (int w = 0; w < F::SB / 4; ++w) x[w] = reinterpret_cast<const u32x4*>(tile + h * 16 * F::SB + value_scale)[w];
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int w = 0; w < F::VW; ++w)
            t.vs[4 * h + i][w] = KD == 8 ? x[i >> 1][2 * (i & 1) + w] >> (8 * (m >> 2)) & 255 : x[0][i] >> (8 * (KD == 2 ? m >> 3 : m >> 2)) & 255;
      }
    }
  }
  // This wave's loads have arrived but for those of the `later` tiles asked for since (DEPTH - 1 at most).
  static __device__ __forceinline__ void wait(int later) {
    static_assert(F::DEPTH == 2, "a tile is on its way while one is worked on");
    if (later >= 1) arrived_but<F::LOADS>();
    else arrived_but<0>();
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
  // The first tile is on its way before the queries are asked for: loads come back in order, so who has waited for those has this.
  Fp4Walk<F> walk(a, w);
  const Fp4Ring<F> ring(smem + wave * F::DEPTH * F::TILE, a);
  int into = 0, from = 0;   // slots of the ring
  auto load_ring = [&](int t) {
    walk.halves(t, [&](int h, const uint8_t* kc, const uint8_t* kss, const uint8_t* vc, const uint8_t* vss) { ring.load(into, h, kc, kss, vc, vss); });
    into = into + 1 < F::DEPTH ? into + 1 : 0;
    if (t + 1 < t1) walk.ask(t + 1);
  };
  if constexpr (F::MODE != ANY)
    if (t0 < t1) {
      walk.ask(t0);
      load_ring(t0);
    }
  // the queries: values 8 (KD kq + c) .. of the lane's row of every column, as they are or in three terms; zeros past the head's end
  auto load_query = [&](int nb, u32x4 (&q)[F::QT][F::KD]) {
    const int node = mine(nb) / group, head = w.hk * group + mine(nb) % group;
    const T* const from = static_cast<const T*>(a.q) + (int64_t)(w.n0 + node) * a.q_strides[0] + head * a.q_strides[1];
#pragma unroll
    for (int c = 0; c < F::KD; ++c) {
      const int d = 8 * (F::KD * kq + c);
      float x[8] = {};
      if (d < D) load8(from + d, x);
      u32x4 terms[F::QT];
      if constexpr (F::F32) cut8(x, terms);
      else terms8<F::QT>(x, terms);
#pragma unroll
      for (int term = 0; term < F::QT; ++term) q[term][c] = terms[term];
    }
  };
  u32x4 q[F::SHARED ? 1 : NB][F::QT][F::KD];
  u32x4* const shared = reinterpret_cast<u32x4*>(smem + F::TILES) + lane;
  if constexpr (F::SHARED) {
    if (wave < NB) {
      load_query(wave, q[0]);
#pragma unroll
      for (int term = 0; term < F::QT; ++term)
#pragma unroll
        for (int c = 0; c < F::KD; ++c) shared[((wave * F::QT + term) * F::KD + c) * 64] = q[0][term][c];
    }
    __syncthreads();
  } else {
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) load_query(nb, q[nb]);
  }
  auto query = [&](int nb, int term, int w) {
    if constexpr (F::SHARED) return shared[((nb * F::QT + term) * F::KD + w) * 64];
    else return q[nb][term][w];
  };
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
    Fp4Tile<F> x;
    bool strange = false;
    auto attend = [&](Fp4Tile<F>& tile, int t) {
      strange |= fp4_attend<F>(st, query, tile, c, (t + 1) * 32 > w.cached, [&](int nb) { return visible(nb, t * 32); });
    };
    if constexpr (F::MODE != ANY) {
      // (a wait that the compiler puts before the queries' first use would wait for the ring's loads, too)
      if constexpr (!F::SHARED)
#pragma unroll
        for (int nb = 0; nb < NB; ++nb)
#pragma unroll
          for (int term = 0; term < F::QT; ++term)
#pragma unroll
            for (int i = 0; i < F::KD; ++i) asm volatile("" : "+v"(q[nb][term][i]));
      for (int t = t0; t < t1; ++t) {
        if (t + 1 < t1) load_ring(t + 1);   // (where the tile before this one was: it has been read)
        Fp4Ring<F>::wait(t1 - 1 - t);
        ring.read(x, from, walk.at);
        from = from + 1 < F::DEPTH ? from + 1 : 0;
        attend(x, t);
        arrived_but<63>();   // (reads of LDS only)
      }
    } else {
      Fp4Tile<F> y;
      auto load = [&](Fp4Tile<F>& tile, int t) {
        walk.load(tile, t);
        __builtin_amdgcn_sched_barrier(0);   // (they are on their way before the tile at hand is worked on)
      };
      load(x, t0);
      for (int t = t0; t < t1; t += 2) {
        if (t + 1 < t1) load(y, t + 1);
        attend(x, t);
        if (t + 1 >= t1) break;
        if (t + 2 < t1) load(x, t + 2);
        attend(y, t + 1);
      }
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
  // The waves' sums against the largest maximum, added in the order of the waves.  4 DT values of a row are the lane's: DT from DT (4 kq + i) on for each i < 4 (of KD 8: 8
  // of each half).  Wave i takes those; a wave alone takes all of its own.
  float* const sums = reinterpret_cast<float*>(smem) + lane;   // (element by element, so that reads of one element meet no bank twice)
  constexpr int COLUMNS = F::COLUMNS;
  float2* const stats = reinterpret_cast<float2*>(smem + WAVES * COLUMNS * DT * 1024) + lane;
  auto put = [&](int nb) {
    const int at = wave * COLUMNS + nb % COLUMNS;
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
      for (int i = 0; i < 4; ++i) sums[((at * DT + d) * 4 + i) * 64] = st.o[nb][d][i];
    stats[at * 64] = make_float2(st.top[nb], over_keys_sum(st.total[nb]));
  };
  if constexpr (WAVES > 1 && COLUMNS == NB) {
    if constexpr (F::MODE != ANY) __syncthreads();   // (they lie where other waves' tiles were)
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) put(nb);
    __syncthreads();
  }
#pragma unroll
  for (int nb = 0; nb < NB; ++nb) {
    if constexpr (WAVES > 1 && COLUMNS < NB) {
      __syncthreads();   // (where other waves' tiles were, or the column before)
      put(nb);
      __syncthreads();
    }
    float top = st.top[nb], total = 0.0f, factor[WAVES];
    if constexpr (WAVES > 1) {
      top = stats[nb % COLUMNS * 64].x;
#pragma unroll
      for (int x = 1; x < WAVES; ++x) top = fmaxf(top, stats[(x * COLUMNS + nb % COLUMNS) * 64].x);
      const float base = top == -INFINITY ? 0.0f : top;
#pragma unroll
      for (int x = 0; x < WAVES; ++x) {
        const float2 other = stats[(x * COLUMNS + nb % COLUMNS) * 64];
        factor[x] = __builtin_amdgcn_exp2f((other.x - base) * c);
        total += other.y * factor[x];
      }
    } else {
      total = over_keys_sum(st.total[nb]);
    }
    const float inv = w.splits > 1 ? 1.0f : total == 0.0f ? 0.0f : 1.0f / total;
    constexpr int N = DT < 8 ? DT : 8;
    const bool there = row_of(nb) < rows;
    const int node = mine(nb) / group, head = w.hk * group + mine(nb) % group;
    const int64_t row = (int64_t)(w.n0 + node) * a.q_heads + head;
    T* const out = static_cast<T*>(a.out) + (int64_t)(w.n0 + node) * a.out_strides[0] + head * a.out_strides[1];
    float* const part = part_sums(a, p, row, w.split);
#pragma unroll
    for (int i0 = 0; i0 < (WAVES > 1 ? 1 : 4); ++i0) {
      const int i = WAVES > 1 ? wave : i0;
#pragma unroll
      for (int e = 0; e < DT; e += N) {
        float v[N];
#pragma unroll
        for (int n = 0; n < N; ++n) v[n] = 0.0f;
#pragma unroll
        for (int n = 0; n < N; ++n) {
          if constexpr (WAVES == 1) v[n] = st.o[nb][e + n][i0];
          else
#pragma unroll
            for (int x = 0; x < WAVES; ++x) v[n] += sums[(((x * COLUMNS + nb % COLUMNS) * DT + e + n) * 4 + i) * 64] * factor[x];
        }
        const int d = (e >> 3) * 128 + (DT < 8 ? DT : 8) * (4 * kq + i);
        if (!there || d >= D) continue;
        if (w.splits > 1) {
#pragma unroll
          for (int n = 0; n < N; n += 4) *reinterpret_cast<float4*>(part + d + n) = make_float4(v[n], v[n + 1], v[n + 2], v[n + 3]);
        } else {
#pragma unroll
          for (int n = 0; n < N; n += 4) store4(out + d + n, v[n] * inv, v[n + 1] * inv, v[n + 2] * inv, v[n + 3] * inv);
        }
      }
    }
    if (w.splits > 1 && there && wave == 0 && kq == 0) *reinterpret_cast<float2*>(part_stats(a, p, row, w.split)) = make_float2(top, total);
  }
}

// What the kernels are compiled for.  (ANY: for two on a unit the compiler finds pages one after the other; 4 tokens over 32000 keys, 8 heads of 128, pages of 8: 93 us, so 70.)
template <typename T, int KD, int NB, Fp4Mode MODE> constexpr int ON_UNIT = MODE == ANY ? 1 : on_unit(sizeof(T) == 4, KD, NB, MODE);
template <typename T, int KD, int NB, Fp4Mode MODE, bool COUNTED>
__global__ void __launch_bounds__(256, (ON_UNIT<T, KD, NB, MODE>))
    fp4_tree_kernel(fi_fp4_tree_attention_args a, TreeSplit p) {
  using F = Fp4<T, KD, NB, MODE, 4>;
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
// A wave a workgroup, which has the whole history: many short ones.
template <typename T, int KD, int NB, Fp4Mode MODE>
__global__ void __launch_bounds__(64, (sizeof(T) == 2 && KD <= 4 && NB == 1 ? ON_UNIT<T, KD, NB, MODE> : 1)) fp4_small_kernel(fi_fp4_tree_attention_args a, TreeSplit p) {
  using F = Fp4<T, KD, NB, MODE, 1>;
  __shared__ __attribute__((aligned(16))) uint8_t smem[F::LDS];
  TreeWork w;
  if (tree_direct(a, p, w)) fp4_work<T, F>(a, w, p, smem);
}

template <typename T, int KD, int NB, Fp4Mode MODE>
int launch_fp4_tree(const fi_fp4_tree_attention_args& a, const Fp4Plan& p, hipStream_t s) {
  const TreeSplit t = {p.splits, p.least / 32, 32, 8, 16 * NB, p.packed ? 0 : p.blocks, p.header};
  const int64_t direct = p.packed ? p.packed : (int64_t)a.n_seqs * p.blocks, all_rows = a.nodes * a.q_heads;
  if (!p.counted && !one_launch(direct, p.small ? 64 : 256)) return kTooLarge;
  if (p.splits > 1 && !one_launch((all_rows + 3) / 4, 256)) return kTooLarge;
  const dim3 grid((uint32_t)direct, (uint32_t)a.kv_heads, (uint32_t)p.splits);
  if constexpr (NB <= 2)
    if (p.small) {
      fp4_small_kernel<T, KD, NB, MODE><<<grid, 64, 0, s>>>(a, t);
      return (int)hipGetLastError();
    }
  // (counted: as many workgroups as run at a time: 32 beams over up to 5001 keys, 1024 workgroups 20.3 us, 512 of them 21.1, 640, which share units unevenly, 22.7)
  if (p.counted) fp4_tree_kernel<T, KD, NB, MODE, true><<<dim3(256 * p.on_unit), 256, 0, s>>>(a, t);
  else fp4_tree_kernel<T, KD, NB, MODE, false><<<grid, 256, 0, s>>>(a, t);
  constexpr int PER = KD <= 2 ? 1 : KD <= 4 ? 2 : 4;
  if (p.splits > 16 && all_rows <= 1024) tree_join_kernel<fi_fp4_tree_attention_args, T, PER, true><<<dim3((uint32_t)all_rows), 256, 0, s>>>(a, t, p.counted);
  else if (p.splits > 1) tree_join_kernel<fi_fp4_tree_attention_args, T, PER, false><<<dim3((uint32_t)((all_rows + 3) / 4)), 256, 0, s>>>(a, t, p.counted);
  return (int)hipGetLastError();
}
template <typename T, int KD, int NB>
int launch_fp4_mode(const fi_fp4_tree_attention_args& a, const Fp4Plan& p, hipStream_t s) {
  const int64_t far = (1ll << 31) / 16 - 1024;
  bool whole = a.page_size % 16 == 0, ring = a.head_dim == 32 * KD;
  auto look = [&](const void* p, const int64_t* strides, int align) {
    whole = whole && strides[0] < 1ll << 31 && strides[1] < far;
    ring = ring && reinterpret_cast<uintptr_t>(p) % align == 0 && strides[0] % align == 0 && strides[1] % align == 0 && strides[2] % align == 0;
  };
  look(a.k_codes, a.k_codes_strides, 16);
  look(a.v_codes, a.v_codes_strides, 16);
  look(a.k_scales, a.k_scales_strides, KD == 2 ? 2 : 4);
  look(a.v_scales, a.v_scales_strides, KD == 2 ? 2 : 4);
  if constexpr (KD != 3)
    if (whole && ring) return launch_fp4_tree<T, KD, NB, RING>(a, p, s);
  return whole ? launch_fp4_tree<T, KD, NB, WORDS>(a, p, s) : launch_fp4_tree<T, KD, NB, ANY>(a, p, s);
}
template <typename T, int KD>
int launch_fp4_columns(const fi_fp4_tree_attention_args& a, const Fp4Plan& p, hipStream_t s) {
  if (p.nb == 1) return launch_fp4_mode<T, KD, 1>(a, p, s);
  if constexpr (KD < 8)
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
