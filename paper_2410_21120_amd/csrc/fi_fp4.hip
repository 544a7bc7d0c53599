// The paged cache of 4-bit values: the write of a step's keys and values, and attention of drafted trees over it.
//
// A value is an E2M1 code times its block's power of two.  CDNA4 converts two codes with their scale to two bf16 in one instruction, exactly (two significant
// bits), so keys and values enter the bf16 matrix instructions as they are held: nothing is left to apply to sums, whatever blocks a head has.
#include <hip/hip_runtime.h>

#include <type_traits>

#include "fi_device.h"
#include "fi_ops.h"
#include "fi_tree_device.h"

namespace fi {
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

// What a lane does with its eight values, four lanes (fewer in a head's last block) a block.  The smallest e with max <= 6 * 2^e: of max = 2^p * (1 + f) it is
// p - 2 where 1 + f <= 1.5, else p - 1.
template <typename T, bool VEC>
__device__ __forceinline__ void write8(const T* from, bool there, uint8_t* codes, uint8_t* scale, T* held, int sub) {
  float x[8];
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] = 0.0f;
  if (there) load8<VEC>(from, x);
#pragma unroll
  for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(x[i]) & 0x7FFFFFFFu);   // (of magnitudes; a NaN's is the largest)
  top = max(top, (uint32_t)__shfl_xor((int)top, 1));
  top = max(top, (uint32_t)__shfl_xor((int)top, 2));
  const bool finite = top < 0x7F800000u;
  const int e = clamp_int((int)(top >> 23) - 127 - ((top & 0x7FFFFFu) <= 0x400000u ? 2 : 1), -125, 125);
  const uint32_t b = finite ? (uint32_t)(e + 127) : NAN_SCALE;
  const float s = scale_of(finite ? b : 127);
  uint32_t w = 0;   // (rounds to nearest, ties to even codes, cuts to 6)
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[0], x[1], s, 0);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[2], x[3], s, 1);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[4], x[5], s, 2);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[6], x[7], s, 3);
  if (!finite) w = 0;
  if (!there) return;
  if (codes) {
    *reinterpret_cast<uint32_t*>(codes) = w;
    if (sub == 0) *scale = (uint8_t)b;
  }
  if (held) {
    const float r = scale_of(b);
    const u32x4 y = {decode2<0>(w, r), decode2<1>(w, r), decode2<2>(w, r), decode2<3>(w, r)};
    if constexpr (std::is_same<T, bf16_t>::value) {
      if constexpr (VEC) *reinterpret_cast<u32x4*>(held) = y;
      else
#pragma unroll
        for (int i = 0; i < 4; ++i) held[2 * i] = (bf16_t)(y[i] & 0xFFFFu), held[2 * i + 1] = (bf16_t)(y[i] >> 16);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) held[2 * i] = __uint_as_float(y[i] << 16), held[2 * i + 1] = __uint_as_float(y[i] & 0xFFFF0000u);
    }
  }
}

// A thread keeps its place in a token (key or value, head, eight values) and goes through the tokens, so it divides once.  per: places of a token.
template <typename T, bool VEC>
__global__ void __launch_bounds__(256) fp4_write_kernel(fi_fp4_cache_write_args a, int blocks, int per, int tokens_at_once) {
  const int at = blockIdx.y * 256 + threadIdx.x, ahead = at / per, place = at - ahead * per;
  if (ahead >= tokens_at_once) return;
  const int sub = place & 3, unit = place >> 2, row = unit / blocks, block = unit - row * blocks;   // row: key head, then value head
  const bool is_v = row >= a.kv_heads;
  const int h = is_v ? row - a.kv_heads : row, d = block * BLOCK + sub * 8;
  const bool there = d < a.head_dim;
  const T* const from = static_cast<const T*>(is_v ? a.v : a.k) + h * (is_v ? a.v_strides[1] : a.k_strides[1]) + d;
  T* const held = static_cast<T*>(is_v ? a.v_held : a.k_held);
  uint8_t* const codes = is_v ? a.v_codes : a.k_codes;
  uint8_t* const scales = is_v ? a.v_scales : a.k_scales;
  const int64_t in_token = is_v ? a.v_strides[0] : a.k_strides[0];
  const int64_t held_token = is_v ? a.v_held_strides[0] : a.k_held_strides[0], held_at = h * (is_v ? a.v_held_strides[1] : a.k_held_strides[1]) + d;
  const int64_t c0 = is_v ? a.v_codes_strides[0] : a.k_codes_strides[0], c1 = is_v ? a.v_codes_strides[1] : a.k_codes_strides[1];
  const int64_t s0 = is_v ? a.v_scales_strides[0] : a.k_scales_strides[0], s1 = is_v ? a.v_scales_strides[1] : a.k_scales_strides[1];
  const int64_t code_at = h * (is_v ? a.v_codes_strides[2] : a.k_codes_strides[2]) + d / 2, scale_at = h * (is_v ? a.v_scales_strides[2] : a.k_scales_strides[2]) + block;
  for (int64_t t = (int64_t)blockIdx.x * tokens_at_once + ahead; t < a.tokens; t += (int64_t)gridDim.x * tokens_at_once) {
    const int64_t slot = a.slots[t];
    const bool kept = slot >= 0 && slot < a.n_slots;
    const int64_t page = kept ? slot / a.page_size : 0, r = kept ? slot - page * a.page_size : 0;
    write8<T, VEC>(from + t * in_token, there, kept ? codes + page * c0 + r * c1 + code_at : nullptr, scales + page * s0 + r * s1 + scale_at,
                   held ? held + t * held_token + held_at : nullptr, sub);
  }
}

// ---------------------------------------------------------------------------------------------------
// Attention
// ---------------------------------------------------------------------------------------------------
// A wave has 16 NB queries (rows: node and head) as columns and keys of its own, 32 at a time: scores S^T = K Q^T, outputs O^T = V^T P^T, by 16 x 16 x 32 products.
// Lane l holds scores of query l & 15, of the keys 4 (l >> 4) + i and 16 + 4 (l >> 4) + i, i < 4, of a tile, and these registers are the operand of the second product
// as they stand: its lane l has to bring values of just these eight keys.  The reduction over a head's values may run in any order, so lane l brings the KD dwords
// of codes from KD (l >> 4) on, of key l & 15.  Values: DT of a head's, from DT (l & 15) on, of each of the eight keys; two keys' are paired by a byte permute.
// All loads go to registers, a tile ahead: lanes of a key read 64 bytes and more that follow each other.
template <typename T, int KD_, int NB_>
struct Fp4 {
  static constexpr int KD = KD_, NB = NB_;                                             // dwords of codes of a key per lane; columns of queries
  static constexpr bool F32 = sizeof(T) == 4;
  static constexpr int QT = F32 ? 3 : 1, PT = F32 ? 3 : NB <= 2 ? 2 : 1;               // bf16 terms of a query's value, of a weight
  static constexpr int VW = KD == 8 ? 2 : 1, DT = KD == 2 ? 4 : 8 * VW;                // words of codes of a value row per lane; values in them
  static constexpr int KS = KD == 8 ? 2 : KD == 3 ? 3 : 1;                             // scales of a key per lane
  static constexpr int WAVES = 4;
  static constexpr int LDS = WAVES * (NB * DT * 1024 + NB * 512);
};
struct Fp4Codes {
  const uint8_t *k, *ks, *v, *vs;   // the key head's part
};

template <typename F>
struct Fp4Tile {
  uint32_t k[2][F::KD], ks[2][F::KS], v[8][F::VW], vs[8][F::VW];
};

// Words of codes at `p`, aligned to four bytes only.
template <int N>
__device__ __forceinline__ void load_words(const uint8_t* p, uint32_t (&w)[N]) {
  typedef uint32_t vec __attribute__((ext_vector_type(N == 3 ? 4 : N), aligned(4)));
  if constexpr (N == 8) {
    typedef uint32_t vec4 __attribute__((ext_vector_type(4), aligned(4)));
    const vec4 x = reinterpret_cast<const vec4*>(p)[0], y = reinterpret_cast<const vec4*>(p)[1];
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = x[i], w[4 + i] = y[i];
  } else if constexpr (N == 4 || N == 2) {
    const vec x = *reinterpret_cast<const vec*>(p);
#pragma unroll
    for (int i = 0; i < N; ++i) w[i] = x[i];
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) w[i] = reinterpret_cast<const uint32_t*>(p)[i];
  }
}

// The lane's place in rows of codes, the same for every key.
template <typename F>
struct Fp4Lane {
  int k[F::KD], ks[F::KS], v[F::VW], vs[F::VW];
  bool whole;   // the lane's dwords of a key are in one piece (a head that KD dwords a lane fill)
  __device__ __forceinline__ explicit Fp4Lane(int D) {
    const int lane = threadIdx.x & 63, kq = lane >> 4, m = lane & 15, words = D / 8, blocks = (D + BLOCK - 1) / BLOCK;
    auto most = [](int x, int n) { return x < n ? x : n - 1; };
    whole = words == 4 * F::KD;
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
  if (at.whole) load_words<F::KD>(codes + at.k[0], t.k[h]);
  else
#pragma unroll
    for (int c = 0; c < F::KD; ++c) t.k[h][c] = *reinterpret_cast<const uint32_t*>(codes + at.k[c]);
#pragma unroll
  for (int c = 0; c < F::KS; ++c) t.ks[h][c] = scales[at.ks[c]];
}
template <typename F>
__device__ __forceinline__ void fp4_load_value(Fp4Tile<F>& t, int j, const Fp4Lane<F>& at, const uint8_t* codes, const uint8_t* scales) {
#pragma unroll
  for (int c = 0; c < F::VW; ++c) {
    t.v[j][c] = F::DT == 4 ? (uint32_t)*reinterpret_cast<const uint16_t*>(codes + at.v[c]) : *reinterpret_cast<const uint32_t*>(codes + at.v[c]);
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
  for (int w = 0; w < F::VW; ++w) {
    constexpr int PAIRS = F::DT == 4 ? 2 : 4;   // two values each, of a word
    uint32_t x[8][PAIRS];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float scale = scale_of(t.vs[j][w]);
      x[j][0] = decode2<0>(t.v[j][w], scale);
      x[j][1] = decode2<1>(t.v[j][w], scale);
      if constexpr (PAIRS == 4) {
        x[j][2] = decode2<2>(t.v[j][w], scale);
        x[j][3] = decode2<3>(t.v[j][w], scale);
      }
    }
#pragma unroll
    for (int u = 0; u < PAIRS; ++u)
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        u32x4 v;
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = __builtin_amdgcn_perm(x[2 * j + 1][u], x[2 * j][u], half ? 0x07060302u : 0x05040100u);
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

// Which keys' rows the lanes load.  WHOLE: pages hold a multiple of 16 keys, so the 16 keys of half a tile lie in one page, whose number is the wave's; else every
// lane looks up its own ten keys.  Keys past the last one read the place that they would have (there is one in its page), or the last key's page.
template <typename F, bool WHOLE>
struct Fp4Walk {
  const fi_fp4_tree_attention_args& a;
  const int32_t* table;
  Fp4Codes c;
  int keys, last_column;
  __device__ __forceinline__ Fp4Walk(const fi_fp4_tree_attention_args& args, const TreeWork& w) : a(args), table(args.block_table + w.b * args.table_stride), keys(w.keys) {
    c = Fp4Codes{args.k_codes + w.hk * args.k_codes_strides[2], args.k_scales + w.hk * args.k_scales_strides[2], args.v_codes + w.hk * args.v_codes_strides[2],
                 args.v_scales + w.hk * args.v_scales_strides[2]};
    last_column = (w.keys - 1) / args.page_size;
  }
  __device__ __forceinline__ int64_t page_at(int column) const { return clamp_int(table[column], 0, a.n_pages - 1); }
  __device__ __forceinline__ void load(Fp4Tile<F>& t, int tile, const Fp4Lane<F>& at) const {
    const int lane = threadIdx.x & 63, kq = lane >> 4, r = lane & 15;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int first = tile * 32 + 16 * h;
      if constexpr (WHOLE) {
        const int column = __builtin_amdgcn_readfirstlane(first / a.page_size), row = first - column * a.page_size;
        const int64_t page = __builtin_amdgcn_readfirstlane((int)page_at(column < last_column ? column : last_column));
        fp4_load_key<F>(t, h, at, c.k + page * a.k_codes_strides[0] + (row + r) * a.k_codes_strides[1], c.ks + page * a.k_scales_strides[0] + (row + r) * a.k_scales_strides[1]);
#pragma unroll
        for (int i = 0; i < 4; ++i)
          fp4_load_value<F>(t, 4 * h + i, at, c.v + page * a.v_codes_strides[0] + (row + 4 * kq + i) * a.v_codes_strides[1],
                            c.vs + page * a.v_scales_strides[0] + (row + 4 * kq + i) * a.v_scales_strides[1]);
      } else {
        auto find = [&](int key, int64_t& page, int& row) {
          key = key < keys ? key : keys - 1;
          const int column = key / a.page_size;
          row = key - column * a.page_size;
          page = page_at(column);
        };
        int64_t page;
        int row;
        find(first + r, page, row);
        fp4_load_key<F>(t, h, at, c.k + page * a.k_codes_strides[0] + row * a.k_codes_strides[1], c.ks + page * a.k_scales_strides[0] + row * a.k_scales_strides[1]);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          find(first + 4 * kq + i, page, row);
          fp4_load_value<F>(t, 4 * h + i, at, c.v + page * a.v_codes_strides[0] + row * a.v_codes_strides[1], c.vs + page * a.v_scales_strides[0] + row * a.v_scales_strides[1]);
        }
      }
    }
  }
  __device__ __forceinline__ const uint8_t* value_scales(int key) const {
    const int column = key / a.page_size;
    return c.vs + page_at(column) * a.v_scales_strides[0] + (key - column * a.page_size) * a.v_scales_strides[1];
  }
};

template <typename T, typename F, bool WHOLE>
__device__ __forceinline__ void fp4_work(const fi_fp4_tree_attention_args& a, const TreeWork& w, const TreeSplit& p, uint8_t* smem) {
  constexpr int NB = F::NB, DT = F::DT, WAVES = F::WAVES;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), kq = lane >> 4;
  const int D = a.head_dim, group = a.q_heads / a.kv_heads, rows = w.nodes * group, first = w.block * 16 * NB;
  if (first >= rows) return;
  auto share = [&](int x) { return w.t0 + (int)((int64_t)(w.t1 - w.t0) * x / WAVES); };
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
    const Fp4Lane<F> at(D);
    const Fp4Walk<F, WHOLE> walk(a, w);
    Fp4Tile<F> x, y;
    bool strange = false;
    auto attend = [&](Fp4Tile<F>& tile, int t) {
      strange |= fp4_attend<F>(st, q, tile, c, (t + 1) * 32 > w.cached, [&](int nb) { return visible(nb, t * 32); });
    };
    walk.load(x, t0, at);
    for (int t = t0; t < t1; t += 2) {
      if (t + 1 < t1) walk.load(y, t + 1, at);
      attend(x, t);
      if (t + 1 >= t1) break;
      if (t + 2 < t1) walk.load(x, t + 2, at);
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

template <typename T, int KD, int NB, bool WHOLE, bool COUNTED>
__global__ void __launch_bounds__(256, 1) fp4_tree_kernel(fi_fp4_tree_attention_args a, TreeSplit p) {
  using F = Fp4<T, KD, NB>;
  __shared__ __attribute__((aligned(16))) uint8_t smem[F::LDS];
  if constexpr (COUNTED) {
    __shared__ TreeLine line;
    line_up(a, p, line);
    along_the_line(a, p, line, [&](const TreeWork& w) {
      __syncthreads();   // (the piece before has been joined)
      fp4_work<T, F, WHOLE>(a, w, p, smem);
    });
  } else {
    TreeWork w;
    if (tree_direct(a, p, w)) fp4_work<T, F, WHOLE>(a, w, p, smem);
  }
}

// How a call is shared out, from its sizes alone (the workspace goes by it).
struct Fp4Plan { int kd, nb, blocks, splits, least, header; bool counted; int64_t packed; };
Fp4Plan plan_fp4(const fi_fp4_tree_attention_args& a) {
  Fp4Plan p;
  const int64_t nodes = a.max_nodes < a.nodes ? a.max_nodes : a.nodes, rows = nodes * (a.q_heads / a.kv_heads);
  p.kd = a.head_dim <= 64 ? 2 : a.head_dim <= 96 ? 3 : a.head_dim <= 128 ? 4 : 8;
  const int most = a.dtype == FI_F32 ? (p.kd == 8 ? 1 : 2) : p.kd == 8 ? 2 : 4;
  p.nb = rows <= 16 ? 1 : rows <= 32 || most < 4 ? (most < 2 ? most : 2) : 4;
  const int per_block = 16 * p.nb;
  p.blocks = (int)((rows + per_block - 1) / per_block);
  const int64_t streams = (int64_t)a.n_seqs * a.kv_heads, units = streams * p.blocks;
  auto some = [](int64_t n) { return n < 1 << 20 ? n : 1 << 20; };   // (products of two stay in 64 bits)
  auto parts = [&](int least) { return ((int64_t)a.max_length + least - 1) / least; };
  p.least = 128;
  const double line = (double)units * ((double)a.page_size * a.table_columns / 32 + 64);   // (tiles, beginnings)
  p.counted = a.n_seqs > 1 && a.n_seqs <= SEQS && parts(p.least) > 1 && some(units) * parts(p.least) > 256 && line < 2147483648.0;
  int64_t splits;
  if (p.counted) {
    p.least = 256;
    splits = (511 + (int64_t)a.kv_heads * p.blocks) / ((int64_t)a.kv_heads * p.blocks);
  } else {
    splits = units > 0 ? (1023 + units) / units : 1;
  }
  if (splits > parts(p.least)) splits = parts(p.least);
  const int64_t room = (64ll << 20) / ((int64_t)a.nodes * a.q_heads * (a.head_dim + 2) * 4 + 1);   // the workspace stays below 64 MB as far as the chip is full
  if (splits > room && splits * some(units) > 512) splits = room * some(units) > 512 ? room : (512 + units - 1) / units;
  p.splits = splits < 1 ? 1 : splits > 63 ? 63 : (int)splits;
  if (p.splits == 1) p.counted = false;
  if (p.counted) ++p.splits;   // (a stretch may begin and end inside a part)
  p.header = p.counted ? 4 + (a.n_seqs + 3) / 4 * 4 : 0;
  const int64_t packed = a.nodes * (a.q_heads / a.kv_heads) / per_block + a.n_seqs;
  p.packed = !p.counted && (int64_t)a.n_seqs * p.blocks > 4 * packed ? packed : 0;
  return p;
}

template <typename T, int KD, int NB, bool WHOLE>
int launch_fp4_tree(const fi_fp4_tree_attention_args& a, const Fp4Plan& p, hipStream_t s) {
  const TreeSplit t = {p.splits, p.least / 32, 32, 8, 16 * NB, p.packed ? 0 : p.blocks, p.header};
  const int64_t direct = p.packed ? p.packed : (int64_t)a.n_seqs * p.blocks, all_rows = a.nodes * a.q_heads;
  if (!p.counted && !one_launch(direct, 256)) return kTooLarge;
  if (p.splits > 1 && !one_launch((all_rows + 3) / 4, 256)) return kTooLarge;
  if (p.counted) fp4_tree_kernel<T, KD, NB, WHOLE, true><<<dim3(512), 256, 0, s>>>(a, t);
  else fp4_tree_kernel<T, KD, NB, WHOLE, false><<<dim3((uint32_t)direct, (uint32_t)a.kv_heads, (uint32_t)p.splits), 256, 0, s>>>(a, t);
  constexpr int PER = KD <= 2 ? 1 : KD <= 4 ? 2 : 4;
  if (p.splits > 16 && all_rows <= 1024) tree_join_kernel<fi_fp4_tree_attention_args, T, PER, true><<<dim3((uint32_t)all_rows), 256, 0, s>>>(a, t, p.counted);
  else if (p.splits > 1) tree_join_kernel<fi_fp4_tree_attention_args, T, PER, false><<<dim3((uint32_t)((all_rows + 3) / 4)), 256, 0, s>>>(a, t, p.counted);
  return (int)hipGetLastError();
}
template <typename T, int KD, int NB>
int launch_fp4_pages(const fi_fp4_tree_attention_args& a, const Fp4Plan& p, hipStream_t s) {
  return a.page_size % 16 == 0 ? launch_fp4_tree<T, KD, NB, true>(a, p, s) : launch_fp4_tree<T, KD, NB, false>(a, p, s);
}
template <typename T, int KD>
int launch_fp4_columns(const fi_fp4_tree_attention_args& a, const Fp4Plan& p, hipStream_t s) {
  if (p.nb == 1) return launch_fp4_pages<T, KD, 1>(a, p, s);
  if constexpr (sizeof(T) == 2 || KD < 8)
    if (p.nb == 2) return launch_fp4_pages<T, KD, 2>(a, p, s);
  if constexpr (sizeof(T) == 2 && KD < 8)
    if (p.nb == 4) return launch_fp4_pages<T, KD, 4>(a, p, s);
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

// Whether every row of a tensor starts on 16 bytes (counts as they are: a dimension of one may have any stride).
bool rows_on_16(const void* p, const int64_t* strides, int es) {
  return reinterpret_cast<uintptr_t>(p) % 16 == 0 && strides[0] * es % 16 == 0 && strides[1] * es % 16 == 0;
}

}  // namespace

int launch_fp4_cache_write(const fi_fp4_cache_write_args& a, void* stream) {
  const hipStream_t s = static_cast<hipStream_t>(stream);
  const int es = elem_size(a.dtype), blocks = (a.head_dim + BLOCK - 1) / BLOCK, per = (a.v ? 2 : 1) * a.kv_heads * blocks * 4;
  const bool vec = rows_on_16(a.k, a.k_strides, es) && (!a.v || rows_on_16(a.v, a.v_strides, es)) && (!a.k_held || rows_on_16(a.k_held, a.k_held_strides, es)) &&
                   (!a.v_held || rows_on_16(a.v_held, a.v_held_strides, es));
  const int at_once = per < 256 ? 256 / per : 1, ys = per < 256 ? 1 : (per + 255) / 256;
  const int64_t xs = ((int64_t)a.tokens + at_once - 1) / at_once, most = ys < 4096 ? (4096 + ys - 1) / ys : 1;
  const dim3 grid((uint32_t)(xs < most ? xs : most), (uint32_t)ys);
  if (a.dtype == FI_F32) {
    if (vec) fp4_write_kernel<float, true><<<grid, 256, 0, s>>>(a, blocks, per, at_once);
    else fp4_write_kernel<float, false><<<grid, 256, 0, s>>>(a, blocks, per, at_once);
  } else {
    if (vec) fp4_write_kernel<bf16_t, true><<<grid, 256, 0, s>>>(a, blocks, per, at_once);
    else fp4_write_kernel<bf16_t, false><<<grid, 256, 0, s>>>(a, blocks, per, at_once);
  }
  return (int)hipGetLastError();
}

uint64_t fp4_tree_workspace(const fi_fp4_tree_attention_args& a) {
  const Fp4Plan p = plan_fp4(a);
  return p.splits > 1 ? ((uint64_t)a.nodes * a.q_heads * p.splits * (a.head_dim + 2) + p.header) * 4 : 0;
}

int launch_fp4_tree_attention(const fi_fp4_tree_attention_args& a, void* stream) {
  const hipStream_t s = static_cast<hipStream_t>(stream);
  return a.dtype == FI_F32 ? launch_fp4_type<float>(a, s) : launch_fp4_type<bf16_t>(a, s);
}

}  // namespace fi
