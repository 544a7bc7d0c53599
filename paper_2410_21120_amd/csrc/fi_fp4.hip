// The paged cache of 4-bit values: the write of a step's keys and values, and attention over it for bf16 queries.
#include <hip/hip_runtime.h>

#include "fi_fp4_device.h"

namespace fi {
namespace {

// What a lane does with its eight values, four lanes (fewer in a head's last block) a block.  The smallest e with max <= 6 * 2^e: of max = 2^p * (1 + f) it is
// p - 2 where 1 + f <= 1.5, else p - 1.
template <typename T>
__device__ __forceinline__ void write8(const T* from, bool there, uint8_t* codes, uint8_t* scale, T* held, int sub) {
  float x[8];
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] = 0.0f;
  if (there) load8(from, x);
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
    typedef uint32_t piece __attribute__((ext_vector_type(4), aligned(sizeof(bf16_t))));
    if constexpr (sizeof(T) == 2) {
      *reinterpret_cast<piece*>(held) = piece{y[0], y[1], y[2], y[3]};
    } else {
      reinterpret_cast<piece*>(held)[0] = piece{y[0] << 16, y[0] & 0xFFFF0000u, y[1] << 16, y[1] & 0xFFFF0000u};
      reinterpret_cast<piece*>(held)[1] = piece{y[2] << 16, y[2] & 0xFFFF0000u, y[3] << 16, y[3] & 0xFFFF0000u};
    }
  }
}

// A thread keeps its place in a token (head, eight values) and goes through the tokens, those of an XCD's workgroups next to each other: rows of codes are often half a
// cache line.  per: places of a token.  What a thread works out before its first token is as much as a token's instructions, so no more workgroups start than run at a time
// (1472 tokens of 32 heads of 128: 8.8 us, twice as many workgroups 11.7; 16384 of 8 heads, with what is held, 35.4 and 36.6, 4.3 TB/s).
template <typename T>
__global__ void __launch_bounds__(256) fp4_write_kernel(fi_fp4_cache_write_args a, int blocks, int per, int tokens_at_once, uint32_t inv) {
  const int at = blockIdx.y * 256 + threadIdx.x, ahead = at / per, place = at - ahead * per;
  if (ahead >= tokens_at_once) return;
  const int sub = place & 3, unit = place >> 2, h = unit / blocks, block = unit - h * blocks, d = block * BLOCK + sub * 8;
  const bool is_v = blockIdx.z, there = d < a.head_dim;
  const int64_t *const in = is_v ? a.v_strides : a.k_strides, *const out = is_v ? a.v_held_strides : a.k_held_strides;
  const int64_t *const cs = is_v ? a.v_codes_strides : a.k_codes_strides, *const ss = is_v ? a.v_scales_strides : a.k_scales_strides;
  int64_t t = (int64_t)xcd_contiguous(blockIdx.x, gridDim.x) * tokens_at_once + ahead;
  const int64_t step = (int64_t)gridDim.x * tokens_at_once;
  const T* from = static_cast<const T*>(is_v ? a.v : a.k) + t * in[0] + h * in[1] + d;
  T* held = static_cast<T*>(is_v ? a.v_held : a.k_held);
  const bool hold = held != nullptr;
  held += t * out[0] + h * out[1] + d;
  uint8_t* const codes = (is_v ? a.v_codes : a.k_codes) + h * cs[2] + d / 2;
  uint8_t* const scales = (is_v ? a.v_scales : a.k_scales) + h * ss[2] + block;
  for (; t < a.tokens; t += step, from += step * in[0], held += step * out[0]) {
    const int64_t slot = a.slots[t];
    const bool kept = slot >= 0 && slot < a.n_slots;
    int64_t page = 0;
    uint32_t r = 0;
    if (a.n_slots <= 0xFFFFFFFFll) {   // (a quotient by inv, floor(2^32 / page size), is right or one too small)
      const uint32_t place = kept ? (uint32_t)slot : 0;
      uint32_t q = __umulhi(place, inv);
      r = place - q * (uint32_t)a.page_size;
      if (r >= (uint32_t)a.page_size) ++q, r -= (uint32_t)a.page_size;
      page = q;
    } else if (kept) {
      page = slot / a.page_size, r = (uint32_t)(slot - page * a.page_size);
    }
    write8<T>(from, there, kept ? codes + page * cs[0] + (int64_t)r * cs[1] : nullptr, scales + page * ss[0] + (int64_t)r * ss[1], hold ? held : nullptr, sub);
  }
}

}  // namespace

Fp4Plan plan_fp4(const fi_fp4_tree_attention_args& a) {
  Fp4Plan p;
  const int64_t nodes = a.max_nodes < a.nodes ? a.max_nodes : a.nodes, rows = nodes * (a.q_heads / a.kv_heads);
  p.kd = a.head_dim <= 64 ? 2 : a.head_dim <= 96 ? 3 : a.head_dim <= 128 ? 4 : 8;
  // (heads of 256: two columns leave room for one workgroup on a unit, one for two; 16 heads on 2, 16 nodes, 12 histories of 2000 keys 44.0 us and 37.2, 4 nodes, 100 of 2000 66.0 and 58.1)
  const int most = p.kd == 8 ? 1 : a.dtype == FI_F32 ? 2 : 4;
  p.nb = rows <= 16 ? 1 : rows <= 32 && most > 2 ? 2 : most;
  const int per_block = 16 * p.nb;
  p.blocks = (int)((rows + per_block - 1) / per_block);
  const int64_t streams = (int64_t)a.n_seqs * a.kv_heads, units = streams * p.blocks;
  // How tiles will be loaded, as sizes have it (strides and addresses may make words of pieces, or any of whole pages: the workspace is asked for before they are known).
  const Fp4Mode mode = a.page_size % 16 ? ANY : p.kd != 3 && a.head_dim == 32 * p.kd ? RING : WORDS;
  p.on_unit = on_unit(a.dtype == FI_F32, p.kd, p.nb, mode);
  auto some = [](int64_t n) { return n < 1 << 20 ? n : 1 << 20; };   // (products of two stay in 64 bits)
  auto parts = [&](int least) { return ((int64_t)a.max_length + least - 1) / least; };
  // Short histories: a wave for each, nothing to join (us, four waves / one; 8 heads of 128 in bf16, lengths up to 60: 4 sequences 7.4 / 6.1, 256 of them 14.6 / 8.6; 250: 10.5 / 11.8
  // and 22.4 / 18.7; 256 sequences of 32 heads of 72, 500: 113 / 92).
  p.small = p.nb <= 2 && (a.max_length <= 64 || (int64_t)a.max_length * 8 <= units);
  // Counted, where there is much to share out for what runs at a time and histories are long beside their number: where they are all as long that loses some microseconds, where they are
  // ragged it gains more (us, direct / counted, all as long and, r, spread over their logarithm. 8 heads of 128, a node each: 4 sequences of 32000 keys 33.4 / 37.3, r 30.4 / 24.3; 16 of 8000
  // 32.7 / 38.7, r 29.0 / 21.2; 256 of 2000 121 / 121, r 45.4 / 49.3. Eight nodes: 12 of 2000 28.7 / 29.3, r 18.2 / 19.4; of 4000 37.1 / 35.7, r 23.5 / 21.9; 100 of 1000 46.9 / 71.2,
  // r 27.6 / 42.2. 37 nodes: 2 of 2000 25.7 / 28.8, r 20.8 / 22.9; 12 of 2000 59 / 62, r 33 / 34; of 4000
  // 91 / 88, r 48 / 40.  Heads of 256, 4 nodes, 16 heads on 2: 12 of 4000 30.3 / 29.4,
  // r 18.1 / 17.5.  fp32, a node each, 32 heads on 8 of 128: 12 of 8000 31.8 / 36.9, r 23.1 / 23.1; 32 of 4000 39.1 / 45.7, r 33.8 / 24.2).
  // Pages of 8, 32 heads on 8 of 128: a node each, 12 of 2000 22.5 / 24.7, r 16.4 / 15.4; of 4000 37.6 / 34.4, r 24.3 / 19.2.  Eight nodes: 12 of 2000 45.0 / 49.9, r 27.5 / 20.5; 2 of 16000
  // 38.7 / 55.3, r 38.4 / 36.9; 4 of 32000 98 / 225, r 93 / 59.  37 nodes: 12 of 2000 163 / 146, r 56 / 48.  fp32, a node each: 12 of 4000 34 / 42, r 24 / 20; 4 of 32000 89 / 89, r 82 / 32.
  // Heads of 64, pages of 1, 37 nodes, 16 heads on 4: 2 of 2000 17.6 / 20.4, r 16.7 / 19.2; 4 of 4000 44.6 / 36.3, r 21.1 / 20.8.
  const int64_t much = 1024ll * (p.kd == 8 ? (p.on_unit == 1 ? 80 : 180) : p.on_unit == 4 ? 960 : p.on_unit == 3 || (p.on_unit == 1 && p.nb == 1) ? 640 : p.on_unit == 2 || p.nb < most ? 360 : 180);
  const double line = (double)units * ((double)a.page_size * a.table_columns / 32 + 64);   // (tiles, beginnings)
  p.counted = !p.small && a.n_seqs > 1 && a.n_seqs <= SEQS && some(units) * a.max_length >= much && a.max_length >= 2 * units && line < 2147483648.0;
  // Stretches: as many as run at a time.  Parts: as many as would with pieces of 16 bytes (for what does run they are fewer, and their last round is as likely to be a short one. Pages of 8, 32
  // heads on 8 of 128, so / for what runs: a node each, 12 of 2000 22.5 / 26.4, of 4000 37.6 / 39.1; eight nodes, 4 of 4000 29.3 / 23.4; fp32, a node each, 12 of 2000 23.2 / 28.1).
  const int64_t at_once = 256 * (p.counted ? p.on_unit : on_unit(a.dtype == FI_F32, p.kd, p.nb, RING));
  int64_t splits;
  if (p.counted) {
    p.least = 256;
    splits = (at_once - 1 + (int64_t)a.kv_heads * p.blocks) / ((int64_t)a.kv_heads * p.blocks);
  } else {
    // Parts of fewer keys where parts are few (2 sequences of 2000 keys, parts of 128 / 256: 10.2 us / 11.7; of 8000 14.5 / 12.7); below 384 keys a second launch costs more than it saves (250: 10.5, 8.5).
    p.least = some(units) * parts(128) > 256 ? 256 : 128;
    splits = a.max_length <= 384 || p.small || units == 0 ? 1 : (at_once - 1 + units) / units;
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

int launch_fp4_cache_write(const fi_fp4_cache_write_args& a, void* stream) {
  const hipStream_t s = static_cast<hipStream_t>(stream);
  const int blocks = (a.head_dim + BLOCK - 1) / BLOCK, per = a.kv_heads * blocks * 4, halves = a.v ? 2 : 1;
  const int at_once = per < 256 ? 256 / per : 1, ys = (per * at_once + 255) / 256;
  const int64_t xs = ((int64_t)a.tokens + at_once - 1) / at_once, most = (2048 + ys * halves - 1) / (ys * halves);   // what runs at a time
  const dim3 grid((uint32_t)(xs < most ? xs : most), (uint32_t)ys, (uint32_t)halves);
  const uint32_t inv = a.page_size == 1 ? ~0u : (uint32_t)((1ull << 32) / (uint32_t)a.page_size);
  if (a.dtype == FI_F32) fp4_write_kernel<float><<<grid, 256, 0, s>>>(a, blocks, per, at_once, inv);
  else fp4_write_kernel<bf16_t><<<grid, 256, 0, s>>>(a, blocks, per, at_once, inv);
  return (int)hipGetLastError();
}

uint64_t fp4_tree_workspace(const fi_fp4_tree_attention_args& a) {
  const Fp4Plan p = plan_fp4(a);
  return p.splits > 1 ? ((uint64_t)a.nodes * a.q_heads * p.splits * (a.head_dim + 2) + p.header) * 4 : 0;
}

int launch_fp4_tree_attention(const fi_fp4_tree_attention_args& a, void* stream) {
  const hipStream_t s = static_cast<hipStream_t>(stream);
  return a.dtype == FI_F32 ? launch_fp4_tree_f32(a, stream) : launch_fp4_type<bf16_t>(a, s);
}

}  // namespace fi
