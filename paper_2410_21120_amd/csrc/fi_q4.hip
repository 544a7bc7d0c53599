// Products of a few rows with 4-bit weights and group scales.
//
// y[m][n] = sum over groups of scale * sum of (q - zero) x.  Every weight is read once, so HBM bounds it as long as the rows are few.  The products run on the
// matrix cores, 16 rows x 16 outputs x 32 inputs an instruction.  A weight becomes bf16 in one operation and a share of a shift: 16 + q is the bit
// pattern 0x4180 | q << 3, two of them at a time, exact; sums of (16 + q) x and of x (the same instruction with ones) are kept in fp32 over a group,
// and (16 + zero) times the second comes off the first when the scale is applied.  fp32 rows are split into three bf16 terms
// (24 bits), so that they enter exactly, too (down to 1e-33: what is left for the third is subnormal then).
#include <hip/hip_runtime.h>

#include <type_traits>

#include "fi_device.h"
#include "fi_ops.h"
#include "fi_ops_device.h"

namespace fi {
namespace {

constexpr int ROWS = 8;   // rows that a wave of the row kernel has sums of

// One result, term by term as the formula says: what a kernel stores in place of a sum that is no finite number.  Sums of (16 + q) x overflow earlier than those of
// (q - zero) x, and an infinite x makes them NaN, where the formula may have an infinity or a number.  Rare, so it takes few registers and its time (us, without / with
// a row of NaN: 24 x 25088 x 4096 inputs x outputs 28 / 810, 1 x 4096 x 4096 4 / 105; the test for it: 24 rows 0.2, 5 rows of 4096 x 1000 0.07).
template <typename T>
__device__ __forceinline__ float q4_term_by_term(const fi_q4_matmul_args& a, int64_t m, int64_t n) {
  const uint8_t* w = a.w + n * a.w_stride;
  const T* x = static_cast<const T*>(a.x) + m * a.x_stride;
  float y = 0.0f;
#pragma unroll 1
  for (int g = 0; g < a.inputs / a.group; ++g) {
    const float scale = a.scales[n * a.scales_stride + g], zero = a.zeros ? (float)a.zeros[n * a.zeros_stride + g] : 8.0f;
#pragma unroll 1
    for (int k = 0; k < a.group; k += 8, w += 4, x += 8)
#pragma unroll
      for (int t = 0; t < 8; ++t) y += ((float)(w[t / 2] >> (t % 2 * 4) & 15) - zero) * scale * ld(x + t);
  }
  return y;
}
template <typename T>
__device__ __forceinline__ float q4_result(const fi_q4_matmul_args& a, int64_t m, int64_t n, float y) {
  return __builtin_isfinite(y) ? y : q4_term_by_term<T>(a, m, n);
}

// Any strides and alignment: one wave per output, a lane takes eight weights at a time.
template <typename T>
__global__ void __launch_bounds__(256) q4_row_kernel(fi_q4_matmul_args a) {
  const int lane = threadIdx.x & 63, n = blockIdx.x * 4 + (threadIdx.x >> 6);
  if (n >= a.outputs) return;
  const uint8_t* const w = a.w + n * a.w_stride;
  for (int m0 = 0; m0 < a.rows; m0 += ROWS) {
    float sum[ROWS] = {};
    for (int k = lane * 8; k < a.inputs; k += 512) {
      const int g = k / a.group;
      const float scale = a.scales[n * a.scales_stride + g], zero = a.zeros ? (float)a.zeros[n * a.zeros_stride + g] : 8.0f;
      float q[8];
#pragma unroll
      for (int t = 0; t < 8; ++t) q[t] = (float)((w[k / 2 + t / 2] >> (t % 2 * 4)) & 15) - zero;
#pragma unroll
      for (int m = 0; m < ROWS; ++m) {
        if (m0 + m >= a.rows) break;
        const T* const x = static_cast<const T*>(a.x) + (m0 + m) * a.x_stride + k;
        float part = 0.0f;   // (eight inputs lie in one group)
#pragma unroll
        for (int t = 0; t < 8; ++t) part += q[t] * ld(x + t);
        sum[m] += scale * part;
      }
    }
#pragma unroll
    for (int m = 0; m < ROWS; ++m) {
      if (m0 + m >= a.rows) break;
      float v = sum[m];
      for (int o = 32; o; o >>= 1) v += __shfl_xor(v, o);
      if (lane == 0) st(static_cast<T*>(a.out) + (m0 + m) * a.out_stride + n, q4_result<T>(a, m0 + m, n, v));
    }
  }
}

typedef float f32x4 __attribute__((ext_vector_type(4)));
constexpr int WAVES = 8;          // of a workgroup: they share its inputs, 128 at a time, and their sums are added in LDS
constexpr uint32_t ONES = 0x3F803F80u;

__device__ __forceinline__ f32x4 mfma16(const u32x4 a, const u32x4 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

// Eight rows' values as operands, in the order in which the weights of a dword come apart: 0 4 1 5 2 6 3 7.
__device__ __forceinline__ u32x4 weave(const u32x4 v) {
  return u32x4{__builtin_amdgcn_perm(v[2], v[0], 0x05040100u), __builtin_amdgcn_perm(v[2], v[0], 0x07060302u), __builtin_amdgcn_perm(v[3], v[1], 0x05040100u),
               __builtin_amdgcn_perm(v[3], v[1], 0x07060302u)};
}

template <typename T>
struct Run8;
template <>
struct Run8<bf16_t> {
  static constexpr int TERMS = 1;
  u32x4 v;
  __device__ __forceinline__ void load(const bf16_t* p, bool there) {
    v = u32x4{0, 0, 0, 0};
    if (there) v = *reinterpret_cast<const u32x4*>(p);
  }
  __device__ __forceinline__ void terms(u32x4 (&t)[1]) const { t[0] = weave(v); }
};
template <>
struct Run8<float> {
  static constexpr int TERMS = 3;
  float4 v[2];
  __device__ __forceinline__ void load(const float* p, bool there) {
    v[0] = v[1] = make_float4(0, 0, 0, 0);
    if (there) {
      v[0] = reinterpret_cast<const float4*>(p)[0];
      v[1] = reinterpret_cast<const float4*>(p)[1];
    }
  }
  // x = a + b + c with a, b, c in bf16: each takes eight bits of what is left
  __device__ __forceinline__ void terms(u32x4 (&t)[3]) const {
    const float* const f = &v[0].x;
#pragma unroll
    for (int p = 0; p < 4; ++p) {   // pair p: values p and p + 4
      float lo = f[p], hi = f[p + 4];
#pragma unroll
      for (int k = 0; k < 3; ++k) {
        const uint32_t both = pack_bf16x2(lo, hi);
        t[k][p] = both;
        lo -= __uint_as_float(both << 16);
        hi -= __uint_as_float(both & 0xFFFF0000u);
      }
    }
  }
};

// A workgroup computes 16 MB rows x 16 NB outputs over a share of the inputs (part `split` of `splits`).  A wave's step is 128 inputs; lane (q, i) = (lane / 16,
// lane % 16) holds, of output i of a block, VW dwords of weights in each of 4 / VW pieces: inputs 32 VW piece + 8 VW q .. + 8 VW of the step, all in one group,
// and of row i the same inputs.
template <typename T, int NB, int VW, int WAVES>
__global__ void __launch_bounds__(64 * WAVES, WAVES / 4) q4_tile_kernel(fi_q4_matmul_args a, uint32_t inv_group) {
  constexpr int MB = 1;
  constexpr int PIECES = 4 / VW, TERMS = Run8<T>::TERMS;
  __shared__ f32x4 sums[WAVES][MB * NB][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), q = lane >> 4, i = lane & 15;
  const int n0 = (int)blockIdx.x * 16 * NB, m0 = blockIdx.y * 16 * MB, K = a.inputs;
  const int steps = (K + 127) / 128, s0 = (int)((int64_t)steps * wave / WAVES), s1 = (int)((int64_t)steps * (wave + 1) / WAVES);
  struct Step {
    uint32_t w[NB][PIECES][VW];
    float scale[NB][PIECES];
    uint32_t zero[NB][PIECES];
    Run8<T> x[MB][4];
  };
  int n[NB];
  const T* x[MB];
#pragma unroll
  for (int b = 0; b < NB; ++b) n[b] = n0 + 16 * b + i < a.outputs ? n0 + 16 * b + i : a.outputs - 1;   // (past the last: once more, not stored)
#pragma unroll
  for (int b = 0; b < MB; ++b) x[b] = static_cast<const T*>(a.x) + (int64_t)(m0 + 16 * b + i) * a.x_stride;
  // k / group by a reciprocal (floor(2^32 / group): the quotient is right or one too small)
  auto group_of = [&](int k) {
    const uint32_t g = __umulhi((uint32_t)k, inv_group);
    return (int)(g + ((uint32_t)k - g * (uint32_t)a.group >= (uint32_t)a.group ? 1u : 0u));
  };
  auto load = [&](Step& s, int step) {
#pragma unroll
    for (int p = 0; p < PIECES; ++p) {
      const int k = step * 128 + p * 32 * VW;
      const bool inside = k < K;   // (a step at the end may be short by whole pieces)
      const int g = inside ? group_of(k) : 0;
#pragma unroll
      for (int b = 0; b < NB; ++b) {
        const uint8_t* const at = a.w + (int64_t)n[b] * a.w_stride + (inside ? (k >> 1) + 4 * VW * q : 0);
        if constexpr (VW == 4) *reinterpret_cast<u32x4*>(s.w[b][p]) = *reinterpret_cast<const u32x4*>(at);
        else if constexpr (VW == 2) *reinterpret_cast<u32x2*>(s.w[b][p]) = *reinterpret_cast<const u32x2*>(at);
        else s.w[b][p][0] = *reinterpret_cast<const uint32_t*>(at);
        s.scale[b][p] = a.scales[n[b] * a.scales_stride + g];
        s.zero[b][p] = a.zeros ? a.zeros[n[b] * a.zeros_stride + g] : 8u;
      }
#pragma unroll
      for (int b = 0; b < MB; ++b)
#pragma unroll
        for (int d = 0; d < VW; ++d) s.x[b][p * VW + d].load(x[b] + k + 8 * VW * q + 8 * d, inside && m0 + 16 * b + i < a.rows);
    }
  };
  f32x4 acc[MB][NB];
#pragma unroll
  for (int m = 0; m < MB; ++m)
#pragma unroll
    for (int b = 0; b < NB; ++b) acc[m][b] = f32x4{0, 0, 0, 0};
  Step now, next;
  if (s0 < s1) load(next, s0);
  for (int step = s0; step < s1; ++step) {
    now = next;
    if (step + 1 < s1) load(next, step + 1);
#pragma unroll
    for (int p = 0; p < PIECES; ++p) {
      f32x4 dot[MB][NB], all[MB];
#pragma unroll
      for (int m = 0; m < MB; ++m) {
        all[m] = f32x4{0, 0, 0, 0};
#pragma unroll
        for (int b = 0; b < NB; ++b) dot[m][b] = f32x4{0, 0, 0, 0};
      }
#pragma unroll
      for (int d = 0; d < VW; ++d) {
        u32x4 v[MB][TERMS];
#pragma unroll
        for (int m = 0; m < MB; ++m) {
          now.x[m][p * VW + d].terms(v[m]);
#pragma unroll
          for (int t = 0; t < TERMS; ++t) all[m] = mfma16(v[m][t], u32x4{ONES, ONES, ONES, ONES}, all[m]);
        }
#pragma unroll
        for (int b = 0; b < NB; ++b) {
          const uint32_t w = now.w[b][p][d];
          const u32x4 f = {(w << 3 & 0x00780078u) | 0x41804180u, (w >> 1 & 0x00780078u) | 0x41804180u, (w >> 5 & 0x00780078u) | 0x41804180u, (w >> 9 & 0x00780078u) | 0x41804180u};
#pragma unroll
          for (int m = 0; m < MB; ++m)
#pragma unroll
            for (int t = 0; t < TERMS; ++t) dot[m][b] = mfma16(v[m][t], f, dot[m][b]);
        }
      }
#pragma unroll
      for (int b = 0; b < NB; ++b) {
        const float scale = now.scale[b][p], zero = 16.0f + (float)now.zero[b][p];
#pragma unroll
        for (int m = 0; m < MB; ++m)
#pragma unroll
          for (int e = 0; e < 4; ++e) acc[m][b][e] += scale * (dot[m][b][e] - zero * all[m][e]);
      }
    }
  }
  // the waves' sums, added in their order: thread by thread one run of four rows of an output
#pragma unroll
  for (int m = 0; m < MB; ++m)
#pragma unroll
    for (int b = 0; b < NB; ++b) sums[wave][m * NB + b][lane] = acc[m][b];
  __syncthreads();
  for (int u = wave; u < MB * NB; u += WAVES) {
    f32x4 y = sums[0][u][lane];
#pragma unroll
    for (int v = 1; v < WAVES; ++v) y += sums[v][u][lane];
    const int col = n0 + 16 * (u % NB) + i, row = m0 + 16 * (u / NB) + 4 * q;
    if (col >= a.outputs) continue;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if (row + e >= a.rows) continue;
      st(static_cast<T*>(a.out) + (row + e) * a.out_stride + col, q4_result<T>(a, row + e, col, y[e]));
    }
  }
}

// Few rows: the vector unit.  A lane has 32 inputs at a time, 16 bytes of weights of each of OUTS outputs, all in one group; M rows.  The rows' inputs come
// through LDS, in the order in which the lanes want them, together with their sums (a lane's own 64 bytes of a row, loaded as they lie, touch a
// line per lane and load: twice the time).  bf16 weights come two by two as above and are multiplied two by two (v_dot2); fp32 rows
// take them as numbers.  WK waves share an output's inputs, each 2048 of a chunk.
typedef __attribute__((__vector_size__(2 * sizeof(__bf16)))) __bf16 bf16x2;
__device__ __forceinline__ float dot2(uint32_t a, uint32_t b, float c) { return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, a), __builtin_bit_cast(bf16x2, b), c, false); }
template <typename T, int M, int OUTS, int WK>
__global__ void __launch_bounds__(256) q4_few_kernel(fi_q4_matmul_args a, uint32_t inv_group) {
  constexpr bool F32 = sizeof(T) == 4;
  constexpr int NX = F32 ? 2 : 1, CHUNK = WK * 2048;   // 16-byte pieces of eight inputs; inputs of a chunk
  __shared__ u32x4 xs[M * WK * 4 * NX * 64];           // [row][part][eighth d of a lane's 32][half of it][lane]
  __shared__ float sums[M * WK * 64];                  // [row][part][lane]
  __shared__ float parts[4][OUTS * M];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, m0 = blockIdx.y * M, K = a.inputs;
  const int n0 = ((int)blockIdx.x * (4 / WK) + wave / WK) * OUTS, part = wave % WK;
  const uint8_t* w[OUTS];
  const float* scales[OUTS];
  const uint8_t* zeros[OUTS];
#pragma unroll
  for (int o = 0; o < OUTS; ++o) {
    const int64_t n = n0 + o < a.outputs ? n0 + o : a.outputs - 1;   // (past the last: once more, not stored)
    w[o] = a.w + n * a.w_stride;
    scales[o] = a.scales + n * a.scales_stride;
    zeros[o] = a.zeros ? a.zeros + n * a.zeros_stride : nullptr;
  }
  const T* x[M];
#pragma unroll
  for (int m = 0; m < M; ++m) x[m] = static_cast<const T*>(a.x) + (int64_t)(m0 + m < a.rows ? m0 + m : a.rows - 1) * a.x_stride;
  struct Chunk {
    u32x4 q[OUTS], x[M][WK][NX];
    float scale[OUTS];
    uint32_t zero[OUTS];
  };
  auto load = [&](Chunk& c, int from) {   // inputs past the end: zeros, times the row's first weights
    const int mine = from + (part * 64 + lane) * 32, k = mine < K ? mine : 0;
    uint32_t g = __umulhi((uint32_t)k, inv_group);   // k / group: right or one too small
    g += (uint32_t)k - g * (uint32_t)a.group >= (uint32_t)a.group ? 1u : 0u;
#pragma unroll
    for (int o = 0; o < OUTS; ++o) {
      c.q[o] = *reinterpret_cast<const u32x4*>(w[o] + (k >> 1));
      c.scale[o] = scales[o][g];
      c.zero[o] = zeros[o] ? zeros[o][g] : 8u;
    }
#pragma unroll
    for (int m = 0; m < M; ++m)
#pragma unroll
      for (int j = 0; j < WK; ++j) {
        const int kx = from + j * 2048 + tid * 8;
#pragma unroll
        for (int u = 0; u < NX; ++u) c.x[m][j][u] = kx < K ? reinterpret_cast<const u32x4*>(x[m] + kx)[u] : u32x4{0, 0, 0, 0};
      }
  };
  float acc[OUTS][M];
#pragma unroll
  for (int o = 0; o < OUTS; ++o)
#pragma unroll
    for (int m = 0; m < M; ++m) acc[o][m] = 0.0f;
  Chunk c;
  load(c, 0);
  for (int from = 0; from < K; from += CHUNK) {
#pragma unroll
    for (int m = 0; m < M; ++m)
#pragma unroll
      for (int j = 0; j < WK; ++j) {   // thread t has piece t % 4 of lane t / 4
        float sum = 0.0f;
        u32x4* const at = xs + (((m * WK + j) * 4 + (tid & 3)) * NX) * 64 + (tid >> 2);
        if constexpr (F32) {
#pragma unroll
          for (int t = 0; t < 8; ++t) sum += __uint_as_float(c.x[m][j][t / 4][t % 4]);
          at[0] = c.x[m][j][0];
          at[64] = c.x[m][j][1];
        } else {
#pragma unroll
          for (int t = 0; t < 4; ++t) sum = dot2(c.x[m][j][0][t], ONES, sum);
          at[0] = weave(c.x[m][j][0]);
        }
        sum += __shfl_xor(sum, 1);
        sum += __shfl_xor(sum, 2);
        if ((tid & 3) == 0) sums[(m * WK + j) * 64 + (tid >> 2)] = sum;
      }
    __syncthreads();
    u32x4 q[OUTS];
    float scale[OUTS], zero[OUTS], dot[OUTS][M];
#pragma unroll
    for (int o = 0; o < OUTS; ++o) {
      q[o] = c.q[o];
      scale[o] = c.scale[o];
      zero[o] = (F32 ? 0.0f : 16.0f) + (float)c.zero[o];
#pragma unroll
      for (int m = 0; m < M; ++m) dot[o][m] = 0.0f;
    }
    if (from + CHUNK < K) load(c, from + CHUNK);
#pragma unroll
    for (int d = 0; d < 4; ++d) {
      u32x4 v[M][NX];
#pragma unroll
      for (int m = 0; m < M; ++m)
#pragma unroll
        for (int u = 0; u < NX; ++u) v[m][u] = xs[(((m * WK + part) * 4 + d) * NX + u) * 64 + lane];
#pragma unroll
      for (int o = 0; o < OUTS; ++o) {
        if constexpr (F32) {
          const uint32_t low = q[o][d] & 0x0F0F0F0Fu, high = q[o][d] >> 4 & 0x0F0F0F0Fu;
#pragma unroll
          for (int t = 0; t < 8; ++t) {
            const float f = (float)(((t & 1 ? high : low) >> (8 * (t >> 1))) & 255u);
#pragma unroll
            for (int m = 0; m < M; ++m) dot[o][m] = __builtin_fmaf(f, __uint_as_float(v[m][t / 4][t % 4]), dot[o][m]);
          }
        } else {
#pragma unroll
          for (int t = 0; t < 4; ++t) {
            const uint32_t f = ((t == 0 ? q[o][d] << 3 : q[o][d] >> (4 * t - 3)) & 0x00780078u) | 0x41804180u;
#pragma unroll
            for (int m = 0; m < M; ++m) dot[o][m] = dot2(v[m][0][t], f, dot[o][m]);
          }
        }
      }
    }
#pragma unroll
    for (int m = 0; m < M; ++m) {
      const float all = sums[(m * WK + part) * 64 + lane];
#pragma unroll
      for (int o = 0; o < OUTS; ++o) acc[o][m] += scale[o] * (dot[o][m] - zero[o] * all);
    }
    __syncthreads();
  }
  // Sums over the lanes: at every step a lane hands half of its values to the lane opposite and takes that one's other half, until it has one.
  constexpr int V = OUTS * M;
  float v[V];
#pragma unroll
  for (int o = 0; o < OUTS; ++o)
#pragma unroll
    for (int m = 0; m < M; ++m) v[o * M + m] = acc[o][m];
  int h = 32;
#pragma unroll
  for (int left = V / 2; left >= 1; left /= 2, h /= 2) {
    const bool upper = (lane & h) != 0;
#pragma unroll
    for (int u = 0; u < left; ++u) {
      const float keep = upper ? v[u + left] : v[u], give = upper ? v[u] : v[u + left];
      v[u] = keep + __shfl_xor(give, h);
    }
  }
  for (; h; h /= 2) v[0] += __shfl_xor(v[0], h);
  if (lane % (64 / V) == 0) parts[wave][lane / (64 / V)] = v[0];
  __syncthreads();
  // the WK waves' sums, in their order
  if (part || lane >= V) return;
  float y = parts[wave][lane];
#pragma unroll
  for (int v = 1; v < WK; ++v) y += parts[wave + v][lane];
  const int n = n0 + lane / M, m = m0 + lane % M;
  if (n < a.outputs && m < a.rows) st(static_cast<T*>(a.out) + m * a.out_stride + n, q4_result<T>(a, m, n, y));
}

// More rows: a workgroup computes 16 MB rows x 256 outputs over a share of the inputs, 128 at a time.  Everything comes into LDS by direct loads, AHEAD
// steps ahead: each wave's weights (32 outputs) and their scales and zero points for itself, of the rows a share each, which it weaves and sums by groups a step
// before they are used.  What the zero points take off, scale * (16 + zero) * (sum of the group's x), is a product of its own over the groups: an fp32 matrix
// instruction takes four of them, once a chunk.  The vector unit bounds it about as much as HBM (64 operations a step to unpack 2 KB of weights, 16 MB for the groups' scales).
// GP: groups in a step (1: groups of 128 inputs and multiples).  Scales and zero points come in chunks of CS steps, so that a load takes pieces of rows
// (two values of 32 rows at a time cost 7 of 37 us): every step brings S of the instructions that fill the chunk after its own.
// fp32 rows: each eight inputs are woven as three bf16 terms, which meet the weights one after the other; 16 rows a workgroup.
template <typename T, int MB, int GP>
struct Wide {
  static constexpr int TERMS = Run8<T>::TERMS;
  static constexpr int S = GP == 4 ? 2 : 1, CS = GP == 4 ? 1 : 4, GC = GP * CS;            // (a chunk's groups: 8 of 64 inputs, else 4)
  static constexpr int CHUNK = 32 * GC * 4, CHUNKS = GP == 4 ? 6 : 3;                       // of a wave: as much for scales as for zero points
  static constexpr int WSTEP = WAVES * 2048, XSTEP = MB * 2048 * (int)sizeof(T), WOVEN_STEP = TERMS * MB * 4096, SUMS = GC * 16 * MB * 4;   // a step's weights, its rows, woven; a chunk's sums of the rows
  static constexpr int LEFT = 160 * 1024 - CHUNKS * WAVES * 2 * CHUNK - 2 * WOVEN_STEP - 2 * SUMS + XSTEP, MOST = LEFT / (WSTEP + XSTEP);
  static constexpr int BUFS = MOST < 5 ? MOST : 5, AHEAD = BUFS - 1, L = 3 + 2 * S;         // L: loads of a wave in a step, its rows' first
  // in LDS: AHEAD + 1 steps of weights, AHEAD of rows as they come, two of woven rows, two chunks' sums, the waves' chunks
  static constexpr int X = BUFS * WSTEP, WOVEN = X + AHEAD * XSTEP, ALL = WOVEN + 2 * WOVEN_STEP, SCALES = ALL + 2 * SUMS, BYTES = SCALES + CHUNKS * WAVES * 2 * CHUNK;
  static_assert(BUFS >= 3 && (TERMS == 1 || MB == 1) && AHEAD * L < 64 && (CS - 1 + AHEAD) / CS + 1 < CHUNKS, "waits can be counted; the chunk in use is not loaded over");
};
template <int CTRL>
__device__ __forceinline__ float swapped(float v) {   // of another lane of the row of 16
  return __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(v), CTRL, 0xF, 0xF, true));
}
template <typename T, int MB, int GP>
__global__ void __launch_bounds__(64 * WAVES, 1) q4_wide_kernel(fi_q4_matmul_args a, int splits, int per_group) {
  using Z = Wide<T, MB, GP>;
  constexpr bool F32 = sizeof(T) == 4;
  constexpr int TERMS = Z::TERMS;
  constexpr int AHEAD = Z::AHEAD, GC = Z::GC, CS = Z::CS;
  __shared__ __attribute__((aligned(1024))) uint8_t smem[Z::BYTES];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), q = lane >> 4, i = lane & 15, K = a.inputs;
  const int split = blockIdx.x % splits, n0 = (int)(blockIdx.x / splits) * 32 * WAVES + 32 * wave, m0 = blockIdx.y * 16 * MB;
  const uint32_t steps = (K + 127) / 128, s0 = (uint32_t)((uint64_t)steps * split / splits), s1 = (uint32_t)((uint64_t)steps * (split + 1) / splits);
  const int last = a.outputs - 1, groups = K / a.group;
  // What this lane loads: weights of two outputs (past the last one: the last once more, not stored), a piece of a row, a scale and a zero point or two.  All
  // from bases that the wave shares (the strides are below 2^24 elements).
  const int first_n = n0 < last ? n0 : last, left_n = last - first_n;
  const int piece_w = (lane & 3) ^ (q & 3), share = F32 ? wave : wave & (4 * MB - 1);
  const int row_x = F32 ? 2 * wave + (lane >> 5) : 4 * share + q, piece_x = F32 ? lane & 31 : i ^ (row_x & 15);
  const uint8_t* const w = a.w + (int64_t)first_n * a.w_stride;
  const float* const scale0 = a.scales + (int64_t)first_n * a.scales_stride;
  const uint8_t* const zero0 = a.zeros ? a.zeros + (int64_t)first_n * a.zeros_stride : nullptr;
  uint32_t off_w[2];
#pragma unroll
  for (int b = 0; b < 2; ++b) {
    const int n = 16 * b + (lane >> 2);
    off_w[b] = (uint32_t)(n < left_n ? n : left_n) * (uint32_t)a.w_stride + 16 * piece_w;
  }
  const int left_m = a.rows - 1 - m0;
  const T* const x = static_cast<const T*>(a.x) + (int64_t)m0 * a.x_stride;
  const uint32_t off_x = (uint32_t)(row_x < left_m ? row_x : left_m) * (uint32_t)a.x_stride * (uint32_t)sizeof(T) + 16 * piece_x;
  uint8_t* const own = smem + Z::SCALES + wave * Z::CHUNKS * 2 * Z::CHUNK;   // the wave's chunks
  // instruction `part` of a chunk (64 / GC rows of it), into buffer `to`
  constexpr int PARTS = GC / 2;
  auto load_scales = [&](uint32_t chunk, uint32_t part, uint32_t to) {
    const int row = (int)part * (64 / GC) + lane / GC, n = row < left_n ? row : left_n;
    const int first = (int)(GP > 1 ? chunk * GC : chunk * CS / (uint32_t)per_group), g = first + lane % GC < groups ? first + lane % GC : groups - 1;
    uint8_t* const at = own + to * 2 * Z::CHUNK + part * 256;
    load_lds_off<4>(scale0, (__umul24(n, (uint32_t)a.scales_stride) + g) * 4, at);
    if (zero0) load_lds_off<1>(zero0, __umul24(n, (uint32_t)a.zeros_stride) + g, at + Z::CHUNK);
    else load_lds_off<1>(scale0, 0, at + Z::CHUNK);   // (not looked at)
  };
  uint32_t slot = 0, slot_x = 0, to = (s0 / CS + 1) % Z::CHUNKS;   // of the next step to load: its slots, the buffer of the chunk after its own
  auto load = [&](uint32_t step) {
    uint8_t* const at = smem + slot * Z::WSTEP + wave * 2048;
    uint8_t* const at_x = smem + Z::X + slot_x * Z::XSTEP + share * 1024;
    const int k = (int)step * 128;
    if (k + 128 <= K) {
      load_lds_off<16>(x + k, off_x, at_x);
#pragma unroll
      for (int b = 0; b < 2; ++b) load_lds_off<16>(w + (k >> 1), off_w[b], at + b * 1024);
    } else {   // pieces past the end of the inputs: the step's first once more, not multiplied
      load_lds_off<16>(x + k, off_x - (k + 16 / (int)sizeof(T) * piece_x < K ? 0 : 16 * piece_x), at_x);
#pragma unroll
      for (int b = 0; b < 2; ++b) load_lds_off<16>(w + (k >> 1), off_w[b] - (k + 32 * piece_w < K ? 0 : 16 * piece_w), at + b * 1024);
    }
#pragma unroll
    for (int u = 0; u < Z::S; ++u) load_scales(step / CS + 1, (step % CS * Z::S + u) % PARTS, to);
    slot = slot + 1 < Z::BUFS ? slot + 1 : 0;
    slot_x = slot_x + 1 < AHEAD ? slot_x + 1 : 0;
    if ((step + 1) % CS == 0) to = to + 1 < Z::CHUNKS ? to + 1 : 0;
  };
  // The wave's own share of a step's rows (which it loaded itself), for all: woven, and summed by groups.
  uint32_t raw = 0;
  auto weave_step = [&](uint32_t step) {
    const uint8_t* const from_raw = smem + Z::X + raw * Z::XSTEP + share * 1024;
    uint8_t* const to_woven = smem + Z::WOVEN + (step & 1) * Z::WOVEN_STEP;
    if (F32 ? lane < 32 : wave < 4 * MB) {
      float sum;
      int row = row_x, octet = piece_x;
      if constexpr (F32) {   // a lane has eight inputs of one of the wave's two rows
        row = 2 * wave + q;
        octet = i;
        Run8<float> v;
        v.v[0] = reinterpret_cast<const float4*>(from_raw + q * 512 + i * 32)[0];
        v.v[1] = reinterpret_cast<const float4*>(from_raw + q * 512 + i * 32)[1];
        u32x4 terms[TERMS];
        v.terms(terms);
#pragma unroll
        for (int t = 0; t < TERMS; ++t) *reinterpret_cast<u32x4*>(to_woven + t * 4096 + row * 256 + ((i ^ row) << 4)) = terms[t];
        sum = (v.v[0].x + v.v[0].y) + (v.v[0].z + v.v[0].w) + ((v.v[1].x + v.v[1].y) + (v.v[1].z + v.v[1].w));
      } else {
        const u32x4 v = *reinterpret_cast<const u32x4*>(from_raw + lane * 16);
        *reinterpret_cast<u32x4*>(to_woven + share * 1024 + lane * 16) = weave(v);
        sum = dot2(v[0], ONES, dot2(v[1], ONES, 0.0f)) + dot2(v[2], ONES, dot2(v[3], ONES, 0.0f));
      }
      sum += swapped<0xB1>(sum);                          // lane ^ 1
      sum += swapped<0x4E>(sum);                          // lane ^ 2
      if constexpr (GP < 4) sum += swapped<0x141>(sum);   // 7 - lane of eight
      if constexpr (GP < 2) sum += swapped<0x140>(sum);   // 15 - lane
      if (i % (16 / GP) == 0) {
        float* const all = reinterpret_cast<float*>(smem + Z::ALL + (step / CS & 1) * Z::SUMS);
        all[(step % CS * GP + octet / (16 / GP)) * 16 * MB + row] = sum;
      }
    }
    raw = raw + 1 < AHEAD ? raw + 1 : 0;
  };
  uint32_t mask = 0x00780078u, sixteen = 0x41804180u;
  asm("" : "+v"(mask), "+v"(sixteen));   // (in registers: as literals they take an operation each)
  f32x4 acc[MB][2];
#pragma unroll
  for (int r = 0; r < MB; ++r)
#pragma unroll
    for (int b = 0; b < 2; ++b) acc[r][b] = f32x4{0, 0, 0, 0};
  // the first chunk, and what the steps before the first one of its chunk would have brought of the next
#pragma unroll
  for (int u = 0; u < PARTS; ++u) load_scales(s0 / CS, u, s0 / CS % Z::CHUNKS);
  for (uint32_t u = 0; u < s0 % CS * Z::S; ++u) load_scales(s0 / CS + 1, u % PARTS, to);
#pragma unroll
  for (int u = 0; u < AHEAD; ++u)
    if (s0 + u < s1) load(s0 + u);
  if (s0 + AHEAD <= s1) arrived_but<AHEAD * Z::L - 1>();   // (the first step's rows)
  else arrived();
  weave_step(s0);
  uint32_t now = 0, from = s0 / CS % Z::CHUNKS;
  for (uint32_t step = s0; step < s1; ++step) {
    // this step's weights and the next one's rows are here
    if (step + AHEAD <= s1) meet_but<(AHEAD - 1) * Z::L - 1>();
    else meet();
    if (step + 1 < s1) weave_step(step + 1);
    if (step + AHEAD < s1) load(step + AHEAD);   // into the slots that this wave has read
    const uint8_t* const at = smem + now * Z::WSTEP + wave * 2048 + i * 64 + q * 4;
    const uint8_t* const rows = smem + Z::WOVEN + (step & 1) * Z::WOVEN_STEP + i * 256;
    now = now + 1 < Z::BUFS ? now + 1 : 0;
    // the step's first group in its chunk
    const uint8_t* const chunk = own + from * 2 * Z::CHUNK;
    const uint8_t* const scales = chunk + 4 * (GP > 1 ? step % CS * GP : step / (uint32_t)per_group - step / CS * CS / (uint32_t)per_group);
    // all that the step multiplies, read at once
    u32x4 v[4][MB * TERMS];   // (block of rows, or term)
    uint32_t d[4][2];
    float scale[GP][2];
#pragma unroll
    for (int r = 0; r < 4; ++r) {
#pragma unroll
      for (int b = 0; b < 2; ++b) d[r][b] = *reinterpret_cast<const uint32_t*>(at + b * 1024 + ((r ^ (i >> 2)) << 4));
#pragma unroll
      for (int t = 0; t < MB * TERMS; ++t) v[r][t] = *reinterpret_cast<const u32x4*>(rows + t * 4096 + (((4 * r + q) ^ i) << 4));
    }
#pragma unroll
    for (int g = 0; g < GP; ++g)
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        const float f = *reinterpret_cast<const float*>(scales + ((16 * b + i) * GC + g) * 4);
        scale[g][b] = GP == 1 || (int)step * 128 + g * (128 / GP) < K ? f : 0.0f;   // (a last step may be short by whole groups)
      }
#pragma unroll
    for (int g = 0; g < GP; ++g) {
      f32x4 dot[MB][2];
#pragma unroll
      for (int r = 4 / GP * g; r < 4 / GP * (g + 1); ++r)
#pragma unroll
        for (int b = 0; b < 2; ++b) {
          const uint32_t w4 = d[r][b];
          const u32x4 f = {(w4 << 3 & mask) | sixteen, (w4 >> 1 & mask) | sixteen, (w4 >> 5 & mask) | sixteen, (w4 >> 9 & mask) | sixteen};
#pragma unroll
          for (int t = 0; t < MB * TERMS; ++t) dot[t % MB][b] = mfma16(v[r][t], f, r == 4 / GP * g && t < MB ? f32x4{0, 0, 0, 0} : dot[t % MB][b]);
        }
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int t = 0; t < MB; ++t)
#pragma unroll
          for (int e = 0; e < 4; ++e) acc[t][b][e] += scale[g][b] * dot[t][b][e];
    }
    if ((step + 1) % CS == 0 || step + 1 == s1) {   // the chunk's zero points (its groups that lie in this share)
      const uint32_t c = step / CS;
      const float* const all = reinterpret_cast<const float*>(smem + Z::ALL + (c & 1) * Z::SUMS);
#pragma unroll
      for (int u = 0; u < GC; u += 4) {
        const uint32_t k = u + q, at_step = c * CS + k / GP;   // this lane's group of the chunk
        const bool mine = at_step >= s0 && at_step < s1 && (GP == 1 || c * GC + k < (uint32_t)groups);
        const uint32_t entry = GP > 1 ? k : at_step / (uint32_t)per_group - c * CS / (uint32_t)per_group;
        float taken[2];
#pragma unroll
        for (int b = 0; b < 2; ++b) {
          const uint8_t* const e = chunk + ((16 * b + i) * GC + entry) * 4;
          const float zero = 16.0f + (zero0 ? (float)*reinterpret_cast<const uint32_t*>(e + Z::CHUNK) : 8.0f);
          taken[b] = mine ? -zero * *reinterpret_cast<const float*>(e) : 0.0f;
        }
#pragma unroll
        for (int t = 0; t < MB; ++t) {
          const float sum = mine ? all[k * 16 * MB + 16 * t + i] : 0.0f;
#pragma unroll
          for (int b = 0; b < 2; ++b) acc[t][b] = __builtin_amdgcn_mfma_f32_16x16x4f32(sum, taken[b], acc[t][b], 0, 0, 0);
        }
      }
      from = from + 1 < Z::CHUNKS ? from + 1 : 0;
    }
  }
  const uint32_t stride = splits > 1 ? (uint32_t)a.outputs : (uint32_t)a.out_stride;
  float* const part = static_cast<float*>(a.workspace) + ((int64_t)split * a.rows + m0) * a.outputs + n0;
  T* const out = static_cast<T*>(a.out) + (int64_t)m0 * a.out_stride + n0;
#pragma unroll
  for (int t = 0; t < MB; ++t)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int row = 16 * t + 4 * q + e;
      if (m0 + row >= a.rows) continue;
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        const int col = 16 * b + i;
        if (n0 + col > last) continue;
        const uint32_t to = row * stride + col;
        if (splits > 1) part[to] = acc[t][b][e];
        else st(out + to, q4_result<T>(a, m0 + row, n0 + col, acc[t][b][e]));
      }
    }
}

// Adds the parts of every result, in their order, eight on their way at a time.
template <typename T>
__global__ void __launch_bounds__(256) q4_join_kernel(fi_q4_matmul_args a, int splits, uint32_t blocks) {
  const uint32_t row = blockIdx.x / blocks, col = blockIdx.x % blocks * 256 + threadIdx.x;
  if (col >= (uint32_t)a.outputs) return;
  const int64_t size = (int64_t)a.rows * a.outputs;
  const float* at = static_cast<const float*>(a.workspace) + (int64_t)row * a.outputs + col;
  float y = 0.0f;
  for (int s = 0; s < splits; s += 8) {
    float part[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) part[u] = s + u < splits ? at[u * size] : 0.0f;
#pragma unroll
    for (int u = 0; u < 8; ++u) y += part[u];
    at += 8 * size;
  }
  st(static_cast<T*>(a.out) + (int64_t)row * a.out_stride + col, q4_result<T>(a, row, col, y));
}

// Which kernel takes a call, from its sizes and type alone (the workspace goes by it), where the addresses allow all of them.
//  FEW:  reads 2048 inputs a step; its time grows with rows x outputs (us, few / tile: 4096 x 1000 inputs x outputs, 1 row 3.2 / 8.4, 4 rows 5.2 / 9.1, 16 rows 7.9 / 11.3;
//        4096 x 4096, 4 rows 7.8 / 10.0, 8 rows 10.9 / 10.8; 1024 x 16384, 2 rows 8.2 / 8.2, 4 rows 12.6 / 8.4; 512 x 8192, 1 row 4.2 / 3.6).
//  TILE: its time is that of a wave's walk over its share of the inputs, once a round of 256 workgroups; smaller groups and fp32 rows make a step longer.
//  WIDE: has two launches and about 10 us whatever it does, and the least time per weight (us, wide / tile, groups of 64, 16 rows: 2048 x 4096 10.9 / 7.2, 4096 x 4096 12.0 / 11.8,
//        8192 x 3000 13.6 / 20.5, 2048 x 8000, two rounds, 11.9 / 12.6; 1024 x 16384, four times the work a step, 12.1 / 8.8, 32 rows 15.5 / 15.8; groups of 32: 2048 x 4096 12.2 / 9.9,
//        4096 x 2048 12.8 / 17.0, 1024 x 16384 13.2 / 14.9; fp32: 2048 x 4096 11.9 / 9.3, 4096 x 4096 12.8 / 15.8, 1024 x 16384 13.1 / 10.2, 64 rows x 16384 x 4096 52 / 203;
//        wide / few: 8192 x 1024, 8 rows 11.4 / 9.2; 12288 x 600, 8 rows 11.9 / 12.5; 25088 x 300, 8 rows 16.1 / 19.4; 16384 x 4096, 4 rows 18.8 / 19.8, 25088 x 4096 26.0 / 29.7,
//        fp32 30 / 41).
enum Kernel { FEW, TILE, WIDE };
struct Plan { Kernel kernel; int mb, splits; };
Plan plan(const fi_q4_matmul_args& a) {
  Plan p = {TILE, 1, 1};
  const int64_t blocks = ((int64_t)a.outputs + 32 * WAVES - 1) / (32 * WAVES), steps = ((int64_t)a.inputs + 127) / 128;
  const bool f32 = a.dtype == FI_F32, few = a.inputs >= 2048 && a.rows <= 16 && a.outputs < 2048;
  const int64_t per = a.outputs >= 16384 ? 64 : 16, tiles = (a.outputs + per - 1) / per * (((int64_t)a.rows + 15) / 16);
  const int64_t walk = a.inputs * ((tiles + 255) / 256) * (per == 64 ? 3 : 1);   // (of TILE)
  const int64_t most = a.group < 64 ? 3000 : a.group < 128 ? (f32 ? 4000 : 5000) : (f32 ? 5000 : 7000);
  const bool wide = a.rows > 4 ? a.inputs >= 12288 || (!few && walk >= most) : a.rows > 2 && a.inputs >= 16384;
  if (wide) {
    p.kernel = WIDE;
    p.mb = a.rows > 16 && a.dtype == FI_BF16 ? 2 : 1;
    const int64_t groups = blocks * (((int64_t)a.rows + 16 * p.mb - 1) / (16 * p.mb));
    int64_t splits = groups > 0 ? 256 / groups : 1;                   // a workgroup per compute unit at most: they run one at a time
    if (splits > steps / 4) splits = steps / 4;                       // (a join costs about as much as four steps)
    p.splits = splits < 1 ? 1 : splits > 32 ? 32 : (int)splits;
  } else if (few || (a.inputs >= 1024 && a.rows <= 2) || (a.inputs >= 2048 && a.rows <= 4)) {
    p.kernel = FEW;
  }
  return p;
}

// The rows start on 16 bytes, weights on the VW dwords that a lane of the tile kernel takes at once.
bool on_tiles(const fi_q4_matmul_args& a, int& vw) {
  const int es = elem_size(a.dtype);
  if (reinterpret_cast<uintptr_t>(a.x) % 16 || a.x_stride * es % 16) return false;
  const uintptr_t w = reinterpret_cast<uintptr_t>(a.w) | (uintptr_t)a.w_stride;
  vw = a.group % 128 == 0 && w % 16 == 0 ? 4 : a.group % 64 == 0 && w % 8 == 0 ? 2 : 1;
  return w % 4 == 0;
}

template <typename T, int NB, int W>
void launch_tiles(const fi_q4_matmul_args& a, int vw, hipStream_t s) {
  const dim3 grid((uint32_t)(((int64_t)a.outputs + 16 * NB - 1) / (16 * NB)), (uint32_t)(((int64_t)a.rows + 15) / 16));
  const uint32_t inv = (uint32_t)((1ull << 32) / (uint32_t)a.group);
  if (vw == 4) q4_tile_kernel<T, NB, 4, W><<<grid, 64 * W, 0, s>>>(a, inv);
  else if (vw == 2) q4_tile_kernel<T, NB, 2, W><<<grid, 64 * W, 0, s>>>(a, inv);
  else q4_tile_kernel<T, NB, 1, W><<<grid, 64 * W, 0, s>>>(a, inv);
}
template <typename T, int M>
void launch_few(const fi_q4_matmul_args& a, hipStream_t s) {
  const uint32_t inv = (uint32_t)((1ull << 32) / (uint32_t)a.group);
  const uint32_t passes = (uint32_t)((a.rows + M - 1) / M);
  auto grid = [&](int outs, int wk) { return dim3((uint32_t)(((int64_t)a.outputs + outs * (4 / wk) - 1) / (outs * (4 / wk))), passes); };
  // two outputs share what is read of the rows, once that leaves enough waves (4096 x 1000, 4 rows: one 5.2 us, two 6.0; 8 rows, two passes: 7.2, 6.2; 4096 x 4096, 4 rows: 11.9, 7.8)
  if ((int64_t)a.outputs * passes >= 1536) q4_few_kernel<T, M, 2, 1><<<grid(2, 1), 256, 0, s>>>(a, inv);
  else if (a.inputs > 2048) q4_few_kernel<T, M, 1, 2><<<grid(1, 2), 256, 0, s>>>(a, inv);
  else q4_few_kernel<T, M, 1, 1><<<grid(1, 1), 256, 0, s>>>(a, inv);
}
template <typename T, int MB>
void launch_wide(const fi_q4_matmul_args& a, const Plan& p, hipStream_t s) {
  const dim3 grid((uint32_t)(((int64_t)a.outputs + 32 * WAVES - 1) / (32 * WAVES) * p.splits), (uint32_t)(((int64_t)a.rows + 16 * MB - 1) / (16 * MB)));
  if (a.group == 32) q4_wide_kernel<T, MB, 4><<<grid, 64 * WAVES, 0, s>>>(a, p.splits, 1);
  else if (a.group == 64) q4_wide_kernel<T, MB, 2><<<grid, 64 * WAVES, 0, s>>>(a, p.splits, 1);
  else q4_wide_kernel<T, MB, 1><<<grid, 64 * WAVES, 0, s>>>(a, p.splits, a.group / 128);
}
template <typename T>
int launch_t(const fi_q4_matmul_args& a, hipStream_t s) {
  int vw;
  if (a.inputs == 0 || !on_tiles(a, vw)) {
    q4_row_kernel<T><<<dim3((uint32_t)(((int64_t)a.outputs + 3) / 4)), 256, 0, s>>>(a);
    return (int)hipGetLastError();
  }
  const Plan p = plan(a);
  const bool aligned = (reinterpret_cast<uintptr_t>(a.w) | (uintptr_t)a.w_stride) % 16 == 0;
  const bool near = a.x_stride < 1 << 24 && a.out_stride < 1 << 24 && a.w_stride < 1 << 24 && a.scales_stride < 1 << 24 && (!a.zeros || a.zeros_stride < 1 << 24);   // (32 rows lie within 2^31 bytes)
  if (p.kernel == FEW && aligned) {
    if (a.rows == 1) launch_few<T, 1>(a, s);
    else if (a.rows == 2) launch_few<T, 2>(a, s);
    else launch_few<T, 4>(a, s);
  } else if (p.kernel == WIDE && aligned && near) {
    if constexpr (sizeof(T) == 4) launch_wide<T, 1>(a, p, s);
    else if (p.mb == 1) launch_wide<T, 1>(a, p, s);
    else launch_wide<T, 2>(a, p, s);
    const uint32_t blocks = (uint32_t)((a.outputs + 255) / 256);
    if (p.splits > 1) q4_join_kernel<T><<<dim3(blocks * (uint32_t)a.rows), 256, 0, s>>>(a, p.splits, blocks);
  } else if (a.outputs >= 16384) {   // (four blocks of outputs share the rows' inputs; fewer leave compute units without work)
    launch_tiles<T, 4, 8>(a, vw, s);
  } else if (a.inputs >= 2048) {
    launch_tiles<T, 1, 16>(a, vw, s);
  } else {
    launch_tiles<T, 1, 8>(a, vw, s);
  }
  return (int)hipGetLastError();
}

}  // namespace

uint64_t q4_workspace(const fi_q4_matmul_args& a) {
  const Plan p = plan(a);
  return p.splits > 1 ? (uint64_t)p.splits * a.rows * a.outputs * 4 : 0;
}

int launch_q4_matmul(const fi_q4_matmul_args& a, void* stream) {
  const hipStream_t s = static_cast<hipStream_t>(stream);
  return a.dtype == FI_F32 ? launch_t<float>(a, s) : launch_t<bf16_t>(a, s);
}

}  // namespace fi
