// Products of a few rows with 4-bit weights and group scales.
//
// y[m][n] = sum over groups of scale * sum of (q - zero) x.  Every weight is read once, so HBM bounds it as long as the rows are few.  The products run on the
// matrix cores, 16 rows x 16 outputs x 32 inputs an instruction.  A weight becomes bf16 in one operation and a share of a shift: 16 + q is the bit
// pattern 0x4180 | q << 3, two of them at a time, exact; sums of (16 + q) x and of x (the same instruction with ones) are kept in fp32 over a group,
// and (16 + zero) times the second comes off the first when the scale is applied.  fp32 rows are split into three bf16 terms
// (24 bits), so that they enter exactly, too.
#include <hip/hip_runtime.h>

#include "fi_device.h"
#include "fi_ops.h"

namespace fi {
namespace {

constexpr int ROWS = 8;   // rows that a wave of the row kernel has sums of

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
      for (int t = 0; t < 8; ++t) q[t] = ((float)((w[k / 2 + t / 2] >> (t % 2 * 4)) & 15) - zero) * scale;
#pragma unroll
      for (int m = 0; m < ROWS; ++m) {
        if (m0 + m >= a.rows) break;
        const T* const x = static_cast<const T*>(a.x) + (m0 + m) * a.x_stride + k;
#pragma unroll
        for (int t = 0; t < 8; ++t) sum[m] += q[t] * ld(x + t);
      }
    }
#pragma unroll
    for (int m = 0; m < ROWS; ++m) {
      if (m0 + m >= a.rows) break;
      float v = sum[m];
      for (int o = 32; o; o >>= 1) v += __shfl_xor(v, o);
      if (lane == 0) st(static_cast<T*>(a.out) + (m0 + m) * a.out_stride + n, v);
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
template <typename T, int MB, int NB, int VW>
__global__ void __launch_bounds__(64 * WAVES, 2) q4_tile_kernel(fi_q4_matmul_args a, int splits) {
  constexpr int PIECES = 4 / VW, TERMS = Run8<T>::TERMS;
  __shared__ f32x4 sums[WAVES][MB * NB][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), q = lane >> 4, i = lane & 15;
  const int split = blockIdx.x % splits, n0 = (int)(blockIdx.x / splits) * 16 * NB, m0 = blockIdx.y * 16 * MB, K = a.inputs;
  const int steps = (K + 127) / 128, share = split * WAVES + wave, shares = splits * WAVES;
  const int s0 = (int)((int64_t)steps * share / shares), s1 = (int)((int64_t)steps * (share + 1) / shares);
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
  auto load = [&](Step& s, int step) {
#pragma unroll
    for (int p = 0; p < PIECES; ++p) {
      const int k = step * 128 + p * 32 * VW;
      const bool inside = k < K;   // (a step at the end may be short by whole pieces)
      const int g = inside ? k / a.group : 0;
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
      if (splits > 1) static_cast<float*>(a.workspace)[((int64_t)split * a.rows + row + e) * a.outputs + col] = y[e];
      else st(static_cast<T*>(a.out) + (row + e) * a.out_stride + col, y[e]);
    }
  }
}

// Adds the parts of every result, in their order.
template <typename T>
__global__ void __launch_bounds__(256) q4_join_kernel(fi_q4_matmul_args a, int splits) {
  const int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x, size = (int64_t)a.rows * a.outputs;
  if (at >= size) return;
  const float* const parts = static_cast<const float*>(a.workspace) + at;
  float y = parts[0];
  for (int s = 1; s < splits; ++s) y += parts[s * size];
  const int row = (int)(at / a.outputs);
  st(static_cast<T*>(a.out) + row * a.out_stride + (at - (int64_t)row * a.outputs), y);
}

// Blocks of 16 rows and of 16 outputs that a workgroup computes, parts of the inputs.
struct Plan { int mb, nb, splits; };
Plan plan(const fi_q4_matmul_args& a) {
  Plan p;
  p.mb = a.rows <= 16 ? 1 : 2;
  const int64_t blocks = ((int64_t)a.outputs + 15) / 16, passes = ((int64_t)a.rows + 16 * p.mb - 1) / (16 * p.mb);
  // A workgroup reads its rows' inputs beside its weights: from a few rows on more outputs share them, and parts of the inputs fill the chip.
  p.nb = a.rows > 8 || blocks >= 1024 ? 4 : 1;
  const int64_t groups = (blocks + p.nb - 1) / p.nb * passes, steps = ((int64_t)a.inputs + 127) / 128;
  int64_t splits = groups > 0 && p.nb > 1 ? (256 + groups - 1) / groups : 1;
  if (splits > steps / (2 * WAVES)) splits = steps / (2 * WAVES);
  p.splits = splits < 1 ? 1 : splits > 16 ? 16 : (int)splits;
  return p;
}

bool on_tiles(const fi_q4_matmul_args& a, int& vw) {
  const int es = elem_size(a.dtype);
  if (reinterpret_cast<uintptr_t>(a.x) % 16 || a.x_stride * es % 16) return false;
  const uintptr_t w = reinterpret_cast<uintptr_t>(a.w) | (uintptr_t)a.w_stride;
  vw = a.group % 128 == 0 && w % 16 == 0 ? 4 : a.group % 64 == 0 && w % 8 == 0 ? 2 : 1;
  return w % 4 == 0;
}

template <typename T, int MB, int NB>
void launch_tiles(const fi_q4_matmul_args& a, const Plan& p, int vw, hipStream_t s) {
  const dim3 grid((uint32_t)((((int64_t)a.outputs + 16 * NB - 1) / (16 * NB)) * p.splits), (uint32_t)(((int64_t)a.rows + 16 * MB - 1) / (16 * MB)));
  if (vw == 4) q4_tile_kernel<T, MB, NB, 4><<<grid, 64 * WAVES, 0, s>>>(a, p.splits);
  else if (vw == 2) q4_tile_kernel<T, MB, NB, 2><<<grid, 64 * WAVES, 0, s>>>(a, p.splits);
  else q4_tile_kernel<T, MB, NB, 1><<<grid, 64 * WAVES, 0, s>>>(a, p.splits);
}
template <typename T>
int launch_t(const fi_q4_matmul_args& a, hipStream_t s) {
  int vw;
  if (!on_tiles(a, vw)) {
    q4_row_kernel<T><<<dim3((uint32_t)(((int64_t)a.outputs + 3) / 4)), 256, 0, s>>>(a);
    return (int)hipGetLastError();
  }
  const Plan p = plan(a);
  if (p.nb == 1) launch_tiles<T, 1, 1>(a, p, vw, s);
  else if (p.mb == 1) launch_tiles<T, 1, 4>(a, p, vw, s);
  else launch_tiles<T, 2, 4>(a, p, vw, s);
  if (p.splits > 1) q4_join_kernel<T><<<dim3((uint32_t)(((int64_t)a.rows * a.outputs + 255) / 256)), 256, 0, s>>>(a, p.splits);
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
