// Products of a few rows with 4-bit weights and group scales.
#include <hip/hip_runtime.h>

#include "fi_device.h"
#include "fi_ops.h"

namespace fi {
namespace {

constexpr int ROWS = 8;   // rows that a wave has sums of

// One wave per output: a lane takes eight weights at a time, scaled group by group.
template <typename T>
__global__ void __launch_bounds__(256) q4_kernel(fi_q4_matmul_args a) {
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

}  // namespace

int launch_q4_matmul(const fi_q4_matmul_args& a, void* stream) {
  const hipStream_t s = static_cast<hipStream_t>(stream);
  const dim3 grid((uint32_t)(((int64_t)a.outputs + 3) / 4));
  if (a.dtype == FI_F32) q4_kernel<float><<<grid, 256, 0, s>>>(a);
  else q4_kernel<bf16_t><<<grid, 256, 0, s>>>(a);
  return (int)hipGetLastError();
}

}  // namespace fi
