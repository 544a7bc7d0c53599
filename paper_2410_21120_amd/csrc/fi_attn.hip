// Attention over whole prompts (packed sequences) and of drafted trees over a paged cache.
#include <hip/hip_runtime.h>

#include "fi_device.h"
#include "fi_ops.h"

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
  const int n0 = clamp_int(a.cu_nodes[b], 0, total), n1 = clamp_int(a.cu_nodes[b + 1], n0, total);
  if (row - n0 >= a.max_nodes) return;
  const int places = a.n_pages ? a.page_size * a.table_columns : 0;
  const int cached = clamp_int(a.cached[b], 0, places), keys = n1 - n0 < places - cached ? cached + n1 - n0 : places;
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

}  // namespace

int launch_prompt_attention(const fi_prompt_attention_args& a, void* stream) {
  const hipStream_t s = static_cast<hipStream_t>(stream);
  const dim3 grid((uint32_t)a.q_tokens, (uint32_t)a.q_heads);
  if (a.dtype == FI_F32) prompt_row_kernel<float><<<grid, 64, 0, s>>>(a);
  else prompt_row_kernel<bf16_t><<<grid, 64, 0, s>>>(a);
  return (int)hipGetLastError();
}

uint64_t tree_workspace(const fi_tree_attention_args&) { return 0; }

int launch_tree_attention(const fi_tree_attention_args& a, void* stream) {
  const hipStream_t s = static_cast<hipStream_t>(stream);
  const dim3 grid((uint32_t)a.nodes, (uint32_t)a.q_heads);
  if (a.dtype == FI_F32) tree_row_kernel<float><<<grid, 64, 0, s>>>(a);
  else tree_row_kernel<bf16_t><<<grid, 64, 0, s>>>(a);
  return (int)hipGetLastError();
}

}  // namespace fi
