// Norms of queries and keys for every head, the position rotation and the write into the paged cache, in one launch.
//
// y = rotate(x * w / sqrt(mean(x^2) + eps)).  Every value is read once and written once, so HBM bounds it.  A head's row is held by
// a group of lanes, in registers from the load to the store: a lane has NP pairs (both halves of each, whichever way pairs are formed) or
// 2 NP of the values behind the rotated part, so a rotation needs no neighbour and the mean one reduction over the group.  The lane keeps
// its pairs from head to head of a token: sines and cosines are computed once per token and lane.
#include <hip/hip_runtime.h>

#include "fi_device.h"
#include "fi_ops.h"

namespace fi {
namespace {

constexpr int HEADS = 4;   // rows that a group has in flight

template <typename T, int N>
struct alignas(sizeof(T) * N) Run { T v[N]; };

// NP pairs per lane; ITEMS runs of them per lane (2: one pair at a time, rows that are not a whole number of longer runs).
// lanes: lanes of a group, a power of two.  waves: waves that share a token.
template <typename T, int NP, int ITEMS>
__global__ void __launch_bounds__(256) rope_kernel(fi_qk_norm_rope_args a, int lanes, int waves) {
  const int lane = threadIdx.x & 63, D = a.head_dim, half = a.rot_dim / 2;
  const int64_t wave = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  const int token = (int)(wave / waves), part = (int)(wave - (int64_t)token * waves);
  if (token >= a.tokens) return;
  const int per_wave = 64 / lanes, group = part * per_wave + lane / lanes, groups = waves * per_wave;
  const int turned = half / NP;                                       // runs of the rotated part
  const int items = turned + (D - a.rot_dim + 2 * NP - 1) / (2 * NP); // and of the whole row

  int first[ITEMS], second[ITEMS];   // where the lane's values stand in a row; an absent value: -1
  float c[ITEMS][NP], s[ITEMS][NP], wq[ITEMS][2 * NP], wk[ITEMS][2 * NP];
#pragma unroll
  for (int u = 0; u < ITEMS; ++u) {
    const int item = (lane & (lanes - 1)) + u * lanes;
    first[u] = second[u] = -1;
#pragma unroll
    for (int t = 0; t < NP; ++t) c[u][t] = 1.0f, s[u][t] = 0.0f;
    if (item < turned) {
      first[u] = a.interleaved ? item * 2 * NP : item * NP;
      second[u] = a.interleaved ? first[u] + NP : half + first[u];
#pragma unroll
      for (int t = 0; t < NP; ++t) {
        const int pair = item * NP + t;
        int axis = 0, end = a.sections[0];
#pragma unroll
        for (int x = 1; x < FI_MAX_AXES; ++x)
          if (x < a.n_axes) { axis += pair >= end ? 1 : 0; end += a.sections[x]; }
        // the angle is one fp32 product, as models form it when they are trained
        sincosf((float)a.positions[(int64_t)token * a.n_axes + axis] * a.inv_freq[pair], &s[u][t], &c[u][t]);
      }
    } else if (item < items) {
      first[u] = a.rot_dim + (item - turned) * 2 * NP;
      second[u] = first[u] + NP < D ? first[u] + NP : -1;   // (an odd row's last value, one pair at a time)
    }
#pragma unroll
    for (int t = 0; t < 2 * NP; ++t) {
      const int at = (t < NP ? first[u] : second[u]) + t % NP;
      const bool there = t < NP ? first[u] >= 0 : second[u] >= 0;
      wq[u][t] = there && a.q_weight ? a.q_weight[at] : 1.0f;
      wk[u][t] = there && a.k_weight ? a.k_weight[at] : 1.0f;
    }
  }
  const float inv_d = 1.0f / (float)D;
  // where the token's keys and values go
  int64_t page = 0, place = token;
  bool keep = true;
  if (a.slots) {
    const int64_t slot = a.slots[token];
    keep = slot >= 0 && slot < a.n_slots;
    page = slot / a.page_size;
    place = slot - page * a.page_size;
  }
  // The interleaved order of a run: values 2t, 2t + 1 are pair t; first / second hold its two halves in memory order.
  const bool inter = a.interleaved != 0;
  const int heads = a.q_heads + a.kv_heads + (a.v ? a.kv_heads : 0);
  for (int h0 = group; h0 < heads; h0 += groups * HEADS) {
    Run<T, NP> x0[HEADS][ITEMS], x1[HEADS][ITEMS];
#pragma unroll
    for (int j = 0; j < HEADS; ++j) {
      const int h = h0 + j * groups;
      if (h >= heads) break;
      const int hk = h - a.q_heads, hv = hk - a.kv_heads;
      const T* const row = hk < 0   ? static_cast<const T*>(a.q) + token * a.q_strides[0] + h * a.q_strides[1]
                           : hv < 0 ? static_cast<const T*>(a.k) + token * a.k_strides[0] + hk * a.k_strides[1]
                                    : static_cast<const T*>(a.v) + token * a.v_strides[0] + hv * a.v_strides[1];
#pragma unroll
      for (int u = 0; u < ITEMS; ++u) {
        x0[j][u] = Run<T, NP>{};
        x1[j][u] = Run<T, NP>{};
        if (first[u] >= 0) x0[j][u] = *reinterpret_cast<const Run<T, NP>*>(row + first[u]);
        if (second[u] >= 0) x1[j][u] = *reinterpret_cast<const Run<T, NP>*>(row + second[u]);
      }
    }
#pragma unroll
    for (int j = 0; j < HEADS; ++j) {
      const int h = h0 + j * groups;
      if (h >= heads) break;
      const int hk = h - a.q_heads, hv = hk - a.kv_heads;
      T* const row = hk < 0   ? static_cast<T*>(a.q_out) + token * a.q_out_strides[0] + h * a.q_out_strides[1]
                     : hv < 0 ? static_cast<T*>(a.k_out) + page * a.k_out_strides[0] + place * a.k_out_strides[1] + hk * a.k_out_strides[2]
                              : static_cast<T*>(a.v_out) + page * a.v_out_strides[0] + place * a.v_out_strides[1] + hv * a.v_out_strides[2];
      const bool store = hk < 0 || keep;
      if (hv < 0) {
        float v[ITEMS][2 * NP], sum = 0.0f;
#pragma unroll
        for (int u = 0; u < ITEMS; ++u)
#pragma unroll
          for (int t = 0; t < 2 * NP; ++t) {
            v[u][t] = ld(t < NP ? &x0[j][u].v[t % NP] : &x1[j][u].v[t % NP]);
            sum += v[u][t] * v[u][t];
          }
        for (int o = lanes >> 1; o; o >>= 1) sum += __shfl_xor(sum, o);
        const float r = 1.0f / sqrtf(sum * inv_d + a.eps);
#pragma unroll
        for (int u = 0; u < ITEMS; ++u) {
          float y[2 * NP];
#pragma unroll
          for (int t = 0; t < 2 * NP; ++t) v[u][t] *= r * (hk < 0 ? wq[u][t] : wk[u][t]);
          const bool turns = (lane & (lanes - 1)) + u * lanes < turned;
#pragma unroll
          for (int t = 0; t < NP; ++t) {
            const int i0 = t, i1 = NP + t, k0 = 2 * t, k1 = 2 * t + 1;
            const float p = inter ? v[u][k0] : v[u][i0], q = inter ? v[u][k1] : v[u][i1];
            const float yp = turns ? p * c[u][t] - q * s[u][t] : p, yq = turns ? q * c[u][t] + p * s[u][t] : q;
            if (inter) { y[k0] = yp; y[k1] = yq; }
            else { y[i0] = yp; y[i1] = yq; }
          }
#pragma unroll
          for (int t = 0; t < 2 * NP; ++t) st(t < NP ? &x0[j][u].v[t % NP] : &x1[j][u].v[t % NP], y[t]);
        }
      }
      if (!store) continue;
#pragma unroll
      for (int u = 0; u < ITEMS; ++u) {
        if (first[u] >= 0) *reinterpret_cast<Run<T, NP>*>(row + first[u]) = x0[j][u];
        if (second[u] >= 0) *reinterpret_cast<Run<T, NP>*>(row + second[u]) = x1[j][u];
      }
    }
  }
}

// Whether every row of a tensor starts on a multiple of `bytes`.
bool starts_on(const void* p, const int64_t* strides, int n, int es, int bytes) {
  if (!p) return true;
  if (reinterpret_cast<uintptr_t>(p) % bytes) return false;
  for (int i = 0; i < n; ++i)
    if (strides[i] * es % bytes) return false;
  return true;
}

template <typename T, int NP, int ITEMS>
int launch_np(const fi_qk_norm_rope_args& a, hipStream_t s) {
  const int items = a.rot_dim / 2 / NP + (a.head_dim - a.rot_dim + 2 * NP - 1) / (2 * NP);
  int lanes = 1;
  while (lanes * ITEMS < items) lanes *= 2;
  // A wave per token computes the fewest sines; with few tokens more waves share one, down to a row per group.
  const int heads = a.q_heads + a.kv_heads * (a.v ? 2 : 1), most = (heads + 64 / lanes - 1) / (64 / lanes);
  int waves = 1;
  while (waves < most && (int64_t)a.tokens * waves < 8192) waves *= 2;
  const int64_t blocks = ((int64_t)a.tokens * waves + 3) / 4;
  rope_kernel<T, NP, ITEMS><<<dim3((uint32_t)blocks), 256, 0, s>>>(a, lanes, waves);
  return (int)hipGetLastError();
}

template <typename T>
int launch_t(const fi_qk_norm_rope_args& a, hipStream_t s) {
  const int es = sizeof(T);
  auto whole = [&](int np) {   // rows are whole runs of np pairs, on addresses that a run of np values needs
    return a.rot_dim % (2 * np) == 0 && a.head_dim % (2 * np) == 0 && starts_on(a.q, a.q_strides, 2, es, np * es) && starts_on(a.k, a.k_strides, 2, es, np * es) &&
           starts_on(a.v, a.v_strides, 2, es, np * es) && starts_on(a.q_out, a.q_out_strides, 2, es, np * es) &&
           starts_on(a.k_out, a.k_out_strides, 3, es, np * es) && starts_on(a.v_out, a.v_out_strides, 3, es, np * es);
  };
  if (whole(4)) return launch_np<T, 4, 1>(a, s);
  if (whole(2)) return launch_np<T, 2, 1>(a, s);
  return launch_np<T, 1, 2>(a, s);
}

}  // namespace

int launch_qk_norm_rope(const fi_qk_norm_rope_args& a, void* stream) {
  const hipStream_t s = static_cast<hipStream_t>(stream);
  return a.dtype == FI_F32 ? launch_t<float>(a, s) : launch_t<bf16_t>(a, s);
}

}  // namespace fi
