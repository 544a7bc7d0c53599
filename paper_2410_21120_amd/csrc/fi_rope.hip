// Norms of queries and keys for every head, the position rotation and the write into the paged cache, in one launch.
//
// y = rotate(x * w / sqrt(mean(x^2) + eps)).  Every value is read once and written once, so HBM bounds it, if the vector unit is kept from doing so.  A head's
// row is held by a group of lanes, in registers from the load to the store: a lane has NP pairs (both halves of each, whichever way pairs are
// formed) or 2 NP of the values behind the rotated part, so a rotation needs no neighbour, and the mean is one reduction over the group (in the
// registers' own rotations: 4 additions for 16 lanes).  The lane keeps its pairs from head to head of a token: each sine is computed once (one per lane, handed out
// through LDS to the waves of a workgroup that share the token: for each wave again, 500 tokens took 13.4 us, not 6.6), and weight, cosine and sine become two
// factors per value before the first head.
#include <hip/hip_runtime.h>

#include "fi_device.h"
#include "fi_ops.h"

namespace fi {
namespace {

// Waves of a call, where it has rows for them, at least (2187 tokens of 48 fp32 heads of 72: one wave a token 15.7 us, two 14.4; 3000 of 20 heads of 128 13.8, 14.9), and
// up to which waves without a row in their last turn cost nothing (64 tokens of 48 bf16 heads of 128: 8 waves a token 4.3 us, 16 3.9; 903 of 20: 4 waves 5.6, 8 8.2).
constexpr int64_t FEWEST_WAVES = 2560, LATENCY_WAVES = 1024;
constexpr int HEADS = 4;                 // rows that a group has in flight (16384 tokens of 48 bf16 heads of 128: one 101 us, two 95, three 88, four 88)

template <typename T, int N>
struct alignas(sizeof(T) * N) Run { T v[N]; };

template <int CTRL>
__device__ __forceinline__ float rotated(float v) {   // the value of another lane of the same 16
  return __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(v), CTRL, 0xF, 0xF, true));
}
// The sum over aligned groups of `lanes` lanes (a power of two, the same for the wave), in all of them.  Groups of fewer than 16 do not take whole rows of
// lanes: they exchange.
__device__ __forceinline__ float group_sum(float v, int lanes) {
  if (lanes >= 16) {
    v += rotated<0x128>(v);   // row_ror:8, 4, 2, 1
    v += rotated<0x124>(v);
    v += rotated<0x122>(v);
    v += rotated<0x121>(v);
    if (lanes >= 32) v += __shfl_xor(v, 16);
    if (lanes >= 64) v += __shfl_xor(v, 32);
    return v;
  }
  for (int o = lanes >> 1; o; o >>= 1) v += __shfl_xor(v, o);
  return v;
}

// NP pairs per lane; ITEMS of them (2: one pair at a time, rows that are not a whole number of longer runs).  A lane's values are two runs of NP, the same run of
// each half.  INTER: pairs are neighbours, inside the runs, else value t of one run and of the other.  lanes: of a group, 1 << wave_bits: waves that share a token.
template <typename T, int NP, int ITEMS, bool INTER>
__global__ void __launch_bounds__(256) rope_kernel(fi_qk_norm_rope_args a, int lanes, int wave_bits) {
  __shared__ float2 turns[4][FI_MAX_HEAD_DIM / 2];
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, D = a.head_dim, half = a.rot_dim / 2;
  const uint32_t wave = blockIdx.x * 4 + w;
  const int token = (int)(wave >> wave_bits), part = (int)(wave & ((1u << wave_bits) - 1u));
  const int shift = __builtin_ctz(lanes), group = (part << (6 - shift)) + (lane >> shift), groups = 64 >> shift << wave_bits, in_group = lane & (lanes - 1);
  const int turned = half / NP;                                       // runs of the rotated part
  const int items = turned + (D - a.rot_dim + 2 * NP - 1) / (2 * NP); // and of the whole row
  // The sines of a token, once for the two or four waves of a workgroup that share it.
  const int sharing = wave_bits >= 2 ? 4 : 1 << wave_bits;
  float2* const turn_of = turns[w & ~(sharing - 1)];
  const int first_pair = token < a.tokens ? lane + 64 * (w & (sharing - 1)) : half;
  for (int pair = first_pair; pair < half; pair += 64 * sharing) {
    int axis = 0, end = a.sections[0];
#pragma unroll
    for (int x = 1; x < FI_MAX_AXES; ++x)
      if (x < a.n_axes) { axis += pair >= end ? 1 : 0; end += a.sections[x]; }
    // the angle is one fp32 product, as models form it when they are trained
    float2 t;
    sincosf((float)a.positions[(int64_t)token * a.n_axes + axis] * a.inv_freq[pair], &t.y, &t.x);
    turn_of[pair] = t;
  }
  if (sharing > 1) __syncthreads();
  else asm volatile("" ::: "memory");   // (a wave's writes and reads of LDS are done in order)
  if (token >= a.tokens) return;

  int first[ITEMS], second[ITEMS];   // where the lane's values stand in a row; an absent value: -1
  bool turn[ITEMS];
  // value t of a run becomes r * (own[t] * it + other[t] * its partner), r = 1 / sqrt(..)
  float own[2][ITEMS][2 * NP], other[2][ITEMS][2 * NP];   // [queries, keys]
#pragma unroll
  for (int u = 0; u < ITEMS; ++u) {
    const int item = in_group + u * lanes;
    first[u] = second[u] = -1;
    turn[u] = item < turned;
    if (turn[u]) {
      first[u] = INTER && NP == 1 ? 2 * item : item * NP;
      second[u] = INTER && NP == 1 ? first[u] + 1 : half + first[u];
    } else if (item < items) {
      first[u] = a.rot_dim + (item - turned) * 2 * NP;
      second[u] = first[u] + NP < D ? first[u] + NP : -1;   // (an odd row's last value, one pair at a time)
    }
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      const float* const weight = x ? a.k_weight : a.q_weight;
      float wt[2 * NP];
#pragma unroll
      for (int t = 0; t < 2 * NP; ++t) wt[t] = 1.0f;
      if (weight && first[u] >= 0) __builtin_memcpy(wt, weight + first[u], NP * 4);
      if (weight && second[u] >= 0) __builtin_memcpy(wt + NP, weight + second[u], NP * 4);
#pragma unroll
      for (int t = 0; t < NP; ++t) {
        const int i = INTER ? 2 * t : t, j = INTER ? 2 * t + 1 : NP + t;
        const int pair = INTER && NP > 1 ? (2 * t < NP ? first[u] : second[u] - NP) / 2 + t : item * NP + t;   // (runs start on even values)
        const float2 cs = turn[u] ? turn_of[pair] : make_float2(1.0f, 0.0f);
        own[x][u][i] = wt[i] * cs.x;
        other[x][u][i] = -wt[j] * cs.y;
        own[x][u][j] = wt[j] * cs.x;
        other[x][u][j] = wt[i] * cs.y;
      }
    }
  }
  const bool rest = a.rot_dim < D;   // some lanes' values are not rotated
  const float inv_d = 1.0f / (float)D;
  // where the token's keys and values go
  int64_t page = 0, place = token;
  bool keep = true;
  if (a.slots) {
    const int64_t slot = a.slots[token];
    keep = slot >= 0 && slot < a.n_slots;
    if ((uint64_t)slot >> 32 == 0) {
      page = (uint32_t)slot / (uint32_t)a.page_size;
      place = (uint32_t)slot - (uint32_t)page * (uint32_t)a.page_size;
    } else {
      page = slot / a.page_size;
      place = slot - page * a.page_size;
    }
  }
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
      if (hv < 0) {
        float v[ITEMS][2 * NP], sum = 0.0f;
#pragma unroll
        for (int u = 0; u < ITEMS; ++u)
#pragma unroll
          for (int t = 0; t < 2 * NP; ++t) {
            v[u][t] = ld(t < NP ? &x0[j][u].v[t % NP] : &x1[j][u].v[t % NP]);
            sum = __builtin_fmaf(v[u][t], v[u][t], sum);
          }
        const float r = __builtin_amdgcn_rsqf(__builtin_fmaf(group_sum(sum, lanes), inv_d, a.eps));
#pragma unroll
        for (int u = 0; u < ITEMS; ++u) {
          float y[2 * NP];
#pragma unroll
          for (int t = 0; t < 2 * NP; ++t) {
            const int partner = INTER ? t ^ 1 : (t + NP) % (2 * NP);
            const float f = hk < 0 ? own[0][u][t] : own[1][u][t], g = hk < 0 ? other[0][u][t] : other[1][u][t];
            const float mine = v[u][t] * f;
            y[t] = __builtin_fmaf(v[u][partner], g, mine);
            if (rest) y[t] = turn[u] ? y[t] : mine;   // (an infinite partner times zero would not vanish)
            y[t] *= r;
          }
          if constexpr (sizeof(T) == 2 && NP % 2 == 0) {
#pragma unroll
            for (int t = 0; t < NP; t += 2) {
              reinterpret_cast<uint32_t*>(x0[j][u].v)[t / 2] = pack_bf16x2(y[t], y[t + 1]);
              reinterpret_cast<uint32_t*>(x1[j][u].v)[t / 2] = pack_bf16x2(y[NP + t], y[NP + t + 1]);
            }
          } else {
#pragma unroll
            for (int t = 0; t < 2 * NP; ++t) st(t < NP ? &x0[j][u].v[t % NP] : &x1[j][u].v[t % NP], y[t]);
          }
        }
      }
      if (hk >= 0 && !keep) continue;
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
  // A wave per token does the fewest preparations; with few tokens more waves share one, down to a row per group.
  const int heads = a.q_heads + a.kv_heads * (a.v ? 2 : 1), most = (heads + 64 / lanes - 1) / (64 / lanes);
  int bits = 0;
  auto waves = [&] { return (int64_t)a.tokens << bits; };
  while ((2 << bits <= most && waves() < FEWEST_WAVES) || (1 << bits < most && waves() < LATENCY_WAVES)) ++bits;
  if (!one_launch((waves() + 3) / 4, 256)) return kTooLarge;
  const dim3 grid((uint32_t)((waves() + 3) / 4));
  if (a.interleaved) rope_kernel<T, NP, ITEMS, true><<<grid, 256, 0, s>>>(a, lanes, bits);
  else rope_kernel<T, NP, ITEMS, false><<<grid, 256, 0, s>>>(a, lanes, bits);
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
