// Entry points of the decoder operators: argument checks, then the launch.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <initializer_list>

#include "fi_internal.h"
#include "fi_ops.h"

namespace fi {
namespace {

constexpr int64_t kRows = (1ll << 31) - 1024;   // row indices are 32 bits, a tile past the last row included
constexpr int64_t kStride = 1ll << 40; // elements: products of strides and indices stay below 2^63

fi_status done(int e, const char* where) {
  if (e == 0) return FI_OK;
  if (e == kTooLarge) {
    set_error("%s: more work than one launch takes", where);
    return FI_EUNSUPPORTED;
  }
  set_error("%s: %s", where, hipGetErrorString(static_cast<hipError_t>(e)));
  return FI_EHIP;
}

// A tensor pointer of `size`-byte elements: present and aligned to its elements.
bool good(const void* p, uintptr_t size, const char* name) {
  if (!p) { set_error("%s is null", name); return false; }
  if (reinterpret_cast<uintptr_t>(p) % size) { set_error("%s is not aligned to its elements", name); return false; }
  return true;
}

bool good_strides(const int64_t* s, int n, const char* name) {
  for (int i = 0; i < n; ++i)
    if (s[i] < 0 || s[i] > kStride) { set_error("%s: stride %lld", name, (long long)s[i]); return false; }
  return true;
}

// Rows of an output (`row` elements each) may not share memory: every dimension, from the shortest stride on, strides over all that the ones before it reach.
bool apart(std::initializer_list<int64_t> strides, std::initializer_list<int64_t> counts, int64_t row, const char* name) {
  struct Dim { int64_t stride, count; } dims[3];
  int n = 0;
  for (size_t i = 0; i < strides.size(); ++i)
    if (counts.begin()[i] > 1) dims[n++] = Dim{strides.begin()[i], counts.begin()[i]};
  std::sort(dims, dims + n, [](const Dim& a, const Dim& b) { return a.stride < b.stride; });
  __int128 reach = row;
  for (int i = 0; i < n; ++i) {
    if (dims[i].stride < reach) {
      set_error("%s: its rows overlap (a stride of %lld over %.0f elements)", name, (long long)dims[i].stride, (double)reach);
      return false;
    }
    reach += (__int128)dims[i].stride * (dims[i].count - 1);
  }
  return true;
}

bool good_dtype(int32_t d) {
  if (d == FI_F32 || d == FI_BF16) return true;
  set_error("bad dtype %d", d);
  return false;
}

fi_status good_heads(int32_t q_heads, int32_t kv_heads, int32_t head_dim) {
  if (q_heads < 1 || kv_heads < 1 || q_heads % kv_heads) { set_error("%d query heads over %d key heads", q_heads, kv_heads); return FI_EINVAL; }
  if (head_dim < 1) { set_error("head_dim %d", head_dim); return FI_EINVAL; }
  if (head_dim > FI_MAX_HEAD_DIM || q_heads > 65535) { set_error("head_dim %d, %d heads: at most %d and 65535", head_dim, q_heads, FI_MAX_HEAD_DIM); return FI_EUNSUPPORTED; }
  return FI_OK;
}

bool good_scale(float s) {
  if (std::isfinite(s) && s > 0.0f) return true;
  set_error("scale has to be finite and above zero");
  return false;
}

fi_status check_tree_sizes(const fi_tree_attention_args& a) {
  if (!good_dtype(a.dtype)) return FI_EINVAL;
  if (a.n_seqs < 0 || a.nodes < 0 || a.page_size < 1 || a.n_pages < 0 || a.table_columns < 0 || a.mask_words < 0 || a.max_nodes < 0 || a.max_length < 0) {
    set_error("negative size");
    return FI_EINVAL;
  }
  if (fi_status st = good_heads(a.q_heads, a.kv_heads, a.head_dim)) return st;
  if (!good_scale(a.scale)) return FI_EINVAL;
  if (a.nodes >= kRows || a.nodes * a.q_heads >= kRows || (int64_t)a.page_size * a.table_columns >= kRows || a.mask_words > 1024) {
    set_error("%lld nodes, %d x %d places, %d mask words: too many", (long long)a.nodes, a.table_columns, a.page_size, a.mask_words);
    return FI_EUNSUPPORTED;
  }
  return FI_OK;
}

fi_status check_q4_sizes(const fi_q4_matmul_args& a) {
  if (!good_dtype(a.dtype)) return FI_EINVAL;
  if (a.rows < 0 || a.inputs < 0 || a.outputs < 0 || a.group < 1 || a.inputs % a.group) { set_error("%d x %d x %d in groups of %d", a.rows, a.outputs, a.inputs, a.group); return FI_EINVAL; }
  if (a.group != 32 && a.group != 64 && a.group % 128) { set_error("groups of %d: 32, 64 and multiples of 128 are covered", a.group); return FI_EUNSUPPORTED; }
  if (a.rows > 1 << 19 || a.inputs > 1 << 24 || a.outputs > 1 << 24) { set_error("%d x %d x %d: too many", a.rows, a.outputs, a.inputs); return FI_EUNSUPPORTED; }
  return FI_OK;
}

bool good_workspace(const void* p, uint64_t bytes, uint64_t need) {
  if (!need) return true;
  if (!good(p, 16, "workspace")) return false;
  if (bytes < need) { set_error("the workspace has %llu bytes, %llu are needed", (unsigned long long)bytes, (unsigned long long)need); return false; }
  return true;
}

}  // namespace
}  // namespace fi

using namespace fi;

extern "C" {

fi_status fi_qk_norm_rope(const fi_qk_norm_rope_args* args, void* hip_stream) {
  if (!args) { set_error("null argument"); return FI_EINVAL; }
  const fi_qk_norm_rope_args& a = *args;
  if (!good_dtype(a.dtype)) return FI_EINVAL;
  if (a.tokens < 0 || a.q_heads < 0 || a.kv_heads < 0 || a.head_dim < 1) { set_error("%d tokens, %d and %d heads of %d", a.tokens, a.q_heads, a.kv_heads, a.head_dim); return FI_EINVAL; }
  if (a.rot_dim < 0 || a.rot_dim % 2 || a.rot_dim > a.head_dim) { set_error("rot_dim %d of head_dim %d", a.rot_dim, a.head_dim); return FI_EINVAL; }
  if (a.interleaved < 0 || a.interleaved > 1) { set_error("interleaved is 0 or 1"); return FI_EINVAL; }
  if (a.n_axes < 1 || a.n_axes > FI_MAX_AXES) { set_error("%d axes", a.n_axes); return FI_EINVAL; }
  int64_t pairs = 0;
  for (int i = 0; i < a.n_axes; ++i) {
    if (a.sections[i] < 0) { set_error("section %d is negative", i); return FI_EINVAL; }
    pairs += a.sections[i];
  }
  if (pairs != a.rot_dim / 2) { set_error("the sections hold %lld pairs, rot_dim %d", (long long)pairs, a.rot_dim / 2); return FI_EINVAL; }
  if (!(a.eps >= 0.0f) || !std::isfinite(a.eps)) { set_error("eps has to be finite and not negative"); return FI_EINVAL; }
  if (a.head_dim > FI_MAX_HEAD_DIM || a.q_heads > 65535 || a.kv_heads > 65535) { set_error("head_dim %d, %d and %d heads: too many", a.head_dim, a.q_heads, a.kv_heads); return FI_EUNSUPPORTED; }
  if (a.tokens == 0 || a.q_heads + a.kv_heads == 0) return FI_OK;
  const int es = elem_size(a.dtype), D = a.head_dim;
  if (a.rot_dim && (!good(a.positions, 4, "positions") || !good(a.inv_freq, 4, "inv_freq"))) return FI_EINVAL;
  if (a.q_heads && (!good(a.q, es, "q") || !good(a.q_out, es, "q_out") || !good_strides(a.q_strides, 2, "q") || !good_strides(a.q_out_strides, 2, "q_out") ||
                    !apart({a.q_out_strides[0], a.q_out_strides[1]}, {a.tokens, a.q_heads}, D, "q_out"))) return FI_EINVAL;
  if ((a.q_weight && !good(a.q_weight, 4, "q_weight")) || (a.k_weight && !good(a.k_weight, 4, "k_weight"))) return FI_EINVAL;
  if (a.kv_heads) {
    if (a.slots && (!good(a.slots, 8, "slots") || a.page_size < 1 || a.n_slots < 0)) {
      if (a.page_size < 1 || a.n_slots < 0) set_error("pages of %d tokens, %lld slots", a.page_size, (long long)a.n_slots);
      return FI_EINVAL;
    }
    const bool kept = !a.slots || a.n_slots > 0;   // a cache without pages has no address, and takes nothing
    if (!good(a.k, es, "k") || (kept && !good(a.k_out, es, "k_out")) || !good_strides(a.k_strides, 2, "k") || !good_strides(a.k_out_strides, 3, "k_out")) return FI_EINVAL;
    if (kept && !a.v != !a.v_out) { set_error("v and v_out come together"); return FI_EINVAL; }
    if (a.v && (!good(a.v, es, "v") || (kept && !good(a.v_out, es, "v_out")) || !good_strides(a.v_strides, 2, "v") || !good_strides(a.v_out_strides, 3, "v_out"))) return FI_EINVAL;
    const int64_t pages = a.slots ? a.n_slots / a.page_size + (a.n_slots % a.page_size != 0) : 1, rows = a.slots ? a.page_size : a.tokens;
    for (int t = 0; t < (a.v ? 2 : 1); ++t) {
      const int64_t* s = t ? a.v_out_strides : a.k_out_strides;
      if (!apart({s[0], s[1], s[2]}, {pages, rows, a.kv_heads}, D, t ? "v_out" : "k_out")) return FI_EINVAL;
    }
  }
  return done(launch_qk_norm_rope(a, hip_stream), "fi_qk_norm_rope");
}

fi_status fi_prompt_attention(const fi_prompt_attention_args* args, void* hip_stream) {
  if (!args) { set_error("null argument"); return FI_EINVAL; }
  const fi_prompt_attention_args& a = *args;
  if (!good_dtype(a.dtype)) return FI_EINVAL;
  if (a.n_seqs < 0 || a.q_tokens < 0 || a.k_tokens < 0) { set_error("negative size"); return FI_EINVAL; }
  if (a.causal < 0 || a.causal > 1) { set_error("causal is 0 or 1"); return FI_EINVAL; }
  if (fi_status st = good_heads(a.q_heads, a.kv_heads, a.head_dim)) return st;
  if (!good_scale(a.scale)) return FI_EINVAL;
  if (a.q_tokens >= kRows || a.k_tokens >= kRows || (a.q_tokens + 64ll * a.n_seqs) * a.q_heads >= 32 * kRows) {
    set_error("%lld queries, %lld keys: too many", (long long)a.q_tokens, (long long)a.k_tokens);
    return FI_EUNSUPPORTED;
  }
  if (a.n_seqs == 0 || a.q_tokens == 0) return FI_OK;
  const int es = elem_size(a.dtype);
  if (!good(a.q, es, "q") || !good(a.out, es, "out") || !good(a.cu_q, 4, "cu_q") || !good(a.cu_k, 4, "cu_k")) return FI_EINVAL;
  if (a.k_tokens && (!good(a.k, es, "k") || !good(a.v, es, "v"))) return FI_EINVAL;
  if (!good_strides(a.q_strides, 2, "q") || !good_strides(a.k_strides, 2, "k") || !good_strides(a.v_strides, 2, "v") || !good_strides(a.out_strides, 2, "out")) return FI_EINVAL;
  if (!apart({a.out_strides[0], a.out_strides[1]}, {a.q_tokens, a.q_heads}, a.head_dim, "out")) return FI_EINVAL;
  return done(launch_prompt_attention(a, hip_stream), "fi_prompt_attention");
}

fi_status fi_tree_attention_workspace(const fi_tree_attention_args* args, uint64_t* bytes) {
  if (!args || !bytes) { set_error("null argument"); return FI_EINVAL; }
  if (fi_status st = check_tree_sizes(*args)) return st;
  *bytes = tree_workspace(*args);
  return FI_OK;
}

fi_status fi_tree_attention(const fi_tree_attention_args* args, void* hip_stream) {
  if (!args) { set_error("null argument"); return FI_EINVAL; }
  const fi_tree_attention_args& a = *args;
  if (fi_status st = check_tree_sizes(a)) return st;
  if (a.n_seqs == 0 || a.nodes == 0 || a.max_nodes == 0) return FI_OK;
  const int es = elem_size(a.dtype);
  if (!good(a.q, es, "q") || !good(a.out, es, "out") || !good(a.cached, 4, "cached") || !good(a.cu_nodes, 4, "cu_nodes")) return FI_EINVAL;
  if (a.n_pages && a.table_columns && (!good(a.k_cache, es, "k_cache") || !good(a.v_cache, es, "v_cache") || !good(a.block_table, 4, "block_table"))) return FI_EINVAL;
  if (a.mask && (!good(a.mask, 8, "mask") || a.mask_words < 1)) {
    if (a.mask_words < 1) set_error("a mask of %d words", a.mask_words);
    return FI_EINVAL;
  }
  if (!good_strides(a.q_strides, 2, "q") || !good_strides(a.k_strides, 3, "k_cache") || !good_strides(a.v_strides, 3, "v_cache") || !good_strides(a.out_strides, 2, "out") ||
      !good_strides(&a.table_stride, 1, "block_table")) return FI_EINVAL;
  if (!apart({a.out_strides[0], a.out_strides[1]}, {a.nodes, a.q_heads}, a.head_dim, "out")) return FI_EINVAL;
  if (!good_workspace(a.workspace, a.workspace_bytes, tree_workspace(a))) return FI_EINVAL;
  return done(launch_tree_attention(a, hip_stream), "fi_tree_attention");
}

fi_status fi_q4_matmul_workspace(const fi_q4_matmul_args* args, uint64_t* bytes) {
  if (!args || !bytes) { set_error("null argument"); return FI_EINVAL; }
  if (fi_status st = check_q4_sizes(*args)) return st;
  *bytes = q4_workspace(*args);
  return FI_OK;
}

fi_status fi_q4_matmul(const fi_q4_matmul_args* args, void* hip_stream) {
  if (!args) { set_error("null argument"); return FI_EINVAL; }
  const fi_q4_matmul_args& a = *args;
  if (fi_status st = check_q4_sizes(a)) return st;
  if (a.rows == 0 || a.outputs == 0) return FI_OK;
  const int es = elem_size(a.dtype);
  if (!good(a.out, es, "out")) return FI_EINVAL;
  if (a.inputs && (!good(a.x, es, "x") || !good(a.w, 1, "w") || !good(a.scales, 4, "scales"))) return FI_EINVAL;
  const int64_t strides[5] = {a.x_stride, a.w_stride, a.scales_stride, a.zeros ? a.zeros_stride : 0, a.out_stride};
  if (!good_strides(strides, 5, "x, w, scales, zeros or out") || !apart({a.out_stride}, {a.rows}, a.outputs, "out")) return FI_EINVAL;
  if (!good_workspace(a.workspace, a.workspace_bytes, q4_workspace(a))) return FI_EINVAL;
  return done(launch_q4_matmul(a, hip_stream), "fi_q4_matmul");
}

}  // extern "C"
