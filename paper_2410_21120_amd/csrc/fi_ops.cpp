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

template <typename A>
fi_status check_tree_sizes(const A& a) {
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

// Codes and scales of one half of a 4-bit cache.
bool good_fp4(const uint8_t* codes, const int64_t* code_strides, const uint8_t* scales, const int64_t* scale_strides, const char* name) {
  if (!good(codes, 4, name) || !good(scales, 1, name) || !good_strides(code_strides, 3, name) || !good_strides(scale_strides, 3, name)) return false;
  for (int i = 0; i < 3; ++i)
    if (code_strides[i] % 4) { set_error("%s: a stride of %lld bytes between codes, multiples of 4 are covered", name, (long long)code_strides[i]); return false; }
  return true;
}
fi_status good_fp4_heads(int32_t kv_heads, int32_t head_dim) {
  if (kv_heads < 0 || head_dim < 1) { set_error("%d heads of %d", kv_heads, head_dim); return FI_EINVAL; }
  if (head_dim % 8 || head_dim > FI_MAX_HEAD_DIM || kv_heads > 65535) { set_error("%d heads of %d: multiples of 8 up to %d, and 65535 heads are covered", kv_heads, head_dim, FI_MAX_HEAD_DIM); return FI_EUNSUPPORTED; }
  return FI_OK;
}

struct Range { const void* p; uint64_t bytes; const char* name; };
// The outputs share no memory with each other or an input.
bool separate(std::initializer_list<Range> outputs, std::initializer_list<Range> inputs) {
  auto meet = [](const Range& x, const Range& y) {
    const uintptr_t a = reinterpret_cast<uintptr_t>(x.p), b = reinterpret_cast<uintptr_t>(y.p);
    if (!x.p || !y.p || !x.bytes || !y.bytes || a >= b + y.bytes || b >= a + x.bytes) return false;
    set_error("%s overlaps %s", x.name, y.name);
    return true;
  };
  for (const Range* x = outputs.begin(); x != outputs.end(); ++x) {
    for (const Range* y = x + 1; y != outputs.end(); ++y)
      if (meet(*x, *y)) return false;
    for (const Range& y : inputs)
      if (meet(*x, y)) return false;
  }
  return true;
}
uint64_t reach(int64_t rows, int64_t stride, int64_t row, int size) { return rows > 0 && row > 0 ? (uint64_t)((rows - 1) * stride + row) * size : 0; }

fi_status check_beam_sizes(const fi_beam_select_args& a) {
  if (!good_dtype(a.dtype)) return FI_EINVAL;
  if (a.n_seqs < 0 || a.beams < 1 || a.keep < 1 || a.vocab < 0) { set_error("%d sequences of %d beams, %d kept, %d tokens", a.n_seqs, a.beams, a.keep, a.vocab); return FI_EINVAL; }
  if (a.end >= a.vocab && a.end >= 0) { set_error("token %d of %d ends a sequence", a.end, a.vocab); return FI_EINVAL; }
  if (a.beams > FI_MAX_BEAMS || a.keep > FI_MAX_BEAMS || (int64_t)a.beams * a.vocab >= kRows || (int64_t)a.n_seqs * a.beams >= kRows || (int64_t)a.n_seqs * a.keep >= kRows) {
    set_error("%d sequences of %d beams, %d kept, %d tokens: too many", a.n_seqs, a.beams, a.keep, a.vocab);
    return FI_EUNSUPPORTED;
  }
  return FI_OK;
}

constexpr int32_t kTableRows = 1 << 16, kRoom = 1 << 16;
fi_status check_table(int32_t rows, int32_t columns, int32_t n_pages, int32_t n_caches) {
  if (rows < 0 || columns < 0 || n_pages < 0 || n_caches < 0) { set_error("negative size"); return FI_EINVAL; }
  if (rows > kTableRows || columns >= kRows || n_pages >= kRows || n_caches > FI_MAX_PAGE_CACHES) {
    set_error("%d rows of %d columns, %d pages of %d caches: too many", rows, columns, n_pages, n_caches);
    return FI_EUNSUPPORTED;
  }
  return FI_OK;
}
fi_status check_fork_sizes(const fi_fork_pages_args& a) {
  if (a.page_size < 1 || a.room < 0 || a.new_rows < 0) { set_error("pages of %d tokens, room for %d, %d rows", a.page_size, a.room, a.new_rows); return FI_EINVAL; }
  if (fi_status st = check_table(a.rows, a.columns, a.n_pages, a.n_caches)) return st;
  if (a.new_rows > kTableRows || a.room > kRoom || (int64_t)a.page_size * a.columns >= kRows) {
    set_error("%d rows, %d columns of %d tokens, room for %d: too many", a.new_rows, a.columns, a.page_size, a.room);
    return FI_EUNSUPPORTED;
  }
  if (!a.parents && a.new_rows != a.rows) { set_error("%d rows continue %d without parents", a.new_rows, a.rows); return FI_EINVAL; }
  return FI_OK;
}
fi_status good_caches(const fi_page_cache* caches, int32_t n, int32_t n_pages) {
  if (n && !caches) { set_error("caches is null"); return FI_EINVAL; }
  for (int i = 0; i < n; ++i) {
    const fi_page_cache& c = caches[i];
    if (c.page_bytes < 0 || c.page_stride < 0 || (n_pages > 1 && c.page_stride < c.page_bytes) || (n_pages && c.page_bytes && !c.base)) {
      set_error("cache %d: pages of %lld bytes, %lld apart", i, (long long)c.page_bytes, (long long)c.page_stride);
      return FI_EINVAL;
    }
    if (c.page_bytes > 1ll << 32 || c.page_stride > kStride) { set_error("cache %d: pages of %lld bytes, %lld apart: too large", i, (long long)c.page_bytes, (long long)c.page_stride); return FI_EUNSUPPORTED; }
  }
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

fi_status fi_fp4_cache_write(const fi_fp4_cache_write_args* args, void* hip_stream) {
  if (!args) { set_error("null argument"); return FI_EINVAL; }
  const fi_fp4_cache_write_args& a = *args;
  if (!good_dtype(a.dtype)) return FI_EINVAL;
  if (a.tokens < 0 || a.page_size < 1 || a.n_slots < 0) { set_error("%d tokens, pages of %d, %lld slots", a.tokens, a.page_size, (long long)a.n_slots); return FI_EINVAL; }
  if (fi_status st = good_fp4_heads(a.kv_heads, a.head_dim)) return st;
  if (a.tokens == 0 || a.kv_heads == 0) return FI_OK;
  if (!a.v && (a.v_codes || a.v_scales || a.v_held)) { set_error("v and its cache come together"); return FI_EINVAL; }
  const int es = elem_size(a.dtype);
  if (!good(a.slots, 8, "slots")) return FI_EINVAL;
  const int64_t pages = a.n_slots / a.page_size + (a.n_slots % a.page_size != 0), D = a.head_dim, blocks = (D + FI_FP4_BLOCK - 1) / FI_FP4_BLOCK;
  for (int t = 0; t < (a.v ? 2 : 1); ++t) {
    const char* const name = t ? "v" : "k";
    const int64_t* const held = t ? a.v_held_strides : a.k_held_strides;
    const int64_t* const codes = t ? a.v_codes_strides : a.k_codes_strides;
    const int64_t* const scales = t ? a.v_scales_strides : a.k_scales_strides;
    const void* const h = t ? a.v_held : a.k_held;
    if (!good(t ? a.v : a.k, es, name) || !good_strides(t ? a.v_strides : a.k_strides, 2, name)) return FI_EINVAL;
    if (h && (!good(h, es, t ? "v_held" : "k_held") || !good_strides(held, 2, name) || !apart({held[0], held[1]}, {a.tokens, a.kv_heads}, D, t ? "v_held" : "k_held"))) return FI_EINVAL;
    if (a.n_slots == 0) continue;   // a cache without pages has no address, and takes nothing
    if (!good_fp4(t ? a.v_codes : a.k_codes, codes, t ? a.v_scales : a.k_scales, scales, t ? "v_codes or v_scales" : "k_codes or k_scales")) return FI_EINVAL;
    if (!apart({codes[0], codes[1], codes[2]}, {pages, a.page_size, a.kv_heads}, D / 2, t ? "v_codes" : "k_codes") ||
        !apart({scales[0], scales[1], scales[2]}, {pages, a.page_size, a.kv_heads}, blocks, t ? "v_scales" : "k_scales")) return FI_EINVAL;
  }
  return done(launch_fp4_cache_write(a, hip_stream), "fi_fp4_cache_write");
}

fi_status fi_fp4_tree_attention_workspace(const fi_fp4_tree_attention_args* args, uint64_t* bytes) {
  if (!args || !bytes) { set_error("null argument"); return FI_EINVAL; }
  if (fi_status st = check_tree_sizes(*args)) return st;
  if (fi_status st = good_fp4_heads(args->kv_heads, args->head_dim)) return st;
  *bytes = fp4_tree_workspace(*args);
  return FI_OK;
}

fi_status fi_fp4_tree_attention(const fi_fp4_tree_attention_args* args, void* hip_stream) {
  if (!args) { set_error("null argument"); return FI_EINVAL; }
  const fi_fp4_tree_attention_args& a = *args;
  if (fi_status st = check_tree_sizes(a)) return st;
  if (fi_status st = good_fp4_heads(a.kv_heads, a.head_dim)) return st;
  if (a.n_seqs == 0 || a.nodes == 0 || a.max_nodes == 0) return FI_OK;
  const int es = elem_size(a.dtype);
  if (!good(a.q, es, "q") || !good(a.out, es, "out") || !good(a.cached, 4, "cached") || !good(a.cu_nodes, 4, "cu_nodes")) return FI_EINVAL;
  if (a.n_pages && a.table_columns &&
      (!good_fp4(a.k_codes, a.k_codes_strides, a.k_scales, a.k_scales_strides, "k_codes or k_scales") ||
       !good_fp4(a.v_codes, a.v_codes_strides, a.v_scales, a.v_scales_strides, "v_codes or v_scales") || !good(a.block_table, 4, "block_table"))) return FI_EINVAL;
  if (a.mask && (!good(a.mask, 8, "mask") || a.mask_words < 1)) {
    if (a.mask_words < 1) set_error("a mask of %d words", a.mask_words);
    return FI_EINVAL;
  }
  if (!good_strides(a.q_strides, 2, "q") || !good_strides(a.out_strides, 2, "out") || !good_strides(&a.table_stride, 1, "block_table")) return FI_EINVAL;
  if (!apart({a.out_strides[0], a.out_strides[1]}, {a.nodes, a.q_heads}, a.head_dim, "out")) return FI_EINVAL;
  if (!good_workspace(a.workspace, a.workspace_bytes, fp4_tree_workspace(a))) return FI_EINVAL;
  return done(launch_fp4_tree_attention(a, hip_stream), "fi_fp4_tree_attention");
}

fi_status fi_beam_select_workspace(const fi_beam_select_args* args, uint64_t* bytes) {
  if (!args || !bytes) { set_error("null argument"); return FI_EINVAL; }
  if (fi_status st = check_beam_sizes(*args)) return st;
  *bytes = beam_workspace(*args);
  return FI_OK;
}

fi_status fi_beam_select(const fi_beam_select_args* args, void* hip_stream) {
  if (!args) { set_error("null argument"); return FI_EINVAL; }
  const fi_beam_select_args& a = *args;
  if (fi_status st = check_beam_sizes(a)) return st;
  if (a.end < 0 && (a.ended || a.ended_out)) { set_error("beams that have ended, and no token that ends them"); return FI_EINVAL; }
  if (a.n_seqs == 0) return FI_OK;
  const int64_t rows = (int64_t)a.n_seqs * a.beams, kept = (int64_t)a.n_seqs * a.keep;
  const int es = elem_size(a.dtype);
  if ((a.vocab && !good(a.logits, es, "logits")) || !good(a.scores, 4, "scores") || !good(a.tokens_out, 4, "tokens_out") || !good(a.parents_out, 4, "parents_out") ||
      !good(a.scores_out, 4, "scores_out") || (a.end >= 0 && !good(a.ended_out, 1, "ended_out")) || !good_strides(&a.logits_stride, 1, "logits")) return FI_EINVAL;
  if (!good_workspace(a.workspace, a.workspace_bytes, beam_workspace(a))) return FI_EINVAL;
  if (!separate({{a.tokens_out, (uint64_t)kept * 4, "tokens_out"}, {a.parents_out, (uint64_t)kept * 4, "parents_out"}, {a.scores_out, (uint64_t)kept * 4, "scores_out"},
                 {a.ended_out, (uint64_t)kept, "ended_out"}, {a.workspace, beam_workspace(a), "the workspace"}},
                {{a.scores, (uint64_t)rows * 4, "scores"}, {a.ended, (uint64_t)rows, "ended"}, {a.logits, reach(rows, a.logits_stride, a.vocab, es), "logits"}})) return FI_EINVAL;
  return done(launch_beam_select(a, hip_stream), "fi_beam_select");
}

fi_status fi_fork_pages_workspace(const fi_fork_pages_args* args, uint64_t* bytes) {
  if (!args || !bytes) { set_error("null argument"); return FI_EINVAL; }
  if (fi_status st = check_fork_sizes(*args)) return st;
  *bytes = fork_workspace(*args);
  return FI_OK;
}

fi_status fi_fork_pages(const fi_fork_pages_args* args, void* hip_stream) {
  if (!args) { set_error("null argument"); return FI_EINVAL; }
  const fi_fork_pages_args& a = *args;
  if (fi_status st = check_fork_sizes(a)) return st;
  if (fi_status st = good_caches(a.caches, a.n_caches, a.n_pages)) return st;
  if (a.rows == 0 && a.new_rows == 0 && a.n_pages == 0) return FI_OK;
  const bool entries = a.columns > 0;
  if ((a.rows && ((entries && !good(a.block_table, 4, "block_table")) || !good(a.lengths, 4, "lengths") || (a.held && !good(a.held, 4, "held")))) ||
      (a.n_pages && (!good(a.refs, 4, "refs") || !good(a.refs_out, 4, "refs_out"))) || (a.new_rows && a.parents && !good(a.parents, 4, "parents")) ||
      (a.new_rows && ((entries && !good(a.table_out, 4, "table_out")) || !good(a.lengths_out, 4, "lengths_out") || !good(a.held_out, 4, "held_out") ||
                      (a.room && !good(a.slots_out, 8, "slots_out"))))) return FI_EINVAL;
  const int64_t strides[2] = {a.table_stride, a.table_out_stride};
  if (!good_strides(strides, 2, "block_table or table_out") || !apart({a.table_out_stride}, {a.new_rows}, a.columns, "table_out")) return FI_EINVAL;
  if (!good_workspace(a.workspace, a.workspace_bytes, fork_workspace(a))) return FI_EINVAL;
  if (!separate({{a.table_out, reach(a.new_rows, a.table_out_stride, a.columns, 4), "table_out"}, {a.lengths_out, 4ull * a.new_rows, "lengths_out"},
                 {a.held_out, 4ull * a.new_rows, "held_out"}, {a.refs_out, 4ull * a.n_pages, "refs_out"}, {a.slots_out, 8ull * a.new_rows * a.room, "slots_out"},
                 {a.workspace, fork_workspace(a), "the workspace"}},
                {{a.block_table, reach(a.rows, a.table_stride, a.columns, 4), "block_table"}, {a.lengths, 4ull * a.rows, "lengths"}, {a.held, 4ull * a.rows, "held"},
                 {a.refs, 4ull * a.n_pages, "refs"}, {a.parents, 4ull * a.new_rows, "parents"}})) return FI_EINVAL;
  return done(launch_fork_pages(a, hip_stream), "fi_fork_pages");
}

fi_status fi_compact_pages_workspace(const fi_compact_pages_args* args, uint64_t* bytes) {
  if (!args || !bytes) { set_error("null argument"); return FI_EINVAL; }
  if (fi_status st = check_table(args->rows, args->columns, args->n_pages, args->n_caches)) return st;
  *bytes = compact_workspace(*args);
  return FI_OK;
}

fi_status fi_compact_pages(const fi_compact_pages_args* args, void* hip_stream) {
  if (!args) { set_error("null argument"); return FI_EINVAL; }
  const fi_compact_pages_args& a = *args;
  if (fi_status st = check_table(a.rows, a.columns, a.n_pages, a.n_caches)) return st;
  if (fi_status st = good_caches(a.caches, a.n_caches, a.n_pages)) return st;
  const bool table = a.rows && a.columns;
  if (!good(a.live_out, 4, "live_out") || (table && (!good(a.block_table, 4, "block_table") || !good(a.table_out, 4, "table_out"))) ||
      (a.n_pages && (!good(a.refs, 4, "refs") || !good(a.refs_out, 4, "refs_out") || !good(a.moved_out, 4, "moved_out")))) return FI_EINVAL;
  const int64_t strides[2] = {a.table_stride, a.table_out_stride};
  if (!good_strides(strides, 2, "block_table or table_out") || !apart({a.table_out_stride}, {a.rows}, a.columns, "table_out")) return FI_EINVAL;
  if (!good_workspace(a.workspace, a.workspace_bytes, compact_workspace(a))) return FI_EINVAL;
  if (!separate({{a.table_out, reach(a.rows, a.table_out_stride, a.columns, 4), "table_out"}, {a.refs_out, 4ull * a.n_pages, "refs_out"},
                 {a.moved_out, 4ull * a.n_pages, "moved_out"}, {a.live_out, 4, "live_out"}, {a.workspace, compact_workspace(a), "the workspace"}},
                {{a.block_table, reach(a.rows, a.table_stride, a.columns, 4), "block_table"}, {a.refs, 4ull * a.n_pages, "refs"}})) return FI_EINVAL;
  return done(launch_compact_pages(a, hip_stream), "fi_compact_pages");
}

}  // extern "C"
