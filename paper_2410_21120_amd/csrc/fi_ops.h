// Launchers of the decoder operators: implemented in fi_rope.hip, fi_attn.hip, fi_q4.hip, fi_fp4.hip, fi_beam.hip and fi_pages.hip, called by fi_ops.cpp once the
// arguments are checked.  Each returns a hipError_t as int, or kTooLarge before it launches anything.
#pragma once

#include "fi_internal.h"

namespace fi {

constexpr int kTooLarge = -1;   // a launch would have 2^32 threads or more along its first dimension, which HIP does not take
inline bool one_launch(int64_t workgroups, int threads) { return workgroups < (1ll << 32) / threads; }

inline int32_t elem_size(int32_t dtype) { return dtype == FI_F32 ? 4 : 2; }

int launch_qk_norm_rope(const fi_qk_norm_rope_args& a, void* stream);
int launch_prompt_attention(const fi_prompt_attention_args& a, void* stream);
int launch_tree_attention(const fi_tree_attention_args& a, void* stream);
int launch_q4_matmul(const fi_q4_matmul_args& a, void* stream);
int launch_fp4_cache_write(const fi_fp4_cache_write_args& a, void* stream);
int launch_fp4_tree_attention(const fi_fp4_tree_attention_args& a, void* stream);
int launch_beam_select(const fi_beam_select_args& a, void* stream);
int launch_fork_pages(const fi_fork_pages_args& a, void* stream);
int launch_compact_pages(const fi_compact_pages_args& a, void* stream);
uint64_t q4_workspace(const fi_q4_matmul_args& a);
uint64_t tree_workspace(const fi_tree_attention_args& a);
uint64_t fp4_tree_workspace(const fi_fp4_tree_attention_args& a);
uint64_t beam_workspace(const fi_beam_select_args& a);
uint64_t fork_workspace(const fi_fork_pages_args& a);
uint64_t compact_workspace(const fi_compact_pages_args& a);

}  // namespace fi
