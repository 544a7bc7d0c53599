"""MI355X-native fused multi-model CNN inference (FusedInf hot path).

The product is the C-ABI library `libfusedinf.so` (see include/fusedinf.h); this
package is a thin ctypes binding with the same entry-point names.  Every step
of the path runs in the library's HIP kernels: nothing here computes.
"""
from .binding import *  # noqa: F401,F403
from .operators import (fi_beam_select, fi_beam_select_args, fi_beam_select_workspace, fi_compact_pages, fi_compact_pages_args, fi_compact_pages_workspace,  # noqa: F401
                        fi_fork_pages, fi_fork_pages_args, fi_fork_pages_workspace, fi_fp4_cache_write, fi_fp4_cache_write_args, fi_fp4_tree_attention,
                        fi_fp4_tree_attention_args, fi_fp4_tree_attention_workspace, fi_page_cache, fi_prompt_attention, fi_prompt_attention_args, fi_q4_matmul,
                        fi_q4_matmul_args, fi_q4_matmul_workspace, fi_qk_norm_rope, fi_qk_norm_rope_args, fi_tree_attention, fi_tree_attention_args,
                        fi_tree_attention_workspace, beam_select, compact_pages, fork_pages, fp4_cache, fp4_cache_write, fp4_tree_attention, prompt_attention, q4_matmul,
                        qk_norm_rope, tree_attention)
