"""The decoder operators on tensors: argument marshalling for the fi_* entry points of the same names.

qk_norm_rope, prompt_attention, tree_attention and q4_matmul take PyTorch tensors (device memory with a shape and strides),
check that they fit together, fill the argument struct of include/fusedinf.h and make the call on the tensors' device and on
`stream` (a hipStream_t as an integer; by default torch's current stream of that device).  Nothing here computes; the checks
and the structs are done in csrc/fi_tensors.cpp (a call of fi_qk_norm_rope or fi_q4_matmul takes the host 3 to 4 us that way, in
Python 11 and 8, more than the kernels of a decoding step).

A tensor that is used on another stream than the one it was made on is the caller's to order, as for any launch.  What a call makes
itself (outputs that are None, workspaces) comes from the memory that torch keeps for the call's stream, so `stream` has nothing to wait
for there; such an output belongs to that stream.  There are no gradients: a tensor that requires one is refused
unless torch's gradient mode is off, and outputs count as changed in place.  ValueError and TypeError tell what does not fit; what the library itself refuses is FiError.
"""
from __future__ import annotations

import ctypes as C
import os

from . import binding as _b
from . import build as _build

FI_MAX_AXES, FI_MAX_HEAD_DIM = 4, 256
_I32, _I64, _P, _F = C.c_int32, C.c_int64, C.c_void_p, C.c_float


def _fields(text):
    kinds = {"i": _I32, "l": _I64, "p": _P, "f": _F, "u": C.c_uint64}
    return [(name, kinds[kind]) for kind, name in (word.split(":") for word in text.split())]


# The structs of the header, their small arrays as single fields (same layout), so that a call fills them in one go.
class fi_qk_norm_rope_args(C.Structure):
    _fields_ = _fields("i:dtype i:tokens i:q_heads i:kv_heads i:head_dim i:rot_dim i:interleaved i:n_axes i:section0 i:section1 i:section2 i:section3 "
                       "f:eps i:page_size l:n_slots p:q p:k p:v p:q_weight p:k_weight p:positions p:inv_freq p:slots p:q_out p:k_out p:v_out "
                       "l:q_token l:q_head l:k_token l:k_head l:v_token l:v_head l:q_out_token l:q_out_head "
                       "l:k_out_page l:k_out_token l:k_out_head l:v_out_page l:v_out_token l:v_out_head")


class fi_prompt_attention_args(C.Structure):
    _fields_ = _fields("i:dtype i:n_seqs i:q_heads i:kv_heads i:head_dim i:causal f:scale i:reserved l:q_tokens l:k_tokens "
                       "p:q p:k p:v p:cu_q p:cu_k p:out l:q_token l:q_head l:k_token l:k_head l:v_token l:v_head l:out_token l:out_head")


class fi_tree_attention_args(C.Structure):
    _fields_ = _fields("i:dtype i:n_seqs i:q_heads i:kv_heads i:head_dim i:page_size i:n_pages i:table_columns i:mask_words i:max_nodes i:max_length "
                       "f:scale l:nodes p:q p:k_cache p:v_cache p:block_table p:cached p:cu_nodes p:mask p:out p:workspace u:workspace_bytes "
                       "l:q_token l:q_head l:out_token l:out_head l:k_page l:k_token l:k_head l:v_page l:v_token l:v_head l:table_stride")


class fi_q4_matmul_args(C.Structure):
    _fields_ = _fields("i:dtype i:rows i:inputs i:outputs i:group i:reserved p:x p:w p:scales p:zeros p:out p:workspace u:workspace_bytes "
                       "l:x_stride l:w_stride l:scales_stride l:zeros_stride l:out_stride")


# ---- the entry points, same names as the header --------------------------------------------
def fi_qk_norm_rope(args: fi_qk_norm_rope_args, stream_ptr=0) -> None:
    _b._check(_b.lib().fi_qk_norm_rope(C.byref(args), stream_ptr), "fi_qk_norm_rope")


def fi_prompt_attention(args: fi_prompt_attention_args, stream_ptr=0) -> None:
    _b._check(_b.lib().fi_prompt_attention(C.byref(args), stream_ptr), "fi_prompt_attention")


def fi_tree_attention_workspace(args: fi_tree_attention_args) -> int:
    n = C.c_uint64(0)
    _b._check(_b.lib().fi_tree_attention_workspace(C.byref(args), C.byref(n)), "fi_tree_attention_workspace")
    return n.value


def fi_tree_attention(args: fi_tree_attention_args, stream_ptr=0) -> None:
    _b._check(_b.lib().fi_tree_attention(C.byref(args), stream_ptr), "fi_tree_attention")


def fi_q4_matmul_workspace(args: fi_q4_matmul_args) -> int:
    n = C.c_uint64(0)
    _b._check(_b.lib().fi_q4_matmul_workspace(C.byref(args), C.byref(n)), "fi_q4_matmul_workspace")
    return n.value


def fi_q4_matmul(args: fi_q4_matmul_args, stream_ptr=0) -> None:
    _b._check(_b.lib().fi_q4_matmul(C.byref(args), stream_ptr), "fi_q4_matmul")


# ---- on tensors ------------------------------------------------------------------------------
_ext = None


def _load():
    """The extension, bound to the library's entry points."""
    global _ext
    import torch   # (its libraries are the extension's)
    library = _b.lib()
    if not os.path.exists(_build.TENSORS):
        _build.build_tensors()
    from . import _tensors

    kinds = {"Byte": torch.uint8, "BFloat16": torch.bfloat16, "Float": torch.float32}

    def room(shape, kind, stream, index):
        with torch.cuda.stream(torch.cuda.ExternalStream(stream, device=index)):
            return torch.empty(shape, dtype=kinds[kind], device=torch.device("cuda", index))

    entries = ("fi_qk_norm_rope", "fi_prompt_attention", "fi_tree_attention", "fi_q4_matmul", "fi_tree_attention_workspace", "fi_q4_matmul_workspace")
    stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda index: torch.cuda.current_stream(index).cuda_stream)
    _tensors.bind(*(C.cast(getattr(library, name), C.c_void_p).value for name in entries), _b._check, stream, room)
    _ext = _tensors
    return _ext


def qk_norm_rope(q, k, v, positions, inv_freq, *, q_weight=None, k_weight=None, eps=1e-6, sections=None, interleaved=False, slots=None,
                 q_out=None, k_out=None, v_out=None, stream=None):
    """Norms every head of q [tokens, q heads, head dim] and k [tokens, kv heads, head dim], rotates them by their positions, copies v.

    positions: int32 [tokens] or [tokens, axes]; inv_freq: fp32 [pairs], turned by the axes in order, sections[a] pairs each.
    q_weight, k_weight: fp32 [head dim].  With slots (int64 [tokens]) k_out and v_out are paged caches [pages, page size, kv heads,
    head dim] and a token goes to place slot % page size of page slot // page size, or nowhere if the slot is outside;
    without, they are [tokens, kv heads, head dim] and made here if None.  v may be None.  Returns (q_out, k_out, v_out)."""
    return (_ext or _load()).qk_norm_rope(q, k, v, positions, inv_freq, q_weight, k_weight, eps, interleaved, sections, slots, q_out, k_out, v_out, stream)


def prompt_attention(q, k, v, cu_q, cu_k=None, *, causal=True, scale=None, out=None, stream=None):
    """softmax(scale * q k^T) v over packed sequences: q [query tokens, q heads, head dim], k and v [key tokens, kv heads, head dim], cu_q and
    cu_k (default: cu_q) int32 [sequences + 1] the offsets of the sequences.  causal: the last query of a sequence sees all its keys.
    scale: head dim ** -0.5 by default.  Returns out [query tokens, q heads, head dim]."""
    return (_ext or _load()).prompt_attention(q, k, v, cu_q, cu_k, causal, scale, out, stream)


def tree_attention(q, k_cache, v_cache, block_table, cached, cu_nodes, mask=None, *, scale=None, max_nodes=None, max_length=None, out=None, workspace=None,
                   stream=None):
    """Attention of drafted trees, or single tokens, over a paged cache.

    q [nodes, q heads, head dim], packed by cu_nodes (int32 [sequences + 1]); k_cache and v_cache [pages, page size, kv heads, head dim];
    block_table int32 [sequences, columns]; cached int32 [sequences]: committed tokens, whose pages the nodes' own keys and values follow;
    mask int64 [nodes, words]: bit j of a row is set where the node sees node j of its sequence, None for chains.
    max_nodes: most nodes of a sequence, later ones are neither computed nor seen (default: all nodes), max_length: most committed tokens and nodes together (default: what
    the table can name; it guides how the work is shared out).  workspace: uint8, fi_tree_attention_workspace bytes; made here if
    None.  Returns out [nodes, q heads, head dim]."""
    return (_ext or _load()).tree_attention(q, k_cache, v_cache, block_table, cached, cu_nodes, mask, scale, max_nodes, max_length, out, workspace, stream)


def q4_matmul(x, w, scales, zeros=None, *, group=None, out=None, workspace=None, stream=None):
    """x [rows, inputs] times 4-bit weights: w uint8 [outputs, inputs / 2], two weights per byte, the even one in the low half; scales fp32 and
    zeros uint8 (8 where None) [outputs, inputs / group].  workspace: uint8, fi_q4_matmul_workspace bytes; made here if None.  Returns out [rows,
    outputs] in x's type."""
    return (_ext or _load()).q4_matmul(x, w, scales, zeros, group, out, workspace, stream)
