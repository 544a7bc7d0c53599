"""The decoder operators on tensors: argument marshalling for the fi_* entry points of the same names.

qk_norm_rope, prompt_attention, tree_attention, q4_matmul, and for beams over a 4-bit cache fp4_cache_write,
fp4_tree_attention, beam_select, fork_pages and compact_pages take PyTorch tensors (device memory with a shape and
strides), check that they fit together, fill the argument struct of include/fusedinf.h and make the call on the tensors'
device and on `stream` (a hipStream_t as an integer; by default torch's current stream of that device).  Nothing here
computes; the checks and the structs are done in csrc/fi_tensors.cpp (a call of fi_qk_norm_rope or fi_q4_matmul takes the
host 3 to 4 us that way, in Python 11 and 8, more than the kernels of a decoding step).

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


class fi_fp4_cache_write_args(C.Structure):
    _fields_ = _fields("i:dtype i:tokens i:kv_heads i:head_dim i:page_size i:reserved l:n_slots p:k p:v p:slots p:k_codes p:k_scales p:v_codes p:v_scales p:k_held p:v_held "
                       "l:k_token l:k_head l:v_token l:v_head l:k_held_token l:k_held_head l:v_held_token l:v_held_head "
                       "l:k_codes_page l:k_codes_token l:k_codes_head l:k_scales_page l:k_scales_token l:k_scales_head "
                       "l:v_codes_page l:v_codes_token l:v_codes_head l:v_scales_page l:v_scales_token l:v_scales_head")


class fi_fp4_tree_attention_args(C.Structure):
    _fields_ = _fields("i:dtype i:n_seqs i:q_heads i:kv_heads i:head_dim i:page_size i:n_pages i:table_columns i:mask_words i:max_nodes i:max_length "
                       "f:scale l:nodes p:q p:k_codes p:k_scales p:v_codes p:v_scales p:block_table p:cached p:cu_nodes p:mask p:out p:workspace u:workspace_bytes "
                       "l:q_token l:q_head l:out_token l:out_head l:k_codes_page l:k_codes_token l:k_codes_head l:k_scales_page l:k_scales_token l:k_scales_head "
                       "l:v_codes_page l:v_codes_token l:v_codes_head l:v_scales_page l:v_scales_token l:v_scales_head l:table_stride")


class fi_beam_select_args(C.Structure):
    _fields_ = _fields("i:dtype i:n_seqs i:beams i:keep i:vocab i:end l:logits_stride p:logits p:scores p:ended p:tokens_out p:parents_out p:scores_out p:ended_out "
                       "p:workspace u:workspace_bytes")


class fi_page_cache(C.Structure):
    _fields_ = _fields("p:base l:page_stride l:page_bytes")


class fi_fork_pages_args(C.Structure):
    _fields_ = _fields("i:rows i:new_rows i:columns i:page_size i:n_pages i:room i:n_caches i:reserved l:table_stride l:table_out_stride p:block_table p:lengths p:held p:refs "
                       "p:parents p:caches p:table_out p:lengths_out p:held_out p:refs_out p:slots_out p:workspace u:workspace_bytes")


class fi_compact_pages_args(C.Structure):
    _fields_ = _fields("i:rows i:columns i:n_pages i:n_caches l:table_stride l:table_out_stride p:block_table p:refs p:caches p:table_out p:refs_out p:moved_out p:live_out "
                       "p:workspace u:workspace_bytes")


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


def fi_fp4_cache_write(args: fi_fp4_cache_write_args, stream_ptr=0) -> None:
    _b._check(_b.lib().fi_fp4_cache_write(C.byref(args), stream_ptr), "fi_fp4_cache_write")


def fi_fp4_tree_attention_workspace(args: fi_fp4_tree_attention_args) -> int:
    n = C.c_uint64(0)
    _b._check(_b.lib().fi_fp4_tree_attention_workspace(C.byref(args), C.byref(n)), "fi_fp4_tree_attention_workspace")
    return n.value


def fi_fp4_tree_attention(args: fi_fp4_tree_attention_args, stream_ptr=0) -> None:
    _b._check(_b.lib().fi_fp4_tree_attention(C.byref(args), stream_ptr), "fi_fp4_tree_attention")


def fi_beam_select_workspace(args: fi_beam_select_args) -> int:
    n = C.c_uint64(0)
    _b._check(_b.lib().fi_beam_select_workspace(C.byref(args), C.byref(n)), "fi_beam_select_workspace")
    return n.value


def fi_beam_select(args: fi_beam_select_args, stream_ptr=0) -> None:
    _b._check(_b.lib().fi_beam_select(C.byref(args), stream_ptr), "fi_beam_select")


def fi_fork_pages_workspace(args: fi_fork_pages_args) -> int:
    n = C.c_uint64(0)
    _b._check(_b.lib().fi_fork_pages_workspace(C.byref(args), C.byref(n)), "fi_fork_pages_workspace")
    return n.value


def fi_fork_pages(args: fi_fork_pages_args, stream_ptr=0) -> None:
    _b._check(_b.lib().fi_fork_pages(C.byref(args), stream_ptr), "fi_fork_pages")


def fi_compact_pages_workspace(args: fi_compact_pages_args) -> int:
    n = C.c_uint64(0)
    _b._check(_b.lib().fi_compact_pages_workspace(C.byref(args), C.byref(n)), "fi_compact_pages_workspace")
    return n.value


def fi_compact_pages(args: fi_compact_pages_args, stream_ptr=0) -> None:
    _b._check(_b.lib().fi_compact_pages(C.byref(args), stream_ptr), "fi_compact_pages")


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

    kinds = {"Byte": torch.uint8, "BFloat16": torch.bfloat16, "Float": torch.float32, "Int": torch.int32, "Long": torch.int64, "Bool": torch.bool}

    def room(shape, kind, stream, index):
        with torch.cuda.stream(torch.cuda.ExternalStream(stream, device=index)):
            return torch.empty(shape, dtype=kinds[kind], device=torch.device("cuda", index))

    entries = ("fi_qk_norm_rope", "fi_prompt_attention", "fi_tree_attention", "fi_q4_matmul", "fi_tree_attention_workspace", "fi_q4_matmul_workspace",
               "fi_fp4_cache_write", "fi_fp4_tree_attention", "fi_beam_select", "fi_fork_pages", "fi_compact_pages", "fi_fp4_tree_attention_workspace",
               "fi_beam_select_workspace", "fi_fork_pages_workspace", "fi_compact_pages_workspace")
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


FP4_BLOCK = 32


def fp4_cache(pages, page_size, kv_heads, head_dim, device="cuda"):
    """Half of an empty 4-bit cache, keys or values: codes uint8 [pages, page size, kv heads, head dim / 2] and scales uint8 [pages, page size, kv heads,
    head dim / 32, rounded up], a head's tokens of a page together in memory, as the kernels like them best."""
    import torch
    codes, scales = (torch.zeros((pages, kv_heads, page_size, n), dtype=torch.uint8, device=device) for n in (head_dim // 2, -(-head_dim // FP4_BLOCK)))
    return codes.permute(0, 2, 1, 3), scales.permute(0, 2, 1, 3)


def fp4_cache_write(k, v, slots, k_codes, k_scales, v_codes=None, v_scales=None, *, k_held=None, v_held=None, stream=None):
    """Writes k and v (or None) [tokens, kv heads, head dim] to their slots (int64 [tokens]) of a 4-bit cache: blocks of 32 values, E2M1 codes, two to a byte, the even value in
    the low half, times 2 ** (scale - 127); a token whose slot is outside of the cache is left out.  Codes and scales are shaped as fp4_cache makes them, with any
    strides; the head dim is a multiple of 8.  k_held, v_held: tensors like k and v that take what the cache then holds for the tokens.  Returns (k_held, v_held)."""
    return (_ext or _load()).fp4_cache_write(k, v, slots, k_codes, k_scales, v_codes, v_scales, k_held, v_held, stream)


def fp4_tree_attention(q, k_codes, k_scales, v_codes, v_scales, block_table, cached, cu_nodes, mask=None, *, scale=None, max_nodes=None, max_length=None, out=None,
                       workspace=None, stream=None):
    """tree_attention over a 4-bit cache, whose values enter the products exactly; fastest with pages of multiples of 16 tokens.  The other arguments are those of tree_attention.  workspace: uint8,
    fi_fp4_tree_attention_workspace bytes; made here if None.  Returns out [nodes, q heads, head dim]."""
    return (_ext or _load()).fp4_tree_attention(q, k_codes, k_scales, v_codes, v_scales, block_table, cached, cu_nodes, mask, scale, max_nodes, max_length, out, workspace, stream)


def beam_select(logits, scores, *, keep=None, end=None, ended=None, tokens_out=None, parents_out=None, scores_out=None, ended_out=None, workspace=None, stream=None):
    """The `keep` (default: beams) best continuations of every sequence: logits [sequences * beams, vocabulary], bf16 or fp32; scores fp32 [sequences, beams], to which the
    log-softmax of the logits is added.  Best first; equal scores by beam, then the larger logit, then the lower token first.  A logit of minus
    infinity masks its token; beams with score minus infinity, and rows with a NaN or plus infinity, have no continuations; where there are fewer than `keep`, token and
    parent are -1.
    end: the token that ends a sequence; ended bool [sequences, beams]: beams that have, and go on as themselves (token `end`, score unchanged).
    Returns tokens and parents (rows of logits) int32, scores fp32, and with end bool ended, else None, all [sequences, keep]."""
    return (_ext or _load()).beam_select(logits, scores, keep, end, ended, tokens_out, parents_out, scores_out, ended_out, workspace, stream)


def fork_pages(block_table, lengths, refs, parents=None, *, page_size, held=None, room=0, caches=(), table_out=None, lengths_out=None, held_out=None, refs_out=None,
               slots_out=None, workspace=None, stream=None):
    """The rows of a block table after a selection.  block_table int32 [rows, columns]; lengths int32 [rows]: committed tokens; held int32 [rows]: tokens that a
    row has pages for (default: lengths); refs int32 [pages]: how often a page is held, 0: free.  New row i continues row parents[i] (int32; -1: it is empty; None: row i
    itself), whose pages of committed tokens it shares; everything else that rows held is let go.  With room every continuing row gets pages for so many
    tokens more, the lowest free ones, in the order of the rows; a partly filled last page that others hold is copied first, in every tensor of `caches` [pages, ...].
    Where pages run out, a row gets nothing, as does one that would write over what such a row holds: its held is its length, its slots are -1.  No output may overlap an input.
    Returns table int32 [new rows, columns] (-1 behind a row's pages), lengths, held, refs, and slots int64 [new rows, room] of the tokens to come."""
    return (_ext or _load()).fork_pages(block_table, lengths, refs, parents, page_size, held, room, caches, table_out, lengths_out, held_out, refs_out, slots_out, workspace, stream)


def compact_pages(block_table, refs, *, caches=(), table_out=None, refs_out=None, moved_out=None, live_out=None, workspace=None, stream=None):
    """Moves the pages in use (refs > 0) of every tensor of `caches` [pages, ...] to the lowest numbers: those above move into the free ones below, in ascending order.
    Returns the renumbered table int32 [rows, columns] and refs int32 [pages], moved int32 [pages]: the new number of every page, -1 for free ones, and
    live int32 [1]: pages in use.  No output may overlap an input."""
    return (_ext or _load()).compact_pages(block_table, refs, caches, table_out, refs_out, moved_out, live_out, workspace, stream)
