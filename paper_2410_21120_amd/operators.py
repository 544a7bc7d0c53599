"""The decoder operators on tensors: argument marshalling for the fi_* entry points of the same names.

qk_norm_rope, prompt_attention, tree_attention and q4_matmul take PyTorch tensors (device memory with a shape and strides),
check that they fit together, fill the argument struct of include/fusedinf.h and make the call on the tensors' device and on
`stream` (a hipStream_t as an integer; by default torch's current stream of that device).  Nothing here computes.

A tensor that is used on another stream than the one it was made on is the caller's to order, as for any launch.  ValueError
and TypeError tell what does not fit; what the library itself refuses is FiError.
"""
from __future__ import annotations

import ctypes as C

from . import binding as _b

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
# A decoding step is a handful of launches of a few microseconds, so the checks are short: a tensor's type, device index, shape and
# strides are read once each (0.05 to 0.1 us), and the stream is asked for as a number.
_torch = None
_dtypes = {}
_stream_of = None


def _setup():
    global _torch, _stream_of
    import torch
    _dtypes.update({torch.bfloat16: _b.FI_BF16, torch.float32: _b.FI_F32})
    _stream_of = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda index: torch.cuda.current_stream(index).cuda_stream)
    _torch = torch


def _kind(t, name):
    """fi_dtype, type and device index of the tensor that the others go by."""
    if _torch is None:
        _setup()
    dtype, index = t.dtype, t.get_device()
    if dtype not in _dtypes:
        raise TypeError(f"{name}: {dtype}, bfloat16 and float32 are covered")
    if index < 0:
        raise ValueError(f"{name} is not in device memory")
    return _dtypes[dtype], dtype, index


def _misfit(t, name, dtype, shape, index, more=""):
    raise ValueError(f"{name}: {t.dtype} {tuple(t.shape)} strides {t.stride()} on {t.device}, {more}{dtype} {tuple(shape)} on device {index} is wanted")


def _rows(t, name, shape, dtype, index):
    """Strides of a data tensor of this shape, in elements."""
    s = t.stride()
    if t.shape != shape or t.dtype is not dtype or t.get_device() != index or (s[-1] != 1 and shape[-1] > 1):
        _misfit(t, name, dtype, shape, index, "contiguous in its last dimension ")
    return s


def _plain(t, name, dtype, shape, index):
    """Pointer of a contiguous tensor of this type and shape."""
    if t.dtype is not dtype or t.shape != shape or t.get_device() != index or not t.is_contiguous():
        _misfit(t, name, dtype, shape, index, "contiguous ")
    return t.data_ptr()


def _call(entry, args, index, stream):
    if index != _torch.cuda.current_device():
        with _torch.cuda.device(index):
            entry(args, _stream_of(index) if stream is None else stream)
    else:
        entry(args, _stream_of(index) if stream is None else stream)


def _workspace(args, needed, workspace, index, stream):
    """Puts the caller's workspace, or one made here, into args.  Returns what has to live until the call is made."""
    if workspace is None:
        need = needed(args)
        if not need:
            return None
        workspace = _torch.empty(need, dtype=_torch.uint8, device=_torch.device("cuda", index))
        if stream is not None:   # the memory may be handed out again only after that stream is done with it
            workspace.record_stream(_torch.cuda.ExternalStream(stream, device=index))
    elif workspace.dtype is not _torch.uint8 or workspace.get_device() != index or not workspace.is_contiguous():
        _misfit(workspace, "workspace", _torch.uint8, workspace.shape, index, "contiguous ")
    args.workspace, args.workspace_bytes = workspace.data_ptr(), workspace.numel()
    return workspace


def qk_norm_rope(q, k, v, positions, inv_freq, *, q_weight=None, k_weight=None, eps=1e-6, sections=None, interleaved=False, slots=None,
                 q_out=None, k_out=None, v_out=None, stream=None):
    """Norms every head of q [tokens, q heads, head dim] and k [tokens, kv heads, head dim], rotates them by their positions, copies v.

    positions: int32 [tokens] or [tokens, axes]; inv_freq: fp32 [pairs], turned by the axes in order, sections[a] pairs each.
    q_weight, k_weight: fp32 [head dim].  With slots (int64 [tokens]) k_out and v_out are paged caches [pages, page size, kv heads,
    head dim] and a token goes to place slot % page size of page slot // page size, or nowhere if the slot is outside;
    without, they are [tokens, kv heads, head dim] and made here if None.  v may be None.  Returns (q_out, k_out, v_out)."""
    kind, dtype, index = _kind(q, "q")
    q_shape, k_shape, p_shape, f_shape = q.shape, k.shape, positions.shape, inv_freq.shape
    if len(q_shape) != 3 or len(k_shape) != 3 or not 1 <= len(p_shape) <= 2 or len(f_shape) != 1:
        raise ValueError("q and k are [tokens, heads, head dim], positions [tokens] or [tokens, axes], inv_freq [pairs]")
    tokens, heads, dim = q_shape
    kv_heads, pairs = k_shape[1], f_shape[0]
    axes = p_shape[1] if len(p_shape) == 2 else 1
    s0, s1, s2, s3 = (pairs, 0, 0, 0) if sections is None else (*sections, 0, 0, 0)[:4]
    if (1 if sections is None else len(sections)) != axes or not 1 <= axes <= FI_MAX_AXES:
        raise ValueError(f"sections {sections} for {axes} axes, 1 to {FI_MAX_AXES} are covered")
    kv_shape = (tokens, kv_heads, dim)
    qs, ks = _rows(q, "q", q_shape, dtype, index), _rows(k, "k", kv_shape, dtype, index)
    if q_out is None:
        q_out = _torch.empty(q_shape, dtype=dtype, device=q.device)
    page = n_slots = slots_ptr = 0
    out_shape = kv_shape
    if slots is not None:
        if k_out is None or k_out.dim() != 4 or (v is not None and v_out is None):
            raise ValueError("with slots, k_out and v_out are caches [pages, page size, kv heads, head dim]")
        pages, page = k_out.shape[:2]
        n_slots, out_shape = pages * page, (pages, page, kv_heads, dim)
        slots_ptr = _plain(slots, "slots", _torch.int64, (tokens,), index)
    elif k_out is None:
        k_out = _torch.empty(kv_shape, dtype=dtype, device=q.device)
    qos, kos = _rows(q_out, "q_out", q_shape, dtype, index), _rows(k_out, "k_out", out_shape, dtype, index)
    v_ptr = v_out_ptr = 0
    vs = vos = (0, 0, 0, 0)
    if v is not None:
        if v_out is None:
            v_out = _torch.empty(kv_shape, dtype=dtype, device=q.device)
        vs, vos = _rows(v, "v", kv_shape, dtype, index), _rows(v_out, "v_out", out_shape, dtype, index)
        v_ptr, v_out_ptr = v.data_ptr(), v_out.data_ptr()
    if slots is None:
        kos, vos = (0, *kos), (0, *vos)
    f32 = _torch.float32
    args = fi_qk_norm_rope_args(
        kind, tokens, heads, kv_heads, dim, 2 * pairs, 1 if interleaved else 0, axes, s0, s1, s2, s3, eps, page, n_slots,
        q.data_ptr(), k.data_ptr(), v_ptr, 0 if q_weight is None else _plain(q_weight, "q_weight", f32, (dim,), index),
        0 if k_weight is None else _plain(k_weight, "k_weight", f32, (dim,), index),
        _plain(positions, "positions", _torch.int32, (tokens,) if len(p_shape) == 1 else (tokens, axes), index), _plain(inv_freq, "inv_freq", f32, f_shape, index),
        slots_ptr, q_out.data_ptr(), k_out.data_ptr(), v_out_ptr, qs[0], qs[1], ks[0], ks[1], vs[0], vs[1], qos[0], qos[1], kos[0], kos[1], kos[2], vos[0], vos[1], vos[2])
    _call(fi_qk_norm_rope, args, index, stream)
    return q_out, k_out, v_out if v is not None else None


def prompt_attention(q, k, v, cu_q, cu_k=None, *, causal=True, scale=None, out=None, stream=None):
    """softmax(scale * q k^T) v over packed sequences: q [query tokens, q heads, head dim], k and v [key tokens, kv heads, head dim], cu_q and
    cu_k (default: cu_q) int32 [sequences + 1] the offsets of the sequences.  causal: the last query of a sequence sees all its keys.
    scale: head dim ** -0.5 by default.  Returns out [query tokens, q heads, head dim]."""
    kind, dtype, index = _kind(q, "q")
    q_shape, k_shape, seqs = q.shape, k.shape, cu_q.shape
    if len(q_shape) != 3 or len(k_shape) != 3 or len(seqs) != 1 or seqs[0] < 1:
        raise ValueError("q, k and v are [tokens, heads, head dim], cu_q is [sequences + 1]")
    tokens, heads, dim = q_shape
    kv_shape = (k_shape[0], k_shape[1], dim)
    qs, ks, vs = _rows(q, "q", q_shape, dtype, index), _rows(k, "k", kv_shape, dtype, index), _rows(v, "v", kv_shape, dtype, index)
    if out is None:
        out = _torch.empty(q_shape, dtype=dtype, device=q.device)
    outs, i32 = _rows(out, "out", q_shape, dtype, index), _torch.int32
    q_ptr = _plain(cu_q, "cu_q", i32, seqs, index)
    args = fi_prompt_attention_args(
        kind, seqs[0] - 1, heads, kv_shape[1], dim, 1 if causal else 0, dim ** -0.5 if scale is None else scale, 0, tokens, kv_shape[0],
        q.data_ptr(), k.data_ptr(), v.data_ptr(), q_ptr, q_ptr if cu_k is None else _plain(cu_k, "cu_k", i32, seqs, index), out.data_ptr(),
        qs[0], qs[1], ks[0], ks[1], vs[0], vs[1], outs[0], outs[1])
    _call(fi_prompt_attention, args, index, stream)
    return out


def tree_attention(q, k_cache, v_cache, block_table, cached, cu_nodes, mask=None, *, scale=None, max_nodes=None, max_length=None, out=None, workspace=None,
                   stream=None):
    """Attention of drafted trees, or single tokens, over a paged cache.

    q [nodes, q heads, head dim], packed by cu_nodes (int32 [sequences + 1]); k_cache and v_cache [pages, page size, kv heads, head dim];
    block_table int32 [sequences, columns]; cached int32 [sequences]: committed tokens, whose pages the nodes' own keys and values follow;
    mask int64 [nodes, words]: bit j of a row is set where the node sees node j of its sequence, None for chains.
    max_nodes: most nodes of a sequence (default: all nodes), max_length: most committed tokens and nodes together (default: what
    the table can name; it guides how the work is shared out).  workspace: uint8, fi_tree_attention_workspace bytes; made here if
    None.  Returns out [nodes, q heads, head dim]."""
    kind, dtype, index = _kind(q, "q")
    q_shape, kv_shape, t_shape, cu_shape = q.shape, k_cache.shape, block_table.shape, cu_nodes.shape
    if len(q_shape) != 3 or len(kv_shape) != 4 or len(t_shape) != 2 or len(cu_shape) != 1 or cu_shape[0] < 1:
        raise ValueError("q is [nodes, heads, head dim], the caches [pages, page size, heads, head dim], block_table [sequences, columns], cu_nodes [sequences + 1]")
    nodes, heads, dim = q_shape
    pages, page, kv_heads, _ = kv_shape
    kv_shape = (pages, page, kv_heads, dim)
    seqs, i32 = cu_shape[0] - 1, _torch.int32
    columns, words, mask_ptr = t_shape[1], 0, 0
    ts = _rows(block_table, "block_table", (seqs, columns), i32, index)
    if mask is not None:
        words = mask.shape[-1]
        mask_ptr = _plain(mask, "mask", _torch.int64, (nodes, words), index)
    qs, ks, vs = _rows(q, "q", q_shape, dtype, index), _rows(k_cache, "k_cache", kv_shape, dtype, index), _rows(v_cache, "v_cache", kv_shape, dtype, index)
    if out is None:
        out = _torch.empty(q_shape, dtype=dtype, device=q.device)
    outs = _rows(out, "out", q_shape, dtype, index)
    args = fi_tree_attention_args(
        kind, seqs, heads, kv_heads, dim, page, pages, columns, words, nodes if max_nodes is None else max_nodes,
        min(page * columns, 2 ** 31 - 1) if max_length is None else max_length, dim ** -0.5 if scale is None else scale, nodes,
        q.data_ptr(), k_cache.data_ptr(), v_cache.data_ptr(), block_table.data_ptr(), _plain(cached, "cached", i32, (seqs,), index),
        _plain(cu_nodes, "cu_nodes", i32, cu_shape, index), mask_ptr, out.data_ptr(), 0, 0,
        qs[0], qs[1], outs[0], outs[1], ks[0], ks[1], ks[2], vs[0], vs[1], vs[2], ts[0])
    workspace = _workspace(args, fi_tree_attention_workspace, workspace, index, stream)
    _call(fi_tree_attention, args, index, stream)
    return out


def q4_matmul(x, w, scales, zeros=None, *, group=None, out=None, workspace=None, stream=None):
    """x [rows, inputs] times 4-bit weights: w uint8 [outputs, inputs / 2], two weights per byte, the even one in the low half; scales fp32 and
    zeros uint8 (8 where None) [outputs, inputs / group].  workspace: uint8, fi_q4_matmul_workspace bytes; made here if None.  Returns out [rows,
    outputs] in x's type."""
    kind, dtype, index = _kind(x, "x")
    x_shape, w_shape, s_shape = x.shape, w.shape, scales.shape
    if len(x_shape) != 2 or len(w_shape) != 2 or len(s_shape) != 2:
        raise ValueError("x is [rows, inputs], w [outputs, inputs / 2], scales [outputs, groups]")
    (rows, inputs), outputs, groups = x_shape, w_shape[0], s_shape[1]
    if group is None:
        group = inputs // groups if groups else 128
    if inputs % 2 or groups * group != inputs:
        raise ValueError(f"{inputs} inputs do not make {groups} groups of {group}")
    s_shape = (outputs, groups)
    xs, ws, ss = _rows(x, "x", x_shape, dtype, index), _rows(w, "w", (outputs, inputs // 2), _torch.uint8, index), _rows(scales, "scales", s_shape, _torch.float32, index)
    zs = _rows(zeros, "zeros", s_shape, _torch.uint8, index) if zeros is not None else (0, 0)
    if out is None:
        out = _torch.empty((rows, outputs), dtype=dtype, device=x.device)
    outs = _rows(out, "out", (rows, outputs), dtype, index)
    args = fi_q4_matmul_args(kind, rows, inputs, outputs, group, 0, x.data_ptr(), w.data_ptr(), scales.data_ptr(), zeros.data_ptr() if zeros is not None else 0,
                             out.data_ptr(), 0, 0, xs[0], ws[0], ss[0], zs[0], outs[0])
    workspace = _workspace(args, fi_q4_matmul_workspace, workspace, index, stream)
    _call(fi_q4_matmul, args, index, stream)
    return out
