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
_torch = None
_dtypes = {}


def _setup():
    global _torch
    import torch
    _torch = torch
    _dtypes.update({torch.bfloat16: _b.FI_BF16, torch.float32: _b.FI_F32})


def _kind(t, name):
    if _torch is None:
        _setup()
    if t.dtype not in _dtypes:
        raise TypeError(f"{name}: {t.dtype}, bfloat16 and float32 are covered")
    if not t.is_cuda:
        raise ValueError(f"{name} is not in device memory")
    return _dtypes[t.dtype]


def _rows(t, name, shape, like):
    """Strides of a data tensor of this shape, in elements, without the last one."""
    if t.shape != shape or t.dtype != like.dtype or t.device != like.device:
        raise ValueError(f"{name}: {t.dtype} {tuple(t.shape)} on {t.device}, {like.dtype} {tuple(shape)} on {like.device} is wanted")
    s = t.stride()
    if s[-1] != 1 and shape[-1] > 1:
        raise ValueError(f"{name}: its last dimension is not contiguous")
    return s


def _plain(t, name, dtype, shape, like):
    """Pointer of a contiguous tensor of this type and shape."""
    if t.dtype != dtype or t.shape != shape or t.device != like.device or not t.is_contiguous():
        raise ValueError(f"{name}: {t.dtype} {tuple(t.shape)} on {t.device}, contiguous {dtype} {tuple(shape)} on {like.device} is wanted")
    return t.data_ptr()


def _call(entry, args, like, stream):
    cuda, index = _torch.cuda, like.device.index
    if index != cuda.current_device():
        with cuda.device(index):
            entry(args, cuda.current_stream().cuda_stream if stream is None else stream)
    else:
        entry(args, cuda.current_stream().cuda_stream if stream is None else stream)


def _workspace(args, needed, workspace, like, stream):
    """Puts the caller's workspace, or one made here, into args.  Returns what has to live until the call is made."""
    if workspace is None:
        need = needed(args)
        if not need:
            return None
        workspace = _torch.empty(need, dtype=_torch.uint8, device=like.device)
        if stream is not None:   # the memory may be handed out again only after that stream is done with it
            workspace.record_stream(_torch.cuda.ExternalStream(stream, device=like.device))
    elif workspace.dtype != _torch.uint8 or workspace.device != like.device or not workspace.is_contiguous():
        raise ValueError(f"workspace: contiguous uint8 on {like.device} is wanted")
    args.workspace, args.workspace_bytes = workspace.data_ptr(), workspace.numel()
    return workspace


def qk_norm_rope(q, k, v, positions, inv_freq, *, q_weight=None, k_weight=None, eps=1e-6, sections=None, interleaved=False, slots=None,
                 q_out=None, k_out=None, v_out=None, stream=None):
    """Norms every head of q [tokens, q heads, head dim] and k [tokens, kv heads, head dim], rotates them by their positions, copies v.

    positions: int32 [tokens] or [tokens, axes]; inv_freq: fp32 [pairs], turned by the axes in order, sections[a] pairs each.
    q_weight, k_weight: fp32 [head dim].  With slots (int64 [tokens]) k_out and v_out are paged caches [pages, page size, kv heads,
    head dim] and a token goes to place slot % page size of page slot // page size, or nowhere if the slot is outside;
    without, they are [tokens, kv heads, head dim] and made here if None.  v may be None.  Returns (q_out, k_out, v_out)."""
    kind = _kind(q, "q")
    if q.dim() != 3 or k.dim() != 3 or positions.dim() not in (1, 2) or inv_freq.dim() != 1:
        raise ValueError("q and k are [tokens, heads, head dim], positions [tokens] or [tokens, axes], inv_freq [pairs]")
    tokens, heads, dim = q.shape
    kv_heads, pairs = k.shape[1], inv_freq.shape[0]
    axes = positions.shape[1] if positions.dim() == 2 else 1
    sections = (pairs,) if sections is None else tuple(sections)
    if len(sections) != axes or not 1 <= axes <= FI_MAX_AXES:
        raise ValueError(f"{len(sections)} sections for {axes} axes, 1 to {FI_MAX_AXES} are covered")
    kv_shape = (tokens, kv_heads, dim)
    qs, ks = _rows(q, "q", (tokens, heads, dim), q), _rows(k, "k", kv_shape, q)
    vs = _rows(v, "v", kv_shape, q) if v is not None else (0, 0)
    q_out = _torch.empty((tokens, heads, dim), dtype=q.dtype, device=q.device) if q_out is None else q_out
    page = n_slots = slots_ptr = 0
    if slots is not None:
        if k_out is None or k_out.dim() != 4 or (v is not None and v_out is None):
            raise ValueError("with slots, k_out and v_out are caches [pages, page size, kv heads, head dim]")
        page = k_out.shape[1]
        n_slots, kv_shape = k_out.shape[0] * page, (k_out.shape[0], page, kv_heads, dim)
        slots_ptr = _plain(slots, "slots", _torch.int64, (tokens,), q)
    elif k_out is None:
        k_out = _torch.empty(kv_shape, dtype=q.dtype, device=q.device)
    if v is not None and v_out is None:
        v_out = _torch.empty(kv_shape, dtype=q.dtype, device=q.device)
    qos, kos = _rows(q_out, "q_out", (tokens, heads, dim), q), _rows(k_out, "k_out", kv_shape, q)
    vos = _rows(v_out, "v_out", kv_shape, q) if v is not None else (0, 0, 0, 0)
    if slots is None:
        kos, vos = (0,) + tuple(kos), (0,) + tuple(vos)
    f32 = _torch.float32
    args = fi_qk_norm_rope_args(
        kind, tokens, heads, kv_heads, dim, 2 * pairs, 1 if interleaved else 0, axes, *sections, *(0,) * (FI_MAX_AXES - axes), eps, page, n_slots,
        q.data_ptr(), k.data_ptr(), v.data_ptr() if v is not None else 0,
        _plain(q_weight, "q_weight", f32, (dim,), q) if q_weight is not None else 0, _plain(k_weight, "k_weight", f32, (dim,), q) if k_weight is not None else 0,
        _plain(positions, "positions", _torch.int32, (tokens, axes) if positions.dim() == 2 else (tokens,), q), _plain(inv_freq, "inv_freq", f32, (pairs,), q),
        slots_ptr, q_out.data_ptr(), k_out.data_ptr(), v_out.data_ptr() if v is not None else 0,
        qs[0], qs[1], ks[0], ks[1], vs[0], vs[1], qos[0], qos[1], kos[0], kos[1], kos[2], vos[0], vos[1], vos[2])
    _call(fi_qk_norm_rope, args, q, stream)
    return q_out, k_out, v_out if v is not None else None


def prompt_attention(q, k, v, cu_q, cu_k=None, *, causal=True, scale=None, out=None, stream=None):
    """softmax(scale * q k^T) v over packed sequences: q [query tokens, q heads, head dim], k and v [key tokens, kv heads, head dim], cu_q and
    cu_k (default: cu_q) int32 [sequences + 1] the offsets of the sequences.  causal: the last query of a sequence sees all its keys.
    scale: head dim ** -0.5 by default.  Returns out [query tokens, q heads, head dim]."""
    kind = _kind(q, "q")
    if q.dim() != 3 or k.dim() != 3 or cu_q.dim() != 1 or cu_q.shape[0] < 1:
        raise ValueError("q, k and v are [tokens, heads, head dim], cu_q is [sequences + 1]")
    tokens, heads, dim = q.shape
    cu_k = cu_q if cu_k is None else cu_k
    kv_shape = (k.shape[0], k.shape[1], dim)
    qs, ks, vs = _rows(q, "q", (tokens, heads, dim), q), _rows(k, "k", kv_shape, q), _rows(v, "v", kv_shape, q)
    out = _torch.empty((tokens, heads, dim), dtype=q.dtype, device=q.device) if out is None else out
    os, seqs = _rows(out, "out", (tokens, heads, dim), q), cu_q.shape
    args = fi_prompt_attention_args(
        kind, seqs[0] - 1, heads, kv_shape[1], dim, 1 if causal else 0, dim ** -0.5 if scale is None else scale, 0, tokens, kv_shape[0],
        q.data_ptr(), k.data_ptr(), v.data_ptr(), _plain(cu_q, "cu_q", _torch.int32, seqs, q), _plain(cu_k, "cu_k", _torch.int32, seqs, q), out.data_ptr(),
        qs[0], qs[1], ks[0], ks[1], vs[0], vs[1], os[0], os[1])
    _call(fi_prompt_attention, args, q, stream)
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
    kind = _kind(q, "q")
    if q.dim() != 3 or k_cache.dim() != 4 or block_table.dim() != 2 or cu_nodes.dim() != 1 or cu_nodes.shape[0] < 1:
        raise ValueError("q is [nodes, heads, head dim], the caches [pages, page size, heads, head dim], block_table [sequences, columns], cu_nodes [sequences + 1]")
    nodes, heads, dim = q.shape
    pages, page, kv_heads, _ = k_cache.shape
    seqs, i32 = cu_nodes.shape[0] - 1, _torch.int32
    if block_table.dtype != i32 or block_table.shape[0] != seqs or block_table.device != q.device or (block_table.stride(1) != 1 and block_table.shape[1] > 1):
        raise ValueError("block_table: int32 [sequences, columns] with contiguous rows is wanted")
    columns, words, mask_ptr = block_table.shape[1], 0, 0
    if mask is not None:
        words = mask.shape[-1]
        mask_ptr = _plain(mask, "mask", _torch.int64, (nodes, words), q)
    kv_shape = (pages, page, kv_heads, dim)
    qs, ks, vs = _rows(q, "q", (nodes, heads, dim), q), _rows(k_cache, "k_cache", kv_shape, q), _rows(v_cache, "v_cache", kv_shape, q)
    out = _torch.empty((nodes, heads, dim), dtype=q.dtype, device=q.device) if out is None else out
    os = _rows(out, "out", (nodes, heads, dim), q)
    args = fi_tree_attention_args(
        kind, seqs, heads, kv_heads, dim, page, pages, columns, words, nodes if max_nodes is None else max_nodes,
        min(page * columns, 2 ** 31 - 1) if max_length is None else max_length, dim ** -0.5 if scale is None else scale, nodes,
        q.data_ptr(), k_cache.data_ptr(), v_cache.data_ptr(), block_table.data_ptr(), _plain(cached, "cached", i32, (seqs,), q),
        _plain(cu_nodes, "cu_nodes", i32, (seqs + 1,), q), mask_ptr, out.data_ptr(), 0, 0,
        qs[0], qs[1], os[0], os[1], ks[0], ks[1], ks[2], vs[0], vs[1], vs[2], block_table.stride(0))
    workspace = _workspace(args, fi_tree_attention_workspace, workspace, q, stream)
    _call(fi_tree_attention, args, q, stream)
    return out


def q4_matmul(x, w, scales, zeros=None, *, group=None, out=None, workspace=None, stream=None):
    """x [rows, inputs] times 4-bit weights: w uint8 [outputs, inputs / 2], two weights per byte, the even one in the low half; scales fp32 and
    zeros uint8 (8 where None) [outputs, inputs / group].  workspace: uint8, fi_q4_matmul_workspace bytes; made here if None.  Returns out [rows,
    outputs] in x's type."""
    kind = _kind(x, "x")
    if x.dim() != 2 or w.dim() != 2 or scales.dim() != 2:
        raise ValueError("x is [rows, inputs], w [outputs, inputs / 2], scales [outputs, groups]")
    (rows, inputs), outputs, groups = x.shape, w.shape[0], scales.shape[1]
    if group is None:
        group = inputs // groups if groups else 128
    if inputs % 2 or w.shape[1] * 2 != inputs or scales.shape[0] != outputs or groups * group != inputs:
        raise ValueError(f"x {tuple(x.shape)}, w {tuple(w.shape)} and scales {tuple(scales.shape)} do not fit groups of {group}")
    for t, name, dtype in ((w, "w", _torch.uint8), (scales, "scales", _torch.float32), (zeros, "zeros", _torch.uint8)):
        if t is not None and (t.dtype != dtype or t.device != x.device or (t.stride(1) != 1 and t.shape[1] > 1)):
            raise ValueError(f"{name}: {dtype} on {x.device} with contiguous rows is wanted")
    if zeros is not None and zeros.shape != scales.shape:
        raise ValueError("zeros have the shape of scales")
    out = _torch.empty((rows, outputs), dtype=x.dtype, device=x.device) if out is None else out
    xs, os = _rows(x, "x", (rows, inputs), x), _rows(out, "out", (rows, outputs), x)
    args = fi_q4_matmul_args(kind, rows, inputs, outputs, group, 0, x.data_ptr(), w.data_ptr(), scales.data_ptr(), zeros.data_ptr() if zeros is not None else 0,
                             out.data_ptr(), 0, 0, xs[0], w.stride(0), scales.stride(0), zeros.stride(0) if zeros is not None else 0, os[0])
    workspace = _workspace(args, fi_q4_matmul_workspace, workspace, x, stream)
    _call(fi_q4_matmul, args, x, stream)
    return out
