"""What the decoder operators refuse, and the layouts of their argument structs (no device is touched: the checks come before any launch)."""
import ctypes as C
import os
import re

import pytest

import paper_2410_21120_amd as fi

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = 4096   # stands for a device address: aligned, never read


def rope(**kw):
    a = fi.fi_qk_norm_rope_args(dtype=fi.FI_BF16, tokens=3, q_heads=4, kv_heads=2, head_dim=64, rot_dim=64, n_axes=1, section0=32, eps=1e-6, q=P, k=P, v=P,
                                positions=P, inv_freq=P, q_out=P, k_out=P, v_out=P, q_token=256, q_head=64, k_token=128, k_head=64, v_token=128, v_head=64,
                                q_out_token=256, q_out_head=64, k_out_token=128, k_out_head=64, v_out_token=128, v_out_head=64)
    for name, value in kw.items():
        setattr(a, name, value)
    return fi.fi_qk_norm_rope, a


def prompt(**kw):
    a = fi.fi_prompt_attention_args(dtype=fi.FI_BF16, n_seqs=1, q_heads=4, kv_heads=2, head_dim=64, causal=1, scale=0.125, q_tokens=3, k_tokens=3, q=P, k=P, v=P,
                                    cu_q=P, cu_k=P, out=P, q_token=256, q_head=64, k_token=128, k_head=64, v_token=128, v_head=64, out_token=256, out_head=64)
    for name, value in kw.items():
        setattr(a, name, value)
    return fi.fi_prompt_attention, a


def tree(**kw):
    a = fi.fi_tree_attention_args(dtype=fi.FI_BF16, n_seqs=1, q_heads=4, kv_heads=2, head_dim=64, page_size=16, n_pages=4, table_columns=4, mask_words=1, max_nodes=3,
                                  max_length=50, scale=0.125, nodes=3, q=P, k_cache=P, v_cache=P, block_table=P, cached=P, cu_nodes=P, mask=P, out=P, workspace=P,
                                  workspace_bytes=1 << 40, q_token=256, q_head=64, out_token=256, out_head=64, k_page=2048, k_token=128, k_head=64, v_page=2048,
                                  v_token=128, v_head=64, table_stride=4)
    for name, value in kw.items():
        setattr(a, name, value)
    return fi.fi_tree_attention, a


def q4(**kw):
    a = fi.fi_q4_matmul_args(dtype=fi.FI_BF16, rows=2, inputs=256, outputs=8, group=64, x=P, w=P, scales=P, zeros=P, out=P, x_stride=256, w_stride=128,
                             scales_stride=4, zeros_stride=4, out_stride=8)
    for name, value in kw.items():
        setattr(a, name, value)
    return fi.fi_q4_matmul, a


INVALID = [
    (rope, dict(dtype=2)), (rope, dict(tokens=-1)), (rope, dict(head_dim=0)), (rope, dict(rot_dim=63)), (rope, dict(rot_dim=66)), (rope, dict(rot_dim=-2)),
    (rope, dict(interleaved=2)), (rope, dict(n_axes=0)), (rope, dict(n_axes=5)), (rope, dict(section0=31)), (rope, dict(n_axes=2, section0=40, section1=-8)),
    (rope, dict(eps=-1.0)), (rope, dict(eps=float("nan"))), (rope, dict(q=0)), (rope, dict(k=0)), (rope, dict(v=0)), (rope, dict(v_out=0)), (rope, dict(positions=0)),
    (rope, dict(inv_freq=P + 2)), (rope, dict(q=P + 1)), (rope, dict(q_token=-1)), (rope, dict(q_out_head=63)), (rope, dict(q_out_token=0)), (rope, dict(k_out_token=32)),
    (rope, dict(slots=P, page_size=0, n_slots=16)), (rope, dict(slots=P + 4, page_size=16, n_slots=16)), (rope, dict(slots=P, page_size=16, n_slots=-1)),
    (rope, dict(slots=P, page_size=16, n_slots=64, k_out_page=0)), (rope, dict(q_weight=P + 1)), (rope, dict(k_token=1 << 50)),
    (prompt, dict(dtype=-1)), (prompt, dict(n_seqs=-1)), (prompt, dict(q_tokens=-1)), (prompt, dict(causal=2)), (prompt, dict(kv_heads=3)), (prompt, dict(kv_heads=0)),
    (prompt, dict(head_dim=0)), (prompt, dict(scale=0.0)), (prompt, dict(scale=float("inf"))), (prompt, dict(scale=float("nan"))), (prompt, dict(q=0)), (prompt, dict(k=0)),
    (prompt, dict(out=0)), (prompt, dict(cu_q=0)), (prompt, dict(cu_k=P + 2)), (prompt, dict(v=P + 1)), (prompt, dict(k_token=-8)), (prompt, dict(out_token=10)),
    (prompt, dict(out_head=0)),
    (tree, dict(dtype=7)), (tree, dict(n_seqs=-1)), (tree, dict(page_size=0)), (tree, dict(n_pages=-1)), (tree, dict(table_columns=-1)), (tree, dict(nodes=-1)),
    (tree, dict(max_nodes=-1)), (tree, dict(max_length=-1)), (tree, dict(q_heads=5)), (tree, dict(scale=-1.0)), (tree, dict(q=0)), (tree, dict(k_cache=0)),
    (tree, dict(v_cache=P + 1)), (tree, dict(block_table=0)), (tree, dict(cached=0)), (tree, dict(cu_nodes=P + 1)), (tree, dict(mask=P + 4)), (tree, dict(mask_words=0)),
    (tree, dict(table_stride=-1)), (tree, dict(out_token=1)),
    (q4, dict(dtype=3)), (q4, dict(rows=-1)), (q4, dict(inputs=250)), (q4, dict(group=0)), (q4, dict(x=0)), (q4, dict(w=0)), (q4, dict(scales=P + 2)), (q4, dict(out=P + 1)),
    (q4, dict(x_stride=-1)), (q4, dict(out_stride=7)), (q4, dict(w_stride=-1)),
]
UNSUPPORTED = [
    (rope, dict(head_dim=258, rot_dim=0, section0=0)), (prompt, dict(head_dim=257)), (prompt, dict(q_tokens=1 << 31)), (tree, dict(head_dim=300)),
    (tree, dict(page_size=1 << 20, table_columns=1 << 12)), (tree, dict(nodes=1 << 31)), (tree, dict(mask_words=1025)), (q4, dict(inputs=240, group=16)),
    (q4, dict(inputs=192, group=96)),
]
NOTHING = [
    (rope, dict(tokens=0)), (prompt, dict(n_seqs=0)), (prompt, dict(q_tokens=0)), (tree, dict(n_seqs=0)), (tree, dict(nodes=0)), (tree, dict(max_nodes=0)),
    (q4, dict(rows=0)), (q4, dict(outputs=0)),
]


@pytest.mark.parametrize("make,change", INVALID, ids=lambda v: getattr(v, "__name__", None) or "-".join(v))
def test_invalid_arguments_are_refused(make, change):
    call, args = make(**change)
    with pytest.raises(fi.FiError) as e:
        call(args)
    assert e.value.status == fi.FI_EINVAL and fi.fi_last_error()


@pytest.mark.parametrize("make,change", UNSUPPORTED, ids=lambda v: getattr(v, "__name__", None) or "-".join(v))
def test_uncovered_sizes_are_refused(make, change):
    call, args = make(**change)
    with pytest.raises(fi.FiError) as e:
        call(args)
    assert e.value.status == fi.FI_EUNSUPPORTED and fi.fi_last_error()


@pytest.mark.parametrize("make,change", NOTHING, ids=lambda v: getattr(v, "__name__", None) or "-".join(v))
def test_empty_problems_are_no_error(make, change):
    call, args = make(**change)
    call(args)


def test_null_structs_are_refused():
    for name in ("fi_qk_norm_rope", "fi_prompt_attention", "fi_tree_attention", "fi_q4_matmul"):
        assert getattr(fi.lib(), name)(None, None) == fi.FI_EINVAL
    n = C.c_uint64(7)
    assert fi.lib().fi_tree_attention_workspace(None, C.byref(n)) == fi.FI_EINVAL and n.value == 7


def test_a_workspace_that_is_too_small_is_refused():
    _, a = tree(n_seqs=1, max_length=60000, page_size=64, n_pages=1000, table_columns=1000)
    need = fi.fi_tree_attention_workspace(a)
    if need:
        for change in (dict(workspace_bytes=need - 1), dict(workspace=0), dict(workspace=P + 8)):
            call, b = tree(n_seqs=1, max_length=60000, page_size=64, n_pages=1000, table_columns=1000, **change)
            with pytest.raises(fi.FiError) as e:
                call(b)
            assert e.value.status == fi.FI_EINVAL


def test_structs_have_the_headers_layout(tmp_path):
    """Sizes and field offsets as a C compiler sees them, against the ctypes structs."""
    import shutil
    import subprocess
    gcc = shutil.which("gcc")
    if gcc is None:
        pytest.skip("needs gcc")
    header = open(os.path.join(ROOT, "include", "fusedinf.h")).read()
    # arrays of the header are single fields here: their first ones are compared
    arrays = {"section0": "sections", "q_token": "q_strides", "k_token": "k_strides", "v_token": "v_strides", "q_out_token": "q_out_strides", "out_token": "out_strides",
              "k_out_page": "k_out_strides", "v_out_page": "v_out_strides", "k_page": "k_strides", "v_page": "v_strides"}
    inner = {"section1", "section2", "section3", "q_head", "k_head", "v_head", "q_out_head", "out_head", "k_out_token", "k_out_head", "v_out_token", "v_out_head"}
    lines, want = [], []
    for cls in (fi.fi_qk_norm_rope_args, fi.fi_prompt_attention_args, fi.fi_tree_attention_args, fi.fi_q4_matmul_args):
        assert re.search(r"\}\s*%s;" % cls.__name__, header)
        lines.append('printf("%%zu\\n", sizeof(%s));' % cls.__name__)
        want.append(C.sizeof(cls))
        for name, _ in cls._fields_:
            if name in inner or (cls is fi.fi_tree_attention_args and name in ("k_token", "v_token")):
                continue
            lines.append('printf("%%zu\\n", offsetof(%s, %s));' % (cls.__name__, arrays.get(name, name)))
            want.append(getattr(cls, name).offset)
    src = tmp_path / "layout.c"
    src.write_text('#include "fusedinf.h"\n#include <stdio.h>\nint main(void) { %s return 0; }\n' % " ".join(lines))
    exe = str(tmp_path / "layout")
    subprocess.run([gcc, "-I" + os.path.join(ROOT, "include"), str(src), "-o", exe], check=True)
    got = [int(v) for v in subprocess.run([exe], stdout=subprocess.PIPE, text=True, check=True).stdout.split()]
    assert got == want


def test_tensors_that_do_not_fit_are_refused():
    import torch
    cpu = torch.zeros((2, 4, 64), dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        fi.prompt_attention(cpu, cpu, cpu, torch.tensor([0, 2], dtype=torch.int32))
    with pytest.raises(TypeError):
        fi.prompt_attention(cpu.half(), cpu, cpu, torch.tensor([0, 2], dtype=torch.int32))
