"""What the operators of beam search over a 4-bit cache refuse, the layouts of their argument structs, and their definitions on the CPU (no device is touched)."""
import ctypes as C
import os
import re

import pytest

import paper_2410_21120_amd as fi

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = 1 << 20   # stands for a device address: aligned, never read


def write(**kw):
    a = fi.fi_fp4_cache_write_args(dtype=fi.FI_BF16, tokens=3, kv_heads=2, head_dim=64, page_size=16, n_slots=64, k=P, v=P, slots=P, k_codes=P, k_scales=P, v_codes=P, v_scales=P,
                                   k_held=P, v_held=P)
    for x in "kv":
        for name, value in (("token", 128), ("head", 64), ("held_token", 128), ("held_head", 64), ("codes_page", 1024), ("codes_token", 32), ("codes_head", 512),
                            ("scales_page", 64), ("scales_token", 2), ("scales_head", 32)):
            setattr(a, x + "_" + name, value)
    return _set(fi.fi_fp4_cache_write, a, kw)


def attend(**kw):
    a = fi.fi_fp4_tree_attention_args(dtype=fi.FI_BF16, n_seqs=1, q_heads=4, kv_heads=2, head_dim=64, page_size=16, n_pages=4, table_columns=4, mask_words=1, max_nodes=3,
                                      max_length=50, scale=0.125, nodes=3, q=P, k_codes=P, k_scales=P, v_codes=P, v_scales=P, block_table=P, cached=P, cu_nodes=P, mask=P, out=P,
                                      workspace=P, workspace_bytes=1 << 40, q_token=256, q_head=64, out_token=256, out_head=64, table_stride=4)
    for x in "kv":
        for name, value in (("codes_page", 1024), ("codes_token", 32), ("codes_head", 512), ("scales_page", 64), ("scales_token", 2), ("scales_head", 32)):
            setattr(a, x + "_" + name, value)
    return _set(fi.fi_fp4_tree_attention, a, kw)


def beams(**kw):
    a = fi.fi_beam_select_args(dtype=fi.FI_BF16, n_seqs=2, beams=4, keep=4, vocab=100, end=3, logits_stride=100, logits=P, scores=2 * P, ended=3 * P, tokens_out=4 * P,
                               parents_out=5 * P, scores_out=6 * P, ended_out=7 * P, workspace=8 * P, workspace_bytes=P)
    return _set(fi.fi_beam_select, a, kw)


CACHES = (fi.fi_page_cache * 2)(fi.fi_page_cache(P, 4096, 4096), fi.fi_page_cache(P, 8192, 4096))
BAD = {name: (fi.fi_page_cache * 2)(CACHES[0], fi.fi_page_cache(*c)) for name, c in dict(close=(P, 4095, 4096), none=(0, 4096, 4096), negative=(P, 4096, -1), back=(P, -4096, 4096),
                                                                                        large=(P, 1 << 40, 1 << 33)).items()}


def fork(**kw):
    a = fi.fi_fork_pages_args(rows=3, new_rows=4, columns=5, page_size=16, n_pages=20, room=1, n_caches=2, table_stride=5, table_out_stride=5, block_table=P, lengths=2 * P, held=3 * P,
                              refs=4 * P, parents=5 * P, caches=C.addressof(CACHES), table_out=6 * P, lengths_out=7 * P, held_out=8 * P, refs_out=9 * P, slots_out=10 * P,
                              workspace=11 * P, workspace_bytes=P)
    return _set(fi.fi_fork_pages, a, kw)


def compact(**kw):
    a = fi.fi_compact_pages_args(rows=3, columns=5, n_pages=20, n_caches=2, table_stride=5, table_out_stride=5, block_table=P, refs=2 * P, caches=C.addressof(CACHES), table_out=3 * P,
                                 refs_out=4 * P, moved_out=5 * P, live_out=6 * P, workspace=7 * P, workspace_bytes=P)
    return _set(fi.fi_compact_pages, a, kw)


def _set(call, a, kw):
    for name, value in kw.items():
        assert hasattr(a, name)
        setattr(a, name, C.addressof(BAD[value]) if name == "caches" and value in BAD else value)
    return call, a


INVALID = [
    (write, dict(dtype=2)), (write, dict(tokens=-1)), (write, dict(kv_heads=-1)), (write, dict(head_dim=0)), (write, dict(page_size=0)), (write, dict(n_slots=-1)), (write, dict(k=0)),
    (write, dict(k=P + 1)), (write, dict(slots=0)), (write, dict(slots=P + 4)), (write, dict(v=0)), (write, dict(k_codes=0)), (write, dict(k_scales=0)), (write, dict(v_codes=P + 2)),
    (write, dict(k_codes_token=33)), (write, dict(k_codes_token=30)), (write, dict(k_codes_page=-4)), (write, dict(k_codes_token=28)), (write, dict(v_codes_head=480)),
    (write, dict(k_scales_token=1)), (write, dict(v_scales_page=63)), (write, dict(k_held_token=64)), (write, dict(v_held=P + 1)), (write, dict(k_token=-1)),
    (attend, dict(dtype=7)), (attend, dict(n_seqs=-1)), (attend, dict(page_size=0)), (attend, dict(n_pages=-1)), (attend, dict(nodes=-1)), (attend, dict(kv_heads=3)),
    (attend, dict(scale=0.0)), (attend, dict(scale=float("nan"))), (attend, dict(q=0)), (attend, dict(k_codes=0)), (attend, dict(v_scales=0)), (attend, dict(k_codes=P + 1)),
    (attend, dict(v_codes_page=1022)), (attend, dict(block_table=0)), (attend, dict(cached=P + 1)), (attend, dict(mask=P + 4)), (attend, dict(mask_words=0)), (attend, dict(out=0)),
    (attend, dict(out_token=10)), (attend, dict(out_head=0)), (attend, dict(q_token=-1)), (attend, dict(k_scales_head=-1)), (attend, dict(table_stride=-4)), (attend, dict(max_nodes=-1)),
    (beams, dict(dtype=5)), (beams, dict(n_seqs=-1)), (beams, dict(beams=0)), (beams, dict(keep=0)), (beams, dict(vocab=-1)), (beams, dict(end=100)), (beams, dict(end=-1)),
    (beams, dict(end=-1, ended=0)), (beams, dict(logits=0)), (beams, dict(logits=P + 1)), (beams, dict(scores=0)), (beams, dict(tokens_out=0)), (beams, dict(parents_out=5 * P + 2)),
    (beams, dict(scores_out=0)), (beams, dict(ended_out=0)), (beams, dict(logits_stride=-1)), (beams, dict(workspace=0)), (beams, dict(workspace_bytes=100)), (beams, dict(workspace=8 * P + 8)),
    (beams, dict(scores_out=2 * P)), (beams, dict(tokens_out=5 * P + 4)), (beams, dict(ended_out=3 * P + 7)), (beams, dict(workspace=P)), (beams, dict(scores_out=P + 1596)),
    (fork, dict(rows=-1)), (fork, dict(new_rows=-1)), (fork, dict(columns=-1)), (fork, dict(page_size=0)), (fork, dict(n_pages=-1)), (fork, dict(room=-1)), (fork, dict(n_caches=-1)),
    (fork, dict(parents=0)), (fork, dict(block_table=0)), (fork, dict(lengths=2 * P + 1)), (fork, dict(held=3 * P + 2)), (fork, dict(refs=0)), (fork, dict(parents=5 * P + 1)),
    (fork, dict(caches=0)), (fork, dict(caches="close")), (fork, dict(caches="none")), (fork, dict(caches="negative")), (fork, dict(caches="back")), (fork, dict(table_out=0)),
    (fork, dict(lengths_out=0)), (fork, dict(held_out=0)), (fork, dict(refs_out=0)), (fork, dict(slots_out=0)), (fork, dict(slots_out=10 * P + 4)), (fork, dict(table_out_stride=4)),
    (fork, dict(table_stride=-1)), (fork, dict(workspace=0)), (fork, dict(workspace_bytes=64)), (fork, dict(refs_out=4 * P)), (fork, dict(table_out=P + 56)), (fork, dict(held_out=2 * P)),
    (fork, dict(lengths_out=5 * P)), (fork, dict(slots_out=9 * P + 72)), (fork, dict(workspace=6 * P)),
    (compact, dict(rows=-1)), (compact, dict(columns=-1)), (compact, dict(n_pages=-1)), (compact, dict(n_caches=-1)), (compact, dict(caches=0)), (compact, dict(caches="close")),
    (compact, dict(block_table=0)), (compact, dict(table_out=0)), (compact, dict(refs=0)), (compact, dict(refs_out=0)), (compact, dict(moved_out=0)), (compact, dict(live_out=0)),
    (compact, dict(live_out=6 * P + 1)), (compact, dict(table_out_stride=3)), (compact, dict(workspace=0)), (compact, dict(workspace_bytes=8)), (compact, dict(refs_out=2 * P + 76)),
    (compact, dict(table_out=P)), (compact, dict(moved_out=4 * P)), (compact, dict(live_out=2 * P)),
]
UNSUPPORTED = [
    (write, dict(head_dim=60)), (write, dict(head_dim=264)), (write, dict(kv_heads=70000)), (attend, dict(head_dim=60)), (attend, dict(head_dim=264)),
    (attend, dict(table_columns=1 << 30)), (attend, dict(mask_words=2000)), (attend, dict(nodes=1 << 31)), (attend, dict(nodes=1 << 28, n_seqs=1 << 28, max_nodes=1)),
    (beams, dict(beams=65)), (beams, dict(keep=65)), (beams, dict(vocab=1 << 30)), (beams, dict(n_seqs=1 << 30)), (beams, dict(n_seqs=1 << 25, workspace_bytes=1 << 50, ended=0, logits=1 << 50,
     scores=1 << 46, tokens_out=1 << 43, parents_out=1 << 44, scores_out=1 << 45, ended_out=1 << 47, workspace=1 << 52)),
    (fork, dict(rows=70000)), (fork, dict(new_rows=70000)), (fork, dict(room=70000)), (fork, dict(columns=1 << 29)), (fork, dict(n_caches=129)), (fork, dict(caches="large")),
    (compact, dict(rows=70000)), (compact, dict(n_caches=129)), (compact, dict(caches="large")),
]


@pytest.mark.parametrize("make,change", INVALID, ids=lambda v: getattr(v, "__name__", None) or "-".join(v))
def test_invalid_arguments_are_refused(make, change):
    call, args = make(**change)
    with pytest.raises(fi.FiError) as e:
        call(args)
    assert e.value.status == fi.FI_EINVAL and fi.fi_last_error()


@pytest.mark.parametrize("make,change", UNSUPPORTED, ids=lambda v: getattr(v, "__name__", None) or "-".join(v))
def test_sizes_beyond_the_kernels_are_refused(make, change):
    call, args = make(**change)
    with pytest.raises(fi.FiError) as e:
        call(args)
    assert e.value.status == fi.FI_EUNSUPPORTED and fi.fi_last_error()


EMPTY = [
    (write, dict(tokens=0, k=0, v=0, slots=0)), (write, dict(kv_heads=0, k=0)), (attend, dict(n_seqs=0)), (attend, dict(nodes=0, q=0, out=0)), (attend, dict(max_nodes=0)),
    (beams, dict(n_seqs=0, logits=0, scores=0)), (fork, dict(rows=0, new_rows=0, n_pages=0, block_table=0, lengths=0, refs=0)),
]


@pytest.mark.parametrize("make,change", EMPTY, ids=lambda v: getattr(v, "__name__", None) or "-".join(v))
def test_empty_problems_are_no_error(make, change):
    call, args = make(**change)
    call(args)


def test_null_structs_are_refused():
    n = C.c_uint64(7)
    for name in ("fi_fp4_cache_write", "fi_fp4_tree_attention", "fi_beam_select", "fi_fork_pages", "fi_compact_pages"):
        assert getattr(fi.lib(), name)(None, None) == fi.FI_EINVAL
        if name != "fi_fp4_cache_write":
            assert getattr(fi.lib(), name + "_workspace")(None, C.byref(n)) == fi.FI_EINVAL and n.value == 7


def test_workspaces_go_by_the_sizes_alone():
    """And a byte less than what is asked for is refused."""
    for make, name, size in ((attend, "fi_fp4_tree_attention", dict(max_length=60000, page_size=64, n_pages=1000, table_columns=1000)), (beams, "fi_beam_select", {}),
                             (fork, "fi_fork_pages", {}), (compact, "fi_compact_pages", {})):
        _, a = make(**size)
        need = getattr(fi, name + "_workspace")(a)
        assert need > 0
        for field, kind in a._fields_:
            if kind is C.c_void_p:
                setattr(a, field, None)
        if make is fork:
            a.new_rows = a.rows   # (without parents)
            assert getattr(fi, name + "_workspace")(a) > 0
        else:
            assert getattr(fi, name + "_workspace")(a) == need
        call, b = make(**size, workspace_bytes=need - 1)
        with pytest.raises(fi.FiError, match="workspace") as e:
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
    lines, want = [], []
    for cls in (fi.fi_fp4_cache_write_args, fi.fi_fp4_tree_attention_args, fi.fi_beam_select_args, fi.fi_page_cache, fi.fi_fork_pages_args, fi.fi_compact_pages_args):
        body = re.search(r"typedef struct \{([^}]*)\} %s;" % cls.__name__, header).group(1)
        lines.append('printf("%%zu\\n", sizeof(%s));' % cls.__name__)
        want.append(C.sizeof(cls))
        for name, _ in cls._fields_:
            # arrays of the header are single fields here: their first ones are compared
            array = re.sub(r"_(page|token|head)$", "_strides", name)
            if array != name and array + "[" in body:
                first = next(n for n, _ in cls._fields_ if n.startswith(array[:-7]) and re.fullmatch(array[:-7] + "(page|token|head)", n))
                if name != first:
                    continue
                name_c = array
            else:
                name_c = name
            lines.append('printf("%%zu\\n", offsetof(%s, %s));' % (cls.__name__, name_c))
            want.append(getattr(cls, name).offset)
    src = tmp_path / "layout.c"
    src.write_text('#include "fusedinf.h"\n#include <stdio.h>\n#include <stddef.h>\nint main(void) { %s return 0; }\n' % " ".join(lines))
    exe = str(tmp_path / "layout")
    subprocess.run([gcc, "-I" + os.path.join(ROOT, "include"), str(src), "-o", exe], check=True)
    assert [int(v) for v in subprocess.run([exe], stdout=subprocess.PIPE, text=True, check=True).stdout.split()] == want


def test_tensors_in_host_memory_are_refused():
    import torch
    x, i, b = torch.zeros((4, 2, 64)), torch.zeros(4, dtype=torch.int32), torch.zeros((3, 16, 2, 32), dtype=torch.uint8)
    for call in (lambda: fi.fp4_cache_write(x, None, i.long(), b, b[..., :2]), lambda: fi.fp4_tree_attention(x, b, b, b, b, i[None], i, i), lambda: fi.beam_select(x[0], x[:1, :, 0]),
                 lambda: fi.fork_pages(i[None], i, i, page_size=4), lambda: fi.compact_pages(i[None], i)):
        with pytest.raises(ValueError, match="device memory"):
            call()
    codes, scales = fi.fp4_cache(3, 16, 2, 72, device="cpu")
    assert codes.shape == (3, 16, 2, 36) and scales.shape == (3, 16, 2, 3) and codes.stride(1) == 36 and scales.stride(1) == 3
