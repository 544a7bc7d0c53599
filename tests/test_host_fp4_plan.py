"""How attention over a 4-bit cache is shared out where lengths may differ: stretches for as many workgroups as run at a time, which goes by how tiles are loaded and so by the
page size and the head's; the workspace tells (no device is touched)."""
import pytest

import paper_2410_21120_amd as fi

# head dim, page size, nodes of a sequence (rows of a block: 16, 32, 64), type, workgroups on a unit: what the registers of these kernels leave room for
KERNELS = [
    (128, 16, 1, "bf16", 4), (128, 8, 1, "bf16", 2), (112, 16, 1, "bf16", 3), (96, 48, 1, "bf16", 4), (72, 1, 1, "bf16", 2), (64, 16, 1, "bf16", 4), (64, 1, 1, "bf16", 3),
    (128, 16, 20, "bf16", 2), (128, 5, 20, "bf16", 1), (64, 64, 20, "bf16", 2), (64, 7, 20, "bf16", 2), (128, 16, 40, "bf16", 2), (96, 16, 40, "bf16", 2), (64, 24, 40, "bf16", 1),
    (128, 24, 40, "bf16", 1), (256, 16, 1, "bf16", 2), (192, 16, 1, "bf16", 1), (256, 8, 1, "bf16", 1), (128, 16, 1, "f32", 3), (72, 16, 1, "f32", 3), (128, 8, 1, "f32", 1),
    (64, 16, 1, "f32", 3), (64, 8, 1, "f32", 2), (72, 48, 20, "f32", 2), (72, 3, 20, "f32", 1), (64, 3, 20, "f32", 2), (256, 16, 1, "f32", 1),
]


@pytest.mark.parametrize("d,page,nodes,dtype,on_unit", KERNELS)
def test_stretches_for_as_many_workgroups_as_run_at_a_time(d, page, nodes, dtype, on_unit):
    seqs, heads, length = 4, 32, 32000
    a = fi.fi_fp4_tree_attention_args(dtype=fi.FI_F32 if dtype == "f32" else fi.FI_BF16, n_seqs=seqs, q_heads=heads, kv_heads=heads, head_dim=d, page_size=page, n_pages=1 << 20,
                                      table_columns=-(-length // page), mask_words=1, max_nodes=nodes, max_length=length, scale=0.1, nodes=seqs * nodes)
    per_part, header = seqs * nodes * heads * (d + 2), 4 + seqs
    parts = (fi.fi_fp4_tree_attention_workspace(a) // 4 - header) / per_part
    assert parts == -(-256 * on_unit // heads) + 1   # (of a history: one more than it has whole stretches)
