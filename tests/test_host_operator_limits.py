"""What the decoder operators refuse beyond single arguments: outputs whose rows share memory (no device is touched: the checks come before any launch)."""
import pytest

import paper_2410_21120_amd as fi
from tests.test_host_operators import P, prompt, rope, tree

PAGED = dict(slots=P, page_size=16, n_slots=64, k_out_page=2048, v_out_page=2048)   # 4 pages of 16 tokens, 2 heads of 64
OVERLAPPING = [
    # (token 0, head 1) and (token 1, head 0) are one row, or share a part of one
    (rope, dict(q_out_token=64, q_out_head=64)), (rope, dict(q_out_token=255)), (rope, dict(q_out_token=64, q_out_head=191)), (rope, dict(k_out_token=64)),
    (rope, dict(v_out_token=127, v_out_head=64)), (prompt, dict(out_token=64, out_head=64)), (prompt, dict(out_token=255)), (prompt, dict(out_token=64, out_head=190)),
    (tree, dict(out_token=64, out_head=64)), (tree, dict(out_token=192)),
    # pages
    (rope, dict(PAGED, k_out_page=64)), (rope, dict(PAGED, v_out_page=2047)), (rope, dict(PAGED, k_out_token=64, k_out_head=64)),
    (rope, dict(PAGED, k_out_page=64, k_out_token=256, k_out_head=255)), (rope, dict(PAGED, v_out_token=127)),
]


@pytest.mark.parametrize("make,change", OVERLAPPING, ids=lambda v: getattr(v, "__name__", None) or "-".join(v))
def test_outputs_whose_rows_share_memory_are_refused(make, change):
    call, args = make(**change)
    with pytest.raises(fi.FiError) as e:
        call(args)
    assert e.value.status == fi.FI_EINVAL and "overlap" in fi.fi_last_error()


MORE_THAN_A_LAUNCH = [
    # 2^32 threads and more along a grid's first dimension: well-formed, not covered, nothing launched
    (rope, dict(tokens=1 << 27)), (prompt, dict(q_tokens=1 << 30, k_tokens=1 << 30)), (prompt, dict(q_tokens=1 << 27, q_token=257)),
    (prompt, dict(n_seqs=1 << 25, q_tokens=1 << 25)), (tree, dict(nodes=1 << 27, q_token=257)), (tree, dict(nodes=1 << 28, n_seqs=1 << 28, max_nodes=1)),
    (tree, dict(nodes=1 << 28, n_seqs=1 << 28, max_nodes=1 << 28)), (tree, dict(nodes=1 << 28, n_seqs=1 << 28, max_nodes=1 << 28, dtype=fi.FI_F32)),
]


@pytest.mark.parametrize("make,change", MORE_THAN_A_LAUNCH, ids=lambda v: getattr(v, "__name__", None) or "-".join(v))
def test_more_work_than_a_launch_takes_is_refused(make, change):
    call, args = make(**change)
    with pytest.raises(fi.FiError) as e:
        call(args)
    assert e.value.status == fi.FI_EUNSUPPORTED and "launch" in fi.fi_last_error()


def test_tensors_that_want_a_derivative_are_refused():
    """There is none to give: a result that is cut off from its inputs would train nothing, in silence."""
    import torch
    from torch.autograd import forward_ad
    x, cu = torch.zeros((2, 4, 64)), torch.tensor([0, 2], dtype=torch.int32)
    wants = torch.zeros((2, 4, 64), requires_grad=True)
    for q, k, v in ((wants, x, x), (x, wants, x), (x, x, wants * 2)):
        with pytest.raises(ValueError, match="gradient"):
            fi.prompt_attention(q, k, v, cu)
        with torch.no_grad(), pytest.raises(ValueError, match="device memory"):
            fi.prompt_attention(q, k, v, cu)
    with forward_ad.dual_level():
        with pytest.raises(ValueError, match="tangent"):
            fi.prompt_attention(forward_ad.make_dual(x, torch.ones_like(x)), x, x, cu)
    with pytest.raises(ValueError, match="negated"):
        fi.prompt_attention(x, torch._neg_view(x), x, cu)
