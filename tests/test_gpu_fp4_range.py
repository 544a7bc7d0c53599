"""Attention over a 4-bit cache by queries that fill the range of their type.  Bounds as in test_gpu_fp4_cache.py."""
import pytest

from tests.test_gpu_fp4_cache import _held, _ref
from tests.test_gpu_operators import _cu, _inside, _kind, _tree_mask, fi, torch  # noqa: F401

pytestmark = pytest.mark.gpu

# by every way of loading a tile, one column of queries, two and four
CALLS = [([300], [1], 16, 64), ([900, 31], [1, 3], 16, 128), ([40, 7], [9, 3], 5, 128), ([2000], [2], 16, 72), ([150], [17], 48, 96), ([70, 300], [40, 33], 16, 64), ([90], [40], 3, 72),
         ([500, 80], [3, 20], 32, 256), ([60], [5], 7, 256), ([20000, 40], [37, 33], 64, 128)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("cached,counts,page,d", CALLS)
def test_queries_up_to_the_largest_number(torch, fi, dtype, cached, counts, page, d):  # noqa: F811
    """Up to two values of a query are within 4 % of the largest number of its type, the others zero.  Keys are at most 6 / 32, so that scores and their differences stay in fp32's
    range, and a scale of 2^-124 makes ordinary ones of them."""
    g, kind = torch.Generator().manual_seed(21), _kind(torch, dtype)
    (k, v), table, dense = _held(torch, g, cached, counts, page, 2, d, "head")
    ks = k[1].clone()
    ks[ks != 255] -= 5
    for kv in dense:
        kv[0] /= 32
    n = sum(counts)
    q = torch.zeros((n, 4, d))
    largest = torch.finfo(kind).max
    for _ in range(2):
        where = torch.randint(0, d, (n, 4, 1), generator=g)
        q.scatter_(2, where, (1 - 0.04 * torch.rand((n, 4, 1), generator=g)) * largest * (1 - 2 * torch.randint(0, 2, (n, 4, 1), generator=g)))
    q[0, 0, 3], q[0, 1, 5], q[0, 2, d - 1] = largest, -largest, largest
    q = q.to(kind).cuda()
    assert q.isfinite().all()
    bits, scale = _tree_mask(torch, g, counts, "tree"), 2.0 ** -124
    got = fi.fp4_tree_attention(q, k[0], ks, *v, table, torch.tensor(cached, dtype=torch.int32).cuda(), _cu(torch, counts), bits.cuda(), scale=scale, max_nodes=max(counts),
                                max_length=max(c + m for c, m in zip(cached, counts)))
    want, bound = _ref(torch, q, dense, cached, counts, bits, scale, dtype)
    assert want.isfinite().all() and want.abs().max() > 0.1
    _inside(got.double().cpu(), want, bound)
