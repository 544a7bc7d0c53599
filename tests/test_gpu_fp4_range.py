"""Attention over a 4-bit cache by queries that fill the range of their type, and how many bits its softmax weights have.  Bounds as in test_gpu_fp4_cache.py."""
import pytest

from tests.test_gpu_fp4_cache import _held, _ref
from tests.test_gpu_operators import H, U, _cu, _inside, _kind, _rows, _tree_mask, fi, torch  # noqa: F401

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


# up to 32 rows a key head (any number in heads of more than 128), a wave a workgroup and four, by every way of loading a tile: nodes, cached, page, query heads, key heads, head dim
WEIGHTS = [(1, 30, 16, 32, 8, 128), (8, 40, 16, 32, 8, 128), (1, 150, 16, 32, 8, 128), (8, 190, 64, 32, 8, 128), (5, 100, 48, 8, 2, 72), (3, 120, 5, 8, 2, 64), (6, 30, 16, 8, 2, 64),
           (1, 90, 1, 8, 8, 96), (9, 100, 16, 6, 2, 112), (40, 20, 16, 4, 2, 256), (4, 100, 7, 16, 2, 192)]


@pytest.mark.parametrize("nodes,cached,page,hq,hk,d", WEIGHTS)
def test_weights_have_16_bits(torch, fi, nodes, cached, page, hq, hk, d):  # noqa: F811
    """Of n keys, with e the error of a score as in test_gpu_operators.py: 2 (e + 68 u) + 2 (n + 8) u and, for weights of two bf16 terms, h^2, relative to sum of weight times |value|, and the result's
    rounding.  Small queries make e small and the weights alike.  Weights of one term (done here in 64 bits) are outside of that bound."""
    g = torch.Generator().manual_seed(22)
    (k, v), table, dense = _held(torch, g, [cached], [nodes], page, hk, d, "head")
    q = (0.1 * _rows(torch, g, (nodes, hq, d), torch.bfloat16, "plain")).contiguous()
    got = fi.fp4_tree_attention(q, *k, *v, table, torch.tensor([cached], dtype=torch.int32).cuda(), _cu(torch, [nodes]), max_nodes=nodes, max_length=cached + nodes)
    x, n, scale, coarse = q.double().cpu(), cached + nodes, d ** -0.5, 0
    seen = torch.ones((nodes, n), dtype=torch.bool).tril(cached)
    for h in range(hq):
        keys, values = dense[0][:, :, h // (hq // hk)]
        s = (x[:, h] @ keys.t() * scale).masked_fill(~seen, float("-inf"))
        e = ((d + 2) * U * (x[:, h].abs() @ keys.abs().t()) * scale).amax(1, keepdim=True)
        w = (s - s.amax(1, keepdim=True)).exp()
        total = w.sum(1, keepdim=True)
        want, size = w @ values / total, w @ values.abs() / total
        bound = size * (2 * (e + 68 * U) + 2 * (n + 8) * U + 1.01 * H * H) + 1.01 * H * want.abs() + 1e-30
        _inside(got[:, h].double().cpu(), want, bound)
        coarse += int(((w.bfloat16().double() @ values / total - want).abs() > bound).sum())
    assert coarse > 0
