"""The 4-bit cache against its definition: codes and scales bit for bit, attention against 64 bits over the values that the cache holds.

Bounds of attention as in test_gpu_operators.py; the cache's values enter exactly.  fp32 queries and weights enter in three bf16 terms (24 bits), so a score is a sum of 3 D
products and a weight is rounded by 2^-24 more: three times that bound's term for scores, and 4 u beside its 64."""
import math

import pytest

from tests import fp4_oracle as oracle
from tests.test_gpu_operators import H, U, _cu, _inside, _kind, _rows, _tree_mask, fi, torch  # noqa: F401

pytestmark = pytest.mark.gpu


def _cache(torch, pages, page, heads, d, order, fill=0xA5):  # noqa: F811
    """Codes and scales of one half, in memory by head ('head'), by token ('token') or with gaps ('wide')."""
    blocks = (d + 31) // 32
    if order == "head":
        c, s = (torch.full((pages, heads, page, n), fill, dtype=torch.uint8).cuda().permute(0, 2, 1, 3) for n in (d // 2, blocks))
        return c, s
    if order == "token":
        return tuple(torch.full((pages, page, heads, n), fill, dtype=torch.uint8).cuda() for n in (d // 2, blocks))
    c = torch.full((pages, page, heads + 1, d // 2 + 4), fill, dtype=torch.uint8).cuda()[:, :, 1:, 4:]
    return c, torch.full((pages, page + 1, heads, blocks + 1), fill, dtype=torch.uint8).cuda()[:, 1:, :, 1:]


WRITES = [
    # tokens, heads, head dim, page, rows, order
    (1, 8, 128, 16, "plain", "head"), (7, 1, 64, 1, "wide", "token"), (130, 4, 72, 48, "plain", "head"), (33, 5, 80, 3, "odd", "wide"), (257, 2, 256, 64, "wide", "head"),
    (65, 3, 96, 16, "plain", "token"), (9, 2, 8, 4, "plain", "head"), (19, 1, 40, 5, "odd", "wide"), (5000, 2, 128, 16, "wide", "head"), (3, 70, 256, 2, "plain", "head"),
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("tokens,heads,d,page,layout,order", WRITES)
def test_write(torch, fi, dtype, tokens, heads, d, page, layout, order):  # noqa: F811
    g, kind = torch.Generator().manual_seed(1), _kind(torch, dtype)
    k, v = (_rows(torch, g, (tokens, heads, d), kind, layout) for _ in range(2))
    k *= torch.exp2(torch.randint(-30, 30, (tokens, heads, 1), generator=g)).to(kind).cuda()
    pages = (tokens + page - 1) // page + 2
    slots = torch.randperm(pages * page, generator=g)[:tokens]
    slots[::7] = torch.tensor([-1, pages * page, -(1 << 40), 1 << 40])[torch.arange(len(slots[::7])) % 4]   # not for the cache
    inside = (slots >= 0) & (slots < pages * page)
    kc, ks = _cache(torch, pages, page, heads, d, order)
    vc, vs = _cache(torch, pages, page, heads, d, order)
    held = [torch.zeros_like(k), torch.zeros_like(v)]
    assert fi.fp4_cache_write(k, v, slots.cuda(), kc, ks, vc, vs, k_held=held[0], v_held=held[1])[1] is held[1]
    for x, c, s, h in ((k, kc, ks, held[0]), (v, vc, vs, held[1])):
        codes, scales, values = oracle.write(x)
        want_c, want_s = torch.full((pages * page, heads, d // 2), 0xA5, dtype=torch.uint8), torch.full((pages * page, heads, scales.shape[-1]), 0xA5, dtype=torch.uint8)
        want_c[slots[inside]], want_s[slots[inside]] = codes[inside], scales[inside]
        assert torch.equal(c.reshape(want_c.shape).cpu(), want_c) and torch.equal(s.reshape(want_s.shape).cpu(), want_s)
        assert torch.equal(h.double().cpu(), values)
    k1, s1 = _cache(torch, pages, page, heads, d, order)
    assert fi.fp4_cache_write(k, None, slots.cuda(), k1, s1) == (None, None)
    assert torch.equal(k1, kc) and torch.equal(s1, ks)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_write_on_borders_and_at_the_ends_of_the_range(torch, fi, dtype):  # noqa: F811
    """Every border between codes and scales in every binade, the largest and smallest numbers, zeros of both signs; blocks with NaN or an infinity."""
    kind, info = _kind(torch, dtype), torch.finfo(_kind(torch, dtype))
    borders = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0, 7.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0])
    rows = []
    for e in list(range(-140, 126, 7)) + [-126, -125, -124, 124, 125]:
        for top in (6.0, 3.0625, 4.0, 5.5):
            x = torch.cat([torch.tensor([top]), borders, -borders, torch.tensor([-0.0])]).double() * 2.0 ** e
            rows += [x, x * (1 + info.eps), x * (1 - info.eps)]
    x = torch.stack(rows).clamp(-info.max, info.max).to(kind)
    special = torch.zeros((8, 32), dtype=kind)
    special[0, 3], special[1, 31], special[2, 0], special[3, 5], special[4], special[5], special[6, 1] = math.nan, math.inf, -math.inf, info.max, -info.max, info.tiny, info.smallest_normal / 2
    x = torch.cat([x, special])[:, None].cuda()
    n = x.shape[0]
    codes, scales = _cache(torch, n, 1, 1, 32, "head")
    held = torch.zeros_like(x)
    fi.fp4_cache_write(x, None, torch.arange(n).cuda(), codes, scales, k_held=held)
    want = oracle.write(x)
    assert torch.equal(scales.reshape(want[1].shape).cpu(), want[1])
    assert torch.equal(codes.reshape(want[0].shape).cpu(), want[0])
    assert torch.equal(held.double().cpu().nan_to_num(1e300), want[2].nan_to_num(1e300))


# ---- attention ----------------------------------------------------------------------------------
def _held(torch, g, cached, counts, page, hk, d, order, spare=3):  # noqa: F811
    """A cache whose unwritten places hold NaN, its table in random order, and what every sequence holds."""
    need = [(c + n + page - 1) // page for c, n in zip(cached, counts)]
    pages = sum(need) + spare
    halves = [_cache(torch, pages, page, hk, d, order, fill=255) for _ in range(2)]
    numbers, table, at, dense = torch.randperm(pages, generator=g), torch.full((len(need), max(need + [1]) + 1), pages - 1, dtype=torch.int32), 0, []
    for b, (c, n, count) in enumerate(zip(cached, counts, need)):
        table[b, :count] = numbers[at:at + count].int()
        at += count
        kv, place = [], torch.arange(c + n)
        where = (table[b, place // page].long().cuda(), (place % page).cuda())
        for codes, scales in halves:
            w, s = torch.randint(0, 256, (c + n, hk, d // 2), generator=g, dtype=torch.uint8), torch.randint(124, 128, (c + n, hk, (d + 31) // 32), generator=g).to(torch.uint8)
            codes[where], scales[where] = w.cuda(), s.cuda()
            kv.append(oracle.read(w, s))
        dense.append(torch.stack(kv))
    return halves, table.cuda(), dense


def _ref(torch, q, dense, cached, counts, bits, scale, dtype, max_nodes=None):  # noqa: F811
    want, bound = torch.zeros(q.shape).double(), torch.full(q.shape, 1e-30).double()
    q, at = q.cpu().double(), 0
    half, terms = (H, 1) if dtype == "bf16" else (0.0, 3)
    for kv, c, n in zip(dense, cached, counts):
        m = n if max_nodes is None else min(n, max_nodes)
        seen = torch.ones((m, c + m), dtype=torch.bool)
        if bits is None:
            seen = seen.tril(c)
        else:
            for j in range(m):
                seen[:, c + j] = (bits[at:at + m, j // 64] >> (j % 64)) & 1 == 1
        group, d = q.shape[1] // kv.shape[2], q.shape[2]
        for h in range(q.shape[1]) if c + m else []:
            k, v, x = kv[0, :c + m, h // group], kv[1, :c + m, h // group], q[at:at + m, h]
            s = x @ k.t() * scale
            e = (terms * (d + 2) * U * (x.abs() @ k.abs().t()) * scale).masked_fill(~seen, 0.0).amax(1, keepdim=True)
            p = torch.softmax(s.masked_fill(~seen, -math.inf), 1).nan_to_num(0.0)
            y, size = p @ v, p @ v.abs()
            want[at:at + m, h] = y
            bound[at:at + m, h] = size * (2 * (e + 68 * U) + 2 * (terms * (c + m) + 8) * U + 1.01 * half) + y.abs() * 1.01 * half + 1e-30
        at += n
    return want, bound


TREES = [
    # cached, counts, page, hq, hk, d, rows, order, mask
    ([1003], [1], 16, 32, 8, 128, "plain", "head", None),
    ([0], [1], 16, 4, 4, 64, "plain", "head", None),
    ([5, 0, 31, 32, 33], [1, 1, 1, 1, 1], 16, 8, 2, 128, "wide", "token", None),
    ([64, 7, 200], [1, 1, 1], 1, 5, 5, 72, "odd", "wide", None),
    ([130, 0, 3], [5, 0, 2], 48, 16, 2, 72, "plain", "head", "tree"),
    ([77, 500], [37, 12], 64, 28, 4, 128, "wide", "head", "tree"),
    ([77, 50], [70, 130], 16, 8, 4, 80, "odd", "token", "tree"),
    ([30, 2], [9, 16], 5, 12, 4, 96, "plain", "wide", "empty"),
    ([100, 1], [3, 20], 256, 8, 1, 256, "plain", "head", "tree"),
    ([300], [40], 16, 2, 2, 256, "odd", "token", "tree"),
    ([700], [2], 7, 3, 1, 40, "plain", "wide", None),
    ([65], [1], 32, 40, 1, 8, "plain", "head", None),
    ([4000], [1], 16, 8, 8, 64, "plain", "head", None),
    ([90, 11], [64, 3], 16, 1, 1, 64, "plain", "head", "tree"),
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("cached,counts,page,hq,hk,d,layout,order,mask", TREES)
def test_attention(torch, fi, dtype, cached, counts, page, hq, hk, d, layout, order, mask):  # noqa: F811
    g, kind = torch.Generator().manual_seed(2), _kind(torch, dtype)
    (k, v), table, dense = _held(torch, g, cached, counts, page, hk, d, order)
    q = _rows(torch, g, (sum(counts), hq, d), kind, layout)
    bits = None if mask is None else _tree_mask(torch, g, counts, mask)
    want, bound = _ref(torch, q, dense, cached, counts, bits, d ** -0.5, dtype)
    for hint in (dict(), dict(max_nodes=max(counts), max_length=max(c + n for c, n in zip(cached, counts)))):
        out = torch.full((sum(counts), hq + 1, d + 8), math.nan, dtype=kind).cuda()[:, 1:, 8:]
        got = fi.fp4_tree_attention(q, *k, *v, table, torch.tensor(cached, dtype=torch.int32).cuda(), _cu(torch, counts), None if bits is None else bits.cuda(), out=out, **hint)
        assert got is out
        _inside(got.double().cpu(), want, bound)


LINES = [
    ([5000, 3, 900, 40, 0, 2500], [1] * 6, 16, 32, 8, 128), ([3000, 10, 800], [37, 5, 20], 64, 16, 4, 72), ([9000, 100], [2, 3], 48, 4, 4, 64),
    ([2000, 1999, 1, 64], [6, 6, 6, 6], 3, 8, 2, 256), ([1200] * 40, [1] * 40, 32, 8, 8, 128), ([700, 20] * 8, [33, 64] * 8, 16, 8, 1, 128),
]


# much to share out for a call of one column of queries, of two, of four and of heads of 256, by every way of loading a tile
SHARED = [
    ([60000, 3, 9000, 0, 700], [1] * 5, 16, 16, 4, 64), ([70000, 12, 20000], [2, 5, 1], 64, 5, 5, 72), ([50000, 300, 4000, 31], [2] * 4, 16, 24, 6, 128),
    ([60000, 3, 800, 9, 65], [1, 2, 1, 1, 3], 3, 12, 4, 128), ([20000, 40, 900], [6, 1, 8], 32, 12, 2, 256), ([24000, 7, 500, 2100], [12, 3, 9, 1], 16, 8, 4, 64),
    ([30000, 10, 800], [37, 5, 20], 64, 16, 4, 72), ([30000, 3, 700], [64, 9, 30], 16, 8, 2, 128), ([30000, 40], [64, 33], 48, 8, 4, 64), ([16000, 40], [64, 33], 5, 8, 4, 64),
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("cached,counts,page,hq,hk,d", LINES + SHARED)
def test_attention_of_ragged_histories(torch, fi, dtype, cached, counts, page, hq, hk, d):  # noqa: F811
    """Histories that are cut and joined, and such that all workgroups share."""
    g, kind = torch.Generator().manual_seed(3), _kind(torch, dtype)
    (k, v), table, dense = _held(torch, g, cached, counts, page, hk, d, "head")
    q = _rows(torch, g, (sum(counts), hq, d), kind, "plain")
    bits = _tree_mask(torch, g, counts, "tree")
    got = fi.fp4_tree_attention(q, *k, *v, table, torch.tensor(cached, dtype=torch.int32).cuda(), _cu(torch, counts), bits.cuda(), max_nodes=max(counts),
                                max_length=max(c + n for c, n in zip(cached, counts)))
    _inside(got.double().cpu(), *_ref(torch, q, dense, cached, counts, bits, d ** -0.5, dtype))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("scale", [1e-3, 30.0])
def test_attention_of_even_and_far_apart_scores(torch, fi, dtype, scale):  # noqa: F811
    """Weights all alike, or one that leaves the others nothing: the running maximum moves or never does."""
    g, kind, cached, counts = torch.Generator().manual_seed(4), _kind(torch, dtype), [1500, 9], [3, 2]
    (k, v), table, dense = _held(torch, g, cached, counts, 16, 2, 64, "head")
    q = _rows(torch, g, (5, 4, 64), kind, "plain")
    got = fi.fp4_tree_attention(q, *k, *v, table, torch.tensor(cached, dtype=torch.int32).cuda(), _cu(torch, counts), scale=scale)
    want, bound = _ref(torch, q, dense, cached, counts, None, scale, dtype)
    if scale > 1:   # the argument of exp is rounded at its own size: |score| u, twice
        top = max(float((q.cpu().double().abs().amax() * kv[0].abs().amax() * 64 * scale)) for kv in dense)
        bound = bound + 4 * top * U * max(float(kv[1].abs().amax()) for kv in dense)
    _inside(got.double().cpu(), want, bound)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,counts,page", [(64, [5, 9], 16), (72, [40, 33], 3), (128, [3, 4], 16), (256, [6, 7], 32), (96, [20, 70], 16)])
def test_a_branch_does_not_see_another(torch, fi, dtype, d, counts, page):  # noqa: F811
    """A block of NaN in the keys or values of one node reaches the nodes below it and no other; of a value, its own 32 results."""
    g, kind, cached, hk = torch.Generator().manual_seed(5), _kind(torch, dtype), [70, 33], 2
    (k, v), table, _ = _held(torch, g, cached, counts, page, hk, d, "head")
    q, bits = _rows(torch, g, (sum(counts), 8, d), kind, "plain"), _tree_mask(torch, g, counts, "tree")
    args = (table, torch.tensor(cached, dtype=torch.int32).cuda(), _cu(torch, counts), bits.cuda())
    clean = fi.fp4_tree_attention(q, *k, *v, *args)
    assert clean.isfinite().all()
    sees = torch.zeros(sum(counts), dtype=torch.bool)
    sees[counts[0]:] = (bits[counts[0]:, 0] >> 2) & 1 == 1
    assert sees[counts[0] + 2] and not sees.all()
    sees, place, block = sees.cuda(), cached[1] + 2, (d - 1) // 32
    where = (int(table[1, place // page]), place % page, 1, block)
    for half in (k, v):
        bad = half[1].clone()
        bad[where] = 255
        got = fi.fp4_tree_attention(q, *((half[0], bad) if half is k else k), *((half[0], bad) if half is v else v), *args)
        assert torch.equal(got[~sees], clean[~sees]) and torch.equal(got[:, :4], clean[:, :4])
        hit = got[sees][:, 4:]
        assert hit.isnan().all() if half is k else hit[..., 32 * block:].isnan().all() and torch.equal(hit[..., :32 * block], clean[sees][:, 4:, :32 * block])
    # of a committed token: all nodes of the sequence
    bad = v[1].clone()
    bad[int(table[1, 4 // page]), 4 % page, 0, 0] = 255
    got = fi.fp4_tree_attention(q, *k, v[0], bad, *args)
    assert got[counts[0]:, :4, :32].isnan().all() and torch.equal(got[:counts[0]], clean[:counts[0]]) and torch.equal(got[:, 4:], clean[:, 4:])
    assert torch.equal(got[counts[0]:, :4, 32:], clean[counts[0]:, :4, 32:])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_no_history_no_nodes_no_pages(torch, fi, dtype):  # noqa: F811
    kind = _kind(torch, dtype)
    q, lengths = torch.ones((3, 4, 64), dtype=kind).cuda(), torch.zeros(2, dtype=torch.int32).cuda()
    (kc, ks), (vc, vs) = (_cache(torch, 2, 16, 2, 64, "head", fill=255) for _ in range(2))
    table, cu = torch.zeros((2, 1), dtype=torch.int32).cuda(), _cu(torch, [1, 2])
    none = torch.zeros((3, 1), dtype=torch.int64).cuda()
    out = torch.full_like(q, math.nan)
    assert not fi.fp4_tree_attention(q, kc, ks, vc, vs, table, lengths, cu, none, out=out).any()   # rows that see nothing
    empty = [x[:0] for x in (kc, ks, vc, vs)]
    assert not fi.fp4_tree_attention(q, *empty, table, lengths + 5, cu, out=torch.full_like(q, math.nan)).any()
    assert not fi.fp4_tree_attention(q, kc, ks, vc, vs, table[:, :0], lengths + 5, cu, out=torch.full_like(q, math.nan)).any()
    assert fi.fp4_tree_attention(q[:0], kc, ks, vc, vs, table, lengths, cu * 0).shape == (0, 4, 64)
    x = torch.ones((2, 2, 64), dtype=kind).cuda()
    held = torch.zeros_like(x)
    fi.fp4_cache_write(x, x, torch.tensor([0, 16]).cuda(), *empty, k_held=held)
    assert torch.equal(held, x)
    fi.fp4_cache_write(x[:0], x[:0], torch.zeros(0, dtype=torch.int64).cuda(), kc, ks, vc, vs)
    assert (kc == 255).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("nodes", [5, 90])
def test_nodes_past_max_nodes_are_neither_computed_nor_seen(torch, fi, dtype, nodes):  # noqa: F811
    g, kind, most = torch.Generator().manual_seed(6), _kind(torch, dtype), nodes - 3
    (k, v), table, dense = _held(torch, g, [10], [nodes], 16, 2, 64, "head")
    q = _rows(torch, g, (nodes, 4, 64), kind, "plain")
    mask = torch.full((nodes, 2), -1, dtype=torch.int64)
    out = torch.full((nodes, 4, 64), 7.0, dtype=kind).cuda()
    fi.fp4_tree_attention(q, *k, *v, table, torch.tensor([10], dtype=torch.int32).cuda(), _cu(torch, [nodes]), mask.cuda(), max_nodes=most, out=out)
    want, bound = _ref(torch, q, dense, [10], [nodes], mask, 64 ** -0.5, dtype, max_nodes=most)
    _inside(out[:most].double().cpu(), want[:most], bound[:most])
    assert (out[most:] == 7).all()


def test_thousands_of_single_tokens_with_nothing_said_about_them(torch, fi):  # noqa: F811
    g, n = torch.Generator().manual_seed(7), 24000
    (k, v), _, _ = _held(torch, g, [0], [16 * 50], 16, 2, 64, "head", spare=0)
    table = torch.randint(0, 50, (n, 1), generator=g, dtype=torch.int32).cuda()
    q = torch.randn((n, 8, 64), generator=g).bfloat16().cuda()
    got = fi.fp4_tree_attention(q, *k, *v, table, torch.full((n,), 3, dtype=torch.int32).cuda(), torch.arange(n + 1, dtype=torch.int32).cuda())
    pick = torch.randint(0, n, (40,), generator=g)
    dense = [torch.stack([oracle.read(*(x[int(table[i, 0]), :4] for x in half)) for half in (k, v)]) for i in pick]
    _inside(got[pick.cuda()].double().cpu(), *_ref(torch, q[pick.cuda()], dense, [3] * 40, [1] * 40, None, 0.125, "bf16"))


def test_cache_offsets_beyond_32_bits(torch, fi):  # noqa: F811
    """Codes and scales past 2^32 bytes, written through slots and read through the table."""
    page, hk, d = 256, 8, 128
    many = (1 << 32) // (page * hk * d // 2) + 40
    g = torch.Generator().manual_seed(8)
    x = torch.randn((600, 2 * hk, d), generator=g).bfloat16().cuda()
    place, q = torch.arange(600), torch.randn((1, 16, d), generator=g).bfloat16().cuda()
    lengths, cu = torch.tensor([599], dtype=torch.int32).cuda(), _cu(torch, [1])
    want = None
    for n in (40, many):
        halves = [fi.fp4_cache(n, page, hk, d) for _ in range(2)]
        order = n - 1 - torch.tensor([4, 0, 2], dtype=torch.int32)
        slots = (order[place // page].long() * page + place % page).cuda()
        fi.fp4_cache_write(x[:, :hk], x[:, hk:], slots, *halves[0], *halves[1])
        got = fi.fp4_tree_attention(q, *halves[0], *halves[1], order[None].cuda(), lengths, cu)
        want = got if want is None else want
        assert torch.equal(got, want) and got.abs().sum() > 0
        del halves
    # scales far apart: a page stride that passes 32 bits over the pages
    codes = [torch.zeros((3, hk, page, d // 2), dtype=torch.uint8, device="cuda").permute(0, 2, 1, 3) for _ in range(2)]
    wide = torch.zeros((2 << 32) + (1 << 20), dtype=torch.uint8, device="cuda")
    scales = [torch.as_strided(wide, (3, page, hk, 4), (1 << 32, hk * 4, 4, 1), at) for at in (0, 1 << 19)]
    slots = (torch.tensor([2, 0, 1])[place // page] * page + place % page).cuda()
    fi.fp4_cache_write(x[:, :hk], x[:, hk:], slots, codes[0], scales[0], codes[1], scales[1])
    got = fi.fp4_tree_attention(q, codes[0], scales[0], codes[1], scales[1], torch.tensor([[2, 0, 1]], dtype=torch.int32).cuda(), lengths, cu)
    assert torch.equal(got, want)


def test_more_slots_than_32_bits_count(torch, fi):  # noqa: F811
    page, g = 4099, torch.Generator().manual_seed(12)
    pages = (1 << 32) // page + 3
    codes, scales = (torch.empty((pages, page, 1, n), dtype=torch.uint8, device="cuda") for n in (4, 1))
    slots = torch.tensor([pages * page - 1, 5, -1, (1 << 32) + 7, 1 << 32, pages * page, (1 << 32) - 1])
    for t in (codes, scales):
        t.view(pages * page, -1)[slots[[0, 1, 3, 4, 6]].cuda()] = 77
    x = torch.randn((7, 1, 8), generator=g).bfloat16().cuda()
    fi.fp4_cache_write(x, None, slots.cuda(), codes, scales)
    want = oracle.write(x)
    kept = [0, 1, 3, 4, 6]
    at = slots[kept].cuda()
    assert torch.equal(codes.view(pages * page, 4)[at].cpu(), want[0][kept][:, 0]) and torch.equal(scales.view(-1)[at].cpu(), want[1][kept].view(-1))


def test_damaged_tables_stay_inside_the_cache(torch, fi):  # noqa: F811
    g, cached, counts = torch.Generator().manual_seed(9), [100, 60], [4, 4]
    (k, v), table, _ = _held(torch, g, cached, counts, 16, 2, 64, "head")
    q, cu = _rows(torch, g, (8, 4, 64), torch.bfloat16, "plain"), _cu(torch, counts)
    lengths = torch.tensor(cached, dtype=torch.int32).cuda()
    want = fi.fp4_tree_attention(q, *k, *v, table, lengths, cu)
    bad, long, negative = table.clone(), lengths.clone(), lengths.clone()
    bad[1, 1], bad[1, 2], long[1], negative[1] = -7, 1 << 30, 1 << 30, -5
    for t, c in ((bad, lengths), (table, long), (bad, long), (table, negative)):
        assert torch.equal(fi.fp4_tree_attention(q, *k, *v, t, c, cu)[:4], want[:4])
    fi.fp4_tree_attention(q, *k, *v, table, lengths, torch.tensor([3, 1 << 30, -2], dtype=torch.int32).cuda())
    torch.cuda.synchronize()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("cached,counts", [([40, 3], [1, 2]), ([900, 33], [1, 2]), ([30000, 5, 9000], [9, 0, 7])])
def test_rows_behind_the_last_sequence_stay_as_they_were(torch, fi, dtype, cached, counts):  # noqa: F811
    """A padded batch: a wave for each history, parts that are joined, stretches that all workgroups share."""
    g, kind, all_rows = torch.Generator().manual_seed(10), _kind(torch, dtype), sum(counts) + 21
    (k, v), table, dense = _held(torch, g, cached, counts, 16, 2, 128, "head")
    q = _rows(torch, g, (all_rows, 16, 128), kind, "plain")
    q[sum(counts):] = math.nan
    out = torch.full((all_rows, 16, 128), 7.0, dtype=kind).cuda()
    want, bound = _ref(torch, q[:sum(counts)], dense, cached, counts, None, 128 ** -0.5, dtype)
    args = (table, torch.tensor(cached, dtype=torch.int32).cuda(), _cu(torch, counts))
    for hint in (dict(), dict(max_nodes=max(counts), max_length=max(c + n for c, n in zip(cached, counts)))):
        fi.fp4_tree_attention(q, *k, *v, *args, out=out, **hint)
        _inside(out[:sum(counts)].double().cpu(), want, bound)
        assert (out[sum(counts):] == 7).all()


def test_calls_on_two_streams_at_once(torch, fi):  # noqa: F811
    """Each call has a workspace of its own, so neither sees the other."""
    g, cached, counts = torch.Generator().manual_seed(11), [30000, 5, 9000], [9, 0, 7]
    (k, v), table, _ = _held(torch, g, cached, counts, 16, 2, 128, "head")
    q = [_rows(torch, g, (16, 16, 128), torch.bfloat16, "plain") for _ in range(2)]
    args = (table, torch.tensor(cached, dtype=torch.int32).cuda(), _cu(torch, counts))
    want = [fi.fp4_tree_attention(x, *k, *v, *args, max_nodes=9, max_length=30009) for x in q]
    streams, got = [torch.cuda.Stream() for _ in q], [[], []]
    torch.cuda.synchronize()
    for _ in range(10):
        for x, s, into in zip(q, streams, got):
            with torch.cuda.stream(s):
                into.append(fi.fp4_tree_attention(x, *k, *v, *args, max_nodes=9, max_length=30009))
    torch.cuda.synchronize()
    assert all(torch.equal(x, w) for into, w in zip(got, want) for x in into)
