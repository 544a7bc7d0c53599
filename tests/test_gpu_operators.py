"""The decoder operators against their definitions in 64 bits on the CPU, on the sizes, strides and masks where they can go wrong.

Bounds are derived, element by element, from what the operators round.  u = 2^-24 is the unit of fp32 (24 significant bits), h = 2^-8 that of bf16 (8):
* norm and rotation: a dozen fp32 operations on values no larger than the pair's, the mean of D squares in fp32, one rounding on store;
* attention: a score's fp32 sum of D products is off by at most (D + 2) u sum |q k| scale =: e; a weight by 2 e relatively (numerator and
  denominator); the sums of n weights and products by (n + 8) u each; on bf16 every weight is rounded (h) before it multiplies
  a value, and the result is rounded (h).  All relative to sum of weight times |value|, the last to |result|;
* 4-bit products: sums of K fp32 terms no larger than 31 scale |x| (a weight may carry an offset through the sum): (K + 8) u of their sum.
"""
import math

import pytest

pytestmark = pytest.mark.gpu

U, H = 2.0 ** -24, 2.0 ** -8


@pytest.fixture(scope="module")
def torch():
    import torch
    return torch


@pytest.fixture(scope="module")
def fi():
    import paper_2410_21120_amd as fi
    return fi


def _kind(torch, dtype):
    return torch.float32 if dtype == "f32" else torch.bfloat16


def _rows(torch, g, shape, kind, layout):
    """A tensor of this shape on the GPU: 'plain', 'wide' (rows of a larger buffer, 16-byte starts) or 'odd' (rows that start on odd elements)."""
    if layout == "plain":
        return torch.randn(shape, generator=g).to(kind).cuda()
    t, heads, d = shape
    pad = 8 if layout == "wide" else 3
    big = torch.randn((t, heads + 2, d + pad), generator=g).to(kind).cuda()
    return big[:, 1:-1, pad - (0 if layout == "wide" else 2):][..., :d] if layout == "odd" else big[:, 1:-1, :d]


def _inside(got, want, bound):
    bad = ~((got - want).abs() <= bound)
    assert not bad.any(), f"{int(bad.sum())} of {bad.numel()} values, worst {float(((got - want).abs() / bound)[bad].max())} of its bound"


# ---- norms, rotation, cache ---------------------------------------------------------------------
def _rope_ref(torch, x, w, positions, inv_freq, sections, eps, interleaved):
    """x [t, heads, d] in 64 bits; the angle is one fp32 product.  Returns the values and their bound before the store."""
    x = x.double().cpu()
    d = x.shape[-1]
    axis = [a for a, n in enumerate(sections) for _ in range(n)]
    pairs = len(axis)
    w = torch.ones(d).double() if w is None else w.double().cpu()
    y = x / (x.square().mean(-1, keepdim=True) + eps).sqrt() * w
    bound = (d / 2 + 16) * U * y.abs()
    angle = (positions.cpu().reshape(x.shape[0], -1)[:, axis].float() * inv_freq.cpu()).double()[:, None]
    c, s = angle.cos(), angle.sin()
    i, j = (slice(0, 2 * pairs, 2), slice(1, 2 * pairs, 2)) if interleaved else (slice(0, pairs), slice(pairs, 2 * pairs))
    a, b = y[..., i].clone(), y[..., j].clone()
    y[..., i], y[..., j] = a * c - b * s, b * c + a * s
    size = (d / 2 + 32) * U * (a.abs() + b.abs())
    bound[..., i], bound[..., j] = size, size
    return y, bound


ROPE = [
    # tokens, q heads, kv heads, head dim, rot, sections, interleaved, layout, page (0: no cache)
    (1, 32, 8, 128, 128, (64,), False, "wide", 16),
    (1, 1, 1, 64, 64, (32,), True, "plain", 0),
    (7, 5, 5, 72, 72, (12, 12, 12), True, "plain", 3),
    (130, 12, 4, 72, 36, (10, 8), False, "wide", 48),
    (33, 28, 4, 80, 40, (20,), True, "odd", 1),
    (257, 8, 1, 256, 256, (64, 32, 32), False, "plain", 64),
    (3, 3, 3, 256, 128, (61, 1, 1, 1), False, "odd", 5),
    (65, 4, 2, 7, 6, (3,), False, "plain", 2),
    (9, 2, 1, 1, 0, (0,), False, "plain", 4),
    (5, 3, 3, 250, 2, (1,), True, "plain", 7),
    (9000, 2, 1, 64, 32, (16,), False, "wide", 16),
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("tokens,hq,hk,d,rot,sections,interleaved,layout,page", ROPE)
def test_norm_rotation_and_cache(torch, fi, dtype, tokens, hq, hk, d, rot, sections, interleaved, layout, page):
    g, kind = torch.Generator().manual_seed(tokens * 1000 + d), _kind(torch, dtype)
    q, k, v = (_rows(torch, g, (tokens, h, d), kind, layout) for h in (hq, hk, hk))
    positions = torch.randint(0, 5000, (tokens, len(sections)), generator=g, dtype=torch.int32).cuda()
    inv_freq = (10000.0 ** -(torch.arange(rot // 2) / max(1, rot // 2))).float().cuda()
    qw, kw = (1 + 0.2 * torch.randn(d, generator=g)).cuda(), None if d == 80 else (1 + 0.2 * torch.randn(d, generator=g)).cuda()
    eps = 1e-5
    want_q, bound_q = _rope_ref(torch, q, qw, positions, inv_freq, sections, eps, interleaved)
    want_k, bound_k = _rope_ref(torch, k, kw, positions, inv_freq, sections, eps, interleaved)
    more = dict(q_weight=qw, k_weight=kw, eps=eps, sections=sections, interleaved=interleaved)
    if not page:
        yq, yk, yv = fi.qk_norm_rope(q, k, v, positions, inv_freq, **more)
    else:
        pages = (tokens + page - 1) // page + 2
        slots = torch.randperm(pages * page, generator=g)[:tokens]
        if tokens > 4:   # padding tokens leave the cache as it is
            slots[1], slots[3] = -1, pages * page
        kept = (slots >= 0) & (slots < pages * page)
        before = torch.randn((2, pages, page, hk, d), generator=g).to(kind).cuda()
        k_cache, v_cache = before.clone()
        yq, _, _ = fi.qk_norm_rope(q, k, v, positions, inv_freq, slots=slots.cuda(), k_out=k_cache, v_out=v_cache, **more)
        at = slots[kept].cuda()
        others = torch.ones(pages * page, dtype=torch.bool)
        others[slots[kept]] = False
        for cache, was in zip((k_cache, v_cache), before):
            assert torch.equal(cache.view(-1, hk, d)[others.cuda()], was.view(-1, hk, d)[others.cuda()])
        yk, yv = k_cache.view(-1, hk, d)[at], v_cache.view(-1, hk, d)[at]
        want_k, bound_k, v = want_k[kept], bound_k[kept], v[kept.cuda()]
    half = H if dtype == "bf16" else 0.0
    for got, want, bound in ((yq, want_q, bound_q), (yk, want_k, bound_k)):
        _inside(got.double().cpu(), want, bound * (1 + half) + half * want.abs() + 1e-30)
    assert torch.equal(yv, v)


def test_norm_rotation_in_place_and_without_values(torch, fi):
    g = torch.Generator().manual_seed(5)
    qkv = torch.randn((37, 12, 64), generator=g).bfloat16().cuda()
    q, k = qkv[:, :8], qkv[:, 8:]
    positions, inv_freq = torch.arange(37, dtype=torch.int32).cuda(), torch.rand(32, generator=g).cuda()
    want_q, want_k, none = fi.qk_norm_rope(q, k, None, positions, inv_freq)
    assert none is None
    fi.qk_norm_rope(q, k, None, positions, inv_freq, q_out=q, k_out=k)
    assert torch.equal(q, want_q) and torch.equal(k, want_k)


def test_norm_of_zeros_infinities_and_no_tokens(torch, fi):
    x = torch.zeros((3, 2, 64), dtype=torch.float32).cuda()
    x[1, 0, 5] = math.inf
    x[2, 1, 7] = math.nan
    positions, inv_freq = torch.arange(3, dtype=torch.int32).cuda(), torch.ones(16).cuda()
    y, yk, _ = fi.qk_norm_rope(x, x[:, :1], None, positions, inv_freq, eps=1e-6)
    assert torch.equal(y[0], torch.zeros(2, 64).cuda()) and torch.equal(y[1, 1], torch.zeros(64).cuda()) and torch.equal(y[2, 0], torch.zeros(64).cuda())
    assert y[2, 1].isnan().all() and y[1, 0, 5].isnan()   # inf / inf
    none = fi.qk_norm_rope(x[:0], x[:0, :1], None, positions[:0], inv_freq)
    assert none[0].shape == (0, 2, 64)


# ---- attention --------------------------------------------------------------------------------------
def _attend_ref(torch, q, k, v, seen, scale, dtype):
    """One head in 64 bits: q [n, d], k and v [keys, d], seen [n, keys].  Returns the values and their bound."""
    q, k, v = q.double(), k.double(), v.double()
    n, d = q.shape
    if k.shape[0] == 0:
        return torch.zeros_like(q), torch.full_like(q, 1e-30)
    k = torch.where(seen.any(0)[:, None], k, 0.0)   # (what nobody sees)
    v = torch.where(seen.any(0)[:, None], v, 0.0)
    s = (q @ k.t()) * scale
    e = ((d + 2) * U * (q.abs() @ k.abs().t()) * scale).masked_fill(~seen, 0.0).amax(1, keepdim=True)
    p = torch.softmax(s.masked_fill(~seen, -math.inf), 1).nan_to_num(0.0)
    y, size = p @ v, p @ v.abs()
    half = H if dtype == "bf16" else 0.0
    # exp's own error and the rounding of its argument (scores up to some tens: 64 u) beside the score's
    bound = size * (2 * (e + 64 * U) + 2 * (k.shape[0] + 8) * U + 1.01 * half) + y.abs() * half * 1.01 + 1e-30
    return y, bound


PROMPTS = [
    # query lengths, extra keys per sequence, q heads, kv heads, head dim, causal, layout
    ([1], [0], 1, 1, 64, True, "plain"),
    ([1, 1, 1], [0, 7, 100], 4, 2, 128, True, "wide"),
    ([33, 1, 0, 64, 129], [0, 0, 0, 0, 0], 12, 4, 64, True, "wide"),
    ([200, 65], [0, 31], 8, 1, 128, True, "plain"),
    ([127, 130], [3, 0], 5, 5, 72, True, "plain"),
    ([127, 130], [3, 0], 5, 5, 72, False, "odd"),
    ([50, 31], [-20, -31], 4, 2, 96, True, "plain"),      # fewer keys than queries: the first queries see nothing, a sequence has no keys
    ([40, 9], [-39, -9], 4, 4, 64, False, "wide"),
    ([70], [0], 2, 1, 256, True, "plain"),
    ([66, 3], [5, 260], 4, 1, 80, True, "wide"),
    ([100], [0], 3, 3, 40, False, "odd"),
    ([64, 128, 192], [64, 0, 1], 2, 2, 32, True, "plain"),
    ([300], [0], 2, 2, 7, True, "plain"),
    ([513], [0], 4, 2, 128, True, "odd"),
]


def _packed(torch, g, counts, heads, d, kind, layout):
    return _rows(torch, g, (sum(counts), heads, d), kind, layout)


def _cu(torch, counts):
    return torch.tensor([sum(counts[:i]) for i in range(len(counts) + 1)], dtype=torch.int32).cuda()


def _prompt_ref(torch, q, k, v, nq, nk, causal, scale, dtype):
    q, k, v = q.cpu(), k.cpu(), v.cpu()
    want, bound = torch.zeros(q.shape).double(), torch.zeros(q.shape).double()
    group, a, b = q.shape[1] // k.shape[1], 0, 0
    for n, keys in zip(nq, nk):
        seen = torch.ones((n, keys), dtype=torch.bool)
        seen = seen.tril(keys - n) if causal else seen
        for h in range(q.shape[1]):
            want[a:a + n, h], bound[a:a + n, h] = _attend_ref(torch, q[a:a + n, h], k[b:b + keys, h // group], v[b:b + keys, h // group], seen, scale, dtype)
        a, b = a + n, b + keys
    return want, bound


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("nq,extra,hq,hk,d,causal,layout", PROMPTS)
def test_prompt_attention(torch, fi, dtype, nq, extra, hq, hk, d, causal, layout):
    g, kind = torch.Generator().manual_seed(sum(nq) * 100 + d), _kind(torch, dtype)
    nk = [n + e for n, e in zip(nq, extra)]
    q, k, v = _packed(torch, g, nq, hq, d, kind, layout), _packed(torch, g, nk, hk, d, kind, layout), _packed(torch, g, nk, hk, d, kind, layout)
    scale = 1.3 * d ** -0.5
    out = torch.full((sum(nq), hq, d), math.nan, dtype=kind).cuda()
    got = fi.prompt_attention(q, k, v, _cu(torch, nq), _cu(torch, nk), causal=causal, scale=scale, out=out)
    want, bound = _prompt_ref(torch, q, k, v, nq, nk, causal, scale, dtype)
    _inside(got.double().cpu(), want, bound)
    again = fi.prompt_attention(q, k, v, _cu(torch, nq), _cu(torch, nk), causal=causal, scale=scale)
    assert torch.equal(again, got)


# Enough rows and heads for the kernel of large calls, whose base addresses also pass 2^31 in their low word somewhere among several tensors
LARGE = [
    ([1100], [0], 128, 8, 128, True), ([515, 700, 1, 300], [0, 77, 600, -120], 104, 4, 64, True), ([1200, 64], [0, 0], 128, 128, 72, False), ([900, 400], [-450, 33], 128, 2, 96, True),
]


@pytest.mark.parametrize("nq,extra,hq,hk,d,causal", LARGE)
def test_prompt_attention_of_many_rows(torch, fi, nq, extra, hq, hk, d, causal):
    g = torch.Generator().manual_seed(sum(nq) + d)
    nk = [n + e for n, e in zip(nq, extra)]
    pad = torch.empty((1 << 30) + 4096 * d, dtype=torch.uint8, device="cuda")   # (moves what follows to other addresses)
    q, k, v = _packed(torch, g, nq, hq, d, torch.bfloat16, "plain"), _packed(torch, g, nk, hk, d, torch.bfloat16, "wide"), _packed(torch, g, nk, hk, d, torch.bfloat16, "plain")
    out = torch.full(q.shape, math.nan, dtype=torch.bfloat16, device="cuda")
    got = fi.prompt_attention(q, k, v, _cu(torch, nq), _cu(torch, nk), causal=causal, out=out)
    want, bound = _prompt_ref(torch, q, k, v, nq, nk, causal, d ** -0.5, "bf16")
    _inside(got.double().cpu(), want, bound)
    assert torch.equal(fi.prompt_attention(q, k, v, _cu(torch, nq), _cu(torch, nk), causal=causal), got)
    if causal:   # nothing leaks from behind the diagonal
        at = nk[0] - 100
        bad_k, bad_v = k.clone(), v.clone()
        bad_k[at, 0, 1], bad_v[at, 1, 2] = math.nan, math.inf
        again = fi.prompt_attention(q, bad_k, bad_v, _cu(torch, nq), _cu(torch, nk))
        blind, group = nq[0] - 100, hq // hk
        assert torch.equal(again[:blind], got[:blind]) and torch.equal(again[nq[0]:], got[nq[0]:]) and torch.equal(again[:, 2 * group:], got[:, 2 * group:])
        assert again[blind:nq[0], :group].isnan().all() and (again[blind:nq[0], group:2 * group, 2] == math.inf).all()
        assert torch.equal(again[:nq[0], group:2 * group, 3:], got[:nq[0], group:2 * group, 3:])
    del pad


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_prompt_attention_of_far_apart_scores(torch, fi, dtype):
    """Scores from -300 to 300 in rising, falling and mixed order: the running maximum moves late, early and often."""
    g, kind, n, d = torch.Generator().manual_seed(3), _kind(torch, dtype), 260, 64
    q, v = torch.zeros((n, 3, d)), torch.randn((n, 3, d), generator=g)
    k = torch.zeros((n, 3, d))
    q[:, :, 0] = 16.0
    ramp = torch.linspace(-18, 18, n)
    k[:, 0, 0], k[:, 1, 0], k[:, 2, 0] = ramp, ramp.flip(0), ramp[torch.randperm(n, generator=g)]
    q, k, v = q.to(kind).cuda(), k.to(kind).cuda(), v.to(kind).cuda()
    for causal in (True, False):
        got = fi.prompt_attention(q, k, v, _cu(torch, [n]), causal=causal, scale=1.0)
        want, bound = _prompt_ref(torch, q, k, v, [n], [n], causal, 1.0, dtype)
        _inside(got.double().cpu(), want, bound + 600 * U * want.abs().amax())   # (the argument of exp: up to 600 before it is rounded)


@pytest.mark.parametrize("dtype,d", [("bf16", 64), ("bf16", 128), ("bf16", 72), ("f32", 64), ("f32", 128), ("bf16", 256), ("bf16", 50)])
def test_what_a_query_does_not_see_has_no_influence(torch, fi, dtype, d):
    """NaN and infinities in keys and values behind the diagonal: rows before them keep their bits, rows that see them carry them."""
    g, kind, n = torch.Generator().manual_seed(4), _kind(torch, dtype), 150
    q, k, v = (torch.randn((n, 2, d), generator=g).to(kind).cuda() for _ in range(3))
    clean = fi.prompt_attention(q, k, v, _cu(torch, [n]))
    for at, value in ((101, math.nan), (75, math.inf), (149, -math.inf), (64, math.nan), (33, math.inf)):
        bad = v.clone()
        bad[at, 0, 3] = value
        got = fi.prompt_attention(q, k, bad, _cu(torch, [n]))
        assert torch.equal(got[:at], clean[:at]) and torch.equal(got[:, 1], clean[:, 1])
        if math.isnan(value):
            assert got[at:, 0, 3].isnan().all()
        else:
            assert (got[at:, 0, 3] == value).all()
        others = [i for i in range(d) if i != 3]
        assert torch.equal(got[:, 0, others], clean[:, 0, others])
        bad = k.clone()
        bad[at, 0, 3] = math.nan
        got = fi.prompt_attention(q, bad, v, _cu(torch, [n]))
        assert torch.equal(got[:at], clean[:at]) and torch.equal(got[:, 1], clean[:, 1]) and got[at:, 0].isnan().all()


def test_prompt_attention_with_one_key_head_for_all_by_broadcasting(torch, fi):
    g = torch.Generator().manual_seed(6)
    q = torch.randn((90, 4, 64), generator=g).bfloat16().cuda()
    k, v = (torch.randn((90, 1, 64), generator=g).bfloat16().cuda() for _ in range(2))
    want = fi.prompt_attention(q, k, v, _cu(torch, [60, 30]))
    got = fi.prompt_attention(q, k.expand(-1, 4, -1), v.expand(-1, 4, -1), _cu(torch, [60, 30]))
    assert torch.equal(got, want)


# ---- trees over a cache --------------------------------------------------------------------------------
TREES = [
    # committed, nodes per sequence, page, q heads, kv heads, head dim, layout, mask
    ([0], [1], 16, 1, 1, 64, "plain", "tree"),
    ([1003], [1], 16, 32, 8, 128, "plain", "tree"),
    ([1, 0, 64, 333, 31], [1, 1, 1, 1, 1], 16, 8, 1, 128, "plain", None),
    ([100, 7, 0], [37, 1, 12], 48, 12, 4, 64, "plain", "tree"),
    ([260, 0, 31], [70, 130, 5], 16, 4, 2, 128, "plain", "tree"),
    ([77, 5], [9, 33], 5, 5, 5, 72, "plain", "tree"),
    ([50, 64], [3, 2], 1, 4, 2, 96, "odd", "tree"),
    ([200], [20], 64, 16, 2, 256, "plain", "tree"),
    ([513, 2], [6, 0], 256, 8, 2, 80, "wide", "tree"),
    ([90, 40], [8, 20], 16, 4, 4, 128, "plain", "empty"),     # some nodes see no node, not even themselves
    ([0, 0], [6, 40], 16, 4, 1, 64, "plain", "empty"),        # ... and nothing is committed: rows that see nothing
    ([5000, 17, 2100], [2, 1, 3], 16, 16, 2, 128, "plain", "tree"),
    ([3000], [100], 32, 8, 8, 64, "plain", None),
    ([40], [9], 8, 6, 3, 21, "odd", "tree"),
    ([7 * i % 50 for i in range(530)], [i % 3 for i in range(530)], 16, 4, 2, 64, "plain", "tree"),     # more sequences than a workgroup counts
    ([1500 if i == 40 else i % 9 for i in range(90)], [1 + i % 2 for i in range(90)], 16, 8, 1, 128, "plain", "tree"),   # one long among many short ones
    ([2500, 3, 0, 700], [40, 33, 1, 2], 16, 8, 1, 128, "plain", "tree"),
]


def _paged(torch, g, need, page, heads, d, kind, layout, spare=3):
    """A cache whose pages hold NaN wherever nothing was written, and the table that hands them out in random order."""
    pages = sum(need) + spare
    pad = {"plain": 0, "wide": 8, "odd": 3}[layout]
    shape = (pages, page, heads + (1 if pad else 0), d + pad)
    caches = [torch.full(shape, math.nan, dtype=kind).cuda()[:, :, :heads, pad - 2 if layout == "odd" else 0:][..., :d] for _ in range(2)]
    order = torch.randperm(pages, generator=g).to(torch.int32)
    columns = max(need + [1]) + 1
    table = torch.full((len(need), columns), pages - 1, dtype=torch.int32)
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n]
        at += n
    return caches, table


def _tree_mask(torch, g, counts, kind):
    words = max(1, (max(counts + [1]) + 63) // 64)
    rows = []
    for n in counts:
        seen = []
        for i in range(n):
            parent = int(torch.randint(-1, i, (1,), generator=g)) if i else -1
            bits = (seen[parent] if parent >= 0 else 0) | 1 << i
            seen.append(bits)
        if kind == "empty":
            seen = [0 if i % 3 != 1 else m for i, m in enumerate(seen)]
        rows += [[(m >> 64 * w) & (2 ** 64 - 1) for w in range(words)] for m in seen]
    return torch.tensor([[w - 2 ** 64 if w >= 2 ** 63 else w for w in row] for row in rows], dtype=torch.int64).reshape(-1, words)


def _tree_case(torch, g, cached, counts, page, hq, hk, d, kind, layout, mask):
    need = [(c + n + page - 1) // page for c, n in zip(cached, counts)]
    caches, table = _paged(torch, g, need, page, hk, d, kind, layout)
    dense = []
    for b, (c, n) in enumerate(zip(cached, counts)):
        kv = torch.randn((2, c + n, hk, d), generator=g).to(kind)
        j = torch.arange(c + n)
        for cache, rows in zip(caches, kv):
            cache[table[b, j // page].long().cuda(), (j % page).cuda()] = rows.cuda()
        dense.append(kv)
    q = _rows(torch, g, (sum(counts), hq, d), kind, layout)
    bits = None if mask is None else _tree_mask(torch, g, counts, mask)
    return q, caches, table.cuda(), dense, bits


def _tree_ref(torch, q, dense, cached, counts, bits, scale, dtype):
    want, bound = torch.zeros(q.shape).double(), torch.zeros(q.shape).double()
    q, at = q.cpu(), 0
    for kv, c, n in zip(dense, cached, counts):
        seen = torch.ones((n, c + n), dtype=torch.bool)
        if bits is None:
            seen = seen.tril(c)
        else:
            for j in range(n):
                seen[:, c + j] = (bits[at:at + n, j // 64] >> (j % 64)) & 1 == 1
        group = q.shape[1] // kv.shape[2]
        for h in range(q.shape[1]):
            want[at:at + n, h], bound[at:at + n, h] = _attend_ref(torch, q[at:at + n, h], kv[0, :, h // group], kv[1, :, h // group], seen, scale, dtype)
        at += n
    return want, bound


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("cached,counts,page,hq,hk,d,layout,mask", TREES)
def test_tree_attention(torch, fi, dtype, cached, counts, page, hq, hk, d, layout, mask):
    g, kind = torch.Generator().manual_seed(sum(cached) + 10 * sum(counts)), _kind(torch, dtype)
    q, (k, v), table, dense, bits = _tree_case(torch, g, cached, counts, page, hq, hk, d, kind, layout, mask)
    scale = 0.9 * d ** -0.5
    want, bound = _tree_ref(torch, q, dense, cached, counts, bits, scale, dtype)
    lengths, cu, m = torch.tensor(cached, dtype=torch.int32).cuda(), _cu(torch, counts), None if bits is None else bits.cuda()
    got = None
    # the work is shared out by what is said about the lengths: nothing, the truth, far too little
    for more in (dict(), dict(max_nodes=max(counts), max_length=max(c + n for c, n in zip(cached, counts))), dict(max_length=1)):
        out = torch.full(q.shape, math.nan, dtype=kind).cuda()
        y = fi.tree_attention(q, k, v, table, lengths, cu, m, scale=scale, out=out, **more)
        _inside(y.double().cpu(), want, bound)
        again = fi.tree_attention(q, k, v, table, lengths, cu, m, scale=scale, **more)
        assert torch.equal(again, y)
        got = y
    assert got is not None


LINES = [
    # few long histories among short ones: workgroups take stretches that begin and end inside a sequence
    ([3000 if i in (3, 17) else 40 * i % 700 for i in range(24)], [i % 4 for i in range(24)], 16, 16, 4, 128),
    ([2900 if i == 5 else 60 * i for i in range(12)], [33 if i == 5 else 3 * i % 31 for i in range(12)], 64, 16, 4, 128),
    ([0 if i else 2700 for i in range(14)], [12 - i % 13 for i in range(14)], 48, 32, 4, 72),
    ([1500 if i == 199 else i % 11 for i in range(200)], [(i + 1) % 2 for i in range(200)], 16, 1, 1, 64),
    ([9000, 5], [1, 2], 256, 8, 4, 128),
    ([700 + 90 * i for i in range(9)], [40] * 9, 32, 8, 8, 64),
    ([2000, 0, 2000, 1, 2000], [9, 0, 20, 0, 1], 16, 32, 16, 256),
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("cached,counts,page,hq,hk,d", LINES)
def test_trees_of_ragged_histories(torch, fi, dtype, cached, counts, page, hq, hk, d):
    g, kind = torch.Generator().manual_seed(sum(cached)), _kind(torch, dtype)
    q, (k, v), table, dense, bits = _tree_case(torch, g, cached, counts, page, hq, hk, d, kind, "plain", "tree")
    want, bound = _tree_ref(torch, q, dense, cached, counts, bits, d ** -0.5, dtype)
    lengths, cu, longest = torch.tensor(cached, dtype=torch.int32).cuda(), _cu(torch, counts), max(c + n for c, n in zip(cached, counts))
    for said in (longest, longest // 3, None):   # what is said about the lengths only guides how the work is shared out
        out = torch.full(q.shape, math.nan, dtype=kind).cuda()
        fi.tree_attention(q, k, v, table, lengths, cu, bits.cuda(), out=out, max_nodes=max(counts), max_length=said)
        _inside(out.double().cpu(), want, bound)
        again = fi.tree_attention(q, k, v, table, lengths, cu, bits.cuda(), max_nodes=max(counts), max_length=said)
        assert torch.equal(again, out)


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 72), ("f32", 64)])
@pytest.mark.parametrize("counts", [[5, 9], [40, 64]])
def test_a_branch_does_not_see_another(torch, fi, dtype, d, counts):
    """NaN and infinities in the keys and values of one node reach the nodes below it and no other."""
    g, kind, cached = torch.Generator().manual_seed(8), _kind(torch, dtype), [70, 33]
    q, (k, v), table, dense, bits = _tree_case(torch, g, cached, counts, 16, 8, 2, d, kind, "plain", "tree")
    lengths, cu = torch.tensor(cached, dtype=torch.int32).cuda(), _cu(torch, counts)
    clean = fi.tree_attention(q, k, v, table, lengths, cu, bits.cuda())
    at = counts[0] + 2   # the second sequence's node 2
    sees = torch.zeros(sum(counts), dtype=torch.bool)
    sees[counts[0]:] = (bits[counts[0]:, 0] >> 2) & 1 == 1
    assert sees[at] and not sees.all()
    place = cached[1] + 2
    where = (int(table[1, place // 16]), place % 16)
    for value in (math.nan, math.inf, -math.inf):
        bad = v.clone()
        bad[where[0], where[1], 1, 5] = value
        got = fi.tree_attention(q, k, bad, table, lengths, cu, bits.cuda())
        hit = got[sees.cuda()][:, 4:, 5]
        assert torch.equal(got[~sees.cuda()], clean[~sees.cuda()]) and torch.equal(got[:, :4], clean[:, :4])
        assert hit.isnan().all() if math.isnan(value) else (hit == value).all()
    bad = k.clone()
    bad[where[0], where[1], 1, 5] = math.nan
    got = fi.tree_attention(q, bad, v, table, lengths, cu, bits.cuda())
    assert torch.equal(got[~sees.cuda()], clean[~sees.cuda()]) and torch.equal(got[:, :4], clean[:, :4]) and got[sees.cuda()][:, 4:].isnan().all()


def test_cache_offsets_beyond_32_bits(torch, fi):
    """Pages whose offsets pass 2^31 elements and 2^32 bytes, written through slots and read through the table."""
    page, hk, d = 64, 8, 128
    pages = (1 << 31) // (page * hk * d) + 5000
    k, v = (torch.zeros((pages, page, hk, d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    assert k.numel() > 1 << 31
    g = torch.Generator().manual_seed(9)
    n, cached = 3, 150
    order = pages - 1 - torch.tensor([4, 0, 2], dtype=torch.int32)
    total = n + cached
    x = torch.randn((total, 8 + 2 * hk, d), generator=g).bfloat16().cuda()
    place = torch.arange(total)
    slots = (order[place // page].long() * page + place % page).cuda()
    q, _, _ = fi.qk_norm_rope(x[:, :8], x[:, 8:8 + hk], x[:, 8 + hk:], place.int().cuda(), torch.rand(64, generator=g).cuda(), slots=slots, k_out=k, v_out=v)
    small_k, small_v = (c[order.long().cuda()] for c in (k, v))
    lengths, cu = torch.tensor([cached], dtype=torch.int32).cuda(), _cu(torch, [n])
    got = fi.tree_attention(q[-n:], k, v, order[None].cuda(), lengths, cu)
    want = fi.tree_attention(q[-n:], small_k, small_v, torch.arange(3, dtype=torch.int32)[None].cuda(), lengths, cu)
    assert torch.equal(got, want) and got.abs().sum() > 0
    alone = fi.prompt_attention(q, small_k.view(-1, hk, d)[:total], small_v.view(-1, hk, d)[:total], _cu(torch, [total]))
    assert (alone[-n:].float() - got.float()).abs().max() <= 2.0 ** -6


def test_damaged_tables_stay_inside_the_cache(torch, fi):
    """Page numbers, lengths and offsets out of range are clamped to the tensors: the call ends, other sequences keep their results."""
    g = torch.Generator().manual_seed(10)
    cached, counts = [100, 60], [4, 4]
    q, (k, v), table, dense, bits = _tree_case(torch, g, cached, counts, 16, 4, 2, 64, torch.bfloat16, "plain", "tree")
    lengths, cu = torch.tensor(cached, dtype=torch.int32).cuda(), _cu(torch, counts)
    want = fi.tree_attention(q, k, v, table, lengths, cu, bits.cuda())
    bad = table.clone()
    bad[1, 1], bad[1, 2] = -7, 1 << 30
    long = lengths.clone()
    long[1] = 1 << 30
    for t, c in ((bad, lengths), (table, long), (bad, long)):
        assert torch.equal(fi.tree_attention(q, k, v, t, c, cu, bits.cuda())[:4], want[:4])
    torch.cuda.synchronize()


# ---- 4-bit products -------------------------------------------------------------------------------------
Q4 = [
    # rows, inputs, outputs, group, zeros
    (1, 32, 1, 32, False), (1, 4096, 1000, 128, False), (2, 64, 17, 64, True), (3, 256, 33, 32, True), (5, 4096, 100, 32, True), (8, 1280, 257, 256, True),
    (16, 512, 64, 128, False), (17, 192, 130, 64, True), (24, 25088, 40, 64, True), (33, 384, 48, 384, True), (64, 2048, 200, 64, False), (65, 128, 31, 128, True),
    (130, 320, 16, 32, False), (1, 16384, 5, 16384, True),
]


def _q4_case(torch, g, rows, inputs, outputs, group, zeros, kind, layout):
    pad = {"plain": 0, "wide": 16, "odd": 3}[layout]
    x = torch.randn((rows, inputs + pad), generator=g).to(kind).cuda()[:, :inputs]
    w = torch.randint(0, 256, (outputs, inputs // 2 + pad), generator=g, dtype=torch.uint8).cuda()[:, :inputs // 2]
    s = (torch.rand((outputs, inputs // group), generator=g) - 0.2).cuda()
    z = torch.randint(0, 16, (outputs, inputs // group), generator=g, dtype=torch.uint8).cuda() if zeros else None
    return x, w, s, z


def _q4_ref(torch, x, w, s, z, group, dtype):
    x, w, s = x.double().cpu(), w.cpu(), s.double().cpu()
    q = torch.stack([w & 15, w >> 4], -1).reshape(w.shape[0], -1).double().view(w.shape[0], -1, group)
    zero = 8.0 if z is None else z.double().cpu()[..., None]
    want = x @ ((q - zero) * s[..., None]).flatten(1).t()
    size = x.abs() @ (31 * s.abs()[..., None].expand_as(q)).flatten(1).t()
    half = H if dtype == "bf16" else 0.0
    return want, size * (x.shape[1] + 8) * U * (1 + half) + want.abs() * half * 1.01 + 1e-30


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("layout", ["plain", "odd", "wide"])
@pytest.mark.parametrize("rows,inputs,outputs,group,zeros", Q4)
def test_q4_products(torch, fi, dtype, layout, rows, inputs, outputs, group, zeros):
    g, kind = torch.Generator().manual_seed(rows * inputs + outputs), _kind(torch, dtype)
    x, w, s, z = _q4_case(torch, g, rows, inputs, outputs, group, zeros, kind, layout)
    out = torch.full((rows, outputs + 3), math.nan, dtype=kind).cuda()
    got = fi.q4_matmul(x, w, s, z, group=group, out=out[:, :outputs])
    want, bound = _q4_ref(torch, x, w, s, z, group, dtype)
    _inside(got.double().cpu(), want, bound)
    assert out[:, outputs:].isnan().all()
    # in the 2-norm the sums' errors do not line up: a bf16 result is off by its rounding, an fp32 one by some units
    off = float((got.double().cpu() - want).norm() / want.norm())
    assert off <= (H if dtype == "bf16" else 64 * U) or rows * outputs < 16
    assert torch.equal(fi.q4_matmul(x, w, s, z, group=group), got)


@pytest.mark.parametrize("rows,inputs,outputs,group,zeros", [
    (5, 12320, 33, 32, True), (17, 8288, 300, 32, False), (40, 12352, 270, 64, True), (9, 12352, 1, 64, False), (6, 12288, 17, 128, True), (20, 12288, 257, 384, True),
    (64, 8192, 5, 4096, False), (33, 8192, 513, 2048, True)])
def test_q4_products_shared_out_over_the_inputs(torch, fi, rows, inputs, outputs, group, zeros):
    """Long rows, whose groups end inside a step, a chunk of scales and a share of the inputs.  The bounds are those of the other products."""
    g = torch.Generator().manual_seed(inputs + outputs)
    x, w, s, z = _q4_case(torch, g, rows, inputs, outputs, group, zeros, torch.bfloat16, "wide")
    got = fi.q4_matmul(x, w, s, z, group=group)
    want, bound = _q4_ref(torch, x, w, s, z, group, "bf16")
    _inside(got.double().cpu(), want, bound)
    assert float((got.double().cpu() - want).norm() / want.norm()) <= H or rows * outputs < 16
    assert torch.equal(fi.q4_matmul(x, w, s, z, group=group), got)
    x[rows // 2, inputs - 1] = math.inf
    kept = [i for i in range(rows) if i != rows // 2]
    again = fi.q4_matmul(x, w, s, z, group=group)
    assert torch.equal(again[kept], got[kept]) and not again[rows // 2].isfinite().any()


@pytest.mark.parametrize("rows,inputs,outputs,group,zeros", [
    (5, 12320, 33, 32, True), (17, 8288, 300, 32, False), (40, 12352, 270, 64, True), (9, 12352, 1, 64, False), (16, 12288, 17, 128, True), (20, 12288, 257, 384, True),
    (7, 2048, 12300, 256, False), (33, 8192, 513, 2048, True)])
def test_q4_fp32_products_shared_out_over_the_inputs(torch, fi, rows, inputs, outputs, group, zeros):
    """The same for fp32 rows, blocks of 16."""
    g = torch.Generator().manual_seed(inputs + outputs)
    x, w, s, z = _q4_case(torch, g, rows, inputs, outputs, group, zeros, torch.float32, "wide")
    got = fi.q4_matmul(x, w, s, z, group=group)
    want, bound = _q4_ref(torch, x, w, s, z, group, "f32")
    _inside(got.double().cpu(), want, bound)
    assert float((got.double().cpu() - want).norm() / want.norm()) <= 64 * U or rows * outputs < 16
    assert torch.equal(fi.q4_matmul(x, w, s, z, group=group), got)
    x[rows // 2, inputs - 1] = math.inf
    kept = [i for i in range(rows) if i != rows // 2]
    again = fi.q4_matmul(x, w, s, z, group=group)
    assert torch.equal(again[kept], got[kept]) and not again[rows // 2].isfinite().any()


def test_q4_rows_do_not_touch_each_other(torch, fi):
    """A row of NaN or infinities stays a row; weights of zero times infinity are NaN, as in the formula."""
    g = torch.Generator().manual_seed(12)
    x, w, s, z = _q4_case(torch, g, 9, 512, 50, 64, True, torch.bfloat16, "plain")
    clean = fi.q4_matmul(x, w, s, z)
    x[4, 100] = math.nan
    got = fi.q4_matmul(x, w, s, z)
    keep = [i for i in range(9) if i != 4]
    assert torch.equal(got[keep], clean[keep]) and got[4].isnan().all()


def test_q4_no_inputs_and_no_rows(torch, fi):
    x, w, s = torch.ones((3, 0)).cuda(), torch.zeros((5, 0), dtype=torch.uint8).cuda(), torch.zeros((5, 0)).cuda()
    assert torch.equal(fi.q4_matmul(x, w, s, group=32), torch.zeros((3, 5)).cuda())
    x, w, s = torch.ones((0, 64)).cuda(), torch.zeros((5, 32), dtype=torch.uint8).cuda(), torch.zeros((5, 1)).cuda()
    assert fi.q4_matmul(x, w, s).shape == (0, 5)


# ---- streams and graphs -------------------------------------------------------------------------------------
def _all_four(torch, fi, state, stream=None):
    """A decoder step's operators one after the other, each reading what the one before wrote."""
    y = fi.q4_matmul(state["x"], state["w"], state["s"], out=state["qkv"], stream=stream)
    rows = y.view(-1, 12, 128)
    q, _, _ = fi.qk_norm_rope(rows[:, :8], rows[:, 8:10], rows[:, 10:], state["positions"], state["inv_freq"], slots=state["slots"], q_out=state["q"],
                              k_out=state["k_cache"], v_out=state["v_cache"], stream=stream)
    a = fi.tree_attention(q, state["k_cache"], state["v_cache"], state["table"], state["cached"], state["cu"], out=state["tree"], max_nodes=3,
                          max_length=2003, workspace=state["workspace"], stream=stream)
    b = fi.prompt_attention(q, rows[:, 8:10], rows[:, 10:], state["cu"], out=state["prompt"], stream=stream)
    return y, a, b


def _step(torch):
    g = torch.Generator().manual_seed(11)
    page, cached, n = 16, [2000, 7], [3, 3]
    pages = sum((c + m + page - 1) // page for c, m in zip(cached, n))
    table = torch.zeros((2, 126), dtype=torch.int32)
    table[0], table[1, 0] = torch.arange(126), 126
    slots = torch.tensor([int(table[b, (cached[b] + i) // page]) * page + (cached[b] + i) % page for b in range(2) for i in range(3)])
    dev = dict(x=torch.randn((6, 1024), generator=g).bfloat16(), w=torch.randint(0, 256, (12 * 128, 512), generator=g, dtype=torch.uint8),
               s=torch.rand((12 * 128, 8), generator=g) * 0.02, positions=torch.tensor([2000, 2001, 2002, 7, 8, 9], dtype=torch.int32), inv_freq=torch.rand(64, generator=g),
               slots=slots, k_cache=torch.randn((pages, page, 2, 128), generator=g).bfloat16(), v_cache=torch.randn((pages, page, 2, 128), generator=g).bfloat16(),
               table=table, cached=torch.tensor(cached, dtype=torch.int32), cu=torch.tensor([0, 3, 6], dtype=torch.int32),
               qkv=torch.zeros((6, 12 * 128)).bfloat16(), q=torch.zeros((6, 8, 128)).bfloat16(), tree=torch.zeros((6, 8, 128)).bfloat16(),
               prompt=torch.zeros((6, 8, 128)).bfloat16(), workspace=torch.zeros(8 << 20, dtype=torch.uint8))
    return {k: v.cuda() for k, v in dev.items()}


def test_operators_on_a_stream_of_their_own(torch, fi):
    state = _step(torch)
    want = [t.clone() for t in _all_four(torch, fi, state)]
    torch.cuda.synchronize()
    for name in ("qkv", "q", "tree", "prompt"):
        state[name].zero_()
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    got = _all_four(torch, fi, state, stream.cuda_stream)
    stream.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_operators_in_a_graph(torch, fi):
    """Recorded once, replayed with new inputs, eager work between the replays: every replay gives the eager call's bits."""
    state = _step(torch)
    _all_four(torch, fi, state)
    torch.cuda.synchronize()
    graph, stream = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=stream):
        outs = _all_four(torch, fi, state)
    for turn in range(4):
        state["x"].copy_(torch.randn((6, 1024), generator=torch.Generator().manual_seed(turn)).bfloat16())
        want = [t.clone() for t in _all_four(torch, fi, state)]
        for t in outs:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, want)), turn


# ---- tensors that do not fit --------------------------------------------------------------------------------
def test_tensors_that_do_not_fit_are_refused(torch, fi):
    """Every check on the way from tensors to the entry points: types, shapes, strides, devices; nothing is launched."""
    d = dict(dtype=torch.bfloat16, device="cuda")
    i32 = dict(dtype=torch.int32, device="cuda")
    q, k, cu = torch.zeros((4, 4, 64), **d), torch.zeros((4, 2, 64), **d), torch.tensor([0, 4], **i32)
    positions, freq = torch.zeros(4, **i32), torch.zeros(32, device="cuda")
    cache, slots = torch.zeros((2, 16, 2, 64), **d), torch.zeros(4, dtype=torch.int64, device="cuda")
    table, cached = torch.zeros((1, 2), **i32), torch.zeros(1, **i32)
    x, w, s = torch.zeros((3, 128), **d), torch.zeros((8, 64), dtype=torch.uint8, device="cuda"), torch.zeros((8, 2), device="cuda")
    wrong = [
        (TypeError, lambda: fi.qk_norm_rope(q.half(), k, k, positions, freq)),
        (TypeError, lambda: fi.qk_norm_rope(q, None, k, positions, freq)),
        (ValueError, lambda: fi.qk_norm_rope(q, k.float(), k, positions, freq)),
        (ValueError, lambda: fi.qk_norm_rope(q, k[:3], k, positions, freq)),
        (ValueError, lambda: fi.qk_norm_rope(q, k, k.cpu(), positions, freq)),
        (ValueError, lambda: fi.qk_norm_rope(q, k, k, positions.long(), freq)),
        (ValueError, lambda: fi.qk_norm_rope(q, k, k, positions, freq, sections=[16, 16])),
        (ValueError, lambda: fi.qk_norm_rope(q, k, k, positions, freq, q_weight=torch.ones(63, device="cuda"))),
        (ValueError, lambda: fi.qk_norm_rope(q, k, k, positions, freq, slots=slots)),
        (ValueError, lambda: fi.qk_norm_rope(q, k, k, positions, freq, slots=slots, k_out=cache)),
        (ValueError, lambda: fi.qk_norm_rope(q, k, k, positions, freq, q_out=torch.zeros((4, 64, 4), **d).transpose(1, 2))),
        (TypeError, lambda: fi.qk_norm_rope(q, k, k, positions, freq, eps="small")),
        (fi.FiError, lambda: fi.qk_norm_rope(q, k, k, positions, torch.zeros(40, device="cuda"))),
        (ValueError, lambda: fi.prompt_attention(q, k, k[:, :1], cu)),
        (ValueError, lambda: fi.prompt_attention(q, k, k, cu.long())),
        (ValueError, lambda: fi.prompt_attention(q, k, k, cu, torch.tensor([0, 2, 4], **i32))),
        (ValueError, lambda: fi.prompt_attention(q, k, k, cu, out=torch.zeros((4, 4, 32), **d))),
        (fi.FiError, lambda: fi.prompt_attention(q[:, :3], k, k, cu)),
        (fi.FiError, lambda: fi.prompt_attention(q, k, k, cu, scale=-1.0)),
        (ValueError, lambda: fi.tree_attention(q, cache, cache[:1], table, cached, cu)),
        (ValueError, lambda: fi.tree_attention(q, cache, cache, table, cached, cu, torch.zeros((3, 1), dtype=torch.int64, device="cuda"))),
        (ValueError, lambda: fi.tree_attention(q, cache, cache, table, torch.zeros(2, **i32), cu)),
        (ValueError, lambda: fi.tree_attention(q, cache, cache, table, cached, cu, max_length=1 << 40)),
        (ValueError, lambda: fi.tree_attention(q, cache, cache, table, cached, cu, workspace=torch.zeros(64, device="cuda"))),
        (ValueError, lambda: fi.q4_matmul(x, w[:, :63], s)),
        (ValueError, lambda: fi.q4_matmul(x, w, s, group=32)),
        (ValueError, lambda: fi.q4_matmul(x, w, s, torch.zeros((8, 1), dtype=torch.uint8, device="cuda"))),
        (ValueError, lambda: fi.q4_matmul(x, w.t().contiguous().t(), s)),
        (TypeError, lambda: fi.q4_matmul(x, w, s, out="here")),
    ]
    for number, (kind, call) in enumerate(wrong):
        with pytest.raises(kind):
            call()
            pytest.fail(f"number {number} was taken")
    assert torch.equal(fi.q4_matmul(x, w, s), torch.zeros((3, 8), **d))


def test_a_workspace_of_the_callers(torch, fi):
    """Products that are shared out take the caller's workspace, and refuse one that is too small."""
    g = torch.Generator().manual_seed(4)
    x, w, s, z = _q4_case(torch, g, 9, 12288, 70, 64, True, torch.bfloat16, "plain")
    args = fi.fi_q4_matmul_args(dtype=fi.FI_BF16, rows=9, inputs=12288, outputs=70, group=64)
    need = fi.fi_q4_matmul_workspace(args)
    assert need > 0
    want = fi.q4_matmul(x, w, s, z)
    assert torch.equal(fi.q4_matmul(x, w, s, z, workspace=torch.empty(need, dtype=torch.uint8, device="cuda")), want)
    with pytest.raises(fi.FiError):
        fi.q4_matmul(x, w, s, z, workspace=torch.empty(need - 16, dtype=torch.uint8, device="cuda"))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = fi.q4_matmul(x, w, s, z, stream=side.cuda_stream)
    side.synchronize()
    assert torch.equal(got, want)
