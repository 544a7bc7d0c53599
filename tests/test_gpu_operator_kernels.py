"""The decoder operators at sizes that every kernel and every way of dealing out the work takes, against their definitions in 64 bits; bounds as in test_gpu_operators.py."""
import math

import pytest

from tests.test_gpu_operators import H, U, _cu, _inside, _kind, _packed, _prompt_ref, _q4_case, _q4_ref, _rope_ref, _tree_case, _tree_ref, fi, torch  # noqa: F401

pytestmark = pytest.mark.gpu


# ---- prompts in blocks of 128 queries ---------------------------------------------------------------------
MIDDLE = [
    # query lengths, extra keys, q heads, kv heads, head dim, causal: more blocks of 32 queries than are taken alone, fewer blocks of 256 than fill the chip
    ([900], [0], 32, 4, 64, True), ([3, 700, 1, 260], [100, 0, 64, 31], 28, 4, 64, True), ([31] * 20 + [1, 0, 129], [i % 3 * 40 for i in range(23)], 32, 8, 64, True),
    ([640], [-500], 48, 4, 40, True), ([333, 400], [-333, 7], 40, 8, 64, False),
    ([500], [0], 20, 4, 72, True), ([130, 129, 127], [0, 300, -100], 24, 24, 72, False), ([30] * 17, [2] * 17, 32, 4, 80, True), ([600, 5], [0, 0], 20, 5, 96, True),
    ([28] * 19, [0] * 19, 32, 4, 96, False), ([511], [0], 24, 3, 128, True), ([257, 1, 300], [64, 0, 128], 32, 8, 128, True), ([33] * 18, [1] * 18, 16, 2, 128, True),
    ([200, 200], [-150, 20], 32, 4, 128, False), ([640], [0], 40, 4, 256, True), ([100, 64, 3], [0, 30, 900], 48, 6, 256, False), ([20] * 9, [0] * 9, 96, 12, 200, True),
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("nq,extra,hq,hk,d,causal", MIDDLE)
def test_prompts_of_middle_sizes(torch, fi, dtype, nq, extra, hq, hk, d, causal):  # noqa: F811
    g, kind = torch.Generator().manual_seed(sum(nq) * 7 + d), _kind(torch, dtype)
    if dtype == "f32" and d <= 128:   # twice the heads: fp32 calls go to these blocks later
        hq, hk = 2 * hq, 2 * hk
    nk = [n + e for n, e in zip(nq, extra)]
    q, k, v = _packed(torch, g, nq, hq, d, kind, "wide"), _packed(torch, g, nk, hk, d, kind, "plain"), _packed(torch, g, nk, hk, d, kind, "wide")
    out = torch.full((sum(nq), hq, d), math.nan, dtype=kind).cuda()
    got = fi.prompt_attention(q, k, v, _cu(torch, nq), _cu(torch, nk), causal=causal, scale=1.2 * d ** -0.5, out=out)
    want, bound = _prompt_ref(torch, q, k, v, nq, nk, causal, 1.2 * d ** -0.5, dtype)
    _inside(got.double().cpu(), want, bound)
    assert torch.equal(fi.prompt_attention(q, k, v, _cu(torch, nq), _cu(torch, nk), causal=causal, scale=1.2 * d ** -0.5), got)


@pytest.mark.parametrize("dtype,d,heads,n", [
    ("bf16", 64, 40, 700), ("bf16", 72, 20, 500), ("bf16", 96, 20, 500), ("bf16", 128, 20, 500), ("bf16", 128, 4, 2200), ("bf16", 256, 40, 640), ("f32", 64, 64, 640),
    ("f32", 72, 64, 640), ("f32", 128, 64, 640), ("f32", 256, 40, 640)])
def test_middle_prompts_do_not_see_behind_the_diagonal(torch, fi, dtype, d, heads, n):  # noqa: F811
    """NaN and infinities in one key or value: rows before it and other heads keep their bits, rows that see it carry it."""
    g, kind = torch.Generator().manual_seed(31), _kind(torch, dtype)
    q, k, v = (torch.randn((n, h, d), generator=g).to(kind).cuda() for h in (heads, 4, 4))
    clean, group = fi.prompt_attention(q, k, v, _cu(torch, [n])), heads // 4
    others = [i for i in range(d) if i != 3]
    for at, value in ((n - 1, math.nan), (n - 77, math.inf), (130, -math.inf), (127, math.nan), (64, math.inf), (n - 128, -math.inf)):
        bad = v.clone()
        bad[at, 1, 3] = value
        got = fi.prompt_attention(q, k, bad, _cu(torch, [n]))
        hit = got[:, group:2 * group]
        assert torch.equal(got[:at], clean[:at]) and torch.equal(got[:, :group], clean[:, :group]) and torch.equal(got[:, 2 * group:], clean[:, 2 * group:])
        assert hit[at:, :, 3].isnan().all() if math.isnan(value) else (hit[at:, :, 3] == value).all()
        assert torch.equal(hit[..., others], clean[:, group:2 * group][..., others])
        bad = k.clone()
        bad[at, 1, 3] = math.nan
        got = fi.prompt_attention(q, bad, v, _cu(torch, [n]))
        assert torch.equal(got[:at], clean[:at]) and torch.equal(got[:, :group], clean[:, :group]) and got[at:, group:2 * group].isnan().all()
    bad = v.clone()
    bad[50, 0, 5], bad[n - 60, 0, 5] = math.inf, -math.inf   # both signs: no number for rows that see both
    got = fi.prompt_attention(q, k, bad, _cu(torch, [n]))[:, :group, 5]
    assert torch.equal(got[:50], clean[:50, :group, 5]) and (got[50:n - 60] == math.inf).all() and got[n - 60:].isnan().all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,heads,d", [(900, 66, 64), (650, 66, 128), (640, 66, 256)])
def test_middle_prompts_of_far_apart_scores(torch, fi, dtype, n, heads, d):  # noqa: F811
    """Scores from -300 to 300 in rising, falling and mixed order, as in the test of short prompts; both groups of waves meet them."""
    g, kind = torch.Generator().manual_seed(32), _kind(torch, dtype)
    q, k, v = torch.zeros((n, heads, d)), torch.zeros((n, 3, d)), torch.randn((n, 3, d), generator=g)
    q[:, :, 0] = 16.0
    ramp = torch.linspace(-18, 18, n)
    k[:, 0, 0], k[:, 1, 0], k[:, 2, 0] = ramp, ramp.flip(0), ramp[torch.randperm(n, generator=g)]
    q, k, v = q.to(kind).cuda(), k.to(kind).cuda(), v.to(kind).cuda()
    for causal in (True, False):
        got = fi.prompt_attention(q, k, v, _cu(torch, [n]), causal=causal, scale=1.0)
        group = heads // 3
        want, bound = _prompt_ref(torch, q[:, ::group], k, v, [n], [n], causal, 1.0, dtype)
        _inside(got[:, ::group].double().cpu(), want, bound + 600 * U * want.abs().amax())
        assert torch.equal(got[:, 1::group], got[:, ::group])


# ---- trees with many rows a sequence ------------------------------------------------------------------------
WIDE_TREES = [
    # committed, nodes, page, q heads, kv heads, head dim, mask: more than 128 rows of a key head, heads up to 128: eight waves share the tiles
    ([3000], [200], 16, 32, 8, 64, "tree"), ([900, 5, 2500, 0], [61, 64, 1, 40], 64, 32, 4, 64, "tree"), ([1500, 1200], [70, 44], 48, 16, 4, 72, "tree"),
    ([2000], [130], 16, 8, 4, 80, None), ([1100, 0, 700, 64, 2000], [50, 60, 0, 33, 1], 16, 28, 4, 96, "tree"), ([1024, 777], [100, 128], 32, 16, 2, 96, "empty"),
    ([1800, 3, 900], [64, 10, 90], 1, 12, 2, 128, "tree"), ([700] * 3, [37, 40, 2], 256, 40, 8, 32, "tree"),
    # fewer rows, histories of any length: four waves that share, or that have keys of their own, on stretches of the line
    ([2600 - 290 * i for i in range(9)] + [0, 3, 64], [12 - i for i in range(12)], 16, 32, 8, 64, "tree"), ([300 * i for i in range(10)], [20, 1] * 5, 64, 24, 8, 128, "tree"),
    ([2700, 0, 5, 1900, 40, 700, 1, 1300, 64, 2222], [1 + i % 3 for i in range(10)], 16, 32, 16, 72, "tree"),
    ([2700, 0, 5, 1900, 40, 700, 1, 1300, 64, 2222], [1] * 10, 48, 32, 16, 256, None),
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("cached,counts,page,hq,hk,d,mask", WIDE_TREES)
def test_trees_of_many_rows(torch, fi, dtype, cached, counts, page, hq, hk, d, mask):  # noqa: F811
    g, kind = torch.Generator().manual_seed(sum(cached) + d), _kind(torch, dtype)
    q, (k, v), table, dense, bits = _tree_case(torch, g, cached, counts, page, hq, hk, d, kind, "plain", mask)
    want, bound = _tree_ref(torch, q, dense, cached, counts, bits, d ** -0.5, dtype)
    lengths, cu, longest = torch.tensor(cached, dtype=torch.int32).cuda(), _cu(torch, counts), max(c + n for c, n in zip(cached, counts))
    m = None if bits is None else bits.cuda()
    for more in (dict(max_nodes=max(counts), max_length=longest), dict()):
        out = torch.full(q.shape, math.nan, dtype=kind).cuda()
        fi.tree_attention(q, k, v, table, lengths, cu, m, out=out, **more)
        _inside(out.double().cpu(), want, bound)
        assert torch.equal(fi.tree_attention(q, k, v, table, lengths, cu, m, **more), out)


# ---- norms and rotation -------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("tokens,d,rot,sections,interleaved", [(50, 68, 36, (18,), True), (3, 76, 76, (20, 10, 8), True), (700, 60, 12, (2, 4), False), (1, 20, 20, (10,), True)])
def test_norms_of_heads_of_four_values_at_a_time(torch, fi, dtype, tokens, d, rot, sections, interleaved):  # noqa: F811
    g, kind = torch.Generator().manual_seed(tokens + d), _kind(torch, dtype)
    x = torch.randn((tokens, 9, d), generator=g).to(kind).cuda()
    positions = torch.randint(0, 3000, (tokens, len(sections)), generator=g, dtype=torch.int32).cuda()
    freq, w = (500.0 ** -(torch.arange(rot // 2) / (rot // 2))).float().cuda(), (1 + 0.2 * torch.randn(d, generator=g)).cuda()
    y, yk, yv = fi.qk_norm_rope(x[:, :5], x[:, 5:7], x[:, 7:], positions, freq, q_weight=w, sections=sections, interleaved=interleaved, eps=1e-5)
    half = H if dtype == "bf16" else 0.0
    for got, rows, weight in ((y, x[:, :5], w), (yk, x[:, 5:7], None)):
        want, bound = _rope_ref(torch, rows, weight, positions, freq, sections, 1e-5, interleaved)
        _inside(got.double().cpu(), want, bound * (1 + half) + half * want.abs() + 1e-30)
    assert torch.equal(yv, x[:, 7:])


# ---- 4-bit products -----------------------------------------------------------------------------------------
PRODUCTS = [
    # rows, inputs, outputs, group, zeros
    (1, 4096, 1600, 128, False), (1, 2048, 1537, 32, True), (2, 4096, 1001, 64, True), (2, 1024, 16400, 128, False), (3, 4096, 1540, 64, True), (5, 4096, 1000, 32, True),
    (16, 2080, 400, 32, False), (7, 2048, 777, 256, True), (1, 2048, 500, 64, False), (4, 4128, 300, 32, True), (1, 25088, 33, 64, True),
    (5, 320, 16401, 64, True), (3, 512, 16390, 128, True), (20, 96, 16500, 32, False), (17, 2048, 3000, 64, True), (40, 640, 500, 128, False), (9, 2080, 600, 32, True),
    (2, 1792, 500, 64, True), (19, 2080, 500, 32, True),
    (520, 512, 4100, 64, True), (530, 512, 4099, 32, False), (300, 1024, 8200, 128, True), (24, 25088, 260, 64, True),
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,inputs,outputs,group,zeros", PRODUCTS)
def test_q4_products_of_every_kernel(torch, fi, dtype, rows, inputs, outputs, group, zeros):  # noqa: F811
    g, kind = torch.Generator().manual_seed(rows + inputs + outputs), _kind(torch, dtype)
    x, w, s, z = _q4_case(torch, g, rows, inputs, outputs, group, zeros, kind, "wide")
    out = torch.full((rows, outputs + 5), math.nan, dtype=kind).cuda()
    got = fi.q4_matmul(x, w, s, z, group=group, out=out[:, :outputs])
    want, bound = _q4_ref(torch, x, w, s, z, group, dtype)
    _inside(got.double().cpu(), want, bound)
    assert float((got.double().cpu() - want).norm() / want.norm()) <= (H if dtype == "bf16" else 64 * U)
    assert out[:, outputs:].isnan().all() and torch.equal(fi.q4_matmul(x, w, s, z, group=group), got)


# ---- graphs of calls whose launches depend on each other --------------------------------------------------------
@pytest.mark.parametrize("dtype,nodes", [("bf16", 3), ("bf16", 40), ("f32", 3)])
def test_shared_out_work_in_a_graph(torch, fi, dtype, nodes):  # noqa: F811
    """Products and trees whose parts a second launch joins, replayed with other lengths, offsets and inputs: every replay gives the eager call's bits."""
    g, kind = torch.Generator().manual_seed(33), _kind(torch, dtype)
    x, w, s, z = _q4_case(torch, g, 9, 12288, 70, 64, True, kind, "plain")
    cached, counts = [4000, 5, 900, 2000, 0, 1700], [nodes] * 6
    q, (k, v), table, _, bits = _tree_case(torch, g, [4000] * 6, counts, 16, 16, 16, 128, kind, "plain", "tree")
    k.nan_to_num_(0.5), v.nan_to_num_(0.5)   # (every place holds something)
    lengths, cu, bits = torch.tensor(cached, dtype=torch.int32).cuda(), _cu(torch, counts), bits.cuda()
    said = dict(max_nodes=nodes, max_length=4000 + nodes)
    sizes = dict(dtype=fi.FI_F32 if dtype == "f32" else fi.FI_BF16, n_seqs=6, q_heads=16, kv_heads=16, head_dim=128, page_size=16, n_pages=k.shape[0], table_columns=table.shape[1],
                 mask_words=1, scale=1.0, nodes=6 * nodes, **said)
    spaces = [torch.zeros(fi.fi_tree_attention_workspace(fi.fi_tree_attention_args(**sizes)), dtype=torch.uint8).cuda(),
              torch.zeros(fi.fi_q4_matmul_workspace(fi.fi_q4_matmul_args(dtype=sizes["dtype"], rows=9, inputs=12288, outputs=70, group=64)), dtype=torch.uint8).cuda()]
    assert all(len(space) for space in spaces)
    outs = [torch.zeros_like(q), torch.zeros((9, 70), dtype=kind).cuda()]

    def step(outs, spaces):
        fi.tree_attention(q, k, v, table, lengths, cu, bits, out=outs[0], workspace=spaces[0], **said)
        fi.q4_matmul(x, w, s, z, group=64, out=outs[1], workspace=spaces[1])

    step(outs, spaces)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(outs, spaces)
    turns = [(cached, counts), ([1, 4000, 0, 3, 3999, 2], counts), ([0] * 6, counts), ([4000] * 6, counts), ([10, 20, 4000, 30, 40, 50], [nodes, 0, nodes, 1, 0, nodes - 1])]
    for turn, (c, n) in enumerate(turns):
        lengths.copy_(torch.tensor(c, dtype=torch.int32))
        cu.copy_(_cu(torch, n))
        q.copy_(torch.randn(q.shape, generator=g))
        x.copy_(torch.randn(x.shape, generator=g))
        want = [torch.zeros_like(t) for t in outs]
        step(want, [None, None])
        for t in outs:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, want)), turn
        assert outs[0][:sum(n)].isfinite().all() and outs[0][:sum(n)].abs().sum() > 0


# ---- single tokens and small trees: nothing but the result is rounded to bf16 ------------------------------------
@pytest.mark.parametrize("cached,counts,page,hq,hk,d", [
    ([4000], [1], 16, 32, 8, 128), ([1003, 5, 64], [1, 1, 1], 64, 8, 8, 64), ([2000, 0, 700, 31], [4, 2, 1, 3], 16, 16, 2, 72), ([900], [7], 1, 8, 2, 256),
    ([100 + i for i in range(40)], [1] * 40, 16, 32, 32, 96), ([3000, 100, 900] * 8, [1, 2, 3] * 8, 48, 16, 16, 128)])
def test_few_nodes_keep_their_weights(torch, fi, cached, counts, page, hq, hk, d):  # noqa: F811
    """Weights that meet the values in two terms of bf16 are off by (2^-8)^2; the bound has no rounding of 2^-8 but that of the result."""
    g = torch.Generator().manual_seed(sum(cached) + d)
    q, (k, v), table, dense, bits = _tree_case(torch, g, cached, counts, page, hq, hk, d, torch.bfloat16, "plain", "tree")
    want, bound = _tree_ref(torch, q, dense, cached, counts, bits, d ** -0.5, "f32")
    size, _ = _tree_ref(torch, q, [torch.stack([kv[0], kv[1].abs()]) for kv in dense], cached, counts, bits, d ** -0.5, "f32")
    lengths, cu, longest = torch.tensor(cached, dtype=torch.int32).cuda(), _cu(torch, counts), max(c + n for c, n in zip(cached, counts))
    got = fi.tree_attention(q, k, v, table, lengths, cu, bits.cuda(), max_nodes=max(counts), max_length=longest)
    _inside(got.double().cpu(), want, bound + size * H * H + 1.01 * H * want.abs())
