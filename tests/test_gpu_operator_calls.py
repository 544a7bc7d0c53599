"""Calls of the decoder operators on tensors: the memory that a call makes for itself, and on which stream."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    import torch
    return torch


@pytest.fixture(scope="module")
def fi():
    import paper_2410_21120_amd as fi
    return fi


def _stream_of(torch, t):
    """The stream whose pool a tensor's memory comes from."""
    for s in torch.cuda.memory_snapshot():
        if s["address"] <= t.data_ptr() < s["address"] + s["total_size"]:
            return s["stream"]
    raise AssertionError("not torch's memory")


def _pool(torch, stream):
    return sum(s["total_size"] for s in torch.cuda.memory_snapshot() if s["stream"] == stream)


def _shared_product(torch):
    """Arguments of a product that needs a workspace."""
    g = torch.Generator().manual_seed(21)
    return (torch.randn((9, 12288), generator=g).bfloat16().cuda(), torch.randint(0, 256, (70, 6144), generator=g, dtype=torch.uint8).cuda(),
            torch.rand((70, 192), generator=g).cuda())


def test_what_a_call_makes_on_a_stream_is_that_streams_memory(torch, fi):
    """Outputs and workspaces made inside a call come from the pool of the call's stream: another pool's block may still be in use on its own stream."""
    g = torch.Generator().manual_seed(20)
    q, k = torch.randn((40, 4, 64), generator=g).bfloat16().cuda(), torch.randn((40, 2, 64), generator=g).bfloat16().cuda()
    cu, positions, freq = torch.tensor([0, 40], dtype=torch.int32).cuda(), torch.arange(40, dtype=torch.int32).cuda(), torch.rand(32, generator=g).cuda()
    cache, table, cached = k.view(10, 4, 2, 64).clone(), torch.arange(10, dtype=torch.int32)[None].cuda(), torch.tensor([39], dtype=torch.int32).cuda()
    x, w, s = _shared_product(torch)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    calls = [lambda **m: fi.qk_norm_rope(q, k, k, positions, freq, **m), lambda **m: (fi.prompt_attention(q, k, k, cu, **m),),
             lambda **m: (fi.tree_attention(q[:1], cache, cache, table, cached, cu.clamp(max=1), **m),), lambda **m: (fi.q4_matmul(x, w, s, group=64, **m),)]
    for call in calls:
        want = call()
        torch.cuda.synchronize()
        got = call(stream=side.cuda_stream)
        side.synchronize()
        for a, b in zip(got, want):
            assert _stream_of(torch, a) == side.cuda_stream and _stream_of(torch, b) != side.cuda_stream
            assert torch.equal(a, b)
    # the workspace
    del got, a
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    out = torch.empty((9, 70), dtype=torch.bfloat16, device="cuda")
    assert _pool(torch, side.cuda_stream) == 0
    fi.q4_matmul(x, w, s, group=64, out=out, stream=side.cuda_stream)
    assert _pool(torch, side.cuda_stream) > 0
    side.synchronize()
    assert torch.equal(out, want[0])


def test_a_block_that_another_stream_is_still_at_work_on(torch, fi):
    """A temporary of the workspace's size is freed with its kernels pending on the current stream; the call's stream owes that one no wait."""
    x, w, s = _shared_product(torch)
    need = fi.fi_q4_matmul_workspace(fi.fi_q4_matmul_args(dtype=fi.FI_BF16, rows=9, inputs=12288, outputs=70, group=64))
    want = fi.q4_matmul(x, w, s, group=64)
    side, a = torch.cuda.Stream(), torch.randn((4096, 4096), device="cuda")
    torch.cuda.synchronize()
    for _ in range(8):
        a @ a
    temporary = torch.empty(need, dtype=torch.uint8, device="cuda")
    for _ in range(200):
        temporary.fill_(255)   # NaN, to the sums
    del temporary
    got = fi.q4_matmul(x, w, s, group=64, stream=side.cuda_stream)
    side.synchronize()
    torch.cuda.synchronize()
    assert torch.equal(got, want)


def test_outputs_of_any_order(torch, fi):
    """Heads in front of tokens, in outputs and caches: the rows lie apart, so they are taken, and hold what others do."""
    g = torch.Generator().manual_seed(22)
    q, k = torch.randn((40, 4, 64), generator=g).bfloat16().cuda(), torch.randn((40, 2, 64), generator=g).bfloat16().cuda()
    cu, positions, freq = torch.tensor([0, 40], dtype=torch.int32).cuda(), torch.arange(40, dtype=torch.int32).cuda(), torch.rand(32, generator=g).cuda()
    turned = lambda heads: torch.zeros((heads, 40, 64), dtype=torch.bfloat16, device="cuda").transpose(0, 1)
    want = fi.qk_norm_rope(q, k, k, positions, freq)
    got = fi.qk_norm_rope(q, k, k, positions, freq, q_out=turned(4), k_out=turned(2), v_out=turned(2))
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    assert torch.equal(fi.prompt_attention(q, k, k, cu, out=turned(4)), fi.prompt_attention(q, k, k, cu))
    caches = torch.zeros((2, 5, 2, 8, 64), dtype=torch.bfloat16, device="cuda").transpose(2, 3)   # 5 pages of 8 tokens
    slots = torch.randperm(40, generator=g).cuda()
    fi.qk_norm_rope(q, k, k, positions, freq, slots=slots, k_out=caches[0], v_out=caches[1])
    flat = caches.reshape(2, 40, 2, 64)
    assert torch.equal(flat[0][slots], want[1]) and torch.equal(flat[1][slots], want[2])
    table, cached, one = torch.arange(5, dtype=torch.int32)[None].cuda(), torch.tensor([20], dtype=torch.int32).cuda(), cu.clamp(max=20)
    plain = caches.contiguous()
    assert torch.equal(fi.tree_attention(q[:20], caches[0], caches[1], table, cached, one, out=turned(4)[:20]), fi.tree_attention(q[:20], plain[0], plain[1], table, cached, one))


@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
def test_thousands_of_single_tokens_with_nothing_said_about_them(torch, fi, dtype):
    """Without max_nodes a sequence may have all the nodes: the workgroups grow with the nodes and the sequences, not with their product."""
    n, hq, hk, d, before = 24000, 8, 2, 64, 3
    kind, g = getattr(torch, dtype), torch.Generator(device="cuda").manual_seed(23)
    q = torch.randn((n, hq, d), generator=g, device="cuda").to(kind)
    k, v = (torch.randn((n, before + 1, hk, d), generator=g, device="cuda").to(kind) for _ in range(2))   # a page a sequence
    table = torch.randperm(n, generator=g, device="cuda").to(torch.int32)[:, None]
    cached, cu = torch.full((n,), before, dtype=torch.int32, device="cuda"), torch.arange(n + 1, dtype=torch.int32, device="cuda")
    got = fi.tree_attention(q, k, v, table, cached, cu, out=torch.full_like(q, float("nan"))).double()
    keys, values = (x[table[:, 0].long()].double().repeat_interleave(hq // hk, 2) for x in (k, v))   # [n, keys, heads, d]
    p = torch.softmax((q.double()[:, None] * keys).sum(-1) * d ** -0.5, 1)[..., None]
    want, size = (p * values).sum(1), (p * values.abs()).sum(1)
    # a score: d + 2 roundings of sum |q k|, at most |q| |k| < 256; a weight of bf16 and a result of bf16 a rounding each
    u, h = 2.0 ** -24, 2.0 ** -8 if dtype == "bfloat16" else 0.0
    assert ((got - want).abs() <= size * (2 * (d + 2) * 256 * d ** -0.5 * u + 200 * u + 1.01 * h) + want.abs() * 1.01 * h + 1e-30).all()


@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
@pytest.mark.parametrize("nodes", [5, 90])
def test_nodes_past_max_nodes_are_neither_computed_nor_seen(torch, fi, dtype, nodes):
    """Whatever the strides: rows that start on odd elements go to another kernel."""
    kind, g, most, before, d = getattr(torch, dtype), torch.Generator().manual_seed(24), nodes - 3, 10, 64
    q = torch.randn((nodes, 4, d), generator=g).to(kind)
    kv = torch.randn((2, (before + nodes + 15) // 16, 16, 2, d), generator=g).to(kind)
    mask = torch.full((nodes, 2), -1, dtype=torch.int64).cuda()   # every node sees every node
    table = torch.arange(kv.shape[1], dtype=torch.int32)[None].cuda()
    cached, cu = torch.tensor([before], dtype=torch.int32).cuda(), torch.tensor([0, nodes], dtype=torch.int32).cuda()
    k, v = kv.flatten(1, 2)[:, :before + most].double().repeat_interleave(2, 2)
    p = torch.softmax(torch.einsum("nhd,khd->hnk", q[:most].double(), k) * d ** -0.5, 2)
    want, size = torch.einsum("hnk,khd->nhd", p, v), torch.einsum("hnk,khd->nhd", p, v.abs())
    u, h = 2.0 ** -24, 2.0 ** -8 if dtype == "bfloat16" else 0.0
    bound = size * (2 * (d + 2) * 256 * d ** -0.5 * u + 400 * u + 1.01 * h) + want.abs() * 1.01 * h + 1e-30
    for pad in (0, 3):
        wide = torch.zeros((*kv.shape[:-1], d + pad), dtype=kind).cuda()
        wide[..., pad:] = kv.cuda()
        out = torch.full(q.shape, 7.0, dtype=kind).cuda()
        fi.tree_attention(q.cuda(), wide[0][..., pad:], wide[1][..., pad:], table, cached, cu, mask, max_nodes=most, out=out)
        assert ((out[:most].double().cpu() - want).abs() <= bound).all() and (out[most:] == 7).all()


def test_no_gradients_and_outputs_that_count_as_changed(torch, fi):
    """Every tensor of every call: refused where it requires a gradient, taken without gradient mode; what autograd has saved of an output is known to be stale."""
    g = torch.Generator().manual_seed(25)
    q, k = torch.randn((40, 4, 64), generator=g).cuda(), torch.randn((40, 2, 64), generator=g).cuda()
    cu, positions, freq, ones = torch.tensor([0, 40], dtype=torch.int32).cuda(), torch.arange(40, dtype=torch.int32).cuda(), torch.rand(32, generator=g).cuda(), torch.ones(64).cuda()
    cache, table, cached = k.view(10, 4, 2, 64).clone(), torch.arange(10, dtype=torch.int32)[None].cuda(), torch.tensor([39], dtype=torch.int32).cuda()
    x, w, s = torch.randn((3, 256), generator=g).cuda(), torch.randint(0, 256, (8, 128), generator=g, dtype=torch.uint8).cuda(), torch.rand((8, 4), generator=g).cuda()
    calls = [
        (fi.qk_norm_rope, dict(q=q, k=k, v=k.clone(), positions=positions, inv_freq=freq, q_weight=ones, k_weight=ones.clone(), slots=torch.arange(40).cuda(),
                               q_out=torch.zeros_like(q), k_out=torch.zeros_like(cache), v_out=torch.zeros_like(cache)), ("q_out", "k_out", "v_out")),
        (fi.prompt_attention, dict(q=q, k=k, v=k.clone(), cu_q=cu, out=torch.zeros_like(q)), ("out",)),
        (fi.tree_attention, dict(q=q[:1].clone(), k_cache=cache, v_cache=cache.clone(), block_table=table, cached=cached, cu_nodes=cu.clamp(max=1), out=torch.zeros_like(q[:1])), ("out",)),
        (fi.q4_matmul, dict(x=x, w=w, scales=s, out=torch.zeros((3, 8)).cuda()), ("out",)),
    ]
    for call, args, outs in calls:
        call(**args)
        want = [args[o].clone() for o in outs]
        for name, t in args.items():
            if not t.is_floating_point():
                continue
            wants = t.detach().clone().requires_grad_()
            with pytest.raises(ValueError, match=name + " requires a gradient"):
                call(**{**args, name: wants})
            with torch.no_grad():
                call(**{**args, name: wants})
        assert all(torch.equal(args[o], y) for o, y in zip(outs, want))
        for o in outs:
            before = args[o]._version
            call(**args)
            assert args[o]._version == before + 1
        factor = torch.ones((), device="cuda", requires_grad=True)
        loss = (factor * args[outs[0]]).sum()   # (saves the output)
        call(**args)
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            loss.backward()
        with torch.inference_mode():
            made = torch.zeros_like(args[outs[0]])
        call(**{**args, outs[0]: made})   # inference tensors have no counter
        assert torch.equal(made, want[0])


def test_a_mask_without_words_is_refused(torch, fi):
    """It has no address, as no mask at all has none, which stands for chains; no node would see another, or itself."""
    q, cache = torch.ones((3, 2, 64), device="cuda"), torch.ones((1, 16, 2, 64), device="cuda")
    table, cached, cu = torch.zeros((1, 1), dtype=torch.int32).cuda(), torch.zeros(1, dtype=torch.int32).cuda(), torch.tensor([0, 3], dtype=torch.int32).cuda()
    with pytest.raises(ValueError, match="no words"):
        fi.tree_attention(q, cache, cache, table, cached, cu, torch.zeros((3, 0), dtype=torch.int64).cuda())
    assert torch.equal(fi.tree_attention(q, cache, cache, table, cached, cu, torch.zeros((3, 1), dtype=torch.int64).cuda()), torch.zeros_like(q))


def test_a_cache_without_pages_takes_nothing(torch, fi):
    """Every slot is outside then: the queries are written, and nothing else."""
    x = torch.randn((5, 8, 64), generator=torch.Generator().manual_seed(26)).cuda()
    positions, freq, none = torch.arange(5, dtype=torch.int32).cuda(), torch.ones(32).cuda(), torch.zeros((0, 16, 2, 64)).cuda()
    want, _, _ = fi.qk_norm_rope(x[:, :4], x[:, 4:6], x[:, 6:], positions, freq)
    for v in (x[:, 6:], None):
        q, k_out, v_out = fi.qk_norm_rope(x[:, :4], x[:, 4:6], v, positions, freq, slots=torch.tensor([0, 1, -1, 5, 16]).cuda(), k_out=none, v_out=none.clone())
        assert torch.equal(q, want) and k_out.shape == none.shape
