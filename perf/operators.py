"""What the performance of the decoder operators is measured on.

A case names one operator of a decoder member's serving path and its sizes:

* "qk_norm_rope":     root-mean-square norms of the queries and keys of every head, the position rotation (one or several
                      axes), and the step's keys and values written to their slots of the paged cache;
* "prompt_attention": attention over whole prompts, packed sequences of different lengths, grouped heads, causal or not,
                      where asked with a prefix of keys in front of the queries;
* "tree_attention":   attention of trees of drafted tokens over a paged cache; a tree of one node is a decoding step;
* "q4_matmul":        products of a few rows with 4-bit weights that have a scale (and a zero point) per group.

Queries, keys, values and rows are N(0, 1), what a norm leaves; cache pages are handed out in random order, as an allocator
does after a while; lengths are ragged.  `own` chooses who computes: elementary torch operations in 32 bits, or this
repository's kernels.
"""
import math
import random

import torch

own = False

LONGEST_BYTES = 4 * 131072 * 8 * 128 * 2 * 2     # the largest listed cache
MOST_PAIRS = 32 * 8192 * 8192                    # query-key pairs of the largest listed prompt


def listed():
    return [
        # one decoding step of one sequence: latency only
        dict(name="rope_step", op="qk_norm_rope", dtype="bf16", tokens=1, q_heads=32, kv_heads=8, head_dim=128, rot=128, axes=1,
             interleaved=False, page=16),
        # three frames of 27 x 27 patches with time, height and width positions, an unconverted fp32 model, odd head size
        dict(name="rope_video_f32", op="qk_norm_rope", dtype="f32", tokens=2187, q_heads=16, kv_heads=16, head_dim=72, rot=72, axes=3,
             interleaved=True, page=48),
        # a long prompt
        dict(name="rope_prompt", op="qk_norm_rope", dtype="bf16", tokens=16384, q_heads=32, kv_heads=8, head_dim=128, rot=128, axes=1,
             interleaved=False, page=64),
        # a round of short ragged requests for a small member
        dict(name="prompt_short", op="prompt_attention", dtype="bf16", seqs=7, longest=301, prefix=0, q_heads=12, kv_heads=4, head_dim=64,
             causal=True, ragged=1),
        # the patches of four images, every one seen by every one, fp32, odd head size
        dict(name="prompt_images_f32", op="prompt_attention", dtype="f32", seqs=4, longest=729, prefix=0, q_heads=16, kv_heads=16, head_dim=72,
             causal=False, ragged=2),
        # one long document
        dict(name="prompt_long", op="prompt_attention", dtype="bf16", seqs=1, longest=8192, prefix=0, q_heads=32, kv_heads=8, head_dim=128,
             causal=True, ragged=0),
        # interactive decoding: one token, an ordinary history
        dict(name="tree_step", op="tree_attention", dtype="bf16", seqs=1, nodes=1, longest=1003, page=16, q_heads=32, kv_heads=8, head_dim=128,
             ragged=0),
        # a round of drafts of up to 37 tokens, ragged histories
        dict(name="tree_drafts", op="tree_attention", dtype="bf16", seqs=12, nodes=37, longest=5001, page=64, q_heads=32, kv_heads=8, head_dim=128,
             ragged=3),
        # long histories, one token each: the cache is all that counts
        dict(name="tree_long", op="tree_attention", dtype="bf16", seqs=4, nodes=1, longest=131071, page=16, q_heads=32, kv_heads=8, head_dim=128,
             ragged=0),
        # one row, a square layer
        dict(name="q4_row", op="q4_matmul", dtype="bf16", rows=1, inputs=4096, outputs=4096, group=128, zeros=False),
        # five rows of an fp32 member's last layer, small groups with zero points
        dict(name="q4_classes_f32", op="q4_matmul", dtype="f32", rows=5, inputs=4096, outputs=1000, group=32, zeros=True),
        # the widest fully connected layer of this repository's families, for the nodes of a drafted tree
        dict(name="q4_wide", op="q4_matmul", dtype="bf16", rows=24, inputs=25088, outputs=4096, group=64, zeros=True),
    ]


def draw(rng):
    def spread(lo, hi):   # over the logarithm, odd values among them
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    while True:
        op = rng.choice(["qk_norm_rope", "prompt_attention", "tree_attention", "q4_matmul"])
        dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
        q_heads, kv_heads = rng.choice([(32, 8), (32, 32), (28, 4), (16, 2), (12, 4), (8, 1), (5, 5)])
        head_dim = rng.choice([64, 72, 80, 96, 128, 128, 256])
        page = rng.choice([1, 16, 16, 32, 48, 64, 256])
        ragged = rng.randint(0, 9999)
        if op == "qk_norm_rope":
            case = dict(op=op, dtype=dtype, tokens=spread(1, 16384), q_heads=q_heads, kv_heads=kv_heads, head_dim=head_dim,
                        rot=rng.choice([head_dim, head_dim, head_dim // 2]), axes=rng.choice([1, 1, 2, 3]), interleaved=rng.random() < 0.5, page=page)
            fits = work(case)["bytes"] <= 16384 * 48 * 128 * 2 * 2 * 1.02
        elif op == "prompt_attention":
            case = dict(op=op, dtype=dtype, seqs=spread(1, 24), longest=spread(1, 8192), prefix=rng.choice([0, 0, spread(1, 2000)]), q_heads=q_heads,
                        kv_heads=kv_heads, head_dim=head_dim, causal=rng.random() < 0.8, ragged=ragged)
            pairs = case["seqs"] * q_heads * case["longest"] * (case["longest"] + case["prefix"])
            fits = pairs * head_dim <= MOST_PAIRS * 128 / (2 if case["causal"] else 4) / (8 if dtype == "f32" else 1) and pairs <= MOST_PAIRS
        elif op == "tree_attention":
            case = dict(op=op, dtype=dtype, seqs=spread(1, 64), nodes=rng.choice([1, spread(1, 100)]), longest=spread(1, 131072), page=page,
                        q_heads=q_heads, kv_heads=kv_heads, head_dim=head_dim, ragged=ragged)
            keys = case["seqs"] * (case["longest"] + case["nodes"])
            fits = (keys * kv_heads * head_dim * 4 * (2 if dtype == "f32" else 1) <= LONGEST_BYTES
                    and keys * q_heads * case["nodes"] * head_dim <= MOST_PAIRS * 16)
        else:
            group = rng.choice([32, 64, 128])
            case = dict(op=op, dtype=dtype, rows=spread(1, 64), inputs=group * spread(4, 25088 // group), outputs=spread(100, 16384), group=group,
                        zeros=rng.random() < 0.5)
            fits = case["inputs"] * case["outputs"] <= 25088 * 4096 and case["inputs"] * case["outputs"] * case["rows"] <= 25088 * 4096 * 24
        if fits:
            return case


def lengths(case):
    """Tokens of every sequence: the longest for all where nothing is ragged, else the first as long as the longest and the others spread below it."""
    most = case["longest"]
    if not case["ragged"]:
        return [most] * case["seqs"]
    r = random.Random(case["ragged"])
    return [most] + [int(round(math.exp(r.uniform(0, math.log(most))))) for _ in range(case["seqs"] - 1)]


def nodes(case):
    """Drafted tokens of every sequence."""
    r = random.Random(case["ragged"] + 1)
    return [case["nodes"]] + [case["nodes"] if not case["ragged"] else r.randint(1, case["nodes"]) for _ in range(case["seqs"] - 1)]


def sections(case):
    pairs, axes = case["rot"] // 2, case["axes"]
    return [pairs - (axes - 1) * (pairs // axes)] + [pairs // axes] * (axes - 1)


def stored(case):
    return torch.float32 if case["dtype"] == "f32" else torch.bfloat16


def offsets(counts):
    total, out = 0, [0]
    for n in counts:
        total += n
        out.append(total)
    return torch.tensor(out, dtype=torch.int32, device="cuda")


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    kind = stored(case)

    def normal(*shape):
        return torch.randn(shape, generator=g, device="cuda").to(kind)

    state = dict(op=case["op"])
    if case["op"] == "q4_matmul":
        n, k, groups = case["outputs"], case["inputs"], case["inputs"] // case["group"]
        state.update(x=normal(case["rows"], k), w=torch.randint(0, 256, (n, k // 2), dtype=torch.uint8, generator=g, device="cuda"),
                     scales=(0.5 + torch.rand((n, groups), generator=g, device="cuda")) / (4.6 * math.sqrt(k)),
                     zeros=torch.randint(5, 12, (n, groups), dtype=torch.uint8, generator=g, device="cuda") if case["zeros"] else None,
                     group=case["group"], out=torch.zeros((case["rows"], n), dtype=kind, device="cuda"))
        return state
    hq, hk, d = case["q_heads"], case["kv_heads"], case["head_dim"]
    if case["op"] == "qk_norm_rope":
        t, page = case["tokens"], case["page"]
        qkv = normal(t, hq + 2 * hk, d)   # the three parts of one projection's rows
        pages = (t + page - 1) // page + 1
        order = torch.randperm(pages, generator=g, device="cuda")
        at = torch.arange(t, device="cuda")
        place = torch.arange(t, dtype=torch.int32, device="cuda")
        first = torch.randint(0, 4096, (1,), generator=g, device="cuda", dtype=torch.int32)
        if case["axes"] == 1:
            positions = (first + place)[:, None]
        else:   # frames of 27 x 27 patches: time, height, width; two axes: height, width
            positions = torch.stack([first + place // 729, place // 27 % 27, place % 27][3 - case["axes"]:], 1)
        inv_freq = torch.cat([1e4 ** -(torch.arange(s, device="cuda", dtype=torch.float32) / s) for s in sections(case)])
        axis = [a for a, count in enumerate(sections(case)) for _ in range(count)]   # of every pair
        state.update(q=qkv[:, :hq], k=qkv[:, hq:hq + hk], v=qkv[:, hq + hk:], positions=positions.contiguous(), inv_freq=inv_freq,
                     axis=torch.tensor(axis, device="cuda"),
                     q_weight=1 + 0.1 * torch.randn(d, generator=g, device="cuda"), k_weight=1 + 0.1 * torch.randn(d, generator=g, device="cuda"),
                     eps=1e-6, sections=sections(case), interleaved=case["interleaved"], slots=order[at // page] * page + at % page,
                     q_out=torch.zeros((t, hq, d), dtype=kind, device="cuda"), k_cache=torch.zeros((pages, page, hk, d), dtype=kind, device="cuda"),
                     v_cache=torch.zeros((pages, page, hk, d), dtype=kind, device="cuda"))
        return state
    state["scale"] = 1.0 / math.sqrt(d)
    if case["op"] == "prompt_attention":
        new = lengths(case)
        seen = [n + case["prefix"] for n in new]
        state.update(q=normal(sum(new), hq, d), k=normal(sum(seen), hk, d), v=normal(sum(seen), hk, d), cu_q=offsets(new), cu_k=offsets(seen),
                     longest_q=max(new), longest_k=max(seen), causal=case["causal"], out=torch.zeros((sum(new), hq, d), dtype=kind, device="cuda"))
        return state
    cached, drafted, page = lengths(case), nodes(case), case["page"]
    need = [(c + n + page - 1) // page for c, n in zip(cached, drafted)]
    order = torch.randperm(sum(need) + 3, generator=g, device="cuda").to(torch.int32)
    start = [sum(need[:i]) for i in range(len(need))]
    column = torch.arange(max(need), device="cuda")
    inside = column[None] < torch.tensor(need, device="cuda")[:, None]
    table = torch.where(inside, order[(torch.tensor(start, device="cuda")[:, None] + column[None]).clamp(max=sum(need) - 1)], 0)
    r, words = random.Random(seed), (max(drafted) + 63) // 64
    rows = []
    for n in drafted:   # every node hangs from one before it or from the last committed token
        seen = []
        for i in range(n):
            parent = r.randint(max(-1, i - 5), i - 1)
            seen.append((seen[parent] if parent >= 0 else 0) | 1 << i)
        rows += [[(m >> 64 * w) & (2 ** 64 - 1) for w in range(words)] for m in seen]
    mask = torch.tensor([[w - 2 ** 64 if w >= 2 ** 63 else w for w in row] for row in rows], dtype=torch.int64, device="cuda")
    pages = sum(need) + 3
    state.update(q=normal(sum(drafted), hq, d), k_cache=normal(pages, page, hk, d), v_cache=normal(pages, page, hk, d), table=table.contiguous(),
                 cached=torch.tensor(cached, dtype=torch.int32, device="cuda"), cu_nodes=offsets(drafted), mask=mask,
                 longest=max(c + n for c, n in zip(cached, drafted)), most_nodes=max(drafted),
                 out=torch.zeros((sum(drafted), hq, d), dtype=kind, device="cuda"))
    return state


def run(state):
    if own:
        return run_own(state)
    return {"qk_norm_rope": plain_rope, "prompt_attention": plain_prompt, "tree_attention": plain_tree, "q4_matmul": plain_q4}[state["op"]](state)


def run_own(s):
    import paper_2410_21120_amd as fi
    if s["op"] == "qk_norm_rope":
        fi.qk_norm_rope(s["q"], s["k"], s["v"], s["positions"], s["inv_freq"], q_weight=s["q_weight"], k_weight=s["k_weight"], eps=s["eps"],
                        sections=s["sections"], interleaved=s["interleaved"], slots=s["slots"], q_out=s["q_out"], k_out=s["k_cache"], v_out=s["v_cache"])
        return {"q": s["q_out"], "k_cache": s["k_cache"], "v_cache": s["v_cache"]}
    if s["op"] == "prompt_attention":
        return fi.prompt_attention(s["q"], s["k"], s["v"], s["cu_q"], s["cu_k"], causal=s["causal"], scale=s["scale"], out=s["out"])
    if s["op"] == "tree_attention":
        return fi.tree_attention(s["q"], s["k_cache"], s["v_cache"], s["table"], s["cached"], s["cu_nodes"], s["mask"], scale=s["scale"],
                                 max_nodes=s["most_nodes"], max_length=s["longest"], out=s["out"])
    return fi.q4_matmul(s["x"], s["w"], s["scales"], s["zeros"], group=s["group"], out=s["out"])


def normed_and_rotated(x, weight, angles, eps, interleaved):
    x = x.float()
    x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + eps) * weight
    half = angles.shape[-1]
    c, s, turned, rest = angles.cos()[:, None], angles.sin()[:, None], x[..., :2 * half], x[..., 2 * half:]
    if interleaved:
        a, b = turned[..., 0::2], turned[..., 1::2]
        return torch.cat([torch.stack([a * c - b * s, b * c + a * s], -1).flatten(-2), rest], -1)
    a, b = turned[..., :half], turned[..., half:]
    return torch.cat([a * c - b * s, b * c + a * s, rest], -1)


def plain_rope(s):
    angles = s["positions"][:, s["axis"]].float() * s["inv_freq"]
    kind = s["q"].dtype
    q = normed_and_rotated(s["q"], s["q_weight"], angles, s["eps"], s["interleaved"]).to(kind)
    k = normed_and_rotated(s["k"], s["k_weight"], angles, s["eps"], s["interleaved"]).to(kind)
    s["k_cache"].view(-1, *k.shape[1:])[s["slots"]] = k
    s["v_cache"].view(-1, *k.shape[1:])[s["slots"]] = s["v"]
    return {"q": q, "k_cache": s["k_cache"], "v_cache": s["v_cache"]}


def padded(cu, longest):
    """Row of every (sequence, place), and whether there is one."""
    place = torch.arange(longest, device=cu.device)
    inside = place[None] < (cu[1:] - cu[:-1])[:, None]
    return torch.where(inside, cu[:-1, None] + place[None], 0), inside


def owners(cu, rows):
    """Sequence and place in it of every packed row."""
    at = torch.arange(rows, device=cu.device)
    seq = (at[:, None] >= cu[None, 1:]).sum(1)
    return seq, at - cu[seq]


def softmax_product(q, k, v, visible, scale):
    """q [b, kv heads, group, n, d], k and v [b, kv heads, keys, d], visible [b, n, keys]; rows that see nothing are zero."""
    b, hk, group, n, d = q.shape
    scores = torch.matmul(q.reshape(b, hk, group * n, d), k.transpose(-1, -2)).view(b, hk, group, n, -1) * scale
    scores = torch.where(visible[:, None, None], scores, -math.inf)
    top = scores.amax(-1, keepdim=True)
    e = torch.exp(scores - torch.where(top == -math.inf, 0.0, top))
    total = e.sum(-1, keepdim=True)
    out = torch.matmul(e.view(b, hk, group * n, -1), v).view(b, hk, group, n, d)
    return out / torch.where(total == 0, 1.0, total)


def plain_prompt(s):
    hq, hk = s["q"].shape[1], s["k"].shape[1]
    rows, _ = padded(s["cu_q"], s["longest_q"])
    keys, there = padded(s["cu_k"], s["longest_k"])
    q = s["q"].float()[rows].view(*rows.shape, hk, hq // hk, -1).permute(0, 2, 3, 1, 4)
    k, v = (s[x].float()[keys].permute(0, 2, 1, 3) for x in ("k", "v"))
    visible = there[:, None].expand(-1, rows.shape[1], -1)
    if s["causal"]:   # the last query sees every key
        more = (s["cu_k"][1:] - s["cu_k"][:-1]) - (s["cu_q"][1:] - s["cu_q"][:-1])
        i, j = torch.arange(rows.shape[1], device=rows.device), torch.arange(keys.shape[1], device=rows.device)
        visible = visible & (j[None, None] <= i[None, :, None] + more[:, None, None])
    out = softmax_product(q, k, v, visible, s["scale"]).permute(0, 3, 1, 2, 4).flatten(2, 3)
    seq, place = owners(s["cu_q"], s["q"].shape[0])
    return out[seq, place].to(s["q"].dtype)


def plain_tree(s):
    hq, hk, page = s["q"].shape[1], s["k_cache"].shape[2], s["k_cache"].shape[1]
    rows, there = padded(s["cu_nodes"], s["most_nodes"])
    q = s["q"].float()[rows].view(*rows.shape, hk, hq // hk, -1).permute(0, 2, 3, 1, 4)
    j = torch.arange(s["longest"], device=rows.device)
    slot = s["table"][:, j // page].long() * page + j % page
    k, v = (s[x].view(-1, hk, s["q"].shape[2])[slot].permute(0, 2, 1, 3).float() for x in ("k_cache", "v_cache"))
    node = j[None] - s["cached"][:, None]                      # which node of the tree a key is
    words = s["mask"][rows]                                    # [b, nodes, words]
    at = node.clamp(0, s["most_nodes"] - 1)
    bits = torch.gather(words, 2, (at // 64)[:, None].expand(-1, rows.shape[1], -1)) >> (at % 64)[:, None] & 1
    drafted = (s["cu_nodes"][1:] - s["cu_nodes"][:-1])[:, None]
    visible = (node < 0)[:, None] | ((node >= 0) & (node < drafted))[:, None] & (bits == 1)
    out = softmax_product(q, k, v, visible, s["scale"]).permute(0, 3, 1, 2, 4).flatten(2, 3)
    seq, place = owners(s["cu_nodes"], s["q"].shape[0])
    return out[seq, place].to(s["q"].dtype)


def plain_q4(s):
    w = torch.stack([s["w"] & 15, s["w"] >> 4], -1).view(s["w"].shape[0], -1, s["group"]).float()   # the low half of a byte comes first
    w = (w - (8.0 if s["zeros"] is None else s["zeros"].float()[..., None])) * s["scales"][..., None]
    return torch.matmul(s["x"].float(), w.flatten(1).t()).to(s["x"].dtype)


def exact(case, seed):
    """The operator's definition in 64 bits, sequence by sequence, head by head."""
    s = prepare(case, seed)
    return {"qk_norm_rope": exact_rope, "prompt_attention": exact_prompt, "tree_attention": exact_tree, "q4_matmul": exact_q4}[case["op"]](s)


def exact_rope(s):
    ends, table = 0, []
    for axis, count in enumerate(s["sections"]):
        table.append(s["positions"][:, axis:axis + 1].double() * s["inv_freq"][ends:ends + count].double())
        ends += count
    turn = torch.polar(torch.ones(()).double().cuda(), torch.cat(table, 1))[:, None]   # the rotation as a complex factor

    def one(x, weight):
        x = x.double()
        x = x / (x.square().sum(-1, keepdim=True) / x.shape[-1] + s["eps"]).sqrt() * weight.double()
        y = x.clone()
        first, second = (slice(0, 2 * ends, 2), slice(1, 2 * ends, 2)) if s["interleaved"] else (slice(0, ends), slice(ends, 2 * ends))
        z = torch.complex(x[..., first].contiguous(), x[..., second].contiguous()) * turn
        y[..., first], y[..., second] = z.real, z.imag
        return y

    k_cache, v_cache = s["k_cache"].double(), s["v_cache"].double()
    page = k_cache.shape[1]
    k_cache[s["slots"] // page, s["slots"] % page] = one(s["k"], s["k_weight"])
    v_cache[s["slots"] // page, s["slots"] % page] = s["v"].double()
    return {"q": one(s["q"], s["q_weight"]), "k_cache": k_cache, "v_cache": v_cache}


def exact_rows(q, k, v, seen, scale):
    """q [n, d], k and v [keys, d], seen [n, keys]."""
    scores = (q @ k.t() * scale).masked_fill(~seen, -math.inf)
    return torch.softmax(scores, 1).nan_to_num(0.0) @ v if k.shape[0] else torch.zeros_like(q)


def exact_prompt(s):
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    group, cu_q, cu_k = s["q"].shape[1] // s["k"].shape[1], s["cu_q"].tolist(), s["cu_k"].tolist()
    for b in range(len(cu_q) - 1):
        n, keys = cu_q[b + 1] - cu_q[b], cu_k[b + 1] - cu_k[b]
        seen = torch.ones((n, keys), dtype=torch.bool, device="cuda")
        if s["causal"]:
            seen = seen.tril(keys - n)
        for h in range(s["q"].shape[1]):
            k, v = (s[x][cu_k[b]:cu_k[b + 1], h // group].double() for x in ("k", "v"))
            out[cu_q[b]:cu_q[b + 1], h] = exact_rows(s["q"][cu_q[b]:cu_q[b + 1], h].double(), k, v, seen, s["scale"])
    return out


def exact_tree(s):
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    group, page, cu = s["q"].shape[1] // s["k_cache"].shape[2], s["k_cache"].shape[1], s["cu_nodes"].tolist()
    for b, before in enumerate(s["cached"].tolist()):
        n = cu[b + 1] - cu[b]
        places = s["table"][b, :(before + n + page - 1) // page].long()
        k, v = (s[x][places].flatten(0, 1)[:before + n].double() for x in ("k_cache", "v_cache"))
        seen = torch.ones((n, before + n), dtype=torch.bool, device="cuda")
        words = s["mask"][cu[b]:cu[b + 1]]
        for j in range(n):
            seen[:, before + j] = (words[:, j // 64] >> (j % 64)) % 2 != 0
        for h in range(s["q"].shape[1]):
            out[cu[b]:cu[b + 1], h] = exact_rows(s["q"][cu[b]:cu[b + 1], h].double(), k[:, h // group], v[:, h // group], seen, s["scale"])
    return out


def exact_q4(s):
    n, k = s["w"].shape[0], s["x"].shape[1]
    w = torch.empty((n, k), dtype=torch.float64, device="cuda")
    w[:, 0::2], w[:, 1::2] = s["w"] % 16, s["w"] // 16
    zero = torch.full_like(s["scales"], 8).double() if s["zeros"] is None else s["zeros"].double()
    w = (w.view(n, -1, s["group"]) - zero[:, :, None]) * s["scales"].double()[:, :, None]
    return s["x"].double() @ w.view(n, k).t()


def work(case):
    """Inputs in once, outputs out once; products of a query with the keys that it sees (a node: its history
    and itself), two operations per multiply-add."""
    size = 4 if case["dtype"] == "f32" else 2
    if case["op"] == "q4_matmul":
        m, k, n = case["rows"], case["inputs"], case["outputs"]
        return {"bytes": n * k // 2 + n * (k // case["group"]) * (5 if case["zeros"] else 4) + m * (k + n) * size, "flops": 2 * m * n * k}
    hq, hk, d = case["q_heads"], case["kv_heads"], case["head_dim"]
    if case["op"] == "qk_norm_rope":
        t = case["tokens"]
        return {"bytes": t * (2 * (hq + 2 * hk) * d * size + 4 * case["axes"] + 8) + 8 * d + 2 * case["rot"], "flops": t * (hq + hk) * d * 7}
    if case["op"] == "prompt_attention":
        new, before = lengths(case), case["prefix"]
        pairs = sum(n * before + (n * (n + 1) // 2 if case["causal"] else n * n) for n in new)
        return {"bytes": 2 * d * size * (hq * sum(new) + hk * sum(n + before for n in new)), "flops": 4 * d * hq * pairs}
    cached, drafted = lengths(case), nodes(case)
    keys = sum(c + n for c, n in zip(cached, drafted))
    return {"bytes": 2 * d * size * (hk * keys + hq * sum(drafted)), "flops": 4 * d * hq * sum(n * (c + 1) for c, n in zip(cached, drafted))}
