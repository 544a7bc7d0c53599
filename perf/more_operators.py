"""What the performance of beam search over a 4-bit cache is measured on.

A case names one operator of a decoder member's serving path and its sizes:

* "fp4_cache_write":    a step's keys and values into a paged cache of 4-bit values: blocks of 32 values of a head, E2M1 codes (0, 0.5, 1, 1.5, 2,
                        3, 4, 6 and a sign) times a power of two; where asked, what the cache then holds for them comes back too;
* "fp4_tree_attention": attention of drafted trees, or single tokens, over that cache; beams share the pages of their prompt;
* "beam_select":        the best continuations of every sequence over its beams and the vocabulary, with their beams and scores;
* "fork_pages":         the cache rows after a selection: children share their parents' pages, the page that is written next is copied
                        where it is shared, room for the next tokens is made, pages of beams that ended are free;
* "compact_pages":      pages in use move to the lowest numbers of the pool, so that the rest of it can be given back.

Keys, values and queries are N(0, 1), what a norm leaves; pages are handed out in random order, as an allocator does after a while.  `own` chooses
who computes: elementary torch operations in 32 bits (64 next to borders), or this repository's kernels.
"""
import math
import random

import torch

own = False

LONGEST_KEYS = 4 * 131072 * 8 * 128       # key values of the largest listed cache
MOST_PAIRS = 12 * 37 * 32 * 5038 * 128    # products of the largest listed round of trees
MOST_LOGITS = 64 * 8 * 131072
MOST_POOL = 4096 * 64 * 8 * 128 * 2 * 4   # bytes of the largest listed pool
BLOCK = 32


def listed():
    return [
        # one decoding step of one sequence: latency only
        dict(name="write_step", op="fp4_cache_write", dtype="bf16", tokens=1, kv_heads=8, head_dim=128, page=16, held=False),
        # a long prompt; attention over it goes by what the cache holds, as later steps will
        dict(name="write_prompt", op="fp4_cache_write", dtype="bf16", tokens=16384, kv_heads=8, head_dim=128, page=64, held=True),
        # interactive decoding: one token, an ordinary history
        dict(name="fp4_step", op="fp4_tree_attention", dtype="bf16", seqs=1, beams=1, nodes=1, longest=1003, page=16, q_heads=32, kv_heads=8, head_dim=128,
             ragged=0),
        # a step of beam search: eight requests of four beams
        dict(name="fp4_beams", op="fp4_tree_attention", dtype="bf16", seqs=8, beams=4, nodes=1, longest=5001, page=64, q_heads=32, kv_heads=8, head_dim=128,
             ragged=3),
        # a round of drafts of up to 37 tokens, ragged histories, an unconverted fp32 model, odd head size
        dict(name="fp4_drafts_f32", op="fp4_tree_attention", dtype="f32", seqs=12, beams=1, nodes=37, longest=2003, page=48, q_heads=16, kv_heads=4, head_dim=72,
             ragged=5),
        # long histories, one token each: the cache is all that counts
        dict(name="fp4_long", op="fp4_tree_attention", dtype="bf16", seqs=4, beams=1, nodes=1, longest=131071, page=16, q_heads=32, kv_heads=8, head_dim=128,
             ragged=0),
        # a step of one request
        dict(name="beam_step", op="beam_select", dtype="bf16", seqs=1, beams=4, keep=4, vocab=32000, ends=False),
        # many requests, twice as many candidates as beams since some may end, a last layer that leaves fp32
        dict(name="beam_batch_f32", op="beam_select", dtype="f32", seqs=64, beams=8, keep=16, vocab=131072, ends=True),
        # the rows of that one request
        dict(name="fork_step", op="fork_pages", seqs=1, beams=4, longest=1003, page=16, kv_heads=8, head_dim=128, layers=1, room=1, scarce=False, ragged=0),
        # the rows of many requests, two layers of caches
        dict(name="fork_batch", op="fork_pages", seqs=64, beams=8, longest=2001, page=32, kv_heads=8, head_dim=128, layers=2, room=1, scarce=False, ragged=7),
        # a small pool between two rounds
        dict(name="compact_small", op="compact_pages", pages=512, page=16, kv_heads=8, head_dim=128, layers=1, rows=12, ragged=1),
        # a large one, a bit over half of it in use
        dict(name="compact_large", op="compact_pages", pages=4096, page=64, kv_heads=8, head_dim=128, layers=2, rows=96, ragged=2),
    ]


def draw(rng):
    def spread(lo, hi):   # over the logarithm, odd values among them
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    while True:
        op = rng.choice(["fp4_cache_write", "fp4_tree_attention", "fp4_tree_attention", "beam_select", "fork_pages", "compact_pages"])
        dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
        q_heads, kv_heads = rng.choice([(32, 8), (32, 32), (28, 4), (16, 2), (12, 4), (8, 1), (5, 5)])
        head_dim = rng.choice([64, 72, 80, 96, 128, 128, 256])
        page = rng.choice([1, 16, 16, 32, 48, 64, 256])
        ragged = rng.randint(0, 9999)
        if op == "fp4_cache_write":
            case = dict(op=op, dtype=dtype, tokens=spread(1, 16384), kv_heads=kv_heads, head_dim=head_dim, page=page, held=rng.random() < 0.5)
            fits = work(case)["bytes"] <= 16384 * 8 * 128 * 2 * 4.6
        elif op == "fp4_tree_attention":
            case = dict(op=op, dtype=dtype, seqs=spread(1, 64), beams=rng.choice([1, 1, 2, 4, 5]), nodes=rng.choice([1, 1, spread(1, 100)]), longest=spread(1, 131072),
                        page=page, q_heads=q_heads, kv_heads=kv_heads, head_dim=head_dim, ragged=ragged)
            keys = case["seqs"] * case["beams"] * (case["longest"] + case["nodes"])
            fits = keys * kv_heads * head_dim <= LONGEST_KEYS and keys * q_heads * case["nodes"] * head_dim <= MOST_PAIRS
        elif op == "beam_select":
            beams = rng.choice([1, 2, 3, 4, 5, 8, 16])
            case = dict(op=op, dtype=dtype, seqs=spread(1, 64), beams=beams, keep=rng.choice([beams, 2 * beams]), vocab=spread(500, 262144), ends=rng.random() < 0.5)
            fits = case["seqs"] * beams * case["vocab"] <= MOST_LOGITS
        elif op == "fork_pages":
            case = dict(op=op, seqs=spread(1, 64), beams=rng.choice([1, 2, 3, 4, 5, 8]), longest=spread(1, 4000), page=page, kv_heads=kv_heads, head_dim=head_dim,
                        layers=rng.choice([1, 1, 2, 3]), room=rng.choice([1, 1, 1, 0, 5, 17]), scarce=rng.random() < 0.2, ragged=ragged)
            held = case["seqs"] * case["beams"] * (case["longest"] + 2 * page + case["room"])
            fits = held * kv_heads * head_dim * 4 * case["layers"] <= MOST_POOL
        else:
            case = dict(op=op, pages=spread(16, 8192), page=page, kv_heads=kv_heads, head_dim=head_dim, layers=rng.choice([1, 1, 2, 3]), rows=spread(1, 100), ragged=ragged)
            fits = case["pages"] * page * kv_heads * head_dim * 4 * case["layers"] <= MOST_POOL
        if fits:
            return case


def lengths(case):
    """Tokens of every sequence: the longest for all where nothing is ragged, else the first as long as the longest and the others spread below it."""
    most = case["longest"]
    if not case["ragged"]:
        return [most] * case["seqs"]
    r = random.Random(case["ragged"])
    return [most] + [int(round(math.exp(r.uniform(0, math.log(most))))) for _ in range(case["seqs"] - 1)]


def drafted(case):
    """Nodes of every row of the batch (a beam of a sequence)."""
    r = random.Random(case["ragged"] + 1)
    return [case["nodes"]] + [case["nodes"] if not case["ragged"] else r.randint(1, case["nodes"]) for _ in range(case["seqs"] * case["beams"] - 1)]


def rows_of_pages(cached, more, beams, page):
    """The pages of every row, numbered from 0: a sequence's beams share the pages of the first half of its tokens, the rest is their own.  Every
    row has pages for its tokens and the `more[row]` behind them.  Returns the rows and how many pages there are."""
    rows, used = [], 0
    for s, n in enumerate(cached):
        shared = n // 2 // page if beams > 1 else 0
        prompt = list(range(used, used + shared))
        used += shared
        for b in range(beams):
            rest = -(-(n + more[s * beams + b]) // page) - shared
            rows.append(prompt + list(range(used, used + rest)))
            used += rest
    return rows, used


def table_of(rows, order, columns, empty):
    """int32 [rows, columns] on the GPU, page i of rows_of_pages being order[i] of the pool."""
    flat = [rows_i + [-1] * (columns - len(rows_i)) for rows_i in rows]
    at = torch.tensor(flat, device="cuda").reshape(len(rows), columns)
    return torch.where(at < 0, empty, order[at.clamp(min=0)]).to(torch.int32).contiguous()


def stored(case):
    return torch.float32 if case.get("dtype") == "f32" else torch.bfloat16


def offsets(counts):
    total, out = 0, [0]
    for n in counts:
        total += n
        out.append(total)
    return torch.tensor(out, dtype=torch.int32, device="cuda")


def ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def blocks(head_dim):
    return (head_dim + BLOCK - 1) // BLOCK


def empty_cache(pages, page, heads, dim):
    """Codes [pages, page, heads, dim / 2] and scales [pages, page, heads, blocks], in memory a head's tokens of a page together."""
    codes = torch.zeros((pages, heads, page, dim // 2), dtype=torch.uint8, device="cuda")
    scales = torch.full((pages, heads, page, blocks(dim)), 127, dtype=torch.uint8, device="cuda")
    return codes.permute(0, 2, 1, 3), scales.permute(0, 2, 1, 3)


def normal_cache(g, pages, page, heads, dim):
    codes, scales = empty_cache(pages, page, heads, dim)
    step = max(1, (1 << 26) // (page * heads * dim))
    for at in range(0, pages, step):
        n = min(step, pages - at)
        c, s = encoded(torch.randn((n, heads, page, dim), generator=g, device="cuda"))
        codes.permute(0, 2, 1, 3)[at:at + n], scales.permute(0, 2, 1, 3)[at:at + n] = c, s
    return codes, scales


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    kind = stored(case)

    def normal(*shape):
        return torch.randn(shape, generator=g, device="cuda").to(kind)

    return dict(op=case["op"]) | {"fp4_cache_write": prepare_write, "fp4_tree_attention": prepare_attention, "beam_select": prepare_beams, "fork_pages": prepare_fork,
                                  "compact_pages": prepare_compact}[case["op"]](case, seed, g, normal)


def prepare_write(case, seed, g, normal):
    t, hk, d, page = case["tokens"], case["kv_heads"], case["head_dim"], case["page"]
    kv = normal(t, 2 * hk, d)   # the two parts of one projection's rows
    pages = (t + page - 1) // page + 1
    order = torch.randperm(pages, generator=g, device="cuda")
    at = torch.arange(t, device="cuda")
    kc, ks = empty_cache(pages, page, hk, d)
    vc, vs = empty_cache(pages, page, hk, d)
    return dict(k=kv[:, :hk], v=kv[:, hk:], slots=order[at // page] * page + at % page, k_codes=kc, k_scales=ks, v_codes=vc, v_scales=vs,
                k_held=torch.zeros((t, hk, d), dtype=kv.dtype, device="cuda") if case["held"] else None,
                v_held=torch.zeros((t, hk, d), dtype=kv.dtype, device="cuda") if case["held"] else None)


def prepare_attention(case, seed, g, normal):
    hq, hk, d, page, beams = case["q_heads"], case["kv_heads"], case["head_dim"], case["page"], case["beams"]
    cached, nodes = lengths(case), drafted(case)
    rows, used = rows_of_pages(cached, nodes, beams, page)
    pages = used + 3
    order = torch.randperm(pages, generator=g, device="cuda")
    table = table_of(rows, order, max(len(x) for x in rows), 0)
    r, words, mask = random.Random(seed), (max(nodes) + 63) // 64, None
    if max(nodes) > 1:   # every node hangs from one before it or from the last committed token
        trees = []
        for n in nodes:
            seen = []
            for i in range(n):
                parent = r.randint(max(-1, i - 5), i - 1)
                seen.append((seen[parent] if parent >= 0 else 0) | 1 << i)
            trees += [[(m >> 64 * w) & (2 ** 64 - 1) for w in range(words)] for m in seen]
        mask = torch.tensor([[w - 2 ** 64 if w >= 2 ** 63 else w for w in row] for row in trees], dtype=torch.int64, device="cuda")
    kc, ks = normal_cache(g, pages, page, hk, d)
    vc, vs = normal_cache(g, pages, page, hk, d)
    every = [n for n in cached for _ in range(beams)]
    return dict(q=normal(sum(nodes), hq, d), k_codes=kc, k_scales=ks, v_codes=vc, v_scales=vs, table=table, cached=ints(every), cu_nodes=offsets(nodes), mask=mask,
                scale=1.0 / math.sqrt(d), longest=max(c + n for c, n in zip(every, nodes)), most_nodes=max(nodes),
                out=torch.zeros((sum(nodes), hq, d), dtype=stored(case), device="cuda"))


def prepare_beams(case, seed, g, normal):
    s, b, keep, vocab = case["seqs"], case["beams"], case["keep"], case["vocab"]
    state = dict(logits=normal(s * b, vocab) * 2, scores=-20 * torch.rand((s, b), generator=g, device="cuda"), keep=keep, end=2 if case["ends"] else None, ended=None,
                 ended_out=None, tokens=torch.zeros((s, keep), dtype=torch.int32, device="cuda"), parents=torch.zeros((s, keep), dtype=torch.int32, device="cuda"),
                 scores_out=torch.zeros((s, keep), device="cuda"))
    if case["ends"]:
        state.update(ended=torch.rand((s, b), generator=g, device="cuda") < 0.2, ended_out=torch.zeros((s, keep), dtype=torch.bool, device="cuda"))
    return state


def prepare_fork(case, seed, g, normal):
    page, beams, room = case["page"], case["beams"], case["room"]
    r = random.Random(seed)
    cached, count = lengths(case), case["seqs"] * beams
    rows, used = rows_of_pages(cached, [0] * count, beams, page)
    every = [n for n in cached for _ in range(beams)]
    wanted = count * (1 + -(-room // page))
    pages = used + (wanted // 3 if case["scarce"] else wanted)
    order = torch.randperm(pages, generator=g, device="cuda")
    columns = -(-(case["longest"] + room) // page) + 1
    refs = torch.zeros(pages, dtype=torch.int32)
    numbers = order.tolist()
    for row in rows:
        for p in row:
            refs[numbers[p]] += 1
    parents = []
    for s in range(case["seqs"]):   # children of the better beams; now and then a request has ended
        over = r.random() < 0.05 and case["seqs"] > 1
        parents += [-1 if over else s * beams + min(r.randrange(beams), r.randrange(beams)) for _ in range(beams)]
    caches = [normal(pages, page, case["kv_heads"], case["head_dim"]) for _ in range(2 * case["layers"])]
    return dict(table=table_of(rows, order, columns, -1), lengths=ints(every), refs=refs.cuda(), parents=ints(parents), page=page, room=room, caches=caches,
                table_out=torch.zeros((count, columns), dtype=torch.int32, device="cuda"), lengths_out=torch.zeros(count, dtype=torch.int32, device="cuda"),
                held_out=torch.zeros(count, dtype=torch.int32, device="cuda"), refs_out=torch.zeros(pages, dtype=torch.int32, device="cuda"),
                slots=torch.zeros((count, room), dtype=torch.int64, device="cuda"))


def prepare_compact(case, seed, g, normal):
    pages, rows = case["pages"], case["rows"]
    r = random.Random(case["ragged"])
    order = torch.randperm(pages, generator=g, device="cuda")
    live = r.randint(pages // 2, pages * 3 // 4)   # pages in use, some of them by several rows
    cuts = sorted(r.randrange(live + 1) for _ in range(rows - 1))
    held = [list(range(a, b)) for a, b in zip([0] + cuts, cuts + [live])]
    held = [held[i - 1][:len(held[i - 1]) // 2] + x if i % 3 == 2 else x for i, x in enumerate(held)]
    refs = torch.zeros(pages, dtype=torch.int32)
    numbers = order.tolist()
    for row in held:
        for p in row:
            refs[numbers[p]] += 1
    columns = max(1, max(len(x) for x in held))
    return dict(table=table_of(held, order, columns, -1), refs=refs.cuda(),
                caches=[normal(pages, case["page"], case["kv_heads"], case["head_dim"]) for _ in range(2 * case["layers"])],
                table_out=torch.zeros((rows, columns), dtype=torch.int32, device="cuda"), refs_out=torch.zeros(pages, dtype=torch.int32, device="cuda"),
                moved=torch.zeros(pages, dtype=torch.int32, device="cuda"), live=torch.zeros(1, dtype=torch.int32, device="cuda"))


def run(state):
    if own:
        return run_own(state)
    return {"fp4_cache_write": plain_write, "fp4_tree_attention": plain_attention, "beam_select": plain_beams, "fork_pages": plain_fork,
            "compact_pages": plain_compact}[state["op"]](state)


def run_own(s):
    import paper_2410_21120_amd as fi
    if s["op"] == "fp4_cache_write":
        fi.fp4_cache_write(s["k"], s["v"], s["slots"], s["k_codes"], s["k_scales"], s["v_codes"], s["v_scales"], k_held=s["k_held"], v_held=s["v_held"])
        return written(s)
    if s["op"] == "fp4_tree_attention":
        return fi.fp4_tree_attention(s["q"], s["k_codes"], s["k_scales"], s["v_codes"], s["v_scales"], s["table"], s["cached"], s["cu_nodes"], s["mask"], scale=s["scale"],
                                     max_nodes=s["most_nodes"], max_length=s["longest"], out=s["out"])
    if s["op"] == "beam_select":
        tokens, parents, scores, ended = fi.beam_select(s["logits"], s["scores"], keep=s["keep"], end=s["end"], ended=s["ended"], tokens_out=s["tokens"],
                                                        parents_out=s["parents"], scores_out=s["scores_out"], ended_out=s["ended_out"])
        return {"tokens": tokens, "parents": parents, "scores": scores, "ended": ended}
    if s["op"] == "fork_pages":
        table, lengths, held, refs, slots = fi.fork_pages(s["table"], s["lengths"], s["refs"], s["parents"], page_size=s["page"], room=s["room"], caches=s["caches"],
                                                          table_out=s["table_out"], lengths_out=s["lengths_out"], held_out=s["held_out"], refs_out=s["refs_out"],
                                                          slots_out=s["slots"])
        return {"table": table, "lengths": lengths, "held": held, "refs": refs, "slots": slots, "caches": s["caches"]}
    table, refs, moved, live = fi.compact_pages(s["table"], s["refs"], caches=s["caches"], table_out=s["table_out"], refs_out=s["refs_out"], moved_out=s["moved"],
                                                live_out=s["live"])
    return {"table": table, "refs": refs, "moved": moved, "live": live, "caches": s["caches"]}


def written(s):
    """What a write leaves.  Codes are two to a byte, so the bytes are returned: equal bytes are equal values; beside them, where asked, the values themselves."""
    return {"k_codes": s["k_codes"], "k_scales": s["k_scales"], "v_codes": s["v_codes"], "v_scales": s["v_scales"], "k_held": s["k_held"], "v_held": s["v_held"]}


def exponents(x):
    """x [..., blocks, 32] in 32 bits: the smallest e in [-125, 125] with |x| <= 6 * 2^e in the whole block (what is larger still is cut to that)."""
    part, power = torch.frexp(x.abs().amax(-1))   # amax = part * 2^power, part in [0.5, 1)
    return torch.where(part <= 0.75, power - 3, power - 2).clamp(-125, 125).where(part > 0, -125)


def encoded(x):
    """x [..., dim] in 32 bits: codes [..., dim / 2], the even value in the low half of a byte, and scales [..., blocks]."""
    dim = x.shape[-1]
    x = torch.nn.functional.pad(x, (0, -dim % BLOCK)).unflatten(-1, (-1, BLOCK))
    finite = torch.isfinite(x).all(-1)
    x = torch.where(finite[..., None], x, 0.0)
    e = exponents(x)
    y = torch.ldexp(x, -e[..., None])
    a = y.abs()
    # borders between 0, 0.5, 1, 1.5, 2, 3, 4 and 6; a value on one goes to the even code
    code = ((a > 0.25).int() + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5) + (a >= 3.5) + (a > 5.0)) + 8 * torch.signbit(x)
    code = code.flatten(-2)[..., :dim].to(torch.uint8)
    return code[..., 0::2] | code[..., 1::2] << 4, torch.where(finite, e + 127, 255).to(torch.uint8)


def decoded(codes, scales):
    """The values in 32 bits."""
    code = torch.stack([codes & 15, codes >> 4], -1).flatten(-2).int()
    value = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0, -0.0, -0.5, -1.0, -1.5, -2.0, -3.0, -4.0, -6.0], device=codes.device)[code]
    scale = torch.where(scales == 255, math.nan, torch.ldexp(torch.ones((), device=codes.device), scales.int() - 127))
    return value * scale.repeat_interleave(BLOCK, -1)[..., :value.shape[-1]]


def plain_write(s):
    page = s["k_codes"].shape[1]
    where = s["slots"] // page, s["slots"] % page
    k_codes, k_scales = encoded(s["k"].float())
    v_codes, v_scales = encoded(s["v"].float())
    s["k_codes"][where], s["k_scales"][where], s["v_codes"][where], s["v_scales"][where] = k_codes, k_scales, v_codes, v_scales
    if s["k_held"] is not None:
        s["k_held"].copy_(decoded(k_codes, k_scales))
        s["v_held"].copy_(decoded(v_codes, v_scales))
    return written(s)


def padded(cu, longest):
    """Row of every (sequence, place)."""
    place = torch.arange(longest, device=cu.device)
    return torch.where(place[None] < (cu[1:] - cu[:-1])[:, None], cu[:-1, None] + place[None], 0)


def owners(cu, rows):
    """Sequence and place in it of every packed row."""
    at = torch.arange(rows, device=cu.device)
    seq = (at[:, None] >= cu[None, 1:]).sum(1)
    return seq, at - cu[seq]


def plain_attention(s):
    hq, hk, d, page = s["q"].shape[1], s["k_codes"].shape[2], s["q"].shape[2], s["k_codes"].shape[1]
    rows = padded(s["cu_nodes"], s["most_nodes"])
    b, n = rows.shape
    q = s["q"].float()[rows].view(b, n, hk, hq // hk, d).permute(0, 2, 3, 1, 4).flatten(2, 3)
    j = torch.arange(s["longest"], device=rows.device)
    column = (j // page).clamp(max=s["table"].shape[1] - 1)
    where = s["table"][:, column].long(), (j % page)[None].expand(b, -1)
    k = decoded(s["k_codes"][where], s["k_scales"][where]).permute(0, 2, 1, 3)
    v = decoded(s["v_codes"][where], s["v_scales"][where]).permute(0, 2, 1, 3)
    node = j[None] - s["cached"][:, None]                      # which node of the tree a key is
    counts = (s["cu_nodes"][1:] - s["cu_nodes"][:-1])[:, None]
    if s["mask"] is None:
        sees = node[:, None] <= torch.arange(n, device=rows.device)[None, :, None]
    else:
        at = node.clamp(0, s["most_nodes"] - 1)
        sees = (torch.gather(s["mask"][rows], 2, (at // 64)[:, None].expand(-1, n, -1)) >> (at % 64)[:, None] & 1) == 1
    visible = (node < 0)[:, None] | ((node >= 0) & (node < counts))[:, None] & sees
    scores = torch.matmul(q, k.transpose(-1, -2)).view(b, hk, hq // hk, n, -1) * s["scale"]
    scores = torch.where(visible[:, None, None], scores, -math.inf)
    top = scores.amax(-1, keepdim=True)
    e = torch.exp(scores - torch.where(top == -math.inf, 0.0, top))
    total = e.sum(-1, keepdim=True)
    out = torch.matmul(e.flatten(2, 3), v).view(b, hk, hq // hk, n, d) / torch.where(total == 0, 1.0, total)
    seq, place = owners(s["cu_nodes"], s["q"].shape[0])
    return out.permute(0, 3, 1, 2, 4).flatten(2, 3)[seq, place].to(s["q"].dtype)


def plain_beams(s):
    seqs, beams = s["scores"].shape
    keep, vocab = s["keep"], s["logits"].shape[1]
    x = s["logits"].double()   # scores of different beams lie close
    top = x.amax(1, keepdim=True)
    log_sum = torch.log(torch.exp(x - top).sum(1, keepdim=True)) + top
    best, token = torch.sort(x, dim=1, descending=True, stable=True)
    best, token = best[:, :keep], token[:, :keep]
    total = s["scores"].double().view(-1, 1) + (best - log_sum)
    if s["ended"] is not None:   # a beam that has ended goes on as itself
        first = torch.arange(best.shape[1], device=x.device)[None] == 0
        total = torch.where(s["ended"].view(-1, 1), torch.where(first, s["scores"].double().view(-1, 1), -math.inf), total)
        token = torch.where(s["ended"].view(-1, 1), s["end"], token)
    total = torch.where(total > -math.inf, total, -math.inf).reshape(seqs, -1)   # (a candidate that is no number is none)
    total, at = torch.sort(total, dim=1, descending=True, stable=True)
    total, at = total[:, :keep], at[:, :keep]
    there = total > -math.inf
    tokens = torch.where(there, torch.gather(token.reshape(seqs, -1), 1, at), -1).int()
    parents = torch.where(there, at // best.shape[1] + beams * torch.arange(seqs, device=x.device)[:, None], -1).int()
    ended = None
    if s["end"] is not None:
        ended = there & ((tokens == s["end"]) | s["ended"].view(-1)[parents.clamp(min=0).long()])
    return {"tokens": tokens, "parents": parents, "scores": total.float(), "ended": ended}


def counted(pages, chosen, most):
    """How often each page is chosen."""
    return torch.zeros(most, dtype=torch.int32, device=pages.device).index_add_(0, pages.clamp(0, most - 1).flatten().long(), chosen.flatten().int())


def plain_fork(s):
    table, page, room, most = s["table"], s["page"], s["room"], s["refs"].shape[0]
    columns, alive = table.shape[1], s["parents"] >= 0
    parent = s["parents"].clamp(min=0).long()
    column = torch.arange(columns, device=table.device)[None]
    length = torch.where(alive, s["lengths"][parent], 0)
    before, after = (length + page - 1) // page, (length + room + page - 1) // page
    held = (s["lengths"] + page - 1) // page
    mine = table[parent]
    shared = column < before[:, None]
    refs = s["refs"] - counted(table, column < held[:, None], most) + counted(mine, shared, most)
    # the page that a row writes next: its own, or a copy for all but the last row that has it
    fits = alive & (after <= columns)
    last = torch.gather(mine, 1, (length // page).clamp(max=columns - 1)[:, None].long())[:, 0]
    part = fits & (length % page != 0) & (room > 0)
    same = (last[:, None] == last[None]) & part[:, None] & part[None]
    copy = part & (refs[last.clamp(min=0).long()] - same.tril(-1).sum(1) > 1)
    need = torch.where(fits, copy + after - before, 0)
    upto = need.cumsum(0)
    free = refs == 0
    made = fits & ((need == 0) | (upto <= free.sum()))
    pool = torch.cat([torch.argsort((~free).int(), stable=True).int(), torch.zeros(1, dtype=torch.int32, device=table.device)])   # free pages, the lowest first
    copy = copy & made
    fresh = (column >= before[:, None]) & (column < after[:, None]) & made[:, None]
    at = (upto - need)[:, None] + torch.where(fresh, copy[:, None] + column - before[:, None], 0)
    given = pool[at.clamp(max=most).long()]
    new = torch.where(shared, mine, torch.where(fresh, given, -1))
    target = pool[(upto - need).clamp(max=most).long()]
    new = torch.where(copy[:, None] & (column == (length // page)[:, None]), target[:, None], new)
    refs = refs - counted(last, copy, most) + counted(target, copy, most) + counted(given, fresh, most)
    place = length[:, None] + torch.arange(room, device=table.device)[None]
    slots = torch.where(made[:, None], torch.gather(new, 1, (place // page).clamp(max=columns - 1).long()).long() * page + place % page, -1)
    # pages are copied by all rows at once: a row without a copy to make repeats that of the first row that has one
    one = torch.argmax(copy.int())
    source = torch.where(copy, last, torch.where(copy.any(), last[one], 0)).long()
    target = torch.where(copy, target, torch.where(copy.any(), target[one], 0)).long()
    caches = [cache.index_copy_(0, target, cache[source]) for cache in s["caches"]]
    return {"table": new.int(), "lengths": length.int(), "held": torch.where(made, length + room, length).int(), "refs": refs.int(), "slots": slots, "caches": caches}


def plain_compact(s):
    table, refs, pages = s["table"], s["refs"], s["refs"].shape[0]
    number = torch.arange(pages, device=refs.device)
    used = refs > 0
    live = used.sum()
    hole, mover = ~used & (number < live), used & (number >= live)
    holes = torch.zeros(pages + 1, dtype=torch.int64, device=refs.device).scatter_(0, torch.where(hole, hole.cumsum(0) - 1, pages), number)
    moved = torch.where(used, torch.where(mover, holes[(mover.cumsum(0) - 1).clamp(min=0)], number), -1)
    source = torch.cat([number, number[:1]]).scatter_(0, torch.where(mover, moved, pages), number)[:pages]
    caches = [cache.copy_(cache[source]) for cache in s["caches"]]
    there = (table >= 0) & (table < pages)
    entry = moved[table.clamp(0, pages - 1).long()]
    return {"table": torch.where(there & (entry >= 0), entry, table).int(), "refs": torch.where(number < live, refs[source], 0).int(), "moved": moved.int(),
            "live": live.int().view(1), "caches": caches}


def exact(case, seed):
    """The operators' definitions in 64 bits, or one row after the other where they count and move."""
    s = prepare(case, seed)
    return {"fp4_cache_write": exact_write, "fp4_tree_attention": exact_attention, "beam_select": exact_beams, "fork_pages": exact_fork,
            "compact_pages": exact_compact}[case["op"]](s)


MAGNITUDES = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def exact_blocks(x):
    """Nearest representable values of a block each, found by distance: codes, scales and values."""
    dim = x.shape[-1]
    x = torch.cat([x.double(), x.new_zeros((*x.shape[:-1], -dim % BLOCK)).double()], -1).unflatten(-1, (-1, BLOCK))
    e = torch.full(x.shape[:-1], -125.0, dtype=torch.float64, device=x.device)
    largest = x.abs().amax(-1)
    for power in range(-125, 125):
        e += (largest > 6.0 * 2.0 ** power).double()
    unit = torch.exp2(e)[..., None]
    best, code = torch.full_like(x, math.inf), torch.zeros_like(x, dtype=torch.uint8)
    for c in (0, 2, 4, 6, 1, 3, 5, 7):   # even codes first: they keep what is as near
        far = (x.abs() - MAGNITUDES[c] * unit).abs()
        code = torch.where(far < best, c, code)
        best = torch.minimum(best, far)
    value = torch.tensor(MAGNITUDES, dtype=torch.float64, device=x.device)[code.long()] * unit * torch.where(torch.signbit(x), -1.0, 1.0)
    code = (code + 8 * torch.signbit(x)).flatten(-2)[..., :dim].to(torch.uint8)
    return code[..., 0::2] + 16 * code[..., 1::2], (e + 127).to(torch.uint8), value.flatten(-2)[..., :dim]


def exact_write(s):
    out = {}
    page = s["k_codes"].shape[1]
    for x in ("k", "v"):
        codes, scales, value = exact_blocks(s[x])
        out[x + "_codes"], out[x + "_scales"] = s[x + "_codes"].clone(), s[x + "_scales"].clone()
        out[x + "_codes"][s["slots"] // page, s["slots"] % page] = codes
        out[x + "_scales"][s["slots"] // page, s["slots"] % page] = scales
        out[x + "_held"] = value if s[x + "_held"] is not None else None
    return out


def exact_values(codes, scales):
    value = torch.tensor(MAGNITUDES + tuple(-m for m in MAGNITUDES), dtype=torch.float64, device=codes.device)
    out = torch.empty((*codes.shape[:-1], 2 * codes.shape[-1]), dtype=torch.float64, device=codes.device)
    out[..., 0::2], out[..., 1::2] = value[(codes % 16).long()], value[(codes // 16).long()]
    unit = torch.pow(2.0, scales.double() - 127)
    for b in range(scales.shape[-1]):
        out[..., BLOCK * b:BLOCK * (b + 1)] *= unit[..., b:b + 1]
    return out


def exact_attention(s):
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    group, page, cu = s["q"].shape[1] // s["k_codes"].shape[2], s["k_codes"].shape[1], s["cu_nodes"].tolist()
    for b, before in enumerate(s["cached"].tolist()):
        n = cu[b + 1] - cu[b]
        places = s["table"][b, :(before + n + page - 1) // page].long()
        k, v = (exact_values(s[x + "_codes"][places].flatten(0, 1)[:before + n], s[x + "_scales"][places].flatten(0, 1)[:before + n]) for x in ("k", "v"))
        seen = torch.ones((n, before + n), dtype=torch.bool, device="cuda")
        for j in range(n):
            if s["mask"] is None:
                seen[:j, before + j] = False
            else:
                seen[:, before + j] = (s["mask"][cu[b]:cu[b + 1], j // 64] >> (j % 64)) % 2 != 0
        for h in range(s["q"].shape[1]):
            scores = (s["q"][cu[b]:cu[b + 1], h].double() @ k[:, h // group].t() * s["scale"]).masked_fill(~seen, -math.inf)
            out[cu[b]:cu[b + 1], h] = torch.softmax(scores, 1) @ v[:, h // group]
    return out


def exact_beams(s):
    seqs, beams = s["scores"].shape
    keep, vocab = s["keep"], s["logits"].shape[1]
    tokens, parents, ended = ([[-1] * keep for _ in range(seqs)] for _ in range(3))
    scores = torch.full((seqs, keep), -math.inf, dtype=torch.float64, device="cuda")
    for b in range(seqs):
        total = s["logits"][b * beams:(b + 1) * beams].double()
        total = s["scores"][b].double()[:, None] + (total - torch.logsumexp(total, 1, keepdim=True))
        if s["ended"] is not None:
            total[s["ended"][b]] = -math.inf
            total[:, s["end"]] = torch.where(s["ended"][b], s["scores"][b].double(), total[:, s["end"]])
        total = total.flatten()
        border = torch.topk(total, min(keep, beams * vocab)).values[-1]
        at = torch.nonzero(total >= border)[:, 0]   # those on the border, too, by their index
        for i, (x, place) in enumerate(sorted(zip(total[at].tolist(), at.tolist()), key=lambda c: (-c[0], c[1]))):
            if i < keep and x > -math.inf:
                tokens[b][i], parents[b][i], scores[b, i] = place % vocab, b * beams + place // vocab, x
    parents, tokens = ints(parents), ints(tokens)
    if s["end"] is not None:
        ended = (tokens >= 0) & ((tokens == s["end"]) | s["ended"].flatten()[parents.clamp(min=0).long()])
    return {"tokens": tokens, "parents": parents, "scores": scores, "ended": ended if s["end"] is not None else None}


def exact_fork(s):
    table, page, room, columns = s["table"].tolist(), s["page"], s["room"], s["table"].shape[1]
    refs, lengths, parents = s["refs"].tolist(), s["lengths"].tolist(), s["parents"].tolist()
    caches = [c.clone() for c in s["caches"]]
    need = lambda n: -(-n // page)   # noqa: E731
    for row, n in zip(table, lengths):
        for p in row[:need(n)]:
            refs[p] -= 1
    new, length = [], []
    for p in parents:
        n = lengths[p] if p >= 0 else 0
        row = table[p][:need(n)] if p >= 0 else []
        for x in row:
            refs[x] += 1
        new.append(row)
        length.append(n)
    free = [p for p, n in enumerate(refs) if n == 0]
    held, slots, taken, have = list(length), [[-1] * room for _ in parents], 0, dict(enumerate(refs))
    for i, (p, n) in enumerate(zip(parents, length)):
        if p < 0 or need(n + room) > columns:
            continue
        copy = room > 0 and n % page != 0 and have[new[i][-1]] > 1
        if copy:
            have[new[i][-1]] -= 1
        wanted = copy + need(n + room) - need(n)
        taken += wanted
        if wanted and taken > len(free):
            continue
        mine = free[taken - wanted:taken]
        for x in mine:
            refs[x] = 1
        if copy:
            refs[new[i][-1]] -= 1
            for c in caches:
                c[mine[0]] = c[new[i][-1]]
            new[i][-1] = mine.pop(0)
        new[i] = new[i] + mine
        held[i] = n + room
        slots[i] = [new[i][t // page] * page + t % page for t in range(n, n + room)]
    return {"table": ints([row + [-1] * (columns - len(row)) for row in new]), "lengths": ints(length), "held": ints(held), "refs": ints(refs),
            "slots": torch.tensor(slots, dtype=torch.int64, device="cuda").view(len(parents), room), "caches": caches}


def exact_compact(s):
    refs, table = s["refs"].tolist(), s["table"].tolist()
    caches = [c.clone() for c in s["caches"]]
    live = sum(n > 0 for n in refs)
    moved = [p if n > 0 else -1 for p, n in enumerate(refs)]
    to = 0
    for p in range(live, len(refs)):
        if refs[p] > 0:
            while refs[to] > 0:
                to += 1
            for c in caches:
                c[to] = c[p]
            moved[p], refs[to], refs[p] = to, refs[p], 0
    return {"table": ints([[moved[p] if p >= 0 else p for p in row] for row in table]), "refs": ints(refs), "moved": ints(moved), "live": ints([live]), "caches": caches}


def work(case):
    """Inputs in once, outputs out once; two operations per multiply-add.  Shared pages count once, pages that move in and out.  What moves hangs on the
    state, so the expected share of it is taken."""
    size = 4 if case.get("dtype") == "f32" else 2
    if case["op"] == "beam_select":
        n = case["seqs"] * case["beams"] * case["vocab"]
        return {"bytes": n * size + case["seqs"] * (5 * case["beams"] + 13 * case["keep"]), "flops": 3 * n}
    hk, d, page = case["kv_heads"], case["head_dim"], case["page"]
    if case["op"] == "fp4_cache_write":
        values = 2 * case["tokens"] * hk
        return {"bytes": values * (d * size * (2 if case["held"] else 1) + d // 2 + blocks(d)) + 8 * case["tokens"], "flops": 3 * values * d}
    if case["op"] == "fp4_tree_attention":
        cached, nodes, beams = lengths(case), drafted(case), case["beams"]
        _, used = rows_of_pages(cached, nodes, beams, 1)
        every = [n for n in cached for _ in range(beams)]
        return {"bytes": 2 * hk * (d // 2 + blocks(d)) * used + 2 * d * size * case["q_heads"] * sum(nodes),
                "flops": 4 * d * case["q_heads"] * sum(n * (c + 1) for c, n in zip(every, nodes))}
    page_bytes = page * hk * d * 2 * 2 * case["layers"]
    if case["op"] == "fork_pages":
        beams, rows = case["beams"], case["seqs"] * case["beams"]
        columns = -(-(case["longest"] + case["room"]) // page) + 1
        # a beam's children, less the one that keeps its page: rows without those that distinct parents are expected to keep (children of the better of two draws)
        kept = sum(1 - (1 - (2 * (beams - b) - 1) / beams ** 2) ** beams for b in range(beams))
        copies = case["seqs"] * (beams - kept) if case["room"] and page > 1 else 0
        if case["scarce"]:
            copies /= 3
        return {"bytes": int(2 * copies * page_bytes + 8 * rows * columns + 8 * rows * case["room"] + 16 * rows), "flops": rows * columns}
    live = case["pages"] * 5 / 8   # between a half and three quarters, spread evenly over the pool
    return {"bytes": int(2 * live * (1 - live / case["pages"]) * page_bytes + 12 * case["pages"]), "flops": case["pages"]}
