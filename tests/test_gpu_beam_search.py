"""Beam search over a 4-bit cache, all of its operators together: selection, forks, writes and attention, step by step against their definitions on the history that every beam has
on the host; the same steps on a stream of their own and replayed as a graph."""
import math

import pytest

from tests import fp4_oracle as oracle
from tests.test_gpu_fp4_cache import _ref
from tests.test_gpu_operators import _inside, fi, torch  # noqa: F401

pytestmark = pytest.mark.gpu

SEQS, BEAMS, PAGE, PAGES, COLUMNS, HQ, HK, D, VOCAB, END = 3, 4, 8, 90, 9, 8, 2, 64, 1200, 7


def _model(torch, dtype):  # noqa: F811
    g = torch.Generator().manual_seed(61)
    kind = torch.bfloat16 if dtype == "bf16" else torch.float32
    m = dict(q=torch.randn((VOCAB, HQ, D), generator=g).to(kind), k=torch.randn((VOCAB, HK, D), generator=g).to(kind), v=torch.randn((VOCAB, HK, D), generator=g).to(kind),
             out=0.15 * torch.randn((HQ * D, VOCAB), generator=g))
    m["out"][:, END] += 0.02
    return {n: t.cuda() for n, t in m.items()}


def _state(torch):  # noqa: F811
    rows, i32 = SEQS * BEAMS, dict(dtype=torch.int32, device="cuda")
    return dict(table=torch.full((rows, COLUMNS), -1, **i32), lengths=torch.zeros(rows, **i32), held=torch.zeros(rows, **i32), refs=torch.zeros(PAGES, **i32),
                slots=torch.zeros((rows, 1), dtype=torch.int64, device="cuda"), tokens=torch.zeros((SEQS, BEAMS), **i32), parents=torch.zeros((SEQS, BEAMS), **i32),
                scores=torch.zeros((SEQS, BEAMS), device="cuda"), ended=torch.zeros((SEQS, BEAMS), dtype=torch.bool, device="cuda"))


def _begin(torch, fi, m, dtype):  # noqa: F811
    """Prompts of different lengths in the cache of the first beam each, then shared by all; the last prompt token's attention."""
    g = torch.Generator().manual_seed(62)
    prompts = [torch.randint(0, VOCAB, (n,), generator=g) for n in (11, 16, 1)]
    run = dict(caches=[*fi.fp4_cache(PAGES, PAGE, HK, D), *fi.fp4_cache(PAGES, PAGE, HK, D)], cu=torch.arange(SEQS * BEAMS + 1, dtype=torch.int32, device="cuda"))
    table, lengths, refs = torch.full((SEQS, COLUMNS), -1, dtype=torch.int32).cuda(), torch.zeros(SEQS, dtype=torch.int32).cuda(), torch.zeros(PAGES, dtype=torch.int32).cuda()
    most = max(len(p) for p in prompts)
    table, lengths, held, refs, slots = fi.fork_pages(table, lengths, refs, page_size=PAGE, room=most)
    for i, p in enumerate(prompts):
        t = p.cuda()
        fi.fp4_cache_write(m["k"][t], m["v"][t], slots[i, :len(p)].contiguous(), *run["caches"])
    lengths = torch.tensor([len(p) for p in prompts], dtype=torch.int32).cuda()
    a = _state(torch)
    parents = torch.arange(SEQS, dtype=torch.int32).repeat_interleave(BEAMS).cuda()
    a["table"], a["lengths"], a["held"], a["refs"], _ = fi.fork_pages(table, lengths, refs, parents, page_size=PAGE, held=held)
    assert torch.equal(a["held"], a["lengths"])
    a["scores"][:, 1:] = -math.inf   # all beams hold the same
    last = torch.stack([p[-1] for p in prompts]).repeat_interleave(BEAMS).cuda()
    run["attended"] = fi.fp4_tree_attention(m["q"][last], *run["caches"], a["table"], a["lengths"] - 1, run["cu"])
    run["workspace"] = torch.zeros(1 << 20, dtype=torch.uint8, device="cuda")
    return prompts, run, a, _state(torch)


def _step(torch, fi, m, run, old, new, stream=None):  # noqa: F811
    """From `old` to `new`, nothing on the host."""
    run["logits"] = logits = run["attended"].flatten(1).float() @ m["out"]
    fi.beam_select(logits, old["scores"], end=END, ended=old["ended"], tokens_out=new["tokens"], parents_out=new["parents"], scores_out=new["scores"], ended_out=new["ended"],
                   workspace=run["workspace"], stream=stream)
    fi.fork_pages(old["table"], old["lengths"], old["refs"], new["parents"].view(-1), page_size=PAGE, held=old["held"], room=1, caches=run["caches"], table_out=new["table"],
                  lengths_out=new["lengths"], held_out=new["held"], refs_out=new["refs"], slots_out=new["slots"], workspace=run["workspace"], stream=stream)
    at = new["tokens"].view(-1).clamp(min=0).long()
    fi.fp4_cache_write(m["k"][at], m["v"][at], new["slots"].view(-1), *run["caches"], stream=stream)
    fi.fp4_tree_attention(m["q"][at], *run["caches"], new["table"], new["lengths"], run["cu"], max_nodes=1, max_length=PAGE * COLUMNS, out=run["attended"],
                          workspace=run["workspace"], stream=stream)
    new["lengths"].copy_(new["held"])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_search(torch, fi, dtype):  # noqa: F811
    m = _model(torch, dtype)
    prompts, run, old, new = _begin(torch, fi, m, dtype)
    history = [p.tolist() for p in prompts for _ in range(BEAMS)]
    held = {n: oracle.write(m[n])[2] for n in ("k", "v")}
    dense = lambda h: torch.stack([held["k"][h], held["v"][h]])   # noqa: E731
    q = m["q"].cpu()
    for step in range(40):
        before = run["attended"].clone()
        rows = [i for i in range(SEQS * BEAMS) if history[i]]
        want, bound = _ref(torch, q[[history[i][-1] for i in rows]], [dense(history[i]) for i in rows], [len(history[i]) - 1 for i in rows], [1] * len(rows), None, D ** -0.5, dtype)
        _inside(before[rows].double().cpu(), want, bound)
        caches = [c.cpu().contiguous() for c in run["caches"]]
        if step == 15:   # the model hardly ever ends by itself: two beams are told to
            old["ended"][0, 0] = old["ended"][2, 1] = True
        _step(torch, fi, m, run, old, new)
        tokens, parents, scores, ended = oracle.select(run["logits"], old["scores"], BEAMS, END, old["ended"].cpu())
        assert torch.equal(new["tokens"].cpu(), tokens) and torch.equal(new["parents"].cpu(), parents) and torch.equal(new["ended"].cpu(), ended), step
        table, lengths, rest, refs, slots = oracle.fork(old["table"].cpu(), old["lengths"].cpu(), old["refs"].cpu(), parents.view(-1), PAGE, old["held"].cpu(), 1, caches)
        assert torch.equal(new["table"].cpu(), table) and torch.equal(new["held"].cpu(), rest) and torch.equal(new["refs"].cpu(), refs) and torch.equal(new["slots"].cpu(), slots), step
        assert len(set(slots[slots >= 0].tolist())) == int((slots >= 0).sum())   # no two rows write one place
        history = [history[p] + [t] if p >= 0 else [] for p, t in zip(parents.view(-1).tolist(), tokens.view(-1).tolist())]
        assert [len(h) for h in history] == new["lengths"].tolist()
        if step % 10 == 9:   # the pool is tidied up in between
            new["table"], new["refs"], _, live = fi.compact_pages(new["table"], new["refs"], caches=run["caches"])
            assert not new["refs"][live.item():].any() and (new["refs"][:live.item()] > 0).all()
        old, new = new, old
        assert old["scores"].isfinite().all()
    assert old["ended"].any() and max(len(h) for h in history) > PAGE * 5


@pytest.mark.parametrize("way", ["stream", "graph"])
def test_search_on_a_stream_and_as_a_graph(torch, fi, way):  # noqa: F811
    """Forty steps give the bits that they give step by step; a graph holds two of them, there and back, and eager work lies between its replays."""
    m = _model(torch, "bf16")
    seen = []
    for mode in ("eager", way):
        _, run, a, b = _begin(torch, fi, m, "bf16")
        trace, stream = [], torch.cuda.Stream()
        if mode == "graph":
            start = {n: t.clone() for n, t in a.items()}, run["attended"].clone(), [c.clone() for c in run["caches"]]
            stream.wait_stream(torch.cuda.current_stream())
            graph = torch.cuda.CUDAGraph()
            _step(torch, fi, m, run, a, b)   # (libraries' first calls)
            torch.cuda.synchronize()
            with torch.cuda.graph(graph, stream=stream):
                _step(torch, fi, m, run, a, b)
                _step(torch, fi, m, run, b, a)
            for n, t in start[0].items():
                a[n].copy_(t)
            run["attended"].copy_(start[1])
            for c, t in zip(run["caches"], start[2]):
                c.copy_(t)
        for turn in range(20):
            if mode == "graph":
                graph.replay()
                torch.cuda.synchronize()
                m["out"] @ m["out"].t()
            elif mode == "stream":
                stream.wait_stream(torch.cuda.current_stream())
                with torch.cuda.stream(stream):
                    _step(torch, fi, m, run, a, b, stream.cuda_stream)
                    _step(torch, fi, m, run, b, a, stream.cuda_stream)
                torch.cuda.current_stream().wait_stream(stream)
            else:
                _step(torch, fi, m, run, a, b)
                _step(torch, fi, m, run, b, a)
            trace.append([t.clone() for t in (*a.values(), run["attended"])])
        seen.append(trace)
    for turn, (x, y) in enumerate(zip(*seen)):
        assert all(torch.equal(p.nan_to_num(), q.nan_to_num()) if p.is_floating_point() else torch.equal(p, q) for p, q in zip(x, y)), turn
