"""What the operators of a 4-bit cache leave to each other: prompts attend to what the cache holds, as later steps will; forks and compactions carry codes and scales."""
import pytest

from tests import fp4_oracle as oracle
from tests.test_gpu_fp4_cache import _held, _ref
from tests.test_gpu_operators import _cu, _inside, _kind, _rows, fi, torch  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("counts,page,hq,hk,d", [([37, 5, 130, 1], 16, 8, 2, 64), ([300], 64, 32, 8, 128), ([64, 33, 2], 5, 4, 4, 72), ([17, 90], 16, 4, 1, 256), ([700, 20], 16, 8, 2, 128)])
def test_a_prompt_sees_what_later_steps_see(torch, fi, dtype, counts, page, hq, hk, d):  # noqa: F811
    """prompt_attention over k_held and v_held, a chain of the prompt's tokens over the cache, and its last tokens as steps of one token: all within their bounds of the definition over
    the values that the cache holds, and those are the same bits."""
    g, kind, tokens = torch.Generator().manual_seed(71), _kind(torch, dtype), sum(counts)
    q, k, v = (_rows(torch, g, (tokens, h, d), kind, "plain") for h in (hq, hk, hk))
    need = [-(-n // page) for n in counts]
    pages, table, at = sum(need) + 2, torch.zeros((len(counts), max(need)), dtype=torch.int32), 0
    order = torch.randperm(pages, generator=g)
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n].int()
        at += n
    place = [torch.arange(n) for n in counts]
    slots = torch.cat([table[b, p // page].long() * page + p % page for b, p in enumerate(place)]).cuda()
    halves = [fi.fp4_cache(pages, page, hk, d) for _ in range(2)]
    held = [torch.empty_like(k), torch.empty_like(v)]
    fi.fp4_cache_write(k, v, slots, *halves[0], *halves[1], k_held=held[0], v_held=held[1])
    dense, at = [], 0
    for b, (n, p) in enumerate(zip(counts, place)):
        where = (table[b, p // page].long().cuda(), (p % page).cuda())
        dense.append(torch.stack([oracle.read(codes[where], scales[where]) for codes, scales in halves]))
        assert all(torch.equal(x[at:at + n].double().cpu(), y) for x, y in zip(held, dense[b]))
        at += n
    want, bound = _ref(torch, q, dense, [0] * len(counts), counts, None, d ** -0.5, dtype)
    cu, none = _cu(torch, counts), torch.zeros(len(counts), dtype=torch.int32).cuda()
    _inside(fi.prompt_attention(q, *held, cu).double().cpu(), want, bound)
    _inside(fi.fp4_tree_attention(q, *halves[0], *halves[1], table.cuda(), none, cu, max_nodes=max(counts), max_length=max(counts)).double().cpu(), want, bound)
    last = cu[1:].long() - 1
    steps = fi.fp4_tree_attention(q[last], *halves[0], *halves[1], table.cuda(), torch.tensor(counts, dtype=torch.int32).cuda() - 1, _cu(torch, [1] * len(counts)), max_nodes=1,
                                  max_length=max(counts))
    _inside(steps.double().cpu(), want[last.cpu()], bound[last.cpu()])


POOLS = [(16, 8, 128, "head"), (16, 2, 72, "head"), (1, 4, 64, "head"), (5, 3, 40, "token"), (64, 2, 256, "head"), (16, 2, 96, "wide")]


@pytest.mark.parametrize("page,hk,d,order", POOLS)
def test_compaction_of_a_4_bit_cache(torch, fi, page, hk, d, order):  # noqa: F811
    """Codes and scales move with their pages, so attention over the renumbered table gives the same bits."""
    g, cached, counts = torch.Generator().manual_seed(72), [70, 0, 333, 16], [2, 1, 3, 1]
    (k, v), table, _ = _held(torch, g, cached, counts, page, hk, d, order, spare=40)
    need = [-(-(c + n) // page) for c, n in zip(cached, counts)]
    if order == "wide":   # (pages with gaps are refused: those of a cache that has none, and what lies between its pages stays)
        with pytest.raises(ValueError, match="gaps"):
            fi.compact_pages(table, torch.zeros(k[0].shape[0], dtype=torch.int32).cuda(), caches=[k[0]])
        apart = [torch.full((x.shape[0], 2, *x.shape[1:]), 77, dtype=torch.uint8).cuda() for x in (*k, *v)]
        for x, y in zip((*k, *v), apart):
            y[:, 1] = x
        k, v = (apart[0][:, 1], apart[1][:, 1]), (apart[2][:, 1], apart[3][:, 1])
    refs = torch.zeros(k[0].shape[0], dtype=torch.int32)
    for b, n in enumerate(need):
        refs[table[b, :n].cpu().long()] += 1
    q, lengths, cu = _rows(torch, g, (sum(counts), 2 * hk, d), torch.bfloat16, "plain"), torch.tensor(cached, dtype=torch.int32).cuda(), _cu(torch, counts)
    before = fi.fp4_tree_attention(q, *k, *v, table, lengths, cu)
    assert before.isfinite().all()
    table, after, moved, live = fi.compact_pages(table, refs.cuda(), caches=[*k, *v])
    assert live.item() == sum(need) and bool((moved[refs.cuda() > 0] != torch.nonzero(refs.cuda() > 0)[:, 0]).any()) and bool((after[:live.item()] == 1).all())
    assert all(int(table[b, :n].max()) < live.item() for b, n in enumerate(need))
    assert torch.equal(fi.fp4_tree_attention(q, *k, *v, table, lengths, cu), before)
    if order == "wide":
        assert all(bool((x[:, 0] == 77).all()) for x in apart)


@pytest.mark.parametrize("page,hk,d,order", POOLS[:5])
def test_forks_of_a_4_bit_cache(torch, fi, page, hk, d, order):  # noqa: F811
    """Every row holds its parent's tokens, and what it writes next to them, and no other row sees that."""
    g, cached, room = torch.Generator().manual_seed(73), [37, 5, 70], 2
    halves, table, _ = _held(torch, g, cached, [0] * 3, page, hk, d, order, spare=30 + -(-24 // page))
    caches = [*halves[0], *halves[1]]
    columns = max(-(-(n + 3 * room) // page) for n in cached)
    wide = torch.full((3, columns), -1, dtype=torch.int32)
    refs, lengths = torch.zeros(caches[0].shape[0], dtype=torch.int32), torch.tensor(cached, dtype=torch.int32)
    for b, n in enumerate(cached):
        wide[b, :-(-n // page)] = table[b, :-(-n // page)].cpu()
        refs[wide[b][wide[b] >= 0].long()] += 1

    def holds(table, b, n):   # codes and scales of a row's tokens
        p = torch.arange(n)
        where = (table[b].cpu()[p // page].long().cuda(), (p % page).cuda())
        return [c[where] for c in caches]
    state = [wide.cuda(), lengths.cuda(), lengths.cuda(), refs.cuda()]
    truth = [holds(wide, b, n) for b, n in enumerate(cached)]
    for parents in ([0, 0, 1, 2, 2, 0], [5, 1, 1, 3, 4, 2, 0]):
        got = fi.fork_pages(state[0], state[1], state[3], torch.tensor(parents, dtype=torch.int32).cuda(), page_size=page, held=state[2], room=room, caches=caches)
        assert bool((got[4] >= 0).all())
        truth = [truth[p] for p in parents]
        x = torch.randn((len(parents) * room, 2 * hk, d), generator=g).bfloat16()
        fi.fp4_cache_write(x[:, :hk].cuda(), x[:, hk:].cuda(), got[4].view(-1), *caches)
        written = [t.view(len(parents), room, *t.shape[1:]).cuda() for half in (x[:, :hk], x[:, hk:]) for t in oracle.write(half)[:2]]
        truth = [[torch.cat([old, new[b]]) for old, new in zip(row, written)] for b, row in enumerate(truth)]
        for b, row in enumerate(truth):
            assert all(torch.equal(x, y) for x, y in zip(holds(got[0], b, len(row[0])), row)), (parents, b)
        state = [got[0], got[2], got[2], got[3]]
