"""Selection over beams and vocabulary, forks and compaction of pages, against their definitions one after the other (fp4_oracle.py).

Tokens, beams, pages and counts are equal; a score is one rounding of a sum in 64 bits whose log-sum comes from fp32 terms: each exp2 has a few u and
its argument one rounding of at most 64 u for what counts, sums of up to 2^11 terms a lane add (2^11 + 8) u at most: bound 2^11 * 1.1 u + 80 u absolutely, and u |score|."""
import math

import pytest

from tests import fp4_oracle as oracle
from tests.test_gpu_operators import U, _kind, fi, torch  # noqa: F401

pytestmark = pytest.mark.gpu

LOG_SUM = (2 ** 11 * 1.1 + 80) * U


def _same(got, want, end=None):
    import torch
    tokens, parents, scores, ended = got
    assert torch.equal(tokens.cpu(), want[0]) and torch.equal(parents.cpu(), want[1])
    s, w = scores.double().cpu(), want[2]
    fine = w.isfinite()
    assert torch.equal(s[~fine], w[~fine])
    assert ((s - w).abs() <= LOG_SUM + 1.01 * U * w.abs())[fine].all()
    assert ended is None if end is None else torch.equal(ended.cpu(), want[3])


SELECTIONS = [
    # sequences, beams, keep, vocabulary, gap behind a row, end
    (1, 1, 1, 1, 0, None), (1, 4, 4, 32000, 0, None), (3, 5, 10, 777, 3, 5), (2, 1, 64, 50, 0, 0), (7, 3, 2, 2047, 1, None), (1, 64, 64, 4099, 0, 17), (2, 2, 64, 131071, 0, None),
    (5, 8, 16, 20000, 8, 19999), (1, 2, 3, 300000, 5, None), (40, 4, 8, 513, 0, 1), (2, 64, 1, 100, 0, None), (64, 8, 8, 8193, 0, None), (2, 16, 32, 130001, 0, None),
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("seqs,beams,keep,vocab,gap,end", SELECTIONS)
def test_selection(torch, fi, dtype, seqs, beams, keep, vocab, gap, end):  # noqa: F811
    g, kind = torch.Generator().manual_seed(31), _kind(torch, dtype)
    wide = torch.full((seqs * beams, vocab + gap), math.nan, dtype=kind)
    wide[:, :vocab] = (3 * torch.randn((seqs * beams, vocab), generator=g)).to(kind)
    logits, scores = wide[:, :vocab], -10 * torch.rand((seqs, beams), generator=g)
    ended = None if end is None else torch.rand((seqs, beams), generator=g) < 0.3
    got = fi.beam_select(wide.cuda()[:, :vocab], scores.cuda(), keep=keep, end=end, ended=None if ended is None else ended.cuda())
    _same(got, oracle.select(logits, scores, keep, end, ended), end)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("vocab", [37, 5000, 40001])
def test_selection_of_equal_logits(torch, fi, dtype, vocab):  # noqa: F811
    """Ties go to the first beam, and in it to the first token: all logits alike, a few values only, zeros of both signs."""
    g, kind = torch.Generator().manual_seed(32), _kind(torch, dtype)
    for logits in (torch.zeros((6, vocab)), torch.randint(0, 3, (6, vocab), generator=g).float(), torch.where(torch.rand((6, vocab), generator=g) < 0.5, 0.0, -0.0)):
        logits = logits.to(kind)
        logits[3:] = logits[:1]   # rows whose sums are alike to the last bit
        scores = torch.zeros((2, 3))
        for keep in (1, 7, 64):
            _same(fi.beam_select(logits.cuda(), scores.cuda(), keep=keep), oracle.select(logits, scores, keep))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_selection_of_rising_falling_and_masked_logits(torch, fi, dtype):  # noqa: F811
    """Every value beats all before it; none does; most of the vocabulary is masked, by minus infinity or the type's lowest value, whole stretches of it too."""
    kind, vocab = _kind(torch, dtype), 30011
    rise = torch.linspace(-20, 20, vocab).to(kind)
    lowest = torch.finfo(kind).min
    rows = [rise, rise.flip(0), rise.clone(), rise.clone(), rise.clone(), torch.full((vocab,), lowest, dtype=kind)]
    rows[2][100:29000] = -math.inf
    rows[3][5000:] = lowest
    rows[4][:] = -math.inf
    rows[4][12345] = 3.0
    logits, scores = torch.stack(rows), torch.tensor([[-1.0, -2.0, -3.0], [-0.5, -1.5, -9.0]])
    for keep in (1, 6, 64):
        _same(fi.beam_select(logits.cuda(), scores.cuda(), keep=keep), oracle.select(logits, scores, keep))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_selection_without_enough_continuations(torch, fi, dtype):  # noqa: F811
    """Dead beams, rows of NaN, infinity or minus infinity, ended beams, fewer tokens than places."""
    kind, g = _kind(torch, dtype), torch.Generator().manual_seed(33)
    logits = torch.randn((12, 9), generator=g).to(kind)
    logits[1, 4], logits[2, 0], logits[3], logits[4, :7] = math.nan, math.inf, -math.inf, -math.inf
    logits[8] = math.nan   # an ended beam's: not looked at
    scores = torch.tensor([[-1.0, -2.0, -3.0], [-4.0, -1.0, -math.inf], [-1.0, math.nan, -math.inf], [-math.inf] * 3])
    ended = torch.zeros((4, 3), dtype=torch.bool)
    ended[2, 2] = ended[3, 1] = True   # ended, and dead
    scores[2, 2] = -0.25
    for keep in (3, 20, 64):
        got = fi.beam_select(logits.cuda(), scores.cuda(), keep=keep, end=8, ended=ended.cuda())
        want = oracle.select(logits, scores, keep, 8, ended)
        _same(got, want, 8)
        assert (got[0][3] == -1).all() and (got[1][3] == -1).all() and (got[2][3] == -math.inf).all() and not got[3][3].any()
    assert want[0][2, 0] == 8 and want[3][2, 0]
    none = fi.beam_select(logits[:, :0].cuda(), scores.cuda())
    assert (none[0] == -1).all() and none[3] is None
    assert fi.beam_select(logits[:0].cuda(), scores[:0].cuda())[0].shape == (0, 3)


def test_selection_of_large_logits(torch, fi):  # noqa: F811
    """fp32 logits whose multiples leave fp32's range: the sum is made again in 64 bits."""
    logits = torch.tensor([[3e38, 2.9e38, 3e38, 0.0], [-3e38, -3.3e38, -3e38, -3.4e38], [1e30, 1e30, -1e30, 0.0], [-1e37, -1e37, -2e37, -1e37]])
    scores = torch.zeros((2, 2))
    _same(fi.beam_select(logits.cuda(), scores.cuda(), keep=4), oracle.select(logits, scores, 4))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_selection_beyond_32_bits(torch, fi, dtype):  # noqa: F811
    """Rows whose offsets pass 2^32 bytes, and 2^31 values."""
    g, kind, vocab = torch.Generator().manual_seed(47), _kind(torch, dtype), 5003
    gap = (1 << 33) // 5 // torch.finfo(kind).bits * 8 + 3
    wide = torch.empty(5 * gap + vocab, dtype=kind, device="cuda")
    logits = torch.as_strided(wide, (6, vocab), (gap, 1))
    logits.copy_(torch.randn((6, vocab), generator=g))
    scores = -torch.rand((2, 3), generator=g)
    plain = fi.beam_select(logits.contiguous(), scores.cuda())
    assert all(x is None or torch.equal(x, y) for x, y in zip(fi.beam_select(logits, scores.cuda()), plain))


def test_first_step_of_a_search(torch, fi):  # noqa: F811
    """All beams hold the same prompt and only the first is alive."""
    g = torch.Generator().manual_seed(34)
    logits = torch.randn((2, 1, 5000), generator=g).expand(2, 4, 5000).reshape(8, 5000).bfloat16()
    scores = torch.tensor([[0.0, -math.inf, -math.inf, -math.inf]] * 2)
    tokens, parents, best, _ = fi.beam_select(logits.cuda(), scores.cuda())
    _same((tokens, parents, best, None), oracle.select(logits, scores, 4))
    assert torch.equal(parents.cpu(), torch.tensor([[0] * 4, [4] * 4], dtype=torch.int32))


# ---- pages --------------------------------------------------------------------------------------
def _pool(torch, g, rows, columns, page, longest, spare, beams=1, more=0):  # noqa: F811
    """Rows in groups of `beams` that share pages of their first half; counts that go with them, some pages held by someone else too."""
    table, lengths, held, used = [], [], [], 0
    for r in range(rows):
        if r % beams == 0:
            n = int(torch.randint(0, longest + 1, (1,), generator=g))
            shared = list(range(used, used + n // 2 // page if beams > 1 else used))
            used += len(shared)
        m = n + int(torch.randint(0, more + 1, (1,), generator=g)) if more else n
        m = min(m, columns * page)
        own = -(-m // page) - len(shared)
        table.append(shared + list(range(used, used + own)))
        used += own
        lengths.append(n)
        held.append(m)
    pages = used + spare
    order = torch.randperm(pages, generator=g).tolist()
    refs = [0] * pages
    table = [[order[p] for p in row] for row in table]
    for row in table:
        for p in row:
            refs[p] += 1
    for row in table[::5]:   # a prompt that is kept for later requests
        for p in row[:2]:
            refs[p] += 1
    i32 = dict(dtype=torch.int32)
    full = torch.tensor([row + [-7] * (columns - len(row)) for row in table], **i32).view(rows, columns)
    return full, torch.tensor(lengths, **i32), torch.tensor(held, **i32), torch.tensor(refs, **i32)


def _caches(torch, g, pages, page):  # noqa: F811
    """Of several types, page sizes, orders and strides; bytes that are no whole pieces."""
    a = torch.randn((pages, page, 2, 8), generator=g).bfloat16().cuda()
    b = torch.randn((pages, 2, page, 24), generator=g).cuda().permute(0, 2, 1, 3)
    c = torch.randint(0, 256, (pages, page, 3), generator=g, dtype=torch.uint8).cuda()
    d = torch.randn((pages, 2, page * 520), generator=g).cuda()[:, 1]   # with something between the pages
    e = torch.randint(0, 256, (pages * page * 5 + 1,), generator=g, dtype=torch.uint8).cuda()[1:].view(pages, page, 5)
    return [a, b, c, d, e]


FORKS = [
    # rows, columns, page, longest, beams, new rows (None: as they are), room, spare pages, tokens held beyond the committed ones
    (1, 4, 16, 50, 1, 4, 1, 20, 0), (4, 8, 16, 100, 4, 4, 1, 3, 0), (12, 8, 1, 7, 3, 12, 1, 40, 0), (8, 5, 7, 33, 2, None, 5, 100, 9), (6, 9, 48, 400, 3, 11, 0, 0, 0),
    (6, 9, 48, 400, 3, 11, 1, 2, 0), (24, 40, 16, 600, 4, 30, 17, 25, 30), (3, 2, 16, 32, 1, 3, 1, 9, 0), (5, 4, 16, 60, 5, 5, 40, 3, 0), (1, 1, 256, 200, 1, 64, 1, 5, 0),
    (200, 12, 8, 90, 8, 240, 3, 170, 4), (1000, 6, 4, 20, 5, 1024, 2, 900, 3), (1500, 6, 4, 20, 5, 1400, 2, 1100, 3), (40, 3000, 1, 2500, 4, 48, 5, 300, 0), (0, 3, 16, 1, 1, 3, 1, 4, 0),
]


@pytest.mark.parametrize("rows,columns,page,longest,beams,new,room,spare,more", FORKS)
def test_forks(torch, fi, rows, columns, page, longest, beams, new, room, spare, more):  # noqa: F811
    g = torch.Generator().manual_seed(41)
    for turn in range(3):
        table, lengths, held, refs = _pool(torch, g, rows, columns, page, longest, spare, beams, more)
        caches = _caches(torch, g, refs.shape[0], page)
        parents = None if new is None else torch.randint(-1, max(rows, 1), (new,), generator=g).int()
        if new is not None and turn == 1 and rows:
            parents[:] = torch.arange(new) % rows   # all go on, most of them by themselves
        if new is not None and turn == 2 and new > 2:
            parents[1:3] = torch.tensor([1 << 30, -(1 << 30)])
        want_caches = [c.cpu().contiguous() for c in caches]
        want = oracle.fork(table, lengths, refs, parents, page, held if more else None, room, want_caches)
        gap = torch.full((rows, columns + 3), 1 << 29, dtype=torch.int32)
        gap[:, :columns] = table
        got = fi.fork_pages(gap.cuda()[:, :columns], lengths.cuda(), refs.cuda(), None if parents is None else parents.cuda(), page_size=page, held=held.cuda() if more else None,
                            room=room, caches=caches)
        for name, x, y in zip(("table", "lengths", "held", "refs", "slots"), got, want):
            assert x.shape == y.shape and x.dtype == y.dtype and torch.equal(x.cpu(), y), name
        assert all(torch.equal(x.cpu(), y) for x, y in zip(caches, want_caches))


def test_forks_go_on(torch, fi):  # noqa: F811
    """Thirty steps, each on what the one before left: no page is lost or held twice, freed ones are used again, and the pool hardly suffices."""
    g, page, rows = torch.Generator().manual_seed(42), 4, 6
    pages, columns = 60, 12
    table = torch.full((rows, columns), -1, dtype=torch.int32)
    table[0, :3] = torch.tensor([50, 3, 17])
    refs = torch.zeros(pages, dtype=torch.int32)
    refs[[50, 3, 17]] = 1
    lengths = torch.tensor([10, 0, 0, 0, 0, 0], dtype=torch.int32)
    state, mine = [t.cuda() for t in (table, lengths, lengths, refs)], [table, lengths, lengths.clone(), refs]
    cache = torch.randn((pages, page, 3), generator=g)
    own, theirs, lacking = cache.clone(), cache.cuda(), 0
    parents = torch.zeros(rows, dtype=torch.int32)
    for step in range(30):
        want = oracle.fork(mine[0], mine[1], mine[3], parents, page, mine[2], 2, [own])
        got = fi.fork_pages(state[0], state[1], state[3], parents.cuda(), page_size=page, held=state[2], room=2, caches=[theirs])
        assert all(torch.equal(x.cpu(), y) for x, y in zip(got, want)) and torch.equal(theirs.cpu(), own), step
        counts = torch.zeros(pages, dtype=torch.int32)
        for row, n in zip(want[0], want[2]):
            for p in row[:-(-int(n) // page)]:
                counts[p] += 1
        assert torch.equal(counts, want[3])
        written = want[4].clone()
        value = torch.randn((*written.shape, 3), generator=g)
        own.view(-1, 3)[written[written >= 0]] = value[written >= 0]
        theirs.view(-1, 3)[written[written >= 0].cuda()] = value[written >= 0].cuda()
        lacking += int((want[2] == want[1]).sum())
        accepted = torch.where(want[2] > want[1], 1 + torch.randint(0, 2, (rows,), generator=g).int(), 0).int()   # one or two of the two
        mine = [want[0], want[1] + accepted, want[2], want[3]]
        state = [got[0], got[1] + accepted.cuda(), got[2], got[3]]
        parents = torch.randint(0, rows, (rows,), generator=g).int()
        if step % 7 == 6:
            parents[:3] = -1
    assert lacking > 0


@pytest.mark.parametrize("pages,rows,steps,seed", [(7, 6, 60, 0), (9, 6, 60, 3), (9, 6, 60, 6), (12, 6, 60, 1), (700, 1100, 12, 2)])
def test_rows_keep_their_tokens_where_pages_are_lacking(torch, fi, pages, rows, steps, seed):  # noqa: F811
    """Rows that got no copy of a page share it with one that went on in it; later steps, in any order of the rows, write over nobody's tokens."""
    g, page, room = torch.Generator().manual_seed(seed), 4, 2
    table, refs, lengths = torch.full((rows, 12), -1, dtype=torch.int32), torch.zeros(pages, dtype=torch.int32), torch.zeros(rows, dtype=torch.int32)
    table[0, 0], refs[3], lengths[0] = 3, 1, 2
    cache, truth, parents, stamp, without = torch.zeros((pages, page), dtype=torch.int64), [[1, 2]] + [[]] * (rows - 1), torch.zeros(rows, dtype=torch.int32), 3, 0
    cache[3, :2] = torch.tensor([1, 2])
    held, theirs = lengths.clone(), cache.cuda()
    for step in range(steps):
        want = oracle.fork(table, lengths, refs, parents, page, held, room, [cache])
        got = fi.fork_pages(table.cuda(), lengths.cuda(), refs.cuda(), parents.cuda(), page_size=page, held=held.cuda(), room=room, caches=[theirs])
        assert all(torch.equal(x.cpu(), y) for x, y in zip(got, want)) and torch.equal(theirs.cpu(), cache), step
        table, lengths, held, refs, slots = want
        truth = [list(truth[p]) if p >= 0 else [] for p in parents.tolist()]
        for i in range(rows):
            if slots[i, 0] >= 0:
                values = torch.arange(stamp, stamp + room)
                cache.view(-1)[slots[i]] = values
                stamp += room
                truth[i] += values[:int(torch.randint(1, room + 1, (1,), generator=g))].tolist()
            else:
                without += int(parents[i] >= 0)
        lengths = torch.tensor([len(x) for x in truth], dtype=torch.int32)
        theirs.copy_(cache)
        numbers, values = table.tolist(), cache.tolist()
        for i, tokens in enumerate(truth):
            assert [values[numbers[i][j // page]][j % page] for j in range(len(tokens))] == tokens, (step, i)
        parents = torch.arange(rows, dtype=torch.int32)
        parents[torch.randperm(rows, generator=g)[:rows // 2]] = torch.randint(-1, rows, (rows // 2,), generator=g).int()
        if step % 3 == 0:
            parents = parents[torch.randperm(rows, generator=g)]
    assert without > 0


def test_forks_of_damaged_tables(torch, fi):  # noqa: F811
    """Entries that are no pages, and lengths out of range, are clamped and count nowhere; the other rows are as they would be."""
    g = torch.Generator().manual_seed(43)
    table, lengths, _, refs = _pool(torch, g, 6, 5, 8, 40, 30)
    lengths[2:5] = torch.tensor([20, 20, 39])   # (partly filled)
    table[2, :3], table[3, 2], table[4, 1] = torch.tensor([-1, 1 << 30, -5]), refs.shape[0], -(1 << 31)
    lengths[0], lengths[1] = 1 << 30, -9
    cache = torch.randn((refs.shape[0], 64), generator=g)
    for room in (0, 1, 9):
        mine, theirs = cache.clone(), cache.cuda()
        want = oracle.fork(table, lengths, refs, torch.arange(6).int(), 8, None, room, [mine])
        got = fi.fork_pages(table.cuda(), lengths.cuda(), refs.cuda(), page_size=8, room=room, caches=[theirs])
        assert all(torch.equal(x.cpu(), y) for x, y in zip(got, want)) and torch.equal(theirs.cpu(), mine)


COMPACTIONS = [(1, 1, 1, 1.0), (3, 7, 16, 0.5), (1024, 40, 9, 0.6), (1025, 300, 2, 0.3), (5000, 33, 1, 0.97), (4097, 10, 4, 0.02), (300, 0, 16, 0.5), (64, 5, 16, 0.0), (9001, 64, 1, 0.55)]


@pytest.mark.parametrize("pages,rows,page,share", COMPACTIONS)
def test_compaction(torch, fi, pages, rows, page, share):  # noqa: F811
    g = torch.Generator().manual_seed(44)
    for turn in range(2):
        refs = torch.where(torch.rand(pages, generator=g) < share, torch.randint(1, 4, (pages,), generator=g), torch.randint(-1, 1, (pages,), generator=g)).int()
        table = torch.randint(-2, pages + 2, (rows, 13), generator=g).int()   # free pages and no pages among them
        caches = _caches(torch, g, pages, page)
        mine = [c.cpu().contiguous() for c in caches]
        want = oracle.compact(table, refs, mine)
        got = fi.compact_pages(table.cuda(), refs.cuda(), caches=caches)
        for name, x, y in zip(("table", "refs", "moved", "live"), got, want):
            assert x.shape == y.shape and torch.equal(x.cpu(), y), name
        assert all(torch.equal(x.cpu(), y) for x, y in zip(caches, mine))
        again = fi.compact_pages(got[0], got[1], caches=caches)
        assert torch.equal(again[0], got[0]) and torch.equal(again[1], got[1]) and all(torch.equal(x.cpu(), y) for x, y in zip(caches, mine))


def test_many_caches(torch, fi):  # noqa: F811
    """As many as a call takes, among them some without bytes: more than one launch."""
    g = torch.Generator().manual_seed(45)
    table, lengths, _, refs = _pool(torch, g, 3, 5, 8, 37, 12)
    lengths.clamp_(min=1)
    cache = torch.randn((128, refs.shape[0], 33), generator=g)
    theirs, parents = cache.cuda(), torch.tensor([0, 0, 1, 2, 2], dtype=torch.int32)
    caches = [c if i != 70 else c[:, :0] for i, c in enumerate(theirs)]
    mine = list(cache.clone())
    want = oracle.fork(table, lengths, refs, parents, 8, None, 1, mine[:70] + mine[71:])
    got = fi.fork_pages(table.cuda(), lengths.cuda(), refs.cuda(), parents.cuda(), page_size=8, room=1, caches=caches)
    assert all(torch.equal(x.cpu(), y) for x, y in zip(got, want)) and torch.equal(theirs.cpu(), torch.stack(mine))
    want = oracle.compact(want[0], want[3], mine[:70] + mine[71:])
    got = fi.compact_pages(got[0], got[3], caches=caches)
    assert all(torch.equal(x.cpu(), y) for x, y in zip(got, want)) and torch.equal(theirs.cpu(), torch.stack(mine))
    with pytest.raises(ValueError, match="at most 128"):
        fi.fork_pages(table.cuda(), lengths.cuda(), refs.cuda(), page_size=8, caches=caches + caches[:1])


def test_pages_beyond_32_bits(torch, fi):  # noqa: F811
    """Pages whose offsets pass 2^32 bytes are copied whole."""
    pages, size = 40, 1 << 27
    cache = torch.zeros((pages, size), dtype=torch.uint8, device="cuda")
    x = torch.randint(0, 256, (size,), dtype=torch.uint8, generator=torch.Generator(device="cuda").manual_seed(46), device="cuda")
    cache[37] = x
    refs = torch.zeros(pages, dtype=torch.int32).cuda()
    refs[37], refs[:36] = 1, 1
    table, lengths = torch.tensor([[37]], dtype=torch.int32).cuda(), torch.tensor([3], dtype=torch.int32).cuda()
    got = fi.fork_pages(table, lengths, refs, torch.tensor([0, 0], dtype=torch.int32).cuda(), page_size=16, room=1, caches=[cache])
    assert got[0].tolist() == [[36], [37]] and got[4].tolist() == [[36 * 16 + 3], [37 * 16 + 3]]
    assert torch.equal(cache[36], x) and torch.equal(cache[37], x) and not cache[38].any()
    refs[0], refs[38] = 0, 1
    cache[38] = 255 - x
    table, refs, moved, live = fi.compact_pages(table, refs, caches=[cache])
    assert live.item() == 37 and table.item() == 0 and moved[38] == 36 and torch.equal(cache[0], x) and torch.equal(cache[36], 255 - x)


# ---- tensors that do not fit --------------------------------------------------------------------
def test_tensors_that_do_not_fit_are_refused(torch, fi):  # noqa: F811
    i32, f32 = dict(dtype=torch.int32, device="cuda"), dict(device="cuda")
    logits, scores = torch.zeros((6, 10), **f32), torch.zeros((2, 3), **f32)
    yes = torch.zeros((2, 3), dtype=torch.bool, device="cuda")
    for args, kw in [((logits[:5], scores), {}), ((logits.t(), scores), {}), ((logits, scores.double()), {}), ((logits, scores.t()), {}), ((logits, scores), dict(keep=0)),
                     ((logits, scores), dict(end=-1)), ((logits, scores), dict(ended=yes)), ((logits, scores), dict(end=1, ended=yes.int())), ((logits, scores.cpu()), {}),
                     ((logits, scores), dict(tokens_out=torch.zeros((2, 4), **i32))), ((logits, scores), dict(scores_out=scores.double())), ((logits[0], scores), {})]:
        with pytest.raises(ValueError):
            fi.beam_select(*args, **kw)
    with pytest.raises(TypeError):
        fi.beam_select(logits.half(), scores)
    for kw in (dict(keep=65), dict(scores_out=scores), dict(end=10), dict(workspace=torch.zeros(8, dtype=torch.uint8, device="cuda"))):
        with pytest.raises(fi.FiError):
            fi.beam_select(logits, scores, **kw)
    table, lengths, refs = torch.zeros((3, 2), **i32), torch.zeros(3, **i32), torch.zeros(9, **i32)
    cache = torch.zeros((9, 4, 6), **f32)
    for args, kw in [((table[0], lengths, refs), {}), ((table.long(), lengths, refs), {}), ((table, lengths[:2], refs), {}), ((table, lengths, refs.float()), {}),
                     ((table, lengths, refs, lengths[:, None]), {}), ((table, lengths, refs, lengths.long()), {}), ((table, lengths, refs), dict(held=lengths[:1])),
                     ((table, lengths, refs), dict(room=-1)), ((table, lengths, refs), dict(caches=[cache[:8]])), ((table, lengths, refs), dict(caches=[cache[:, :, :5]])),
                     ((table, lengths, refs), dict(caches=[cache[:, ::2]])), ((table, lengths, refs), dict(caches=[cache.cpu()])), ((table.cpu(), lengths, refs), {}),
                     ((table, lengths, refs), dict(caches=[cache[:1].expand(9, 4, 6)[:, :1].expand(9, 4, 6)])), ((table, lengths, refs), dict(slots_out=table, room=2))]:
        with pytest.raises(ValueError):
            fi.fork_pages(*args, page_size=4, **kw)
    with pytest.raises(TypeError):
        fi.fork_pages(table, lengths, refs, page_size=4, caches=[3])
    for kw in (dict(page_size=0), dict(page_size=4, refs_out=refs), dict(page_size=4, table_out=table), dict(page_size=4, held_out=lengths), dict(page_size=4, held=refs[:3], refs_out=refs),
               dict(page_size=4, caches=[cache[:1].expand(9, 4, 6)])):
        with pytest.raises(fi.FiError):
            fi.fork_pages(table, lengths, refs, **kw)
    for args, kw in [((table, refs[None]), {}), ((table, refs.long()), {}), ((table, refs), dict(live_out=torch.zeros(2, **i32))), ((table, refs), dict(caches=[cache[:3]]))]:
        with pytest.raises(ValueError):
            fi.compact_pages(*args, **kw)
    for kw in (dict(refs_out=refs), dict(table_out=table), dict(moved_out=refs)):
        with pytest.raises(fi.FiError):
            fi.compact_pages(table, refs, **kw)
    k, q, cu = torch.zeros((4, 2, 64), **f32), torch.zeros((4, 4, 64), **f32), torch.tensor([0, 4], **i32)
    c, s = fi.fp4_cache(3, 16, 2, 64)
    slots = torch.arange(4).cuda()
    for args, kw in [((k, k, slots.int(), c, s, c, s), {}), ((k, k, slots, c, s), {}), ((k, None, slots, c, s, c, s), {}), ((k, None, slots, c[..., :-1], s), {}),
                     ((k, None, slots, c.float(), s), {}), ((k, None, slots, c, s[..., :1]), {}), ((k[..., :60], None, slots, c[..., :30], s), {}), ((k.cpu(), None, slots, c, s), {}),
                     ((k, None, slots[:3], c, s), {}), ((k, None, slots, c, s), dict(k_held=k.bfloat16()))]:
        with pytest.raises((ValueError, TypeError)):
            fi.fp4_cache_write(*args, **kw)
    for codes in (torch.zeros((3, 16, 2, 33), dtype=torch.uint8).cuda()[..., 1:], c[:1].expand(3, 16, 2, 32)):   # rows off four bytes; pages that share memory
        with pytest.raises(fi.FiError):
            fi.fp4_cache_write(k, None, slots, codes, s)
    table, lengths = torch.zeros((1, 3), **i32), torch.zeros(1, **i32)
    for args, kw in [((q, c, s, c, s[:2], table, lengths, cu), {}), ((q[..., :56], c, s, c, s, table, lengths, cu), {}), ((q, c, s, c, s, table.long(), lengths, cu), {}),
                     ((q, c, s, c, s, table, lengths, cu), dict(out=q.bfloat16())), ((q, c, s, c, s, table, lengths, cu, torch.zeros((4, 0), dtype=torch.int64).cuda()), {})]:
        with pytest.raises(ValueError):
            fi.fp4_tree_attention(*args, **kw)
    for kw in (dict(scale=0.0), dict(max_nodes=-1), dict(out=q[:, :1].expand(4, 4, 64))):
        with pytest.raises(fi.FiError):
            fi.fp4_tree_attention(q, c, s, c, s, table, lengths, cu, **kw)


def test_no_gradients_and_outputs_that_count_as_changed(torch, fi):  # noqa: F811
    g = torch.Generator().manual_seed(47)
    k, q = torch.randn((4, 2, 64), generator=g).cuda(), torch.randn((4, 4, 64), generator=g).cuda()
    c, s = fi.fp4_cache(3, 16, 2, 64)
    i32 = dict(dtype=torch.int32, device="cuda")
    table, lengths, cu, refs = torch.tensor([[1, 0, 2]], **i32), torch.tensor([20], **i32), torch.tensor([0, 4], **i32), torch.ones(3, **i32)
    cache = torch.randn((3, 16, 2), generator=g).cuda()
    calls = [
        (fi.fp4_cache_write, dict(k=k, v=k.clone(), slots=torch.arange(4).cuda(), k_codes=c, k_scales=s, v_codes=c.clone(), v_scales=s.clone(), k_held=torch.zeros_like(k),
                                  v_held=torch.zeros_like(k)), ("k_codes", "k_scales", "v_codes", "v_scales", "k_held", "v_held")),
        (fi.fp4_tree_attention, dict(q=q, k_codes=c, k_scales=s, v_codes=c, v_scales=s, block_table=table, cached=lengths, cu_nodes=cu, out=torch.zeros_like(q)), ("out",)),
        (fi.beam_select, dict(logits=q.view(16, 64), scores=torch.zeros((4, 4)).cuda(), scores_out=torch.zeros((4, 4)).cuda(), tokens_out=torch.zeros((4, 4), **i32)),
         ("scores_out", "tokens_out")),
        (fi.fork_pages, dict(block_table=table, lengths=lengths, refs=refs, page_size=16, room=1, caches=[cache], refs_out=torch.zeros(3, **i32)), ("refs_out", "caches")),
        (fi.compact_pages, dict(block_table=table, refs=refs, caches=[cache], moved_out=torch.zeros(3, **i32)), ("moved_out", "caches")),
    ]
    one = lambda args, name: args[name][0] if name == "caches" else args[name]   # noqa: E731
    for call, args, outs in calls:
        for name in args:
            if name == "page_size" or name == "room" or not one(args, name).is_floating_point():
                continue
            wants = one(args, name).detach().clone().requires_grad_()
            wants = [wants] if name == "caches" else wants
            with pytest.raises(ValueError, match="requires a gradient"):
                call(**{**args, name: wants})
            with torch.no_grad():
                call(**{**args, name: wants})
        before = [one(args, o)._version for o in outs]
        call(**args)
        assert [one(args, o)._version for o in outs] == [v + 1 for v in before]
        with torch.inference_mode():
            made = torch.zeros_like(one(args, outs[0]))
        call(**{**args, outs[0]: made})
        assert torch.equal(made, one(args, outs[0]))
