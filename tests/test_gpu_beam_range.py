"""Selection and forks where their sizes end: the largest vocabulary, the last few logits of a row, the largest pool of pages; and a list of caches that changes during the call.

A score is a sum in 64 bits, rounded once to fp32, whose log-sum comes from fp32 terms: each exp2 has a few u, its argument one rounding of at most 64 u for what
counts, a lane adds at most 64 of them in fp32 (u each), lanes and waves are added in 64 bits: bound (64 * 1.1 + 80) u absolutely, and u |score|."""
import math

import pytest

from tests import fp4_oracle as oracle
from tests.test_gpu_operators import U, _kind, fi, torch  # noqa: F401

pytestmark = pytest.mark.gpu

LOG_SUM = (64 * 1.1 + 80) * U
MOST, LAST = (1 << 31) - 1025, (1 << 31) - 4096   # tokens or pages; where the last stretch of so many logits begins


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_selection_from_the_largest_vocabulary(torch, fi, dtype):  # noqa: F811
    """The last stretch of a row ends next to 2^31; its last piece is moved forward by one place, so the eighth logit from the end is read twice and counts once."""
    kind = _kind(torch, dtype)
    logits = torch.full((1, MOST), -30.0, dtype=kind, device="cuda")
    planted = {MOST - 8: 5.0, MOST - 1: 4.0, 0: 3.0, MOST - 700: 2.5, 1 << 30: 2.0, LAST: 1.5, LAST - 1: 1.0, MOST - 1100: 0.5}
    for token, x in planted.items():
        logits[0, token] = x
    tokens, parents, scores, _ = fi.beam_select(logits, torch.tensor([[-2.0]]).cuda(), keep=8)
    log_sum = math.log(math.fsum([math.exp(x) for x in planted.values()] + [(MOST - len(planted)) * math.exp(-30.0)]))
    want = torch.tensor([-2.0 + (x - log_sum) for x in planted.values()]).double()
    assert tokens.tolist() == [list(planted)] and not parents.any()
    assert ((scores[0].double().cpu() - want).abs() <= LOG_SUM + 1.01 * U * want.abs()).all()


def test_forks_in_the_largest_pool(torch, fi):  # noqa: F811
    """One page is free, the last one, and two rows need one: the pages are gone through to their end and no further."""
    i32 = dict(dtype=torch.int32, device="cuda")
    refs = torch.ones(MOST, **i32)
    refs[MOST - 1] = 0
    table, lengths = torch.tensor([[0, -1], [1, -1]], **i32), torch.tensor([16, 16], **i32)
    table, lengths, held, after, slots = fi.fork_pages(table, lengths, refs, page_size=16, room=1)
    assert table.tolist() == [[0, MOST - 1], [1, -1]] and lengths.tolist() == [16, 16] and held.tolist() == [17, 16]
    assert slots.tolist() == [[(MOST - 1) * 16], [-1]]
    refs[MOST - 1] = 1
    assert torch.equal(after, refs)


TAILS = [512 + 1, 512 + 7, 3 * 512 + 4, 2048 + 5, 16384 + 1, 16384 + 7, 2 * 16384 + 3, 8 * 16384 - 1, 13, 8, 7, 1]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("vocab", TAILS)
def test_the_last_logits_of_a_row_count_once(torch, fi, dtype, vocab):  # noqa: F811
    """The last few logits, which a piece that was moved forward brings, hold most of the softmax's mass: one left out, or taken twice, would be seen in every score."""
    g, kind = torch.Generator().manual_seed(51), _kind(torch, dtype)
    logits = torch.randn((6, vocab), generator=g) - 10
    for row, n in enumerate((1, 2, 5, 7, 8, 9)):   # of logits at the end
        logits[row, -n:] = 4 + torch.rand(min(n, vocab), generator=g)
    logits = logits.to(kind)
    scores = -torch.rand((3, 2), generator=g)
    for keep in (1, 9, 64):
        tokens, parents, best, _ = fi.beam_select(logits.cuda(), scores.cuda(), keep=keep)
        want = oracle.select(logits, scores, keep)
        assert torch.equal(tokens.cpu(), want[0]) and torch.equal(parents.cpu(), want[1])
        there = want[0] >= 0
        assert ((best.double().cpu() - want[2]).abs() <= LOG_SUM + 1.01 * U * want[2].abs())[there].all() and (best.cpu()[~there] == -math.inf).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("seqs,beams,keep,vocab", [(1, 4, 4, 32000), (3, 5, 10, 777), (1, 64, 64, 4099), (2, 2, 64, 131071), (5, 8, 16, 20000), (1, 16, 32, 131072), (64, 8, 16, 32000)])
def test_scores_are_as_exact_as_terms_of_32_bits(torch, fi, dtype, seqs, beams, keep, vocab):  # noqa: F811
    g, kind = torch.Generator().manual_seed(52), _kind(torch, dtype)
    logits, scores = (3 * torch.randn((seqs * beams, vocab), generator=g)).to(kind), -10 * torch.rand((seqs, beams), generator=g)
    tokens, parents, best, _ = fi.beam_select(logits.cuda(), scores.cuda(), keep=keep)
    want = oracle.select(logits, scores, keep)
    assert torch.equal(tokens.cpu(), want[0]) and torch.equal(parents.cpu(), want[1])
    assert ((best.double().cpu() - want[2]).abs() <= LOG_SUM + 1.01 * U * want[2].abs()).all()


def test_caches_are_those_of_the_call_whatever_becomes_of_their_list(torch, fi, monkeypatch):  # noqa: F811
    """A caller's list that changes while the call allocates its outputs."""
    i32, made = dict(dtype=torch.int32, device="cuda"), torch.empty
    cache, caches = torch.arange(24.0).cuda().view(3, 8), []
    table, refs, one = torch.zeros((1, 2), **i32), torch.tensor([1, 0, 0], **i32), torch.tensor([3], **i32)
    now = torch.cuda.current_stream().cuda_stream

    def empty(*args, **kw):
        caches.clear()
        return made(*args, **kw)
    caches.append(cache)
    before = cache._version
    monkeypatch.setattr(torch, "empty", empty)
    got = fi.fork_pages(table, one, refs, torch.tensor([0, 0], **i32), page_size=4, room=1, caches=caches, stream=now)
    assert not caches and cache._version == before + 1 and got[0].tolist() == [[1, -1], [0, -1]]
    assert torch.equal(cache[1], cache[0]) and cache[2, 0] == 16
    caches.append(cache)
    fi.compact_pages(table + 2, torch.tensor([0, 0, 1], **i32), caches=caches, stream=now)
    assert not caches and cache._version == before + 2 and cache[0, 0] == 16
