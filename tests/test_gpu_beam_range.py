"""Selection and forks where their sizes end: the largest vocabulary, the last few logits of a row, the largest pool of pages.

A score is a sum in 64 bits, rounded once to fp32, whose log-sum comes from fp32 terms: each exp2 has a few u, its argument one rounding of at most 64 u for what
counts, a lane adds at most 64 of them in fp32 (u each), lanes and waves are added in 64 bits: bound (64 * 1.1 + 80) u absolutely, and u |score|."""
import math

import pytest

from tests import fp4_oracle as oracle
from tests.test_gpu_operators import U, _kind, fi, torch  # noqa: F401

pytestmark = pytest.mark.gpu

LOG_SUM = (64 * 1.1 + 80) * U
MOST = (1 << 31) - 1025


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_selection_from_the_largest_vocabulary(torch, fi, dtype):  # noqa: F811
    """The last stretch of a row ends next to 2^31; its last piece is moved forward by one place, so the eighth logit from the end is read twice and counts once."""
    kind = _kind(torch, dtype)
    logits = torch.full((1, MOST), -30.0, dtype=kind, device="cuda")
    planted = {MOST - 8: 5.0, MOST - 1: 4.0, 0: 3.0, MOST - 700: 2.5, 1 << 30: 2.0, MOST - 3071: 1.5, MOST - 3072: 1.0, MOST - 1100: 0.5}
    for token, x in planted.items():
        logits[0, token] = x
    tokens, parents, scores, _ = fi.beam_select(logits, torch.tensor([[-2.0]]).cuda(), keep=8)
    log_sum = math.log(math.fsum([math.exp(x) for x in planted.values()] + [(MOST - len(planted)) * math.exp(-30.0)]))
    want = torch.tensor([-2.0 + (x - log_sum) for x in planted.values()]).double()
    assert tokens.tolist() == [list(planted)] and not parents.any()
    assert ((scores[0].double().cpu() - want).abs() <= LOG_SUM + 1.01 * U * want.abs()).all()
