"""4-bit products of rows that fill the range of their type, of rows with an offset and of infinities, on every kernel that may take a call.

Bounds as in test_gpu_operators.py, from the formula's own terms: sums of K fp32 terms scale * (q - zero) * x, (K + 8) u of the sum of their sizes, twice where
a kernel carries (16 + q) through it, and a rounding to bf16."""
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


CALLS = [
    # rows, inputs, outputs, group, zeros, odd strides
    (1, 4096, 1600, 128, False, False), (2, 2048, 1601, 64, True, False), (5, 4096, 1000, 32, True, False), (1, 4096, 300, 64, True, False), (3, 2048, 40, 32, False, False),
    (5, 512, 70, 32, True, False), (9, 640, 33, 64, False, False), (17, 1024, 48, 256, True, False), (2, 256, 16400, 64, True, False), (6, 2048, 2100, 128, True, False),
    (9, 12288, 70, 64, True, False), (40, 12352, 270, 32, False, False), (6, 12288, 17, 128, True, False), (520, 512, 4100, 64, True, False), (3, 512, 37, 64, True, True),
    (12, 4096, 20, 256, False, True),
]


def _case(torch, rows, inputs, outputs, group, zeros, odd, kind):
    g = torch.Generator().manual_seed(rows * inputs + outputs)
    pad = 3 if odd else 0
    x = torch.randn((rows, inputs + pad), generator=g)
    w = torch.randint(0, 256, (outputs, inputs // 2 + pad), generator=g, dtype=torch.uint8)
    s = (torch.rand((outputs, inputs // group), generator=g) + 0.5) / (4.6 * math.sqrt(inputs))
    z = torch.randint(0, 16, s.shape, generator=g, dtype=torch.uint8) if zeros else None
    x, w = x.to(kind)[:, :inputs], w[:, :inputs // 2]
    q = torch.stack([w & 15, w >> 4], -1).reshape(outputs, -1).double().view(outputs, -1, group)
    weights = ((q - (8.0 if z is None else z.double()[..., None])) * s.double()[..., None]).flatten(1)
    return x, w, s, z, weights


def _product(torch, fi, x, w, s, z, group, odd):
    x, w = x.cuda(), w.cuda()
    if odd:   # rows that start on odd elements
        x = torch.nn.functional.pad(x, (3, 0))[:, 3:]
        w = torch.nn.functional.pad(w, (3, 0))[:, 3:]
    return fi.q4_matmul(x, w, s.cuda(), None if z is None else z.cuda(), group=group).double().cpu()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,inputs,outputs,group,zeros,odd", CALLS)
def test_infinities_are_the_formulas(torch, fi, dtype, rows, inputs, outputs, group, zeros, odd):
    """Infinite inputs of both signs and NaN: what the formula gives, whichever kernel takes the call; other rows keep their bits."""
    kind = torch.float32 if dtype == "f32" else torch.bfloat16
    x, w, s, z, weights = _case(torch, rows, inputs, outputs, group, zeros, odd, kind)
    clean = _product(torch, fi, x, w, s, z, group, odd)
    for row, put in ((rows // 2, {1: math.inf}), (rows - 1, {inputs - 1: -math.inf, 7: -math.inf}), (0, {5: math.inf, inputs // 2: -math.inf}), (rows // 3, {inputs - 2: math.nan})):
        bad = x.clone()
        for at, value in put.items():
            bad[row, at] = value
        got = _product(torch, fi, bad, w, s, z, group, odd)
        want = sum(weights[:, at] * value for at, value in put.items())   # the finite rest does not matter
        assert not want.isfinite().any()
        assert torch.equal(got[row].isnan(), want.isnan()) and torch.equal(got[row][~want.isnan()], want[~want.isnan()])
        others = [i for i in range(rows) if i != row]
        assert torch.equal(got[others], clean[others])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,inputs,outputs,group,zeros,odd", CALLS)
def test_inputs_near_the_largest_number(torch, fi, dtype, rows, inputs, outputs, group, zeros, odd):
    """Inputs up to 3.39e38, whose sums with whole weights overflow; with the scales the results are finite."""
    kind = torch.float32 if dtype == "f32" else torch.bfloat16
    x, w, s, z, weights = _case(torch, rows, inputs, outputs, group, zeros, odd, kind)
    weights = weights / 64
    g = torch.Generator().manual_seed(1)
    for row in {0, rows // 2, rows - 1}:
        at = torch.randperm(inputs, generator=g)[:24]
        x[row, at] = (torch.randn(24, generator=g).sign() * torch.tensor([3.39e38, 1e38, 2e37, 1e30] * 6)).to(kind)
    got = _product(torch, fi, x, w, s / 64, z, group, odd)
    want, size = x.double() @ weights.t(), x.double().abs() @ weights.abs().t()
    half = H if dtype == "bf16" else 0.0
    assert size.max() < 3e38
    # (terms as they lie in a kernel that adds (16 + q) x: 31 units of scale where the formula has q - zero)
    assert ((got - want).abs() <= (inputs + 8) * U * (size + x.double().abs() @ (31 / 64 * s.double().repeat_interleave(group, 1)).t()) + 1.01 * half * want.abs()).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,inputs,outputs,group,zeros,odd", CALLS)
def test_rows_with_an_offset(torch, fi, dtype, rows, inputs, outputs, group, zeros, odd):
    """Inputs around 100, as ahead of a norm: the offset times the weights' mean stays in the results, the bound is that of the formula's own terms."""
    kind = torch.float32 if dtype == "f32" else torch.bfloat16
    x, w, s, z, weights = _case(torch, rows, inputs, outputs, group, zeros, odd, kind)
    x = (x.float() + 100).to(kind)
    got = _product(torch, fi, x, w, s, z, group, odd)
    want, size = x.double() @ weights.t(), x.double().abs() @ weights.abs().t()
    assert ((got - want).abs() <= 2 * (inputs + 8) * U * size + (1.01 * H * want.abs() if dtype == "bf16" else 0)).all()
