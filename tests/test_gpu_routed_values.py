"""Routed products: the quantiser's rounding over all values of its types."""
import pytest
import torch

import paper_2607_22866_b200 as gm
from test_gpu_routed import BF16, F16, quantize_reference

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows", [1, 128])
@pytest.mark.parametrize("dtype", [BF16, F16])
def test_quantize_all_values_under_many_maxima(dtype, rows):
    # every finite value of the type, of either sign, in a block whose largest magnitude is m, for maxima m from the least to the largest: the
    # definition is of exact quotients, so values and scales are those of the formula, ties included
    every = torch.arange(65536, dtype=torch.int32, device="cuda").to(torch.int16).view(dtype)
    every = every[every.isfinite()]
    size = every.double().abs()
    positive = every[every.double() > 0]
    most = torch.cat([positive[:: 97 if dtype == BF16 else 61], positive[-1:]])
    per = 128 * rows - 1
    codes, small = set(), 0
    for m in most:
        under = every[size <= float(m)]
        under = under[torch.randperm(under.numel(), generator=torch.Generator(device="cuda").manual_seed(1), device="cuda")]
        under = torch.nn.functional.pad(under, (0, -under.numel() % per)).view(-1, per)
        X = torch.cat([m.expand(under.shape[0], 1), under], 1).view(-1, rows, 128).view(-1, 128)
        Q, S = gm.block_quantize(X, rows)
        q, s = quantize_reference(X, rows)
        assert torch.equal(Q.double(), q), float(m)
        assert bool(((S.double() - s).abs() <= 2.0 ** -24 * s).all()), float(m)
        ratio = X.double() / float(m)
        small += int(((ratio < 0) & (ratio > -2.0 ** -19)).any() and ((ratio > 0) & (ratio < 2.0 ** -19)).any())
        codes.update(Q.double().unique().tolist())
    assert len(codes) == 2 * 126 + 1  # every finite value of e4m3 came out, of both signs (the zeros count once)
    assert small > 100                # blocks that go down to what rounds to zero: 448 x 2^-19 is less than half the least step, 2^-10
