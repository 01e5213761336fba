"""Routed products: the quantiser's rounding over all values of its types, gradients against differences, direction by direction."""
import pytest
import torch

import paper_2607_22866_b200 as gm
from test_gpu_routed import BF16, F16, F32, make_route, quantize_reference

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


def test_gradients_are_the_differences():
    # L = <G, sum of r * (X W^T)> is linear in X, in W and in the r: (L(+d) - L(-d)) / 2 is <gradient, d>.  Small whole numbers (and weights that are
    # powers of two) make every product, sum and rounding on the way exact, so both sides are equal, for single elements as for whole directions.
    n, E, K, N = 60, 5, 48, 40
    R = make_route(n, E, 3, 2, drop=0.1)
    g = torch.Generator(device="cuda").manual_seed(3)
    whole = lambda shape, most: torch.randint(-most, most + 1, shape, generator=g, device="cuda").float()  # noqa: E731
    R.val.copy_(torch.tensor([-2.0, -1.0, 0.5, 1.0], device="cuda")[torch.randint(0, 4, R.val.shape, generator=g, device="cuda")])
    X, W, G = whole((n, K), 3), whole((E, N, K), 3), whole((n, N), 2)
    route = gm.route_plan(R)

    def loss(X, W, val):
        route = gm.route_plan(gm.DeviceCSR(n, E, R.row_ptr, R.col, val))
        P = gm.route_product(route, X.to(BF16), W.to(BF16), dtype=F32)
        return float((gm.route_sum(route, P).double() * G.double()).sum())

    P = gm.route_product(route, X.to(BF16), W.to(BF16), dtype=F32)
    dP, dval = gm.route_sum_grads(route, G, P)
    assert torch.equal(dP.to(BF16).float(), dP)
    dX = gm.route_product_dx(route, dP.to(BF16), W.to(BF16), dtype=F32)
    dW = gm.route_product_dw(route, dP.to(BF16), X.to(BF16), dtype=F32)
    for name, grad, at in (("X", dX, X), ("W", dW, W), ("val", dval, R.val)):
        some = torch.randperm(at.numel(), generator=g, device="cuda")[:40]
        directions = [whole(at.shape, 1)] + [torch.zeros(at.numel(), device="cuda").index_fill(0, i, 1.0).view(at.shape) for i in some]
        nonzero = 0
        for d in directions:
            args = lambda v: (v if name == "X" else X, v if name == "W" else W, v if name == "val" else R.val)  # noqa: E731
            diff = (loss(*args(at + d)) - loss(*args(at - d))) / 2
            assert diff == float((grad.double() * d.double()).sum()), name
            nonzero += diff != 0
        assert nonzero > 20, name
