"""Routed products as a program may call them: arrays of R replaced."""
import pytest
import torch

import paper_2607_22866_b200 as gm
from test_gpu_routed import BF16, make_route, randn

pytestmark = pytest.mark.gpu


def refused(call):
    with pytest.raises(gm.GmError) as e:
        call()
    assert e.value.status == -1


def test_replaced_arrays_of_r_are_refused_where_they_are_read():
    R = make_route(50, 4, 3, 1)
    route = gm.route_plan(R)
    P, W = randn((R.nnz, 64), BF16, 2), randn((4, 64, 32), BF16, 3)
    G = randn((50, 64), BF16, 4)
    dX = gm.route_product_dx(route, P, W)
    plain = gm.route_sum(route, P, weighted=False)
    val, row_ptr = R.val, R.row_ptr
    R.val = torch.zeros_like(val)
    refused(lambda: gm.route_sum(route, P))
    refused(lambda: gm.route_sum_grads(route, G, P))
    assert torch.equal(gm.route_sum(route, P, weighted=False), plain) and torch.equal(gm.route_product_dx(route, P, W), dX)  # (read no values)
    R.val = val
    want = gm.route_sum(route, P)
    R.row_ptr = row_ptr.clone()
    refused(lambda: gm.route_sum(route, P))
    refused(lambda: gm.route_sum(route, P, weighted=False))
    refused(lambda: gm.route_sum_grads(route, G, P))
    refused(lambda: gm.route_product_dx(route, P, W))
    gm.route_product_dx(route, P, W, by_entry=True)  # (reads neither)
    R.row_ptr = row_ptr
    assert torch.equal(gm.route_sum(route, P), want)
    # the same tensor with other memory
    R.val.data = torch.ones_like(val)
    refused(lambda: gm.route_sum(route, P))
