"""Routed products as a program may call them: arrays of R replaced, routes used inside captures, captures that fork."""
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


def test_route_made_before_a_capture():
    # a graph reads the route's arrays and R's values at every replay: values and inputs may change in place between replays
    R = make_route(300, 6, 4, 3, drop=0.1)
    route = gm.route_plan(R)
    X, W = randn((300, 200), BF16, 1), randn((6, 136, 200), BF16, 2)
    G = randn((300, 136), BF16, 3)

    def step():
        P = gm.route_product(route, X, W)
        Y = gm.route_sum(route, P)
        dP, dval = gm.route_sum_grads(route, G, P)
        return P, Y, dP, dval, gm.route_product_dx(route, dP, W), gm.route_product_dw(route, dP, X)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for k in range(3):
        R.val.mul_(-0.5)
        X.copy_(randn((300, 200), BF16, 10 + k))
        for t in out:
            t.fill_(float("nan"))
        graph.replay()
        assert all(torch.equal(a, b) for a, b in zip(out, step())), k
    torch.cuda.synchronize()
    route.status()


def test_captures_that_fork_and_join():
    # kernels that may begin while the one before them ends, with more than one before them: behind a fork, behind a join, behind other kernels and a memset
    R = make_route(400, 6, 4, 5, drop=0.1)
    X, W, G = randn((400, 200), BF16, 1), randn((6, 136, 200), BF16, 2), randn((400, 136), BF16, 3)
    side = torch.cuda.Stream()

    def step():
        main = torch.cuda.current_stream()
        route = gm.route_plan(R)
        side.wait_stream(main)
        with torch.cuda.stream(side):
            Xq, Xs = gm.block_quantize(X)
            Wq, Ws = gm.block_quantize(W, 128)
            Q = gm.route_product_scaled(route, Xq, Xs, Wq, Ws)
            Z = gm.route_sum(route, Q)
        P = gm.route_product(route, X, W)
        dP, dval = gm.route_sum_grads(route, G, P)
        main.wait_stream(side)
        dW = gm.route_product_dw(route, (dP + Q), X)  # behind both
        Y = gm.route_sum(route, P + Q)
        side.wait_stream(main)
        with torch.cuda.stream(side):
            dX = gm.route_product_dx(route, dP, W)
        A = torch.zeros_like(Y)
        A.add_(Y)
        main.wait_stream(side)
        return P, Q, Z, dP, dval, dW, Y, dX, A, gm.block_quantize(A)[0].float()

    want = [t.clone() for t in step()]
    torch.cuda.synchronize()
    assert torch.equal(want[6], want[8])
    for _ in range(5):
        got = step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for _ in range(10):
        for t in out:
            t.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want))
