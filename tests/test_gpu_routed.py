"""Routed products against their formulas in 64 bits: routes, products and their gradients, sums over entries, 8-bit forms.

Tolerances.  A result of type T is rounded once: at most eps_T / 2 of its size.  Before that, sums of n terms are kept in 32 bits; every
addition is off by at most one unit of the last place of a partial sum (a matrix unit may cut off instead of rounding), so by at
most n * 2^-23 * sum |terms| altogether.  f16 results below its smallest normal number are off by at most half its smallest step, 2^-25.
"""
import os
import subprocess
import sys
import threading

import numpy as np
import pytest
import torch

import paper_2607_22866_b200 as gm

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32


def make_route(n, E, k, seed, drop=0.0, empty=0.0, skew=0.0):
    """A CSR matrix with rows of 0 .. k entries, columns in any order and sometimes twice, some of them outside [0, E)."""
    rng = np.random.default_rng(seed)
    length = rng.integers(0, k + 1, n) if k > 1 else np.ones(n, dtype=np.int64)
    length[rng.random(n) < empty] = 0
    p = (1.0 + np.arange(E)) ** -skew
    col = rng.choice(E, int(length.sum()), p=p / p.sum()).astype(np.int32)
    out = rng.random(col.size) < drop
    col[out] = rng.choice(np.array([-1, E, -2**31, 2**31 - 1]), int(out.sum()))
    row_ptr = np.concatenate([[0], np.cumsum(length)]).astype(np.int64)
    val = rng.uniform(-1, 1, col.size).astype(np.float32)
    return gm.DeviceCSR(n, E, torch.from_numpy(row_ptr).cuda(), torch.from_numpy(col).cuda(), torch.from_numpy(val).cuda())


def reference_route(R):
    row_ptr, col = R.row_ptr.cpu().numpy(), R.col.cpu().numpy()
    row = np.repeat(np.arange(R.n_rows), np.diff(row_ptr))
    key = np.where((col >= 0) & (col < R.n_cols), col, R.n_cols)
    order = np.argsort(key, kind="stable")
    offsets = np.searchsorted(key[order], np.arange(R.n_cols + 1))
    pos = np.empty_like(order)
    pos[order] = np.arange(order.size)
    return row, key, order, offsets, pos


def check_route(R, route):
    row, key, order, offsets, pos = reference_route(R)
    assert np.array_equal(route.offsets.cpu().numpy(), offsets)
    assert np.array_equal(route.order.cpu().numpy(), order)
    assert np.array_equal(route.rows.cpu().numpy(), row[order])
    assert np.array_equal(route.pos.cpu().numpy(), pos)


def randn(shape, dtype, seed, scale=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(shape, generator=g, device="cuda") * scale).to(dtype)


def close(got, ref, magnitude, terms):
    """Every element within the rounding of its type and of `terms` additions whose absolute values sum to `magnitude`."""
    eps = torch.finfo(got.dtype).eps / 2 if got.dtype != F32 else 2.0 ** -24
    least = 2.0 ** -25 if got.dtype == F16 else 0.0
    err = (got.double() - ref).abs()
    # (the rounding is of the computed sum, which the second term may have moved)
    bound = terms * 2.0 ** -23 * magnitude * (1 + eps) + eps * ref.abs() + least
    assert got.shape == ref.shape
    assert bool((err <= bound).all()), f"off by {float((err - bound).max())} more than {float(bound.max())} allowed"


def product_reference(R, X, W, by_entry):
    """P, and the sum of the absolute terms."""
    row, key, order, offsets, _ = reference_route(R)
    N = W.shape[1]
    P = torch.zeros(order.size, N, dtype=torch.float64, device="cuda")
    A = torch.zeros_like(P)
    for e in range(R.n_cols):
        a, b = int(offsets[e]), int(offsets[e + 1])
        if a < b:
            x = X[a:b].double() if by_entry else X[torch.from_numpy(row[order[a:b]]).cuda()].double()
            P[a:b] = x @ W[e].double().T
            A[a:b] = x.abs() @ W[e].double().abs().T
    return P, A


ROUTES = [  # n, E, k, drop, empty, skew
    (1, 1, 1, 0.0, 0.0, 0.0), (1, 7, 5, 0.0, 0.0, 0.0), (3, 40, 4, 0.2, 0.3, 0.0), (0, 3, 2, 0.0, 0.0, 0.0), (5, 3, 2, 1.0, 0.0, 0.0),
    (64, 8, 3, 0.1, 0.5, 1.0), (700, 5, 3, 0.05, 0.1, 2.0), (1025, 1, 1, 0.0, 0.0, 0.0), (2000, 33, 6, 0.0, 0.0, 0.7), (40, 2048, 8, 0.1, 0.0, 0.0),
    (30000, 130, 9, 0.1, 0.1, 1.0), (20000, 100, 9, 0.1, 0.1, 1.0), (70000, 1, 1, 0.3, 0.0, 0.0), (300000, 128, 1, 0.0, 0.6, 0.0), (5000, 2048, 9, 0.01, 0.0, 0.5), (100, 600, 300, 0.0, 0.9, 0.0),
]


@pytest.mark.parametrize("n,E,k,drop,empty,skew", ROUTES)
def test_route(n, E, k, drop, empty, skew):
    R = make_route(n, E, k, 11 + n, drop, empty, skew)
    check_route(R, gm.route_plan(R))


def test_route_of_no_columns():
    R = gm.DeviceCSR(4, 0, torch.tensor([0, 1, 1, 3, 3], device="cuda"), torch.tensor([0, -1, 5], dtype=torch.int32, device="cuda"), torch.ones(3, device="cuda"))
    route = gm.route_plan(R)
    check_route(R, route)
    X = randn((4, 16), BF16, 1)
    assert not gm.route_product(route, X, torch.empty(0, 24, 16, dtype=BF16, device="cuda")).any()
    assert not gm.route_sum(route, randn((3, 24), BF16, 2)).any()
    assert gm.route_product_dw(route, randn((3, 24), BF16, 3), X).shape == (0, 24, 16)


# n, E, k, N, K: one place, tile borders in every direction, odd widths (copied first), several parts of a column
PRODUCTS = [
    (1, 1, 1, 8, 8), (1, 6, 5, 1, 64), (3, 40, 4, 130, 72), (257, 1, 1, 128, 64), (700, 5, 3, 129, 200), (64, 8, 3, 40, 1), (50, 3, 2, 33, 77),
    (900, 2, 2, 384, 264), (1, 3, 3, 256, 2048), (2500, 17, 4, 96, 128), (16, 2, 1, 2, 8200), (5, 3, 2, 0, 16), (5, 3, 2, 16, 0),
]


@pytest.mark.parametrize("dtype,out", [(BF16, BF16), (F16, F16), (BF16, F32), (F16, BF16)])
@pytest.mark.parametrize("by_entry", [False, True])
@pytest.mark.parametrize("n,E,k,N,K", PRODUCTS)
def test_product(n, E, k, N, K, by_entry, dtype, out):
    R = make_route(n, E, k, 3 * n + K, drop=0.1, empty=0.1, skew=0.5)
    route = gm.route_plan(R)
    X, W = randn((R.nnz if by_entry else n, K), dtype, 1), randn((E, N, K), dtype, 2)
    P = gm.route_product(route, X, W, by_entry, dtype=out)
    ref, mag = product_reference(R, X, W, by_entry)
    assert P.dtype == out
    close(P, ref, mag, K)
    assert torch.equal(P, gm.route_product(route, X, W, by_entry, dtype=out))  # the same call, the same bits
    torch.cuda.synchronize()
    route.status()


def dx_reference(R, dP, W, by_entry):
    row, key, order, offsets, _ = reference_route(R)
    T = torch.zeros(order.size, W.shape[2], dtype=torch.float64, device="cuda")
    A = torch.zeros_like(T)
    for e in range(R.n_cols):
        a, b = int(offsets[e]), int(offsets[e + 1])
        T[a:b] = dP[a:b].double() @ W[e].double()
        A[a:b] = dP[a:b].double().abs() @ W[e].double().abs()
    if by_entry:
        return T, A
    rows = torch.from_numpy(row[order]).cuda()
    zero = torch.zeros(R.n_rows, W.shape[2], dtype=torch.float64, device="cuda")
    return zero.index_add(0, rows, T), zero.index_add(0, rows, A)


@pytest.mark.parametrize("dtype,out", [(BF16, BF16), (F16, F16), (BF16, F32)])
@pytest.mark.parametrize("by_entry", [False, True])
@pytest.mark.parametrize("n,E,k,N,K", PRODUCTS)
def test_product_dx(n, E, k, N, K, by_entry, dtype, out):
    R = make_route(n, E, k, 5 * n + K, drop=0.1, empty=0.1, skew=0.5)
    route = gm.route_plan(R)
    dP, W = randn((R.nnz, N), dtype, 1), randn((E, N, K), dtype, 2)
    dP[int(route.offsets[-1]):] = float("nan")  # routed nowhere: not looked at
    dX = gm.route_product_dx(route, dP, W, by_entry, dtype=out)
    ref, mag = dx_reference(R, dP, W, by_entry)
    assert dX.dtype == out
    close(dX, ref, mag, N + k)
    torch.cuda.synchronize()
    route.status()


def dw_reference(R, dP, X, by_entry):
    row, key, order, offsets, _ = reference_route(R)
    dW = torch.zeros(R.n_cols, dP.shape[1], X.shape[1], dtype=torch.float64, device="cuda")
    A = torch.zeros_like(dW)
    for e in range(R.n_cols):
        a, b = int(offsets[e]), int(offsets[e + 1])
        x = X[a:b].double() if by_entry else X[torch.from_numpy(row[order[a:b]]).cuda()].double()
        dW[e] = dP[a:b].double().T @ x
        A[e] = dP[a:b].double().abs().T @ x.abs()
    return dW, A, int(np.diff(offsets).max())


@pytest.mark.parametrize("dtype,out", [(BF16, BF16), (F16, F16), (BF16, F32)])
@pytest.mark.parametrize("by_entry", [False, True])
@pytest.mark.parametrize("n,E,k,N,K", PRODUCTS)
def test_product_dw(n, E, k, N, K, by_entry, dtype, out):
    R = make_route(n, E, k, 7 * n + K, drop=0.1, empty=0.1, skew=0.5)
    route = gm.route_plan(R)
    dP, X = randn((R.nnz, N), dtype, 1), randn((R.nnz if by_entry else n, K), dtype, 2)
    ref, mag, most = dw_reference(R, dP, X, by_entry)
    dP[int(route.offsets[-1]):] = float("nan")
    dW = gm.route_product_dw(route, dP, X, by_entry, dtype=out)
    assert dW.dtype == out
    close(dW, ref, mag, most)
    torch.cuda.synchronize()
    route.status()


def test_neighbours_with_nan_and_infinities_stay_apart():
    # a column's rows of P, X and dP lie next to another's in memory: what is not finite there must not get across
    R = gm.DeviceCSR(40, 2, torch.arange(41, device="cuda"), torch.tensor([0, 1] * 20, dtype=torch.int32, device="cuda"), torch.ones(40, device="cuda"))
    route = gm.route_plan(R)
    X, W, dP = randn((40, 72), BF16, 1), randn((2, 136, 72), BF16, 2), randn((40, 136), BF16, 3)
    bad_x, bad_w, bad_p = X.clone(), W.clone(), dP.clone()
    bad_x[1::2] = float("nan")
    bad_w[1] = float("inf")
    bad_p[20:] = float("-inf")
    good = lambda a, b: torch.equal(a, b) and bool(a.isfinite().all())  # noqa: E731
    assert good(gm.route_product(route, bad_x, bad_w)[:20], gm.route_product(route, X, W)[:20])
    assert good(gm.route_product_dx(route, bad_p, bad_w)[0::2], gm.route_product_dx(route, dP, W)[0::2])
    assert good(gm.route_product_dw(route, bad_p, bad_x)[0], gm.route_product_dw(route, dP, X)[0])
    by_place = bad_x[route.rows.long()]
    assert good(gm.route_product_dw(route, bad_p, by_place, True)[0], gm.route_product_dw(route, dP, X)[0])
    assert good(gm.route_product(route, by_place, bad_w, True)[:20], gm.route_product(route, X, W)[:20])


def layouts(t):
    """The same values with other strides."""
    yield "transposed", t.transpose(-1, -2).contiguous().transpose(-1, -2)
    wide = torch.zeros(*t.shape[:-1], t.shape[-1] + 8, dtype=t.dtype, device=t.device)
    wide[..., :-8] = t
    yield "padded rows", wide[..., :-8]
    wide = torch.zeros(*t.shape[:-1], t.shape[-1] + 3, dtype=t.dtype, device=t.device)
    wide[..., 3:] = t
    yield "off by three", wide[..., 3:]
    every = torch.zeros(*t.shape[:-1], 2 * t.shape[-1], dtype=t.dtype, device=t.device)
    every[..., ::2] = t
    yield "every other", every[..., ::2]


def test_strides():
    R = make_route(90, 4, 3, 5, drop=0.1)
    route = gm.route_plan(R)
    X, W, dP = randn((90, 136), BF16, 1), randn((4, 152, 136), BF16, 2), randn((R.nnz, 152), BF16, 3)
    P, dX, dW = gm.route_product(route, X, W), gm.route_product_dx(route, dP, W), gm.route_product_dw(route, dP, X)
    for name, w in layouts(W):
        assert torch.equal(w, W) and torch.equal(gm.route_product(route, X, w), P), name
        assert torch.equal(gm.route_product_dx(route, dP, w), dX), name
    for name, x in layouts(X):
        assert torch.equal(gm.route_product(route, x, W), P) and torch.equal(gm.route_product_dw(route, dP, x), dW), name
    for name, d in layouts(dP):
        assert torch.equal(gm.route_product_dx(route, d, W), dX) and torch.equal(gm.route_product_dw(route, d, X), dW), name
    # one block for all columns, one row for all rows
    assert torch.equal(gm.route_product(route, X, W[:1].expand(4, -1, -1)), gm.route_product(route, X, W[:1].repeat(4, 1, 1)))
    assert torch.equal(gm.route_product(route, X[:1].expand(90, -1), W), gm.route_product(route, X[:1].repeat(90, 1), W))


def test_unusual_layouts():
    R = make_route(90, 4, 3, 5, drop=0.1)
    route = gm.route_plan(R)
    X, dP = randn((90, 136), BF16, 1), randn((R.nnz, 152), BF16, 3)
    W = randn((152, 4, 136), BF16, 2).transpose(0, 1)  # blocks between each other's rows
    V = W.contiguous()
    assert torch.equal(gm.route_product(route, X, W), gm.route_product(route, X, V))
    assert torch.equal(gm.route_product_dx(route, dP, W), gm.route_product_dx(route, dP, V))
    W = randn((136, 152, 4), BF16, 2).permute(2, 1, 0)  # blocks innermost
    V = W.contiguous()
    assert torch.equal(gm.route_product(route, X, W), gm.route_product(route, X, V))
    assert torch.equal(gm.route_product_dx(route, dP, W), gm.route_product_dx(route, dP, V))
    long = randn((90 * 8 + 136,), BF16, 4)  # rows that share most of their values
    X = long.as_strided((90, 136), (8, 1))
    P = gm.route_product(route, X, V)
    assert torch.equal(P, gm.route_product(route, X.contiguous(), V))
    G = long.as_strided((R.nnz, 136), (8, 1)) if R.nnz <= 90 else torch.cat([long, long]).as_strided((R.nnz, 136), (8, 1))
    assert torch.equal(gm.route_product(route, G, V, True), gm.route_product(route, G.contiguous(), V, True))
    assert torch.equal(gm.route_product_dw(route, G, X), gm.route_product_dw(route, G.contiguous(), X.contiguous()))
    assert torch.equal(gm.route_product_dw(route, G, G, True), gm.route_product_dw(route, G.contiguous(), G.contiguous(), True))
    for rows in (1, 128):
        for a, b in zip(gm.block_quantize(X, rows), gm.block_quantize(X.contiguous(), rows)):
            assert torch.equal(a.float(), b.float())


SUMS = [(1, 1, 1, 1), (1, 9, 5, 4096), (3, 40, 4, 130), (700, 5, 3, 1032), (64, 8, 9, 77), (300, 16, 6, 24), (5, 3, 2, 0), (20, 600, 300, 16), (0, 3, 2, 8)]


@pytest.mark.parametrize("dtype,out", [(BF16, BF16), (F16, F16), (F32, F32), (F32, BF16), (BF16, F32)])
@pytest.mark.parametrize("weighted", [True, False])
@pytest.mark.parametrize("n,E,k,N", SUMS)
def test_sum(n, E, k, N, weighted, dtype, out):
    R = make_route(n, E, k, 13 * n + N, drop=0.1, empty=0.2)
    route = gm.route_plan(R)
    P = randn((R.nnz, N), dtype, 4)
    P[int(route.offsets[-1]):] = float("nan")
    row, key, order, offsets, pos = reference_route(R)
    ok = torch.from_numpy(key < E).cuda()
    rows, at = torch.from_numpy(row).cuda()[ok], torch.from_numpy(pos).cuda()[ok]
    w = R.val.double()[ok] if weighted else torch.ones(int(ok.sum()), dtype=torch.float64, device="cuda")
    zero = torch.zeros(n, N, dtype=torch.float64, device="cuda")
    ref = zero.index_add(0, rows, w[:, None] * P[at].double())
    mag = zero.index_add(0, rows, (w[:, None] * P[at].double()).abs())
    close(gm.route_sum(route, P, weighted, dtype=out), ref, mag, k)


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("n,E,k,N", SUMS)
def test_sum_grads(n, E, k, N, dtype):
    R = make_route(n, E, k, 17 * n + N, drop=0.1, empty=0.2)
    route = gm.route_plan(R)
    P, dY = randn((R.nnz, N), dtype, 4), randn((n, N), dtype, 5)
    P[int(route.offsets[-1]):] = float("nan")
    dP, dval = gm.route_sum_grads(route, dY, P)
    row, key, order, offsets, pos = reference_route(R)
    ok = torch.from_numpy(key < E).cuda()
    rows, pos = torch.from_numpy(row).cuda(), torch.from_numpy(pos).cuda()
    terms = torch.where(ok[:, None], dY[rows].double() * P[pos].double(), 0.0)
    close(dval, terms.sum(1), terms.abs().sum(1), N)
    ref = torch.zeros(R.nnz, N, dtype=torch.float64, device="cuda")
    ref[pos] = torch.where(ok[:, None], R.val.double()[:, None] * dY[rows].double(), 0.0)
    close(dP, ref, ref.abs(), 1)


def test_sum_strides():
    R = make_route(90, 4, 3, 5, drop=0.1)
    route = gm.route_plan(R)
    P, dY = randn((R.nnz, 136), BF16, 1), randn((90, 136), BF16, 2)
    Y, (dP, dval) = gm.route_sum(route, P), gm.route_sum_grads(route, dY, P)
    same = lambda a, b: torch.equal(a[0], b[0]) and torch.allclose(a[1], b[1], rtol=1e-5, atol=1e-5)  # noqa: E731
    for name, p in layouts(P):  # (rows that are not aligned are added up in another order: the dot products' last bits)
        assert torch.equal(gm.route_sum(route, p), Y) and same(gm.route_sum_grads(route, dY, p), (dP, dval)), name
    for name, g in layouts(dY):
        assert same(gm.route_sum_grads(route, g, P), (dP, dval)), name
    # the gradient of a plain sum is one value repeated
    one = torch.ones((), dtype=BF16, device="cuda")
    assert same(gm.route_sum_grads(route, one.expand(90, 136), P), gm.route_sum_grads(route, one.repeat(90, 136), P))
    assert torch.equal(gm.route_sum(route, one.expand(R.nnz, 136)), gm.route_sum(route, one.repeat(R.nnz, 136)))


def test_gradients_against_differences():
    # L = <G, sum of r * (X W^T)>: along a random direction, (L(+h) - L(-h)) / 2h is linear in each argument, so exact up to rounding
    n, E, K, N = 60, 5, 48, 40
    R = make_route(n, E, 3, 2, drop=0.1)
    route = gm.route_plan(R)
    X, W, G = randn((n, K), BF16, 1), randn((E, N, K), BF16, 2), randn((n, N), F32, 3)
    P = gm.route_product(route, X, W, dtype=F32)
    dP, dval = gm.route_sum_grads(route, G, P)
    half = dP.to(BF16)
    dX, dW = gm.route_product_dx(route, half, W, dtype=F32), gm.route_product_dw(route, half, X, dtype=F32)

    def loss(X, W, val):
        route = gm.route_plan(gm.DeviceCSR(n, E, R.row_ptr, R.col, val))
        return float((gm.route_sum(route, gm.route_product(route, X, W, dtype=F32)).double() * G.double()).sum())

    for name, grad, at in (("X", dX, X), ("W", dW, W), ("val", dval, R.val)):
        d = randn(at.shape, F32, 9).sign()
        up, down = ((at.double() + s * 0.25 * d).to(at.dtype) for s in (1, -1))
        h = (up.double() - down.double()) / 2  # what the rounded arguments differ by
        args = lambda v: (v if name == "X" else X, v if name == "W" else W, v if name == "val" else R.val)  # noqa: E731
        diff = (loss(*args(up)) - loss(*args(down))) / 2
        want = float((grad.double() * h).sum())
        # each term of `want` is off by the rounding of dP to 8 bits (2^-9 of it, independent signs would give far less), and both sums
        # by the 32-bit roundings: bound them by the sum of absolute values
        scale = float((G.double().abs()[torch.from_numpy(reference_route(R)[0]).cuda()] * R.val.double().abs()[:, None]).sum())
        size = float((X.double().abs().max() * W.double().abs().max())) * K * scale
        slack = (2.0 ** -9 if name != "val" else 0.0) * float((grad.double().abs() * h.abs()).sum()) * 8 + 2.0 ** -22 * size
        assert abs(diff - want) <= slack, (name, diff, want, slack)


def e4m3(y):
    step = torch.ldexp(torch.ones_like(y), (torch.frexp(y).exponent - 1).clamp(min=-6) - 3)
    return torch.round(y / step) * step


def quantize_reference(X, rows):
    x = X.double() if X.dim() == 3 else X.double()[None]
    B, N, K = x.shape
    finite = torch.where(x.isfinite(), x, 0.0)
    pad = torch.nn.functional.pad(finite, (0, -K % 128, 0, -N % rows)).view(B, -(-N // rows), rows, -(-K // 128), 128)
    most = pad.abs().amax((2, 4)).clamp(min=2.0 ** -100)
    wide = most.repeat_interleave(rows, 1)[:, :N].repeat_interleave(128, 2)[:, :, :K]
    q = torch.where(x.isfinite(), e4m3(finite * 448 / wide), float("nan"))
    return q.view(X.shape), (most / 448).view(*X.shape[:-2], most.shape[1], most.shape[2])


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("rows", [1, 128])
@pytest.mark.parametrize("shape", [(1, 1), (1, 128), (3, 136), (128, 128), (129, 264), (2, 77, 1000), (5, 200, 131), (3, 0, 16), (2, 16, 0), (3, 300, 512)])
def test_quantize(shape, rows, dtype):
    X = randn(shape, dtype, 6)
    if X.numel():
        X *= torch.exp(2 * randn((1, shape[-1]), F32, 7)).to(dtype)
        X.view(-1)[0] = 0.0
    Q, S = gm.block_quantize(X, rows)
    q, s = quantize_reference(X, rows)
    assert Q.dtype == torch.float8_e4m3fn and Q.shape == X.shape and S.shape == s.shape
    assert torch.equal(Q.double(), q)  # ties included: the definition is of exact quotients
    assert bool(((S.double() - s).abs() <= 2.0 ** -24 * s).all())


@pytest.mark.parametrize("dtype", [BF16, F16])
def test_quantize_every_value(dtype):
    # all finite values of the type next to each of many maxima: no quotient lands on the wrong side of a border
    bits = torch.arange(65536, dtype=torch.int32, device="cuda").to(torch.int16)
    every = bits.view(dtype)
    every = every[every.isfinite()]
    most = every[(every.double().abs() > 0)].abs().unique()[:: 97 if dtype == BF16 else 61]
    blocks = []
    for m in most:
        under = every[every.abs() <= m][-127 * 24:]  # (the last ones reach up to the maximum, with both signs among them)
        under = under[torch.randperm(under.numel(), generator=torch.Generator(device="cuda").manual_seed(1), device="cuda")]
        under = torch.nn.functional.pad(under, (0, -under.numel() % 127)).view(-1, 127)
        blocks.append(torch.cat([m.expand(under.shape[0], 1), under], 1))
    X = torch.cat(blocks)
    Q, S = gm.block_quantize(X, 1)
    q, s = quantize_reference(X, 1)
    assert torch.equal(Q.double(), q)


def test_quantize_values_that_are_not_finite():
    X = randn((4, 300), BF16, 1)
    X[0, 5], X[1, 200], X[2] = float("inf"), float("nan"), float("-inf")
    for rows in (1, 128):
        Q, S = gm.block_quantize(X, rows)
        q, s = quantize_reference(X, rows)
        assert torch.equal(Q.double().isnan(), q.isnan()) and torch.equal(Q.double().nan_to_num(), q.nan_to_num())
        assert bool(S.isfinite().all()) and torch.allclose(S.double(), s, rtol=2.0 ** -23, atol=0)


def test_quantize_strides():
    X = randn((3, 140, 264), BF16, 1)
    for rows in (1, 128):
        Q, S = gm.block_quantize(X, rows)
        for name, x in layouts(X):
            q, s = gm.block_quantize(x, rows)
            assert torch.equal(q.float(), Q.float()) and torch.equal(s, S), name


SCALED = [
    (1, 1, 1, 8, 16), (1, 6, 5, 1, 128), (3, 40, 4, 130, 144), (257, 1, 1, 128, 256), (700, 5, 3, 129, 400), (64, 8, 3, 40, 1), (50, 3, 2, 33, 77),
    (900, 2, 2, 384, 1040), (1, 3, 3, 256, 2048), (2500, 17, 4, 96, 640), (5, 3, 2, 0, 16), (5, 3, 2, 16, 0),
]


@pytest.mark.parametrize("out", [BF16, F16, F32])
@pytest.mark.parametrize("rows", [1, 128])
@pytest.mark.parametrize("by_entry", [False, True])
@pytest.mark.parametrize("n,E,k,N,K", SCALED)
def test_product_scaled(n, E, k, N, K, by_entry, rows, out):
    R = make_route(n, E, k, 19 * n + K, drop=0.1, empty=0.1, skew=0.5)
    route = gm.route_plan(R)
    X, W = randn((R.nnz if by_entry else n, K), BF16, 1), randn((E, N, K), BF16, 2, 0.3)
    if K:
        X *= torch.exp(randn((1, K), F32, 7)).to(BF16)
    (Xq, Xs), (Wq, Ws) = gm.block_quantize(X, 1), gm.block_quantize(W, rows)
    P = gm.route_product_scaled(route, Xq, Xs, Wq, Ws, by_entry, dtype=out)
    x = Xq.double() * Xs.double().repeat_interleave(128, 1)[:, :K]
    w = Wq.double() * Ws.double().repeat_interleave(128, 2)[:, :, :K].repeat_interleave(rows, 1)[:, :N]
    ref, mag = product_reference(R, x, w, by_entry)
    # the products with the scales add three roundings to each block's sum
    close(P, ref, mag, K + 3)
    assert torch.equal(P, gm.route_product_scaled(route, Xq, Xs, Wq, Ws, by_entry, dtype=out))
    torch.cuda.synchronize()
    route.status()


def test_scaled_strides():
    R = make_route(90, 4, 3, 5, drop=0.1)
    route = gm.route_plan(R)
    for rows in (1, 128):
        (Xq, Xs), (Wq, Ws) = gm.block_quantize(randn((90, 272), BF16, 1)), gm.block_quantize(randn((4, 152, 272), BF16, 2), rows)
        P = gm.route_product_scaled(route, Xq, Xs, Wq, Ws)
        for k, t in enumerate((Xq, Xs, Wq, Ws)):
            for name, other in layouts(t.view(torch.uint8) if k in (0, 2) else t):
                args = [Xq, Xs, Wq, Ws]
                args[k] = other.view(torch.float8_e4m3fn) if k in (0, 2) else other
                assert torch.equal(gm.route_product_scaled(route, *args), P), (k, name)


def layer(R, X, W1, W2, G):
    """Forward and backward of a layer: two routed products with a gate between them, weighted sum, all gradients."""
    route = gm.route_plan(R)
    H = gm.route_product(route, X, W1)
    A = torch.nn.functional.silu(H.float())
    B = A.to(X.dtype)
    P = gm.route_product(route, B, W2, by_entry=True)
    Y = gm.route_sum(route, P)
    dP, dval = gm.route_sum_grads(route, G, P)
    dB = gm.route_product_dx(route, dP, W2, by_entry=True)
    dW2 = gm.route_product_dw(route, dP, B, by_entry=True)
    s = torch.sigmoid(H.float())
    dH = (dB.float() * (s * (1 + H.float() * (1 - s)))).to(X.dtype)
    return Y, dval, gm.route_product_dx(route, dH, W1), gm.route_product_dw(route, dH, X), dW2


def layer_inputs(seed, n=150, E=6, d=72, h=104):
    R = make_route(n, E, 3, seed, drop=0.05)
    return R, randn((n, d), BF16, seed + 1), randn((E, h, d), BF16, seed + 2, d ** -0.5), randn((E, d, h), BF16, seed + 3, h ** -0.5), randn((n, d), BF16, seed + 4)


def test_layer():
    R, X, W1, W2, G = layer_inputs(3)
    got = layer(R, X, W1, W2, G)
    row, key, order, offsets, pos = reference_route(R)
    x, w1, w2, val = (t.double().requires_grad_() for t in (X, W1, W2, R.val))
    Y = torch.zeros(R.n_rows, X.shape[1], dtype=torch.float64, device="cuda")
    for e in range(R.n_cols):
        q = torch.from_numpy(order[offsets[e]: offsets[e + 1]]).cuda()
        rows = torch.from_numpy(row).cuda()[q]
        Y = Y.index_add(0, rows, val[q, None] * (torch.nn.functional.silu(x[rows] @ w1[e].T) @ w2[e].T))
    Y.backward(G.double())
    for name, g, ref in zip(("Y", "dval", "dX", "dW1", "dW2"), got, (Y.detach(), val.grad, x.grad, w1.grad, w2.grad)):
        # up to five roundings to 8 bits (2^-9 of a value, 2^-8 at worst) lie on the way to each result; their effect on it
        # adds up no faster than linearly in the norm
        assert float((g.double() - ref).norm() / ref.norm()) <= 5 * 2.0 ** -8, name


def test_graph_and_streams():
    inputs = [layer_inputs(s) for s in (3, 40)]
    inputs = [(gm.DeviceCSR(150, 6, R.row_ptr[:151].clone(), R.col, R.val), *rest) for R, *rest in inputs]
    want = [[t.clone() for t in layer(*i)] for i in inputs]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):  # on a stream of its own, while the first one works on the other inputs
        there = layer(*inputs[0])
    here = layer(*inputs[1])
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(there, want[0])) and all(torch.equal(a, b) for a, b in zip(here, want[1]))
    graphs = []
    for i in inputs:  # two captured layers, replayed at the same time
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            out = layer(*i)
        graphs.append((g, out))
    for _ in range(3):
        for t in graphs[0][1] + graphs[1][1]:
            t.zero_()
        torch.cuda.synchronize()
        graphs[0][0].replay()
        with torch.cuda.stream(side):
            graphs[1][0].replay()
        torch.cuda.synchronize()
        for (_, out), w in zip(graphs, want):
            assert all(torch.equal(a, b) for a, b in zip(out, w))


def test_given_stream_and_route_of_another():
    R, X, W1, W2, G = layer_inputs(5)
    route = gm.route_plan(R)
    want = gm.route_sum(route, gm.route_product(route, X, W1))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    P = gm.route_product(route, X, W1, stream=side)
    Y = gm.route_sum(route, P, stream=side)
    del route, P
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(Y, want)


def test_host_threads():
    inputs = [layer_inputs(s) for s in (3, 40, 77)]
    want = [[t.clone() for t in layer(*i)] for i in inputs]
    torch.cuda.synchronize()
    wrong = []

    def work(k):
        try:
            with torch.cuda.stream(torch.cuda.Stream()):
                for _ in range(20):
                    got = layer(*inputs[k])
                torch.cuda.current_stream().synchronize()
                if not all(torch.equal(a, b) for a, b in zip(got, want[k])):
                    wrong.append(k)
        except Exception as e:  # pragma: no cover
            wrong.append(e)

    threads = [threading.Thread(target=work, args=(k,)) for k in range(3)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not wrong


def test_dx_with_the_librarys_own_scratch():
    R = make_route(80, 5, 3, 6, drop=0.1)
    route = gm.route_plan(R)
    for K in (64, 77):
        dP, W = randn((R.nnz, 40), BF16, 1), randn((5, 40, K), BF16, 2)
        want, dX = gm.route_product_dx(route, dP, W), torch.full((80, K), 7.0, dtype=BF16, device="cuda")
        b = gm.binding
        d = dX.device
        call = lambda terms: b.load_library().gm_route_product_dx(  # noqa: E731
            route._h, b._dense(dP, "", d), b._dense(W, "", d), 0, b._dense(dX, "", d), terms, torch.cuda.current_stream().cuda_stream)
        assert call(None) == 0 and torch.equal(dX, want)
        assert call(dX.data_ptr() + 2) == -1  # not aligned


def test_values_may_change_between_calls():
    R = make_route(50, 4, 3, 1)
    route = gm.route_plan(R)
    P = randn((R.nnz, 64), F32, 2)
    gm.route_sum(route, P)
    R.val.mul_(2)
    assert torch.equal(gm.route_sum(route, P), gm.route_sum(gm.route_plan(R), P))


@pytest.mark.parametrize("k", [1, 5])
def test_many_columns(k):
    # the most columns there may be, with tiles of few places (k = 1) and of many (k = 5: 75000 entries)
    n, E, N, K = 30000, 2048, 24, 72
    R = make_route(n, E, k, 21, drop=0.02)
    route = gm.route_plan(R)
    X, W = randn((n, K), BF16, 1), randn((E, N, K), BF16, 2)
    ref, mag = product_reference(R, X, W, False)
    close(gm.route_product(route, X, W, dtype=F32), ref, mag, K)
    for rows in (1, 128):
        (Xq, Xs), (Wq, Ws) = gm.block_quantize(X), gm.block_quantize(W, rows)
        x, w = Xq.double() * Xs.double(), Wq.double() * Ws.double().repeat_interleave(rows, 1)[:, :N]
        ref, mag = product_reference(R, x, w, False)
        close(gm.route_product_scaled(route, Xq, Xs, Wq, Ws, dtype=F32), ref, mag, K + 3)
    dP = randn((R.nnz, N), BF16, 3)
    ref, mag, most = dw_reference(R, dP, X, False)
    close(gm.route_product_dw(route, dP, X, dtype=F32), ref, mag, most)
    torch.cuda.synchronize()
    route.status()


def test_offsets_beyond_32_bits():
    # rows of P, X, dP and dW whose elements' numbers pass 2^31 (and whose bytes pass 2^32)
    n, E, N, K = 70000, 3, 32776, 16
    R = make_route(n, E, 1, 4)
    route = gm.route_plan(R)
    X, W = randn((n, K), BF16, 1), randn((E, N, K), BF16, 2)
    P = gm.route_product(route, X, W)
    assert P.numel() > 2**31
    row, key, order, offsets, pos = reference_route(R)
    places = np.r_[0:3, n // 2: n // 2 + 3, n - 300: n]
    some = torch.from_numpy(places).cuda()
    x, e = X[torch.from_numpy(row[order[places]]).cuda()].double(), torch.from_numpy(key[order[places]]).cuda()
    ref = torch.einsum("pk,pnk->pn", x, W[e].double())
    mag = torch.einsum("pk,pnk->pn", x.abs(), W[e].double().abs())
    close(P[some], ref, mag, K)
    # the sums over one entry each are the rows themselves, times a weight
    Y = gm.route_sum(route, P)
    last = torch.arange(n - 300, n, device="cuda")
    rows = route.pos.long()[last]
    ref = R.val.double()[last, None] * P[rows].double()
    close(Y[last], ref, ref.abs(), 1)
    dP, dval = gm.route_sum_grads(route, Y, P)
    ref = Y[last].double() * P[rows].double()
    close(dval[last], ref.sum(1), ref.abs().sum(1), N)
    ref = R.val.double()[last, None] * Y[last].double()
    close(dP[rows], ref, ref.abs(), 1)
    dX = gm.route_product_dx(route, P, W)
    at = torch.arange(n - 50, n, device="cuda")
    e, p = torch.from_numpy(key).cuda()[at], P[route.pos.long()[at]].double()
    close(dX[at], torch.einsum("pn,pnk->pk", p, W[e].double()), torch.einsum("pn,pnk->pk", p.abs(), W[e].double().abs()), N + 1)
    dW = gm.route_product_dw(route, P, X)
    a, b = int(offsets[2]), int(offsets[3])
    x, g = X[torch.from_numpy(row[order[a:b]]).cuda()].double(), P[a:b, -64:].double()
    close(dW[2, -64:], g.T @ x, g.abs().T @ x.abs(), b - a)
    by_place = gm.route_product(route, P[:, :4096], randn((E, 24, 4096), BF16, 5), by_entry=True)  # rows 65552 bytes apart
    again = gm.route_product(route, P[:, :4096].contiguous(), randn((E, 24, 4096), BF16, 5), by_entry=True)
    assert torch.equal(by_place, again)


def test_first_calls_of_a_process_in_a_capture():
    # what the library looks up once for itself does not end a capture; 70 routes at a time need more than one slab of its host memory
    code = """
import torch, paper_2607_22866_b200 as gm
n, E, N, K = 40, 3, 24, 64
rp = torch.arange(n + 1, device="cuda")
R = gm.DeviceCSR(n, E, rp, torch.arange(n, device="cuda", dtype=torch.int32) % E, torch.ones(n, device="cuda"))
X, W = torch.ones(n, K, device="cuda").bfloat16(), torch.ones(E, N, K, device="cuda").bfloat16()
torch.cuda.synchronize()
g = torch.cuda.CUDAGraph()
routes = []
with torch.cuda.graph(g):
    for _ in range(70):
        routes.append(gm.route_plan(R))
    P = gm.route_product(routes[-1], X, W)
    Y = gm.route_sum(routes[-1], P)
    dX = gm.route_product_dx(routes[-1], P, W)
    dW = gm.route_product_dw(routes[-1], P, X)
    Q, S = gm.block_quantize(X)
for t in (P, Y, dX, dW):
    t.zero_()
g.replay()
torch.cuda.synchronize()
assert (P == K).all() and (Y == K).all() and (dX == K * N).all() and dW[0, 0, 0] == K * 14, (P, Y, dX, dW)
"""
    done = subprocess.run([sys.executable, "-c", code], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert done.returncode == 0, done.stderr[-2000:]


def refused(status, call):
    with pytest.raises(gm.GmError) as e:
        call()
    assert e.value.status == status, e.value


def test_refusals():
    INVALID, DIM, DTYPE, CAPACITY = -1, -2, -3, -6
    R = make_route(20, 4, 2, 1)
    route = gm.route_plan(R)
    X, W, P = randn((20, 64), BF16, 1), randn((4, 32, 64), BF16, 2), randn((R.nnz, 32), BF16, 3)
    refused(DIM, lambda: gm.route_product(route, X[:19], W))
    refused(DIM, lambda: gm.route_product(route, X[:, :63], W))
    refused(DIM, lambda: gm.route_product(route, X, W[:3]))
    refused(DIM, lambda: gm.route_product(route, X, W[0]))
    refused(DIM, lambda: gm.route_product(route, X, W, by_entry=True))
    refused(DTYPE, lambda: gm.route_product(route, X.half(), W))
    refused(DTYPE, lambda: gm.route_product(route, X.float(), W.float()))
    refused(DTYPE, lambda: gm.route_product(route, X, W, dtype=torch.float64))
    refused(DTYPE, lambda: gm.route_product(route, X.int(), W))
    refused(INVALID, lambda: gm.route_product(route, X.cpu(), W))
    refused(INVALID, lambda: gm.route_product(route, X, W.cpu()))
    refused(DIM, lambda: gm.route_product_dx(route, P[:-1], W))
    refused(DIM, lambda: gm.route_product_dw(route, P, X[:-1]))
    refused(DIM, lambda: gm.route_sum(route, P[:-1]))
    refused(DTYPE, lambda: gm.route_sum(route, P.double()))
    refused(DTYPE, lambda: gm.route_sum_grads(route, randn((20, 32), F16, 1), P))
    refused(DIM, lambda: gm.route_sum_grads(route, randn((20, 31), BF16, 1), P))
    refused(INVALID, lambda: gm.block_quantize(X, 64))
    refused(DTYPE, lambda: gm.block_quantize(X.float()))
    refused(DIM, lambda: gm.block_quantize(X[0]))
    (Xq, Xs), (Wq, Ws) = gm.block_quantize(X), gm.block_quantize(W, 128)
    refused(DTYPE, lambda: gm.route_product_scaled(route, X, Xs, Wq, Ws))
    refused(DIM, lambda: gm.route_product_scaled(route, Xq, Xs[:, :0], Wq, Ws))
    refused(DIM, lambda: gm.route_product_scaled(route, Xq, Xs, Wq, Ws.expand(4, 2, 1)))
    refused(DTYPE, lambda: gm.route_product_scaled(route, Xq, Xs, Wq, Ws.half()))
    wide = gm.DeviceCSR(2, 2049, torch.zeros(3, dtype=torch.int64, device="cuda"), torch.zeros(0, dtype=torch.int32, device="cuda"), torch.zeros(0, device="cuda"))
    refused(CAPACITY, lambda: gm.route_plan(wide))
    refused(DTYPE, lambda: gm.route_plan(gm.DeviceCSR(20, 4, R.row_ptr, R.col, R.val.double())))
    refused(INVALID, lambda: gm.route_plan(gm.DeviceCSR(30, 4, R.row_ptr, R.col, R.val)))
