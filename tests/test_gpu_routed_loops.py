"""Routed products in their main loops: pairs of blocks that go over several tiles (148 SMs: more than 74 tiles), sums of more blocks of k than
there are stages, buffers or slots of scales, sums that last long.

Tolerances.  Every element: as in test_gpu_routed.py.  The norm of all errors, of f32 results of independent terms of mean zero: the partial sum of the
first s of n terms has a norm of about sqrt(s / n) times the result's, every addition is off by at most 2^-23 of the partial sum, and the errors' norms
add up at worst: 2/3 n 2^-23 times the norm of the result.  n 2^-23 leaves half of that again for what "about" means with thousands of results.  One
rounding to bf16 of sums on their way would be off by about 2^-9 / sqrt(3) = 1.1e-3 of it, n 2^-23 is 3.5e-4 at n = 2960.
"""
import pytest
import torch

import paper_2607_22866_b200 as gm
from test_gpu_routed import BF16, F16, F32, close, dw_reference, dx_reference, make_route, product_reference, randn

pytestmark = pytest.mark.gpu


def close_norm(got, ref, terms):
    assert got.dtype == F32
    off, allowed = float((got.double() - ref).norm()), terms * 2.0 ** -23 * float(ref.norm())
    assert off <= allowed, (off, allowed)


def tiles(R, places, rows):
    """Tiles of at most `places` places by 256 rows of a block."""
    count = torch.bincount(R.col[(R.col >= 0) & (R.col < R.n_cols)].long(), minlength=R.n_cols)
    return int(((count + places - 1) // places).sum()) * -(-rows // 256)


def scaled_inputs(rows_x, E, N, K, rows):
    X, W = randn((rows_x, K), BF16, 1), randn((E, N, K), BF16, 2, 0.3)
    (Xq, Xs), (Wq, Ws) = gm.block_quantize(X, 1), gm.block_quantize(W, rows)
    x = Xq.double() * Xs.double().repeat_interleave(128, 1)[:, :K]
    w = Wq.double() * Ws.double().repeat_interleave(128, 2)[:, :, :K].repeat_interleave(rows, 1)[:, :N]
    return (Xq, Xs, Wq, Ws), x, w


# n, E, k, N, K: columns of few places (tiles of 64): some of more than one tile, some of less than half of one
@pytest.mark.parametrize("rows", [1, 128])
@pytest.mark.parametrize("by_entry", [False, True])
@pytest.mark.parametrize("n,E,k,N,K", [(700, 64, 4, 1032, 2960), (90, 50, 3, 520, 1168)])
def test_scaled_few_places_over_many_tiles(n, E, k, N, K, by_entry, rows):
    R = make_route(n, E, k, 23 * n, drop=0.05, skew=0.7)
    route = gm.route_plan(R)
    assert R.nnz <= 48 * E and tiles(R, 64, N) > 74
    (Xq, Xs, Wq, Ws), x, w = scaled_inputs(R.nnz if by_entry else n, E, N, K, rows)
    P = gm.route_product_scaled(route, Xq, Xs, Wq, Ws, by_entry, dtype=F32)
    ref, mag = product_reference(R, x, w, by_entry)
    close(P, ref, mag, K + 3)
    close_norm(P, ref, K + 3)
    for _ in range(5):  # scales that were overwritten too early would show sometimes only
        assert torch.equal(P, gm.route_product_scaled(route, Xq, Xs, Wq, Ws, by_entry, dtype=F32))
    torch.cuda.synchronize()
    route.status()


@pytest.mark.parametrize("by_entry", [False, True])
def test_dw_of_a_column_of_many_places(by_entry):
    # half a million stages in one sum; of -1, 0 and 1, whose partial sums stay far below 2^24: exact in any order
    n, entries = 5000, 32_000_000 + 37
    row_ptr = (torch.arange(n + 1, device="cuda") * entries) // n
    R = gm.DeviceCSR(n, 2, row_ptr, torch.ones(entries, dtype=torch.int32, device="cuda"), torch.ones(entries, device="cuda"))
    route = gm.route_plan(R)
    g = torch.Generator(device="cuda").manual_seed(1)
    ones = lambda rows: torch.randint(-1, 2, (rows, 8), generator=g, device="cuda", dtype=torch.int8).bfloat16()  # noqa: E731
    dP, X = ones(entries), ones(entries if by_entry else n)
    dW = gm.route_product_dw(route, dP, X, by_entry, dtype=F32)
    ref = torch.zeros(8, 8, dtype=torch.float64, device="cuda")
    for a in range(0, entries, 1 << 22):
        d = dP[a: a + (1 << 22)].double()
        ref += d.T @ (X[a: a + (1 << 22)] if by_entry else X[route.rows[a: a + (1 << 22)].long()]).double()
    assert float(ref.abs().max()) < 2.0 ** 20
    assert torch.equal(dW[1].double(), ref) and not dW[0].any()
    torch.cuda.synchronize()
    route.status()


@pytest.mark.parametrize("kind", ["16 bits", "8 bits"])
def test_sums_over_more_than_2_to_30_values(kind):
    # rows whose bytes pass 2^31, in sums that last for seconds; almost all values are zero, the others small whole numbers: exact
    K = 2 ** 30 + 72
    R = gm.DeviceCSR(1, 1, torch.tensor([0, 1], device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda"), torch.ones(1, device="cuda"))
    route = gm.route_plan(R)
    X, W = (torch.zeros(K, dtype=BF16, device="cuda") for _ in range(2))
    at = torch.tensor([0, 63, 64, 2 ** 20 + 5, 2 ** 29, 2 ** 30 - 1, 2 ** 30, 2 ** 30 + 63, 2 ** 30 + 64, K - 1], device="cuda")
    X[at], W[at] = torch.arange(1, 11, device="cuda").bfloat16(), torch.arange(10, 0, -1, device="cuda").bfloat16()
    want = float((X[at].double() * W[at].double()).sum())
    if kind == "16 bits":
        P = gm.route_product(route, X[None], W[None, None], dtype=F32)
        dX = gm.route_product_dx(route, P.bfloat16(), W[None, None], dtype=F32)
        assert torch.equal(dX, (float(P.bfloat16()) * W.float())[None])
    else:
        e4m3, scales = torch.float8_e4m3fn, torch.ones(1, -(-K // 128), device="cuda")
        P = gm.route_product_scaled(route, X.to(e4m3)[None], scales, W.to(e4m3)[None, None], scales[None], dtype=F32)
    assert float(P) == want
    torch.cuda.synchronize()
    route.status()


# n, E, k, N, K: tiles of 256 places (six stages a block of threads) and of 64 (ten): as many blocks of 64 values as stages, one more, many
LOOPS = [(3000, 9, 4, 1000, 840), (3000, 9, 4, 1032, 384), (3000, 9, 4, 1032, 448), (700, 64, 4, 520, 1496), (700, 64, 4, 520, 640), (700, 64, 4, 520, 704)]


def few(R):
    return R.nnz <= 48 * R.n_cols


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("by_entry", [False, True])
@pytest.mark.parametrize("n,E,k,N,K", LOOPS)
def test_products_over_many_tiles(n, E, k, N, K, by_entry, dtype):
    R = make_route(n, E, k, 29 * n + K, drop=0.05, skew=0.7)
    route = gm.route_plan(R)
    assert few(R) == (E == 64) and tiles(R, 64 if few(R) else 256, N) > 74 * 1.25
    X, W, dP = randn((R.nnz if by_entry else n, K), dtype, 1), randn((E, N, K), dtype, 2), randn((R.nnz, N), dtype, 3)
    P = gm.route_product(route, X, W, by_entry, dtype=F32)
    ref, mag = product_reference(R, X, W, by_entry)
    close(P, ref, mag, K)
    close_norm(P, ref, K)
    dX = gm.route_product_dx(route, dP, W, by_entry, dtype=F32)
    ref, mag = dx_reference(R, dP, W, by_entry)
    close(dX, ref, mag, N + k)
    close_norm(dX, ref, N + k)
    dW = gm.route_product_dw(route, dP, X, by_entry, dtype=F32)
    ref, mag, most = dw_reference(R, dP, X, by_entry)
    close(dW, ref, mag, most)
    close_norm(dW, ref, most)
    half = [gm.route_product(route, X, W, by_entry), gm.route_product_dx(route, dP, W, by_entry), gm.route_product_dw(route, dP, X, by_entry)]
    for a, b in zip((P, dX, dW), half):  # the same sums, rounded
        assert b.dtype == dtype and torch.equal(a.to(dtype), b)
    for _ in range(3):
        assert torch.equal(P, gm.route_product(route, X, W, by_entry, dtype=F32)) and torch.equal(dW, gm.route_product_dw(route, dP, X, by_entry, dtype=F32))
    torch.cuda.synchronize()
    route.status()


# tiles of 256 places, two of them per pair of blocks and more, with more blocks of 128 values than stages, buffers of sums and slots of scales
@pytest.mark.parametrize("rows", [1, 128])
@pytest.mark.parametrize("by_entry", [False, True])
@pytest.mark.parametrize("n,E,k,N,K", [(3000, 9, 4, 1032, 1680), (2500, 8, 5, 1536, 1168)])
def test_scaled_many_places_over_many_tiles(n, E, k, N, K, by_entry, rows):
    R = make_route(n, E, k, 31 * n, drop=0.05, skew=0.7)
    route = gm.route_plan(R)
    assert not few(R) and tiles(R, 256, N) > 74 * 1.25
    (Xq, Xs, Wq, Ws), x, w = scaled_inputs(R.nnz if by_entry else n, E, N, K, rows)
    P = gm.route_product_scaled(route, Xq, Xs, Wq, Ws, by_entry, dtype=F32)
    ref, mag = product_reference(R, x, w, by_entry)
    close(P, ref, mag, K + 3)
    close_norm(P, ref, K + 3)
    for dtype in (BF16, F16):
        assert torch.equal(P.to(dtype), gm.route_product_scaled(route, Xq, Xs, Wq, Ws, by_entry, dtype=dtype))
    for _ in range(5):
        assert torch.equal(P, gm.route_product_scaled(route, Xq, Xs, Wq, Ws, by_entry, dtype=F32))
    torch.cuda.synchronize()
    route.status()


def test_large_tiles_with_the_most_columns():
    # 2048 columns with more than 48 places each on average: the shared memory of large tiles and of the most columns
    n, E, N, K = 30000, 2048, 24, 72
    R = make_route(n, E, 9, 21, drop=0.02)
    assert not few(R)
    route = gm.route_plan(R)
    X, W = randn((n, K), BF16, 1), randn((E, N, K), BF16, 2)
    P = gm.route_product(route, X, W, dtype=F32)
    ref, mag = product_reference(R, X, W, False)
    close(P, ref, mag, K)
    close_norm(P, ref, K)
    for rows in (1, 128):
        (Xq, Xs, Wq, Ws), x, w = scaled_inputs(n, E, N, K, rows)
        P = gm.route_product_scaled(route, Xq, Xs, Wq, Ws, dtype=F32)
        ref, mag = product_reference(R, x, w, False)
        close(P, ref, mag, K + 3)
        close_norm(P, ref, K + 3)
    dP = randn((R.nnz, N), BF16, 3)
    dX, dW = gm.route_product_dx(route, dP, W, dtype=F32), gm.route_product_dw(route, dP, X, dtype=F32)
    ref, mag = dx_reference(R, dP, W, False)
    close(dX, ref, mag, N + 9)
    close_norm(dX, ref, N + 9)
    ref, mag, most = dw_reference(R, dP, X, False)
    close(dW, ref, mag, most)
    close_norm(dW, ref, most)
    torch.cuda.synchronize()
    route.status()
