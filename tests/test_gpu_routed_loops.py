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
from test_gpu_routed import BF16, F16, F32, close, make_route, product_reference, randn

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
