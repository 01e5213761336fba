"""Refusals of the routed products that need no GPU: arguments are checked before anything is launched or looked at on a device."""
import ctypes
import struct

import pytest
import torch

import paper_2607_22866_b200 as gm

INVALID, DIM, DTYPE, BAD_CSR, CAPACITY = -1, -2, -3, -4, -6
F32, F64, BF16, F16, E4M3 = range(5)
SOMEWHERE = 0x7F0000000000  # never looked at


CSR = gm.binding._CSR


def dense(rows, cols, dtype, blocks=1, data=SOMEWHERE, block=None, row=None, col=1):
    row = cols if row is None else row
    return struct.pack("=7q2i", data, blocks, rows, cols, rows * row if block is None else block, row, col, dtype, 0)


@pytest.fixture(scope="module")
def lib():
    return gm.load_library()


def plan(lib, R, arrays=(SOMEWHERE,) * 4, out=True):
    h = ctypes.c_void_p()
    rc = lib.gm_route_plan(ctypes.byref(R) if R is not None else None, *arrays, None, ctypes.byref(h) if out else None)
    assert not h.value
    return rc


def test_route_plan_refuses(lib):
    def R(n=4, e=3, nnz=5, rp=SOMEWHERE, col=SOMEWHERE, val=SOMEWHERE, dtype=F32):
        return CSR(n, e, nnz, rp, col, val, dtype, 0)

    assert plan(lib, None) == INVALID and plan(lib, R(), out=False) == INVALID
    assert plan(lib, R(n=-1)) == INVALID and plan(lib, R(nnz=-1)) == INVALID and plan(lib, R(e=-1)) == INVALID
    assert plan(lib, R(nnz=2**31)) == INVALID and plan(lib, R(n=2**31 - 1)) == INVALID
    assert plan(lib, R(e=2049)) == CAPACITY
    assert plan(lib, R(n=0)) == BAD_CSR
    assert plan(lib, R(rp=None)) == INVALID and plan(lib, R(col=None)) == INVALID and plan(lib, R(val=None)) == INVALID
    assert plan(lib, R(dtype=F64)) == DTYPE and plan(lib, R(dtype=BF16)) == DTYPE and plan(lib, R(dtype=17)) == DTYPE
    for k in range(4):
        arrays = [SOMEWHERE] * 4
        arrays[k] = None
        assert plan(lib, R(), arrays) == INVALID


def test_calls_without_a_route_are_refused(lib):
    m = dense(4, 8, BF16)
    assert lib.gm_route_status(None) == INVALID
    assert lib.gm_route_product(None, m, 0, m, m, None) == INVALID
    assert lib.gm_route_product_dx(None, m, m, 0, m, None, None) == INVALID
    assert lib.gm_route_product_dw(None, m, m, 0, m, None) == INVALID
    assert lib.gm_route_sum(None, m, 1, m, None) == INVALID
    assert lib.gm_route_sum_grads(None, m, m, m, None, None) == INVALID
    assert lib.gm_route_product_scaled(None, m, m, 0, m, m, m, None) == INVALID
    lib.gm_route_destroy(None)


def test_block_quantize_refuses(lib):
    X, Q, S = dense(4, 200, BF16), dense(4, 200, E4M3), dense(4, 2, F32)
    call = lambda x=X, rows=1, q=Q, s=S: lib.gm_block_quantize(x, rows, q, s, None)  # noqa: E731
    assert call(x=None) == INVALID and call(q=None) == INVALID and call(s=None) == INVALID
    assert call(rows=2) == INVALID and call(rows=0) == INVALID and call(rows=-128) == INVALID
    assert call(x=dense(4, 200, F32)) == DTYPE and call(x=dense(4, 200, E4M3)) == DTYPE and call(x=dense(4, 200, 9)) == DTYPE
    assert call(q=dense(4, 200, BF16)) == DTYPE and call(s=dense(4, 2, BF16)) == DTYPE
    assert call(q=dense(4, 199, E4M3)) == DIM and call(s=dense(4, 1, F32)) == DIM and call(rows=128) == DIM
    assert call(x=dense(-1, 200, BF16)) == INVALID and call(x=dense(4, 200, BF16, row=-200)) == INVALID
    assert call(x=dense(4, 200, BF16, data=0)) == INVALID and call(x=dense(4, 200, BF16, data=SOMEWHERE + 1)) == INVALID
    assert call(q=dense(4, 200, E4M3, row=208)) == INVALID  # results are contiguous
    assert call(q=dense(4, 200, E4M3, col=2, row=400)) == INVALID and call(q=dense(4, 200, E4M3, row=100)) == INVALID
    # nothing to do is no error, and needs no device
    assert lib.gm_block_quantize(dense(0, 200, BF16), 1, dense(0, 200, E4M3), dense(0, 2, F32), None) == 0
    assert lib.gm_block_quantize(dense(4, 0, F16, data=0), 128, dense(4, 0, E4M3, data=0), dense(1, 0, F32, data=0), None) == 0


def test_tensors_of_the_host_are_refused():
    X = torch.zeros(4, 16, dtype=torch.bfloat16)
    R = gm.DeviceCSR(1, 2, torch.tensor([0, 1]), torch.zeros(1, dtype=torch.int32), torch.ones(1))
    for call in (lambda: gm.block_quantize(X), lambda: gm.route_plan(R)):
        with pytest.raises(gm.GmError) as e:
            call()
        assert e.value.status == INVALID
