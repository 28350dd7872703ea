"""What the operators of a layer in 8 bits refuse, on the host before anything is queued, and the sizes of
their workspaces.  Addresses are made up: a refused call looks at no memory."""
import os
import struct

import pytest

from conftest import ROOT

LIB = os.path.join(ROOT, "paper_1610_02132_amd", "libqsgd.so")
pytestmark = pytest.mark.skipif(not os.path.exists(LIB), reason="libqsgd.so not built")

INVALID, CAPACITY, UNSUPPORTED = -1, -2, -5
F32, BF16, F16, I8 = 0, 1, 2, 3


@pytest.fixture(scope="module")
def b():
    from paper_1610_02132_amd import binding
    return binding


def mat(b, at, rows, cols, kind=F32, ld=None, reserved=0):
    return struct.pack("=QQQQII", at, rows, cols, cols if ld is None else ld, kind, reserved)   # struct qsgd_matrix


def draws(b, row_base=0, reserved=0, iteration_dev=0):
    return struct.pack("=QIIIIQ", 1, 0, 0, row_base, reserved, iteration_dev)                   # struct qsgd_draws


def ref(m):
    return m


A, B, Y, Z = 0x10000000, 0x20000000, 0x30000000, 0x40000000   # far apart, aligned


def test_dropout_refusals(b):
    L = b._load()

    def call(p=0.1, x=None, res=None, y=None, d=None):
        x = mat(b, A, 4, 32) if x is None else x
        y = mat(b, Y, 4, 32) if y is None else y
        return L.qsgd_dropout(ref(draws(b) if d is None else d), p, ref(x), ref(res), ref(y), None)

    for p in (-0.01, 1.01, float("nan"), float("inf")):
        assert call(p=p) == INVALID
    assert L.qsgd_dropout(None, 0.1, ref(mat(b, A, 4, 32)), None, ref(mat(b, Y, 4, 32)), None) == INVALID
    assert L.qsgd_dropout(ref(draws(b)), 0.1, None, None, ref(mat(b, Y, 4, 32)), None) == INVALID
    assert L.qsgd_dropout(ref(draws(b)), 0.1, ref(mat(b, A, 4, 32)), None, None, None) == INVALID
    assert call(d=draws(b, reserved=1)) == INVALID
    assert call(d=draws(b, row_base=2 ** 32 - 3)) == INVALID          # its rows would pass 2^32
    assert call(d=draws(b, iteration_dev=0x1002)) == INVALID          # not aligned to a word
    assert call(x=mat(b, A, 4, 32, reserved=1)) == INVALID
    assert call(x=mat(b, A, 4, 32, I8), y=mat(b, Y, 4, 32, I8)) == INVALID
    assert call(x=mat(b, A, 4, 32, 7), y=mat(b, Y, 4, 32, 7)) == INVALID
    assert call(y=mat(b, Y, 4, 32, BF16)) == INVALID                  # another type
    assert call(y=mat(b, Y, 4, 31)) == INVALID                        # another shape
    assert call(x=mat(b, A, 4, 32, ld=31)) == INVALID                 # rows overlap
    assert call(x=mat(b, A + 2, 4, 32)) == INVALID                    # not aligned to its elements
    assert call(x=mat(b, 0, 4, 32)) == INVALID
    assert call(x=mat(b, A, 2 ** 31, 1), y=mat(b, Y, 2 ** 31, 1)) == INVALID
    assert call(x=mat(b, A, 4, 32, ld=2 ** 45), y=mat(b, Y, 4, 32, ld=2 ** 45)) == INVALID
    assert call(res=mat(b, Z, 4, 31)) == INVALID
    assert call(res=mat(b, Z, 4, 32, F16)) == INVALID
    assert call(y=mat(b, A + 16, 4, 32)) == INVALID                   # overlaps x without being x
    assert call(y=mat(b, A, 4, 32, ld=40)) == INVALID                 # x's place with another distance of rows
    assert call(res=mat(b, Z, 4, 32), y=mat(b, Z + 64, 4, 32)) == INVALID
    assert L.qsgd_dropout_backward(ref(draws(b)), 2.0, ref(mat(b, A, 4, 32)), ref(mat(b, Y, 4, 32)), None) == INVALID


def test_work_that_a_launch_cannot_count(b):
    L = b._load()
    x, y = mat(b, A, 2 ** 30, 64, BF16), mat(b, A + 2 ** 40, 2 ** 30, 64, BF16)
    assert L.qsgd_dropout(draws(b), 0.1, x, None, y, None) == UNSUPPORTED
    rows = mat(b, A + 2 ** 42, 2 ** 25, 4096, I8)
    assert L.qsgd_quantize(None, 0, mat(b, A, 2 ** 25, 4096, BF16), rows, 2 ** 45, None, None, None, 0, None) == UNSUPPORTED
    a, w = mat(b, A, 2 ** 26, 16, I8), mat(b, A + 2 ** 40, 16, 16, I8)
    assert L.qsgd_int_matmul(a, 2 ** 45, w, 2 ** 44, None, mat(b, A + 2 ** 42, 2 ** 26, 16), None, 0, None) == UNSUPPORTED
    a, w = mat(b, A, 2 ** 20, 16, I8), mat(b, A + 2 ** 40, 2 ** 18, 16, I8)
    assert L.qsgd_int_matmul(a, 2 ** 45, w, 2 ** 44, None, mat(b, A + 2 ** 42, 2 ** 20, 2 ** 18), None, 0, None) == UNSUPPORTED


def test_nothing_to_do_is_no_error(b):
    """Matrices without elements: nothing is launched (there need not be a GPU)."""
    L = b._load()
    for rows, cols in ((0, 5), (5, 0), (0, 0)):
        x, y = mat(b, 0, rows, cols), mat(b, 0, rows, cols)
        assert L.qsgd_dropout(ref(draws(b)), 0.1, ref(x), None, ref(y), None) == 0
    e = mat(b, 0, 0, 16, I8)
    assert L.qsgd_int_matmul(ref(e), None, ref(mat(b, B, 4, 16, I8)), Z, None, ref(mat(b, 0, 0, 4)), None, 0, None) == 0
    assert L.qsgd_quantize(None, 0, ref(mat(b, 0, 0, 5)), ref(mat(b, 0, 0, 5, I8, ld=16)), None, None, None, None, 0, None) == 0


def test_quantize_refusals(b):
    L = b._load()
    need = b.qsgd_quantize_workspace_bytes(8, 40)
    assert need > 0
    W = 0x50000000

    def call(d="default", rounding=0, x=None, rows="default", rs=Z, cols="default", cs=Z + 4096, ws=W, size=None):
        d = draws(b) if d == "default" else d
        x = mat(b, A, 8, 40) if x is None else x
        rows = mat(b, B, 8, 40, I8, ld=48) if rows == "default" else rows
        cols = mat(b, Y, 40, 8, I8, ld=16) if cols == "default" else cols
        return L.qsgd_quantize(ref(d), rounding, ref(x), ref(rows), rs, ref(cols), cs, ws, need if size is None else size, None)

    assert call(rounding=2) == INVALID
    assert call(d=None, rounding=1) == INVALID                        # stochastic rounding without draws
    assert call(rows=None, cols=None) == INVALID
    assert call(rs=None) == INVALID
    assert call(cs=None) == INVALID
    assert call(rs=Z + 2) == INVALID
    assert call(x=mat(b, A, 8, 40, I8, ld=48)) == INVALID
    assert call(rows=mat(b, B, 8, 40, F32)) == INVALID
    assert call(rows=mat(b, B, 8, 40, I8, ld=40)) == INVALID          # not a multiple of 16
    assert call(rows=mat(b, B + 8, 8, 40, I8, ld=48)) == INVALID      # not aligned to 16
    assert call(rows=mat(b, B, 40, 8, I8, ld=16)) == INVALID
    assert call(cols=mat(b, Y, 8, 40, I8, ld=48)) == INVALID          # the column form is transposed
    assert call(rows=mat(b, A, 8, 40, I8, ld=48)) == INVALID          # overlaps x
    assert call(cols=mat(b, B, 40, 8, I8, ld=16)) == INVALID          # overlaps the row form
    assert call(rs=A + 64) == INVALID                                 # scales over x, over levels, over each other
    assert call(cs=B + 16) == INVALID
    assert call(cs=Z + 16) == INVALID
    assert call(ws=None) == INVALID
    assert call(ws=W + 8) == INVALID
    assert call(size=need - 1) == CAPACITY


def test_product_refusals(b):
    L = b._load()

    def call(a=None, sa=Z, w=None, sb=Z + 4096, bias=None, y=None, ws=None, size=0):
        a = mat(b, A, 8, 40, I8, ld=48) if a is None else a
        w = mat(b, B, 24, 40, I8, ld=48) if w is None else w
        y = mat(b, Y, 8, 24) if y is None else y
        return L.qsgd_int_matmul(ref(a), sa, ref(w), sb, bias, ref(y), ws, size, None)

    assert call(a=mat(b, A, 8, 40)) == INVALID
    assert call(a=mat(b, A, 8, 41, I8, ld=48)) == INVALID             # another K
    assert call(a=mat(b, A, 8, 40, I8, ld=40)) == INVALID
    assert call(a=mat(b, A + 4, 8, 40, I8, ld=48)) == INVALID
    assert call(sa=None) == INVALID
    assert call(sb=None) == INVALID
    assert call(sa=Z + 1) == INVALID
    assert call(bias=Z + 2) == INVALID
    assert call(y=mat(b, Y, 24, 8)) == INVALID
    assert call(y=mat(b, Y, 8, 24, I8, ld=32)) == INVALID
    assert call(y=mat(b, A, 8, 24)) == INVALID                        # overlaps an operand
    assert call(sa=Y + 64) == INVALID                                 # ... or its scales, or the bias
    assert call(sb=Y + 64) == INVALID
    assert call(bias=Y + 64) == INVALID
    assert call(a=mat(b, A, 8, 40, I8, ld=2 ** 23)) == UNSUPPORTED
    K = 200_000
    long = b.qsgd_int_matmul_workspace_bytes(8, 24, K)                # sums that pass 32 bits are joined from pieces
    assert long > 0
    la, lb = mat(b, A, 8, K, I8), mat(b, B, 24, K, I8)
    assert call(a=la, w=lb) == INVALID
    assert call(a=la, w=lb, ws=0x50000008, size=long) == INVALID
    assert call(a=la, w=lb, ws=0x50000000, size=long - 1) == CAPACITY


def test_linear_refusals(b):
    L = b._load()
    M, N, K = 8, 24, 40
    W = 0x50000000
    need = b.qsgd_linear_forward_workspace_bytes(M, N, K)

    def forward(d="default", rounding=0, x=None, w=None, ws_=Z, bias=None, y=None, ws=W, size=None):
        d = draws(b) if d == "default" else d
        x = mat(b, A, M, K, BF16) if x is None else x
        w = mat(b, B, N, K, I8, ld=48) if w is None else w
        y = mat(b, Y, M, N, BF16) if y is None else y
        return L.qsgd_linear_forward(ref(d), rounding, ref(x), ref(w), ws_, bias, ref(y), ws, need if size is None else size, None)

    assert forward(rounding=3) == INVALID
    assert forward(d=None, rounding=1) == INVALID
    assert forward(x=mat(b, A, M, K + 1, BF16)) == INVALID
    assert forward(y=mat(b, Y, M, N, F32)) == INVALID
    assert forward(w=mat(b, B, N, K, BF16)) == INVALID
    assert forward(ws_=None) == INVALID
    assert forward(y=mat(b, A, M, N, BF16)) == INVALID
    assert forward(ws=None) == INVALID
    assert forward(size=need - 1) == CAPACITY

    need_b = b.qsgd_linear_backward_workspace_bytes(M, N, K)

    def backward(d="default", rounding=1, x=None, w=None, dy=None, dx="default", dw="default", db=None, ws=W, size=None):
        d = draws(b) if d == "default" else d
        x = mat(b, A, M, K, BF16) if x is None else x
        w = mat(b, A + 65536, N, K, BF16) if w is None else w
        dy = mat(b, B, M, N, BF16) if dy is None else dy
        dx = mat(b, Y, M, K, BF16) if dx == "default" else dx
        dw = mat(b, Z, N, K, F32) if dw == "default" else dw
        return L.qsgd_linear_backward(ref(d), rounding, ref(x), ref(w), ref(dy), ref(dx), ref(dw), db, ws,
                                      need_b if size is None else size, None)

    assert backward(d=None) == INVALID
    assert backward(dx=None, dw=None) == INVALID                      # nothing asked for
    assert backward(dy=mat(b, B, N, M, BF16)) == INVALID
    assert backward(dy=mat(b, B, M, N, F16)) == INVALID
    assert backward(dw=mat(b, Z, N, K, BF16)) == INVALID              # the weights' gradient is fp32
    assert backward(dx=mat(b, Y, M, K, F32)) == INVALID
    assert backward(dx=mat(b, A, M, K, BF16)) == INVALID              # over x
    assert backward(dw=mat(b, Y + 64, N, K, F32)) == INVALID          # over dx
    assert backward(db=Z + 2) == INVALID
    assert backward(db=Y + 64) == INVALID                             # over dx
    assert backward(ws=W + 4) == INVALID
    assert backward(size=need_b - 1) == CAPACITY
    assert backward(d=draws(b, row_base=2 ** 32 - 7)) == INVALID


def test_workspace_sizes(b):
    """Sizes depend on the arguments alone, grow with them, and are 0 for sizes that no call takes."""
    assert b.qsgd_quantize_workspace_bytes(1, 1) >= 12
    assert b.qsgd_quantize_workspace_bytes(8192, 4096) < 8192 * 4096
    assert b.qsgd_int_matmul_workspace_bytes(0, 5, 7) == 0
    assert b.qsgd_int_matmul_workspace_bytes(2 ** 31, 5, 7) == 0
    assert b.qsgd_linear_forward_workspace_bytes(8192, 4096, 4096) >= 8192 * 4096
    n = b.qsgd_linear_backward_workspace_bytes(8192, 4096, 4096)
    assert n >= 2 * 8192 * 4096 + 4096 * 4096 and n < 2 ** 33
    assert b.qsgd_linear_backward_workspace_bytes(2 ** 23, 16, 16) == 0
    assert b.qsgd_linear_forward_workspace_bytes(2 ** 31, 16, 16) == 0


def test_binding_refuses_tensors_that_are_no_matrix(b):
    import torch
    x = torch.zeros(4, 32)
    with pytest.raises(ValueError):
        b._matrix(x, "x")                                             # not on the device
    with pytest.raises(ValueError):
        b._matrix(x.double(), "x")
    with pytest.raises(ValueError):
        b._vector(x, 5, "scale")
