"""What lies in an output and what does not.  The word that is added to the iteration must not: a kernel would read it while
another writes it.  Nothing that has no elements does.  On the host, before anything is queued; the addresses are made up, and a
refused call looks at no memory."""
import os
import struct

import pytest

from conftest import ROOT

LIB = os.path.join(ROOT, "paper_1610_02132_amd", "libqsgd.so")
pytestmark = pytest.mark.skipif(not os.path.exists(LIB), reason="libqsgd.so not built")

INVALID, UNSUPPORTED = -1, -5
F32, BF16, I8 = 0, 1, 3
X, W, DY, Y, DW, S, WS = (0x10000000 * i for i in range(1, 8))   # far apart, aligned


@pytest.fixture(scope="module")
def L():
    from paper_1610_02132_amd import binding
    return binding._load()


def mat(at, rows, cols, kind=F32, ld=None):
    return struct.pack("=QQQQII", at, rows, cols, cols if ld is None else ld, kind, 0)   # struct qsgd_matrix


def draws(iteration_dev):
    return struct.pack("=QIIIIQ", 1, 0, 0, 0, 0, iteration_dev)                          # struct qsgd_draws


INSIDE = [0, 4, 4 * 32 - 4, 4 * 40, 4 * (3 * 40 + 31)]   # of 4 rows of 32 floats, 40 apart


@pytest.mark.parametrize("at", INSIDE)
def test_inside_dropouts_result(L, at):
    x, y = mat(X, 4, 32), mat(Y, 4, 32, ld=40)
    assert L.qsgd_dropout(draws(Y + at), 0.1, x, None, y, None) == INVALID
    assert L.qsgd_dropout_backward(draws(Y + at), 0.1, x, y, None) == INVALID


def test_half_inside_a_row_of_16_bit_elements(L):
    x, y = mat(X, 4, 31, BF16), mat(Y, 4, 31, BF16, ld=40)
    assert L.qsgd_dropout(draws(Y + 60), 0.1, x, None, y, None) == INVALID          # the row's last element and what follows
    x, y = mat(X, 4, 31, BF16), mat(Y + 2, 4, 31, BF16, ld=40)
    assert L.qsgd_dropout(draws(Y + 2 * 40), 0.1, x, None, y, None) == INVALID      # what precedes a row, and its first element
    assert L.qsgd_dropout(draws(Y), 0.1, x, None, y, None) == INVALID


def test_between_two_rows_it_is_in_neither(L):
    """(A call that is refused for its size alone, after this check: nothing is queued.)"""
    x, y = mat(X, 2 ** 30, 64, BF16, ld=72), mat(X + 2 ** 40, 2 ** 30, 64, BF16, ld=72)
    for at, rc in ((128, UNSUPPORTED), (140, UNSUPPORTED), (2 * 72 * 2 ** 29 + 132, UNSUPPORTED), (124, INVALID), (144, INVALID)):
        assert L.qsgd_dropout(draws(X + 2 ** 40 + at), 0.1, x, None, y, None) == rc, at
    assert L.qsgd_dropout(draws(X), 0.1, x, None, y, None) == UNSUPPORTED           # in an input it is only read


@pytest.mark.parametrize("rounding", (0, 1))
def test_inside_the_quantizers_results(L, rounding):
    for at in (Y, Y + 48 * 7 + 36, DW, DW + 16 * 39 + 4, S, S + 28, S + 4096, S + 4096 + 156):
        rc = L.qsgd_quantize(draws(at), rounding, mat(X, 8, 40), mat(Y, 8, 40, I8, ld=48), S, mat(DW, 40, 8, I8, ld=16), S + 4096,
                             WS, 1 << 20, None)
        assert rc == INVALID, hex(at)


def test_inside_the_layers_results(L):
    for at in (Y, Y + 2 * (7 * 24 + 22)):
        assert L.qsgd_linear_forward(draws(at), 1, mat(X, 8, 40, BF16), mat(W, 24, 40, I8, ld=48), S, None, mat(Y, 8, 24, BF16),
                                     WS, 1 << 20, None) == INVALID
    for at in (Y, Y + 2 * (7 * 40 + 38), DW, DW + 4 * (24 * 40 - 1), S, S + 4 * 23):
        assert L.qsgd_linear_backward(draws(at), 1, mat(X, 8, 40, BF16), mat(W, 24, 40, BF16), mat(DY, 8, 24, BF16),
                                      mat(Y, 8, 40, BF16), mat(DW, 24, 40), S, WS, 1 << 20, None) == INVALID


def test_a_result_without_elements_holds_nothing(L):
    for rows, cols in ((0, 5), (5, 0), (0, 0)):
        y = mat(Y + 2, rows, cols, BF16)
        assert L.qsgd_dropout(draws(Y), 0.1, mat(X, rows, cols, BF16), None, y, None) == 0


def test_an_operand_without_elements_overlaps_nothing(L):
    """Products of no depth whose operands point into the result.  (Refused for their size alone, which is
    looked at after the overlap: nothing is queued.)"""
    M, N = 2 ** 20, 2 ** 18
    y = mat(X, M, N)
    far, near = X + 2 ** 44, X + 4096
    for a, b in ((far, far), (near, far), (far, near), (near, near)):
        assert L.qsgd_int_matmul(mat(a, M, 0, I8), 2 ** 45, mat(b, N, 0, I8), 2 ** 45 + 2 ** 30, None, y, None, 0, None) == UNSUPPORTED
