"""The integer product's last steps where a row's scale is large: the definition is fl(fl(fl(sum) a_scale) b_scale + bias), the last two in
one rounding, and it overflows only where its value does.  Against exact fractions, bit for bit, in every kernel that ends a
product."""
from fractions import Fraction

import numpy as np
import pytest
import torch

import layer_reference as R
import paper_1610_02132_amd as q

pytestmark = pytest.mark.gpu


def rounded(v):
    """A fraction to 24 bits, ties to even, without limits of the exponent."""
    if v == 0:
        return v
    a, e = abs(v), 0
    while a >= 2 ** 24:
        a, e = a / 2, e + 1
    while a < 2 ** 23:
        a, e = a * 2, e - 1
    return (1 if v > 0 else -1) * Fraction(round(a)) * Fraction(2) ** e


def defined(total, s, t, bias):
    """The result as fp32 (all of them normal here, or infinite)."""
    if total == 0:
        return np.float32(bias)
    v = rounded(rounded(rounded(Fraction(int(total))) * Fraction(s)) * Fraction(t) + Fraction(bias))
    if abs(v) >= 2 ** 128:
        return np.float32(np.inf if v > 0 else -np.inf)
    return np.float32(float(v))


# of the few-row kernel, tiles, no depth to speak of, and pieces that are joined (results four to a thread, and one)
SHAPES = [(3, 20, 100), (70, 40, 100), (1500, 1501, 33), (64, 64, 8192), (33, 71, 20_000)]


@pytest.mark.parametrize("M,N,K", SHAPES, ids=str)
def test_large_scales(M, N, K):
    g = torch.Generator()
    g.manual_seed(M)
    a, b = (R.levels(n, K)[1] for n in (M, N))
    a.copy_(torch.randint(-127, 128, (M, K), generator=g).to(torch.int8))
    b.copy_(torch.randint(-127, 128, (N, K), generator=g).to(torch.int8))
    a[2].zero_()                                                     # sums of nothing under every scale
    rng = np.random.default_rng(M)
    sums = a.cpu().numpy().astype(np.int64)[:3] @ b.cpu().numpy().astype(np.int64).T
    for power in (60, 89, 90, 91, 100, 126):
        for sign in (1, -1):
            sa = (sign * (1 + rng.random(M)) * 2.0 ** power).astype(np.float32)
            tb = ((1 + rng.random(N)) * 2.0 ** -power).astype(np.float32)
            # what the first row's results are nearly, the other way: nothing is left but what the roundings make
            bias = -(sums[0].astype(np.float64) * sa[0] * tb).astype(np.float32)
            tb[3:8], bias[3:8] = 2.0 ** 100, 1.5                     # results that leave fp32, all but a sum of nothing
            tb[8], bias[8] = np.float32(2.0 ** (127 - power - 13)), -3e38   # ... and some that a bias brings back
            tb[9], bias[9] = np.float32(2.0 ** (127 - power - 13)), 3e38
            y = torch.empty(M, N, device="cuda")
            ws = torch.empty(max(16, q.qsgd_int_matmul_workspace_bytes(M, N, K)), dtype=torch.uint8, device="cuda")
            dev = lambda v: torch.from_numpy(v).cuda()  # noqa: E731
            q.qsgd_int_matmul(a, dev(sa), b, dev(tb), y, bias=dev(bias), workspace=ws)
            got = y[:3].cpu().numpy()
            for m in range(3):
                for n in range(min(N, 24)):
                    want = defined(sums[m, n], float(sa[m]), float(tb[n]), float(bias[n]))
                    assert got[m, n] == want, (power, sign, m, n, got[m, n], want)
