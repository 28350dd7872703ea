"""Products in pieces by every kernel, in every type, and both gradients of a layer in one launch or in pieces, by every kernel:
shapes that the host's estimate sends there (see layer_shapes.py)."""
import numpy as np
import pytest
import torch

import layer_reference as R
import layer_shapes as S
import paper_1610_02132_amd as q

pytestmark = pytest.mark.gpu

D = q.Draws(seed=9, stream_id=40, iteration=2)
TOP = 128 ** 2


def levels(rows, cols, seed, low=-128):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    ld = (cols + 15) // 16 * 16
    return torch.randint(low, 128, (rows, ld), generator=g, device="cuda", dtype=torch.int8)[:, :cols]


def space(n):
    """A workspace of exactly n bytes inside a larger buffer whose rest must stay as it is."""
    buf = torch.full((n + 256,), 0x5A, dtype=torch.uint8, device="cuda")
    return buf, buf[:n] if n else None


def exact_sums(a, b):
    """The integer sums in 64-bit floats (below 2^53: exact), a part of k at a time."""
    assert a.shape[1] * TOP < 2 ** 53
    y = torch.zeros(a.shape[0], b.shape[0], dtype=torch.float64, device="cuda")
    for k in range(0, a.shape[1], 16_384):
        y += torch.matmul(a[:, k:k + 16_384].double(), b[:, k:k + 16_384].double().t().contiguous())
    return y


def within(got, sums, sa, sb, bias, what):
    """got against sums * sa * sb + bias: the sum to fp32, two products (the last with the bias in one rounding), and the type."""
    y = sums * sa.double()[:, None] * sb.double()
    tol = 3 * R.U32 * y.abs() * 1.01
    if bias is not None:
        y = y + bias.double()
        tol = tol + R.U32 * y.abs() * 1.01
    t = got.dtype
    tol = tol + R.HALF_STEP[t] * (y.abs() + tol) + R.LEAST[t]
    off = (got.double() - y).abs()
    # a value from half a step above the type's largest on is infinite, one that may be on either side of that is either
    info = torch.finfo(t)
    over = info.max + info.eps / 2 * 2.0 ** int(np.log2(info.max))
    infinite = got.double() == y.sign() * float("inf")
    right = torch.where(y.abs() - tol >= over, infinite, (off <= tol) | (infinite & (y.abs() + tol >= over)))
    assert bool(right.all()), (what, float((off / tol)[~right].max()))


@pytest.mark.parametrize("M,N,K", list(S.IN_PIECES), ids=str)
def test_product_in_pieces(M, N, K):
    need = q.qsgd_int_matmul_workspace_bytes(M, N, K)
    assert need >= 4 * S.IN_PIECES[M, N, K][1] * M * N
    a, b = levels(M, K, 1), levels(N, K, 2)
    a[0].fill_(-128), b[0].fill_(-128)                  # the largest sums there are
    sa, sb = torch.rand(M, device="cuda") * 0.001 + 1e-5, torch.rand(N, device="cuda") * 0.001 + 1e-5
    bias = torch.linspace(-3, 3, N, device="cuda")
    sums = exact_sums(a, b)
    for dtype in R.TYPES:
        for with_bias in (None, bias):
            wsbuf, ws = space(need)
            buf, y = R.framed(M, N, dtype, ld=N + 3, start=1)
            q.qsgd_int_matmul(a, sa, b, sb, y, bias=with_bias, workspace=ws)
            within(y, sums, sa, sb, with_bias, dtype)
            assert R.outside_untouched(buf, y) and bool((wsbuf[need:] == 0x5A).all())


@pytest.mark.parametrize("M,N,K", list(S.PAIRS) + list(S.BACKWARD_IN_PIECES), ids=str)
def test_gradients(M, N, K):
    """dx, dw and db of the layer against the quantizer's levels and their exact products: whole, as they are a few rows at
    a time, and bit for bit as the integer product gives them."""
    dtype = (torch.bfloat16, torch.float32, torch.float16)[(M + N + K) % 3]
    g = torch.Generator(device="cuda")
    g.manual_seed(M + N)
    value = lambda r, c, s: (torch.randn(r, c, generator=g, device="cuda") * s).to(dtype)  # noqa: E731
    x, w, dy = value(M, K, 1.0), value(N, K, 0.05), value(M, N, 0.5)
    need = q.qsgd_linear_backward_workspace_bytes(M, N, K)
    wsbuf, ws = space(need)
    dxbuf, dx = R.framed(M, K, dtype, ld=K + 1)
    dwbuf, dw = R.framed(N, K, torch.float32, ld=K + 2, start=3)
    db = torch.full((N,), 9.0, device="cuda")
    q.qsgd_linear_backward(D, x, w, dy, dx=dx, dw=dw, db=db, workspace=ws, rounding=q.ROUND_STOCHASTIC)
    assert R.outside_untouched(dxbuf, dx) and R.outside_untouched(dwbuf, dw) and bool((wsbuf[need:] == 0x5A).all())

    def quantized(t, by, form):
        r, c = t.shape if form == "rows" else t.shape[::-1]
        out = torch.empty(r, (c + 15) // 16 * 16, dtype=torch.int8, device="cuda")[:, :c]
        scale = torch.empty(r, device="cuda")
        room = torch.empty(q.qsgd_quantize_workspace_bytes(*t.shape), dtype=torch.uint8, device="cuda")
        d = q.Draws(seed=D.seed, stream_id=D.stream_id + by, iteration=D.iteration)
        q.qsgd_quantize(d, t, **{form: out, form[:-1] + "_scale": scale}, workspace=room, rounding=q.ROUND_STOCHASTIC)
        return out, scale

    for what, got, a, b in (("dx", dx, quantized(dy, 0, "rows"), quantized(w, 1, "columns")),
                            ("dw", dw, quantized(dy, 0, "columns"), quantized(x, 2, "columns"))):
        rows = torch.unique(torch.linspace(0, a[0].shape[0] - 1, 40, device="cuda").long())
        within(got[rows], exact_sums(a[0][rows], b[0]), a[1][rows], b[1], None, what)
        y = torch.empty(got.shape, dtype=got.dtype, device="cuda")
        room = torch.empty(q.qsgd_int_matmul_workspace_bytes(a[0].shape[0], b[0].shape[0], a[0].shape[1]), dtype=torch.uint8, device="cuda")
        q.qsgd_int_matmul(a[0], a[1], b[0], b[1], y, workspace=room)
        assert torch.equal(got, y), what
    # M terms in some order of additions
    assert bool(((db.double() - dy.double().sum(0)).abs() <= R.U32 * M * dy.double().abs().sum(0) + 1e-45).all())


@pytest.mark.parametrize("dtype", R.TYPES, ids=str)
@pytest.mark.parametrize("M,N,K", [(1500, 1501, k) for k in (0, 1, 31, 32, 33, 64)] + [(1400, 1500, 0)], ids=str)
def test_product_of_little_or_no_depth(M, N, K, dtype):
    """Many results of at most two matrix instructions each; of none, where the bias is all there is."""
    a, b = levels(M, K, 1), levels(N, K, 2)
    sa, sb = torch.rand(M, device="cuda") + 0.1, torch.rand(N, device="cuda") + 0.1
    bias = torch.linspace(-3, 3, N, device="cuda")
    sums = exact_sums(a, b)
    for with_bias in (None, bias):
        buf, y = R.framed(M, N, dtype, ld=N + 3, start=1)
        q.qsgd_int_matmul(a, sa, b, sb, y, bias=with_bias)
        within(y, sums, sa, sb, with_bias, dtype)
        assert R.outside_untouched(buf, y)
        if K == 0:
            assert torch.equal(y, (torch.zeros(N, device="cuda") if with_bias is None else bias).to(dtype).expand(M, N))
