"""The operators of a layer in 8 bits against plain forms in 64 bits: sizes that end inside a vector, a
draw block or a tile, strides and alignments, empty and non-finite rows, every type and form."""
import itertools
import struct

import numpy as np
import pytest
import torch

import layer_reference as R
import paper_1610_02132_amd as q
from paper_1610_02132_amd import binding

pytestmark = pytest.mark.gpu

D = q.Draws(seed=0xFEDCBA9876543210, stream_id=3, iteration=9)
TYPES = R.TYPES
NAME = {torch.float32: "f32", torch.bfloat16: "bf16", torch.float16: "f16"}
ids = lambda v: NAME.get(v, str(v).replace(" ", ""))  # noqa: E731


def space(n):
    """A workspace of exactly n bytes inside a larger buffer whose rest must stay as it is."""
    buf = torch.full((max(n, 0) + 256,), 0x5A, dtype=torch.uint8, device="cuda")
    return buf, buf[:n] if n else None


def space_kept(buf, n):
    return bool((buf[n:] == 0x5A).all())


# ---- dropout -----------------------------------------------------------------------

SHAPES = [(1, 1), (1, 8), (3, 7), (1, 4096), (5, 9), (64, 64), (7, 1003), (129, 520), (1031, 17), (2, 20000), (300, 1), (33, 8192)]


@pytest.mark.parametrize("dtype", TYPES, ids=ids)
@pytest.mark.parametrize("rows,cols", SHAPES, ids=str)
def test_dropout(rows, cols, dtype):
    x, res = R.values(rows, cols, dtype, 1), R.values(rows, cols, dtype, 2)
    for p, residual in ((0.1, res), (0.5, None), (0.0, res), (1.0, res), (0.003, None)):
        buf, y = R.framed(rows, cols, dtype, ld=cols + 3, start=5)
        q.qsgd_dropout(D, p, x, y, residual=residual)
        want, tol = R.dropout(D, p, x, residual)
        R.check(y, want, tol, f"p={p}")
        assert R.outside_untouched(buf, y)
    buf, dx = R.framed(rows, cols, dtype)
    q.qsgd_dropout_backward(D, 0.25, x, dx)
    want, tol = R.dropout(D, 0.25, x)
    R.check(dx, want, tol)
    assert R.outside_untouched(buf, dx)


@pytest.mark.parametrize("dtype", TYPES, ids=ids)
@pytest.mark.parametrize("ld,start", [(64, 0), (64, 1), (65, 0), (72, 8), (67, 3)])
def test_dropout_does_not_depend_on_layout(dtype, ld, start):
    rows, cols = 37, 61
    x = R.values(rows, cols, dtype, 3)
    res = R.values(rows, cols, dtype, 4)
    want = torch.empty_like(x.contiguous())
    q.qsgd_dropout(D, 0.3, x, want, residual=res)
    xs, rs = R.framed(rows, cols, dtype, ld=ld, start=start)[1], R.framed(rows, cols, dtype, ld=ld + 8, start=start)[1]
    xs.copy_(x), rs.copy_(res)
    buf, y = R.framed(rows, cols, dtype, ld=ld + 16, start=start)
    q.qsgd_dropout(D, 0.3, xs, y, residual=rs)
    assert torch.equal(y, want) and R.outside_untouched(buf, y)
    q.qsgd_dropout(D, 0.3, xs, xs, residual=rs)       # in place of x
    assert torch.equal(xs, want)
    xs.copy_(x)
    q.qsgd_dropout(D, 0.3, xs, rs, residual=rs)       # in place of the residual
    assert torch.equal(rs, want)


def test_dropout_between_columns_of_one_matrix():
    """Column ranges of a larger matrix: they do not overlap, however close."""
    big = R.values(50, 96, torch.bfloat16, 5, ld=96).contiguous()
    want = torch.empty(50, 32, dtype=torch.bfloat16, device="cuda")
    q.qsgd_dropout(D, 0.2, big[:, :32], want, residual=big[:, 64:])
    keep = big.clone()
    q.qsgd_dropout(D, 0.2, big[:, :32], big[:, 32:64], residual=big[:, 64:])
    assert torch.equal(big[:, 32:64], want) and torch.equal(big[:, :32], keep[:, :32]) and torch.equal(big[:, 64:], keep[:, 64:])
    with pytest.raises(q.QsgdError):
        q.qsgd_dropout(D, 0.2, big[:, :32], big[:, 31:63])


def test_dropout_drops_whatever_the_value_is():
    """Infinities and NaN in dropped places leave nothing; in kept ones they stay."""
    x = torch.full((64, 512), float("nan"), device="cuda")
    x[1::2] = float("inf")
    y = torch.empty_like(x)
    q.qsgd_dropout(D, 0.4, x, y)
    keep = torch.from_numpy(R.half_words(D, 64, 512) >= round(0.4 * 65536)).cuda()
    assert bool((y[~keep] == 0).all())
    assert bool(torch.isnan(y[0::2][keep[0::2]]).all()) and bool(torch.isinf(y[1::2][keep[1::2]]).all())
    q.qsgd_dropout(D, 1.0, x, y)
    assert bool((y == 0).all())


def test_dropout_rows_of_a_slice_draw_like_the_whole():
    x = R.values(50, 77, torch.float32, 5)
    whole, part = torch.empty_like(x), torch.empty_like(x)
    q.qsgd_dropout(D, 0.2, x, whole)
    for r0, r1 in ((0, 13), (13, 14), (14, 50)):
        d = q.Draws(seed=D.seed, stream_id=D.stream_id, iteration=D.iteration, row_base=r0)
        q.qsgd_dropout(d, 0.2, x[r0:r1], part[r0:r1])
    assert torch.equal(whole, part)
    last = q.Draws(seed=D.seed, row_base=2 ** 32 - 50)          # the last rows there are
    q.qsgd_dropout(last, 0.2, x, whole)
    want, tol = R.dropout(last, 0.2, x)
    R.check(whole, want, tol)


def test_dropout_past_32_bits_of_elements():
    """Elements behind the first 2^32: drawn by their row, read and written at their own place."""
    rows, cols = 4200, 2 ** 20
    x = torch.ones(rows, cols, dtype=torch.bfloat16, device="cuda")
    y = torch.empty_like(x)
    q.qsgd_dropout(D, 0.5, x, y)
    for r in (0, 4095, 4096, 4199):
        d = q.Draws(seed=D.seed, stream_id=D.stream_id, iteration=D.iteration, row_base=r)
        want, tol = R.dropout(d, 0.5, x[r:r + 1])
        R.check(y[r:r + 1], want, tol)


def test_dropout_share_and_mean():
    """E y = x: the mean of 2^22 kept-or-dropped ones is within six standard deviations of 1."""
    x = torch.ones(2048, 2048, device="cuda")
    y = torch.empty_like(x)
    for p in (0.1, 0.5, 0.9):
        q.qsgd_dropout(D, p, x, y)
        share = round(65536 * p) / 65536
        assert abs(float(y.double().mean()) - 1.0) < 6 * (share / (1 - share) / 2 ** 22) ** 0.5


# ---- quantizer -----------------------------------------------------------------------

def quantized(x, rounding, form, draws=D, ld_extra=0):
    rows, cols = x.shape
    need = q.qsgd_quantize_workspace_bytes(rows, cols) if form != "rows" else 0
    wsbuf, ws = space(need)
    kw, bufs = {}, []
    if form != "columns":
        buf, kw["rows"] = R.levels(rows, cols, ld=max(16, (cols + 15) // 16 * 16) + ld_extra)
        kw["row_scale"] = torch.full((rows,), 5.0, device="cuda")
        bufs.append((buf, kw["rows"]))
    if form != "rows":
        buf, kw["columns"] = R.levels(cols, rows, ld=max(16, (rows + 15) // 16 * 16) + ld_extra)
        kw["column_scale"] = torch.full((cols,), 5.0, device="cuda")
        bufs.append((buf, kw["columns"]))
    q.qsgd_quantize(draws, x, workspace=ws, rounding=rounding, **kw)
    torch.cuda.synchronize()
    assert all(R.outside_untouched(b, v) for b, v in bufs) and space_kept(wsbuf, need)
    return kw


def check_levels(x, got, rounding, draws=D):
    h = R.half_words(draws, *x.shape) if rounding else None
    for axis, name, scale in ((1, "rows", "row_scale"), (0, "columns", "column_scale")):
        if name not in got:
            continue
        level, s = R.quantize(x, axis, rounding, h)
        g = got[name].cpu().numpy().astype(np.int64)
        assert np.array_equal(g if axis else g.T, level), name
        R.check(got[scale], s, R.U32 * np.abs(s) * 1.01, scale)


QSHAPES = [(1, 1), (1, 16), (2, 7), (1, 5000), (64, 128), (65, 127), (128, 64), (3, 8192), (257, 1003), (1029, 33), (5000, 3),
           (33, 16400), (2, 70001)]


@pytest.mark.parametrize("rounding", (0, 1), ids=("nearest", "stochastic"))
@pytest.mark.parametrize("dtype", TYPES, ids=ids)
@pytest.mark.parametrize("rows,cols", QSHAPES, ids=str)
def test_quantize(rows, cols, dtype, rounding):
    x = R.values(rows, cols, dtype, 6)
    for form in ("rows", "columns", "both"):
        check_levels(x, quantized(x, rounding, form, ld_extra=16), rounding)


@pytest.mark.parametrize("dtype", TYPES, ids=ids)
@pytest.mark.parametrize("ld,start", [(104, 0), (104, 1), (101, 0), (99, 3)])
def test_quantize_does_not_depend_on_layout(dtype, ld, start):
    x = R.values(133, 99, dtype, 7, ld=ld, start=start)
    check_levels(x, quantized(x, 1, "both"), 1)


@pytest.mark.parametrize("rounding", (0, 1), ids=("nearest", "stochastic"))
@pytest.mark.parametrize("dtype", TYPES, ids=ids)
def test_quantize_rows_without_a_scale(dtype, rounding):
    """Rows of zeros, rows too small for a scale, rows with the type's extreme values, an infinity or a NaN."""
    x = R.values(96, 200, dtype, 8)
    info = torch.finfo(dtype)
    x[0] = 0.0
    x[1] = -0.0
    x[2, :] = info.smallest_normal / 4                # (bf16, fp32: below 2^-119)
    x[3] = info.min
    x[4, 7] = info.max
    x[5, 11] = float("inf")
    x[6, 0] = -float("inf")
    x[7, 199] = float("nan")
    x[8, 3], x[8, 4] = float("nan"), float("inf")
    x[9] = 1.0                                        # all at the top level
    if dtype != torch.float16:
        x[10], x[11] = 2.0 ** -119, 2.0 ** -120       # on the two sides of the smallest scale
    check_levels(x, quantized(x, rounding, "both"), rounding)
    x[:, 50] = 0.0
    x[:, 51] = info.min
    check_levels(x, quantized(x, rounding, "both"), rounding)


def test_quantize_no_rows_and_no_columns():
    got = quantized(torch.empty(0, 37, device="cuda"), 0, "both")
    assert bool((got["column_scale"] == 0).all())
    got = quantized(torch.empty(37, 0, device="cuda"), 0, "both")
    assert bool((got["row_scale"] == 0).all())


@pytest.mark.parametrize("rows,cols,dtype,rounding", [(70_001, 1003, torch.float16, 1), (66_000, 1024, torch.bfloat16, 0),
                                                      (40_000, 1700, torch.float32, 1)], ids=str)
def test_quantize_columns_of_many_rows(rows, cols, dtype, rounding):
    """Matrices whose column form takes 512 rows to a workgroup, 128 at a time, and is read past the caches."""
    x = R.values(rows, cols, dtype, 9)
    got = quantized(x, rounding, "both")
    m = x.float().abs().amax(0).cpu().numpy()
    R.check(got["column_scale"], m.astype(np.float64) / 127, R.U32 * m / 127 * 1.01)
    inv = np.float32(127) / m
    some = sorted({0, 1, 127, 128, 511, 512, 640, rows // 2, rows - 100, rows - 2, rows - 1} | set(range(1000, rows, 997)))
    at = torch.tensor(some, device="cuda")
    v, levels = R.host(x[at]), got["columns"].t()[at].cpu().numpy().astype(np.int64)
    for i, r in enumerate(some):
        t = (v[i] * inv).astype(np.float32).astype(np.float64)
        if rounding:
            h = R.half_words(q.Draws(seed=D.seed, stream_id=D.stream_id, iteration=D.iteration, row_base=D.row_base + r), 1, cols)[0]
            low = np.floor(np.abs(t))
            want = np.sign(t) * np.minimum(low + ((h + 0.5) / 65536 < np.abs(t) - low), 127)
        else:
            want = np.rint(t)
        assert np.array_equal(levels[i], want), r


def test_quantize_past_32_bits_of_elements():
    """Both forms of a matrix of more than 2^32 elements: its last rows and columns."""
    rows, cols = 70_016, 65_536
    x = torch.empty(rows, cols, dtype=torch.bfloat16, device="cuda").normal_()
    got = {"rows": torch.empty(rows, cols, dtype=torch.int8, device="cuda"), "row_scale": torch.empty(rows, device="cuda"),
           "columns": torch.empty(cols, rows, dtype=torch.int8, device="cuda"), "column_scale": torch.empty(cols, device="cuda")}
    ws = torch.empty(q.qsgd_quantize_workspace_bytes(rows, cols), dtype=torch.uint8, device="cuda")
    q.qsgd_quantize(None, x, workspace=ws, rounding=0, **got)
    for r in (0, 65_535, 65_536, rows - 1):
        level, scale = R.quantize(x[r:r + 1], 1, 0)
        assert np.array_equal(got["rows"][r:r + 1].cpu().numpy(), level)
        R.check(got["row_scale"][r:r + 1], scale, R.U32 * scale * 1.01)
    for c in (0, 61_345, cols - 1):
        level, scale = R.quantize(x[:, c:c + 1], 0, 0)
        assert np.array_equal(got["columns"][c].cpu().numpy(), level[:, 0])
        R.check(got["column_scale"][c:c + 1], scale, R.U32 * scale * 1.01)


def test_quantize_is_unbiased():
    """The mean of 512 stochastic levels times the scale against the value: 2 levels apart at most, so a standard
    deviation of half a level; six of the mean's, plus the half step of a 16-bit draw."""
    x = R.values(64, 64, torch.float32, 9)
    total = torch.zeros(64, 64, dtype=torch.float64, device="cuda")
    for i in range(512):
        got = quantized(x, 1, "rows", q.Draws(seed=4, iteration=i))
        total += got["rows"].double()
    step = got["row_scale"].double()[:, None]
    off = (total / 512 - x.double() / step).abs()
    assert float(off.max()) < 6 * 0.5 / 512 ** 0.5 + 2.0 ** -17 + 1e-4


# ---- product -----------------------------------------------------------------------

def int_levels(rows, cols, seed, full=False):
    g = torch.Generator()
    g.manual_seed(seed)
    v = torch.randint(-128 if full else -127, 128, (rows, cols), generator=g).to(torch.int8)
    buf, view = R.levels(rows, cols)
    view.copy_(v)
    return view


def scales(n, seed, device="cuda"):
    g = torch.Generator()
    g.manual_seed(seed)
    return (torch.rand(n, generator=g) * 0.01 + 1e-4).to(device)


def multiplied(a, sa, b, sb, dtype, bias=None, ld=None, start=0):
    M, N, K = a.shape[0], b.shape[0], a.shape[1]
    need = q.qsgd_int_matmul_workspace_bytes(M, N, K)
    wsbuf, ws = space(need)
    buf, y = R.framed(M, N, dtype, ld=ld, start=start)
    q.qsgd_int_matmul(a, sa, b, sb, y, bias=bias, workspace=ws)
    torch.cuda.synchronize()
    assert R.outside_untouched(buf, y) and space_kept(wsbuf, need)
    return y


PSHAPES = [(1, 1, 1), (1, 16, 16), (1, 4096, 4096), (1, 100, 65), (2, 17, 31), (3, 64, 64), (7, 33, 129), (15, 300, 500), (16, 256, 64),
           (17, 1000, 2000), (32, 127, 128), (33, 65, 63), (64, 64, 64), (65, 129, 255), (100, 2048, 96), (127, 128, 129), (128, 128, 128),
           (129, 127, 1003), (200, 4096, 33), (255, 257, 256), (256, 256, 256), (257, 255, 300), (300, 500, 4100), (513, 1025, 77),
           (1000, 1000, 1000), (1500, 700, 2000), (4096, 130, 520), (70, 5000, 16), (20, 20, 60000), (2048, 2048, 1024)]


@pytest.mark.parametrize("M,N,K", PSHAPES, ids=str)
def test_product(M, N, K):
    a, b = int_levels(M, K, 1, full=True), int_levels(N, K, 2, full=True)
    sa, sb = scales(M, 3), scales(N, 4)
    bias = torch.linspace(-3, 3, N, device="cuda")
    an, bn = a.cpu().numpy(), b.cpu().numpy()
    for dtype, with_bias in zip(TYPES, (True, False, True)):
        y = multiplied(a, sa, b, sb, dtype, bias if with_bias else None, ld=N + 5, start=3)
        want, tol = R.product(an, sa.cpu().double().numpy(), bn, sb.cpu().double().numpy(), dtype,
                              bias.cpu().numpy() if with_bias else None)
        R.check(y, want, tol, NAME[dtype])


def on_device(a, sa, b, sb):
    """The product in 64 bits on the device (sums below 2^53: exact), and its tolerance in fp32."""
    y = torch.matmul(a.double().contiguous(), b.double().t().contiguous()) * sa.double()[:, None] * sb.double()
    return y, 3 * R.U32 * y.abs() * 1.01 + R.LEAST[torch.float32] + R.U32 * y.abs()


# sizes that go to each of the kernels, with depths that end in, before and behind every stage of its loop
DEPTHS = ([(20, 300, 256 * j + r) for j in range(0, 18, 4) for r in (1, 15, 16, 255)] +
          [(200, 300, 128 * j + r) for j in range(0, 20) for r in (0, 1, 100, 127) if 128 * j + r > 0] +
          [(1024, 4096, 128 * j + r) for j in range(4, 10) for r in (0, 127)] + [(1030, 4090, 1000), (2500, 2500, 300), (2500, 2470, 129)] +
          [(4096, 4096, 128 * j + r) for j in range(11, 15) for r in (0, 1)] + [(4090, 4095, 1500), (5000, 5000, 2001)] +
          [(2041, 2040, 128 * j + r) for j in range(3, 17) for r in (0, 1, 127)] + [(1000, 4000, 2001), (1024, 4096, 4096)])


@pytest.mark.parametrize("M,N", sorted(set(d[:2] for d in DEPTHS)), ids=str)
def test_product_depths(M, N):
    most = max(K for m, n, K in DEPTHS if (m, n) == (M, N))
    big_a, big_b = int_levels(M, most, 1, full=True), int_levels(N, most, 2, full=True)
    sa, sb = scales(M, 3), scales(N, 4)
    for K in [K for m, n, K in DEPTHS if (m, n) == (M, N)]:
        a, b = big_a[:, :K], big_b[:, :K]
        y = multiplied(a, sa, b, sb, torch.float32)
        want, tol = on_device(a, sa, b, sb)
        assert bool(((y.double() - want).abs() <= tol).all()), K


@pytest.mark.parametrize("M,N,K", [(1500, 1501, k) for k in (1, 15, 16, 31, 32, 33, 47, 63, 64)] + [(70, 40_000, 17), (16_401, 130, 64), (3, 700_000, 5)],
                         ids=str)
def test_product_of_little_depth(M, N, K):
    a, b = int_levels(M, K, 1, full=True), int_levels(N, K, 2, full=True)
    sa, sb = scales(M, 3), scales(N, 4)
    bias = torch.linspace(-2, 2, N, device="cuda")
    for dtype, with_bias in zip(TYPES, (True, False, True)):
        y = multiplied(a, sa, b, sb, dtype, bias if with_bias else None, ld=N + 5, start=3)
        want, tol = on_device(a, sa, b, sb)
        if with_bias:
            want, tol = want + bias.double(), tol + R.U32 * (want.abs() + bias.double().abs())
        tol = tol + R.HALF_STEP[dtype] * want.abs() * 1.01 + R.LEAST[dtype]
        assert bool(((y.double() - want).abs() <= tol).all()), dtype


def test_product_in_pieces():
    """Depths that are summed in pieces and joined, results four to a thread and one."""
    for M, N, K in ((64, 64, 8192), (33, 70, 20_000), (50, 71, 9001), (1500, 1500, 20_000), (300, 302, 16_384)):
        assert q.qsgd_int_matmul_workspace_bytes(M, N, K) > 0
        a, b = int_levels(M, K, 1, full=True), int_levels(N, K, 2, full=True)
        sa, sb = scales(M, 3), scales(N, 4)
        bias = torch.linspace(-2, 2, N, device="cuda")
        y = multiplied(a, sa, b, sb, torch.float32, bias)
        want, tol = on_device(a, sa, b, sb)
        want = want + bias.double()
        assert bool(((y.double() - want).abs() <= tol + R.U32 * want.abs()).all()), (M, N, K)


@pytest.mark.parametrize("M,N", [(8200, 8200), (4100, 4101)], ids=str)
def test_pieces_of_more_results_than_one_pass_of_a_launch(M, N):
    """2^26 results four to a thread, 2^24 one to a thread, and some more: the last rows come with a second pass."""
    K = 130_817
    g = torch.Generator(device="cuda")
    g.manual_seed(5)
    ld = (K + 15) // 16 * 16
    a, b = (torch.randint(-127, 128, (n, ld), generator=g, device="cuda", dtype=torch.int8)[:, :K] for n in (M, N))
    sa, sb = scales(M, 3), scales(N, 4)
    y = torch.full((M, N), float("nan"), device="cuda")
    ws = torch.empty(q.qsgd_int_matmul_workspace_bytes(M, N, K), dtype=torch.uint8, device="cuda")
    q.qsgd_int_matmul(a, sa, b, sb, y, workspace=ws)
    assert not bool(y.isnan().any())
    rows = torch.tensor([0, 1, M // 2, M - 2, M - 1], device="cuda")
    want, tol = on_device(a[rows], sa[rows], b, sb)
    assert bool(((y[rows].double() - want).abs() <= tol).all())


@pytest.mark.parametrize("M,N", [(5, 7), (40, 70), (300, 500)], ids=str)
def test_product_of_no_depth_is_the_bias(M, N):
    a, b = int_levels(M, 0, 1), int_levels(N, 0, 2)
    bias = torch.arange(float(N), device="cuda")
    assert torch.equal(multiplied(a, scales(M, 1), b, scales(N, 2), torch.float32, bias), bias.expand(M, N))
    assert bool((multiplied(a, scales(M, 1), b, scales(N, 2), torch.float32) == 0).all())


@pytest.mark.parametrize("M,N,K", [(1, 3, 300_000), (5, 9, 131_072), (70, 40, 131_009), (2, 2, 1_000_003)], ids=str)
def test_product_sums_past_32_bits(M, N, K):
    """All products of one sign and the largest there are: the sums pass 2^31 from 131072 terms on (131009 * 2^14 is
    just below) and stay exact."""
    a, b = int_levels(M, K, 1), int_levels(N, K, 2)
    a.fill_(-128), b.fill_(-128)
    a[0, :5] = 1
    one = torch.ones(M, device="cuda"), torch.ones(N, device="cuda")
    y = multiplied(a, one[0], b, one[1], torch.float32)
    want = (a.cpu().numpy().astype(np.float64) @ b.cpu().numpy().astype(np.float64).T)
    assert (abs(want).max() >= 2 ** 31) == (K >= 131_072)
    R.check(y, want, R.U32 * np.abs(want))


@pytest.mark.parametrize("times", (1, 7, 200), ids=str)
def test_product_scales_at_the_ends_of_the_range(times):
    """Scales whose product, or whose product with the sum, leaves fp32 while the result does not; NaN and zero rows."""
    a, b = int_levels(6 * times, 64, 1), int_levels(6 * times, 64, 2)
    a.fill_(100), b.fill_(100)
    sa = torch.tensor([2.0 ** -120, 2.0 ** 120, 0.0, 1.0, float("nan"), 1e-30] * times, device="cuda")
    sb = torch.tensor([2.0 ** 120, 2.0 ** -120, 1.0, 1e-30, 1.0, float("nan")] * times, device="cuda")
    y = multiplied(a, sa, b, sb, torch.float32)
    with np.errstate(all="ignore"):
        want = 640000.0 * sa.double().cpu().numpy()[:, None] * sb.double().cpu().numpy()[None]
    over = np.abs(want) > torch.finfo(torch.float32).max
    g = y.double().cpu().numpy()
    assert np.isinf(g[over]).all()
    R.check(np.where(over, 0, g), np.where(over, 0, want), R.U32 * 3 * np.where(over, 0, np.abs(np.nan_to_num(want))) * 1.01 + 2.0 ** -149)


@pytest.mark.parametrize("M,N", [(2, 3), (70, 40)], ids=str)
def test_product_of_long_sums_and_large_scales(M, N):
    """A sum near 2^37 times a scale of 2^95 leaves fp32, the result of the two scales does not."""
    K = 8_000_000
    a, b = (torch.full((n, K), 127, dtype=torch.int8, device="cuda") for n in (M, N))
    for s, t in ((2.0 ** 95, 2.0 ** -100), (2.0 ** -100, 2.0 ** 95), (2.0 ** 91, 2.0 ** -30), (2.0 ** 89, 1.0)):
        y = torch.empty(M, N, device="cuda")
        ws = torch.empty(q.qsgd_int_matmul_workspace_bytes(M, N, K), dtype=torch.uint8, device="cuda")
        q.qsgd_int_matmul(a, torch.full((M,), s, device="cuda"), b, torch.full((N,), t, device="cuda"), y, workspace=ws)
        want = K * 127.0 ** 2 * s * t
        assert bool(((y.double() - want).abs() <= 4 * R.U32 * want).all()), (s, t)


def test_product_past_32_bits_of_results():
    M, N, K = 66_000, 66_001, 48
    a, b = int_levels(M, K, 1, full=True), int_levels(N, K, 2, full=True)
    sa, sb = scales(M, 3), scales(N, 4)
    y = torch.empty(M, N, device="cuda")
    q.qsgd_int_matmul(a, sa, b, sb, y)
    at = torch.tensor([0, 1, 65_074, 65_075, M - 1], device="cuda")    # (65075 N is behind 2^32)
    want, tol = on_device(a[at], sa[at], b, sb)
    assert bool(((y[at].double() - want).abs() <= tol).all())


@pytest.mark.parametrize("M", [7, 1100], ids=str)
def test_product_of_rows_far_apart(M):
    """Operands that span more than 2^32 bytes, for the kernels of few rows and of tiles."""
    N, K, ld = 1100, 300, 2 ** 22 + 16
    a, b = (torch.empty(n, ld, dtype=torch.int8, device="cuda")[:, 1600:1600 + K] for n in (M, N))
    a.copy_(int_levels(M, K, 1, full=True)), b.copy_(int_levels(N, K, 2, full=True))
    sa, sb = scales(M, 3), scales(N, 4)
    y = multiplied(a, sa, b, sb, torch.float32)
    want, tol = on_device(a, sa, b, sb)
    assert bool(((y.double() - want).abs() <= tol).all())


def test_product_operands_in_larger_matrices():
    """Column ranges of wider matrices: what stands behind K in a row, levels and all, changes nothing."""
    big_a, big_b = int_levels(90, 400, 1, full=True), int_levels(110, 400, 2, full=True)
    sa, sb = scales(90, 3), scales(110, 4)
    for k0, k1 in ((0, 400), (16, 377), (128, 129), (0, 15), (160, 352)):
        y = multiplied(big_a[:, k0:k1], sa, big_b[:, k0:k1], sb, torch.float32)
        want, tol = R.product(big_a[:, k0:k1].cpu().numpy(), sa.double().cpu().numpy(), big_b[:, k0:k1].cpu().numpy(),
                              sb.double().cpu().numpy(), torch.float32)
        R.check(y, want, tol, f"{k0}:{k1}")


# ---- linear layer -------------------------------------------------------------------

LSHAPES = [(1, 1, 1), (1, 64, 64), (1, 4096, 1024), (2, 100, 333), (4, 1000, 2048), (5, 7, 9), (16, 300, 500), (17, 257, 1030), (64, 64, 64),
           (100, 515, 129), (130, 70, 2000), (777, 130, 65), (1000, 260, 300), (3, 2, 20000), (1, 48, 40000)]


@pytest.mark.parametrize("dtype", TYPES, ids=ids)
@pytest.mark.parametrize("M,N,K", LSHAPES, ids=str)
def test_linear_forward(M, N, K, dtype):
    x = R.values(M, K, dtype, 1)
    if M > 2:
        x[1] = 0.0
    w, ws = int_levels(N, K, 2), scales(N, 3)
    bias = torch.linspace(-1, 1, N, device="cuda")
    need = q.qsgd_linear_forward_workspace_bytes(M, N, K)
    for rounding, b in ((0, bias), (1, None)):
        wsbuf, work = space(need)
        buf, y = R.framed(M, N, dtype, ld=N + 3)
        q.qsgd_linear_forward(D if rounding else None, x, w, ws, y, bias=b, workspace=work, rounding=rounding)
        torch.cuda.synchronize()
        level, scale = R.quantize(x, 1, rounding, R.half_words(D, M, K) if rounding else None)
        want, tol = R.product(level, scale, w.cpu().numpy(), ws.double().cpu().numpy(), dtype,
                              None if b is None else b.cpu().numpy(), scale_roundings=1)
        R.check(y, want, tol)
        assert R.outside_untouched(buf, y) and space_kept(wsbuf, need)


@pytest.mark.parametrize("M,N,K", [(1, 1, 1), (1, 4096, 4096), (1, 300, 47_000), (3, 77, 1000), (4, 500, 8192), (7, 33, 129), (16, 64, 2700),
                                   (16, 100, 255), (16, 8192, 2048), (40, 300, 512), (3, 12_288, 100), (1, 12_289, 4096),
                                   (2, 32_768, 2048), (1, 32_769, 48)], ids=str)
def test_linear_forward_is_quantizer_and_product(M, N, K):
    """Bit for bit, whichever way it takes."""
    for dtype, rounding in zip(TYPES, (1, 0, 1)):
        x, w, ws = R.values(M, K, dtype, 1), int_levels(N, K, 2), scales(N, 3)
        bias = torch.linspace(-1, 1, N, device="cuda")
        work = torch.empty(q.qsgd_linear_forward_workspace_bytes(M, N, K), dtype=torch.uint8, device="cuda")
        y = torch.empty(M, N, dtype=dtype, device="cuda")
        q.qsgd_linear_forward(D, x, w, ws, y, bias=bias, workspace=work, rounding=rounding)
        got = quantized(x, rounding, "rows")
        assert torch.equal(y, multiplied(got["rows"], got["row_scale"], w, ws, dtype, bias))


def test_linear_forward_rows_without_a_scale():
    """A token of zeros gives the bias, one with an infinity or a NaN gives NaN, and the others are as without it."""
    for M in (4, 40):
        x = R.values(M, 200, torch.bfloat16, 1)
        w, ws, bias = int_levels(70, 200, 2), scales(70, 3), torch.linspace(-1, 1, 70, device="cuda")
        work = torch.empty(max(16, q.qsgd_linear_forward_workspace_bytes(M, 70, 200)), dtype=torch.uint8, device="cuda")
        y, z = torch.empty(M, 70, dtype=torch.bfloat16, device="cuda"), torch.empty(M, 70, dtype=torch.bfloat16, device="cuda")
        q.qsgd_linear_forward(None, x, w, ws, y, bias=bias, workspace=work)
        x[0], x[1, 5], x[2, 6] = 0.0, float("inf"), float("nan")
        q.qsgd_linear_forward(None, x, w, ws, z, bias=bias, workspace=work)
        assert torch.equal(z[0], bias.bfloat16()) and bool(torch.isnan(z[1:3]).all()) and torch.equal(y[3:], z[3:])


def backward(x, w, dy, rounding=1, draws=D, want=("dx", "dw", "db")):
    M, N, K = dy.shape[0], dy.shape[1], x.shape[1]
    need = q.qsgd_linear_backward_workspace_bytes(M, N, K)
    wsbuf, ws = space(need)
    out, bufs = {}, []
    for name, (r, c, t) in {"dx": (M, K, x.dtype), "dw": (N, K, torch.float32)}.items():
        if name in want:
            buf, out[name] = R.framed(r, c, t)
            bufs.append((buf, out[name]))
    if "db" in want:
        out["db"] = torch.full((N,), 9.0, device="cuda")
    q.qsgd_linear_backward(draws, x, w, dy, workspace=ws, rounding=rounding, **out)
    torch.cuda.synchronize()
    assert all(R.outside_untouched(b, v) for b, v in bufs) and space_kept(wsbuf, need)
    return out


def shifted(d, by, base):
    return q.Draws(seed=d.seed, stream_id=d.stream_id + by, iteration=d.iteration, row_base=base)


def expected_gradients(x, w, dy, rounding, d=D):
    M, N, K = dy.shape[0], dy.shape[1], x.shape[1]
    hd, hw, hx = (R.half_words(d, M, N), R.half_words(shifted(d, 1, 0), N, K),
                  R.half_words(shifted(d, 2, d.row_base), M, K)) if rounding else (None,) * 3
    r, rs = R.quantize(dy, 1, rounding, hd)
    c, cs = R.quantize(dy, 0, rounding, hd)
    wq, wsc = R.quantize(w, 0, rounding, hw)
    xq, xs = R.quantize(x, 0, rounding, hx)
    g = R.host(dy).astype(np.float64)
    return {"dx": R.product(r, rs, wq.T, wsc, x.dtype, scale_roundings=2),
            "dw": R.product(c.T, cs, xq.T, xs, torch.float32, scale_roundings=2),
            # M terms in some order of additions
            "db": (g.sum(0), R.U32 * M * np.abs(g).sum(0) + 1e-45)}


@pytest.mark.parametrize("dtype", TYPES, ids=ids)
@pytest.mark.parametrize("M,N,K", LSHAPES, ids=str)
def test_linear_backward(M, N, K, dtype):
    x, w, dy = R.values(M, K, dtype, 1), R.values(N, K, dtype, 2, scale=0.05), R.values(M, N, dtype, 3, scale=0.5)
    if M > 3:
        dy[1], x[2] = 0.0, 0.0
    for rounding in (0, 1):
        want = expected_gradients(x, w, dy, rounding)
        got = backward(x, w, dy, rounding)
        for name, (v, tol) in want.items():
            R.check(got[name], v, tol, name)


@pytest.mark.parametrize("M,N,K", [(40, 1500, 1600), (2100, 60, 1100), (60, 64, 40_000), (1, 1460, 1460)], ids=str)
def test_linear_backward_of_few_tokens_or_outputs(M, N, K):
    """Gradients of many values and little depth: the weights', the input's, both."""
    x, w, dy = R.values(M, K, torch.bfloat16, 1), R.values(N, K, torch.bfloat16, 2), R.values(M, N, torch.bfloat16, 3)
    for name, (v, tol) in expected_gradients(x, w, dy, 1, D).items():
        R.check(backward(x, w, dy)[name], v, tol, name)


@pytest.mark.parametrize("M,N,K", [(0, 5, 8), (5, 0, 8), (5, 8, 0), (300, 8, 0)], ids=str)
def test_linear_of_no_tokens_outputs_or_inputs(M, N, K):
    x, w, ws = torch.ones(M, K, device="cuda"), int_levels(N, K, 1), scales(N, 2)
    bias = torch.arange(float(N), device="cuda")
    y = torch.full((M, N), 7.0, device="cuda")
    work = torch.empty(q.qsgd_linear_forward_workspace_bytes(M, N, K), dtype=torch.uint8, device="cuda")
    q.qsgd_linear_forward(D, x, w, ws, y, bias=bias, workspace=work, rounding=1)
    assert torch.equal(y, bias.expand(M, N))
    dx, dw, db = (torch.full(s, 7.0, device="cuda") for s in ((M, K), (N, K), (N,)))
    work = torch.empty(q.qsgd_linear_backward_workspace_bytes(M, N, K), dtype=torch.uint8, device="cuda")
    q.qsgd_linear_backward(D, x, torch.ones(N, K, device="cuda"), torch.ones(M, N, device="cuda"), dx, dw, db, work, 1)
    # (a NaN or a 7 would say that something was not written)
    assert bool((dx == 0).all()) and bool((dw == 0).all()) and bool((db == M).all())


def test_linear_backward_of_no_tokens():
    got = backward(torch.empty(0, 40, device="cuda"), R.values(24, 40, torch.float32, 1), torch.empty(0, 24, device="cuda"))
    assert bool((got["dw"] == 0).all()) and bool((got["db"] == 0).all())


def test_linear_backward_any_choice_of_gradients():
    x, w, dy = R.values(70, 90, torch.bfloat16, 1), R.values(50, 90, torch.bfloat16, 2), R.values(70, 50, torch.bfloat16, 3)
    whole = backward(x, w, dy)
    for k in (1, 2):
        for want in itertools.combinations(("dx", "dw", "db"), k):
            for name, v in backward(x, w, dy, want=want).items():
                assert torch.equal(v, whole[name]), (want, name)


def test_gradients_are_those_of_the_formula_where_levels_are_exact():
    """Whole numbers with 127 in every row and column are their own levels: the gradients are exact, and equal the
    differences of the layer's output, which is linear in each of its arguments."""
    M, N, K = 40, 24, 56
    g = np.random.default_rng(5)

    def whole(r, c):
        v = g.integers(-127, 128, (r, c)).astype(np.float64)
        v[np.arange(max(r, c)) % r, np.arange(max(r, c)) % c] = 127
        return v

    x, w, dy = whole(M, K), whole(N, K), whole(M, N)
    t = lambda v: torch.from_numpy(v).float().cuda()  # noqa: E731
    for rounding in (0, 1):
        got = backward(t(x), t(w), t(dy), rounding)
        for name, want in (("dx", dy @ w), ("dw", dy.T @ x), ("db", dy.sum(0))):
            R.check(got[name], want, 5 * R.U32 * np.abs(want), name)
    loss = lambda x, w, b: float(((x @ w.T + b) * dy).sum())  # noqa: E731  (its gradient by y is dy)
    b = np.zeros(N)
    for r, c in ((0, 0), (3, 7), (23, 55)):
        for name, arg in (("dx", 0), ("dw", 1)):
            e = [np.zeros_like(x), np.zeros_like(w)]
            e[arg][r, c] = 1.0
            diff = (loss(x + e[0], w + e[1], b) - loss(x - e[0], w - e[1], b)) / 2
            assert abs(float(got[name][r, c]) - diff) <= 5 * R.U32 * abs(diff) + 1e-6
        eb = np.zeros(N)
        eb[r] = 1.0
        assert abs(float(got["db"][r]) - (loss(x, w, b + eb) - loss(x, w, b - eb)) / 2) <= 1e-3


def test_gradients_are_unbiased():
    """Means of 256 gradients from stochastic levels against dy w and dy^T x.  A level is off by at most one step,
    with variance at most step^2 / 4; the variance of a sum of products of independent factors is the sum of
    (a^2 + va)(b^2 + vb) - a^2 b^2, and six standard deviations of the mean are allowed."""
    M, N, K, runs = 48, 40, 32, 256
    x, w, dy = R.values(M, K, torch.float32, 1), R.values(N, K, torch.float32, 2), R.values(M, N, torch.float32, 3)
    total = {"dx": 0.0, "dw": 0.0}
    for i in range(runs):
        got = backward(x, w, dy, 1, q.Draws(seed=11, iteration=i), want=("dx", "dw"))
        for k in total:
            total[k] = total[k] + got[k].double()
    X, W, G = (R.host(t).astype(np.float64) for t in (x, w, dy))
    var = lambda v, axis: np.broadcast_to((np.abs(v).max(axis=axis, keepdims=True) / 127) ** 2 / 4, v.shape)  # noqa: E731

    def spread(a, va, b, vb):   # sums over the first one's last axis
        return np.sqrt((a ** 2 + va) @ (b ** 2 + vb) - (a ** 2) @ (b ** 2))

    for name, want, sd in (("dx", G @ W, spread(G, var(G, 1), W, var(W, 0))),
                           ("dw", G.T @ X, spread(G.T, var(G, 0).T, X, var(X, 0)))):
        off = np.abs(total[name].cpu().numpy() / runs - want)
        # (the draws' half step, 2^-17 of a level, is far below the spread)
        assert (off <= 6 * sd / runs ** 0.5 + 1e-5 * np.abs(want)).all(), (name, (off / sd).max() * runs ** 0.5)


def test_weights_draw_by_their_own_rows():
    """A slice of tokens with row_base: its dx are the whole batch's rows."""
    x, w, dy = R.values(60, 64, torch.float32, 1), R.values(40, 64, torch.float32, 2), R.values(60, 40, torch.float32, 3)
    whole = backward(x, w, dy, want=("dx",))["dx"]
    part = backward(x[20:50], w, dy[20:50], 1, shifted(D, 0, 20), want=("dx",))["dx"]
    assert torch.equal(part, whole[20:50])


# ---- as they are used ----------------------------------------------------------------

class Block:
    """y = residual + dropout(linear(x)) with its backward pass, and the weights' update through the codec."""

    def __init__(self, M, N, K, dtype):
        self.w = R.values(N, K, dtype, 20, scale=0.05).contiguous()
        self.master = self.w.float().clone()
        self.bias = torch.linspace(-0.1, 0.1, N, device="cuda")
        self.x, self.res = R.values(M, K, dtype, 21).contiguous(), R.values(M, N, dtype, 22).contiguous()
        self.dy = R.values(M, N, dtype, 23, scale=0.1).contiguous()
        new = lambda r, c, t: torch.empty(r, c, dtype=t, device="cuda")  # noqa: E731
        self.wq, self.wscale = R.levels(N, K)[1], torch.empty(N, device="cuda")
        self.lin, self.y, self.dlin = (new(M, N, dtype) for _ in range(3))
        self.dx = new(M, K, dtype)
        self.dw, self.db = new(N, K, torch.float32), torch.empty(N, device="cuda")
        need = max(q.qsgd_linear_forward_workspace_bytes(M, N, K), q.qsgd_linear_backward_workspace_bytes(M, N, K),
                   q.qsgd_quantize_workspace_bytes(N, K))
        self.ws = torch.empty(need, dtype=torch.uint8, device="cuda")
        self.P = q.Params(n=N * K, s=16, d=512, seed=1)
        self.msg = torch.zeros(q.qsgd_max_encoded_bytes(self.P) // 4, dtype=torch.int32, device="cuda")
        self.cws = torch.zeros(q.qsgd_workspace_bytes(self.P, 1) // 4, dtype=torch.int32, device="cuda")

    def step(self, draws):
        drop = q.Draws(seed=draws.seed, stream_id=draws.stream_id + 8, iteration=draws.iteration, iteration_dev=draws.iteration_dev)
        self.w.copy_(self.master)
        q.qsgd_quantize(None, self.w, rows=self.wq, row_scale=self.wscale)
        q.qsgd_linear_forward(None, self.x, self.wq, self.wscale, self.lin, bias=self.bias, workspace=self.ws)
        q.qsgd_dropout(drop, 0.1, self.lin, self.y, residual=self.res)
        q.qsgd_dropout_backward(drop, 0.1, self.dy, self.dlin)
        q.qsgd_linear_backward(draws, self.x, self.w, self.dlin, dx=self.dx, dw=self.dw, db=self.db, workspace=self.ws,
                               rounding=q.ROUND_STOCHASTIC)
        q.qsgd_encode(self.P, self.dw.view(-1), self.msg, self.cws)
        q.qsgd_sgd_step(self.P, [self.msg], 0.1, self.master.view(-1), self.cws)

    def results(self):
        return {k: getattr(self, k).clone() for k in ("lin", "y", "dlin", "dx", "dw", "db", "master", "wq", "wscale")}


@pytest.mark.parametrize("dtype", TYPES, ids=ids)
@pytest.mark.parametrize("M,N,K", [(64, 128, 256), (333, 130, 100)], ids=str)
def test_training_step(M, N, K, dtype):
    """The operators one after the other and the codec behind them, each against its plain form on what it got."""
    b = Block(M, N, K, dtype)
    before = b.master.clone()
    d = q.Draws(seed=77, stream_id=1, iteration=2)
    b.step(d)
    torch.cuda.synchronize()
    drop = shifted(d, 8, 0)
    wl, wsc = R.quantize(b.w, 1, 0)
    assert np.array_equal(b.wq.cpu().numpy(), wl)
    xl, xs = R.quantize(b.x, 1, 0)
    R.check(b.lin, *R.product(xl, xs, wl, wsc, dtype, b.bias.cpu().numpy(), scale_roundings=2), "lin")
    R.check(b.y, *R.dropout(drop, 0.1, b.lin, b.res), "y")
    R.check(b.dlin, *R.dropout(drop, 0.1, b.dy), "dlin")
    for name, (v, tol) in expected_gradients(b.x, b.w, b.dlin, 1, d).items():
        R.check(getattr(b, name), v, tol, name)
    from oracle import qsgd_oracle as qo
    words = qo.encode(qo.Params(n=N * K, s=16, d=512, code=0, seed=1), b.dw.view(-1).cpu().numpy())
    assert np.array_equal(b.msg.cpu().numpy().view(np.uint32)[:len(words)], words)
    want = qo.sgd_step([words], 0.1, before.view(-1).cpu().numpy())
    assert np.array_equal(b.master.view(-1).cpu().numpy(), want)


def test_training_step_in_a_graph():
    """Captured with the iteration in device memory: every replay gives what eager steps give, draws and all, with
    eager work of the same operators between the replays."""
    eager, block, other = (Block(100, 72, 130, torch.bfloat16) for _ in range(3))
    it = torch.zeros(1, dtype=torch.int32, device="cuda")
    draws = q.Draws(seed=5, iteration=10, iteration_dev=it)
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        block.step(draws)                 # (warm)
    torch.cuda.synchronize()
    block.master.copy_(eager.master)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        block.step(draws)
        it.add_(1)
    it.zero_()
    block.master.copy_(eager.master)
    torch.cuda.synchronize()
    seen = []
    for i in range(4):
        graph.replay()
        torch.cuda.synchronize()
        eager.step(q.Draws(seed=5, iteration=10 + i))
        other.step(q.Draws(seed=6, iteration=i))
        torch.cuda.synchronize()
        want, got = eager.results(), block.results()
        for k in want:
            assert torch.equal(want[k], got[k]), (i, k)
        seen.append(got["dlin"])
    assert not torch.equal(seen[0], seen[1])


def test_calls_on_two_streams():
    """Two blocks of their own, each on its stream, interleaved call by call."""
    one, two = Block(200, 96, 160, torch.bfloat16), Block(200, 96, 160, torch.bfloat16)
    ref = Block(200, 96, 160, torch.bfloat16)
    ref.step(D)
    torch.cuda.synchronize()
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    for _ in range(3):
        for b, s in ((one, s1), (two, s2)):
            with torch.cuda.stream(s):
                b.master.copy_(ref.w)
                b.step(D)
    torch.cuda.synchronize()
    want = ref.results()
    for b in (one, two):
        got = b.results()
        assert all(torch.equal(want[k], got[k]) for k in want)


def test_a_stream_of_the_callers_choice():
    x, y = R.values(64, 96, torch.float32, 1).contiguous(), torch.zeros(64, 96, device="cuda")
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    q.qsgd_dropout(D, 0.1, x, y, stream=s)
    s.synchronize()
    R.check(y, *R.dropout(D, 0.1, x))


def test_kernels_are_timed_by_name():
    x = R.values(64, 96, torch.float32, 1).contiguous()
    y = torch.empty_like(x)
    q.qsgd_timing_enable(True)
    q.qsgd_timing_reset()
    q.qsgd_dropout(D, 0.1, x, y)
    ms, launches = q.qsgd_timing_get("dropout")
    q.qsgd_timing_enable(False)
    q.qsgd_timing_reset()
    assert launches == 1 and ms > 0


def test_the_c_abi_takes_a_null_residual_and_counts_rows_apart():
    """Straight through the C ABI: a matrix whose single row has any ld."""
    L = binding._load()
    x = torch.ones(1, 40, device="cuda")
    y = torch.zeros(1, 40, device="cuda")
    matrix = lambda t, ld: struct.pack("=QQQQII", t.data_ptr(), 1, 40, ld, 0, 0)  # noqa: E731  (struct qsgd_matrix)
    assert L.qsgd_dropout(D.c(), 0.5, matrix(x, 1000), None, matrix(y, 40), None) == 0
    torch.cuda.synchronize()
    R.check(y, *R.dropout(D, 0.5, x))
