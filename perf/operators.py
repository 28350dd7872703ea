"""The operators of a layer in 8 bits, with cases on which their speed is watched.

Next to the codec, the library has what stands in front of it in a training program: dropout whose
mask is drawn from the counter-based generator and never stored, the quantizer with a scale per row
or per column, the product of 8-bit integers with those scales, and the linear layer made of the
two, forward and backward.  Its weight gradient is what `qsgd_encode` takes.

A case is
  op      dropout | dropout_backward | quantize | product | linear | linear_backward
  type    f32 | bf16 | f16: of the activations (product: of the result)
  M, N, K dropout and quantize: a matrix of M rows and K columns (N = 0); product: M x K times
          (N x K) transposed; linear: M tokens, K inputs, N outputs
  p       share that is dropped          residual, bias   whether there is one
  round   nearest | stochastic           form             rows | columns | both (quantize)

Definitions that both forms below keep.  Draw of element (r, c) of a matrix: the 16-bit half word
c % 8 of the Philox-4x32-10 block with counter (c / 8, r, stream, iteration) and the seed as key.
Dropout keeps where the draw is at least D = rint(65536 p), times 65536 / (65536 - D).  A level is
fl(|x| fl(127 / m)) in fp32, m the largest magnitude of the row or column, rounded to nearest (ties
to even) or up where (draw + 0.5) / 65536 is below its fraction; it stands for level * m / 127.
"""
from __future__ import annotations

import numpy as np
import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}
SEED, STREAM, ITERATION = 0x1234567890ABCDEF, 5, 7   # of every case's draws
TINY = 2.0 ** -119                                   # below it a row counts as zero


def _case(name, op, kind, M, N, K, p=0.0, residual=False, bias=False, rounding="nearest", form="rows"):
    return {"name": name, "op": op, "type": kind, "M": M, "N": N, "K": K, "p": p, "residual": residual,
            "bias": bias, "round": rounding, "form": form}


def listed():
    return [
        # a few tokens of a small model: launch and the host's part of a call; the last draw block is cut
        _case("dropout_few", "dropout", "bf16", 4, 0, 1004, p=0.1, residual=True),
        # the end of a block in training, added to the residual stream
        _case("dropout_residual", "dropout", "bf16", 8192, 0, 4096, p=0.1, residual=True),
        # its gradient in fp32; rows that no vector load fits
        _case("dropout_backward_odd", "dropout_backward", "f32", 5003, 0, 2049, p=0.25),
        # activations of a batch, a scale per token
        _case("quantize_tokens", "quantize", "bf16", 8192, 0, 4096),
        # a gradient that is needed along both axes, unbiased; odd sizes
        _case("quantize_both_odd", "quantize", "f16", 2047, 0, 1001, rounding="stochastic", form="both"),
        # a single token: the weights' bytes are all there is to it
        _case("product_token", "product", "bf16", 1, 4096, 4096),
        # a ragged batch, nothing a multiple of a tile
        _case("product_ragged", "product", "f16", 333, 1111, 2223, bias=True),
        # the largest product
        _case("product_large", "product", "bf16", 8192, 8192, 8192),
        # a few requests at once, activations quantized on the way
        _case("linear_few", "linear", "bf16", 16, 8192, 4096, bias=True),
        # a training batch forward
        _case("linear_batch", "linear", "bf16", 8192, 4096, 4096, bias=True),
        # a small layer's gradients in fp32, odd sizes
        _case("linear_backward_odd", "linear_backward", "f32", 777, 515, 1001, rounding="stochastic"),
        # a training batch backward: gradients of input, weights and bias
        _case("linear_backward_batch", "linear_backward", "bf16", 8192, 4096, 4096, bias=True, rounding="stochastic"),
    ]


def _size(rng, lo, hi):
    """A whole number, its logarithm spread evenly; rounded to a multiple of 64 half of the time, as sizes of layers are."""
    v = lo * (hi / lo) ** rng.random()
    return max(lo, int(v / 64 + 0.5) * 64) if rng.random() < 0.5 and v >= 64 else max(lo, int(v))


def draw(rng):
    op = rng.choice(["dropout", "dropout_backward", "quantize", "product", "linear", "linear_backward"])
    c = {"op": op, "type": rng.choice(["f32", "bf16", "f16"]), "M": 0, "N": 0, "K": 0, "p": 0.0, "residual": False,
         "bias": False, "round": "nearest", "form": "rows"}
    c["M"], c["K"] = _size(rng, 1, 8192), _size(rng, 16, 8192)
    if op.startswith("dropout"):
        c["p"] = rng.choice([0.05, 0.1, 0.2, 0.5])
        c["residual"] = op == "dropout" and rng.random() < 0.7
    elif op == "quantize":
        c["round"], c["form"] = rng.choice(["nearest", "stochastic"]), rng.choice(["rows", "columns", "both"])
    else:
        c["N"] = _size(rng, 16, 8192 if op != "linear_backward" else 4096)
        c["bias"] = rng.random() < 0.5
        if op != "product":
            c["round"] = "stochastic" if op == "linear_backward" else "nearest"
    return c


# ---- inputs ---------------------------------------------------------------------------------------

def _values(g, rows, cols, dtype, scale):
    """Normal values, channels of different sizes, some of them far above the rest; the last row in 64 is padding."""
    x = torch.randn(rows, cols, device="cuda", generator=g)
    x *= scale * torch.exp(0.7 * torch.randn(cols, device="cuda", generator=g))
    x[63::64] = 0.0
    return x.to(dtype)


def _padded(rows, cols):
    """A matrix of bytes whose rows start at multiples of 16, as the products want them."""
    return torch.empty(rows, (cols + 15) // 16 * 16, dtype=torch.int8, device="cuda")[:, :cols]


def _levels(g, rows, cols):
    """8-bit levels as a quantized matrix has them, and a scale for each row."""
    q = _padded(rows, cols)
    q.copy_((torch.randn(rows, cols, device="cuda", generator=g) * 36).round_().clamp_(-127, 127))
    return q, torch.rand(rows, device="cuda", generator=g) * 0.01 + 1e-3


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    op, M, N, K = case["op"], case["M"], case["N"], case["K"]
    t = TYPES[case["type"]]
    s = {"case": case}
    bias = lambda: torch.randn(N, device="cuda", generator=g) * 0.1 if case["bias"] else None  # noqa: E731
    if op == "dropout":
        s["x"] = _values(g, M, K, t, 1.0)
        s["residual"] = _values(g, M, K, t, 1.0) if case["residual"] else None
    elif op == "dropout_backward":
        s["dy"] = _values(g, M, K, t, 1e-3)
    elif op == "quantize":
        s["x"] = _values(g, M, K, t, 1.0)
    elif op == "product":
        s["a"], s["a_scale"] = _levels(g, M, K)
        s["b"], s["b_scale"] = _levels(g, N, K)
        s["bias"] = bias()
    elif op == "linear":
        s["x"] = _values(g, M, K, t, 1.0)
        s["w"], s["w_scale"] = _levels(g, N, K)
        s["bias"] = bias()
    else:
        s["x"], s["w"], s["dy"] = _values(g, M, K, t, 1.0), _values(g, N, K, t, 0.02), _values(g, M, N, t, 1e-3)
    return s


# ---- the plain form -------------------------------------------------------------------------------

def _half_words(rows, cols, stream):
    """The 16-bit draws of a matrix, in 64-bit integers."""
    blocks = (cols + 7) // 8
    x = [torch.arange(blocks, device="cuda").repeat(rows, 1), torch.arange(rows, device="cuda")[:, None].repeat(1, blocks)]
    x += [torch.full_like(x[0], stream), torch.full_like(x[0], ITERATION)]
    k0, k1 = SEED & 0xFFFFFFFF, SEED >> 32
    for _ in range(10):
        h0, l0 = _product_words(x[0], 0xD2511F53)
        h1, l1 = _product_words(x[2], 0xCD9E8D57)
        x = [h1 ^ x[1] ^ k0, l1, h0 ^ x[3] ^ k1, l0]
        k0, k1 = (k0 + 0x9E3779B9) & 0xFFFFFFFF, (k1 + 0xBB67AE85) & 0xFFFFFFFF
    w = torch.stack(x, dim=-1)
    return torch.stack((w & 0xFFFF, w >> 16), dim=-1).reshape(rows, 8 * blocks)[:, :cols]


def _product_words(x, m):
    """High and low word of a 32 x 32 bit product: it passes 63 bits, so the high word comes from halves."""
    return (x * (m >> 16) + ((x * (m & 0xFFFF)) >> 16)) >> 16, (x * m) & 0xFFFFFFFF


def _plain_dropout(x, p, residual):
    D = round(65536 * float(np.float32(p)))
    y = torch.where(_half_words(x.shape[0], x.shape[1], STREAM) >= D, x.float() * (65536.0 / (65536 - D)), 0.0)
    return (y if residual is None else residual.float() + y).to(x.dtype)


def _plain_quantize(x, dim, rounding, stream):
    """Levels (int8) and scales along `dim` (1: a scale for each row, 0: for each column)."""
    v = x.float()
    m = v.abs().amax(dim=dim, keepdim=True)
    m = torch.where(m < TINY, 0.0, m)
    t = v * torch.where(m > 0, torch.full_like(m, 127.0) / m, 0.0)
    if rounding == "nearest":
        t = t.round()
    else:
        a = t.abs()
        low = a.floor()
        u = (_half_words(x.shape[0], x.shape[1], stream).float() + 0.5) / 65536
        t = torch.copysign((low + (u < a - low)).clamp(max=127.0), t)
    return t.to(torch.int8), (m / torch.full_like(m, 127.0)).squeeze(dim)


def _plain_product(a, a_scale, b, b_scale, bias, dtype):
    y = (a.float() @ b.float().t()) * a_scale[:, None] * b_scale
    return (y if bias is None else y + bias).to(dtype)


def _plain(s):
    case = s["case"]
    op, rounding = case["op"], case["round"]
    if op == "dropout":
        return _plain_dropout(s["x"], case["p"], s["residual"])
    if op == "dropout_backward":
        return _plain_dropout(s["dy"], case["p"], None)
    if op == "quantize":
        out = {}
        if case["form"] != "columns":
            out["rows"], out["row_scale"] = _plain_quantize(s["x"], 1, rounding, STREAM)
        if case["form"] != "rows":
            q, out["column_scale"] = _plain_quantize(s["x"], 0, rounding, STREAM)
            out["columns"] = q.t().contiguous()
        return out
    if op == "product":
        return _plain_product(s["a"], s["a_scale"], s["b"], s["b_scale"], s["bias"], TYPES[case["type"]])
    if op == "linear":
        q, scale = _plain_quantize(s["x"], 1, rounding, STREAM)
        return _plain_product(q, scale, s["w"], s["w_scale"], s["bias"], TYPES[case["type"]])
    x, w, dy = s["x"], s["w"], s["dy"]
    dy_rows, dy_row_scale = _plain_quantize(dy, 1, rounding, STREAM)
    dy_cols, dy_col_scale = _plain_quantize(dy, 0, rounding, STREAM)
    w_cols, w_scale = _plain_quantize(w, 0, rounding, STREAM + 1)
    x_cols, x_scale = _plain_quantize(x, 0, rounding, STREAM + 2)
    out = {"dx": _plain_product(dy_rows, dy_row_scale, w_cols.t(), w_scale, None, x.dtype),
           "dw": _plain_product(dy_cols.t(), dy_col_scale, x_cols.t(), x_scale, None, torch.float32)}
    if case["bias"]:
        out["db"] = dy.float().sum(0)
    return out


# ---- the library's calls --------------------------------------------------------------------------

def _own(s):
    import paper_1610_02132_amd as q
    case = s["case"]
    op, M, N, K, dtype = case["op"], case["M"], case["N"], case["K"], TYPES[case["type"]]
    if "draws" not in s:   # what a program keeps: its draws' key, its result buffers, a workspace
        s["draws"] = q.Draws(seed=SEED, stream_id=STREAM, iteration=ITERATION)
        s["rounding"] = q.ROUND_STOCHASTIC if case["round"] == "stochastic" else q.ROUND_NEAREST
        new = lambda rows, cols, t=dtype: torch.empty(rows, cols, dtype=t, device="cuda")  # noqa: E731
        if op.startswith("dropout"):
            s["out"], need = new(M, K), 0
        elif op == "quantize":
            s["out"], need = {}, q.qsgd_quantize_workspace_bytes(M, K)
            if case["form"] != "columns":
                s["out"] |= {"rows": _padded(M, K), "row_scale": new(1, M, torch.float32)[0]}
            if case["form"] != "rows":
                s["out"] |= {"columns": _padded(K, M), "column_scale": new(1, K, torch.float32)[0]}
        elif op == "product":
            s["out"], need = new(M, N), q.qsgd_int_matmul_workspace_bytes(M, N, K)
        elif op == "linear":
            s["out"], need = new(M, N), q.qsgd_linear_forward_workspace_bytes(M, N, K)
        else:
            s["out"], need = {"dx": new(M, K), "dw": new(N, K, torch.float32)}, q.qsgd_linear_backward_workspace_bytes(M, N, K)
            if case["bias"]:
                s["out"]["db"] = new(1, N, torch.float32)[0]
        s["workspace"] = torch.empty(max(need, 16), dtype=torch.uint8, device="cuda")
    out, draws, ws = s["out"], s["draws"], s["workspace"]
    if op == "dropout":
        q.qsgd_dropout(draws, case["p"], s["x"], out, residual=s["residual"])
    elif op == "dropout_backward":
        q.qsgd_dropout_backward(draws, case["p"], s["dy"], out)
    elif op == "quantize":
        q.qsgd_quantize(draws, s["x"], workspace=ws, rounding=s["rounding"], **out)
    elif op == "product":
        q.qsgd_int_matmul(s["a"], s["a_scale"], s["b"], s["b_scale"], out, bias=s["bias"], workspace=ws)
    elif op == "linear":
        q.qsgd_linear_forward(draws, s["x"], s["w"], s["w_scale"], out, bias=s["bias"], workspace=ws, rounding=s["rounding"])
    else:
        q.qsgd_linear_backward(draws, s["x"], s["w"], s["dy"], workspace=ws, rounding=s["rounding"], **out)
    return out


def run(state):
    return _own(state) if own else _plain(state)


# ---- what a pass cannot do without ------------------------------------------------------------------

def work(case):
    op, M, N, K, size = case["op"], case["M"], case["N"], case["K"], SIZE[case["type"]]
    if op.startswith("dropout"):
        return {"bytes": M * K * size * (3 if case["residual"] else 2), "flops": 2 * M * K}
    if op == "quantize":
        rows, cols = case["form"] != "columns", case["form"] != "rows"
        return {"bytes": M * K * (size + rows + cols) + 4 * (M * rows + K * cols), "flops": 2 * M * K * (rows + cols)}
    bias = 4 * N if case["bias"] else 0
    if op == "product":
        return {"bytes": M * K + N * K + 4 * (M + N) + bias + M * N * size, "flops": 2 * M * N * K}
    if op == "linear":
        return {"bytes": M * K * size + N * K + 4 * N + bias + M * N * size, "flops": 2 * M * N * K}
    return {"bytes": (2 * M * K + N * K + M * N) * size + 4 * N * K + bias, "flops": 4 * M * N * K}


# ---- the definitions in 64 bits ---------------------------------------------------------------------

def _exact_draws(rows, cols, stream):
    """Philox-4x32-10 on the host, in unsigned 64-bit words."""
    blocks = -(-cols // 8)
    u, mask = np.uint64, np.uint64(0xFFFFFFFF)
    c = np.tile(np.arange(blocks, dtype=u), rows), np.repeat(np.arange(rows, dtype=u), blocks), u(stream), u(ITERATION)
    key = np.array([SEED & 0xFFFFFFFF, SEED >> 32], dtype=u)
    for _ in range(10):
        p, r = u(0xD2511F53) * c[0], u(0xCD9E8D57) * c[2]
        c = (r >> u(32)) ^ c[1] ^ key[0], r & mask, (p >> u(32)) ^ c[3] ^ key[1], p & mask
        key = (key + np.array([0x9E3779B9, 0xBB67AE85], dtype=u)) & mask
    words = np.empty((rows * blocks, 4), dtype="<u4")
    for i in range(4):
        words[:, i] = c[i]
    return words.view("<u2").reshape(rows, 8 * blocks)[:, :cols]


def _exact_quantize(x, axis, rounding, draws):
    """Levels (64 bits) and scales; the level's fp32 product is part of its definition, everything else is exact."""
    v = x.float().cpu().numpy()
    m = np.abs(v).max(axis=axis, keepdims=True)
    m[m < TINY] = 0
    inv = np.zeros_like(m)
    np.divide(np.float32(127), m, out=inv, where=m > 0)
    t = (v * inv).astype(np.float64)
    if rounding == "nearest":
        level = np.rint(t)
    else:
        a = np.abs(t)
        level = np.sign(t) * np.minimum(np.ceil(a - (draws + 0.5) / 65536), 127)
    return torch.from_numpy(level).cuda(), torch.from_numpy(m.astype(np.float64) / 127).squeeze(axis).cuda()


def exact(case, seed):
    s = prepare(case, seed)
    op, M, N, K, rounding = case["op"], case["M"], case["N"], case["K"], case["round"]
    d = torch.float64
    if op.startswith("dropout"):
        x = s["x"] if op == "dropout" else s["dy"]
        D = int(np.rint(np.float32(case["p"]) * np.float32(65536)))
        keep = torch.from_numpy(_exact_draws(M, K, STREAM) >= D).cuda()
        y = x.to(d) * keep * 65536 / (65536 - D)
        return y if s.get("residual") is None else y + s["residual"].to(d)
    if op == "quantize":   # the levels are whole numbers: None
        out = {}
        if case["form"] != "columns":
            out |= {"rows": None, "row_scale": s["x"].to(d).abs().amax(1) / 127}
        if case["form"] != "rows":
            out |= {"columns": None, "column_scale": s["x"].to(d).abs().amax(0) / 127}
        return out
    if op in ("product", "linear"):
        if op == "product":
            a, a_scale, b, b_scale = s["a"].to(d), s["a_scale"], s["b"].to(d), s["b_scale"]
        else:
            a, a_scale = _exact_quantize(s["x"], 1, rounding, _exact_draws(M, K, STREAM) if rounding == "stochastic" else None)
            b, b_scale = s["w"].to(d), s["w_scale"]
        y = torch.matmul(a * a_scale.to(d)[:, None], (b * b_scale.to(d)[:, None]).t().contiguous())
        return y if s["bias"] is None else y + s["bias"].to(d)
    x, w, dy = s["x"], s["w"], s["dy"]
    hd, hw, hx = (_exact_draws(M, N, STREAM), _exact_draws(N, K, STREAM + 1), _exact_draws(M, K, STREAM + 2)) if rounding == "stochastic" else (None,) * 3
    r, rs = _exact_quantize(dy, 1, rounding, hd)
    c, cs = _exact_quantize(dy, 0, rounding, hd)
    wq, ws = _exact_quantize(w, 0, rounding, hw)
    xq, xs = _exact_quantize(x, 0, rounding, hx)
    out = {"dx": torch.matmul(r * rs[:, None], wq * ws), "dw": torch.matmul((c * cs).t().contiguous(), xq * xs)}
    if case["bias"]:
        out["db"] = dy.to(d).sum(0)
    return out
