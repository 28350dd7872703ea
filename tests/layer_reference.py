"""Plain forms of the operators of a layer in 8 bits, on the host in 64 bits (numpy), and the
tolerances that follow from how many roundings the library's results have."""
from __future__ import annotations

import numpy as np
import torch

U32 = 2.0 ** -24                                   # half a step of fp32, relative
HALF_STEP = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
# half of the smallest subnormal
LEAST = {torch.float32: 2.0 ** -150, torch.bfloat16: 2.0 ** -134, torch.float16: 2.0 ** -25}
TYPES = (torch.float32, torch.bfloat16, torch.float16)
TINY = 2.0 ** -119


def half_words(d, rows, cols):
    """Draws of a matrix: d has seed, stream_id, iteration and row_base."""
    blocks = -(-cols // 8)
    m = 0xFFFFFFFF
    r, b = np.meshgrid(np.arange(rows, dtype=np.uint64) + np.uint64(d.row_base), np.arange(blocks, dtype=np.uint64), indexing="ij")
    x = [b, r & np.uint64(m), np.full_like(b, d.stream_id & m), np.full_like(b, d.iteration & m)]
    k = [d.seed & m, (d.seed >> 32) & m]
    for _ in range(10):
        p, q = x[0] * np.uint64(0xD2511F53), x[2] * np.uint64(0xCD9E8D57)
        x = [(q >> np.uint64(32)) ^ x[1] ^ np.uint64(k[0]), q & np.uint64(m),
             (p >> np.uint64(32)) ^ x[3] ^ np.uint64(k[1]), p & np.uint64(m)]
        k = [(k[0] + 0x9E3779B9) & m, (k[1] + 0xBB67AE85) & m]
    halves = [w >> np.uint64(16 * i) & np.uint64(0xFFFF) for w in x for i in (0, 1)]
    return np.stack(halves, axis=-1).reshape(rows, 8 * blocks)[:, :cols].astype(np.int64)


def host(t):
    return t.detach().float().cpu().numpy()


def dropout(d, p, x, residual=None):
    """(result, tolerance) in 64 bits for y of x's type."""
    D = int(np.rint(np.float32(p).astype(np.float64) * 65536))
    keep = half_words(d, *x.shape) >= D
    v = host(x).astype(np.float64)
    drawn = np.where(keep, v, 0.0) * (65536.0 / (65536 - D) if D < 65536 else 0.0)
    y = drawn if residual is None else drawn + host(residual).astype(np.float64)
    # factor and product rounded in fp32, then the sum, then the type
    tol = U32 * (2 * np.abs(drawn) + np.abs(y)) * 1.01 + HALF_STEP[x.dtype] * np.abs(y) * 1.01 + LEAST[x.dtype]
    return y, tol


def quantize(x, axis, rounding, draws=None):
    """Levels (int64) and scales (64 bits) with one per row (axis 1) or column (axis 0).  The level's
    fp32 product is part of its definition."""
    v = host(x)
    if v.shape[axis] == 0:
        return np.zeros(v.shape, np.int64), np.zeros(v.shape[1 - axis])
    m = np.abs(v).max(axis=axis, keepdims=True)    # (NaN if there is one)
    bad, tiny = ~np.isfinite(m), m < TINY
    with np.errstate(all="ignore"):
        inv = np.where(bad | tiny, np.float32(0), np.float32(127) / m).astype(np.float32)
        t = (v * inv).astype(np.float32)
    t = np.where(inv > 0, t, np.float32(0)).astype(np.float64)
    if rounding == 0:
        level = np.rint(t)
    else:
        a = np.abs(t)
        up = (draws + 0.5) / 65536 < a - np.floor(a)
        level = np.sign(t) * np.minimum(np.floor(a) + up, 127)
    scale = np.where(bad, np.nan, np.where(tiny, 0.0, m.astype(np.float64) / 127))
    return level.astype(np.int64), scale.reshape(-1)


def product(a, a_scale, b, b_scale, dtype, bias=None, scale_roundings=0):
    """(result, tolerance): a and b whole numbers, the scales in 64 bits (rounded to fp32 by the library
    `scale_roundings` times in all)."""
    y = (a.astype(np.float64) @ b.astype(np.float64).T) * a_scale[:, None] * b_scale[None, :]
    # the sum to fp32, two products
    tol = U32 * (3 + scale_roundings) * np.abs(y) * 1.01
    if bias is not None:
        y = y + bias.astype(np.float64)
        tol = tol + U32 * np.abs(y) * 1.01
    # ... and the type's rounding, of a value that may already be off by so much
    return y, tol + HALF_STEP[dtype] * (np.abs(y) + tol) + LEAST[dtype]


def check(got, want, tol, what=""):
    g = host(got).astype(np.float64) if torch.is_tensor(got) else got
    assert g.shape == want.shape, (what, g.shape, want.shape)
    nan = np.isnan(want)
    assert np.array_equal(np.isnan(g), nan), f"{what}: NaN in other places"
    off = np.abs(g - want)[~nan]
    over = off > tol[~nan]
    assert not over.any(), f"{what}: {int(over.sum())} of {g.size} off, by up to {(off / np.maximum(tol[~nan], 1e-300)).max():.3g} tolerances"


# ---- device matrices ---------------------------------------------------------------

def framed(rows, cols, dtype, ld=None, start=0, fill=None, device="cuda"):
    """(whole buffer, the matrix inside it): rows `ld` elements apart, `start` elements in; the rest of the
    buffer holds `fill`."""
    ld = cols if ld is None else ld
    buf = torch.empty(start + max(rows, 1) * ld + 64, dtype=dtype, device=device)
    buf.fill_(fill if fill is not None else (77 if dtype == torch.int8 else 12345.0))
    return buf, buf.as_strided((rows, cols), (ld, 1), start)


def levels(rows, cols, ld=None, device="cuda"):
    """(buffer, view) for levels: rows at multiples of 16 bytes."""
    return framed(rows, cols, torch.int8, ld=max(16, (cols + 15) // 16 * 16) if ld is None else ld, device=device)


def outside_untouched(buf, view, fill=None):
    """The buffer's elements that the view does not cover still hold `fill`."""
    fill = fill if fill is not None else (77 if buf.dtype == torch.int8 else 12345.0)
    mask = torch.ones(buf.numel(), dtype=torch.bool, device=buf.device)
    mask.as_strided(view.shape, view.stride(), view.storage_offset()).fill_(False)
    want = torch.full((), fill, dtype=buf.dtype, device=buf.device)
    return bool((buf[mask] == want).all())


def values(rows, cols, dtype, seed, device="cuda", scale=1.0, ld=None, start=0):
    g = torch.Generator()
    g.manual_seed(seed)
    x = torch.randn(rows, cols, generator=g) * scale * torch.exp(0.7 * torch.randn(cols, generator=g))
    _, view = framed(rows, cols, dtype, ld=ld, start=start, device=device)
    view.copy_(x.to(dtype))
    return view
