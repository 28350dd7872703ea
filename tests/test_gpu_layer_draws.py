"""Gradients behind a dropout, with draws that are named as the header says: the means over many steps are those of the formula."""
import numpy as np
import pytest
import torch

import layer_reference as R
import paper_1610_02132_amd as q

pytestmark = pytest.mark.gpu

M, N, K, RUNS = 48, 40, 32, 256


def variance(v, axis):
    """Of stochastic levels times their scale, at most: a quarter of a step squared."""
    return np.broadcast_to((np.abs(v).max(axis=axis, keepdims=True) / 127) ** 2 / 4, v.shape)


def spread(a, va, b, vb):
    """Variance of a sum of products of independent factors, over the first one's last axis."""
    return (a ** 2 + va) @ (b ** 2 + vb) - (a ** 2) @ (b ** 2)


def host(t):
    return R.host(t).astype(np.float64)


@pytest.mark.parametrize("p", [0.1, 0.5])
def test_gradients_behind_a_dropout_are_unbiased(p):
    """dx and dw of what qsgd_dropout_backward leaves, against dlin w and dlin^T x step by step: the mean of the differences is
    within six of its standard deviations.  (The draws' half step, 2^-17 of a level, is far below them.)"""
    peer = 2
    x, w, dy = R.values(M, K, torch.float32, 1), R.values(N, K, torch.float32, 2), R.values(M, N, torch.float32, 3)
    X, W = host(x), host(w)
    dlin, dx, dw = torch.empty(M, N, device="cuda"), torch.empty(M, K, device="cuda"), torch.empty(N, K, device="cuda")
    ws = torch.empty(q.qsgd_linear_backward_workspace_bytes(M, N, K), dtype=torch.uint8, device="cuda")
    off = {"dx": np.zeros((M, K)), "dw": np.zeros((N, K))}
    var = {"dx": np.zeros((M, K)), "dw": np.zeros((N, K))}
    for step in range(RUNS):
        q.qsgd_dropout_backward(q.Draws(seed=100, stream_id=peer, iteration=step), p, dy, dlin)
        q.qsgd_linear_backward(q.Draws(seed=200, stream_id=4 * peer, iteration=step), x, w, dlin, dx=dx, dw=dw, workspace=ws,
                               rounding=q.ROUND_STOCHASTIC)
        G = host(dlin)
        off["dx"] += host(dx) - G @ W
        off["dw"] += host(dw) - G.T @ X
        var["dx"] += spread(G, variance(G, 1), W, variance(W, 0))
        var["dw"] += spread(G.T, variance(G, 0).T, X, variance(X, 0))
    for k in off:
        # (1e-5 of a step's result for the roundings of scales and products)
        assert (np.abs(off[k]) <= 6 * np.sqrt(var[k]) + 1e-5 * RUNS * np.abs(host(dx if k == "dx" else dw)).max()).all(), k


def test_streams_of_the_gradients_wrap():
    """The last stream_ids: w and x draw under 0 and 1."""
    x, w, dy = R.values(9, 20, torch.bfloat16, 1), R.values(12, 20, torch.bfloat16, 2), R.values(9, 12, torch.bfloat16, 3)
    d = q.Draws(seed=6, stream_id=2 ** 32 - 1, iteration=3)
    dx, dw = torch.empty(9, 20, dtype=torch.bfloat16, device="cuda"), torch.empty(12, 20, device="cuda")
    ws = torch.empty(q.qsgd_linear_backward_workspace_bytes(9, 12, 20), dtype=torch.uint8, device="cuda")
    q.qsgd_linear_backward(d, x, w, dy, dx=dx, dw=dw, workspace=ws, rounding=q.ROUND_STOCHASTIC)
    h = lambda s, r, c: R.half_words(q.Draws(seed=6, stream_id=s, iteration=3), r, c)  # noqa: E731
    r, rs = R.quantize(dy, 1, 1, h(2 ** 32 - 1, 9, 12))
    c, cs = R.quantize(dy, 0, 1, h(2 ** 32 - 1, 9, 12))
    wq, wsc = R.quantize(w, 0, 1, h(0, 12, 20))
    xq, xs = R.quantize(x, 0, 1, h(1, 9, 20))
    R.check(dx, *R.product(r, rs, wq.T, wsc, torch.bfloat16, scale_roundings=2), "dx")
    R.check(dw, *R.product(c.T, cs, xq.T, xs, torch.float32, scale_roundings=2), "dw")
