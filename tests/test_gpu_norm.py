"""Layer norm, forward and backward, against the oracle in 64 bits.

Bounds.  U = 2^-24.  The mean of n values of magnitude up to M carries at most (log2-like, taken as 32) units of M, so a deviation is
off by 32 U M, in units of the row's spread s = 1 / rstd: d = 32 U M / s.  rstd is off by about d^2 + 32 U, h by
d + 64 U |h|, and results by that times their factors; a bf16 result is rounded once more, 2^-8 of its value.
"""
import numpy as np
import pytest

import oracle.f8 as of8

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


def _host(t):
    import torch
    torch.cuda.synchronize()
    return t.double().cpu().numpy()


def _draw(rng, T, D, dtype, mean=1.0):
    import torch
    x = rng.standard_normal((T, D)) * np.exp(rng.standard_normal((T, 1))) + mean * rng.standard_normal((T, 1))
    t = torch.from_numpy(x.astype(np.float32)).to(torch.bfloat16 if dtype == "bf16" else torch.float32)
    return t.double().numpy(), t.cuda()


def _check(x, w, b, dtype, eps, y, mean, rstd):
    ry, rm, rr = of8.layer_norm(x, w, b, eps)
    M = np.abs(x).max(1, keepdims=True)
    d = 32 * U * M * rr[:, None]
    h = np.abs((x - rm[:, None]) * rr[:, None])
    w1 = 1.0 if w is None else np.abs(w)
    tol = (d * (1 + h) + 64 * U * h) * w1 + 8 * U * np.abs(ry) + (2.0 ** -8 * np.abs(ry) if dtype == "bf16" else 0) + 2.0 ** -120
    if b is not None:
        tol = tol + 4 * U * np.abs(b)
    assert (np.abs(y - ry) <= tol).all(), float((np.abs(y - ry) / tol).max())
    assert (np.abs(mean - rm) <= 32 * U * M[:, 0]).all()
    assert (np.abs(rstd - rr) <= rr * (64 * U + d[:, 0])).all()


SHAPES = [(1, 1), (1, 7), (3, 64), (5, 127), (2, 128), (9, 512), (4, 520), (6, 1000), (3, 1024), (4, 1032), (7, 2048), (3, 2050), (5, 4096), (2, 4104), (3, 8192),
          (2, 8200), (2, 16384), (2, 16392), (1, 30001), (1021, 260), (700, 1000), (513, 4096), (3000, 96), (9000, 130), (8300, 8), (2500, 300), (130, 129), (129, 256), (33, 384)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,D", SHAPES)
def test_forward_and_backward(T, D, dtype):
    import torch
    import paper_2407_09453_amd as bsp
    rng = np.random.default_rng([T, D])
    x, xt = _draw(rng, T, D, dtype)
    dy, dyt = _draw(rng, T, D, dtype, 0.1)
    w, b = (rng.standard_normal(D) + 1).astype(np.float32), rng.standard_normal(D).astype(np.float32)
    wt, bt = torch.from_numpy(w).cuda(), torch.from_numpy(b).cuda()
    y, mean, rstd = bsp.layer_norm(xt, wt, bt)
    _check(x, w, b, dtype, 1e-5, _host(y), _host(mean), _host(rstd))
    dx, dw, db = bsp.layer_norm_grad(dyt, xt, mean, rstd, wt)
    rx, rw, rb = of8.layer_norm_grad(dy, x, w)
    _, rm, rr = of8.layer_norm(x)
    h, g = np.abs((x - rm[:, None]) * rr[:, None]), np.abs(dy * w)
    d = 32 * U * np.abs(x).max(1, keepdims=True) * rr[:, None]
    spread = g + g.mean(1, keepdims=True) + h * (g * h).mean(1, keepdims=True)
    tol = rr[:, None] * (64 * U + 4 * d * (1 + h)) * (spread + (g * h).mean(1, keepdims=True) + g.mean(1, keepdims=True)) + (2.0 ** -8 * np.abs(rx) if dtype == "bf16" else 0)
    assert (np.abs(_host(dx) - rx) <= tol + 2.0 ** -120).all(), float((np.abs(_host(dx) - rx) / tol).max())
    n = min(T, 520) + T // 512 + 8  # terms added one after the other, in a thread and over the partial sums
    tw = (n * U + 64 * U) * (np.abs(dy) * h).sum(0) + (np.abs(dy) * d * (1 + h)).sum(0)
    assert (np.abs(_host(dw) - rw) <= tw + 2.0 ** -120).all()
    assert (np.abs(_host(db) - rb) <= n * U * np.abs(dy).sum(0) + 2.0 ** -120).all()


@pytest.mark.parametrize("code", ["e4m3", "e5m2"])
@pytest.mark.parametrize("T,D", [(1, 1), (1, 4096), (17, 1000), (5, 129), (40, 2048), (3, 8192), (2, 17000), (300, 520)])
def test_forward_to_codes(T, D, code):
    """The codes of the fp32 result: each within a rounding of the oracle's, and equal to those of the kernel's own fp32 result."""
    import torch
    import paper_2407_09453_amd as bsp
    rng = np.random.default_rng([T, D, 3])
    x, xt = _draw(rng, T, D, "f32")
    w, b = torch.from_numpy((rng.standard_normal(D) + 1).astype(np.float32)).cuda(), torch.from_numpy(rng.standard_normal(D).astype(np.float32)).cuda()
    y, mean, rstd = bsp.layer_norm(xt, w, b)
    c, mean2, rstd2 = bsp.layer_norm(xt, w, b, code=code)
    assert torch.equal(mean, mean2) and torch.equal(rstd, rstd2)
    direct = bsp.save8(y, code)
    torch.cuda.synchronize()
    assert torch.equal(c.codes, direct.codes) and torch.equal(c.scale[:, :T], direct.scale[:, :T])
    layer = bsp.BspLayerF8(rng.standard_normal((130, D)).astype(np.float32) / np.sqrt(D))
    assert torch.equal(layer.fc(c), layer.fc(direct))


def test_no_weight_no_bias_and_eps():
    import paper_2407_09453_amd as bsp
    x, xt = _draw(np.random.default_rng(5), 9, 300, "f32")
    for eps in (0.0, 1e-3):
        y, mean, rstd = bsp.layer_norm(xt, eps=eps)
        _check(x, None, None, "f32", eps, _host(y), _host(mean), _host(rstd))
    dx, _, db = bsp.layer_norm_grad(xt, xt, mean, rstd)
    rx, _, _ = of8.layer_norm_grad(x, x, eps=1e-3)
    assert np.abs(_host(dx) - rx).max() <= 2e-5 * np.abs(x).max() * _host(rstd).max()


def test_constant_and_offset_rows():
    """A row without spread gives the bias; one whose mean is a thousand times its spread keeps its digits."""
    import torch
    import paper_2407_09453_amd as bsp
    x = np.random.default_rng(6).standard_normal((3, 2048)) + 1000.0
    x[0] = 3.0
    xt = torch.from_numpy(x.astype(np.float32)).cuda()
    y, mean, rstd = bsp.layer_norm(xt)
    x = _host(xt)
    assert (_host(y)[0] == 0).all()
    _check(x[1:], None, None, "f32", 1e-5, _host(y)[1:], _host(mean)[1:], _host(rstd)[1:])


def test_rare_values_stay_in_their_row():
    import torch
    import paper_2407_09453_amd as bsp
    x, xt = _draw(np.random.default_rng(7), 6, 1000, "bf16")
    clean, _, _ = bsp.layer_norm(xt)
    xt[2, 5], xt[4, 999] = float("nan"), float("inf")
    y, mean, rstd = bsp.layer_norm(xt)
    y, clean = _host(y), _host(clean)
    assert np.isnan(y[[2, 4]]).all() and (y[[0, 1, 3, 5]] == clean[[0, 1, 3, 5]]).all()
    dx, _, _ = bsp.layer_norm_grad(xt, xt, mean, rstd)
    assert np.isfinite(_host(dx)[[0, 1, 3, 5]]).all()


def test_rows_anywhere_and_none():
    import torch
    import paper_2407_09453_amd as bsp
    base = torch.randn(70, 1111, device="cuda")
    w = torch.randn(700, device="cuda")
    for X in (base[:, :700], base[::3, 11:711], base.to(torch.bfloat16)[:, 3:703], base[:1, :700].expand(50, 700)):
        X2 = X.contiguous()
        y, mean, rstd = bsp.layer_norm(X, w)
        y2, mean2, rstd2 = bsp.layer_norm(X2, w)
        x = _host(X)
        _check(x, w.double().cpu().numpy(), None, "bf16" if X.dtype == torch.bfloat16 else "f32", 1e-5, _host(y), _host(mean), _host(rstd))
        a = bsp.layer_norm_grad(X, X, mean, rstd, w)
        b = bsp.layer_norm_grad(X2, X2, mean, rstd, w)
        for p, q in zip(a, b):
            assert torch.equal(p, q)
    y, mean, rstd = bsp.layer_norm(torch.empty(0, 300, device="cuda"))
    dx, dw, db = bsp.layer_norm_grad(torch.empty(0, 300, device="cuda"), torch.empty(0, 300, device="cuda"), mean, rstd)
    torch.cuda.synchronize()
    assert y.shape == dx.shape == (0, 300) and not dw.any() and not db.any()
    dx, dw, db = bsp.layer_norm_grad(torch.empty(0, 20000, device="cuda"), torch.empty(0, 20000, device="cuda"), mean, rstd)
    assert not dw.any() and not db.any()


def test_same_bits_every_time():
    import torch
    import paper_2407_09453_amd as bsp
    _, xt = _draw(np.random.default_rng(8), 3000, 520, "bf16")
    y, mean, rstd = bsp.layer_norm(xt)
    a = bsp.layer_norm_grad(xt, xt, mean, rstd)
    for _ in range(3):
        b = bsp.layer_norm_grad(xt, xt, mean, rstd)
        assert all(torch.equal(p, q) for p, q in zip(a, b))
