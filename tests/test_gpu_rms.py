"""Root-mean-square norm with the residual's addition, forward and backward, against the oracle in 64 bits.

Bounds.  U = 2^-24.  h is one fp32 addition rounded to its type: exact.  A sum of D squares, up to 160 of them one after the other in a thread
and the rest in pairs, carries at most 192 U of itself, rstd half of that and 4 U, so y carries 128 U.  The gradient's sum carries
192 U of its terms' magnitudes; a bf16 result is rounded once more, 2^-8 of its value.
"""
import numpy as np
import pytest

import oracle.lm as olm

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
TINY = 2.0 ** -120


def _host(t):
    import torch
    torch.cuda.synchronize()
    return t.double().cpu().numpy()


def _draw(rng, T, D, dtype):
    import torch
    x = rng.standard_normal((T, D)) * np.exp(rng.standard_normal((T, 1)))
    return torch.from_numpy(x.astype(np.float32)).to(torch.bfloat16 if dtype == "bf16" else torch.float32).cuda()


def _check_forward(y, rstd, h, w, dtype, eps=1e-6):
    ry, rr = olm.rms_norm(h, w, eps)
    assert (np.abs(rstd - rr) <= 128 * U * rr).all()
    tol = (128 * U + (2.0 ** -8 if dtype == "bf16" else 0)) * np.abs(ry) + TINY
    assert (np.abs(y - ry) <= tol).all(), float((np.abs(y - ry) / tol).max())


def _check_backward(dx, dw, dy, h, w, dh, dtype):
    rx, rw = olm.rms_norm_grad(dy, h, w, dh=dh)
    n, rr = olm.rms_norm(h)
    g = np.abs(dy if w is None else dy * w)
    spread = rr[:, None] * (g + np.abs(n) * (g * np.abs(n)).mean(1, keepdims=True))
    tol = 512 * U * spread + (0 if dh is None else 4 * U * np.abs(dh)) + (2.0 ** -8 if dtype == "bf16" else 0) * np.abs(rx) + TINY
    assert (np.abs(dx - rx) <= tol).all(), float((np.abs(dx - rx) / tol).max())
    terms = min(len(dy), 520) + len(dy) // 512 + 8  # added one after the other, in a thread and over the partial sums
    assert (np.abs(dw - rw) <= (terms + 160) * U * np.abs(dy * n).sum(0) + TINY).all()


SHAPES = [(1, 1), (1, 7), (3, 64), (5, 127), (2, 128), (9, 512), (4, 520), (6, 1000), (3, 1024), (4, 1032), (7, 2048), (3, 2050), (5, 4096), (2, 4104), (3, 8192),
          (2, 8200), (2, 16384), (2, 16392), (1, 30001), (1021, 260), (700, 1000), (513, 4096), (3000, 96), (9000, 130), (2500, 300), (33, 384)]


@pytest.mark.parametrize("residual", [True, False])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,D", SHAPES)
def test_forward_and_backward(T, D, dtype, residual):
    import torch
    import paper_2407_09453_amd as bsp
    rng = np.random.default_rng([T, D, residual])
    x, r, dy, dh = (_draw(rng, T, D, dtype) for _ in range(4))
    w = (rng.standard_normal(D) + 1).astype(np.float32)
    wt = torch.from_numpy(w).cuda()
    y, h, rstd = bsp.rms_norm(x, wt, r if residual else None)
    if residual:
        assert torch.equal(h, (x.float() + r.float()).to(x.dtype))
    else:
        assert h is x
    _check_forward(_host(y), _host(rstd), _host(h), w, dtype)
    dx, dw = bsp.rms_norm_grad(dy, h, rstd, wt, dH=dh if residual else None)
    _check_backward(_host(dx), _host(dw), _host(dy), _host(h), w, _host(dh) if residual else None, dtype)


@pytest.mark.parametrize("code", ["e4m3", "e5m2"])
@pytest.mark.parametrize("T,D", [(1, 1), (1, 4096), (17, 1000), (5, 129), (40, 2048), (3, 8192), (2, 17000), (300, 520)])
def test_forward_to_codes(T, D, code):
    """The codes of the fp32 result, as a checkpoint of the kernel's own fp32 result has them; and a layer that reads them."""
    import torch
    import paper_2407_09453_amd as bsp
    rng = np.random.default_rng([T, D, 3])
    x, r = _draw(rng, T, D, "f32"), _draw(rng, T, D, "f32")
    w = torch.from_numpy((rng.standard_normal(D) + 1).astype(np.float32)).cuda()
    y, h, rstd = bsp.rms_norm(x, w, r)
    c, h2, rstd2 = bsp.rms_norm(x, w, r, code=code)
    direct = bsp.save8(y, code)
    torch.cuda.synchronize()
    assert torch.equal(h, h2) and torch.equal(rstd, rstd2) and torch.equal(c.codes, direct.codes) and torch.equal(c.scale[:, :T], direct.scale[:, :T])
    layer = bsp.BspLayerF8(rng.standard_normal((130, D)).astype(np.float32) / np.sqrt(D))
    assert torch.equal(layer.fc(c), layer.fc(direct))


def test_gradient_against_differences():
    """The loss sum(dy y) + sum(dh h), moved by small steps of x in 64 bits, and the kernel's gradient of it."""
    import torch
    import paper_2407_09453_amd as bsp
    rng = np.random.default_rng(11)
    x, dy, dh = (_draw(rng, 3, 300, "f32") for _ in range(3))
    w = (rng.standard_normal(300) + 1).astype(np.float32)
    _, h, rstd = bsp.rms_norm(x, torch.from_numpy(w).cuda())
    dx = _host(bsp.rms_norm_grad(dy, h, rstd, torch.from_numpy(w).cuda(), dH=dh)[0])
    x, dy, dh = _host(x), _host(dy), _host(dh)
    loss = lambda x: float((dy * olm.rms_norm(x, w)[0]).sum() + (dh * x).sum())  # noqa: E731
    step = 1e-5
    for at in ((0, 0), (0, 299), (1, 7), (2, 255), (2, 256)):
        d = np.zeros_like(x)
        d[at] = step
        num = (loss(x + d) - loss(x - d)) / (2 * step)
        # (second differences leave step^2 of the third derivative, rounding 2^-52 of the loss over a step)
        assert abs(num - dx[at]) <= 1e-5 * (1 + np.abs(dx).max())


def test_no_weight_eps_zero_rows_and_rare_values():
    import torch
    import paper_2407_09453_amd as bsp
    x = _draw(np.random.default_rng(5), 7, 1000, "bf16")
    x[3] = 0
    for eps in (1e-6, 1e-2):
        y, _, rstd = bsp.rms_norm(x, eps=eps)
        _check_forward(_host(y), _host(rstd), _host(x), None, "bf16", eps)
    dx, dw = bsp.rms_norm_grad(x, x, rstd)
    assert (_host(dx)[3] == 0).all()
    clean, dirty = _host(y), x.clone()
    dirty[2, 5], dirty[4, 999] = float("nan"), float("inf")
    y, _, rstd = bsp.rms_norm(dirty, eps=1e-2)
    y, dx = _host(y), _host(bsp.rms_norm_grad(x, dirty, rstd)[0])
    rest = [0, 1, 3, 5, 6]
    assert np.isnan(y[2]).all() and np.isnan(y[4, 999]) and (y[rest] == clean[rest]).all() and np.isfinite(dx[rest]).all()


def test_rows_anywhere_and_none():
    import torch
    import paper_2407_09453_amd as bsp
    base = torch.randn(70, 1111, device="cuda")
    w = torch.randn(700, device="cuda")
    for X in (base[:, :700], base[::3, 11:711], base.to(torch.bfloat16)[:, 3:703], base[:1, :700].expand(50, 700)):
        X2 = X.contiguous()
        a, b = bsp.rms_norm(X, w, X), bsp.rms_norm(X2, w, X2)
        assert all(torch.equal(p, q) for p, q in zip(a, b))
        a, b = bsp.rms_norm_grad(X, X, a[2], w, dH=X), bsp.rms_norm_grad(X2, X2, b[2], w, dH=X2)
        assert all(torch.equal(p, q) for p, q in zip(a, b))
    for D in (300, 20000):
        none = torch.empty(0, D, device="cuda")
        y, h, rstd = bsp.rms_norm(none, residual=none)
        dx, dw = bsp.rms_norm_grad(none, h, rstd)
        assert y.shape == h.shape == dx.shape == (0, D) and not dw.any()
    wide = torch.randn(4, 1000, device="cuda", dtype=torch.bfloat16)
    guard = torch.full((4, 1000 + 24), 7.0, device="cuda", dtype=torch.bfloat16)  # rows behind and columns past are left as they were
    lib, out = bsp.load_library(), guard[:, 8:1008]
    rstd = torch.empty(4, device="cuda")
    assert lib.bsp_rms_norm(wide.data_ptr(), 1000, None, 0, 1, 3, 1000, None, 1e-6, None, 0, out.data_ptr(), 1024, None, rstd.data_ptr(),
                            torch.cuda.current_stream().cuda_stream) == 0
    y, _, _ = bsp.rms_norm(wide)
    torch.cuda.synchronize()
    assert torch.equal(out[:3], y[:3]) and (guard[3] == 7).all() and (guard[:, :8] == 7).all() and (guard[:, 1008:] == 7).all()


def test_same_bits_every_time_and_in_a_graph():
    import torch
    import paper_2407_09453_amd as bsp
    x, r, dy = (_draw(np.random.default_rng(8 + k), 3000, 520, "bf16") for k in range(3))
    w = torch.randn(520, device="cuda")

    def both():
        y, h, rstd = bsp.rms_norm(x, w, r)
        return (y, h, rstd, *bsp.rms_norm_grad(dy, h, rstd, w, dH=dy))
    want = both()
    for _ in range(2):
        assert all(torch.equal(p, q) for p, q in zip(want, both()))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        both()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = both()
    for k in range(4):
        x.copy_(torch.randn_like(x, dtype=torch.float32))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(both(), got)), k


def test_on_a_stream_of_the_caller():
    import torch
    import paper_2407_09453_amd as bsp
    x, r = _draw(np.random.default_rng(3), 2000, 1000, "bf16"), _draw(np.random.default_rng(4), 2000, 1000, "bf16")
    want = bsp.rms_norm(x, None, r)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    y, h, rstd = bsp.rms_norm(x, None, r, stream=side.cuda_stream)
    dx, dw = bsp.rms_norm_grad(x, h, rstd, stream=side.cuda_stream)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(p, q) for p, q in zip((y, h, rstd), want))
    assert all(torch.equal(p, q) for p, q in zip((dx, dw), bsp.rms_norm_grad(x, want[1], want[2])))
    same, h, _ = bsp.rms_norm(x, stream=side.cuda_stream)
    assert h is x


def test_autograd_is_told():
    import torch
    import paper_2407_09453_amd as bsp
    x = torch.randn(4, 64, device="cuda", requires_grad=True)
    with pytest.warns(UserWarning, match="records nothing"):
        bsp.rms_norm(x)


@pytest.mark.parametrize("D", [700, 20000])
def test_offsets_past_32_bits(D):
    """Rows 2^30 elements apart."""
    import torch
    import paper_2407_09453_amd as bsp
    held = torch.empty(3 * 2 ** 30 + D, dtype=torch.bfloat16, device="cuda")
    far = held.as_strided((4, D), (2 ** 30, 1))
    X = torch.randn(4, D, device="cuda").to(torch.bfloat16)
    far.copy_(X)
    assert all(torch.equal(p, q) for p, q in zip(bsp.rms_norm(far, residual=far), bsp.rms_norm(X, residual=X)))
    _, h, rstd = bsp.rms_norm(X)
    assert all(torch.equal(p, q) for p, q in zip(bsp.rms_norm_grad(far, far, rstd, dH=far), bsp.rms_norm_grad(X, h, rstd, dH=X)))
    out, r = torch.zeros_like(X), torch.empty(4, device="cuda")
    assert bsp.load_library().bsp_rms_norm(X.data_ptr(), D, None, 0, 1, 4, D, None, 1e-6, None, 0, far.data_ptr(), 2 ** 30, None, r.data_ptr(), torch.cuda.current_stream().cuda_stream) == 0
    out.copy_(far)
    assert torch.equal(out, bsp.rms_norm(X)[0])
