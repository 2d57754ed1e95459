"""Log probabilities, entropy, the likeliest tokens and the logits' gradient against the oracle in 64 bits.

Bounds.  U = 2^-24.  With d = (max - x) scale, an exponent carries three roundings, 3 U d, and e^-d that and 4 U more; joining chunks
multiplies by one more such factor.  A sum of them, up to 32 one after the other in a thread, then in pairs, then up to 64 chunks, carries
160 U: in all (6 d + 160) U of each term.  The log of the sum moves by that over the sum and 4 U of itself.  A bf16 gradient is rounded once
more, 2^-8 of its value.
"""
import numpy as np
import pytest

import oracle.lm as olm

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


def _host(t):
    import torch
    torch.cuda.synchronize()
    return t.double().cpu().numpy()


def _bounds(x, scale):
    """(of log S, of the entropy, of every log probability, d) for rows with a token left."""
    with np.errstate(invalid="ignore", over="ignore"):
        z = x * scale
        m = z.max(1, keepdims=True)
        d = m - z
        e = np.exp(-d)
        d = np.where(e == 0, 0.0, np.minimum(d, 1e4))
        S = e.sum(1)
        s_tol = (e * (6 * d + 160)).sum(1) * U
        q_tol = (e * d * (6 * d + 168)).sum(1) * U
        log = np.log(S)
        log_tol = s_tol / S + 4 * U * np.abs(log) + 2.0 ** -100
        q = (e * d).sum(1) / S
        h_tol = log_tol + q_tol / S + q * s_tol / S + 4 * U * (np.abs(log) + q)
        lp = np.where(np.isinf(z), 0.0, m - z) + log[:, None]
        return log_tol, h_tol, log_tol[:, None] + 4 * U * (np.abs(lp) + np.where(np.isinf(z), 0, m - z)), d


def _same(got, want, tol):
    """Within the bound where the value is finite, alike where it is not."""
    with np.errstate(invalid="ignore"):
        fine = np.where(np.isfinite(want), np.abs(got - want) <= tol, (got == want) | (np.isnan(got) & np.isnan(want)))
    assert fine.all(), (got[~fine][:4], want[~fine][:4], np.broadcast_to(tol, want.shape)[~fine][:4])


def _check(x, tokens, top, scale, out, sure=None):
    """Rows whose maximum is finite in bounds, the others exactly."""
    logp, lse, entropy, tl, ti = out
    rl, rs, rh, rt, ri = olm.log_probs(x, tokens, top, scale)
    log_tol, h_tol, lp_tol, _ = _bounds(x, scale)
    fin = np.isfinite(rs)
    log_tol, h_tol, lp_tol = (np.where(fin.reshape((-1,) + (1,) * (t.ndim - 1)), t, 0.0) for t in (log_tol, h_tol, lp_tol))
    token = np.clip(tokens, 0, x.shape[1] - 1)
    _same(_host(logp), rl, lp_tol[np.arange(len(x)), token])
    _same(_host(lse), rs, log_tol + 4 * U * np.abs(np.where(fin, rs, 0)) + 4 * U * np.abs(np.where(fin, (x * scale).max(1), 0)))
    _same(_host(entropy), rh, h_tol)
    if top:
        assert (_host(ti) == ri).all()
        _same(_host(tl), rt, np.take_along_axis(lp_tol, ri, 1))
    else:
        assert tl is None and ti is None


def _check_grad(x, tokens, dl, dh, scale, got, bf16):
    want = olm.log_probs_grad(x, tokens, dl, dh, scale)
    _, lse, h, _, _ = olm.log_probs(x, tokens, 0, scale)
    log_tol, h_tol, _, _ = _bounds(x, scale)
    with np.errstate(invalid="ignore", over="ignore"):
        z = np.where(np.isinf(x), 0.0, x * scale)
        lp = z - np.where(np.isfinite(lse), lse, 0.0)[:, None]
        p = np.where(np.isinf(x), 0.0, np.exp(lp))
        # the log of the sum as it was written, rounded to fp32, the difference, the exponential
        d = (log_tol + 4 * U * np.abs(np.where(np.isfinite(lse), lse, 0)))[:, None] + 4 * U * (np.abs(z) + np.abs(lp))
        al, ah = (np.zeros(len(x)) if v is None else np.abs(v) for v in (dl, dh))
        a = al[:, None] + ah[:, None] * (np.abs(lp) + np.abs(h)[:, None])
        tol = scale * (p * (d + 16 * U) * a + p * ah[:, None] * (d + h_tol[:, None]) + 4 * U * al[:, None] * (np.arange(x.shape[1]) == np.asarray(tokens)[:, None]))
    tol = np.where(np.isfinite(tol), tol, 0) + (2.0 ** -8 if bf16 else 4 * U) * np.abs(np.where(np.isfinite(want), want, 0)) + 2.0 ** -120
    _same(_host(got), want, tol)


def _logits(rng, T, V, dtype, spread=2.5):
    import torch
    z = rng.standard_normal((T, V)) * spread
    z[np.arange(T), rng.integers(0, V, T)] += 8
    return torch.from_numpy(z.astype(np.float32)).to(torch.bfloat16 if dtype == "bf16" else torch.float32).cuda()


SHAPES = [(1, 1, 1), (1, 2, 1), (3, 5, 5), (2, 7, 0), (4, 8, 8), (9, 63, 20), (5, 64, 64), (3, 100, 50), (7, 511, 5), (2, 513, 64), (260, 1000, 5), (4, 1000, 50), (3, 1025, 64), (600, 2047, 20),
          (2, 2049, 1), (700, 4090, 20), (3, 4097, 64), (600, 8192, 0), (550, 8200, 64), (520, 16385, 20), (513, 32768, 8), (513, 32769, 64), (1, 32768, 20), (1, 50001, 64),
          (2, 131072, 20), (1, 200003, 50), (5, 131073, 0), (90, 65536, 64), (2, 1 << 21, 64), (2100, 600, 33)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,V,top", SHAPES)
def test_forward_and_backward(T, V, top, dtype):
    import torch
    import paper_2407_09453_amd as bsp
    rng = np.random.default_rng([T, V])
    X = _logits(rng, T, V, dtype)
    tokens = rng.integers(0, V, T)
    tokens[T // 2] = -1 if T > 1 else tokens[0]
    scale = [1.0, 0.7, 1.25][(T + V) % 3]
    kind = torch.int64 if V % 2 else torch.int32
    tok = torch.from_numpy(tokens).to(kind).cuda()
    out = bsp.log_probs(X, tok, top, scale)
    x, f32scale = _host(X), float(np.float32(scale))
    keep = slice(0, T if T * V < 3e6 else 24)  # (the oracle's time)
    _check(x[keep], tokens[keep], top, f32scale, [None if t is None else t[keep] for t in out])
    dl, dh = (rng.standard_normal(T).astype(np.float32) for _ in range(2))
    dlt, dht = torch.from_numpy(dl).cuda(), torch.from_numpy(dh).cuda()
    g = bsp.log_probs_grad(X, tok, out[1], out[2], dlt, dht, scale)
    _check_grad(x[keep], tokens[keep], dl[keep], dh[keep], f32scale, g[keep], dtype == "bf16")
    again = bsp.log_probs_grad(X, tok, out[1], out[2], dlt, dht, scale, out=X)  # over the logits
    assert again is X and torch.equal(g, X)


@pytest.mark.parametrize("V", [40, 1000, 5000, 40000, 131072])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_masks_ties_and_rare_values(V, dtype):
    """Rows that masks leave little or nothing, rows of one value, of the type's lowest, runs of equal values, NaN and infinities."""
    import torch
    import paper_2407_09453_amd as bsp
    rng = np.random.default_rng(V)
    X = _logits(rng, 14, V, dtype)
    inf = float("inf")
    low = torch.finfo(X.dtype).min
    X[0] = -inf
    X[1, 1:] = -inf
    X[2] = 1.5
    X[3] = low
    X[4, : V // 2] = low
    X[5, torch.from_numpy(rng.random(V) < 0.9).cuda()] = -inf
    X[6] = torch.round(X[6])
    X[7, 7] = float("nan")
    X[8, V - 1] = inf
    X[9] = torch.arange(V, device="cuda").to(X.dtype) / V
    X[10] = -torch.arange(V, device="cuda").to(X.dtype) / V
    X[11, 3] = 40.0  # a sure token: what the others add is far below a bit of 1
    X[12] = 0.0
    X[12, ::2] = -0.0
    X[13] = inf
    tokens = rng.integers(0, V, 14)
    tokens[[1, 6]] = 0, V - 1
    tokens[11] = 3
    out = bsp.log_probs(X, torch.from_numpy(tokens).cuda(), 20)
    x = _host(X)
    rest = [0, 1, 2, 3, 4, 5, 6, 9, 10, 11, 12]
    _check(x[rest], tokens[rest], 20, 1.0, [t[rest] for t in out])
    for r in (7, 8, 13):  # not a number, but whose turn it is stays clear
        assert torch.isnan(out[1][r]) and torch.isnan(out[2][r]) and torch.isnan(out[0][r])
        assert (_host(out[4][r]) == olm.order(x[r:r + 1])[0, :20]).all()
    dl, dh = (rng.standard_normal(14).astype(np.float32) for _ in range(2))
    g = bsp.log_probs_grad(X, torch.from_numpy(tokens).cuda(), out[1], out[2], torch.from_numpy(dl).cuda(), torch.from_numpy(dh).cuda())
    _check_grad(x[rest], tokens[rest], dl[rest], dh[rest], 1.0, g[rest], dtype == "bf16")
    assert torch.isnan(g[7]).all()


def test_tokens_out_of_range():
    import torch
    import paper_2407_09453_amd as bsp
    X = torch.randn(5, 300, device="cuda")
    tokens = torch.tensor([299, 300, -1, -100, 1 << 40], device="cuda")
    logp, lse, entropy, _, _ = bsp.log_probs(X, tokens)
    one = torch.ones(5, device="cuda")
    g = bsp.log_probs_grad(X, tokens, lse, entropy, one, None)
    assert torch.isnan(logp).tolist() == [False, True, False, False, True] and logp[2] == 0 and logp[3] == 0
    assert not g[2:4].any() and torch.isnan(g[[1, 4]]).all() and torch.isfinite(g[0]).all()
    assert not bsp.log_probs_grad(X, tokens.clamp(-1, 299), lse, entropy).any()  # nothing comes in


def test_gradient_against_differences():
    import torch
    import paper_2407_09453_amd as bsp
    rng = np.random.default_rng(2)
    X = _logits(rng, 3, 77, "f32")
    tokens = np.array([5, -1, 76])
    dl, dh = (rng.standard_normal(3).astype(np.float32) for _ in range(2))
    tok = torch.from_numpy(tokens).cuda()
    _, lse, entropy, _, _ = bsp.log_probs(X, tok, scale=0.5)
    g = _host(bsp.log_probs_grad(X, tok, lse, entropy, torch.from_numpy(dl).cuda(), torch.from_numpy(dh).cuda(), scale=0.5))
    x = _host(X)

    def loss(x):
        lp, _, h, _, _ = olm.log_probs(x, tokens, 0, 0.5)
        return float((dl * lp + dh * h).sum())
    for at in ((0, 5), (0, 6), (1, 0), (2, 76), (2, int(x[2].argmax()))):
        d = np.zeros_like(x)
        d[at] = 1e-5
        assert abs((loss(x + d) - loss(x - d)) / 2e-5 - g[at]) <= 1e-6


def test_rows_anywhere_and_none():
    import torch
    import paper_2407_09453_amd as bsp
    base = torch.randn(60, 1111, device="cuda")
    tok = torch.arange(60, device="cuda", dtype=torch.int32)
    d = torch.randn(60, device="cuda")
    for X in (base[:, :700], base[::3, 11:711], base.to(torch.bfloat16)[:, 3:703], base[:1, :700].expand(50, 700)):
        n = len(X)
        a, b = bsp.log_probs(X, tok[:n], 5), bsp.log_probs(X.contiguous(), tok[:n], 5)
        assert all(torch.equal(p, q) for p, q in zip(a, b))
        guard = torch.full((n, 720), 7.0, device="cuda", dtype=X.dtype)
        out = bsp.log_probs_grad(X, tok[:n], a[1], a[2], d[:n], d[:n], out=guard[:, 9:709])
        assert torch.equal(out, bsp.log_probs_grad(X.contiguous(), tok[:n], a[1], a[2], d[:n], d[:n]))
        assert (guard[:, :9] == 7).all() and (guard[:, 709:] == 7).all()
    none = torch.empty(0, 300, device="cuda")
    out = bsp.log_probs(none, tok[:0], 3)
    assert out[0].shape == (0,) and out[3].shape == (0, 3) and bsp.log_probs_grad(none, tok[:0], out[1], out[2]).shape == (0, 300)


def test_offsets_past_32_bits():
    """Rows whose elements lie past 2^32: the last row's results are those of the row by itself."""
    import torch
    import paper_2407_09453_amd as bsp
    T, V = 33000, 131072
    X = torch.empty(T, V, device="cuda", dtype=torch.bfloat16)
    for a in range(0, T, 3000):
        X[a:a + 3000].normal_(0, 2)
    tok = torch.randint(0, V, (T,), device="cuda")
    out = bsp.log_probs(X, tok, 7)
    last = slice(T - 300, T)
    d = torch.randn(T, device="cuda")
    alone = bsp.log_probs(X[last].clone(), tok[last], 7)
    for a, b in zip(out, alone):
        if a.dtype == torch.int32:
            assert torch.equal(a[last], b)
        else:
            assert torch.allclose(a[last], b, rtol=0, atol=3e-5)  # (other chunks: the sums' order)
    want = bsp.log_probs_grad(X[last].clone(), tok[last], out[1][last].clone(), out[2][last].clone(), d[last].clone(), None)
    bsp.log_probs_grad(X, tok, out[1], out[2], d, None, out=X)
    assert torch.equal(X[last], want)


def test_same_bits_every_time_and_in_a_graph():
    import torch
    import paper_2407_09453_amd as bsp
    X = torch.randn(6, 70000, device="cuda").to(torch.bfloat16)  # (many equal values, in chunks)
    tok, d = torch.arange(6, device="cuda"), torch.randn(6, device="cuda")

    def both():
        out = bsp.log_probs(X, tok, 30)
        return (*out, bsp.log_probs_grad(X, tok, out[1], out[2], d, d))
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
        X.copy_(torch.randn(6, 70000, device="cuda"))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(both(), got)), k


def test_on_a_stream_of_the_caller_and_autograd_is_told():
    import torch
    import paper_2407_09453_amd as bsp
    X, tok = torch.randn(500, 3000, device="cuda"), torch.arange(500, device="cuda")
    want = bsp.log_probs(X, tok, 4)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = bsp.log_probs(X, tok, 4, stream=side.cuda_stream)
    g = bsp.log_probs_grad(X, tok, got[1], got[2], got[0], stream=side.cuda_stream)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(p, q) for p, q in zip(want, got))
    assert torch.equal(g, bsp.log_probs_grad(X, tok, want[1], want[2], want[0]))
    with pytest.warns(UserWarning, match="records nothing"):
        bsp.log_probs(X.clone().requires_grad_(), tok)
