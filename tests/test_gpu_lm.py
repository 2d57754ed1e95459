"""Norms, 8-bit layers with adapters and log probabilities strung together as a network is tuned and served.

Each operator's result is the oracle's on the GPU's own inputs to it.  Bounds, U = 2^-24: a code is at most half of its binade's step
from the value; a product of codes with a bf16 result may lose 2^-10 of its magnitudes' sum, and an adapter's part beside it 2^-16 (u as
two parts, sums in fp32); sums of n products in fp32 lose (n + 16) U of their magnitudes; a bf16 result is half a step off, 2^-8.
"""
import os
import sys

import numpy as np
import pytest

import oracle.f8 as of8
import oracle.lm as olm

pytestmark = pytest.mark.gpu
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
U = 2.0 ** -24


def _host(t):
    return t.double().cpu().numpy()


def _network(seed=0, vocabulary=1001, width=260, users=3, rank=5):
    import torch
    import tune_adapters
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    net = tune_adapters.Network(vocabulary, width, users, rank, gen)
    for A, B in net.master:
        B.copy_(torch.randn(B.shape, generator=gen, device="cuda") / rank ** 0.5)
        A.copy_(A.to(torch.bfloat16))
        B.copy_(B.to(torch.bfloat16))
    for w in net.w:
        w.copy_(1 + 0.2 * torch.randn(w.shape, generator=gen, device="cuda"))
    net.take()
    return net, gen


def _batch(net, gen, T, V):
    import torch
    import paper_2407_09453_amd as bsp
    tokens, wanted = torch.randint(0, V, (2, T), generator=gen, device="cuda")
    wanted[::5] = -1  # rows of a prompt: nothing is wanted of them
    which = torch.randint(-1, net.banks[0].N, (T,), generator=gen, device="cuda")
    return tokens, wanted, which, bsp.BspRequests(which, net.banks[0].N)


def test_the_example_runs():
    import tune_adapters
    net, means = tune_adapters.train(steps=3, rows=100, vocabulary=500, width=256, users=3, rank=4)
    assert np.isfinite(means).all()
    import torch
    import paper_2407_09453_amd as bsp
    logp, tokens = net.answer(torch.arange(3, device="cuda"), bsp.BspRequests(torch.arange(3), 3))
    assert torch.isfinite(logp).all() and ((tokens >= 0) & (tokens < 500)).all()


@pytest.mark.parametrize("T", [1, 7, 130])
def test_a_step_is_the_oracles(T, monkeypatch):
    import torch
    import paper_2407_09453_amd as bsp
    weights = []
    made = bsp.BspLayerF8.__init__
    monkeypatch.setattr(bsp.BspLayerF8, "__init__", lambda self, W, *a, **k: (weights.append(_host(W)), made(self, W, *a, **k))[1])
    V, D = 1001, 260
    net, gen = _network(T)
    tokens, wanted, which, requests = _batch(net, gen, T, V)
    logits, kept = net.forward(tokens, requests)
    n1, h0, r1, positive, n2, h1, r2 = kept
    logp, lse, entropy, _, _ = bsp.log_probs(logits, wanted)
    dlogp, dentropy = torch.randn(2, T, generator=gen, device="cuda").unbind(0)
    dlogits = bsp.log_probs_grad(logits, wanted, lse, entropy, dlogp, dentropy)
    dx, (dw1, dw2), (g1, g2) = net.backward(dlogits, kept, requests)
    dn2 = net.layers[1].grad_input(dlogits, adapters=net.banks[1], requests=requests)
    dh1, _ = bsp.rms_norm_grad(dn2, h1, r2, net.w[1])
    dy = dh1 * positive
    dn1 = net.layers[0].grad_input(dy, adapters=net.banks[0], requests=requests)
    y = net.layers[0].fc(n1, relu=True, adapters=net.banks[0], requests=requests)
    torch.cuda.synchronize()
    which, tok = which.cpu().numpy(), wanted.cpu().numpy()
    scale = np.full(net.banks[0].N, net.scale)
    AB = [[_host(m) for m in pair] for pair in net.master]
    full = [np.ones((-(-W.shape[0] // 128), -(-W.shape[1] // 128)), np.uint8) for W in weights]

    def codes_near(codes, want):
        v = _host(codes.load(torch.float32))
        step = np.ldexp(2.0 ** 5, np.repeat(of8.scales(want, "e4m3"), 128, 1)[:, :D])  # the largest binade's, 2^(8 - 3) scales; twice where the scale is on an edge
        assert (np.abs(v - want) <= step).all()
        return v

    def layer_near(got, k, x, xq, relu=False, transposed=False):
        A, B = AB[k] if not transposed else [np.swapaxes(m, 1, 2) for m in AB[k][::-1]]
        low = [olm.low_rank(v, a, b, scale, which)[1] for v, a, b in ((x, A, B), (np.abs(x), np.abs(A), np.abs(B)))]
        want = of8.fc(xq, weights[k], full[k], None, low[0], relu, coded=True, transposed=transposed)
        mag = of8.fc(np.abs(xq), np.abs(weights[k]), full[k], coded=True, transposed=transposed)
        assert (np.abs(_host(got) - want) <= 2.0 ** -8 * np.abs(want) + 2.0 ** -10 * mag + (2.0 ** -16 + (x.shape[1] + 64) * U) * low[1] + 2.0 ** -120).all()

    def sums_near(got, want, mag, n):
        assert (np.abs(_host(got) - want) <= (n + 16) * U * mag + 2.0 ** -120).all()
    H0 = _host(net.embedding[tokens])
    assert (_host(h0) == H0).all()
    v1 = codes_near(n1, olm.rms_norm(H0, _host(net.w[0]))[0])
    layer_near(y, 0, v1, v1, relu=True)
    assert (_host(h1) == _host((y.double() + h0.double()).to(torch.bfloat16))).all()
    v2 = codes_near(n2, olm.rms_norm(_host(h1), _host(net.w[1]))[0])
    layer_near(logits, 1, v2, v2)
    z = _host(logits)
    wlogp, wlse, wh, _, _ = olm.log_probs(z, tok)
    far = 2.0 ** -20 * (1 + np.abs(z).max(1))  # some sixteen steps of fp32 at the size of what goes into a row's sum
    assert (np.abs(_host(logp) - wlogp) <= far).all() and (np.abs(_host(lse) - wlse) <= far).all() and (np.abs(_host(entropy) - wh) <= 8 * far).all()
    wz = olm.log_probs_grad(z, tok, _host(dlogp), _host(dentropy))
    p = np.exp(z - wlse[:, None])
    spread = (np.abs(_host(dlogp)) + np.abs(_host(dentropy)) * (1 + wh))[:, None] * p * (1 + np.abs(z - wlse[:, None])) + np.abs(wz)
    assert (np.abs(_host(dlogits) - wz) <= 2.0 ** -8 * np.abs(wz) + 16 * far[:, None] * spread).all()
    dz = _host(dlogits)
    layer_near(dn2, 1, dz, of8.values(dz, "e5m2"), transposed=True)
    layer_near(dn1, 0, _host(dy), of8.values(_host(dy), "e5m2"), transposed=True)
    for k, got, d, v in ((1, g2, dz, v2), (0, g1, _host(dy), v1)):
        want, mag = olm.low_rank_grad(d, v, *AB[k], scale, which), olm.low_rank_grad(np.abs(d), np.abs(v), *map(np.abs, AB[k]), scale, which)
        for i in (0, 1):
            sums_near(got[i], want[i], mag[i], T + d.shape[1] + D)
    for got, dw, dn, h, w, dh in ((dh1, dw2, dn2, h1, net.w[1], None), (dx, dw1, dn1, h0, net.w[0], dh1)):
        want, ww = olm.rms_norm_grad(_host(dn), _host(h), _host(w), dh=None if dh is None else _host(dh))
        nhat, rstd = olm.rms_norm(_host(h))
        g = np.abs(_host(dn) * _host(w))
        mag = rstd[:, None] * (g + np.abs(nhat) * (g * np.abs(nhat)).mean(1, keepdims=True)) + (0 if dh is None else np.abs(_host(dh)))
        assert (np.abs(_host(got) - want) <= 2.0 ** -8 * np.abs(want) + (D + 32) * U * mag).all()
        sums_near(dw, ww, (np.abs(_host(dn)) * np.abs(nhat)).sum(0), T + D)


def test_the_heads_adapters_against_differences():
    """The loss in 64 bits as the head's adapters move, its inputs and the layer's own part held.  The gradient is of logits rounded to
    bf16, d = 2^-8 of the largest and 2^-10 of the product's magnitudes off: each p by a factor e^(2 d) at most; and rounded itself."""
    import torch
    import paper_2407_09453_amd as bsp
    V, T = 301, 40
    net, gen = _network(9, V, 128, 2, 4)
    tokens, wanted, which, requests = _batch(net, gen, T, V)
    logits, kept = net.forward(tokens, requests)
    n2 = kept[4]
    _, lse, entropy, _, _ = bsp.log_probs(logits, wanted)
    dlogp = torch.randn(T, generator=gen, device="cuda")
    dlogits = bsp.log_probs_grad(logits, wanted, lse, entropy, dlogp)
    grads = net.banks[1].grad(dlogits, n2, requests)
    x, dl, tok, which = _host(n2.load(torch.float32)), _host(dlogp), wanted.cpu().numpy(), which.cpu().numpy()
    AB, scale = [_host(m) for m in net.master[1]], np.full(2, net.scale)
    own = _host(net.layers[1].fc(n2, dtype=torch.float32))

    def loss(A, B):
        z = own + olm.low_rank(x, A, B, scale, which)[1]
        return (dl * olm.log_probs(z, tok)[0]).sum()
    z = own + olm.low_rank(x, *AB, scale, which)[1]
    off = 2.0 ** -8 * np.abs(z).max(1) + np.abs(_host(logits) - z).max(1)
    dz = olm.log_probs_grad(z, tok, dl)
    p = np.exp(z - olm.log_probs(z, tok)[1][:, None])
    err = np.abs(dl)[:, None] * (tok >= 0)[:, None] * p * np.expm1(2 * off)[:, None] + 2.0 ** -8 * np.abs(dz) * np.exp(2 * off)[:, None]
    rng = np.random.default_rng(1)
    for i in (0, 1):
        far = olm.low_rank_grad(err, np.abs(x), *map(np.abs, AB), scale, which)[i]
        got = _host(grads[i])
        for k in rng.integers(0, got.size, 12):
            d = [np.zeros(m.shape) for m in AB]
            d[i].ravel()[k] = 1e-5
            diff = (loss(*(m + e for m, e in zip(AB, d))) - loss(*(m - e for m, e in zip(AB, d)))) / 2e-5
            assert abs(got.ravel()[k] - diff) <= far.ravel()[k] + 1e-6 * (1 + abs(diff)), (i, k, got.ravel()[k], diff)


def test_served_and_tuned_from_graphs():
    """Two graphs of answers and one of a step's gradients, replayed in turn with other tokens and users between, each the eager call's bits."""
    import torch
    import paper_2407_09453_amd as bsp
    V = 1001
    net, gen = _network(4)
    sizes, held = (1, 9, 200), []

    def tuned(tokens, wanted, requests):
        logits, kept = net.forward(tokens, requests)
        _, lse, entropy, _, _ = bsp.log_probs(logits, wanted)
        d = torch.ones(len(tokens), device="cuda")
        dx, dw, g = net.backward(bsp.log_probs_grad(logits, wanted, lse, entropy, d, d, out=logits), kept, requests)
        return (dx, *dw, *g[0], *g[1])
    for T in sizes:
        tokens, wanted, _, requests = _batch(net, gen, T, V)
        call = (lambda t, w, r: tuned(t, w, r)) if T == 200 else (lambda t, w, r: net.answer(t, r, 5))
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            call(tokens, wanted, requests)
        torch.cuda.current_stream().wait_stream(side)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = call(tokens, wanted, requests)
        held.append((graph, tokens, wanted, requests, call, out))
    for turn in range(4):
        for graph, tokens, wanted, requests, call, out in held:
            T = len(tokens)
            t2, w2, which, fresh = _batch(net, gen, T, V)
            tokens.copy_(t2)
            wanted.copy_(w2)
            requests.update(which)
        if turn == 2:
            net.banks[1].set(0, net.master[1][0][1], net.master[1][1][1], 0.5)
        for graph, *_ in held:
            graph.replay()
        torch.cuda.synchronize()
        for graph, tokens, wanted, requests, call, out in held:
            for a, b in zip(call(tokens, wanted, requests), out):
                assert torch.equal(a, b) or (torch.isnan(a) == torch.isnan(b)).all() and torch.equal(a.nan_to_num(), b.nan_to_num())
