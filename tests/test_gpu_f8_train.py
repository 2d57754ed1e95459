"""The example's training step: it learns, and its pieces are the oracle's on the values that it passes from one to the next."""
import os
import sys

import numpy as np
import pytest

import oracle.f8 as of8

pytestmark = pytest.mark.gpu
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


def _host(t):
    return t.double().cpu().numpy()


def test_it_learns():
    import train_f8
    _, losses = train_f8.train()
    assert np.isfinite(losses).all() and losses[-1] < 0.5 * losses[0], losses


def test_a_step_is_the_oracles():
    """Each operator's result against the oracle's on the GPU's own inputs to it, as the training step strings them together."""
    import torch
    import paper_2407_09453_amd as bsp
    import train_f8
    gen = torch.Generator(device="cuda")
    gen.manual_seed(3)
    block = train_f8.Block(256, 384, gen)
    x = torch.randn(70, 256, generator=gen, device="cuda").to(torch.bfloat16)
    y, (_, mean, rstd, n, h) = block.forward(x)
    dy = torch.randn(70, 256, generator=gen, device="cuda").to(torch.bfloat16)
    dx, g = block.backward(dy, (x, mean, rstd, n, h))
    m = {k: _host(v) for k, v in block.master.items()}
    g1, g2 = block.fc1.gamma, block.fc2.gamma
    nv, hv = _host(n.load(torch.float32)), _host(h.load(torch.float32))
    U = 2.0 ** -24

    def near(got, want, S, terms, bf16=True):  # a rounding to bf16 and what the products of codes lose; or fp32 sums of so many terms
        tol = 2.0 ** -8 * np.abs(want) + 2.0 ** -10 * S if bf16 else (terms + 8) * U * S
        assert (np.abs(_host(got) - want) <= tol).all()
    yn, _, _ = of8.layer_norm(_host(x), m["w"], m["b"])
    e = of8.scales(yn, "e4m3")
    step = np.ldexp(2.0 ** 5, np.repeat(e, 128, 1)[:, :256])  # a code is at most half of its largest step from the value
    assert (np.abs(nv - yn) <= 0.5 * step + 1e-5).all()
    h_ref = of8.fc(nv, m["W1"], g1, m["b1"], relu=True, coded=True)
    S = of8.fc(np.abs(nv), np.abs(m["W1"]), g1, np.abs(m["b1"]), coded=True)
    # what is kept is the code of a bf16 result: two roundings, the second of three bits after the leading one
    assert (np.abs(hv - h_ref) <= 2.0 ** -3 * np.abs(h_ref) + 2.0 ** -9 * S + 2.0 ** -9 * np.ldexp(1.0, np.repeat(of8.scales(hv, "e4m3"), 128, 1)[:, :384])).all()
    near(y, of8.fc(hv, m["W2"], g2, m["b2"], residual=_host(x), coded=True), of8.fc(np.abs(hv), np.abs(m["W2"]), g2, np.abs(m["b2"]), residual=np.abs(_host(x)), coded=True), 0)
    dW2, db2 = of8.grad_weight(_host(dy), hv, g2)
    S2, Sb2 = of8.grad_weight(np.abs(_host(dy)), np.abs(hv), g2)
    near(g["W2"], dW2, S2, 70, bf16=False)
    near(g["b2"], db2, Sb2, 70, bf16=False)
    dh = block.fc2.grad_input(dy, relu_of=h)
    near(dh, of8.fc(_host(dy), m["W2"], g2, code="e5m2", transposed=True, gate=hv), of8.fc(np.abs(_host(dy)), np.abs(m["W2"]), g2, code="e5m2", transposed=True), 0)
    dW1, _ = of8.grad_weight(_host(dh), nv, g1)
    near(g["W1"], dW1, of8.grad_weight(np.abs(_host(dh)), np.abs(nv), g1)[0], 70, bf16=False)
    assert (_host(g["W1"])[~of8.mask(g1, 384, 256)] == 0).all() and (_host(g["W2"])[~of8.mask(g2, 256, 384)] == 0).all()
    dn = block.fc1.grad_input(dh)
    rx, rw, rb = of8.layer_norm_grad(_host(dn), _host(x), m["w"])
    assert np.abs(_host(dx) - (rx + _host(dy))).max() <= 2.0 ** -7 * np.abs(rx + _host(dy)).max() + 2.0 ** -7 * np.abs(rx).max()
    near(g["w"], rw, (np.abs(_host(dn)) * np.abs((_host(x) - _host(mean)[:, None]) * _host(rstd)[:, None])).sum(0) + 1e-3, 70 + 120, bf16=False)
    near(g["b"], rb, np.abs(_host(dn)).sum(0), 70, bf16=False)


def test_a_row_served_is_the_batchs():
    """One row through the block as a batch's: the same codes, sums in another order."""
    import torch
    import train_f8
    gen = torch.Generator(device="cuda")
    gen.manual_seed(4)
    block = train_f8.Block(256, 256, gen)
    x = torch.randn(130, 256, generator=gen, device="cuda").to(torch.bfloat16)
    import paper_2407_09453_amd as bsp
    n, _, _ = bsp.layer_norm(x, block.master["w"], block.master["b"], code="e4m3")
    batch, few = _host(block.fc1.fc(n)), []
    for r in (0, 64, 129):
        one, _, _ = bsp.layer_norm(x[r:r + 1], block.master["w"], block.master["b"], code="e4m3")
        assert torch.equal(one.codes[0], n.codes[r]) and torch.equal(one.scale[:, 0], n.scale[:, r])
        few.append(_host(block.fc1.fc(one))[0])
    S = of8.fc(np.abs(_host(n.load(torch.float32))), np.abs(_host(block.master["W1"])), block.fc1.gamma, coded=True)[[0, 64, 129]]
    assert (np.abs(batch[[0, 64, 129]] - np.array(few)) <= 2.0 ** -7 * np.abs(batch[[0, 64, 129]]) + 2.0 ** -9 * S).all()
