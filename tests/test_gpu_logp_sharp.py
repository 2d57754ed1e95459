"""Log probabilities at sharp and dull temperatures and of logits of any size, against the oracle in 64 bits.

Bounds.  U = 2^-24; d = (max - x) scale.  An exponent carries the rounding of a difference, of scale log2 e twice and of their product: 6 U d with what
the constant's own rounding adds.  A sum's term, e^-d, carries that and 160 U for the exponential and the additions (up to 32 in a thread, then in
pairs, then up to 64 chunks).  Where the sum is near 1 the terms that reach the maximum are counted, not added, and carry nothing.  Nothing
here grows with the logits themselves but lse, which is rounded once at its own size, from m scale, rounded at that.

The gradient's probabilities carry their exponent's rounding and the sum's; for results in bf16 those of ordinary rows come from lse, at most 64 U off, and
what the likeliest token leaves, 1 - p, at most 2^-11 of itself.  In fp32, and in every other row, that is the sum of the others, over S.
"""
import numpy as np
import pytest

import oracle.lm as olm

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
MOST = float(np.finfo(np.float32).max)


def _host(t):
    import torch
    torch.cuda.synchronize()
    return t.double().cpu().numpy()


def _same(got, want, tol):
    """Within the bound where a float holds the value, alike where it does not."""
    with np.errstate(invalid="ignore"):
        want = np.where(np.abs(want) > MOST, np.sign(want) * np.inf, want)
        fine = np.where(np.isfinite(want), np.abs(got - want) <= tol, got == want)
    assert fine.all(), (np.argwhere(~fine)[:4], got[~fine][:4], want[~fine][:4], np.broadcast_to(tol, want.shape)[~fine][:4])


class _Row:
    """Exact values of rows with a token left, and how far each may be off."""

    def __init__(self, x, scale):
        with np.errstate(invalid="ignore", over="ignore"):
            m = x.max(1, keepdims=True)
            self.d = np.where(x == m, 0.0, (m - x) * scale)
            self.e = np.exp(-self.d)
            d = np.where(self.e == 0, 0.0, self.d)
            self.at = self.d == 0
            self.n, self.S = self.at.sum(1), self.e.sum(1)
            term = self.e * (6 * d + 160) * U
            self.others = np.where(self.at, 0.0, term).sum(1)  # of what does not reach the maximum
            self.sum = np.where(self.S < 1.2, self.others, term.sum(1))
            self.log = np.where(self.S < 1.2, np.log1p((self.n - 1) + np.where(self.at, 0.0, self.e).sum(1)), np.log(self.S))
            q, q_tol = (self.e * d).sum(1) / self.S, (self.e * d * (6 * d + 168)).sum(1) * U / self.S
            self.h = self.log + q
            self.log_tol = self.sum / self.S + 4 * U * np.abs(self.log) + 2.0 ** -100
            self.h_tol = self.log_tol + q_tol + q * self.sum / self.S + 4 * U * (np.abs(self.log) + q)
            self.lp = -self.d - self.log[:, None]
            self.lp_tol = self.log_tol[:, None] + 4 * U * (np.abs(self.lp) + self.d)


def _check(x, tokens, top, scale, out):
    logp, lse, entropy, tl, ti = out
    _, rs, _, _, ri = olm.log_probs(x, tokens, top, scale)
    r = _Row(x, scale)
    rows = np.arange(len(x))
    _same(_host(logp), r.lp[rows, tokens], r.lp_tol[rows, tokens])
    _same(_host(lse), rs, r.log_tol + 4 * U * (np.abs(rs) + np.abs(x.max(1) * scale)))
    _same(_host(entropy), r.h, r.h_tol)
    assert (_host(ti) == ri).all()
    _same(_host(tl), np.take_along_axis(r.lp, ri, 1), np.take_along_axis(r.lp_tol, ri, 1))


def _logits(V, scale, most, dtype):
    """Rows around `most`: spread over some units, near their largest at this scale, all equal, two that share the largest, a sure token, masked."""
    import torch
    rng = np.random.default_rng([V, int(np.log2(scale)) + 200, int(abs(most)) % 1000])
    z = rng.standard_normal((6, V))
    x = most + 2.5 * z
    step = 2.0 ** -8 * abs(most)
    x[1] = most - np.abs(z[1]) * max(3 / scale, 2.0 ** -22 * abs(most))
    x[2] = most
    x[3] = most - step * (1 + np.abs(z[3]))
    x[3, rng.choice(V, 2, False)] = most
    x[4] = most - (12 + np.abs(z[4])) / min(scale, 1.0)
    x[4, rng.integers(V)] = most
    x[5, rng.random(V) < 0.9] = -np.inf
    x[5, rng.integers(V)] = most
    return torch.from_numpy(x.astype(np.float32)).to(torch.bfloat16 if dtype == "bf16" else torch.float32).cuda()


def _tokens(x, seed):
    """A token that may be given of each row: half of them the likeliest."""
    rng = np.random.default_rng(seed)
    return np.array([int(r.argmax()) if k % 2 else int(rng.choice(np.flatnonzero(np.isfinite(r)))) for k, r in enumerate(x)])


SCALES = [(s, 20.0) for s in (1e-30, 1e-3, 100.0, 1e4, 1e6, 1e8, 1e9, 1e10, 2.0 ** 40, 2.0 ** 70, 2.0 ** 100)]
SIZES = [(1.0, s * m) for m in (1e3, 1e5, 3e6, 1e8, 1e10, 3e12, 1e15, 1e25) for s in (1, -1)] + [(1e4, -90.0), (2.0 ** 60, 1e15)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V", [70, 1000, 5000, 33000])
@pytest.mark.parametrize("scale,most", SCALES + SIZES)
def test_forward_at_any_temperature(scale, most, V, dtype):
    import torch
    import paper_2407_09453_amd as bsp
    X = _logits(V, scale, most, dtype)
    x, scale = _host(X), float(np.float32(scale))
    tokens = _tokens(x, V)
    _check(x, tokens, 5, scale, bsp.log_probs(X, torch.from_numpy(tokens).cuda(), 5, scale))


def test_forward_where_no_float_holds_the_sum():
    """m scale past the largest float: lse is infinite, log probabilities are what they are."""
    import torch
    import paper_2407_09453_amd as bsp
    X = torch.full((4, 3000), -3e38, device="cuda")
    X[0, 5:8] = 3e38
    X[1] = 2e30
    X[2, 9] = 1e20
    tokens = np.array([5, 0, 9, 2])
    x = _host(X)
    _check(x, tokens, 3, 2.0 ** 100, bsp.log_probs(X, torch.from_numpy(tokens).cuda(), 3, 2.0 ** 100))


def _check_grad(x, tokens, dl, dh, scale, got, bf16):
    r = _Row(x, scale)
    rows = np.arange(len(x))
    held = 64 * U if bf16 else 0.0
    al, ah, S, h, log = (v[:, None] for v in (np.abs(dl), np.abs(dh), r.S, r.h, np.abs(r.log)))
    p = r.e / S
    with np.errstate(invalid="ignore"):
        lph = np.where(p == 0, 0.0, r.lp + h)
        d = np.where(p == 0, 0.0, r.d)
    one = np.zeros(x.shape, bool)
    one[rows, tokens] = True
    # 1 - p of each value: what does not reach the maximum, where it is the only one that does
    rest = np.where(r.at, (r.n - 1 + np.where(r.at, 0.0, r.e).sum(1))[:, None] / S, 1 - p)
    p_tol = p * ((6 * d + 16) * U + (r.sum / r.S)[:, None] + held)
    rest_tol = np.where(r.at, r.others[:, None] / S + rest * ((r.sum / r.S)[:, None] + 16 * U), p_tol + 4 * U) + (2.0 ** -11 * rest if bf16 else 0.0)
    want = scale * (dl[:, None] * np.where(one, rest, -p) - dh[:, None] * p * lph)
    lph_tol = r.h_tol[:, None] + r.log_tol[:, None] + 6 * U * d + 8 * U * (h + log + d) + held
    tol = p_tol * (np.where(one, 0.0, al) + ah * np.abs(lph)) + p * (ah * lph_tol + 8 * U * (al + ah * (h + log + d))) + np.where(one, al * (rest_tol + 4 * U * rest), 0.0)
    # (a probability below 2^-125 may be 0)
    tol = scale * (tol + 2.0 ** -125 * (al + ah * 200)) + (2.0 ** -8 if bf16 else 4 * U) * np.abs(want) + 2.0 ** -120
    _same(_host(got), want, tol)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V", [70, 1000, 3000, 5000, 12000, 30000, 33000, 70001])
@pytest.mark.parametrize("scale,most", [(1.0, 20.0)] + SCALES + SIZES)
def test_gradient_at_any_temperature(scale, most, V, dtype):
    import torch
    import paper_2407_09453_amd as bsp
    X = _logits(V, scale, most, dtype)
    x, scale = _host(X), float(np.float32(scale))
    tokens = _tokens(x, V)
    rng = np.random.default_rng(V + 1)
    dl, dh = (rng.standard_normal(len(x)).astype(np.float32) for _ in range(2))
    tok, dlt, dht = (torch.from_numpy(t).cuda() for t in (tokens, dl, dh))
    _, lse, entropy, _, _ = bsp.log_probs(X, tok, 0, scale)
    g = bsp.log_probs_grad(X, tok, lse, entropy, dlt, dht, scale)
    _check_grad(x, tokens, dl.astype(np.float64), dh.astype(np.float64), scale, g, dtype == "bf16")
    _check_grad(x, tokens, dl.astype(np.float64), 0 * dh.astype(np.float64), scale, bsp.log_probs_grad(X, tok, lse, entropy, dlt, None, scale), dtype == "bf16")
    again = bsp.log_probs_grad(X, tok, lse, entropy, dlt, dht, scale, out=X)
    assert again is X and torch.equal(g, X)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_sure_token_keeps_its_gradient(dtype):
    """A token that leaves a 2^-21st to the others: its gradient is minus the sum of theirs, to what the results' own rounding leaves."""
    import torch
    import paper_2407_09453_amd as bsp
    X = torch.zeros(2, 1000, device="cuda", dtype=torch.bfloat16 if dtype == "bf16" else torch.float32)
    X[:, 7] = 25.0
    X[1] += 1000.0 if dtype == "f32" else 0.0
    x, tokens = _host(X), np.array([7, 7])
    tok, one = torch.tensor(tokens, device="cuda"), torch.ones(2, device="cuda")
    _, lse, entropy, _, _ = bsp.log_probs(X, tok)
    g = bsp.log_probs_grad(X, tok, lse, entropy, one)
    _check_grad(x, tokens, np.ones(2), np.zeros(2), 1.0, g, dtype == "bf16")
    g = _host(g)
    assert (g[:, 7] > 0).all() and (np.abs(g.sum(1)) <= (2.0 ** -7 if dtype == "bf16" else 400 * U) * g[:, 7]).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V", [1000, 33000, 140000])
def test_a_row_has_the_same_gradient_in_any_batch(V, dtype):
    """Ordinary and sharp rows in turn, by themselves, among a few and among many (whose workgroups share them out otherwise)."""
    import torch
    import paper_2407_09453_amd as bsp
    gen = torch.Generator(device="cuda")
    gen.manual_seed(V)
    X = torch.randn(260, V, generator=gen, device="cuda")
    X[::2] *= 300
    X = X.to(torch.bfloat16 if dtype == "bf16" else torch.float32)
    tok = torch.randint(0, V, (260,), generator=gen, device="cuda")
    dl, dh = (torch.randn(260, generator=gen, device="cuda") for _ in range(2))
    _, lse, entropy, _, _ = bsp.log_probs(X, tok)
    assert (lse.abs()[::2] > 64).all() and (lse.abs()[1::2] < 64).all()
    g = bsp.log_probs_grad(X, tok, lse, entropy, dl, dh)
    for n in (1, 5, 40):
        for at in (0, 1, 219):
            r = slice(at, at + n)
            assert torch.equal(g[r], bsp.log_probs_grad(X[r].clone(), tok[r], lse[r], entropy[r], dl[r], dh[r]))
    bsp.log_probs_grad(X, tok, lse, entropy, dl, dh, out=X)
    assert torch.equal(g, X)
