"""Low-rank adapters of many requests beside an 8-bit layer, forward and backward, against the oracle in 64 bits.

Bounds.  U = 2^-24.  The layer's own product: 2^-10 of its magnitudes' sum for bf16 results, (terms + 8) U of it for fp32 ones (as the
layer's tests have them).  u = s A x adds bf16 products in fp32, a sixteenth of them one after the other at most: (K / 16 + 96) U of
their magnitudes; fp32 rows enter as three bf16 parts, each of which takes off half a step of 2^-8: 2^-26 of them is left.  For bf16 results u
enters as two parts, 2^-17 of itself is left, for fp32 ones and for gradients as three; at most 3 rank + 16 sums follow.  Gradients
likewise, over an adapter's rows in place of K, in chunks.  A bf16 result is rounded once more, 2^-8 of its value.
"""
import numpy as np
import pytest

import oracle.f8 as of8
import oracle.lm as olm

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


def _host(t):
    import torch
    torch.cuda.synchronize()
    return t.double().cpu().numpy()


def _rows(rng, T, K, dtype):
    import torch
    x = rng.standard_normal((T, K)) * np.exp(0.5 * rng.standard_normal((T, 1))) * np.where(rng.random(K) < 0.02, 10.0, 1.0)
    return torch.from_numpy(x.astype(np.float32)).to(torch.float32 if dtype == "f32" else torch.bfloat16).cuda()


class Case:
    def __init__(self, rng, T, I, O, R, N, density=0.7, which=None, bias=True):
        import torch
        import paper_2407_09453_amd as bsp
        W = rng.standard_normal((O, I)).astype(np.float32) / np.sqrt(I)
        self.gamma = (rng.random((-(-O // 128), -(-I // 128))) < density).astype(np.uint8)
        self.W, self.b = W, rng.standard_normal(O).astype(np.float32) if bias else None
        self.layer = bsp.BspLayerF8(W, self.gamma, bias=self.b)
        self.bank = bsp.BspAdapters(N, R, I, O)
        A = torch.from_numpy((rng.standard_normal((N, R, I)) / np.sqrt(I)).astype(np.float32)).to(torch.bfloat16)
        B = torch.from_numpy((rng.standard_normal((N, O, R))).astype(np.float32)).to(torch.bfloat16)
        self.scale = 2.0 ** rng.integers(-2, 2, N) * 0.75
        for n in range(N):
            self.bank.set(n, A[n].cuda(), B[n].cuda().float() if n % 2 else B[n].cuda(), float(self.scale[n])) if n % 2 == 0 else \
                self.bank.set(n, A[n].cuda().float(), B[n].cuda().float(), float(self.scale[n]))
        self.A, self.B = A.double().numpy(), B.double().numpy()
        self.which = rng.integers(-1, N, T) if which is None else np.asarray(which)
        self.requests = bsp.BspRequests(torch.from_numpy(self.which).to(torch.int32 if T % 2 else torch.int64).cuda(), N)

    def low_tol(self, x, A, B, dtype, out_bf16):
        """How far the adapters' part may be off."""
        amag, _ = olm.low_rank(np.abs(x), np.abs(A), np.abs(B), self.scale, self.which)
        u, _ = olm.low_rank(x, A, B, self.scale, self.which)
        du = ((x.shape[1] / 16 + 96) * U + (2.0 ** -26 if dtype == "f32" else 0)) * amag
        one = np.ones(len(self.scale))
        tol = np.zeros((len(x), B.shape[1]))
        for n in range(len(one)):
            r = np.flatnonzero(self.which == n)
            tol[r] = (du[r] + (2.0 ** (-17 if out_bf16 else -26) + (3 * A.shape[1] + 16) * U) * (np.abs(u[r]) + du[r])) @ np.abs(B[n]).T
        return tol

    def check(self, y, x, xq, dtype, out_bf16, relu=False, residual=None, transposed=False, gate=None):
        A, B = (np.swapaxes(self.B, 1, 2), np.swapaxes(self.A, 1, 2)) if transposed else (self.A, self.B)
        add = olm.low_rank(x, A, B, self.scale, self.which)[1] + (0 if residual is None else residual)
        want = of8.fc(xq, self.W, self.gamma, None if transposed else self.b, add, relu, coded=True, transposed=transposed, gate=gate)
        mag = of8.fc(np.abs(xq), np.abs(self.W), self.gamma, None if transposed else np.abs(self.b), np.abs(add), coded=True, transposed=transposed)
        tol = (2.0 ** -10 if out_bf16 else (x.shape[1] + 16) * U) * mag + self.low_tol(x, A, B, dtype, out_bf16) + (2.0 ** -8 if out_bf16 else 0) * np.abs(want) + 2.0 ** -120
        assert (np.abs(y - want) <= tol).all(), float((np.abs(y - want) / tol).max())


SHAPES = [  # T, I, O, R, N
    (1, 128, 128, 1, 1), (1, 4096, 512, 16, 8), (2, 1000, 520, 8, 3), (7, 129, 127, 3, 2), (16, 2048, 1000, 16, 20), (17, 300, 260, 17, 4), (32, 4096, 256, 64, 32), (31, 520, 4, 128, 3),
    (33, 512, 512, 16, 5), (64, 1000, 1000, 33, 64), (65, 4096, 384, 16, 7), (128, 256, 2048, 128, 2), (197, 2048, 1000, 5, 5), (300, 7, 5, 2, 3), (1021, 640, 520, 16, 300),
    (2048, 512, 1024, 8, 12), (700, 4096, 2048, 64, 3), (4100, 384, 256, 32, 1)]


@pytest.mark.parametrize("dtype", ["bf16", "f32", "codes"])
@pytest.mark.parametrize("T,I,O,R,N", SHAPES)
def test_layer_with_adapters(T, I, O, R, N, dtype):
    import torch
    import paper_2407_09453_amd as bsp
    rng = np.random.default_rng([T, I, O, R])
    c = Case(rng, T, I, O, R, N)
    X = _rows(rng, T, I, dtype)
    x = _host(X)
    xq = of8.values(x, "e4m3")
    bf16 = dtype != "f32"
    res = _rows(rng, T, O, dtype)
    given = bsp.save8(X) if dtype == "codes" else X
    x = xq if dtype == "codes" else x
    c.check(_host(c.layer.fc(given, adapters=c.bank, requests=c.requests)), x, xq, dtype, bf16)
    c.check(_host(c.layer.fc(given, relu=True, residual=res, adapters=c.bank, requests=c.requests)), x, xq, dtype, bf16, True, _host(res))
    if dtype == "codes":
        c.check(_host(c.layer.fc(given, dtype=torch.float32, adapters=c.bank, requests=c.requests)), x, xq, dtype, False)


@pytest.mark.parametrize("code", ["e5m2", "e4m3"])
@pytest.mark.parametrize("T,I,O,R,N", SHAPES)
def test_gradients(T, I, O, R, N, code):
    import paper_2407_09453_amd as bsp
    rng = np.random.default_rng([T, I, O, R, 1])
    c = Case(rng, T, I, O, R, N)
    dY, X = _rows(rng, T, O, "bf16"), _rows(rng, T, I, "bf16")
    dy, x = _host(dY), _host(X)
    dyq = of8.values(dy, code)
    c.check(_host(c.layer.grad_input(dY, code=code, adapters=c.bank, requests=c.requests)), dy, dyq, "bf16", True, transposed=True)
    kept = bsp.save8(X.clamp_min(0), code)
    gate = _host(kept.load())
    c.check(_host(c.layer.grad_input(dY, relu_of=kept, code=code, adapters=c.bank, requests=c.requests)), dy, dyq, "bf16", True, transposed=True, gate=gate)
    coded = bsp.save8(dY, code)
    c.check(_host(c.layer.grad_input(coded, adapters=c.bank, requests=c.requests)), dyq, dyq, "codes", True, transposed=True)
    for given, xs in ((kept, gate), (X, x)):
        dA, dB = (_host(t) for t in c.bank.grad(dY, given, c.requests))
        _check_grad(c, dA, dB, dy, xs)


def _check_grad(c, dA, dB, dy, x):
    rA, rB = olm.low_rank_grad(dy, x, c.A, c.B, c.scale, c.which)
    Bt, At = np.swapaxes(c.B, 1, 2), np.swapaxes(c.A, 1, 2)
    for n in range(len(c.scale)):
        r = np.flatnonzero(c.which == n)
        s = c.scale[n]
        u, v = s * x[r] @ c.A[n].T, s * dy[r] @ c.B[n]
        du = s * (x.shape[1] / 16 + 96) * U * (np.abs(x[r]) @ np.abs(c.A[n]).T)
        dv = s * (dy.shape[1] / 16 + 96) * U * (np.abs(dy[r]) @ np.abs(c.B[n]))
        f = 2.0 ** -26 + (3 * len(r) + 64) * U
        tA, tB = (dv + f * (np.abs(v) + dv)).T @ np.abs(x[r]), np.abs(dy[r]).T @ (du + f * (np.abs(u) + du))
        assert (np.abs(dA[n] - rA[n]) <= tA + 2.0 ** -120).all(), (n, float((np.abs(dA[n] - rA[n]) / (tA + 2.0 ** -120)).max()))
        assert (np.abs(dB[n] - rB[n]) <= tB + 2.0 ** -120).all(), (n, float((np.abs(dB[n] - rB[n]) / (tB + 2.0 ** -120)).max()))
    assert Bt.shape and At.shape


@pytest.mark.parametrize("name,which", [
    ("none", [-1] * 300), ("one", [2] * 300), ("past", [7, 8, 1 << 20, -5] * 75), ("runs", [0] * 100 + [3] * 33 + [-1] * 17 + [1] * 150), ("last", [-1] * 299 + [4]),
    ("turns", list(range(5)) * 60)])
def test_whose_rows(name, which):
    """All of one adapter, of none, of no such adapter, in runs and in turn; the plan itself; gradients of adapters without rows are zero."""
    import torch
    import paper_2407_09453_amd as bsp
    rng = np.random.default_rng(5)
    which = np.array(which)
    c = Case(rng, 300, 384, 260, 8, 5, which=which)
    c.which = np.where((which >= 0) & (which < 5), which, -1)
    X, dY = _rows(rng, 300, 384, "bf16"), _rows(rng, 300, 260, "bf16")
    x, dy = _host(X), _host(dY)
    c.check(_host(c.layer.fc(X, adapters=c.bank, requests=c.requests)), x, of8.values(x, "e4m3"), "bf16", True)
    few = bsp.BspRequests(torch.from_numpy(which[-20:]).cuda(), 5)
    got = c.layer.fc(X[-20:], adapters=c.bank, requests=few)
    d, c.which = c.which, c.which[-20:]
    c.check(_host(got), x[-20:], of8.values(x[-20:], "e4m3"), "bf16", True)
    c.which = d
    dA, dB = (_host(t) for t in c.bank.grad(dY, X, c.requests))
    _check_grad(c, dA, dB, dy, x)
    for n in range(5):
        if not (c.which == n).any():
            assert not dA[n].any() and not dB[n].any()
    if (c.which < 0).any():  # rows without an adapter: the layer's own results, bit for bit
        none = np.flatnonzero(c.which < 0)
        assert torch.equal(c.layer.fc(X)[none], c.layer.fc(X, adapters=c.bank, requests=c.requests)[none])


@pytest.mark.parametrize("T", [1, 63, 64, 65, 1024, 5000, 40000])
@pytest.mark.parametrize("N", [1, 3, 64, 65, 1000, 1024])
def test_plan(T, N):
    """Sorted by adapter, rows in their order within each, those of none last; tiles of up to 64 rows that hold each once."""
    import torch
    import paper_2407_09453_amd as bsp
    rng = np.random.default_rng([T, N])
    which = rng.integers(-2, N + 2, T)
    which[rng.random(T) < 0.3] = N // 2
    q = bsp.BspRequests(torch.from_numpy(which).cuda(), N)
    torch.cuda.synchronize()
    p = q.plan.view(torch.int32).cpu().numpy()
    own = np.where((which >= 0) & (which < N), which, -1)
    at = (N + 1 + 3) & ~3
    start, w = p[:N + 1], p[at:at + T]
    t4 = (T + 3) & ~3
    order, tiles = p[at + t4:at + t4 + T], p[at + 2 * t4:]
    counts = np.bincount(own[own >= 0], minlength=N)
    assert (w == own).all() and (start == np.concatenate([[0], counts.cumsum()])).all()
    want = np.argsort(np.where(own < 0, N, own), kind="stable")
    assert (order == want).all()
    records = [(a, want[s + j:s + min(j + 64, n)]) for a, s, n in [*zip(range(N), start, counts), (-1, start[N], T - start[N])] for j in range(0, n, 64)]
    assert tiles[1] == len(records) and tiles[0] == sum(a >= 0 for a, _ in records)
    for k, (a, rows) in enumerate(records):
        r = tiles[4 + 68 * k:4 + 68 * (k + 1)]
        assert r[0] == a and r[1] == len(rows) and (r[4:4 + len(rows)] == rows).all() and (r[4 + len(rows):] == rows[-1]).all()


def test_nothing_of_another_row_or_adapter():
    """An adapter of NaN and a row of infinities reach their own rows alone, in results and gradients; a slot that is cleared or not set adds nothing."""
    import torch
    import paper_2407_09453_amd as bsp
    for T in (20, 200):
        rng = np.random.default_rng(T)
        c = Case(rng, T, 640, 384, 16, 6, which=np.arange(T) % 7 - 1)
        X, dY = _rows(rng, T, 640, "bf16"), _rows(rng, T, 384, "bf16")
        y, dx, (dA, dB) = c.layer.fc(X, adapters=c.bank, requests=c.requests), c.layer.grad_input(dY, adapters=c.bank, requests=c.requests), c.bank.grad(dY, X, c.requests)
        c.bank.set(3, torch.full((16, 640), float("nan"), device="cuda"), torch.full((384, 16), float("inf"), device="cuda"))
        X[8] = float("inf")  # of adapter 0
        assert c.which[8] == 0
        y2, dx2, (dA2, dB2) = c.layer.fc(X, adapters=c.bank, requests=c.requests), c.layer.grad_input(dY, adapters=c.bank, requests=c.requests), c.bank.grad(dY, X, c.requests)
        sick = c.which == 3
        rest = ~sick & (np.arange(T) != 8)
        for a, b in ((y, y2), (dx, dx2)):
            assert torch.equal(a[rest], b[rest]) and torch.isnan(b[sick]).all()
        keep = [1, 2, 4, 5]
        assert torch.equal(dA[keep], dA2[keep]) and torch.equal(dB[keep], dB2[keep])
        c.bank.clear(3)
        X[8] = 0
        y3 = c.layer.fc(X, adapters=c.bank, requests=c.requests)
        assert torch.equal(y3[sick], c.layer.fc(X)[sick])
        fresh = bsp.BspAdapters(6, 16, 640, 384)
        assert torch.equal(c.layer.fc(X, adapters=fresh, requests=c.requests), c.layer.fc(X))


def test_lower_rank_and_another_step():
    """A slot of a lower rank than the set's, and new weights in it."""
    import torch
    rng = np.random.default_rng(4)
    c = Case(rng, 50, 300, 260, 20, 2)
    X = _rows(rng, 50, 300, "f32")
    x = _host(X)
    for r in (1, 7, 20):
        A, B = torch.from_numpy(rng.standard_normal((r, 300)).astype(np.float32)).cuda(), torch.from_numpy(rng.standard_normal((260, r)).astype(np.float32)).cuda()
        c.bank.set(1, A, B, 0.5)
        c.A[1], c.B[1], c.scale[1] = 0, 0, 0.5
        c.A[1, :r], c.B[1, :, :r] = _host(A.bfloat16()), _host(B.bfloat16())
        c.check(_host(c.layer.fc(X, adapters=c.bank, requests=c.requests)), x, of8.values(x, "e4m3"), "f32", False)


def test_gradient_against_differences():
    """The adapters' part of the loss sum(dy y), linear in A and in B: its change along a direction, in 64 bits, is the gradient along it."""
    rng = np.random.default_rng(9)
    c = Case(rng, 90, 200, 150, 6, 3)
    dY, X = _rows(rng, 90, 150, "bf16"), _rows(rng, 90, 200, "bf16")
    dA, dB = (_host(t) for t in c.bank.grad(dY, X, c.requests))
    dy, x = _host(dY), _host(X)
    loss = lambda A, B: float((dy * olm.low_rank(x, A, B, c.scale, c.which)[1]).sum())  # noqa: E731
    base = loss(c.A, c.B)
    for _ in range(5):
        d, e = rng.standard_normal(c.A.shape), rng.standard_normal(c.B.shape)
        # a sum of n terms, each off by a few hundred U of its size: their spread bounds it
        assert abs(loss(c.A + d, c.B) - base - (dA * d).sum()) <= 2.0 ** -15 * np.sqrt((dA * dA).sum() * (d * d).sum())
        assert abs(loss(c.A, c.B + e) - base - (dB * e).sum()) <= 2.0 ** -15 * np.sqrt((dB * dB).sum() * (e * e).sum())


def test_rows_anywhere_and_none():
    import torch
    import paper_2407_09453_amd as bsp
    rng = np.random.default_rng(6)
    base = torch.randn(60, 1111, device="cuda")
    layer, bank = bsp.BspLayerF8(torch.randn(260, 700, device="cuda") * 0.03), bsp.BspAdapters(4, 8, 700, 260)
    wide = torch.randn(8, 801, device="cuda")
    for n in range(4):
        bank.set(n, wide[:, 50:750], torch.randn(260, 30, device="cuda")[:, 11:19], 1.0)
    for X in (base[:, :700], base[::3, 11:711], base.to(torch.bfloat16)[:, 3:703], base[:1, :700].expand(50, 700)):
        q = bsp.BspRequests(torch.from_numpy(rng.integers(-1, 4, len(X))), 4)
        assert torch.equal(layer.fc(X, adapters=bank, requests=q), layer.fc(X.contiguous(), adapters=bank, requests=q))
    both = base.to(torch.bfloat16)
    q = bsp.BspRequests(torch.from_numpy(rng.integers(-1, 4, 60)).cuda(), 4)
    a = bank.grad(both[:, 3:263], both[:, 5:705], q)
    b = bank.grad(both[:, 3:263].contiguous(), both[:, 5:705].contiguous(), q)
    assert all(torch.equal(x, y) for x, y in zip(a, b))
    q = bsp.BspRequests(torch.empty(0, dtype=torch.int32, device="cuda"), 4)
    none = torch.empty(0, 700, device="cuda", dtype=torch.bfloat16)
    assert layer.fc(none, adapters=bank, requests=q).shape == (0, 260)
    dA, dB = bank.grad(torch.empty(0, 260, device="cuda", dtype=torch.bfloat16), none, q)
    assert not dA.any() and not dB.any() and dA.shape == (4, 8, 700) and dB.shape == (4, 260, 8)


@pytest.mark.parametrize("T", [5, 24, 600])
def test_same_bits_every_time_and_in_a_graph(T):
    """A captured step replayed on other rows and another assignment of them, against eager calls between the replays."""
    import torch
    import paper_2407_09453_amd as bsp
    rng = np.random.default_rng(T)
    c = Case(rng, T, 1000, 520, 16, 9)
    X, dY = _rows(rng, T, 1000, "bf16"), _rows(rng, T, 520, "bf16")
    ids = torch.from_numpy(c.which).cuda()
    q = bsp.BspRequests(ids, 9)

    def both():
        q.update(ids)
        kept = bsp.save8(X)
        return (c.layer.fc(X, adapters=c.bank, requests=q), c.layer.grad_input(dY, adapters=c.bank, requests=q), *c.bank.grad(dY, kept, q))
    want = both()
    for _ in range(2):
        assert all(torch.equal(a, b) for a, b in zip(want, both()))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        both()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = both()
    for k in range(4):
        X.copy_(torch.randn(T, 1000, device="cuda"))
        dY.copy_(torch.randn(T, 520, device="cuda"))
        ids.copy_(torch.randint(-1, 9, (T,), device="cuda"))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(both(), got)), k


def test_on_a_stream_of_the_caller_and_autograd_is_told():
    import torch
    rng = np.random.default_rng(2)
    c = Case(rng, 500, 1000, 520, 16, 9)
    X, dY = _rows(rng, 500, 1000, "bf16"), _rows(rng, 500, 520, "bf16")
    want = (c.layer.fc(X, adapters=c.bank, requests=c.requests), c.layer.grad_input(dY, adapters=c.bank, requests=c.requests), *c.bank.grad(dY, X, c.requests))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    s = side.cuda_stream
    c.requests.update(torch.from_numpy(c.which).cuda(), stream=s)
    got = (c.layer.fc(X, adapters=c.bank, requests=c.requests, stream=s), c.layer.grad_input(dY, adapters=c.bank, requests=c.requests, stream=s),
           *c.bank.grad(dY, X, c.requests, stream=s))
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    with pytest.warns(UserWarning, match="records nothing"):
        c.bank.grad(dY.clone().requires_grad_(), X, c.requests)


def test_refusals():
    import torch
    import paper_2407_09453_amd as bsp
    layer, bank = bsp.BspLayerF8(torch.randn(260, 700, device="cuda")), bsp.BspAdapters(4, 8, 700, 260)
    q = bsp.BspRequests(torch.zeros(3, dtype=torch.int32), 4)
    X = torch.randn(3, 700, device="cuda")
    for kw in (dict(adapters=bank), dict(requests=q), dict(adapters=bsp.BspAdapters(4, 8, 700, 300), requests=q), dict(adapters=bsp.BspAdapters(5, 8, 700, 260), requests=q),
               dict(adapters=bank, requests=bsp.BspRequests(torch.zeros(4, dtype=torch.int32), 4))):
        with pytest.raises(AssertionError):
            layer.fc(X, **kw)
    A, B = torch.randn(8, 700, device="cuda"), torch.randn(260, 8, device="cuda")
    for slot, a, b in ((4, A, B), (-1, A, B), (0, A, B[:, :7]), (0, A[:, :699], B), (0, A.bfloat16(), B), (0, A.half(), B.half()), (0, A.cpu(), B.cpu()), (0, torch.randn(9, 700, device="cuda"), torch.randn(260, 9, device="cuda"))):
        with pytest.raises(AssertionError):
            bank.set(slot, a, b)
    with pytest.raises(AssertionError):
        bank.grad(torch.randn(3, 260, device="cuda"), X.bfloat16(), q)
    with pytest.raises(AssertionError):
        q.update(torch.zeros(4, dtype=torch.int32))
