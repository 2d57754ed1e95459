"""Host side of root-mean-square norm, adapters and log probabilities: refusals, sizes, the packed calls, and the oracle against its own definition."""
import ctypes
import struct

import numpy as np
import pytest

import oracle.lm as olm
import paper_2407_09453_amd as bsp
from paper_2407_09453_amd import binding as b

OK, NULL, SHAPE, DTYPE, CAPACITY, ALIGN = 0, -1, -2, -5, -7, -9
P = 1 << 20  # an address that no call may touch: every one of these is refused before anything is launched
BF, F32 = b.BSP_BF16, b.BSP_F32


def _codes(T=8, K=384, dtype=b.BSP_E4M3, codes=P, scale=P):
    return b.bsp_codes(T, K, dtype, codes, scale)


def _ref(s):
    return None if s is None else ctypes.byref(s)


def _weights(O=256, I=384, **kw):
    w = b.bsp_weights_f8(O, I, 6, P, P, P, P, P, P, P, P)
    for k, v in kw.items():
        setattr(w, k, v)
    return w


def _adapters(N=4, R=16, I=384, O=256, **kw):
    d = b.bsp_f8_adapters(N, R, I, O, P, P, P, P, P)
    for k, v in kw.items():
        setattr(d, k, v)
    return d


def _requests(T=8, N=4, plan=P):
    return b.bsp_f8_requests(T, N, plan)


@pytest.mark.parametrize("want,args", [
    (DTYPE, dict(dt=b.BSP_I8)), (SHAPE, dict(T=-1)), (SHAPE, dict(D=0)), (SHAPE, dict(ldx=383)), (NULL, dict(X=None)), (ALIGN, dict(X=P + 1)), (SHAPE, dict(eps=-1.0)),
    (SHAPE, dict(eps=float("nan"))), (NULL, dict(H=None)), (NULL, dict(r=None)), (SHAPE, dict(ldr=100)), (SHAPE, dict(ldh=0)), (ALIGN, dict(r=P + 1)), (NULL, dict(Y=None)),
    (NULL, dict(c=_codes())), (SHAPE, dict(Y=None, c=_codes(T=7))), (SHAPE, dict(Y=None, c=_codes(K=256))), (DTYPE, dict(Y=None, c=_codes(dtype=BF))), (NULL, dict(rstd=None)),
    (ALIGN, dict(w=P + 2)), (ALIGN, dict(rstd=P + 2)), (SHAPE, dict(ldy=383)), (OK, dict(T=0, X=None, r=None, H=None, Y=None, rstd=None)),
])
def test_rms_refusals(want, args):
    a = {**dict(X=P, ldx=384, r=P, ldr=384, dt=BF, T=8, D=384, w=P, eps=1e-6, H=P, ldh=384, Y=P, ldy=384, c=None, rstd=P), **args}
    assert bsp.load_library().bsp_rms_norm(a["X"], a["ldx"], a["r"], a["ldr"], a["dt"], a["T"], a["D"], a["w"], a["eps"], a["H"], a["ldh"], a["Y"], a["ldy"],
                                           _ref(a["c"]), a["rstd"], None) == want


@pytest.mark.parametrize("want,args", [
    (DTYPE, dict(dt=b.BSP_I8)), (SHAPE, dict(ld=383)), (NULL, dict(dY=None)), (NULL, dict(H=None)), (ALIGN, dict(dH=P + 1)), (NULL, dict(dX=None)), (NULL, dict(rstd=None)),
    (ALIGN, dict(w=P + 1)), (ALIGN, dict(dw=P + 2)), (CAPACITY, dict(T=5000, n=512 * 384 * 4 - 1)), (NULL, dict(T=600, ws=None)), (ALIGN, dict(ws=P + 8)), (SHAPE, dict(D=0)),
])
def test_rms_gradient_refusals(want, args):
    a = {**dict(dY=P, ld=384, H=P, dH=P, dt=BF, T=8, D=384, rstd=P, w=P, dX=P, dw=P, ws=P, n=1 << 30), **args}
    lib = bsp.load_library()
    assert lib.bsp_rms_norm_grad(a["dY"], a["ld"], a["H"], a["ld"], a["dH"], a["ld"], a["dt"], a["T"], a["D"], a["rstd"], a["w"], a["dX"], a["ld"], a["dw"],
                                 a["ws"], a["n"], None) == want
    n = ctypes.c_int64(-1)
    assert lib.bsp_rms_norm_grad_workspace(8, 384, n) == OK and n.value == 0
    assert lib.bsp_rms_norm_grad_workspace(600, 384, None) == NULL and lib.bsp_rms_norm_grad_workspace(-1, 384, n) == SHAPE


@pytest.mark.parametrize("want,args", [
    (DTYPE, dict(dt=b.BSP_I8)), (SHAPE, dict(T=-1)), (SHAPE, dict(V=0)), (SHAPE, dict(V=(1 << 21) + 1, ld=1 << 22)), (SHAPE, dict(ld=999)), (NULL, dict(X=None)), (ALIGN, dict(X=P + 1)),
    (DTYPE, dict(tb=2)), (NULL, dict(tok=None)), (ALIGN, dict(tok=P + 4)), (SHAPE, dict(scale=0.0)), (SHAPE, dict(scale=-1.0)), (SHAPE, dict(scale=float("nan"))),
    (SHAPE, dict(scale=float("inf"))), (SHAPE, dict(scale=2.0 ** 101)), (SHAPE, dict(top=65)), (SHAPE, dict(top=-1)), (SHAPE, dict(V=5, top=6)), (NULL, dict(lse=None)), (NULL, dict(logp=None)),
    (NULL, dict(top=3, tl=None)), (NULL, dict(top=3, ti=None)), (ALIGN, dict(entropy=P + 2)), (CAPACITY, dict(V=20000, ld=20000, top=3, n=8 * 10 * 40 - 1)),
    (NULL, dict(V=20000, ld=20000, top=3, ws=None)), (ALIGN, dict(V=20000, ld=20000, ws=P + 8)), (OK, dict(T=0, X=None, tok=None)),
])
def test_log_probs_refusals(want, args):
    a = {**dict(X=P, ld=1000, dt=BF, T=8, V=1000, tok=P, tb=8, scale=1.0, top=0, logp=P, lse=P, entropy=P, tl=P, ti=P, ws=P, n=1 << 30), **args}
    assert bsp.load_library().bsp_log_probs(a["X"], a["ld"], a["dt"], a["T"], a["V"], a["tok"], a["tb"], a["scale"], a["top"], a["logp"], a["lse"], a["entropy"],
                                            a["tl"], a["ti"], a["ws"], a["n"], None) == want


@pytest.mark.parametrize("want,args", [
    (DTYPE, dict(dt=b.BSP_I8)), (SHAPE, dict(ld=999)), (NULL, dict(X=None)), (NULL, dict(dX=None)), (SHAPE, dict(ldd=0)), (DTYPE, dict(tb=0)), (NULL, dict(tok=None)), (NULL, dict(lse=None)),
    (NULL, dict(entropy=None)), (ALIGN, dict(dlogp=P + 1)), (ALIGN, dict(dentropy=P + 1)), (SHAPE, dict(scale=0.0)), (SHAPE, dict(scale=2.0 ** 101)), (SHAPE, dict(dX=P, ldd=1001)), (OK, dict(T=0, X=None, dX=None)),
])
def test_log_probs_gradient_refusals(want, args):
    a = {**dict(X=P, ld=1000, dt=BF, T=8, V=1000, tok=P, tb=4, scale=1.0, lse=P, entropy=P, dlogp=P, dentropy=P, dX=2 * P, ldd=1000), **args}
    assert bsp.load_library().bsp_log_probs_grad(a["X"], a["ld"], a["dt"], a["T"], a["V"], a["tok"], a["tb"], a["scale"], a["lse"], a["entropy"], a["dlogp"], a["dentropy"],
                                                 a["dX"], a["ldd"], None) == want


def test_adapter_sizes_and_refusals():
    lib = bsp.load_library()
    na, nb, n = ctypes.c_int64(0), ctypes.c_int64(0), ctypes.c_int64(0)
    for R, Rp in ((1, 16), (16, 16), (17, 32), (33, 64), (64, 64), (65, 128), (128, 128)):
        assert lib.bsp_f8_adapters_size(R, 300, 129, na, nb) == OK and (na.value, nb.value) == (Rp * 384, Rp * 256)
    for R, I, O in ((0, 1, 1), (129, 1, 1), (1, 0, 1), (1, 1, 0), (1, (1 << 24) + 1, 1)):
        assert lib.bsp_f8_adapters_size(R, I, O, na, nb) == SHAPE
    assert lib.bsp_f8_adapters_size(1, 1, 1, None, nb) == NULL
    assert lib.bsp_f8_requests_size(-1, 4, n) == SHAPE and lib.bsp_f8_requests_size(8, 0, n) == SHAPE and lib.bsp_f8_requests_size(8, 1025, n) == SHAPE
    assert lib.bsp_f8_requests_size((1 << 26) + 1, 4, n) == SHAPE and lib.bsp_f8_requests_size(8, 4, None) == NULL
    for want, kw in ((NULL, dict(which=None)), (DTYPE, dict(size=2)), (ALIGN, dict(which=P + 4)), (NULL, dict(r=_requests(plan=None))), (ALIGN, dict(r=_requests(plan=P + 8))),
                     (SHAPE, dict(r=_requests(N=0))), (NULL, dict(r=None)), (OK, dict(r=_requests(T=0, plan=None), which=None))):
        a = {**dict(r=_requests(), which=P, size=8), **kw}
        assert lib.bsp_f8_requests_plan(_ref(a["r"]), a["which"], a["size"], None) == want, kw
    for want, kw in ((NULL, dict(d=None)), (SHAPE, dict(slot=4)), (SHAPE, dict(slot=-1)), (SHAPE, dict(rank=17)), (SHAPE, dict(rank=-1)), (NULL, dict(A=None)), (NULL, dict(B=None)),
                     (SHAPE, dict(lda=383)), (SHAPE, dict(ldb=15)), (DTYPE, dict(dt=b.BSP_I8)), (DTYPE, dict(dt=b.BSP_I8, rank=0)), (ALIGN, dict(A=P + 1)), (SHAPE, dict(d=_adapters(R=129))),
                     (SHAPE, dict(d=_adapters(N=1025))), (NULL, dict(d=_adapters(b_t=None))), (ALIGN, dict(d=_adapters(a=P + 8)))):
        a = {**dict(d=_adapters(), slot=0, rank=16, A=P, lda=384, B=P, ldb=16, dt=BF), **kw}
        assert lib.bsp_f8_adapters_set(_ref(a["d"]), a["slot"], a["rank"], a["A"], a["lda"], a["B"], a["ldb"], a["dt"], 1.0, None) == want, kw


@pytest.mark.parametrize("want,args", [
    (NULL, dict(w=None)), (NULL, dict(d=None)), (NULL, dict(q=None)), (SHAPE, dict(q=_requests(T=9))), (SHAPE, dict(q=_requests(N=5))), (SHAPE, dict(d=_adapters(I=256))),
    (SHAPE, dict(d=_adapters(O=384))), (SHAPE, dict(T=7)), (SHAPE, dict(X=_codes(T=9))), (SHAPE, dict(X=_codes(K=256))), (SHAPE, dict(t=1)), (DTYPE, dict(X=_codes(dtype=BF))),
    (NULL, dict(X=None)), (DTYPE, dict(X=None, values=P, code=BF)), (DTYPE, dict(X=None, values=P, xdt=b.BSP_E4M3)), (SHAPE, dict(X=None, values=P, ld=100)),
    (ALIGN, dict(X=None, values=P + 1)), (NULL, dict(Y=None)), (ALIGN, dict(Y=P + 2)), (DTYPE, dict(ydt=b.BSP_I8)), (SHAPE, dict(gate=_codes(K=384))), (CAPACITY, dict(n=8 * 16 * 4 - 1)),
    (NULL, dict(ws=None)), (ALIGN, dict(ws=P + 8)), (NULL, dict(d=_adapters(scale=None))), (OK, dict(T=0, X=_codes(T=0, codes=None, scale=None), q=_requests(T=0), Y=None)),
])
def test_adapted_product_refusals(want, args):
    a = {**dict(w=_weights(), t=0, X=_codes(), values=None, xdt=BF, ld=384, T=8, code=b.BSP_E4M3, d=_adapters(), q=_requests(), r=None, gate=None, Y=P, ydt=BF, ws=P, n=1 << 30), **args}
    lib = bsp.load_library()
    assert lib.bsp_f8_fc_adapted(_ref(a["w"]), a["t"], _ref(a["X"]), a["values"], a["xdt"], a["ld"], a["T"], a["code"], _ref(a["d"]), _ref(a["q"]), None, a["r"], 0, _ref(a["gate"]),
                                 a["Y"], a["ydt"], a["ws"], a["n"], None) == want
    n = ctypes.c_int64(-1)
    assert lib.bsp_f8_fc_adapted_workspace(_weights(), 0, 8, 1, _adapters(), n) == OK and n.value == 8 * 16 * 4
    assert lib.bsp_f8_fc_adapted_workspace(_weights(), 0, 17, 0, _adapters(), n) == OK and n.value == (17 * 384 + 32 * 3 + 15) // 16 * 16 + 17 * 16 * 4
    for T, N, coded, copied in ((32, 4, 1, 0), (33, 4, 1, 1), (33, 1, 1, 0), (33, 1, 0, 1)):  # many rows of several adapters: room for their codes
        assert lib.bsp_f8_fc_adapted_workspace(_weights(), 0, T, coded, _adapters(N=N), n) == OK
        plain = ctypes.c_int64(0)
        assert lib.bsp_f8_fc_workspace(_weights(), 0, T, 1 - copied, plain) == OK
        assert n.value == (plain.value + 15) // 16 * 16 + T * 16 * 4
    assert lib.bsp_f8_fc_adapted_workspace(_weights(), 0, 8, 1, None, n) == NULL and lib.bsp_f8_fc_adapted_workspace(_weights(), 0, 8, 1, _adapters(), None) == NULL


@pytest.mark.parametrize("want,args", [
    (NULL, dict(d=None)), (NULL, dict(q=None)), (SHAPE, dict(q=_requests(T=9))), (SHAPE, dict(q=_requests(N=3))), (SHAPE, dict(T=-1)), (NULL, dict(dY=None)), (SHAPE, dict(ld=255)),
    (SHAPE, dict(X=_codes(K=256))), (SHAPE, dict(X=_codes(T=7))), (NULL, dict(X=None)), (SHAPE, dict(X=None, values=P, ldx=100)), (NULL, dict(dA=None)), (NULL, dict(dB=None)),
    (ALIGN, dict(dA=P + 2)), (CAPACITY, dict(n=2 * 8 * 16 * 4 - 1)), (NULL, dict(ws=None)), (ALIGN, dict(ws=P + 4)),
])
def test_adapters_gradient_refusals(want, args):
    a = {**dict(d=_adapters(), dY=P, ld=256, X=_codes(), values=None, ldx=384, T=8, q=_requests(), dA=P, dB=P, ws=P, n=1 << 30), **args}
    assert bsp.load_library().bsp_f8_adapters_grad(_ref(a["d"]), a["dY"], a["ld"], _ref(a["X"]), a["values"], a["ldx"], a["T"], _ref(a["q"]), a["dA"], a["dB"], a["ws"], a["n"],
                                                   None) == want


def test_packed_calls_refuse_what_the_calls_refuse():
    call = bsp.load_library().bsp_f8_call_packed
    words = lambda *w: struct.pack("=%dq" % len(w), *w)  # noqa: E731
    one = struct.unpack("=q", struct.pack("=d", 1.0))[0]
    rms = [P, 384, 0, 0, BF, 8, 384, P, one, 0, 0, P, 384, 0, 0, 0, 0, 0, P, 0]
    for at, value, want in ((0, 0, NULL), (4, 77, DTYPE), (4, 2**32 + BF, DTYPE), (5, 2**32 + 8, SHAPE), (6, -1, SHAPE), (9, P, NULL), (11, 0, NULL), (18, 0, NULL), (18, P + 1, ALIGN)):
        w = list(rms)
        w[at] = value
        assert call(16, words(*w)) == want, (at, value)
    logp = [P, 1000, BF, 8, 1000, P, 8, one, 0, P, P, P, 0, 0, 0, 0, 0]
    for at, value, want in ((0, 0, NULL), (2, 77, DTYPE), (3, 2**33, SHAPE), (6, 2**32 + 8, DTYPE), (7, 0, SHAPE), (8, 65, SHAPE), (8, 2**32 + 1, SHAPE), (8, 3, NULL), (10, 0, NULL)):
        w = list(logp)
        w[at] = value
        assert call(18, words(*w)) == want, (at, value)
    assert call(17, words(*[0] * 17)) == SHAPE and call(19, words(*[0] * 15)) == SHAPE and call(20, words(*[0] * 27)) == NULL and call(21, words(*[0] * 17)) == NULL
    assert call(22, words(*[0] * 30)) == SHAPE and call(15, words(*[0] * 30)) == SHAPE


def test_oracle_gradients_against_differences():
    rng = np.random.default_rng(0)
    x, dy, dh, w = rng.standard_normal((3, 20)), rng.standard_normal((3, 20)), rng.standard_normal((3, 20)), rng.standard_normal(20)
    dx, dw = olm.rms_norm_grad(dy, x, w, dh=dh)
    A, B, s, which = rng.standard_normal((2, 3, 20)), rng.standard_normal((2, 5, 3)), np.array([0.5, 2.0]), np.array([1, -1, 0])
    d5 = rng.standard_normal((3, 5))
    dA, dB = olm.low_rank_grad(d5, x, A, B, s, which)
    tokens, dl, de = np.array([3, -1, 19]), rng.standard_normal(3), rng.standard_normal(3)
    dz = olm.log_probs_grad(x, tokens, dl, de, 0.7)

    def logp(x):
        lp, _, h, _, _ = olm.log_probs(x, tokens, 0, 0.7)
        return (dl * lp + de * h).sum()
    for f, v, g in ((lambda v: (dy * olm.rms_norm(v, w)[0]).sum() + (dh * v).sum(), x, dx), (lambda v: (dy * olm.rms_norm(x, v)[0]).sum(), w, dw),
                    (lambda v: (d5 * olm.low_rank(x, v, B, s, which)[1]).sum(), A, dA), (lambda v: (d5 * olm.low_rank(x, A, v, s, which)[1]).sum(), B, dB), (logp, x, dz)):
        for k in rng.integers(0, v.size, 8):
            d = np.zeros(v.size)
            d[k] = 1e-6
            d = d.reshape(v.shape)
            assert abs((f(v + d) - f(v - d)) / 2e-6 - g.ravel()[k]) < 1e-7 * (1 + abs(g).max())


def test_oracle_order_and_masks():
    x = np.array([[1.0, 3.0, 3.0, -np.inf, 0.0, -0.0], [np.nan, 1.0, np.inf, 2.0, np.nan, -np.inf], [-np.inf] * 6])
    assert olm.order(x).tolist() == [[1, 2, 0, 4, 5, 3], [0, 4, 2, 3, 1, 5], [0, 1, 2, 3, 4, 5]]
    logp, lse, h, top, ids = olm.log_probs(x, [0, 1, 2], 2)
    assert lse[2] == -np.inf and logp[2] == -np.inf and h[2] == 0 and (top[2] == -np.inf).all() and np.isnan(lse[1])
    assert abs(np.exp(olm.log_probs(x[:1], [0], 6)[3]).sum() - 1) < 1e-12
