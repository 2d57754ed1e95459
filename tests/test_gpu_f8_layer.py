"""What a BspLayerF8 holds and what it takes from its caller: biases, new weights, types, refusals of the tensors' side."""
import numpy as np
import pytest


pytestmark = pytest.mark.gpu


def _bsp():
    import paper_2407_09453_amd as bsp
    return bsp


def _host(t):
    import torch
    torch.cuda.synchronize()
    return t.double().cpu().numpy()


def _whole(T, K, seed):
    """Small whole numbers whose codes are themselves: sums below 2^8 are exact in bf16, so results are compared for equality."""
    import torch
    x = np.zeros((T, K), np.float32)
    rng = np.random.default_rng([5, seed])
    x[np.arange(T), rng.integers(0, K, T)] = rng.integers(1, 9, T)
    return x, torch.from_numpy(x).to(torch.bfloat16).cuda()


def test_a_bias_tensor_stays_its_callers():
    """Two layers made from one bias on the device, one of them trained on; the tensor changed in place between; a parameter."""
    import torch
    bsp = _bsp()
    W = np.eye(128, dtype=np.float32)
    x, t = _whole(3, 128, 1)
    b = torch.full((128,), 2.0, device="cuda")
    one, two = bsp.BspLayerF8(W, bias=b), bsp.BspLayerF8(W, bias=b)
    one.update(W, bias=torch.full((128,), 5.0, device="cuda"))
    assert (_host(b) == 2).all()
    assert (_host(one.fc(t)) == x + 5).all() and (_host(two.fc(t)) == x + 2).all()
    b.fill_(9.0)
    assert (_host(two.fc(t)) == x + 2).all()
    p = torch.nn.Parameter(torch.full((128,), 3.0, device="cuda"))
    layer = bsp.BspLayerF8(W, bias=p)
    assert (_host(layer.fc(t)) == x + 3).all()
    layer.update(W, bias=torch.full((128,), 4.0, device="cuda"))
    assert (_host(p.detach()) == 3).all() and (_host(layer.fc(t)) == x + 4).all()


def test_biases_of_other_places_and_types():
    """numpy in 32 and 64 bits, a list, a bf16 tensor, every second element of one, a host tensor."""
    import torch
    bsp = _bsp()
    W = np.eye(128, dtype=np.float32)
    x, t = _whole(2, 128, 2)
    v = np.arange(128) % 16
    for b in (v.astype(np.float32), v.astype(np.float64), [float(k) for k in v], torch.from_numpy(v).to(torch.bfloat16).cuda(),
              torch.from_numpy(np.repeat(v, 2).astype(np.float32)).cuda()[::2], torch.from_numpy(v.astype(np.float32))):
        assert (_host(bsp.BspLayerF8(W, bias=b).fc(t)) == x + v).all()


def test_new_biases_are_refused_or_taken_whole():
    """A bias of another shape, or one for a layer that has none, is an error that names it; the layer stays as it was."""
    import torch
    bsp = _bsp()
    W = np.eye(128, dtype=np.float32)
    x, t = _whole(2, 128, 3)
    layer = bsp.BspLayerF8(W, bias=np.full(128, 2.0, np.float32))
    for b in (torch.ones(1, device="cuda"), torch.tensor(1.0, device="cuda"), [1.0], torch.ones(1, 128, device="cuda"), np.ones(127, np.float32)):
        with pytest.raises(AssertionError, match="bias"):
            layer.update(2 * W, bias=b)
        assert (_host(layer.fc(t)) == x + 2).all()
    for b in (np.arange(128, dtype=np.float64) % 8, torch.arange(128, device="cuda") % 8):
        layer.update(2 * W, bias=b)
        assert (_host(layer.fc(t)) == 2 * x + np.arange(128) % 8).all()
    plain = bsp.BspLayerF8(W)
    with pytest.raises(AssertionError, match="bias"):
        plain.update(2 * W, bias=np.ones(128, np.float32))
    assert (_host(plain.fc(t)) == x).all()
    for wrong in (np.ones((127, 128), np.float32), torch.ones(128, 128, device="cuda", dtype=torch.float64)):  # no half of an update
        with pytest.raises(AssertionError):
            layer.update(wrong, bias=np.full(128, 7.0, np.float32))
        assert (_host(layer.fc(t)) == 2 * x + np.arange(128) % 8).all()


def test_a_checkpoint_given_is_of_the_type_asked_for():
    """save8 into a BspCodes: its own type where none is asked for, an error where another is, nothing written."""
    import torch
    bsp = _bsp()
    t = torch.randn(5, 200, device="cuda")
    for have, other in (("e4m3", "e5m2"), ("e5m2", "e4m3")):
        c = bsp.BspCodes(5, 200, have)
        c.buffer.fill_(77)
        with pytest.raises(AssertionError, match=have):
            bsp.save8(t, other, out=c)
        assert bool((c.buffer == 77).all())
        want = bsp.save8(t, have)
        for got in (bsp.save8(t, out=c), bsp.save8(t, have, out=c)):
            assert got is c and torch.equal(c.codes, want.codes) and torch.equal(c.scale, want.scale)
    assert bsp.save8(t).kind == "e4m3"


def test_a_graph_that_is_not_recorded_is_said_to_be():
    """No call records what autograd needs: a tensor that requires a gradient is taken with a warning, under no_grad without, with the same results."""
    import warnings
    import torch
    bsp = _bsp()
    rng = np.random.default_rng(9)
    layer = bsp.BspLayerF8(rng.standard_normal((130, 256)).astype(np.float32), bias=rng.standard_normal(130).astype(np.float32))
    x, dy, r = (torch.randn(20, n, device="cuda").to(torch.bfloat16) for n in (256, 130, 130))
    w, b = torch.ones(256, device="cuda"), torch.zeros(256, device="cuda")
    codes = bsp.save8(x)
    _, mean, rstd = bsp.layer_norm(x, w, b)
    calls = {  # what may require a gradient, and the call
        "save8": ([x], lambda x: bsp.save8(x).load()),
        "fc": ([x, r], lambda x, r: layer.fc(x, residual=r)),
        "grad_input": ([dy], lambda dy: layer.grad_input(dy)),
        "grad_weight": ([dy], lambda dy: layer.grad_weight(dy, codes)),
        "layer_norm": ([x, w, b], lambda x, w, b: bsp.layer_norm(x, w, b)),
        "layer_norm_grad": ([torch.randn_like(x), x, w], lambda d, x, w: bsp.layer_norm_grad(d, x, mean, rstd, w)),
    }
    listed = lambda v: list(v) if isinstance(v, tuple) else [v]  # noqa: E731
    for name, (given, call) in calls.items():
        with warnings.catch_warnings():
            warnings.simplefilter("error")
            want = listed(call(*given))
        for k in range(len(given)):
            some = [t.clone().requires_grad_() if i == k else t for i, t in enumerate(given)]
            with pytest.warns(UserWarning, match="autograd"):
                got = listed(call(*some))
            with warnings.catch_warnings(), torch.no_grad():
                warnings.simplefilter("error")
                again = listed(call(*some))
            assert all(torch.equal(g, v) and torch.equal(a, v) and not g.requires_grad for g, a, v in zip(got, again, want)), (name, k)
    with warnings.catch_warnings():  # new weights are taken as values, as an optimiser's are
        warnings.simplefilter("error")
        layer.update(torch.nn.Parameter(torch.randn(130, 256, device="cuda")), bias=torch.nn.Parameter(torch.randn(130, device="cuda")))


@pytest.mark.parametrize("T", [3, 20, 60])
def test_rows_of_the_smallest_values(T):
    """fp32 results and the weights' gradient take codes as bf16: whole multiples of 2^-133 exactly, and of a value between them no
    more than 2^-133 is lost.  Rows of one value and one much smaller; weights of 2^60, so that results are ordinary numbers."""
    import torch
    bsp = _bsp()
    W = np.full((130, 128), 2.0 ** 60, np.float32)
    layer = bsp.BspLayerF8(W)
    for small, lost in ((1.0, 0.0), (5.0, 0.0), (0.75, 1.0)):
        x = torch.zeros(T, 128)
        x[:, 3], x[:, 77] = 2.0 ** -127, small * 2.0 ** -133
        c = bsp.save8(x.cuda(), "e4m3")
        values = _host(c.load(torch.float32))
        assert (values == x.double().numpy()).all()
        ref = values.sum(1)[:, None] * 2.0 ** 60
        assert (np.abs(_host(layer.fc(c, dtype=torch.float32)) - ref) <= lost * 2.0 ** -73 + 2.0 ** -24 * ref).all()
        dy = torch.full((T, 130), 2.0 ** 60, dtype=torch.bfloat16, device="cuda")
        dW, _ = layer.grad_weight(dy, c)
        want = T * values[0] * 2.0 ** 60
        assert (np.abs(_host(dW) - want) <= T * lost * 2.0 ** -73 + (T + 8) * 2.0 ** -24 * want).all()
