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
