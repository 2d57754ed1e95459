"""What the calls of norm, adapters and log probabilities say where an input requires a gradient: on the current stream, on one given by handle."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu


def _cases():
    """(name, call, its tensors that may require a gradient)."""
    import torch
    import paper_2407_09453_amd as bsp
    X, Y, R, w = torch.randn(8, 256, device="cuda"), torch.randn(8, 128, device="cuda"), torch.randn(8, 128, device="cuda"), torch.ones(256, device="cuda")
    layer = bsp.BspLayerF8(torch.randn(128, 256, device="cuda"))
    bank, requests = bsp.BspAdapters(2, 4, 256, 128), bsp.BspRequests(np.arange(8) % 2, 2)
    tok = torch.arange(8, device="cuda")
    _, _, rstd = bsp.rms_norm(X, w)
    _, lse, entropy, _, _ = bsp.log_probs(X, tok)
    d = torch.ones(8, device="cuda")
    both = dict(adapters=bank, requests=requests)
    return [
        ("rms_norm", lambda X, w, r, **k: bsp.rms_norm(X, w, r, **k), [X, w, X.clone()]),
        ("rms_norm_grad", lambda dY, H, w, dH, **k: bsp.rms_norm_grad(dY, H, rstd, w, dH, **k), [X, X.clone(), w, X.clone()]),
        ("log_probs", lambda X, **k: bsp.log_probs(X, tok, **k), [X]),
        ("log_probs_grad", lambda X, dl, dh, **k: bsp.log_probs_grad(X, tok, lse, entropy, dl, dh, **k), [X, d, d.clone()]),
        ("fc", lambda X, r, **k: layer.fc(X, residual=r, **both, **k), [X, R]),
        ("grad_input", lambda dY, **k: layer.grad_input(dY, **both, **k), [Y]),
        ("adapters' grad", lambda dY, X, **k: bank.grad(dY, X, requests, **k), [Y.bfloat16(), X.bfloat16()]),
    ]


@pytest.mark.parametrize("where", ["here", "own", "side"])
def test_autograd_is_told(where):
    import warnings
    import torch
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    at = {"here": {}, "own": {"stream": torch.cuda.current_stream().cuda_stream}, "side": {"stream": side.cuda_stream}}[where]
    for name, call, tensors in _cases():
        torch.cuda.synchronize()
        with warnings.catch_warnings():
            warnings.simplefilter("error")
            call(*tensors, **at)
            with torch.no_grad():
                call(*(t.clone().requires_grad_() for t in tensors), **at)
        for i in range(len(tensors)):
            given = [t.detach().clone().requires_grad_(k == i) for k, t in enumerate(tensors)]
            torch.cuda.synchronize()
            with warnings.catch_warnings(record=True) as said:
                warnings.simplefilter("always")
                call(*given, **at)
            assert any("records nothing" in str(s.message) for s in said), (name, i, where)
    torch.cuda.synchronize()
