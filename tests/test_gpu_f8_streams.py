"""Calls of the 8-bit layers with an explicit stream: the other stream's work is held up by a kernel that spins, and what either
stream reads and writes is compared with the results of calls one after the other."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu
HELD = 10_000_000  # clocks of the spinning kernel: some milliseconds, the calls below take microseconds


def _bsp():
    import paper_2407_09453_amd as bsp
    return bsp


def _flat(v):
    """Clones of a result's tensors, of a checkpoint its codes and the scales of its rows."""
    if isinstance(v, tuple):
        return [t for x in v for t in _flat(x)]
    if isinstance(v, _bsp().BspCodes):
        return [v.codes.clone(), v.scale[:, :v.T].clone()]
    return [v.clone()]


def _buffers(v):
    if isinstance(v, tuple):
        return [t for x in v for t in _buffers(x)]
    return [v.buffer if isinstance(v, _bsp().BspCodes) else v]


@pytest.fixture(scope="module")
def calls():
    """Name -> (call with stream=, bytes of the workspaces that it takes)."""
    import torch
    bsp = _bsp()
    gen = torch.Generator(device="cuda")
    gen.manual_seed(11)
    T, I, O = 700, 1024, 640
    draw = lambda *s: torch.randn(*s, generator=gen, device="cuda")  # noqa: E731
    layer = bsp.BspLayerF8(draw(O, I) / 32, bias=draw(O))
    x, dy, w = draw(T, I).to(torch.bfloat16), draw(T, O).to(torch.bfloat16), draw(I)
    codes = bsp.save8(x)
    long = bsp.BspLayerF8(draw(128, 16384) / 128)  # few outputs of a long contraction: shares
    xs = bsp.save8(draw(40, 16384).to(torch.bfloat16))
    _, mean, rstd = bsp.layer_norm(x, w)
    some = bsp.BspLayerF8(draw(128, 256) / 16)  # few blocks: ranges of rows
    dy2, x2 = draw(4096, 128).to(torch.bfloat16), bsp.save8(draw(4096, 256).to(torch.bfloat16))
    torch.cuda.synchronize()
    norm_bytes = __import__("paper_2407_09453_amd.f8", fromlist=["f8"])._norm_bytes(T, I)
    return {
        "fc": (lambda **k: layer.fc(x, relu=True, **k), layer._bytes(0, T)),
        "fc, shares": (lambda **k: long.fc(xs, **k), long._bytes(1, 40)),
        "fc of codes": (lambda **k: layer.fc(codes, dtype=torch.float32, **k), 0),
        "grad_input": (lambda **k: layer.grad_input(dy, relu_of=codes, **k), layer._bytes(2, T)),
        "grad_weight": (lambda **k: some.grad_weight(dy2, x2, **k), some._bytes("grad", 4096)),
        "save8": (lambda **k: bsp.save8(x, **k), 0),
        "load": (lambda **k: codes.load(**k), 0),
        "layer_norm": (lambda **k: bsp.layer_norm(x, w, **k), 0),
        "layer_norm to codes": (lambda **k: bsp.layer_norm(x, w, code="e4m3", **k), 0),
        "layer_norm_grad": (lambda **k: bsp.layer_norm_grad(x, x, mean, rstd, w, **k), norm_bytes),
    }


NAMES = ["fc", "fc, shares", "fc of codes", "grad_input", "grad_weight", "save8", "load", "layer_norm", "layer_norm to codes", "layer_norm_grad"]


@pytest.mark.parametrize("name", NAMES)
def test_blocks_that_wait_elsewhere_are_not_written(calls, name):
    """Blocks of the call's sizes are dropped in the current stream while a copy of them is still to come there; the call, in a
    stream that is free, writes its workspace and results meanwhile."""
    import torch
    call, ws = calls[name]
    s = torch.cuda.Stream()
    want = _flat(call())
    sizes = [t.numel() * t.element_size() for t in _buffers(call(stream=s.cuda_stream))] + [ws] * (ws > 0)
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    blocks = [torch.full((n,), 91, dtype=torch.uint8, device="cuda") for n in sizes for _ in range(2)]
    at = [b.data_ptr() for b in blocks]
    copies = [torch.empty_like(b) for b in blocks]
    torch.cuda.synchronize()
    torch.cuda._sleep(HELD)
    for b, c in zip(blocks, copies):
        c.copy_(b)
    del b, blocks
    got = call(stream=s.cuda_stream)
    assert not {t.data_ptr() for t in _buffers(got)} & set(at)
    s.synchronize()
    torch.cuda.synchronize()
    assert all(bool((c == 91).all()) for c in copies)
    assert all(torch.equal(a, b) for a, b in zip(_flat(got), want))


@pytest.mark.parametrize("name", NAMES)
def test_results_may_be_dropped_behind_their_use(calls, name):
    """A result read in the current stream, which waited for it, and dropped before the read is done: the next call in the other
    stream writes another block."""
    import torch
    call, _ = calls[name]
    want = _flat(call())
    s = torch.cuda.Stream()
    call(stream=s.cuda_stream)
    torch.cuda.synchronize()
    got = call(stream=s.cuda_stream)
    torch.cuda.current_stream().wait_stream(s)
    torch.cuda._sleep(HELD)
    read = _flat(got)
    at = {t.data_ptr() for t in _buffers(got)}
    del got
    again = call(stream=s.cuda_stream)
    assert not at & {t.data_ptr() for t in _buffers(again)}
    for t in _buffers(again):
        t.record_stream(s)
        with torch.cuda.stream(s):
            t.zero_()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(read, want))


def test_what_calls_of_a_stream_pass_on_may_be_dropped():
    """Codes, results and workspaces that calls in a stream made and others there read, dropped while the stream has it all to do."""
    import torch
    bsp = _bsp()
    gen = torch.Generator(device="cuda")
    gen.manual_seed(12)
    draw = lambda *s: torch.randn(*s, generator=gen, device="cuda")  # noqa: E731
    layer, back = bsp.BspLayerF8(draw(512, 768) / 28, bias=draw(512)), bsp.BspLayerF8(draw(768, 512) / 22)
    x, r, dy = draw(300, 768).to(torch.bfloat16), draw(300, 512).to(torch.bfloat16), draw(300, 512).to(torch.bfloat16)

    def chain(**k):
        n, mean, rstd = bsp.layer_norm(x, code="e4m3", **k)
        y = layer.fc(n, residual=r, relu=True, **k)
        z = back.fc(bsp.save8(y, **k), **k)
        dx = layer.grad_input(dy, relu_of=bsp.save8(z, **k), **k)
        return z, layer.grad_weight(dy, n, **k), bsp.layer_norm_grad(dx, x, mean, rstd, **k)
    want = _flat(chain())
    s = torch.cuda.Stream()
    sizes = [300 * 768 * 2, 300 * 512 * 2, bsp.BspCodes(300, 768).buffer.numel(), bsp.BspCodes(300, 512).buffer.numel(), 2 * 300 * 4, layer._bytes("grad", 300)]
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        torch.cuda._sleep(HELD)
    got = chain(stream=s.cuda_stream)
    litter = [torch.full((n,), 255, dtype=torch.uint8, device="cuda") for n in sizes for _ in range(4)]  # takes what was dropped, where it can
    torch.cuda.synchronize()
    assert all(torch.equal(a, w) for a, w in zip(_flat(got), want)) and len(litter) == 24


def test_a_stream_may_go_before_what_it_worked_on():
    """A stream that is not torch's, destroyed by its owner when its work is done: inputs, layer and results are freed later."""
    import ctypes
    import torch
    bsp = _bsp()
    torch.cuda.synchronize()
    hip = ctypes.CDLL(bsp.lib_path())  # (the runtime that the library itself is linked to)
    x = torch.randn(700, 512, device="cuda").to(torch.bfloat16)
    layer = bsp.BspLayerF8(torch.randn(640, 512, device="cuda"))
    want = layer.fc(x)
    W = torch.randn(640, 512, device="cuda")
    torch.cuda.synchronize()
    h = ctypes.c_void_p()
    assert hip.hipStreamCreate(ctypes.byref(h)) == 0
    codes = bsp.save8(x, stream=h.value)
    y = layer.fc(codes, stream=h.value)
    layer.update(W, stream=h.value)
    assert hip.hipStreamSynchronize(h) == 0 and hip.hipStreamDestroy(h) == 0
    assert torch.equal(y, want)
    del x, layer, W, codes, y
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    assert torch.equal(torch.ones(1000, device="cuda") + 1, torch.full((1000,), 2.0, device="cuda"))


def test_the_default_streams_handle():
    """0 is the default stream, also where another one is current."""
    import torch
    bsp = _bsp()
    x = torch.randn(90, 256, device="cuda").to(torch.bfloat16)
    layer = bsp.BspLayerF8(torch.randn(130, 256, device="cuda"))
    want = layer.fc(x)
    torch.cuda.synchronize()
    t = torch.empty_like(x)
    with torch.cuda.stream(torch.cuda.Stream()):
        torch.cuda.default_stream().synchronize()
        with torch.cuda.stream(torch.cuda.default_stream()):
            torch.cuda._sleep(HELD)
            t.copy_(x)  # in the default stream: the call has to come behind it
        y = layer.fc(t, stream=0)
        torch.cuda.synchronize()
    assert torch.equal(y, want)
    assert torch.equal(layer.fc(x, stream=torch.cuda.current_stream().cuda_stream), want)


def test_in_a_graph_with_a_fork():
    """A capture that forks to a second stream, calls there by handle, and joins."""
    import torch
    bsp = _bsp()
    gen = torch.Generator(device="cuda")
    gen.manual_seed(13)
    x = torch.randn(130, 512, generator=gen, device="cuda").to(torch.bfloat16)
    one, two = (bsp.BspLayerF8(torch.randn(384, 512, generator=gen, device="cuda") / 22) for _ in range(2))
    s = torch.cuda.Stream()

    def step(stream):
        if stream is None:
            return one.fc(x), two.fc(bsp.save8(x))
        here = torch.cuda.current_stream()
        s.wait_stream(here)
        a = two.fc(bsp.save8(x, stream=stream), stream=stream)
        b = one.fc(x)
        here.wait_stream(s)
        return b, a
    step(None), step(s.cuda_stream)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        got = step(s.cuda_stream)
    for k in range(3):
        x.copy_(torch.randn(130, 512, generator=gen, device="cuda").to(torch.bfloat16))
        for o in got:
            o.fill_(float("nan"))
        want = step(None)
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_two_host_threads():
    """Two threads, a stream each, the same layer: each gets the results of its own calls."""
    import threading
    import torch
    bsp = _bsp()
    gen = torch.Generator(device="cuda")
    gen.manual_seed(14)
    layer = bsp.BspLayerF8(torch.randn(640, 512, generator=gen, device="cuda") / 22)
    xs = [[torch.randn(T, 512, generator=gen, device="cuda").to(torch.bfloat16) for T in (1, 33, 200, 700)] for _ in range(2)]
    dys = [[torch.randn(x.shape[0], 640, generator=gen, device="cuda").to(torch.bfloat16) for x in row] for row in xs]

    def step(x, dy):
        c = bsp.save8(x)
        return [layer.fc(x), layer.fc(c), layer.grad_input(dy, relu_of=c), *layer.grad_weight(dy, c)]
    want = [[step(x, dy) for x, dy in zip(a, b)] for a, b in zip(xs, dys)]
    torch.cuda.synchronize()
    got, errors = [None, None], []

    def work(i):
        try:
            with torch.cuda.stream(torch.cuda.Stream()) as _:
                for _ in range(20):
                    got[i] = [step(x, dy) for x, dy in zip(xs[i], dys[i])]
                torch.cuda.current_stream().synchronize()
        except Exception as e:  # (a thread's exception is not the test's)
            errors.append(e)
    threads = [threading.Thread(target=work, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert not errors
    for i in range(2):
        for a, b in zip(got[i], want[i]):
            assert all(torch.equal(p, q) for p, q in zip(a, b))


def test_new_weights_and_bias_in_a_stream():
    """update() with a stream puts the bias there too: a call behind it in that stream has both while the current stream is held,
    and one before it has neither."""
    import torch
    bsp = _bsp()
    gen = torch.Generator(device="cuda")
    gen.manual_seed(15)
    draw = lambda *s: torch.randn(*s, generator=gen, device="cuda")  # noqa: E731
    W, b, W2, b2, x = draw(384, 256), draw(384), draw(384, 256), draw(384), draw(60, 256).to(torch.bfloat16)
    old, new = bsp.BspLayerF8(W, bias=b).fc(x), bsp.BspLayerF8(W2, bias=b2).fc(x)
    layer = bsp.BspLayerF8(W, bias=b)
    s = torch.cuda.Stream()
    for _ in range(2):  # the first turn warms up
        layer.update(W, bias=b)
        Wc, bc = W2.clone(), b2.clone()
        torch.cuda.synchronize()
        torch.cuda._sleep(HELD)
        with torch.cuda.stream(s):
            torch.cuda._sleep(HELD // 4)
        first = layer.fc(x, stream=s.cuda_stream)
        layer.update(Wc, bias=bc, stream=s.cuda_stream)
        second = layer.fc(x, stream=s.cuda_stream)
        s.synchronize()
        with torch.cuda.stream(s):  # (where the results are ready)
            got = torch.equal(first, old), torch.equal(second, new)
        torch.cuda.synchronize()
    assert got == (True, True)
    layer.update(W.cpu(), bias=b.cpu().numpy(), stream=s.cuda_stream)
    y = layer.fc(x, stream=s.cuda_stream)
    s.synchronize()
    assert torch.equal(y, old)


def test_the_current_stream_is_the_callers_afterwards():
    """Also behind a call that is refused, and no other stream's handle is left current."""
    import torch
    bsp = _bsp()
    layer, x = bsp.BspLayerF8(torch.randn(256, 128, device="cuda")), torch.randn(3, 128, device="cuda")
    s, t = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    for here in (torch.cuda.default_stream(), t):
        with torch.cuda.stream(here):
            layer.fc(x, stream=s.cuda_stream)
            assert torch.cuda.current_stream() == here
            with pytest.raises(AssertionError):
                layer.fc(x[:, :100], stream=s.cuda_stream)
            assert torch.cuda.current_stream() == here and torch.cuda.current_device() == 0
    torch.cuda.synchronize()
