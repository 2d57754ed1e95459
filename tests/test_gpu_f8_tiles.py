"""Every tile of the 8-bit products and every shape of the weights' gradient, on ordinary data, with the kernel that ran named: many
steps, shares and ranges, ragged rows and channels, masks, gates, residuals, both types of codes and of results.

The references are sums in 64 bits on the GPU.  Weights are whole numbers up to 15 times a power of two for each block: their codes are
themselves.  What the activations' codes stand for is read back from a checkpoint (test_gpu_f8.py holds that to the oracle).
Bounds as there: a bf16 result is rounded once, 2^-8 of its value, and its products lose less than 2^-10 of the sum of their magnitudes S;
an fp32 result adds n terms in some order, at most (n + 8) 2^-24 S, as the gradients' sums over T rows do.
"""
import pytest

from gpu_util import kernels_of

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
TILES = {"256x256": "<4, 2, 2, 4, 2,", "128x256": "<4, 2, 1, 4, 3,", "128x128": "<2, 2, 2, 2, 2,", "128x64": "<2, 1, 2, 2, 3,", "128x32": "<1, 1, 4, 1, 4,"}


def _blocks(n):
    return -(-n // 128)


def _gen(*key):
    import zlib
    import torch
    return torch.Generator(device="cuda").manual_seed(zlib.crc32(repr(key).encode()))


def _weights(gen, O, I, density):
    """(W, mask of blocks, W under the mask in 64 bits)."""
    import torch
    W = torch.randint(-15, 16, (O, I), generator=gen, device="cuda").float()
    size = torch.exp2(torch.randint(-9, -3, (_blocks(O), _blocks(I)), generator=gen, device="cuda").float())
    W *= size.repeat_interleave(128, 0).repeat_interleave(128, 1)[:O, :I]
    gamma = (torch.rand(_blocks(O), _blocks(I), generator=gen, device="cuda") < density).to(torch.uint8)
    keep = gamma.repeat_interleave(128, 0).repeat_interleave(128, 1)[:O, :I]
    return W, gamma, W.double() * keep


def _rows(gen, T, K):
    """Rows of differing size, some channels much larger than the others, in bf16."""
    import torch
    x = torch.randn(T, K, generator=gen, device="cuda") * torch.exp(torch.randn(T, 1, generator=gen, device="cuda"))
    return (x * torch.where(torch.rand(K, generator=gen, device="cuda") < 0.02, 20.0, 1.0)).to(torch.bfloat16)


def _into(T, width, dtype):
    """(out [T][width] of NaN, the whole buffer that it lies at the start of)."""
    import torch
    buffer = torch.full((T * width + 512,), float("nan"), device="cuda", dtype=dtype)
    return buffer[:T * width].view(T, width), buffer


def _near(out, buffer, ref, S, n):
    """Within the bound, nothing past the end."""
    import torch
    f32 = out.dtype == torch.float32
    tol = (n + 8) * U * S if f32 else 2.0 ** -8 * ref.abs() + 2.0 ** -10 * S + 2.0 ** -133
    ratio = ((out.double() - ref).abs() / tol.clamp_min(2.0 ** -140)).max()
    assert float(ratio) <= 1.0, float(ratio)  # (a NaN fails too)
    assert bool(buffer[out.numel():].isnan().all())


PRODUCTS = [
    # tile, T, contraction, channels, density (which the tile is chosen by: rows, and the kept blocks a block row)
    ("256x256", 4100, 300, 1990, 1.0), ("256x256", 2085, 9400, 4090, 1.0),
    ("128x256", 3001, 1152, 3960, 1.0), ("128x256", 8200, 300, 500, 0.6), ("128x256", 2085, 16000, 2048, 0.6), ("128x256", 3000, 1000, 2990, 0.5),
    ("128x128", 8200, 300, 130, 1.0), ("128x128", 700, 2000, 4003, 0.5), ("128x128", 8200, 9400, 130, 1.0), ("128x128", 517, 4100, 4004, 1.0),
    ("128x64", 4100, 300, 130, 1.0), ("128x64", 4100, 16000, 130, 0.7), ("128x64", 1030, 9100, 130, 0.6),
    ("128x32", 700, 9400, 1000, 1.0), ("128x32", 700, 16000, 1003, 0.6), ("128x32", 390, 9100, 264, 1.0),
]
PRODUCTS_F32 = [
    ("128x128", 8200, 300, 130, 0.6), ("128x128", 700, 2000, 4003, 1.0), ("128x128", 8200, 9400, 130, 1.0), ("128x128", 2085, 16000, 2048, 0.6),
    ("128x128", 2085, 9100, 130, 0.6), ("128x128", 700, 9400, 1000, 1.0),
    ("128x64", 4100, 300, 130, 1.0), ("128x64", 1030, 4100, 130, 0.6),
    ("128x32", 45, 4100, 1030, 1.0), ("128x32", 70, 2000, 1003, 0.6),
]


def _both(rows, rows_f32):
    return [(*r, "bf16") for r in rows] + [(*r, "f32") for r in rows_f32]


@pytest.mark.parametrize("kind", ["e4m3", "e5m2"])
@pytest.mark.parametrize("tile,T,I,O,density,dtype", _both(PRODUCTS, PRODUCTS_F32))
def test_tiles_of_the_product(tile, T, I, O, density, dtype, kind):
    """The layer: bias and relu, then a residual too."""
    import torch
    import paper_2407_09453_amd as bsp
    gen = _gen(T, I, O, kind)
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    W, gamma, Wq = _weights(gen, O, I, density)
    b = torch.randn(O, generator=gen, device="cuda")
    layer = bsp.BspLayerF8(W, gamma, bias=b)
    codes = bsp.save8(_rows(gen, T, I), kind)
    x, Wt = codes.load(torch.float32).double(), Wq.t().contiguous()
    y, S = x @ Wt + b, x.abs() @ Wt.abs() + b.abs()
    del x, Wt, Wq
    out, buffer = _into(T, O, dt)
    ran = kernels_of(lambda: layer.fc(codes, relu=True, out=out))
    name = "f8_wide" + TILES[tile] + (" true" if kind == "e5m2" else " false") + (", true>" if dtype == "f32" else ", false>")
    assert any(name in k for k in ran), ran
    _near(out, buffer, y.relu(), S, I)
    r = torch.randn(T, O, generator=gen, device="cuda").to(dt)
    out, buffer = _into(T, O, dt)
    layer.fc(codes, relu=True, residual=r, out=out)
    _near(out, buffer, (y + r.double()).relu(), S + r.double().abs(), I)
    if kind == "e4m3":  # the rows as values become the same codes: the same bits
        t = codes.load()
        assert torch.equal(layer.fc(t, relu=True, residual=r, dtype=dt), out)


@pytest.mark.parametrize("kind", ["e4m3", "e5m2"])
@pytest.mark.parametrize("tile,T,O,I,density,dtype", _both(PRODUCTS, PRODUCTS_F32))
def test_tiles_of_the_input_gradient(tile, T, O, I, density, dtype, kind):
    """The transposed product, O its contraction: without a gate, and through one of the other type of codes."""
    import torch
    import paper_2407_09453_amd as bsp
    gen = _gen(T, I, O, kind, 2)
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    W, gamma, Wq = _weights(gen, O, I, density)
    layer = bsp.BspLayerF8(W, gamma)
    codes = bsp.save8(_rows(gen, T, O), kind)
    dy = codes.load(torch.float32).double()
    dx, S = dy @ Wq, dy.abs() @ Wq.abs()
    del dy, Wq
    out, buffer = _into(T, I, dt)
    ran = kernels_of(lambda: layer.grad_input(codes, out=out))
    name = "f8_wide" + TILES[tile] + (" true" if kind == "e5m2" else " false") + (", true>" if dtype == "f32" else ", false>")
    assert any(name in k for k in ran), ran
    _near(out, buffer, dx, S, O)
    gate = bsp.save8(_rows(gen, T, I).relu(), "e5m2" if kind == "e4m3" else "e4m3")
    opened = gate.load(torch.float32) > 0
    assert 0.2 < float(opened.float().mean()) < 0.6
    out, buffer = _into(T, I, dt)
    layer.grad_input(codes, relu_of=gate, out=out)
    _near(out, buffer, dx * opened, S, O)
    assert bool((out[~opened] == 0).all())


@pytest.mark.parametrize("T", [1, 16, 17, 20, 32])
@pytest.mark.parametrize("O,I,density", [(4100, 520, 0.6), (16400, 130, 1.0)])
def test_few_rows_in_fp32_through_a_gate(T, O, I, density):
    """Also a contraction so long that its sums are shared out."""
    import torch
    import paper_2407_09453_amd as bsp
    gen = _gen(T, I, O, 3)
    W, gamma, Wq = _weights(gen, O, I, density)
    layer = bsp.BspLayerF8(W, gamma)
    gate = bsp.save8(_rows(gen, T, I).relu())
    opened = gate.load(torch.float32) > 0
    for kind in ("e4m3", "e5m2"):
        codes = bsp.save8(_rows(gen, T, O), kind)
        dy = codes.load(torch.float32).double()
        out, buffer = _into(T, I, torch.float32)
        layer.grad_input(codes, relu_of=gate, out=out)
        _near(out, buffer, (dy @ Wq) * opened, dy.abs() @ Wq.abs(), O)


@pytest.mark.parametrize("T", [17, 20, 31, 32, 33, 64])
def test_rows_as_values_give_the_bits_of_their_codes(T):
    """More rows than become codes inside the product's kernel: the same kernel on the same codes."""
    import torch
    import paper_2407_09453_amd as bsp
    gen = _gen(T, 4)
    W, gamma, _ = _weights(gen, 1000, 2100, 0.6)
    layer = bsp.BspLayerF8(W, gamma, bias=torch.randn(1000, generator=gen, device="cuda"))
    t = _rows(gen, T, 2100)
    for dt in (torch.bfloat16, torch.float32):
        assert torch.equal(layer.fc(t, dtype=dt), layer.fc(bsp.save8(t), dtype=dt))


GRADIENTS = [
    # blocks and waves a workgroup, ranges of rows or one; T, I, O, density
    ("<1, 4,", False, 1003, 4090, 2981, 0.5), ("<1, 4,", False, 1500, 4090, 2990, 0.4), ("<1, 4,", False, 1003, 4090, 4003, 0.4), ("<1, 4,", False, 1024, 4096, 4096, 0.4),
    ("<2, 4,", False, 1003, 8100, 4003, 0.5), ("<2, 4,", False, 1003, 6000, 8100, 0.6), ("<2, 4,", False, 1003, 4000, 2000, 1.0), ("<2, 4,", False, 387, 4090, 8003, 0.4),
    ("<4, 8,", False, 1003, 4090, 4090, 1.0), ("<4, 8,", False, 999, 3000, 3000, 1.0), ("<4, 8,", False, 387, 8190, 4003, 1.0), ("<4, 8,", False, 1056, 4096, 4096, 1.0),
    ("<1, 8,", False, 1000, 2000, 1300, 1.0), ("<1, 8,", False, 515, 1000, 1999, 0.9), ("<1, 8,", False, 1030, 2000, 1303, 1.0), ("<1, 8,", False, 1060, 2000, 1305, 1.0),
    ("<1, 8,", False, 1120, 2000, 1299, 1.0),
    ("<1, 8,", True, 2011, 1000, 2007, 1.0), ("<1, 8,", True, 2011, 2000, 2007, 0.35), ("<1, 8,", True, 5001, 500, 700, 1.0), ("<1, 8,", True, 5001, 120, 130, 1.0),
    ("<1, 8,", True, 1111, 200, 5, 1.0), ("<1, 8,", True, 3333, 300, 500, 0.7),
]


@pytest.mark.parametrize("kind", ["e4m3", "e5m2"])
@pytest.mark.parametrize("shape,ranges,T,I,O,density", GRADIENTS)
def test_shapes_of_the_weight_gradient(shape, ranges, T, I, O, density, kind):
    """Eight steps of 32 rows and more in every range, so that the loop moves on through the rows."""
    import torch
    import paper_2407_09453_amd as bsp
    gen = _gen(T, I, O, kind, 5)
    W, gamma, _ = _weights(gen, O, I, density)
    layer = bsp.BspLayerF8(W, gamma)
    codes = bsp.save8(_rows(gen, T, I), kind)
    dy = _rows(gen, T, O)
    out, buffer = _into(O, I, torch.float32)
    ran = kernels_of(lambda: layer.grad_weight(dy, codes, out=out))
    name = "f8_grad" + shape + (" true," if kind == "e5m2" else " false,") + (" true>" if O < 8 else " false>")
    assert any(name in k for k in ran) and any("f8_grad_finish" in k for k in ran) == ranges, ran
    out.fill_(float("nan"))
    _, db = layer.grad_weight(dy, codes, out=out)
    x, d = codes.load(torch.float32).double(), dy.double().t().contiguous()
    keep = gamma.repeat_interleave(128, 0).repeat_interleave(128, 1)[:O, :I].bool()
    S = d.abs() @ x.abs()
    _near(out, buffer, (d @ x) * keep, S, T)
    assert bool((out[~keep] == 0).all())
    assert bool(((db - d.sum(1)).abs() <= (T + 8) * U * d.abs().sum(1)).all())
