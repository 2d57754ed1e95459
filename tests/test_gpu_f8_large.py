"""Layer norm and checkpoints of so many rows or columns that one dimension of a launch does not hold their threads.  The inputs are one
row, or a few, repeated (a row stride of zero), so every row's result is that of a small call."""
import pytest

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


def _needs(gib):
    import torch
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < gib * 2 ** 30:
        pytest.skip("needs %d GiB" % gib)


def _all_rows_are(t, row):
    import torch
    lo, hi = t[0].clone(), t[0].clone()
    for i in range(0, t.shape[0], 1 << 24):
        lo, hi = torch.minimum(lo, t[i:i + (1 << 24)].amin(0)), torch.maximum(hi, t[i:i + (1 << 24)].amax(0))
    return torch.equal(lo, row) and torch.equal(hi, row)


@pytest.mark.parametrize("T,D,codes,gib", [((1 << 24) + 5, 4, False, 2), ((1 << 28) + 3, 8, False, 12), ((1 << 26) + 2, 264, True, 30),
                                           ((1 << 24) + 1, 1032, False, 38), ((1 << 23) + 1, 4104, True, 42), ((1 << 22) + 3, 8200, False, 72)])
def test_norm_of_many_rows(T, D, codes, gib):
    """Fewer than eight columns; sixteen rows, four rows, one row a workgroup; workgroups of 512 and 1024 threads."""
    import torch
    import paper_2407_09453_amd as bsp
    _needs(gib)
    x = torch.randn(1, D, device="cuda").to(torch.bfloat16)
    w, b = torch.randn(D, device="cuda"), torch.randn(D, device="cuda")
    kind = "e4m3" if codes else None
    small, mean1, rstd1 = bsp.layer_norm(x, w, b, code=kind)
    y, mean, rstd = bsp.layer_norm(x.expand(T, D), w, b, code=kind)
    torch.cuda.synchronize()
    if codes:
        assert _all_rows_are(y.codes, small.codes[0])
        assert all(_all_rows_are(y.scale[k, :T, None], small.scale[k, :1]) for k in range(y.scale.shape[0]))
    else:
        assert _all_rows_are(y, small[0])
    assert _all_rows_are(mean[:, None], mean1) and _all_rows_are(rstd[:, None], rstd1)


@pytest.mark.parametrize("T,D", [((1 << 24) + 5, 4), ((1 << 24) + 3, 7)])
def test_norm_gradient_of_many_short_rows(T, D):
    """dx is a small call's; dweight and dbias against sums in 64 bits: at most T / 512 + 513 terms one after the other, a term off by 8 U of its parts."""
    import torch
    import paper_2407_09453_amd as bsp
    _needs(4)
    x = torch.randn(T, D, device="cuda")
    dy = torch.randn(T, D, device="cuda")
    w = torch.randn(D, device="cuda")
    _, mean, rstd = bsp.layer_norm(x, w)
    dx, dw, db = bsp.layer_norm_grad(dy, x, mean, rstd, w)
    for part in (slice(0, 1000), slice(T - 1000, T)):
        assert torch.equal(dx[part], bsp.layer_norm_grad(dy[part], x[part], mean[part].contiguous(), rstd[part].contiguous(), w)[0])
    n = T // 512 + 513 + 8
    terms = dy.double() * (x.double() - mean.double()[:, None]) * rstd.double()[:, None]
    spread = dy.double().abs() * (x.double().abs() + mean.double().abs()[:, None]) * rstd.double()[:, None]
    assert bool(((dw - terms.sum(0)).abs() <= n * U * terms.abs().sum(0) + 8 * U * spread.sum(0)).all())
    assert bool(((db - dy.double().sum(0)).abs() <= n * U * dy.double().abs().sum(0)).all())


def test_norm_gradient_of_long_rows():
    """2^27 columns and more: dbias is a sum of nine equal whole numbers, dweight of nine equal terms, each off by 4 U, summed in nine steps."""
    import torch
    import paper_2407_09453_amd as bsp
    _needs(40)
    T, D = 9, (1 << 27) + 3
    x = torch.randn(1, D, device="cuda").to(torch.bfloat16)
    dy = torch.randint(-8, 9, (1, D), device="cuda").to(torch.bfloat16)
    mean, rstd = torch.full((T,), 0.25, device="cuda"), torch.full((T,), 0.5, device="cuda")
    dx, dw, db = bsp.layer_norm_grad(dy.expand(T, D), x.expand(T, D), mean, rstd)
    assert torch.equal(db, T * dy[0].float())
    term = dy[0].float() * ((x[0].float() - 0.25) * 0.5)
    assert bool(((dw - T * term).abs() <= (4 + 9 + 1) * U * T * term.abs()).all())
    assert all(torch.equal(dx[0], dx[t]) for t in range(1, T))


@pytest.mark.parametrize("T,K,gib", [((1 << 28) + 17, 3, 40), ((1 << 25) + 1, 1030, 45 + 70)])
def test_checkpoint_of_many_rows(T, K, gib):
    """Rows past the sixteens that one dimension holds, of one and of two workgroups across."""
    import torch
    import paper_2407_09453_amd as bsp
    _needs(gib)
    x = torch.randn(1, K, device="cuda").to(torch.bfloat16)
    small = bsp.save8(x)
    c = bsp.save8(x.expand(T, K))
    assert _all_rows_are(c.codes, small.codes[0])
    assert all(_all_rows_are(c.scale[k, :T, None], small.scale[k, :1]) for k in range(c.scale.shape[0]))
    assert _all_rows_are(c.load(), small.load()[0])


def test_bias_gradient_alone_of_many_channels():
    """Through the C entry point, no dW: 2^24 channels over 2^14, in ranges of rows.  Whole numbers: exact sums."""
    import ctypes
    import torch
    from paper_2407_09453_amd import binding as b
    _needs(2)
    T, O, I = 1200, 1 << 24, 1 << 14
    kept = 3
    row_ptr = torch.full((O // 128 + 1,), kept, dtype=torch.int32, device="cuda")
    row_ptr[0] = 0  # all of them in the first block row
    some = torch.arange(kept, dtype=torch.int32, device="cuda")
    col_ptr = torch.zeros(I // 128 + 1, dtype=torch.int32, device="cuda")
    codes = torch.zeros(kept, 128, 128, dtype=torch.uint8, device="cuda")
    w = b.bsp_weights_f8(O, I, kept, row_ptr.data_ptr(), some.data_ptr(), col_ptr.data_ptr(), some.data_ptr(), codes.data_ptr(), codes.data_ptr(),
                         codes.data_ptr(), codes.data_ptr())
    lib = b.load_library()
    n = ctypes.c_int64(0)
    assert lib.bsp_f8_fc_grad_workspace(w, T, n) == 0 and n.value > 0
    ws = torch.empty(n.value, dtype=torch.uint8, device="cuda")
    import paper_2407_09453_amd as bsp
    x = bsp.save8(torch.ones(1, I, device="cuda").expand(T, I))
    dy = torch.randint(-8, 9, (1, O), device="cuda").to(torch.bfloat16)
    db = torch.full((O,), float("nan"), device="cuda")
    torch.cuda.synchronize()
    assert lib.bsp_f8_fc_grad(w, dy.data_ptr(), 0, ctypes.byref(x.struct), None, db.data_ptr(), ws.data_ptr(), n.value,
                              torch.cuda.current_stream().cuda_stream) == 0
    assert torch.equal(db, T * dy[0].float())
