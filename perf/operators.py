"""The operators of a layer's training step and serving call in 8-bit floating point, as measurable cases.

Three kinds of case:

* ``product``: an FC layer whose weights are e4m3 codes with a power-of-two scale for each 128x128 block, of which a mask
  keeps some; activations in bf16 or fp32 are brought to codes with a scale for each row's 128 columns within the call;
* ``save`` and ``grad``: an activation kept as an 8-bit checkpoint and read back; the backward pass of such a layer, in
  which the checkpoint of its input gives the weights' gradient and the gate of the ReLU that made it;
* ``norm``: layer norm, forward to its own type or straight to a checkpoint, and backward.

The plain forms below are the definitions in single precision.  Sizes are those of the repository's FC layers
(25088, 4096, 2048, 1000 and 512 channels), a multiple of them, and powers of two for the rows.
"""
import math

import torch

own = False

DEV = "cuda"
TORCH = {"bf16": torch.bfloat16, "f32": torch.float32}
BYTES = {"bf16": 2, "f32": 4}
FLOAT8 = {"e4m3": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2}
EPS = 1e-5


# ------------------------------------------------------------------------------- the cases
def listed():
    return [
        # serving, one row at a time: a 4096 x 4096 layer streams its weights once for a single row
        {"name": "product_single", "kind": "product", "T": 1, "I": 4096, "O": 4096, "density": 1.0, "dtype": "bf16", "relu": False},
        # serving a batch of 16 on the widest FC layer of the benchmark networks, half of its blocks kept
        {"name": "product_few", "kind": "product", "T": 16, "I": 25088, "O": 4096, "density": 0.5, "dtype": "bf16", "relu": True},
        # a classifier on an odd number of rows in single precision: ragged in rows and in outputs
        {"name": "product_ragged_f32", "kind": "product", "T": 197, "I": 2048, "O": 1000, "density": 0.75, "dtype": "f32", "relu": False},
        # a training batch through a widening layer, all blocks kept
        {"name": "product_large", "kind": "product", "T": 16384, "I": 4096, "O": 16384, "density": 1.0, "dtype": "bf16", "relu": True},
        # a small activation kept and read back, where latency counts
        {"name": "save_small", "kind": "save", "T": 16, "I": 2048, "code": "e4m3", "dtype": "bf16"},
        # a training batch's activation kept and read back
        {"name": "save_large", "kind": "save", "T": 16384, "I": 4096, "code": "e4m3", "dtype": "bf16"},
        # the backward pass of a small ragged layer on few rows
        {"name": "grad_small", "kind": "grad", "T": 37, "I": 1000, "O": 520, "density": 0.6, "code": "e5m2", "relu": False},
        # the backward pass of a square layer, half of its blocks kept, behind a ReLU
        {"name": "grad_masked", "kind": "grad", "T": 2048, "I": 4096, "O": 4096, "density": 0.5, "code": "e5m2", "relu": True},
        # the backward pass of a widening layer on a training batch, all blocks kept
        {"name": "grad_large", "kind": "grad", "T": 8192, "I": 4096, "O": 16384, "density": 1.0, "code": "e4m3", "relu": True},
        # serving one row: the norm in front of a layer, straight to the codes that the layer reads
        {"name": "norm_single", "kind": "norm", "T": 1, "D": 4096, "dtype": "bf16", "codes": True, "grad": False},
        # forward and backward in single precision at a ragged width
        {"name": "norm_ragged_f32", "kind": "norm", "T": 1021, "D": 1000, "dtype": "f32", "codes": False, "grad": True},
        # forward and backward of a training batch
        {"name": "norm_large", "kind": "norm", "T": 16384, "D": 4096, "dtype": "bf16", "codes": False, "grad": True},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _channels(rng, lo, hi):
    """Mostly whole blocks, as such layers have them; one in three is any number."""
    c = _log(rng, lo, hi)
    return c if rng.random() < 0.34 else max(128, (c + 64) // 128 * 128)


def draw(rng):
    kind = rng.choice(["product", "product", "save", "grad", "grad", "norm"])
    density = rng.choice([0.25, 0.5, 0.75, 1.0, 1.0])
    if kind in ("product", "grad"):
        while True:
            few = kind == "product" and rng.random() < 0.4  # serving
            T = _log(rng, 1, 64) if few else _log(rng, 1, 16384)
            I, O = _channels(rng, 64, 25088), _channels(rng, 64, 16384)
            if T * I * O <= (2 ** 40 if kind == "product" else 2 ** 39) and I * O <= 2 ** 27:
                break
        c = {"kind": kind, "T": T, "I": I, "O": O, "density": density, "relu": rng.random() < 0.5}
        if kind == "product":
            return {**c, "dtype": rng.choice(["bf16", "bf16", "bf16", "f32"])}
        return {**c, "code": rng.choice(["e4m3", "e5m2"])}
    T, D = _log(rng, 1, 16384), _channels(rng, 64, 16384)
    if T * D > 2 ** 26:
        T = max(1, 2 ** 26 // D)
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if kind == "save":
        return {"kind": kind, "T": T, "I": D, "code": rng.choice(["e4m3", "e5m2"]), "dtype": dtype}
    codes = rng.random() < 0.4
    return {"kind": kind, "T": T, "D": D, "dtype": dtype, "codes": codes, "grad": not codes or rng.random() < 0.5}


# ------------------------------------------------------------------------------- inputs
def _activation(gen, T, I, dtype, relu):
    """Rows of differing size, a few channels much larger than the others; not negative behind a ReLU."""
    x = torch.randn(T, I, generator=gen, device=DEV)
    x *= torch.exp(0.5 * torch.randn(T, 1, generator=gen, device=DEV))
    x *= torch.where(torch.rand(I, generator=gen, device=DEV) < 0.01, 20.0, 1.0)
    return (x.clamp_min(0) if relu else x).to(dtype)


def _inputs(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    kind, T = case["kind"], case["T"]
    s = {"kind": kind}
    if kind in ("product", "grad"):
        I, O = case["I"], case["O"]
        W = torch.randn(O, I, generator=gen, device=DEV) * math.sqrt(2.0 / (I * case["density"]))
        nbo, nbi = -(-O // 128), -(-I // 128)
        gamma = (torch.rand(nbo, nbi, generator=gen, device=DEV).argsort().argsort() < max(1, round(case["density"] * nbi))).to(torch.uint8) \
            if nbi > 1 else torch.ones(nbo, nbi, dtype=torch.uint8, device=DEV)
        s |= {"W": W, "gamma": gamma, "bias": torch.randn(O, generator=gen, device=DEV) * 0.1, "relu": case["relu"]}
    if kind == "product":
        s["X"] = _activation(gen, T, I, TORCH[case["dtype"]], False)
    elif kind == "save":
        s |= {"X": _activation(gen, T, case["I"], TORCH[case["dtype"]], False), "code": case["code"]}
    elif kind == "grad":
        s["X"] = _activation(gen, T, I, torch.bfloat16, case["relu"])
        s["dY"] = (torch.randn(T, O, generator=gen, device=DEV) * 1e-3 * torch.exp(torch.randn(T, 1, generator=gen, device=DEV))).to(torch.bfloat16)
        s["code"] = case["code"]
    else:
        D, dt = case["D"], TORCH[case["dtype"]]
        x = torch.randn(T, D, generator=gen, device=DEV) * torch.exp(torch.randn(T, 1, generator=gen, device=DEV)) + torch.randn(T, 1, generator=gen, device=DEV)
        s |= {"X": x.to(dt), "weight": 1 + 0.1 * torch.randn(D, generator=gen, device=DEV), "bias": 0.1 * torch.randn(D, generator=gen, device=DEV),
              "codes": case["codes"], "grad": case["grad"]}
        if case["grad"]:
            s["dY"] = (torch.randn(T, D, generator=gen, device=DEV) * 1e-2).to(dt)
    return s


def prepare(case, seed):
    """Weights are held as their codes and scales, and a checkpoint that the forward pass has left as its own, on either side."""
    s = _inputs(case, seed)
    if own:
        import paper_2407_09453_amd as bsp
        s["bsp"] = bsp
        if "W" in s:
            s["layer"] = bsp.BspLayerF8(s.pop("W"), s.pop("gamma"), bias=s.pop("bias"), device=DEV)
        if case["kind"] == "grad":
            s["checkpoint"] = bsp.save8(s.pop("X"))
        return s
    if "W" in s:
        s["W"] = _codes(s["W"], "e4m3", 128)
    if case["kind"] == "grad":
        s["checkpoint"] = _codes(s.pop("X"), "e4m3")
    return s


# ------------------------------------------------------------------------------- the plain forms
def _power(e):
    """2^e, exactly (a device's pow and ldexp may be off by a unit in the last place)."""
    return ((e.long() + 1023) << 52).view(torch.float64).float()


def _codes(x, kind, rows=1):
    """(codes, scales): a power of two for each block of rows x 128, such that the block's largest value fits the code's range."""
    T, K = x.shape
    Tp, Kp = -(-T // rows) * rows, -(-K // 128) * 128
    full = torch.zeros(Tp, Kp, device=x.device)
    full[:T, :K] = x
    b = full.view(Tp // rows, rows, Kp // 128, 128)
    m, e = torch.frexp(b.abs().amax(dim=(1, 3), keepdim=True))  # amax = m 2^e, 0.5 <= m < 1
    e = e - {"e4m3": 9, "e5m2": 16}[kind] + (m > 0.875).to(e.dtype)
    e = torch.where(m == 0, torch.zeros_like(e), e.clamp(-127, 127))
    q = (b * _power(-e)).to(FLOAT8[kind])
    return q.view(Tp, Kp)[:T, :K], e.view(Tp // rows, Kp // 128), rows


def _values(codes):
    q, e, rows = codes
    s = _power(e).repeat_interleave(rows, 0).repeat_interleave(128, 1)
    return q.float() * s[:q.shape[0], :q.shape[1]]


def _weights(s):
    W = _values(s["W"])
    return W * s["gamma"].repeat_interleave(128, 0).repeat_interleave(128, 1)[:W.shape[0], :W.shape[1]]


def run(s):
    return _run_own(s) if own else _run_plain(s)


def _run_own(s):
    kind = s["kind"]
    if kind == "product":
        return s["layer"].fc(s["X"], relu=s["relu"])
    if kind == "save":
        return s["bsp"].save8(s["X"], s["code"]).load()
    if kind == "grad":
        dX = s["layer"].grad_input(s["dY"], relu_of=s["checkpoint"] if s["relu"] else None, code=s["code"])
        dW, db = s["layer"].grad_weight(s["dY"], s["checkpoint"])
        return {"dX": dX, "dW": dW, "db": db}
    y, mean, rstd = s["bsp"].layer_norm(s["X"], s["weight"], s["bias"], EPS, code="e4m3" if s["codes"] else None)
    out = {"y": y.load() if s["codes"] else y}
    if s["grad"]:
        out["dX"], out["dw"], out["db"] = s["bsp"].layer_norm_grad(s["dY"], s["X"], mean, rstd, s["weight"])
    return out


def _run_plain(s):
    kind = s["kind"]
    if kind == "product":
        y = _values(_codes(s["X"], "e4m3")) @ _weights(s).t() + s["bias"]
        return (y.clamp_min(0) if s["relu"] else y).to(s["X"].dtype)
    if kind == "save":
        return _values(_codes(s["X"], s["code"])).to(torch.bfloat16)
    if kind == "grad":
        x, dy = _values(s["checkpoint"]), s["dY"].float()
        dx = _values(_codes(s["dY"], s["code"])) @ _weights(s)
        if s["relu"]:
            dx = dx * (x > 0)
        gamma = s["gamma"].repeat_interleave(128, 0).repeat_interleave(128, 1)[:dy.shape[1], :x.shape[1]]
        return {"dX": dx.to(torch.bfloat16), "dW": (dy.t() @ x) * gamma, "db": dy.sum(0)}
    x = s["X"].float()
    c = x - x.mean(1, keepdim=True)
    r = torch.rsqrt((c * c).mean(1, keepdim=True) + EPS)
    h = c * r
    y = h * s["weight"] + s["bias"]
    out = {"y": _values(_codes(y, "e4m3")).to(torch.bfloat16) if s["codes"] else y.to(s["X"].dtype)}
    if s["grad"]:
        dy = s["dY"].float()
        g = dy * s["weight"]
        dx = r * (g - g.mean(1, keepdim=True) - h * (g * h).mean(1, keepdim=True))
        out |= {"dX": dx.to(s["X"].dtype), "dw": (dy * h).sum(0), "db": dy.sum(0)}
    return out


# ------------------------------------------------------------------------------- what a pass cannot do without
def work(case):
    kind, T = case["kind"], case["T"]
    if kind in ("product", "grad"):
        I, O = case["I"], case["O"]
        nbo, nbi = -(-O // 128), -(-I // 128)
        kept = max(1, round(case["density"] * nbi)) / nbi
        weights = kept * O * I
        if kind == "product":
            b = BYTES[case["dtype"]]
            return {"bytes": T * I * b + weights + 4 * O + T * O * b, "flops": 2 * T * weights}
        return {"bytes": 2 * T * O + T * I + weights + 2 * T * I + 4 * O * I + 4 * O, "flops": 4 * T * weights}
    if kind == "save":  # read, codes written, values written
        return {"bytes": T * case["I"] * (BYTES[case["dtype"]] + 1 + 2), "flops": 4 * T * case["I"]}
    D, b = case["D"], BYTES[case["dtype"]]
    fwd = T * D * (b + (1 + 2 if case["codes"] else b)) + 8 * D
    return {"bytes": fwd + (T * D * 2 * b + 12 * D if case["grad"] else 0), "flops": T * D * (8 + (14 if case["grad"] else 0))}


# ------------------------------------------------------------------------------- 64 bits
def _floor_log2(a):
    """The exponent of each value (as a whole number), 0 where there is none: the exponent field of a double."""
    return torch.where(a > 0, (a.view(torch.int64) >> 52) - 1023, 0)


def _two(e):
    """2^e in 64 bits from a whole number: 1.0 with its exponent field moved."""
    return (torch.full_like(e, 1023) + e << 52).view(torch.float64)


def _exact_values(x, kind, tall=1):
    """The values that codes stand for, from the rule itself: exponent of the largest, and the grid of the code around each value."""
    x = x.double()
    rows, cols = x.shape
    out = torch.empty_like(x)
    bits, top, low = (3, 8, -6) if kind == "e4m3" else (2, 15, -14)
    group = torch.arange(rows, device=x.device) // tall
    for k in range(0, cols, 128):
        part = x[:, k:k + 128]
        most = torch.zeros(int(group[-1]) + 1, dtype=torch.float64, device=x.device).scatter_reduce(0, group, part.abs().amax(1), "amax")
        exp = _floor_log2(most)
        e = torch.where(most > 1.75 * _two(exp), exp - top + 1, exp - top)
        e = torch.where(most > 0, e.clamp(-127, 127), 0)[group][:, None]
        v = part * _two(-e)
        step = _two(_floor_log2(v.abs()).clamp_min(low) - bits)
        out[:, k:k + 128] = torch.round(v / step) * step * _two(e)
    return out


def _exact_weights(s):
    W = _exact_values(s["W"], "e4m3", 128)
    for o in range(s["gamma"].shape[0]):
        keep = s["gamma"][o].double().repeat_interleave(128)[:W.shape[1]]
        W[o * 128:(o + 1) * 128] *= keep
    return W


def exact(case, seed):
    s = _inputs(case, seed)
    kind = case["kind"]
    if kind == "product":
        y = torch.addmm(s["bias"].double(), _exact_values(s["X"], "e4m3"), _exact_weights(s).t().contiguous())
        return torch.relu(y) if s["relu"] else y
    if kind == "save":
        return _exact_values(s["X"], s["code"])
    if kind == "grad":
        x, dy = _exact_values(s["X"], "e4m3"), s["dY"].double()
        dx = torch.mm(_exact_values(s["dY"], s["code"]), _exact_weights(s))
        if s["relu"]:
            dx = torch.where(x > 0, dx, 0.0)
        dw = torch.mm(dy.t().contiguous(), x)
        for o in range(s["gamma"].shape[0]):
            dw[o * 128:(o + 1) * 128] *= s["gamma"][o].double().repeat_interleave(128)[:dw.shape[1]]
        return {"dX": dx, "dW": dw, "db": dy.sum(0)}
    x, w, b = s["X"].double(), s["weight"].double(), s["bias"].double()
    mean = x.sum(1, keepdim=True) / x.shape[1]
    sd = torch.sqrt(((x - mean) ** 2).sum(1, keepdim=True) / x.shape[1] + EPS)
    h = (x - mean) / sd
    y = h * w + b
    out = {"y": _exact_values(y, "e4m3") if s["codes"] else y}
    if s["grad"]:
        dy = s["dY"].double()
        p = dy * w
        proj = (p * h).sum(1, keepdim=True) / x.shape[1]
        out["dX"] = (p - p.sum(1, keepdim=True) / x.shape[1] - proj * h) / sd
        out["dw"], out["db"] = (dy * h).sum(0), dy.sum(0)
    return out
