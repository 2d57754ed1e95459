"""Operators of fine-tuning and serving a language model on frozen 8-bit layers, as measurable cases.

Four kinds of case:

* ``rms``: root-mean-square norm with the addition of the residual stream, to its own type or straight to the 8-bit codes that
  a layer reads, and its backward pass, in which the gradient that came down the residual stream joins;
* ``adapt``: an 8-bit FC layer with low-rank adapters beside it, each row its own request's: y = W x + b + s B_a A_a x;
* ``tune``: the backward pass of such a layer whose adapters alone are trained: the gradients of its input, and of A and B
  of every adapter;
* ``logp``: log probabilities of given tokens with the entropy, the log of the sum and the top alternatives, from logits, and
  the gradient of the logits.

The plain forms below are the definitions in single precision.  Sizes are those of the repository's FC layers
(25088, 4096, 2048, 1000 and 512 channels), multiples of them, and powers of two or any number for rows and vocabularies.
"""
import math

import torch

own = False

DEV = "cuda"
TORCH = {"bf16": torch.bfloat16, "f32": torch.float32}
BYTES = {"bf16": 2, "f32": 4, "codes": 1}
FLOAT8 = {"e4m3": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2}
EPS = 1e-6


# ------------------------------------------------------------------------------- the cases
def listed():
    return [
        # serving one token: the norm in front of a layer, the residual added, straight to the codes that the layer reads
        {"name": "rms_single", "kind": "rms", "T": 1, "D": 4096, "dtype": "bf16", "residual": True, "codes": True, "grad": False},
        # forward and backward in single precision at a ragged width, as the last norm of a model has it, with no residual
        {"name": "rms_ragged_f32", "kind": "rms", "T": 777, "D": 2966, "dtype": "f32", "residual": False, "codes": False, "grad": True},
        # forward and backward of a training batch, with the residual stream both ways
        {"name": "rms_large", "kind": "rms", "T": 16384, "D": 4096, "dtype": "bf16", "residual": True, "codes": True, "grad": True},
        # serving one token of one request
        {"name": "adapt_single", "kind": "adapt", "T": 1, "I": 4096, "O": 4096, "density": 1.0, "dtype": "bf16", "R": 16, "N": 8, "runs": False, "relu": False},
        # serving a batch of single tokens, each of any of 32 requests' adapters or of none, half of the layer's blocks kept
        {"name": "adapt_batch", "kind": "adapt", "T": 64, "I": 4096, "O": 16384, "density": 0.5, "dtype": "bf16", "R": 16, "N": 32, "runs": False, "relu": True},
        # prompts of twelve requests, packed one behind the other, from the codes that the norm left
        {"name": "adapt_large", "kind": "adapt", "T": 16384, "I": 4096, "O": 4096, "density": 1.0, "dtype": "codes", "R": 16, "N": 12, "runs": True, "relu": False},
        # the backward pass of a small ragged layer on few rows
        {"name": "tune_small", "kind": "tune", "T": 37, "I": 1000, "O": 520, "density": 0.6, "R": 4, "N": 3, "runs": False},
        # the backward pass of a widening layer on a training batch of four tasks
        {"name": "tune_large", "kind": "tune", "T": 8192, "I": 4096, "O": 16384, "density": 1.0, "R": 32, "N": 4, "runs": True},
        # serving one token: its log probability and the twenty likeliest of a long vocabulary
        {"name": "logp_single", "kind": "logp", "T": 1, "V": 131072, "dtype": "bf16", "top": 20, "scale": 1.0, "masked": False, "grad": False},
        # a classifier's loss in single precision with its gradient, and its five likeliest classes
        {"name": "logp_ragged_f32", "kind": "logp", "T": 253, "V": 1000, "dtype": "f32", "top": 5, "scale": 1.0, "masked": False, "grad": True},
        # scoring a prompt under a grammar that leaves some rows few tokens, at a temperature, odd vocabulary
        {"name": "logp_masked", "kind": "logp", "T": 1021, "V": 50001, "dtype": "bf16", "top": 8, "scale": 1.25, "masked": True, "grad": False},
        # the loss of a training batch, with entropy, and its gradient
        {"name": "logp_large", "kind": "logp", "T": 8192, "V": 32768, "dtype": "bf16", "top": 0, "scale": 1.0, "masked": False, "grad": True},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _channels(rng, lo, hi):
    """Mostly whole blocks, as such layers have them; one in three is any number."""
    c = _log(rng, lo, hi)
    return c if rng.random() < 0.34 else max(128, (c + 64) // 128 * 128)


def draw(rng):
    kind = rng.choice(["rms", "adapt", "adapt", "tune", "tune", "logp", "logp"])
    if kind == "rms":
        T, D = _log(rng, 1, 16384), _channels(rng, 64, 16384)
        T = max(1, min(T, 2 ** 26 // D))
        codes = rng.random() < 0.5
        return {"kind": kind, "T": T, "D": D, "dtype": rng.choice(["bf16", "bf16", "f32"]), "residual": rng.random() < 0.7, "codes": codes,
                "grad": not codes or rng.random() < 0.5}
    if kind == "logp":
        T, V = _log(rng, 1, 16384), _log(rng, 100, 200000)
        T = max(1, min(T, 2 ** 28 // V))
        return {"kind": kind, "T": T, "V": V, "dtype": rng.choice(["bf16", "bf16", "f32"]), "top": rng.choice([0, 1, 5, 20, 50]),
                "scale": rng.choice([1.0, 1.0, 0.7, 1.25]), "masked": rng.random() < 0.3, "grad": rng.random() < 0.5}
    while True:
        few = kind == "adapt" and rng.random() < 0.5  # serving single tokens
        T = _log(rng, 1, 64) if few else _log(rng, 1, 16384)
        I, O = _channels(rng, 64, 16384), _channels(rng, 64, 16384)
        R, N = _log(rng, 1, 64), _log(rng, 1, 64)
        if T * I * O <= (2 ** 38 if kind == "adapt" else 2 ** 39) and I * O <= 2 ** 26 and N * R * (I + O) <= 2 ** 25 and T * N * R <= 2 ** 23:
            break
    c = {"kind": kind, "T": T, "I": I, "O": O, "density": rng.choice([0.25, 0.5, 1.0, 1.0]), "R": R, "N": N, "runs": not few and rng.random() < 0.7}
    if kind == "adapt":
        c |= {"dtype": rng.choice(["bf16", "bf16", "codes", "f32"]), "relu": rng.random() < 0.3}
    return c


# ------------------------------------------------------------------------------- inputs
def _activation(gen, T, I):
    """Rows of differing size, a few channels much larger than the others."""
    x = torch.randn(T, I, generator=gen, device=DEV)
    x *= torch.exp(0.5 * torch.randn(T, 1, generator=gen, device=DEV))
    return x * torch.where(torch.rand(I, generator=gen, device=DEV) < 0.01, 20.0, 1.0)


def _which(gen, T, N, runs):
    """Each row's adapter: any of them, or none (-1, one row in eight); or requests one behind the other, of differing lengths."""
    if not runs:
        ids = torch.randint(0, N, (T,), generator=gen, device=DEV)
        return torch.where(torch.rand(T, generator=gen, device=DEV) < 0.125, -1, ids).int()
    ends = torch.rand(N, generator=gen, device=DEV).add_(0.1).cumsum(0)
    at = (torch.arange(T, device=DEV) + 0.5) / T * ends[-1]
    order = torch.rand(N, generator=gen, device=DEV).argsort()
    return order[torch.searchsorted(ends, at).clamp_max(N - 1)].int()


def _inputs(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    kind, T = case["kind"], case["T"]
    s = {"kind": kind}
    if kind == "rms":
        D, dt = case["D"], TORCH[case["dtype"]]
        s |= {"X": _activation(gen, T, D).to(dt), "weight": 1 + 0.1 * torch.randn(D, generator=gen, device=DEV), "codes": case["codes"], "grad": case["grad"],
              "residual": _activation(gen, T, D).to(dt) if case["residual"] else None}
        if case["grad"]:
            s["dY"] = (torch.randn(T, D, generator=gen, device=DEV) * 1e-2).to(dt)
            s["dH"] = (torch.randn(T, D, generator=gen, device=DEV) * 1e-2).to(dt) if case["residual"] else None
    elif kind == "logp":
        V, dt = case["V"], TORCH[case["dtype"]]
        z = torch.randn(T, V, generator=gen, device=DEV) * 2.5
        likely = torch.randint(0, V, (T, 4), generator=gen, device=DEV)  # a few likely tokens, as models have them
        z.scatter_(1, likely, 8 + 2 * torch.randn(T, 4, generator=gen, device=DEV))
        tokens = torch.where(torch.rand(T, generator=gen, device=DEV) < 0.6, likely[:, 0], torch.randint(0, V, (T,), generator=gen, device=DEV))
        if case["masked"]:  # in one row of three one token of 32 is allowed (and more than are asked for)
            rows = torch.rand(T, 1, generator=gen, device=DEV) < 0.34
            off = (torch.arange(V, device=DEV) * 7919 + 31 * torch.arange(T, device=DEV)[:, None]) % 32 != 0
            off &= torch.arange(V, device=DEV) >= 64
            off &= torch.arange(V, device=DEV) != tokens[:, None]
            z.masked_fill_(rows & off, float("-inf"))
        if T > 8:
            tokens = torch.where(torch.rand(T, generator=gen, device=DEV) < 0.05, -1, tokens)  # padding
        s |= {"X": z.to(dt), "tokens": tokens.int(), "top": case["top"], "scale": case["scale"], "grad": case["grad"]}
        if case["grad"]:
            s["dlogp"] = -torch.rand(T, generator=gen, device=DEV) / T
            s["dentropy"] = 0.01 * torch.randn(T, generator=gen, device=DEV) / T
    else:
        I, O, R, N = case["I"], case["O"], case["R"], case["N"]
        W = torch.randn(O, I, generator=gen, device=DEV) * math.sqrt(2.0 / (I * case["density"]))
        nbo, nbi = -(-O // 128), -(-I // 128)
        gamma = (torch.rand(nbo, nbi, generator=gen, device=DEV).argsort().argsort() < max(1, round(case["density"] * nbi))).to(torch.uint8) \
            if nbi > 1 else torch.ones(nbo, nbi, dtype=torch.uint8, device=DEV)
        s |= {"W": W, "gamma": gamma, "bias": torch.randn(O, generator=gen, device=DEV) * 0.1,
              "A": (torch.randn(N, R, I, generator=gen, device=DEV) / math.sqrt(I)).bfloat16(),
              "B": (torch.randn(N, O, R, generator=gen, device=DEV) * 0.2).bfloat16(),
              "s": 2.0 ** torch.randint(-1, 2, (N,), generator=gen, device=DEV).float(), "which": _which(gen, T, N, case["runs"])}
        x = _activation(gen, T, I)
        if kind == "adapt":
            s |= {"X": x.to(TORCH.get(case["dtype"], torch.bfloat16)), "coded": case["dtype"] == "codes", "relu": case["relu"]}
        else:
            s["X"] = x.bfloat16()
            s["dY"] = (torch.randn(T, O, generator=gen, device=DEV) * 1e-3 * torch.exp(torch.randn(T, 1, generator=gen, device=DEV))).bfloat16()
    return s


def prepare(case, seed):
    """Weights are held as their codes and scales, adapters in bf16, and a checkpoint that an earlier call has left as its own, on either side."""
    s = _inputs(case, seed)
    kind = case["kind"]
    coded = kind == "tune" or s.get("coded")
    if own:
        import paper_2407_09453_amd as bsp
        s["bsp"] = bsp
        if kind in ("adapt", "tune"):
            s["layer"] = bsp.BspLayerF8(s.pop("W"), s.pop("gamma"), bias=s.pop("bias"), device=DEV)
            s["adapters"] = bsp.BspAdapters(case["N"], case["R"], case["I"], case["O"], device=DEV)
            A, B, scale = s.pop("A"), s.pop("B"), s.pop("s").tolist()
            for n in range(case["N"]):
                s["adapters"].set(n, A[n], B[n], scale[n])
            s["requests"] = bsp.BspRequests(s.pop("which"), case["N"])
            if coded:
                s["X"] = bsp.save8(s["X"])
        return s
    if "W" in s:
        s["W"] = _codes(s["W"], "e4m3", 128)
        if coded:
            s["X"] = _codes(s["X"], "e4m3")
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
    kind, bsp = s["kind"], s["bsp"]
    if kind == "rms":
        y, h, rstd = bsp.rms_norm(s["X"], s["weight"], s["residual"], EPS, code="e4m3" if s["codes"] else None)
        out = {"y": y.load() if s["codes"] else y, "h": h, "rstd": rstd}
        if s["grad"]:
            out["dX"], out["dw"] = bsp.rms_norm_grad(s["dY"], h, rstd, s["weight"], dH=s["dH"])
        return out
    if kind == "adapt":
        return s["layer"].fc(s["X"], relu=s["relu"], adapters=s["adapters"], requests=s["requests"])
    if kind == "tune":
        dX = s["layer"].grad_input(s["dY"], adapters=s["adapters"], requests=s["requests"])
        dA, dB = s["adapters"].grad(s["dY"], s["X"], s["requests"])
        return {"dX": dX, "dA": dA, "dB": dB}
    logp, lse, entropy, top, ids = bsp.log_probs(s["X"], s["tokens"], top=s["top"], scale=s["scale"])
    out = {"logp": logp, "lse": lse, "entropy": entropy}
    if s["top"]:
        out["top"], out["ids"] = top, ids
    if s["grad"]:
        out["dX"] = bsp.log_probs_grad(s["X"], s["tokens"], lse, entropy, s["dlogp"], s["dentropy"], scale=s["scale"])
    return out


def _low(s, x, A, B):
    """(u, u B) of the rows' adapters: every row against all of them, all but its own set to zero."""
    N, R = A.shape[0], A.shape[1]
    mine = (s["which"][:, None] == torch.arange(N, device=x.device)).float() * s["s"]
    u = (x @ A.reshape(N * R, -1).t()).view(-1, N, R) * mine[:, :, None]
    return u, u.reshape(-1, N * R) @ B.transpose(1, 2).reshape(N * R, -1)


def _run_plain(s):
    kind = s["kind"]
    if kind == "rms":
        dt = s["X"].dtype
        h = s["X"] if s["residual"] is None else (s["X"].float() + s["residual"].float()).to(dt)
        x = h.float()
        r = torch.rsqrt((x * x).mean(1, keepdim=True) + EPS)
        y = x * r * s["weight"]
        out = {"y": _values(_codes(y, "e4m3")).to(torch.bfloat16) if s["codes"] else y.to(dt), "h": h, "rstd": r[:, 0]}
        if s["grad"]:
            dy = s["dY"].float()
            g = dy * s["weight"]
            dx = r * (g - x * (r * r * (g * x).mean(1, keepdim=True)))
            if s["dH"] is not None:
                dx = dx + s["dH"].float()
            out |= {"dX": dx.to(dt), "dw": (dy * x * r).sum(0)}
        return out
    if kind == "adapt":
        x = _values(s["X"]) if s["coded"] else s["X"].float()
        y = (x if s["coded"] else _values(_codes(x, "e4m3"))) @ _weights(s).t() + s["bias"] + _low(s, x, s["A"].float(), s["B"].float())[1]
        return (y.clamp_min(0) if s["relu"] else y).to(torch.bfloat16 if s["coded"] else s["X"].dtype)
    if kind == "tune":
        x, dy, A, B = _values(s["X"]), s["dY"].float(), s["A"].float(), s["B"].float()
        N, R = A.shape[0], A.shape[1]
        u, v = _low(s, x, A, B)[0], None
        v, low = _low(s, dy, B.transpose(1, 2), A.transpose(1, 2))
        dx = _values(_codes(dy, "e5m2")) @ _weights(s) + low
        dA = (v.reshape(-1, N * R).t() @ x).view(N, R, -1)
        dB = (u.reshape(-1, N * R).t() @ dy).view(N, R, -1).transpose(1, 2).contiguous()
        return {"dX": dx.to(torch.bfloat16), "dA": dA, "dB": dB}
    z = s["X"].float() * s["scale"]
    m = z.amax(1, keepdim=True)
    d = z - m
    e = torch.exp(d)
    total = e.sum(1, dtype=torch.float64)
    log = torch.log(total)
    tokens = s["tokens"].long()
    at = d.gather(1, tokens.clamp_min(0)[:, None])[:, 0]
    # (0 times minus infinity is nothing in an entropy)
    entropy = log - (torch.where(e > 0, d, 0.0) * e).sum(1, dtype=torch.float64) / total
    out = {"logp": torch.where(tokens >= 0, at - log, 0.0).float(), "lse": (m[:, 0] + log).float(), "entropy": entropy.float()}
    if s["top"]:
        v, i = torch.sort(s["X"].float(), dim=1, descending=True, stable=True)
        out |= {"top": (v[:, :s["top"]] * s["scale"] - m - log[:, None]).float(), "ids": i[:, :s["top"]].int()}
    if s["grad"]:
        lp = d - log.float()[:, None]
        p = torch.exp(lp)
        dlogp = torch.where(tokens >= 0, s["dlogp"], 0.0)
        dz = p * (-dlogp[:, None] - s["dentropy"][:, None] * (torch.where(p > 0, lp, 0.0) + entropy.float()[:, None]))
        dz.scatter_add_(1, tokens.clamp_min(0)[:, None], dlogp[:, None])
        out["dX"] = (dz * s["scale"]).to(s["X"].dtype)
    return out


# ------------------------------------------------------------------------------- what a pass cannot do without
def work(case):
    kind, T = case["kind"], case["T"]
    if kind == "rms":
        D, b = case["D"], BYTES[case["dtype"]]
        fwd = T * D * (b * (3 if case["residual"] else 1) + (1 + 2 if case["codes"] else b)) + 4 * D + 4 * T
        return {"bytes": fwd + (T * D * b * (4 if case["residual"] else 3) + 8 * D if case["grad"] else 0), "flops": T * D * (5 + (12 if case["grad"] else 0))}
    if kind == "logp":
        V, b = case["V"], BYTES[case["dtype"]]
        return {"bytes": T * V * b * (3 if case["grad"] else 1) + T * (16 + 8 * case["top"]), "flops": T * V * (6 + (8 if case["grad"] else 0))}
    I, O, R = case["I"], case["O"], case["R"]
    nbi = -(-I // 128)
    weights = max(1, round(case["density"] * nbi)) / nbi * O * I
    low, used = T * R * (I + O), min(case["N"], T) * R * (I + O)
    if kind == "adapt":
        b = BYTES[case["dtype"]]
        return {"bytes": T * I * b + weights + 4 * O + 2 * used + T * O * max(b, 2), "flops": 2 * T * weights + 2 * low}
    return {"bytes": 2 * T * O + T * I + weights + 2 * used + 2 * T * I + 4 * case["N"] * R * (I + O), "flops": 2 * T * weights + 6 * low}


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
        W[o * 128:(o + 1) * 128] *= s["gamma"][o].double().repeat_interleave(128)[:W.shape[1]]
    return W


def _exact_logp(s):
    """Row by row in 64 bits (some rows at a time, for memory's sake)."""
    X, tokens, n, scale = s["X"], s["tokens"].long(), s["top"], s["scale"]
    T, V = X.shape
    parts = {k: [] for k in ["logp", "lse", "entropy"] + (["top", "ids"] if n else []) + (["dX"] if s["grad"] else [])}
    for a in range(0, T, max(1, 2 ** 25 // V)):
        rows = slice(a, min(T, a + max(1, 2 ** 25 // V)))
        x, tok = X[rows].double(), tokens[rows]
        lse = torch.logsumexp(x * scale, 1)
        lp = x * scale - lse[:, None]
        p = lp.exp()
        h = -torch.special.xlogy(p, p).sum(1)
        given = tok >= 0
        safe = tok.clamp_min(0)[:, None]
        parts["logp"].append(torch.where(given, lp.gather(1, safe)[:, 0], 0.0))
        parts["lse"].append(lse)
        parts["entropy"].append(h)
        if n:  # by value, and by index where values are equal: the (V - index) breaks ties of the logits' ranks
            rank = torch.unique(x, return_inverse=True)[1] * V + (V - 1 - torch.arange(V, device=x.device))
            ids = rank.topk(n, 1).indices
            parts["ids"].append(ids.int())
            parts["top"].append(lp.gather(1, ids))
        if s["grad"]:
            one = torch.zeros_like(p).scatter_(1, safe, given[:, None].double())
            dl, dh = (s["dlogp"][rows].double() * given)[:, None], s["dentropy"][rows].double()[:, None]
            parts["dX"].append(scale * (dl * (one - p) - dh * (torch.special.xlogy(p, p) + p * h[:, None])))
    return {k: torch.cat(v) for k, v in parts.items()}


def exact(case, seed):
    s = _inputs(case, seed)
    kind = case["kind"]
    if kind == "logp":
        return _exact_logp(s)
    if kind == "rms":
        h = s["X"].double()
        if s["residual"] is not None:  # the residual stream is held in its type, and the norm is that of what is held
            h = (h + s["residual"].double()).to(s["X"].dtype).double()
        D, w = h.shape[1], s["weight"].double()
        q = 1 / torch.sqrt(h.pow(2).sum(1, keepdim=True) / D + EPS)
        y = h * q * w
        out = {"y": _exact_values(y, "e4m3") if s["codes"] else y, "h": h, "rstd": q[:, 0]}
        if s["grad"]:
            n, dy = h * q, s["dY"].double()
            dn = dy * w
            out["dX"] = q * (dn - n * ((dn * n).sum(1, keepdim=True) / D))
            if s["dH"] is not None:
                out["dX"] += s["dH"].double()
            out["dw"] = (dy * n).sum(0)
        return out
    codes = _exact_values(s["X"], "e4m3")
    x = codes if kind == "tune" or s["coded"] else s["X"].double()
    W = _exact_weights(s)
    y = torch.addmm(s["bias"].double(), codes, W.t().contiguous()) if kind == "adapt" else torch.mm(_exact_values(s["dY"], "e5m2"), W)
    dA, dB = torch.zeros(s["A"].shape, dtype=torch.float64, device=DEV), torch.zeros(s["B"].shape, dtype=torch.float64, device=DEV)
    for n in range(case["N"]):
        rows = torch.nonzero(s["which"] == n)[:, 0]
        if rows.numel() == 0:
            continue
        A, B, f = s["A"][n].double(), s["B"][n].double(), s["s"][n].double()
        xs = x[rows]
        if kind == "adapt":
            y[rows] += f * torch.mm(torch.mm(xs, A.t().contiguous()), B.t().contiguous())
        else:
            dy = s["dY"][rows].double()
            v = torch.mm(dy, B) * f
            y[rows] += torch.mm(v, A)
            dA[n] = torch.mm(v.t().contiguous(), xs)
            dB[n] = torch.mm(dy.t().contiguous(), torch.mm(xs, A.t().contiguous()) * f)
    if kind == "adapt":
        return torch.relu(y) if s["relu"] else y
    return {"dX": y, "dA": dA, "dB": dB}
