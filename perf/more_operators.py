"""Dropout without a stored mask, root-mean-square norm with the residual's addition, embedding with its gradient: the cases
that are timed and their plain forms.

Operators (own = True makes the framework's calls, own = False the plain form in torch):

  drop       y = kept * x * scale; the mask comes from a counter-based generator and a seed, which is an input (drop_bwd: of dy)
  rms_fwd    h = residual + drop(x), rstd = 1/sqrt(mean_c h^2 + eps), y = h * rstd * gamma over the C channels of every position
  rms_bwd    dz = rstd (g - xh mean_c(g xh)) + dh with g = dy * gamma, xh = h * rstd; dresidual = dz, dx = drop'(dz), dgamma = sum dy xh
  rms_8bit   y of rms_fwd (no dropout) in e4m3 with one scale a position, for serving
  embed      y = scale * W[token]
  embed_bwd  dW = scale * sum of dy over the positions of each token

Layouts of the norm: "rows" is [rows, C] (channels-last activations, tokens), "planes" is [B, C, H, W].

The generator: element e of a tensor in memory order takes bits 16*(e%4) .. 16*(e%4)+15 of word e//4, word k is
fin(key + GAMMA * (k+1)) with key = fin((seed ^ STREAM) + GAMMA); it is dropped if they are below round(65536 p).
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda:0"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}
EPS = 1e-6
TOP8, LEAST8 = 448.0, 2.0 ** -100       # e4m3's largest value; the least magnitude that a row's scale goes by
GAMMA, M1, M2, STREAM = 0x9E3779B97F4A7C15, 0xBF58476D1CE4E5B9, 0x94D049BB133111EB, 0x3C6EF372FE94F82B


# ---- cases ---------------------------------------------------------------------------------------------------------
def _drop(name, op, n, dtype, p):
    return {"name": name, "op": op, "n": n, "dtype": dtype, "p": p}


def _rows(name, op, rows, channels, dtype, wtype, residual=False, p=0.0):
    return {"name": name, "op": op, "layout": "rows", "rows": rows, "C": channels, "dtype": dtype, "wtype": wtype, "residual": residual, "p": p}


def _planes(name, op, batch, channels, height, width, dtype, wtype, residual=False, p=0.0):
    return {"name": name, "op": op, "layout": "planes", "B": batch, "C": channels, "H": height, "W": width, "dtype": dtype, "wtype": wtype,
            "residual": residual, "p": p}


def _embed(name, op, n, rows, channels, dtype, tokens, scale):
    return {"name": name, "op": op, "N": n, "V": rows, "C": channels, "dtype": dtype, "tokens": tokens, "scale": scale}


def listed():
    return [
        # behind the smallest benchmark layer (C1): latency counts
        _drop("drop C1 f32", "drop", 4 * 16 * 32 * 32, "f32", 0.1),
        # the gradient of the headline layer's activation (C5) in its storage type, at the common rate of wide layers
        _drop("drop bwd C5 f16", "drop_bwd", 256 * 256 * 28 * 28, "f16", 0.5),
        # the end of a residual branch over channels-last activations of C3's input
        _rows("rms fwd C3 rows bf16", "rms_fwd", 64 * 56 * 56, 128, "bf16", "f32", True, 0.1),
        # a ragged small layer: odd channels and odd planes
        _planes("rms fwd ragged planes f16", "rms_fwd", 7, 37, 19, 23, "f16", "f16", True),
        # few long rows: a batch of token vectors in a wide network
        _rows("rms bwd long rows bf16", "rms_bwd", 4096, 4096, "bf16", "bf16", True),
        # the headline layer's activation, whole residual block end
        _planes("rms bwd C5 planes f16", "rms_bwd", 256, 256, 28, 28, "f16", "f32", True, 0.1),
        # serving, single tokens
        _rows("rms 8bit 1 token bf16", "rms_8bit", 1, 4096, "bf16", "bf16", True),
        # serving, a long prompt with rows of an odd length: no row but the first is aligned
        _rows("rms 8bit odd rows f16", "rms_8bit", 8192, 5001, "f16", "f16"),
        # serving, single tokens of a text vocabulary
        _embed("embed 8 tokens bf16", "embed", 8, 32000, 4096, "bf16", "zipf", 1.0),
        # a code map of C2's extent (128 images of 32 x 32) over a small code book
        _embed("embed code map f32", "embed", 128 * 32 * 32, 1024, 64, "f32", "uniform", 8.0),
        # a ragged small batch of texts
        _embed("embed bwd 1999 tokens f16", "embed_bwd", 1999, 5003, 300, "f16", "zipf", 1.0),
        # a training batch of texts: a few tokens make up much of it
        _embed("embed bwd 64k tokens bf16", "embed_bwd", 32 * 2048, 50304, 512, "bf16", "zipf", 22.627416997969522),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["drop", "drop_bwd", "rms_fwd", "rms_bwd", "rms_8bit", "embed", "embed_bwd"])
    dtype = rng.choice(["f32", "bf16", "f16"])
    most = 50_000_000 if dtype != "f32" else 25_000_000
    if op.startswith("drop"):
        return {"op": op, "n": _log(rng, 100, most), "dtype": dtype, "p": rng.choice([0.05, 0.1, 0.25, 0.5, 0.9])}
    if op.startswith("rms"):
        wtype, residual = rng.choice(["f32", dtype]), rng.random() < 0.7
        p = 0.0 if op == "rms_8bit" else rng.choice([0.0, 0.0, 0.1, 0.3])
        elements = _log(rng, 500, most)
        if rng.random() < 0.6:
            channels = _log(rng, 8, 16384)
            return {"op": op, "layout": "rows", "rows": max(1, elements // channels), "C": channels, "dtype": dtype, "wtype": wtype, "residual": residual, "p": p}
        channels, height, width = _log(rng, 8, 1024), _log(rng, 4, 112), _log(rng, 4, 112)
        return {"op": op, "layout": "planes", "B": max(1, min(512, elements // (channels * height * width))), "C": channels, "H": height, "W": width,
                "dtype": dtype, "wtype": wtype, "residual": residual, "p": p}
    channels = _log(rng, 8, 4096)
    return {"op": op, "N": _log(rng, 1, min(500_000, most // channels)), "V": _log(rng, 2, min(200_000, most // channels)), "C": channels, "dtype": dtype,
            "tokens": rng.choice(["zipf", "uniform"]), "scale": rng.choice([1.0, math.sqrt(channels)])}


# ---- inputs --------------------------------------------------------------------------------------------------------
def _normal(gen, *shape):
    return torch.randn(shape, generator=gen, device=DEV, dtype=torch.float32)


def _probabilities(case):
    """Of the tokens: all alike, or falling with the rank as in texts."""
    if case["tokens"] == "uniform":
        return torch.full((case["V"],), 1.0 / case["V"], dtype=torch.float64, device="cpu")
    p = 1.0 / (torch.arange(case["V"], dtype=torch.float64, device="cpu") + 2.7)
    return p / p.sum()


def prepare(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    dt, op = TYPES[case["dtype"]], case["op"]
    s = {"op": op, "seed": (0x1234567 * seed + 11) & 0x7FFFFFFFFFFF, "p": case.get("p", 0.0)}
    if op.startswith("drop"):
        s["x"] = _normal(gen, case["n"]).to(dt)
        return s
    if op.startswith("rms"):
        ch, planes = case["C"], case["layout"] == "planes"
        shape = (case["B"], ch, case["H"], case["W"]) if planes else (case["rows"], ch)
        over = (1, ch, 1, 1) if planes else (1, ch)
        # channels of unlike size around a mean of their own, as a residual stream has them
        x = _normal(gen, *shape).mul_(0.5 + torch.rand(over, generator=gen, device=DEV)).add_(0.3 * _normal(gen, *over)).to(dt)
        s.update(axis=1 if planes else -1, gamma=(1 + 0.1 * _normal(gen, ch)).to(TYPES[case["wtype"]]))
        if op == "rms_bwd":
            s.update(h=x, dy=_normal(gen, *shape).mul_(0.1).to(dt), dh=_normal(gen, *shape).mul_(0.1).to(dt) if case["residual"] else None)
            s["rstd"] = (x.float().square().mean(s["axis"]) + EPS).rsqrt()
        else:
            s.update(x=x, residual=_normal(gen, *shape).to(dt) if case["residual"] else None)
        return s
    cdf = _probabilities(case).cumsum(0).to(DEV)
    u = torch.rand(case["N"], generator=gen, device=DEV, dtype=torch.float64)
    s.update(tokens=torch.searchsorted(cdf, u).clamp_(max=case["V"] - 1), V=case["V"], scale=case["scale"])
    if op == "embed":
        s["W"] = _normal(gen, case["V"], case["C"]).to(dt)
    else:
        s["dy"] = _normal(gen, case["N"], case["C"]).mul_(0.1).to(dt)
    return s


# ---- one pass ------------------------------------------------------------------------------------------------------
def _signed(v):
    return v - (1 << 64) if v >> 63 else v


def _shift(z, k):
    """A logical shift to the right of 64-bit words that torch holds as signed."""
    return (z >> k) & ((1 << (64 - k)) - 1)


def _fin(z):
    z = (z ^ _shift(z, 30)) * _signed(M1)
    z = (z ^ _shift(z, 27)) * _signed(M2)
    return z ^ _shift(z, 31)


def _fin_int(z):
    mask = (1 << 64) - 1
    z = ((z ^ (z >> 30)) * M1) & mask
    z = ((z ^ (z >> 27)) * M2) & mask
    return z ^ (z >> 31)


def _rate(p):
    """(values of 65536 that are dropped, the factor of the others)."""
    q = int(65536 * p + 0.5)
    return q, 65536.0 / (65536 - q)


def _plain_drop(x, p, seed):
    """In 32 bits, in the shape of x."""
    q, scale = _rate(p)
    key = _fin_int(((seed ^ STREAM) + GAMMA) & ((1 << 64) - 1))
    n = x.numel()
    words = _fin(torch.arange(1, (n + 3) // 4 + 1, device=x.device, dtype=torch.int64) * _signed(GAMMA) + _signed(key))
    fields = torch.stack([words & 0xFFFF, (words >> 16) & 0xFFFF, (words >> 32) & 0xFFFF, (words >> 48) & 0xFFFF], 1).view(-1)[:n]
    return torch.where((fields >= q).view(x.shape), x.float() * scale, 0.0)


def _over_channels(t, axis):
    return t.float().view(1, -1, 1, 1) if axis == 1 else t.float()


def _plain_rms(s):
    """(h, rstd with the axis, y) in 32 bits."""
    h = s["x"].float() if s["p"] == 0.0 else _plain_drop(s["x"], s["p"], s["seed"])
    if s["residual"] is not None:
        h = h + s["residual"].float()
    rstd = (h.square().mean(s["axis"], keepdim=True) + EPS).rsqrt()
    return h, rstd, h * rstd * _over_channels(s["gamma"], s["axis"])


def _plain_rms_bwd(s):
    axis = s["axis"]
    dy, rstd = s["dy"].float(), s["rstd"].unsqueeze(axis)
    xh = s["h"].float() * rstd
    dgamma = (dy * xh).sum((0, 2, 3) if axis == 1 else (0,))
    g = dy * _over_channels(s["gamma"], axis)
    dz = (g - xh * (g * xh).mean(axis, keepdim=True)) * rstd
    if s["dh"] is not None:
        dz = dz + s["dh"].float()
    dt = s["h"].dtype
    dx = dz if s["p"] == 0.0 else _plain_drop(dz, s["p"], s["seed"])
    return dx.to(dt), dz.to(dt), dgamma.to(s["gamma"].dtype)


def run(s):
    op = s["op"]
    changed = op == "rms_fwd" or op == "rms_8bit"
    changed = changed and (s["residual"] is not None or s["p"] != 0.0)       # whether h is another tensor than x
    if own:
        from paper_2106_06998_amd import dropout, embedding, norm
        if op == "drop":
            return dropout.dropout_forward(s["x"], s["p"], s["seed"])
        if op == "drop_bwd":
            return dropout.dropout_backward(s["x"], s["p"], s["seed"])
        if op == "rms_fwd":
            y, h, rstd = norm.rms_norm_forward(s["x"], s["gamma"], s["residual"], EPS, s["axis"], s["p"], s["seed"])
            return (y, h, rstd) if changed else (y, rstd)
        if op == "rms_bwd":
            return norm.rms_norm_backward(s["dy"], s["h"], s["rstd"], s["gamma"], s["dh"], s["axis"], s["p"], s["seed"])
        if op == "rms_8bit":
            q, scale, h = norm.rms_norm_8bit(s["x"], s["gamma"], s["residual"], EPS, s["axis"], torch.float8_e4m3fn)
            return (q, scale, h) if changed else (q, scale)
        if op == "embed":
            return embedding.embedding_forward(s["tokens"], s["W"], s["scale"])
        return embedding.embedding_backward(s["dy"], s["tokens"], s["V"], s["scale"])
    if op.startswith("drop"):
        return _plain_drop(s["x"], s["p"], s["seed"]).to(s["x"].dtype)
    if op == "rms_bwd":
        return _plain_rms_bwd(s)
    if op == "rms_fwd":
        h, rstd, y = _plain_rms(s)
        dt = s["x"].dtype
        return (y.to(dt), h.to(dt), rstd.squeeze(s["axis"])) if changed else (y.to(dt), rstd.squeeze(s["axis"]))
    if op == "rms_8bit":
        h, _, y = _plain_rms(s)
        scale = y.abs().amax(s["axis"], keepdim=True).clamp(min=LEAST8) / TOP8
        q = (y / scale).to(torch.float8_e4m3fn)
        return (q, scale.squeeze(s["axis"]), h.to(s["x"].dtype)) if changed else (q, scale.squeeze(s["axis"]))
    if op == "embed":
        return (s["W"].index_select(0, s["tokens"]).float() * s["scale"]).to(s["W"].dtype)
    dw = torch.zeros(s["V"], s["dy"].shape[1], device=s["dy"].device, dtype=torch.float32)
    return (dw.index_add_(0, s["tokens"], s["dy"].float()) * s["scale"]).to(s["dy"].dtype)


# ---- what a pass cannot do without ---------------------------------------------------------------------------------
def work(case):
    size, op = SIZE[case["dtype"]], case["op"]
    if op.startswith("drop"):
        return {"bytes": 2 * case["n"] * size, "flops": 12 * case["n"]}
    if op.startswith("rms"):
        ch = case["C"]
        rows = case["rows"] if case["layout"] == "rows" else case["B"] * case["H"] * case["W"]
        n, w, more = rows * ch, ch * SIZE[case["wtype"]], 12 * rows * ch if case["p"] else 0
        if op == "rms_bwd":
            return {"bytes": (3 + case["residual"] + (case["p"] != 0.0)) * n * size + 4 * rows + 2 * w, "flops": 10 * n + more}
        changed = case["residual"] or case["p"] != 0.0
        return {"bytes": (1 + case["residual"] + changed) * n * size + n * (size if op == "rms_fwd" else 1) + 4 * rows + w, "flops": 6 * n + more}
    n, values = case["N"], case["N"] * case["C"]
    if op == "embed":
        met = float((1 - (1 - _probabilities(case)).pow(n)).sum())       # rows of the table that the tokens name
        return {"bytes": 8 * n + (values + met * case["C"]) * size, "flops": values}
    return {"bytes": 8 * n + (values + case["V"] * case["C"]) * size, "flops": values}


# ---- the definitions in 64 bits ------------------------------------------------------------------------------------
def _kept(n, p, seed):
    """0 or 1 / (share that is kept) of n values, from unsigned words on the host."""
    with np.errstate(over="ignore"):
        def fin(z):
            z = (z ^ (z >> np.uint64(30))) * np.uint64(M1)
            z = (z ^ (z >> np.uint64(27))) * np.uint64(M2)
            return z ^ (z >> np.uint64(31))
        key = fin(np.array([seed ^ STREAM], dtype=np.uint64) + np.uint64(GAMMA))
        words = fin(key + np.uint64(GAMMA) * np.arange(1, n // 4 + 2, dtype=np.uint64))
    fields = words.astype("<u8").view("<u2")[:n]
    dropped = int(65536 * p + 0.5)
    keep = torch.from_numpy(np.greater_equal(fields, dropped)).to(DEV)
    return keep.double() * (65536.0 / (65536 - dropped))


def exact(case, seed):
    s = prepare(case, seed)
    op, p = s["op"], s["p"]
    if op.startswith("drop"):
        return s["x"].double() * _kept(case["n"], p, s["seed"])
    if op == "embed":
        return s["W"].double()[s["tokens"]] * s["scale"]
    if op == "embed_bwd":
        order = torch.argsort(s["tokens"], stable=True)
        first = torch.searchsorted(s["tokens"][order].contiguous(), torch.arange(s["V"] + 1, device=DEV))
        sums = torch.cat([torch.zeros(1, s["dy"].shape[1], dtype=torch.float64, device=DEV), s["dy"][order].double().cumsum(0)])
        return s["scale"] * (sums[first[1:]] - sums[first[:-1]])
    planes = s["axis"] == 1

    def flat(t):
        return (t.permute(0, 2, 3, 1).reshape(-1, t.shape[1]) if planes else t).double()

    like = s["h"] if op == "rms_bwd" else s["x"]
    n = like.shape[1]

    def back(t):
        return t.view(like.shape[0], *like.shape[2:], n).permute(0, 3, 1, 2).contiguous() if planes else t

    def stat(t):
        return t.view(like.shape[0], *like.shape[2:]) if planes else t.view(-1)

    gamma = s["gamma"].double()
    kept = flat(_kept(like.numel(), p, s["seed"]).view(like.shape)) if p else None
    if op == "rms_bwd":
        dy, h, r = flat(s["dy"]), flat(s["h"]), s["rstd"].double().reshape(-1, 1)
        g = dy * gamma
        dz = r * g - r ** 3 / n * h * (g * h).sum(1, keepdim=True)
        if s["dh"] is not None:
            dz += flat(s["dh"])
        return back(dz if kept is None else dz * kept), back(dz), (dy * h * r).sum(0)
    h = flat(s["x"])
    if kept is not None:
        h = h * kept
    if s["residual"] is not None:
        h = h + flat(s["residual"])
    r = 1 / torch.sqrt(torch.linalg.vector_norm(h, dim=1, keepdim=True) ** 2 / n + EPS)
    y = h * r * gamma
    more = [back(h)] if kept is not None or s["residual"] is not None else []
    if op == "rms_fwd":
        return (back(y), *more, stat(r))
    scale = torch.linalg.vector_norm(y, ord=math.inf, dim=1, keepdim=True).clamp(min=LEAST8) / TOP8
    return (back(y / scale), stat(scale), *more)
