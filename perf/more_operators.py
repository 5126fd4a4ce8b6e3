"""The operators on a layer's residual stream, as cases to be timed through the public entry points.

A case is one pass over `rows` rows (tokens, positions, samples, heads) of `cols` columns. Three kinds:

    drop   dropout, with or without the addition of a residual (`dropout`); the gradient is the same call
    norm   total = residual + dropout(x) and its root-mean-square norm (`rms_norm`), whole or, with `bits8`, as e4m3 codes with
           scales by the row (group 0) or by groups of columns
    back   the gradient of that (`rms_norm_backward`): of the residual, of x, of the weight

With `own` the framework's kernels run, without it the same formulas in elementary torch operations, in 32 bits.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
SEED, EPS = 1_906_02367, 1e-5


def _case(name, kind, rows, cols, **kw):
    c = dict(kind=kind, rows=rows, cols=cols, type="bf16", pad=0, p=0.0, residual=False, weight="same", bits8=False, group=0)
    c.update(kw)
    if name is not None:
        c["name"] = name
    return c


def listed():
    return [
        # the local step of the softmax regression: mini-batches of 8 for 15 workers, 784 features and the constant one
        _case("drop_120x785", "drop", 120, 785, type="fp32", p=0.2),
        # a layer's output in training, dropped out and added to the residual stream
        _case("drop_8192x4096_residual", "drop", 8192, 4096, p=0.1, residual=True),
        # an inner layer of odd width in 16-bit floats, padded rows
        _case("drop_4095x11009", "drop", 4095, 11009, type="fp16", p=0.5, pad=7),
        # serving, a single token: latency is all there is
        _case("norm_1x4096", "norm", 1, 4096, residual=True),
        # the features of all samples of the softmax regression
        _case("norm_6000x785", "norm", 6000, 785, type="fp32"),
        # every head of a batch of tokens by itself
        _case("norm_131072x128", "norm", 131072, 128, weight="fp32"),
        # a layer of a training step: the dropped-out output joins the residual stream and is normed for the next one
        _case("norm_16384x4096_drop", "norm", 16384, 4096, p=0.1, residual=True),
        # serving, a batch of tokens, for a product in 8 bits with a scale per token
        _case("norm8_64x8192", "norm", 64, 8192, residual=True, bits8=True),
        # a long prompt, for a product in 8 bits with a scale per 128 columns
        _case("norm8_8192x8192_g128", "norm", 8192, 8192, residual=True, bits8=True, group=128),
        # the features' norm in the local step, backward
        _case("back_120x785", "back", 120, 785, type="fp32", p=0.2),
        # the training step's layer, backward
        _case("back_16384x4096_drop", "back", 16384, 4096, p=0.1, residual=True),
        # odd and wide rows in 16-bit floats, weights in 32 bits
        _case("back_2047x12289", "back", 2047, 12289, type="fp16", pad=5, residual=True, weight="fp32"),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["drop", "norm", "norm", "norm", "back", "back"])
    cols = _log_uniform(rng, 8, 16_384)
    if rng.random() < 0.5:                                                  # the widths that most models have
        cols = max(8, cols // 64 * 64)
    rows = _log_uniform(rng, 1, max(2, min(131_072, 30_000_000 // cols)))
    bits8 = kind == "norm" and rng.random() < 0.4
    return _case(None, kind, rows, cols, type=rng.choice(["fp32", "bf16", "bf16", "fp16"]), pad=rng.choice([0, 0, 1, 24]),
                 p=rng.choice([0.05, 0.1, 0.2, 0.5]) if kind == "drop" or (not bits8 and rng.random() < 0.5) else 0.0, residual=rng.random() < 0.6,
                 weight=rng.choice(["same", "same", "fp32", "none"]), bits8=bits8, group=rng.choice([0, 0, 32, 64, 128]) if bits8 else 0)


def prepare(case, seed):
    dev = torch.device("cuda")
    g = torch.Generator(device=dev)
    g.manual_seed(seed * 7919 + 29)
    N, C, dt = case["rows"], case["cols"], TYPES[case["type"]]

    def rows(spread):
        held = torch.full((N, C + case["pad"]), float("nan"), dtype=dt, device=dev)      # what lies behind a row is not looked at
        v = held[:, :C]
        v.copy_(torch.randn(N, C, generator=g, device=dev).mul_(spread))
        return v

    # a residual stream: some columns are far larger than the others, and some rows
    spread = torch.exp(0.5 * torch.randn(C, generator=g, device=dev)) * torch.exp(0.3 * torch.randn(N, 1, generator=g, device=dev))
    spread = torch.where(torch.rand(C, generator=g, device=dev) < 0.004, 20.0 * spread, spread)
    s = dict(case=case, drop=dict(p=case["p"], seed=SEED + seed, round=seed % 1000, row0=seed % 7 * N), weight=None)
    empty = lambda dtype: torch.empty(N, C, dtype=dtype, device=dev)
    if case["kind"] != "drop" and case["weight"] != "none":
        s["weight"] = (1.0 + 0.2 * torch.randn(C, generator=g, device=dev)).to(torch.float32 if case["weight"] == "fp32" else dt)
    if case["kind"] == "back":
        s.update(total=rows(spread), dy=rows(0.1), dtotal=rows(0.1) if case["residual"] else None, dresidual=empty(dt))
        if case["p"] > 0:
            s["dx"] = empty(dt)
        if s["weight"] is not None:
            s["dweight"] = torch.empty(C, dtype=torch.float32, device=dev)
        return s
    s.update(x=rows(1.0 if case["residual"] else spread), residual=rows(spread) if case["residual"] else None)
    if case["kind"] == "drop":
        s["y"] = empty(dt)
        return s
    if case["residual"] or case["p"] > 0:                                   # else x is the total itself
        s["total"] = empty(dt)
    s["y"] = empty(torch.float8_e4m3fn if case["bits8"] else dt)
    if case["bits8"]:
        s["scales"] = torch.empty(N, -(-C // case["group"]) if case["group"] else 1, device=dev)
    return s


OUTPUTS = {"drop": ("y",), "norm": ("total", "y", "scales"), "back": ("dresidual", "dx", "dweight")}


# ---------------------------------------------------------------------------------------------
# the plain form
# ---------------------------------------------------------------------------------------------
def _plain_words(drop, N, units, dev):
    """Philox4x32-10 of every row's units of eight columns: four words of 32 bits, held in 64."""
    low = 0xFFFFFFFF
    c0 = torch.arange(units, device=dev).expand(N, units)
    c1 = ((torch.arange(N, device=dev) + drop["row0"]) & low).unsqueeze(1)
    c2, c3 = drop["round"] & low, drop["round"] >> 32 | 2 << 30
    k0, k1 = drop["seed"] & low, drop["seed"] >> 32
    for _ in range(10):
        a, b = c0 * 0xD2511F53, c2 * 0xCD9E8D57
        c0, c1, c2, c3 = (b >> 32 & low) ^ c1 ^ k0, b & low, (a >> 32 & low) ^ c3 ^ k1, a & low
        k0, k1 = k0 + 0x9E3779B9 & low, k1 + 0xBB67AE85 & low
    return torch.stack((c0, c1, c2, c3), 2)


def _plain_drop(s, v):
    drop, (N, C) = s["drop"], v.shape
    if not drop["p"]:
        return v
    T = int(math.floor((1.0 - drop["p"]) * 65536.0 + 0.5))
    w = _plain_words(drop, N, -(-C // 8), v.device)
    keep = torch.stack((w & 0xFFFF, w >> 16), 3).reshape(N, -1)[:, :C] < T
    return torch.where(keep, v * (65536.0 / T), 0.0)


def _plain_norm(s):
    case = s["case"]
    h = _plain_drop(s, s["x"].float())
    if s["residual"] is not None:
        h = h + s["residual"].float()
    out = {}
    if "total" in s:
        out["total"] = h.to(s["x"].dtype)
    y = h * torch.rsqrt((h * h).mean(1, keepdim=True) + EPS)
    if s["weight"] is not None:
        y = y * s["weight"].float()
    if not case["bits8"]:
        out["y"] = y.to(s["x"].dtype)
        return out
    N, C = y.shape
    size = case["group"] or C
    groups = torch.nn.functional.pad(y, (0, -C % size)).view(N, -1, size)
    most = groups.abs().amax(2, keepdim=True).clamp_min(2.0 ** -100)
    out["y"] = (groups * (448.0 / most)).view(N, -1)[:, :C].to(torch.float8_e4m3fn)
    out["scales"] = (most / 448.0).squeeze(2)
    return out


def _plain_back(s):
    h, dy = s["total"].float(), s["dy"].float()
    r = torch.rsqrt((h * h).mean(1, keepdim=True) + EPS)
    u = h * r
    g = dy if s["weight"] is None else dy * s["weight"].float()
    d = r * (g - u * (g * u).mean(1, keepdim=True))
    if s["dtotal"] is not None:
        d = d + s["dtotal"].float()
    out = dict(dresidual=d.to(s["total"].dtype))
    if "dx" in s:
        out["dx"] = _plain_drop(s, d).to(s["total"].dtype)
    if "dweight" in s:
        out["dweight"] = (dy * u).sum(0)
    return out


def _own(s):
    from paper_1906_02367_amd import binding as B
    kind = s["case"]["kind"]
    if kind == "drop":
        B.dropout(s["x"], s["y"], residual=s["residual"], **s["drop"])
    elif kind == "norm":
        B.rms_norm(s["x"], s["y"], weight=s["weight"], eps=EPS, residual=s["residual"], total=s.get("total"), scales=s.get("scales"),
                   group=s["case"]["group"], **s["drop"])
    else:
        B.rms_norm_backward(s["total"], s["dy"], weight=s["weight"], eps=EPS, dtotal=s["dtotal"], dresidual=s["dresidual"], dx=s.get("dx"),
                            dweight=s.get("dweight"), **s["drop"])
    return {n: s[n] for n in OUTPUTS[kind] if n in s}


def run(state):
    if own:
        return _own(state)
    kind = state["case"]["kind"]
    if kind == "norm":
        return _plain_norm(state)
    if kind == "back":
        return _plain_back(state)
    y = _plain_drop(state, state["x"].float())
    if state["residual"] is not None:
        y = y + state["residual"].float()
    return dict(y=y.to(state["x"].dtype))


def work(case):
    n, b, kind = case["rows"] * case["cols"], 4 if case["type"] == "fp32" else 2, case["kind"]
    weight = 0 if kind == "drop" or case["weight"] == "none" else case["cols"] * (4 if case["weight"] == "fp32" else b)
    arrays = 2 + case["residual"]                                           # x, y, residual; total, dy and dresidual, dtotal
    if kind == "back":
        arrays += 1 + (case["p"] > 0)
        weight += 4 * case["cols"] if weight else 0
    if kind == "norm":
        arrays += case["residual"] or case["p"] > 0
    small = 0
    if case["bits8"]:
        small = n * (1 - b) + 4 * case["rows"] * (-(-case["cols"] // case["group"]) if case["group"] else 1)
    return {"bytes": arrays * n * b + weight + small, "flops": n * {"drop": 2, "norm": 6, "back": 12}[kind]}


# ---------------------------------------------------------------------------------------------
# the definition in 64 bits
# ---------------------------------------------------------------------------------------------
def _exact_keep(case, drop):
    """1 / (the share that is kept) where a value is kept, 0 elsewhere; the generator in unsigned numbers on the host."""
    N, C = case["rows"], case["cols"]
    units = (C + 7) // 8
    u32 = np.uint64(0xFFFFFFFF)
    word = [np.broadcast_to(np.arange(units, dtype=np.uint64), (N, units)),
            np.broadcast_to(((np.arange(N, dtype=np.uint64) + np.uint64(drop["row0"])) & u32)[:, None], (N, units)),
            np.uint64(drop["round"]) & u32, np.uint64((drop["round"] >> 32) + 2 ** 31)]
    key = [drop["seed"] % 2 ** 32, drop["seed"] // 2 ** 32]
    for _ in range(10):
        first, second = word[0] * np.uint64(0xD2511F53), word[2] * np.uint64(0xCD9E8D57)
        word = [(second >> np.uint64(32)) ^ word[1] ^ np.uint64(key[0]), second & u32, (first >> np.uint64(32)) ^ word[3] ^ np.uint64(key[1]), first & u32]
        key = [(key[0] + 0x9E3779B9) % 2 ** 32, (key[1] + 0xBB67AE85) % 2 ** 32]
    piece = np.stack([np.broadcast_to(w, (N, units)) for w in word], axis=2).astype("<u4").view("<u2").reshape(N, units * 8)[:, :C]
    kept = round((1.0 - drop["p"]) * 65536)
    return (torch.from_numpy(piece.astype(np.int32)).cuda() < kept).double() * (65536.0 / kept)


def _exact_e4m3(v):
    """The nearest of the values that e4m3 holds, |v| <= 448; ties to the even one."""
    _, e = torch.frexp(v)
    step = torch.exp2((e - 1).clamp_min(-6).double() - 3.0)
    return torch.round(v / step) * step


def exact(case, seed):
    s = prepare(case, seed)
    kind, C = case["kind"], case["cols"]
    factor = _exact_keep(case, s["drop"]) if case["p"] > 0 else 1.0
    w = 1.0 if s["weight"] is None else s["weight"].double()
    if kind == "back":
        h, dy = s["total"].double(), s["dy"].double()
        rms = torch.sqrt(torch.linalg.vector_norm(h, dim=1, keepdim=True) ** 2 / C + EPS)
        out = {}
        if "dweight" in s:
            out["dweight"] = torch.einsum("nc,nc->c", dy, h / rms)
        d = dy * w / rms - h * ((dy * w * h).sum(1, keepdim=True) / (C * rms ** 3))
        if s["dtotal"] is not None:
            d += s["dtotal"].double()
        out["dresidual"] = d
        if "dx" in s:
            out["dx"] = d * factor
        return out
    h = s["x"].double() * factor
    if s["residual"] is not None:
        h += s["residual"].double()
    if kind == "drop":
        return dict(y=h)
    out = dict(total=h) if "total" in s else {}
    y = h / torch.sqrt(torch.linalg.vector_norm(h, dim=1, keepdim=True) ** 2 / C + EPS) * w
    if case["bits8"]:
        size = case["group"] or C
        most = torch.stack([part.abs().amax(1) for part in y.split(size, 1)], 1).clamp_min(2.0 ** -100)
        out["scales"] = most / 448
        y = _exact_e4m3(y / out["scales"].repeat_interleave(size, 1)[:, :C])
    out["y"] = y
    return out
