"""The operators on a residual stream in 64 bits, from their definitions, and how far 32-bit results may be off.

Tolerances.  u = 2^-24 (half a step of fp32), 64-bit roundings left out.  A row's sum: a thread adds at most 32 values, then at most 6 steps within
a wave and 16 over the waves: SUM = 54 roundings relative to the sum of the terms' sizes.  Each function below adds up the roundings of its own formula.
An output of fewer bits adds half a step of its type, eps / 2 relative, and half a step of its subnormals."""
import math

import numpy as np
import torch

U = 2.0 ** -24
SUM = 54
INF = float("inf")
SUBNORMAL = {torch.float32: 2.0 ** -149, torch.bfloat16: 2.0 ** -133, torch.float16: 2.0 ** -24, torch.float8_e4m3fn: 2.0 ** -9}
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}


def philox(c0, c1, c2, c3, k0, k1):
    """Philox4x32-10 on arrays of unsigned numbers below 2^32, held in 64 bits."""
    low, s = np.uint64(0xFFFFFFFF), np.uint64(32)
    c0, c1, c2, c3 = (np.asarray(c, dtype=np.uint64) for c in (c0, c1, c2, c3))
    for _ in range(10):
        a, b = c0 * np.uint64(0xD2511F53), c2 * np.uint64(0xCD9E8D57)
        c0, c1, c2, c3 = (b >> s) ^ c1 ^ np.uint64(k0), b & low, (a >> s) ^ c3 ^ np.uint64(k1), a & low
        k0, k1 = (k0 + 0x9E3779B9) & 0xFFFFFFFF, (k1 + 0xBB67AE85) & 0xFFFFFFFF
    return c0, c1, c2, c3


def threshold(p):
    return math.floor((1.0 - p) * 65536.0 + 0.5)


def kept(rows, cols, p, seed=0, round=0, row0=0):
    """Which values are kept, [rows, cols], one at a time from the header's words."""
    T = threshold(p)
    i = np.arange(cols)
    n = (row0 + np.arange(rows, dtype=np.uint64))[:, None]
    r = round % 2 ** 62
    unit = np.broadcast_to((i // 8).astype(np.uint64), (rows, cols))
    words = np.stack(philox(unit, np.broadcast_to(n, (rows, cols)), r & 0xFFFFFFFF, r >> 32 | 2 << 30, seed & 0xFFFFFFFF, seed >> 32))
    piece = i % 8
    word = words[piece // 2, np.arange(rows)[:, None], i[None, :]]
    return torch.from_numpy((((word >> np.uint64(16)) * (piece % 2) + (word & np.uint64(0xFFFF)) * (1 - piece % 2)) < T))


def rounding(x, tol, dtype):
    return torch.finfo(dtype).eps / 2 * (x.abs() + tol) + SUBNORMAL[dtype] / 2


def dropped(v, keep, p):
    """drop(v) and its tolerance: the factor and the product are rounded."""
    T = threshold(p)
    d = torch.where(keep, v * (65536.0 / T if T else 0.0), 0.0)
    return d, (2 * U * d.abs() if p > 0 else torch.zeros_like(d))


def total_of(x, residual=None, keep=None, p=0.0):
    """residual + drop(x) and its tolerance before it is stored: one more rounding."""
    h = x.detach().cpu().double()
    tol = torch.zeros_like(h)
    if keep is not None:
        h, tol = dropped(h, keep, p)
    if residual is not None:
        h = h + residual.detach().cpu().double()
        tol = tol * 1.01 + U * h.abs()
    return h, tol


def norm_of(h, tol, weight, eps):
    """y = w h r, r = 1 / sqrt(sum h^2 / C + eps).  The sum is off by 2 |h| tol_h a term and SUM u; the quotient and the sum with eps add 2 u, the root
    takes half of that and adds 1 u, its inverse 1 u; the two products 2 u."""
    C = h.shape[1]
    w = torch.ones(C, dtype=torch.float64) if weight is None else weight.detach().cpu().double()
    ss = (h * h).sum(1, keepdim=True)
    ms = ss / C + eps
    rel = 0.5 * (((2 * h.abs() * tol).sum(1, keepdim=True) + SUM * U * ss) / C / ms + 2 * U) + 2 * U
    y = h / torch.sqrt(ms) * w
    return y, 1.01 * (w.abs() / torch.sqrt(ms) * tol + y.abs() * (rel + 2 * U))


def scales_of(y, tol, group, Q):
    """Per group: max(a, 2^-100) / Q, its tolerance (that of the largest value, and a division), and both spread over the columns."""
    C = y.shape[1]
    size = group or C
    a = torch.stack([q.abs().amax(1) for q in y.split(size, 1)], 1).clamp_min(2.0 ** -100)
    t = torch.stack([q.amax(1) for q in tol.split(size, 1)], 1)
    return a / Q, 1.01 * t / Q + 2 * U * a / Q, (a / Q).repeat_interleave(size, 1)[:, :C]


def backward(h, dy, weight, eps, dtotal=None):
    """dresidual, dw before they are stored, and their tolerances.  u_i = h_i r: the root's roundings (SUM / 2 + 3) and 1.  g = w dy: 1.  The mean of
    g u: g, the products with h, SUM, then r, the product and the quotient.  The difference: u mean 1 and itself 1, times r 2.  dw: each term as u
    and 1, and a sum of at most `rows` terms and 112 steps over a block's rows and the blocks."""
    h, dy = h.detach().cpu().double(), dy.detach().cpu().double()
    N, C = h.shape
    w = torch.ones(C, dtype=torch.float64) if weight is None else weight.detach().cpu().double()
    r = 1 / torch.sqrt((h * h).sum(1, keepdim=True) / C + eps)
    rr = (SUM / 2 + 3) * U
    un, g = h * r, dy * w
    mean = (g * un).mean(1, keepdim=True)
    t_mean = (SUM + 2) * U * (g * un).abs().mean(1, keepdim=True) + mean.abs() * (rr + 2 * U)
    inner = g - un * mean
    t_inner = U * g.abs() + un.abs() * t_mean + (un * mean).abs() * (rr + 2 * U) + U * inner.abs()
    d = r * inner
    tol = 1.01 * (r * t_inner + d.abs() * (rr + 2 * U))
    if dtotal is not None:
        d = d + dtotal.detach().cpu().double()
        tol = tol + U * (d.abs() + tol)
    terms = dy * un
    return d, tol, terms.sum(0), 1.01 * U * (SUM / 2 + 6 + N + 112) * terms.abs().sum(0)


def check(got, want, tol, what):
    got = got.detach().cpu().double()
    nan = torch.isnan(want)
    assert torch.equal(torch.isnan(got), nan), f"{what}: NaN at other places"
    inf = torch.isinf(want)
    assert torch.equal(got[inf], want[inf]) and not torch.isinf(got[~inf]).any(), f"{what}: infinities at other places"
    fine = ~(nan | inf)
    off = (got - want).abs()[fine] - tol.expand_as(want)[fine]
    if off.numel() and float(off.max()) > 0:
        at = int(off.argmax())
        raise AssertionError(f"{what}: {float(got[fine][at])} instead of {float(want[fine][at])}, allowed {float(tol.expand_as(want)[fine][at]):.3g}, "
                             f"{int((off > 0).sum())} of {off.numel()} values off")
