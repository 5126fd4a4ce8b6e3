"""The operators on logits in 64 bits, row by row from their definitions, and how far 32-bit results may be off.

Tolerances.  u = 2^-24 (half a step of fp32).  y = (z - m) c log2(e) carries at most 4 roundings (the difference, the constant, its product
with c, the product), exp2 at most 2 more: e_i is off by (4 |d_i| + 4) u relative, d_i = c (z_i - m).  A sum over V terms is
made by threads of at most n values each, n = 80 + V / 1024 (a multiple of it for rows that threads of one wave hold), each
value and each change of the running maximum (at most one per value) one rounding, and at most 64 steps to join them:
relative error (2 n + 64) u of a sum of terms of one sign.  With D1 = sum p |d|, D2 = sum p d^2 the logarithm L of the sum is then off by
  tol_L = u (2 n + 64 + 4 D1 + |L|).
Everything else follows by adding up the terms of the formulas; each function below says how.  An output of fewer bits adds half
a step of its type, eps / 2 relative, and half a step of its subnormals."""
import math

import torch

U = 2.0 ** -24
INF = float("inf")
# a step among the smallest values: exp2 gives 0 below 2^-126, here times up to 2^6; fp16 has subnormals of its own
SUBNORMAL = {torch.float32: 2.0 ** -119, torch.bfloat16: 2.0 ** -119, torch.float16: 2.0 ** -24}


def rows_of(logits, c):
    """Per row: d = c (z - m), L, logp, p, and what the tolerances need."""
    z = logits.detach().cpu().double()
    N, V = z.shape
    m = z.amax(1, keepdim=True) if V else z
    empty = m == -INF
    d = c * (z - torch.where(empty, 0.0, m))
    s = torch.exp(d).sum(1, keepdim=True)
    L = torch.log(s)
    logp = torch.where(d == -INF, -INF, d - L)
    p = torch.where(empty, 0.0, torch.exp(logp))
    fin = torch.where(d > -INF, d, 0.0)
    D1, D2 = (p * fin.abs()).sum(1, keepdim=True), (p * fin * fin).sum(1, keepdim=True)
    n = 80 + V / 1024
    sums = 2 * n + 64
    tol_L = U * (sums + 4 * D1 + torch.where(empty, 0.0, L.abs()))
    return dict(z=z, m=m, empty=empty, d=d, fin=fin, L=L, logp=logp, p=p, D1=D1, D2=D2, sums=sums, tol_L=tol_L, c=c,
                tol_logp=tol_L + U * (6 * fin.abs() + 2 * torch.where(empty, 0.0, L.abs()) + 4))


def entropy(r):
    """H = L - ln 2 w / s: L, the sum w (terms of one sign, each off by (4 |d| + 6) u relative), their quotient and difference."""
    plogp = torch.where(r["p"] > 0, r["p"] * r["logp"], 0.0)
    H = -plogp.sum(1, keepdim=True)
    tol = 2 * r["tol_L"] + U * (2 * r["sums"] * r["D1"] + 4 * r["D2"] + 8 * r["D1"] + H.abs())
    return torch.where(r["empty"], 0.0, H), tol


def target_logprob(r, target):
    V = r["z"].shape[1]
    t = target.cpu().long()
    lp = r["logp"].gather(1, t.clamp(0, V - 1).unsqueeze(1)).squeeze(1)
    tol = r["tol_logp"].gather(1, t.clamp(0, V - 1).unsqueeze(1)).squeeze(1)
    lp = torch.where(r["empty"].squeeze(1), -INF, lp)
    return torch.where(t < 0, 0.0, torch.where(t >= V, float("nan"), lp)), tol


def lse(r):
    x = r["c"] * r["m"] + r["L"]
    return torch.where(r["empty"], -INF, x).squeeze(1), (r["tol_L"] + 3 * U * (r["c"] * r["m"]).abs() + U * r["L"].abs()).squeeze(1)


def top(r, K):
    """The K largest, ties to the lower index, by a stable sort."""
    z, index = torch.sort(r["z"] + 0.0, dim=1, descending=True, stable=True)
    index = index[:, :K]
    lp = torch.where(r["empty"], -INF, r["logp"].gather(1, index))
    return index, lp, r["tol_logp"].gather(1, index)


def logprob_gradient(r, target, g, h, dtype):
    """dz_i = c ([i = t] g - p_i (g + h (logp_i + H))): p_i off by tol_logp relative, logp and H by theirs, and 8 roundings of the terms."""
    N, V = r["z"].shape
    c = r["c"]
    H, tol_H = entropy(r)
    gg = torch.zeros(N, 1, dtype=torch.float64) if g is None else g.cpu().double().unsqueeze(1)
    hh = torch.zeros(N, 1, dtype=torch.float64) if h is None else h.cpu().double().unsqueeze(1)
    t = None if target is None else target.cpu().long().unsqueeze(1)
    if t is not None:
        gg = torch.where(t < 0, 0.0, gg)
    lpH = torch.where(r["p"] > 0, r["logp"] + H, 0.0)
    dz = -c * r["p"] * (gg + hh * lpH)
    mag = c * r["p"] * (gg.abs() + hh.abs() * (H.abs() + 2 * torch.where(r["empty"], 0.0, r["L"].abs()) + r["fin"].abs()))
    tol = mag * (r["tol_logp"] + 12 * U) + c * r["p"] * hh.abs() * (tol_H + r["tol_logp"])
    tol = torch.where(r["p"] > 0, tol, 0.0)
    if t is not None and g is not None:
        given = ((t >= 0) & (t < V) & ~r["empty"]).double()
        dz.scatter_add_(1, t.clamp(0, V - 1), c * gg * given)
        tol.scatter_add_(1, t.clamp(0, V - 1), 3 * U * c * gg.abs() * given)
        dz = torch.where(t >= V, float("nan"), dz)
    dz = torch.where(r["empty"], 0.0, dz)
    return dz, tol + rounding(dz, tol, dtype)


def rounding(x, tol, dtype):
    return torch.finfo(dtype).eps / 2 * (x.abs() + tol) + SUBNORMAL[dtype] / 2


def distill(r, index, value, c_t, t_lse, g, dtype):
    """loss, its tolerance, dz, its tolerance.  The entries' part is computed in 64 bits from the row's sums, so the loss is off by
    what the sums put into logp (and, with the rest as a class, into the sum outside): tol_L each, weighed with the teacher's
    probabilities, and its rounding to 32 bits; the teacher's own terms by far less.  A gradient c g p_i is off by tol_logp relative, c g q_i
    by 2 roundings; outside, softmax times (p_r - q_r): tol_logp of that softmax and tol of p_r."""
    N, V = r["z"].shape
    K = index.shape[1]
    loss, tol_loss = torch.zeros(N, dtype=torch.float64), torch.zeros(N, dtype=torch.float64)
    dz, tol = torch.zeros(N, V, dtype=torch.float64), torch.zeros(N, V, dtype=torch.float64)
    c = r["c"]
    for n in range(N):
        entries, bad = {}, False
        for k in range(K):
            i = int(index[n, k])
            if i >= V:
                bad = True
            elif i >= 0 and i not in entries:
                entries[i] = float(value[n, k]) * float(torch.tensor(c_t, dtype=torch.float32))
        gn = 1.0 if g is None else float(g[n])
        if bad:
            loss[n], dz[n] = float("nan"), float("nan")
            continue
        S = sorted(entries)
        u = torch.tensor([entries[i] for i in S], dtype=torch.float64)
        rest = t_lse is not None
        at = torch.tensor(S, dtype=torch.long)
        outside = torch.ones(V, dtype=torch.bool)
        outside[at] = False
        logp, p, tl = r["logp"][n], r["p"][n], r["tol_logp"][n]
        if bool(r["empty"][n]):
            logp = torch.full_like(logp, -INF)
        if rest:
            lq = u - float(t_lse[n])
        elif len(S) and float(u.max()) > -INF:
            lq = u - torch.logsumexp(u, 0)
        else:
            continue                                                          # no entries, or none with any mass
        q = torch.exp(lq)
        some = q > 0
        terms = q[some] * (lq[some] - logp[at][some])
        loss[n] = terms.sum()
        tL = float(r["tol_L"][n])
        tol_loss[n] = float(q.sum()) * tL + 1e-12
        d_in = p[at] - q
        t_in = p[at] * (tl[at] + 6 * U) + 4 * U * (q + p[at])
        if rest:
            q_r = max(0.0, 1.0 - float(q.sum()))
            d = torch.where(outside, r["d"][n], -INF) if not bool(r["empty"][n]) else torch.full((V,), -INF, dtype=torch.float64)
            l_r = float(torch.logsumexp(d, 0)) - float(r["L"][n])
            if l_r > -INF:
                share = torch.exp(d - d.max())                                # (not by its logarithm: d may be as low as -3e38)
                share = share / share.sum()
                p_r = math.exp(l_r)
                fin = torch.where(d > -INF, d - d.max(), 0.0)
                D1 = float((share * fin.abs()).sum())
                t_r = U * (r["sums"] + 4 * D1 + abs(math.log(float(torch.exp(d - d.max()).sum()))))
                if q_r > 0:
                    loss[n] += q_r * (math.log(q_r) - l_r)
                tol_loss[n] += q_r * (tL + t_r)
                dz[n] = share * (p_r - q_r)
                t_share = t_r + U * (6 * fin.abs() + 8)
                tol[n] = share * (abs(p_r - q_r) * t_share + p_r * (tL + t_r) + 4 * U * (p_r + q_r))
                tol[n] = torch.where(outside, tol[n], 0.0)
        else:
            dz[n] = p
            tol[n] = torch.where(p > 0, p * (tl + 8 * U), 0.0)
        dz[n, at], tol[n, at] = d_in, t_in
        if bool(r["empty"][n]):
            dz[n], tol[n] = 0.0, 0.0
        dz[n] *= c * gn
        tol[n] = tol[n] * abs(c * gn) + 4 * U * dz[n].abs()
    tol_loss = tol_loss + 2 * U * torch.where(loss.abs() < INF, loss.abs(), 0.0)
    return loss, tol_loss, dz, tol + rounding(dz, tol, dtype)


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
