"""The operators on a model's logits, as cases to be timed through the public entry points.

A case is one pass over the logits of N rows (positions, or samples) and V classes (tokens).  Four kinds:

    score    log probabilities of given tokens, with the entropy and the top alternatives (`token_logprobs`)
    step     the gradient of a loss in the log probabilities, its weights known beforehand: the local step of training
             (`token_logprobs_backward`, which forms the statistics itself)
    policy   the log probabilities first, weights that depend on them, then the gradient, with the entropy's
             (`token_logprobs` and `token_logprobs_backward`)
    distill  the loss against a teacher's top logits and its gradient (`distill_backward`, which forms the statistics
             itself; with "forward": the loss alone, by `distill`)

With `own` the framework's kernels run, without it the same formulas in elementary torch operations, in 32 bits.
"""
from __future__ import annotations

import math

import torch

own = False

TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}


def _case(name, kind, N, V, **kw):
    c = dict(kind=kind, N=N, V=V, type="bf16", pad=0, top=0, entropy=False, masked=False, scale=1.0, rest=False, forward=False)
    c.update(kw)
    if name is not None:
        c["name"] = name
    return c


def listed():
    return [
        # the loss and the top-1 and top-5 error of the softmax regression (15 workers with 400 samples each, 10 classes)
        _case("score_6000x10_top5", "score", 6000, 10, type="fp32", top=5),
        # serving, a single token: the sampled token's log probability and five alternatives; latency is all there is
        _case("score_1x32000_top5", "score", 1, 32000, top=5, scale=1.25),
        # serving, a batch of requests with a mask of allowed tokens, 20 alternatives each
        _case("score_64x128000_top20", "score", 64, 128000, top=20, entropy=True, masked=True),
        # scoring whole texts: log probability and entropy of every position
        _case("score_4096x128000", "score", 4096, 128000, entropy=True),
        # a teacher's table: the 64 largest of every position, logits with padded rows
        _case("score_2048x50001_top64", "score", 2048, 50001, type="fp32", pad=175, top=64),
        # the local step of the softmax regression: 15 workers, mini-batches of 8
        _case("step_120x10", "step", 120, 10, type="fp32"),
        # a training step's loss gradient, a vocabulary of ordinary size
        _case("step_8192x32000", "step", 8192, 32000),
        # an odd vocabulary in 16-bit floats: rows at every alignment, a mask that leaves some rows without a token
        _case("step_1000x65537", "step", 1000, 65537, type="fp16", masked=True),
        # policy gradients with an entropy bonus over a large vocabulary
        _case("policy_4096x131072", "policy", 4096, 131072, entropy=True),
        # a small student: ten classes, the teacher's three best
        _case("distill_120x10_top3", "distill", 120, 10, type="fp32", top=3),
        # a student's training step: the teacher's 64 best and the rest as one class
        _case("distill_8192x32000_top64", "distill", 8192, 32000, top=64, rest=True),
        # few long rows in 32 bits, a temperature, the teacher's 200 best by themselves
        _case("distill_300x151001_top200", "distill", 300, 151001, type="fp32", top=200, scale=0.5),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["score", "score", "step", "policy", "distill", "distill"])
    V = _log_uniform(rng, 8, 200_000)
    top = 0
    if kind == "score":
        top = min(V, rng.choice([0, 1, 5, 20, 64, 128]))
    if kind == "distill":
        top = min(V, _log_uniform(rng, 1, 256))
    most = 60_000_000 if top and kind == "score" else 200_000_000
    N = _log_uniform(rng, 1, max(2, min(16_384, most // V)))
    return _case(None, kind, N, V, type=rng.choice(["fp32", "bf16", "bf16", "fp16"]), pad=rng.choice([0, 0, 1, 24]), top=top,
                 entropy=kind == "policy" or (kind != "distill" and rng.random() < 0.5), masked=rng.random() < 0.4,
                 scale=rng.choice([1.0, 1.0, 0.5, 1.25]), rest=kind == "distill" and rng.random() < 0.5,
                 forward=kind == "distill" and rng.random() < 0.3)


def prepare(case, seed):
    dev = torch.device("cuda")
    g = torch.Generator(device=dev)
    g.manual_seed(seed * 7919 + 13)
    N, V, dt = case["N"], case["V"], TYPES[case["type"]]

    def randn(*shape):
        return torch.randn(*shape, generator=g, device=dev)

    # a few frequent classes and a long tail; some rows are sharp, some are flat
    tail = -0.7 * torch.log1p(torch.randperm(V, generator=g, device=dev).float())
    z = randn(N, V).mul_(2.0).add_(tail).mul_(torch.exp(0.4 * randn(N, 1)))
    held = torch.full((N, V + case["pad"]), float("nan"), dtype=dt, device=dev)     # what lies behind a row is not looked at
    logits = held[:, :V]
    logits.copy_(z)
    if case["masked"]:                                                             # classes that are not allowed
        out = torch.rand(V, generator=g, device=dev) < 0.2
        out[torch.randint(0, V, (1,), generator=g, device=dev)] = False
        logits.masked_fill_(out, float("-inf"))
        if N >= 16:
            logits[N // 2] = float("-inf")                                         # a row whose mask leaves nothing
    top = min(20, V)
    best = torch.topk(logits.float(), top, dim=1).indices
    target = best.gather(1, torch.randint(0, top, (N, 1), generator=g, device=dev)).squeeze(1)
    if N >= 16:
        target[torch.rand(N, generator=g, device=dev) < 0.1] = -100                # positions that are not trained on
    given = (target >= 0).float()
    S = (8192.0 if case["type"] == "fp16" else 1.0) / N                            # 16-bit floats need a scaled loss
    s = dict(case=case, logits=logits, target=target, share=S, weight=-S * given)
    f32 = dict(dtype=torch.float32, device=dev)
    if case["kind"] == "score":
        s.update(logprob=torch.empty(N, **f32), lse=torch.empty(N, **f32))
        if case["entropy"]:
            s["entropy"] = torch.empty(N, **f32)
        if case["top"]:
            s.update(top_index=torch.empty(N, case["top"], dtype=torch.int32, device=dev), top_logprob=torch.empty(N, case["top"], **f32))
    elif case["kind"] == "distill":
        t = logits + randn(N, V).mul_(1.5 / case["scale"])                            # in 32 bits: another tensor
        value, index = torch.topk(t, case["top"], dim=1)
        index = index.to(torch.int32)
        if case["masked"]:                                                         # tables with fewer entries in some rows
            some = torch.rand(N, 1, generator=g, device=dev) * (case["top"] + 1)
            index.masked_fill_((torch.arange(case["top"], device=dev) >= some) | ~torch.isfinite(value), -1)
            value.masked_fill_(index < 0, 0.0)
        s.update(index=index.contiguous(), value=value.contiguous(), loss=torch.empty(N, **f32), weight=torch.rand(N, generator=g, device=dev) * S)
        if case["rest"]:
            t = t.mul_(case["scale"])
            s["teacher_lse"] = torch.logsumexp(t, 1)
        if not case["forward"]:
            s["dlogits"] = torch.empty(N, V, dtype=dt, device=dev)
    else:
        s.update(logprob=torch.empty(N, **f32), dlogits=torch.empty(N, V, dtype=dt, device=dev))
        if case["entropy"]:
            s.update(entropy=torch.empty(N, **f32), entropy_weight=torch.full((N,), -0.01 * S, **f32))
        if case["kind"] == "policy":
            s.update(stats=torch.empty(N, 4, **f32), advantage=randn(N), old=-1.0 - torch.rand(N, generator=g, device=dev))
    return s


def _policy_weights(s, logprob):
    """d/d logprob of the clipped policy objective: the weights of a step that depend on its log probabilities."""
    ratio = torch.exp((logprob - s["old"]).clamp(-5.0, 5.0))
    live = ((s["advantage"] > 0) & (ratio < 1.2)) | ((s["advantage"] <= 0) & (ratio > 0.8))
    return torch.where(live & (s["target"] >= 0), -s["advantage"] * ratio * s["share"], 0.0)


# ---------------------------------------------------------------------------------------------
# the plain form
# ---------------------------------------------------------------------------------------------
def _plain_stats(s):
    c = s["case"]["scale"]
    z = s["logits"].float()
    m = z.amax(1, keepdim=True)
    empty = m == float("-inf")
    d = (z - torch.where(empty, 0.0, m)).mul_(c)
    e = torch.exp(d)
    total = e.sum(1, keepdim=True)
    L = torch.log(total)
    return z, m, empty, d, e, total, L


def _plain_entropy(empty, d, e, total, L):
    return torch.where(empty, 0.0, L - (e * d.clamp_min(-1e4)).sum(1, keepdim=True) / total)


def _plain_logprob(s, d, L, empty):
    t = s["target"].unsqueeze(1)
    lp = torch.where(empty, float("-inf"), d.gather(1, t.clamp_min(0)) - L)
    return torch.where(t >= 0, lp, 0.0)


def _plain_score(s):
    case = s["case"]
    z, m, empty, d, e, total, L = _plain_stats(s)
    out = dict(logprob=_plain_logprob(s, d, L, empty).squeeze(1),
               lse=torch.where(empty, float("-inf"), m * case["scale"] + L).squeeze(1))
    if case["entropy"]:
        out["entropy"] = _plain_entropy(empty, d, e, total, L).squeeze(1)
    if case["top"]:
        V = case["V"]
        bits = (z + 0.0).view(torch.int32)
        key = (bits ^ ((bits >> 31) & 0x7FFFFFFF)).long() * (1 << 32) + torch.arange(V - 1, -1, -1, device=z.device)
        key = torch.topk(key, case["top"], dim=1).values                            # larger first, ties to the lower index
        index = V - 1 - (key & 0xFFFFFFFF)
        out["top_index"] = index.to(torch.int32)
        out["top_logprob"] = torch.where(empty, float("-inf"), d.gather(1, index) - L)
    return out


def _plain_gradient(s, g, h):
    case = s["case"]
    z, m, empty, d, e, total, L = _plain_stats(s)
    t = s["target"].unsqueeze(1)
    out = dict(logprob=_plain_logprob(s, d, L, empty).squeeze(1))
    if g is None:
        g = _policy_weights(s, out["logprob"])
    g = torch.where(t >= 0, g.unsqueeze(1), 0.0)
    p = e.div_(total)
    if h is not None:
        H = _plain_entropy(empty, d, p, 1.0, L)
        out["entropy"] = H.squeeze(1)
        grad = p * (d.clamp_min_(-1e4).sub_(L).add_(H).mul_(h.unsqueeze(1)).add_(g)).neg_()
    else:
        grad = p * -g
    grad.scatter_add_(1, t.clamp_min(0), g)
    grad = torch.where(empty, 0.0, grad.mul_(case["scale"]))
    out["dlogits"] = grad.to(s["logits"].dtype)
    return out


def _plain_distill(s):
    case = s["case"]
    c = case["scale"]
    z, m, empty, d, e, total, L = _plain_stats(s)
    k = s["index"].long()
    has = k >= 0
    k = k.clamp_min(0)
    u = (s["value"].double() * c).masked_fill(~has, float("-inf"))                   # the entries and their sums in 64 bits
    if case["rest"]:
        lse = s["teacher_lse"].unsqueeze(1)
    else:
        most = u.amax(1, keepdim=True).clamp_min(-1e38)
        lse = torch.log(torch.exp(u - most).sum(1, keepdim=True)) + most
    logq = torch.where(has, u - lse, 0.0)
    q = torch.where(has, torch.exp(logq), 0.0)
    L = torch.log(total.double())
    logp = torch.where(empty, float("-inf"), (z.gather(1, k).double() - m) * c - L)
    loss = torch.where(q > 0, q * (logq - logp), 0.0).sum(1, keepdim=True)
    p = torch.where(empty, 0.0, e / total)
    weight = c * s["weight"].unsqueeze(1)
    taught = torch.zeros_like(z).scatter_add_(1, k, q.float())
    if case["rest"]:
        inside = torch.zeros_like(z).scatter_add_(1, k, has.float()) > 0
        left = torch.where(inside, float("-inf"), z * c)
        most = left.amax(1, keepdim=True).clamp_min(-3e38)
        lse_rest = torch.log(torch.exp(left - most).sum(1, keepdim=True)) + most
        sum_q = q.sum(1, keepdim=True)
        sum_p = torch.where(has, torch.exp(logp), 0.0).sum(1, keepdim=True)
        rest = (1.0 - sum_q).clamp_min(0.0)
        # the student's rest: from what is inside where that is the smaller part
        log_rest = torch.where(sum_p < 0.5, torch.log1p(-sum_p.clamp_max(0.5)), lse_rest.double() - m.double() * c - L)
        log_rest = torch.where(empty | (lse_rest == float("-inf")), float("-inf"), log_rest)
        both = (rest > 0) & (log_rest > float("-inf"))                              # nothing outside: the rest is left out
        loss = loss + torch.where(both, rest * (torch.log1p(-sum_q.clamp_max(1.0)) - log_rest), 0.0)
        outside = torch.where(left > float("-inf"), torch.exp(left - lse_rest), 0.0) * (torch.exp(log_rest) - rest).float()
        grad = torch.where(inside, p - taught, outside)
    else:
        grad = torch.where(has.any(1, keepdim=True), p - taught, 0.0)
    grad = torch.where(empty, 0.0, grad)
    out = dict(loss=loss.squeeze(1).float())
    if not case["forward"]:
        out["dlogits"] = (grad * weight).to(s["logits"].dtype)
    return out


def _own(s):
    from paper_1906_02367_amd import binding as B
    case = s["case"]
    kind, c = case["kind"], case["scale"]
    if kind == "score":
        B.token_logprobs(s["logits"], s["target"], scale=c, logprob=s["logprob"], entropy=s.get("entropy"), lse=s["lse"],
                         top_index=s.get("top_index"), top_logprob=s.get("top_logprob"))
        return {n: s[n] for n in ("logprob", "lse", "entropy", "top_index", "top_logprob") if n in s}
    if kind == "distill":
        teacher = dict(scale=c, teacher_scale=c, teacher_lse=s.get("teacher_lse"), loss=s["loss"])
        if case["forward"]:
            B.distill(s["logits"], s["index"], s["value"], **teacher)
            return dict(loss=s["loss"])
        B.distill_backward(s["logits"], s["index"], s["value"], s["dlogits"], grad_loss=s["weight"], **teacher)
        return dict(loss=s["loss"], dlogits=s["dlogits"])
    if kind == "step":
        B.token_logprobs_backward(s["logits"], s["target"], s["dlogits"], scale=c, grad_logprob=s["weight"],
                                  grad_entropy=s.get("entropy_weight"), logprob=s["logprob"], entropy=s.get("entropy"))
    else:
        B.token_logprobs(s["logits"], s["target"], scale=c, logprob=s["logprob"], entropy=s["entropy"], stats=s["stats"])
        B.token_logprobs_backward(s["logits"], s["target"], s["dlogits"], scale=c, grad_logprob=_policy_weights(s, s["logprob"]),
                                  grad_entropy=s["entropy_weight"], stats=s["stats"])
    return {n: s[n] for n in ("logprob", "entropy", "dlogits") if n in s}


def run(state):
    if own:
        return _own(state)
    kind = state["case"]["kind"]
    if kind == "score":
        return _plain_score(state)
    if kind == "distill":
        return _plain_distill(state)
    return _plain_gradient(state, state["weight"] if kind == "step" else None, state.get("entropy_weight"))


def work(case):
    N, V, K = case["N"], case["V"], case["top"]
    b = 4 if case["type"] == "fp32" else 2
    writes = case["kind"] != "score" and not case["forward"]
    small = N * (8 + 4 * 3 + 8 * K)
    return {"bytes": N * V * b * (2 if writes else 1) + small, "flops": N * V * (9 if writes else 5)}


# ---------------------------------------------------------------------------------------------
# the definition in 64 bits, a few rows at a time
# ---------------------------------------------------------------------------------------------
def _exact_rows(s, r0, r1, out):
    case = s["case"]
    c, V, kind = case["scale"], case["V"], case["kind"]
    lse0 = torch.logsumexp(s["logits"][r0:r1].double() * c, 1)
    live = lse0 > float("-inf")
    logp = s["logits"][r0:r1].double() * c - torch.where(live, lse0, 0.0)[:, None]   # rows that are empty stay at -inf
    p = logp.exp()
    n = torch.arange(r1 - r0, device=p.device)
    if kind != "distill":
        t = s["target"][r0:r1]
        chosen = logp[n, t.clamp_min(0)]
        chosen[t < 0] = 0.0
        out["logprob"][r0:r1] = chosen
        plogp = (p * logp).nan_to_num_(nan=0.0)
        H = -plogp.sum(1)
        if "entropy" in out:
            out["entropy"][r0:r1] = H
    if kind == "score":
        out["lse"][r0:r1] = lse0
        if case["top"]:
            value, index = torch.sort(s["logits"][r0:r1].float(), dim=1, descending=True, stable=True)
            out["top_index"][r0:r1] = index[:, :case["top"]].to(torch.int32)
            out["top_logprob"][r0:r1] = logp.gather(1, index[:, :case["top"]])
    elif kind in ("step", "policy"):
        g = s["weight"][r0:r1].double()
        if kind == "policy":
            part = dict(s, old=s["old"][r0:r1].double(), advantage=s["advantage"][r0:r1].double(), target=t)
            g = _policy_weights(part, chosen)
        g = g * (t >= 0)
        grad = -g[:, None] * p
        if case["entropy"]:
            grad -= s["entropy_weight"][r0:r1].double()[:, None] * (plogp + p * H[:, None])
        grad[n, t.clamp_min(0)] += g * live
        out["dlogits"][r0:r1] = grad * c
    else:
        index = s["index"][r0:r1].long()
        has = index >= 0
        u = torch.where(has, s["value"][r0:r1].double() * c, float("-inf"))
        lse = s["teacher_lse"][r0:r1].double() if case["rest"] else torch.logsumexp(u, 1)
        some = has.any(1)
        q = torch.where(has, torch.exp(u - torch.where(some, lse, 0.0)[:, None]), 0.0)
        at = logp.gather(1, index.clamp_min(0))
        loss = torch.where(q > 0, q * (q.log() - at), 0.0).sum(1)
        taught = torch.zeros_like(p).index_put_((n[:, None].expand_as(index)[has], index[has]), q[has])
        grad = (p - taught) * some[:, None]
        if case["rest"]:
            inside = torch.zeros_like(p, dtype=torch.bool).index_put_((n[:, None].expand_as(index)[has], index[has]), has[has])
            rest = (1.0 - q.sum(1)).clamp_min(0.0)
            lse_rest = torch.logsumexp(logp.masked_fill(inside, float("-inf")), 1)
            loss += torch.where((rest > 0) & (lse_rest > float("-inf")), rest * (rest.log() - lse_rest), 0.0)
            share = torch.exp(logp - torch.where(lse_rest > float("-inf"), lse_rest, 0.0)[:, None])
            grad = torch.where(inside, p - taught, share * (lse_rest.exp() - rest)[:, None])
        out["loss"][r0:r1] = loss
        if "dlogits" in out:
            out["dlogits"][r0:r1] = grad * live[:, None] * (c * s["weight"][r0:r1].double())[:, None]


def exact(case, seed):
    s = prepare(case, seed)
    N, V = case["N"], case["V"]
    names = ("logprob", "lse", "entropy", "top_logprob", "loss", "dlogits")
    out = {n: torch.empty(s[n].shape, dtype=torch.float64, device=s[n].device) for n in names if n in s}
    if case["kind"] in ("step", "policy") and not case["entropy"]:
        out.pop("entropy", None)
    if "top_index" in s:
        out["top_index"] = s["top_index"]
    rows = max(1, (1 << 26) // V)
    for r0 in range(0, N, rows):
        _exact_rows(s, r0, min(N, r0 + rows), out)
    return out
