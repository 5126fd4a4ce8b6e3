"""The operators on a residual stream where the framework uses them, and a chain from a layer's forward pass to the synchronised update."""
import numpy as np
import pytest
import torch

import residual_util as X

pytestmark = pytest.mark.gpu
dev = torch.device("cuda")


def _loss(prob, w, x, y, keep):
    """The loss of one worker's samples in 64 bits, for autograd."""
    from paper_1906_02367_amd import algorithm1 as A
    h = x.double() if keep is None else torch.where(keep, x.double() * (65536 / X.threshold(prob.p)), 0.0)
    h = h / torch.sqrt((h * h).mean(1, keepdim=True) + prob.eps)
    z = h @ w.view(A.N_CLASSES, -1).t()
    return -torch.log_softmax(z, 1).gather(1, y[:, None]).mean() + 0.5 * prob.lam * (w ** 2).sum()


@pytest.mark.parametrize("p", [0.0, 0.2, 0.6])
def test_gradient_of_the_regularised_local_step(p):
    """Against autograd in 64 bits on the same samples and masks, which differ from worker to worker and from step to step.  A logit is a product of
    785 terms, off by at most 785 u sum |n w| <= 785 u |n| |w|, u = 2^-24: |n| = 28 (the norm's), |w| < 31 for one class (785 values of size 1, or
    0.1 of it here): 785 * 2^-24 * 28 * 3.1 = 4e-3 at the very worst.  A class's gradient moves by at most twice that, times |n_j| < 6: 5e-2 at
    worst, a hundredth of it for roundings of random sign; the limit is 2e-3."""
    from paper_1906_02367_amd import algorithm1 as A
    model = A.RegularisedProblem(A.SoftmaxProblem(seed=4, n_per_worker=20, R=3), p=p, seed=11)
    w = 0.1 * torch.randn(3, A.D, generator=torch.Generator().manual_seed(2)).to(dev)
    for step in range(2):
        state = model.gen.get_state()
        got = model.minibatch_grads(w, 6)
        model.gen.set_state(state)
        idx = torch.randint(0, 20, (3, 6), generator=model.gen, device=dev)
        keep = X.kept(18, A.N_FEATURES + 1, p, seed=11, round=step).to(dev) if p else None
        for r in range(3):
            wr = w[r].double().requires_grad_(True)
            want, = torch.autograd.grad(_loss(model, wr, model.x[r, idx[r]], model.y[r, idx[r]], None if keep is None else keep[6 * r:6 * r + 6]), wr)
            assert float((got[r].double() - want).abs().max()) < 2e-3, (step, r)
    whole = _loss(model, w[0].double(), model.x.reshape(model.n, -1), model.y.reshape(-1), None)
    assert model.loss(w[0]) == pytest.approx(float(whole), rel=1e-5)


def test_algorithm1_on_the_regularised_problem_runs():
    from paper_1906_02367_amd import algorithm1 as A, binding as B
    model = A.RegularisedProblem(A.SoftmaxProblem(seed=1, n_per_worker=40, R=4), p=0.3)
    res = A.run_sync(model, A.Operator(quantizer=B.SIGN_L1), H=2, T=20)
    assert res["q"].device_status() == B.OK
    assert res["identity_err"] < 1e-5 and all(np.isfinite(res["loss"])) and res["bits"][-1] == 10 * 4 * (64 + 40 * 14)
    assert model.step == 20 and all(0.0 <= e <= 1.0 for e in model.error(res["x"]))


def test_from_a_layers_pass_to_the_synchronised_update():
    """Two workers' layers y = norm(residual + dropout(x W)): forward, backward, the gradients of W and of the norm's weight compressed as one vector
    of two segments, the master adding the messages up: each step against its own definition on the inputs it had."""
    from oracle import oracle as O
    from paper_1906_02367_amd import binding as B
    N, h, C, R, p, eps = 60, 24, 200, 2, 0.3, 1e-4
    g = torch.Generator().manual_seed(8)
    W, gain = (torch.randn(h, C, generator=g) / 5).to(dev), (1 + 0.2 * torch.randn(C, generator=g)).to(dev)
    d = h * C + C
    seg, k = [0, h * C, d], [h * C // 50, C // 10]
    q = B.Qsl(d, seg, k, 15, B.TOPK, B.QSGD, 5, R, device=dev)
    op = O.OracleOp(d, seg, k, 15, 0, 0, 5)
    delta = torch.empty(R, d, device=dev)
    for r in range(R):
        inputs, residual, dy = (torch.randn(N, n, generator=g).to(dev) for n in (h, C, C))
        out = inputs @ W
        y, total, dx, dgain = torch.empty_like(out), torch.empty_like(out), torch.empty_like(out), torch.empty(C, device=dev)
        drop = dict(p=p, seed=3, round=7, row0=r * N)
        B.rms_norm(out, y, weight=gain, eps=eps, residual=residual, total=total, **drop)
        t, tol = X.total_of(out, residual, X.kept(N, C, **drop), p)
        want, tol_y = X.norm_of(t, tol, gain, eps)
        X.check(total, t, tol + X.rounding(t, tol, torch.float32), "total")
        X.check(y, want, tol_y + X.rounding(want, tol_y, torch.float32), "y")
        B.rms_norm_backward(total, dy, weight=gain, eps=eps, dx=dx, dweight=dgain, **drop)
        want, tol, want_w, tol_w = X.backward(total, dy, gain, eps)
        keep = X.kept(N, C, **drop)
        want, t2 = X.dropped(want, keep, p)
        tol = torch.where(keep, tol * (65536 / X.threshold(p)) * 1.01 + t2, 0.0)
        X.check(dx, want, tol + X.rounding(want, tol, torch.float32), "dx")
        X.check(dgain, want_w, tol_w, "dweight")
        delta[r] = torch.cat([(inputs.t().contiguous() @ dx).reshape(-1), dgain])
    m, msg, x = torch.zeros(R, d, device=dev), q.new_msg(R), torch.zeros(d, device=dev)
    q.compress(m, delta, m, 0, 0, msg)
    q.aggregate(msg, x, -1.0 / R, accumulate=True)
    torch.cuda.synchronize()
    assert q.device_status() == B.OK
    for r in range(R):
        o = op.compress(np.zeros(d, np.float32), delta[r].cpu().numpy(), r, 0)
        assert np.array_equal(msg[r].cpu().numpy(), o["msg"])
    assert np.allclose(x.cpu().numpy(), op.aggregate(msg.cpu().numpy(), -1.0 / R), rtol=1e-6, atol=1e-30)
