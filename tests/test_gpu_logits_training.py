"""The operators on logits where the framework uses them: the errors and the distilled local step of the softmax model, and a chain from
a teacher's logits to the synchronised update."""
import numpy as np
import pytest
import torch

import logits_util as X

pytestmark = pytest.mark.gpu
dev = torch.device("cuda")


def test_error_of_the_softmax_model():
    from paper_1906_02367_amd import algorithm1 as A
    prob = A.SoftmaxProblem(seed=3, n_per_worker=50)
    w = 2.0 * torch.randn(A.D, generator=torch.Generator().manual_seed(1)).to(dev)
    order = torch.sort(prob.logits(w), dim=1, descending=True, stable=True).indices
    for k, got in zip((1, 2, 5), prob.error(w, (1, 2, 5))):
        want = float((order[:, :k] == prob.y.reshape(-1, 1)).any(1).sum())
        assert got == pytest.approx(1.0 - want / prob.n, abs=1e-6)


def _distilled_loss(prob, w, x, y, index, value):
    """The loss of one worker's samples in 64 bits, for autograd."""
    from paper_1906_02367_amd import algorithm1 as A
    z = x.double() @ w.view(A.N_CLASSES, -1).t()
    ce = -torch.log_softmax(z, 1).gather(1, y[:, None]).squeeze(1)
    logp, lq = torch.log_softmax(z / prob.T, 1), value.double()
    q, at = lq.exp(), logp.gather(1, index.long())
    left, p_r = 1 - q.sum(1), 1 - at.exp().sum(1)
    kl = (q * (lq - at)).sum(1) + left * (left.log() - p_r.log())
    return (prob.a * ce + (1 - prob.a) * prob.T ** 2 * kl).mean() + 0.5 * prob.lam * (w ** 2).sum()


@pytest.mark.parametrize("top,a", [(1, 0.5), (3, 0.3), (8, 0.0)])
def test_gradient_of_the_distilled_local_step(top, a):
    """Against autograd in 64 bits on the same samples.  u = 2^-24.  A logit is a product of 785 terms, off by at most 785 u sum |x w|, and sum
    |x w| <= |x| |w| (Cauchy) < 1.5 * 45 = 70: 3.3e-3.  (Twenty times the size that roundings of random sign have.)  A class's gradient
    dz = a (p - y) + (1 - a) T (p_T - q) moves by at most (a + (1 - a)) * 2 times the logits' error, and g by that times |x_j| < 0.3 (four standard
    deviations and the mean of a feature): 3.3e-3 * 2 * 0.3 = 2e-3 at the very worst, 1e-4 for roundings of random sign; what the products
    with x and the operators add (tested apart) is below 1e-5."""
    from paper_1906_02367_amd import algorithm1 as A
    prob = A.SoftmaxProblem(seed=4, n_per_worker=20, R=3)
    g = torch.Generator().manual_seed(2)
    teacher = torch.randn(A.D, generator=g).to(dev)
    dp = A.DistilledProblem(prob, teacher, top=top, a=a)
    w = torch.randn(3, A.D, generator=g).to(dev)
    state = dp.gen.get_state()
    got = dp.minibatch_grads(w, 6)
    dp.gen.set_state(state)
    idx = torch.randint(0, 20, (3, 6), generator=dp.gen, device=dev)
    for r in range(3):
        wr = w[r].double().requires_grad_(True)
        loss = _distilled_loss(dp, wr, dp.x[r, idx[r]], dp.y[r, idx[r]], dp.index[r, idx[r]], dp.value[r, idx[r]])
        want, = torch.autograd.grad(loss, wr)
        assert float((got[r].double() - want).abs().max()) < 1e-4, r
    whole = _distilled_loss(dp, w[0].double(), dp.x.reshape(dp.n, -1), dp.y.reshape(-1), dp.index.reshape(dp.n, -1), dp.value.reshape(dp.n, -1))
    assert dp.loss(w[0]) == pytest.approx(float(whole), rel=1e-5)


def test_algorithm1_on_the_distilled_problem_runs():
    from paper_1906_02367_amd import algorithm1 as A, binding as B
    prob = A.SoftmaxProblem(seed=1, n_per_worker=40, R=4)
    teacher = A.run_sync(prob, A.Operator(quantizer=B.SIGN_L1), H=2, T=20)["x"]
    res = A.run_sync(A.DistilledProblem(prob, teacher), A.Operator(quantizer=B.SIGN_L1), H=2, T=20)
    assert res["q"].device_status() == B.OK
    assert res["identity_err"] < 1e-5 and all(np.isfinite(res["loss"])) and res["bits"][-1] == 10 * 4 * (64 + 40 * 14)
    assert all(0.0 <= e <= 1.0 for e in prob.error(res["x"]))


def test_from_a_teachers_logits_to_the_synchronised_update():
    """A teacher's table is made from its logits, two workers' students are scored and taught, their output layers' gradients are
    compressed and the master adds the messages up: each step against its own definition on the inputs it had."""
    from oracle import oracle as O
    from paper_1906_02367_amd import binding as B
    V, h, N, K, R = 1003, 48, 40, 16, 2
    g = torch.Generator().manual_seed(8)
    hidden = (torch.randn(R, N, h, generator=g) / 4).to(dev)
    W_t, W = (torch.randn(V, h, generator=g).to(dev) for _ in range(2))
    d = V * h
    q = B.Qsl(d, [0, d], [d // 100], 15, B.TOPK, B.QSGD, 5, R, device=dev)
    op = O.OracleOp(d, [0, d], [d // 100], 15, 0, 0, 5)
    delta = torch.empty(R, d, device=dev)
    for r in range(R):
        teacher = (hidden[r] @ W_t.t()).bfloat16()
        index, value, lse = torch.empty(N, K, dtype=torch.int32, device=dev), torch.empty(N, K, device=dev), torch.empty(N, device=dev)
        B.token_logprobs(teacher, lse=lse, top_index=index, top_logprob=value)
        want, lp, tol = X.top(X.rows_of(teacher, 1.0), K)
        assert torch.equal(index.cpu().long(), want)
        X.check(value, lp, tol, "teacher's table")
        z = (hidden[r] @ W.t()).bfloat16()
        loss, dz, ones = torch.empty(N, device=dev), torch.empty_like(z), torch.full((N,), 1.0 / N, device=dev)
        zero = torch.zeros(N, device=dev)
        B.distill_backward(z, index, value, dz, teacher_lse=zero, grad_loss=ones, loss=loss)
        l, tol_l, want, tol = X.distill(X.rows_of(z, 1.0), index.cpu(), value.cpu(), 1.0, zero.cpu(), ones.cpu(), torch.bfloat16)
        X.check(loss, l, tol_l, "loss")
        X.check(dz, want, tol, "gradient")
        delta[r] = (dz.float().t().contiguous() @ hidden[r]).reshape(-1)
    m, msg, x = torch.zeros(R, d, device=dev), q.new_msg(R), torch.zeros(d, device=dev)
    q.compress(m, delta, m, 0, 0, msg)
    q.aggregate(msg, x, -1.0 / R, accumulate=True)
    torch.cuda.synchronize()
    assert q.device_status() == B.OK
    for r in range(R):
        o = op.compress(np.zeros(d, np.float32), delta[r].cpu().numpy(), r, 0)
        assert np.array_equal(msg[r].cpu().numpy(), o["msg"])
    assert np.allclose(x.cpu().numpy(), op.aggregate(msg.cpu().numpy(), -1.0 / R), rtol=1e-6, atol=1e-30)
