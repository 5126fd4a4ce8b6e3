"""The operators on a residual stream at the edges of what the header allows: values next to nothing, weights and totals far from one, large eps, results that
the caches do not hold.  Against the definitions in 64 bits (residual_util), with their tolerances."""
import math

import pytest
import torch

import residual_util as X

pytestmark = pytest.mark.gpu
dev = torch.device("cuda")
E4M3, I8 = torch.float8_e4m3fn, torch.int8


@pytest.fixture(scope="module")
def B():
    from paper_1906_02367_amd import binding
    return binding


def rows_of(N, C, dtype, seed, size=1.0):
    """Normal values, times `size` before they are rounded to the type."""
    g = torch.Generator().manual_seed(seed * 1009 + 7 * C + N)
    return (torch.randn(N, C, generator=g, dtype=torch.float64) * size).to(X.TYPES[dtype]).to(dev)


def check_codes(B, x, w, eps, code, group):
    """Codes and scales of rows without a residual; returns them."""
    N, C = x.shape
    Q = 448.0 if code is E4M3 else 127.0
    q, s = torch.ones(N, C, device=dev).to(code), torch.full((N, -(-C // group) if group else 1), 77.0, device=dev)
    B.rms_norm(x, q, weight=w, eps=eps, scales=s, group=group)
    h, none = X.total_of(x)
    y, tol = X.norm_of(h, none, w, eps)
    want_s, tol_s, spread = X.scales_of(y, tol, group, Q)
    X.check(s, want_s, tol_s, f"{C}: scales, group {group}, eps {eps}")
    v = y / spread
    t_v = 1.01 * (tol / spread + v.abs() * (tol_s / want_s).repeat_interleave(group or C, 1)[:, :C] + 3 * X.U * v.abs())
    X.check(q.float(), v, t_v + (torch.full_like(v, 0.5) if code is I8 else X.rounding(v, t_v, code)), f"{C}: codes, group {group}, eps {eps}")
    return q.float(), s


# ---- 8 bits --------------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("code", [E4M3, I8])
@pytest.mark.parametrize("C", [20, 64, 130, 1000, 4100, 9000, 20000])
def test_codes_of_rows_next_to_nothing(B, C, code):
    """Rows of zeros, of 1e-38, of 2^-130, of 1e-9 with a group of zeros, beside ordinary ones, for eps down to the least that is taken.  (What the sum of
    squares loses below 2^-149 a term is nothing beside eps.)"""
    for eps in (1e-5, 2.7e-12, 1e-12, 2.2e-13, 1e-20, 2.0 ** -100):
        for dtype in ("fp32", "bf16"):
            x = rows_of(9, C, dtype, 1)
            x[1], x[3], x[6] = 0.0, rows_of(1, C, dtype, 2, 1e-38)[0], rows_of(1, C, dtype, 3, 2.0 ** -130)[0]
            x[4] = rows_of(1, C, dtype, 4, 1e-9)[0]
            x[4, 32:64] = 0.0
            for group in (0, 32):
                q, s = check_codes(B, x, None, eps, code, group)
                least = torch.tensor(2.0 ** -100 / (448.0 if code is E4M3 else 127.0), device=dev)
                assert not q[1].any() and (s[1] == least).all() and not q[4, 32:64].any()
                if group and C > 32:
                    assert s[4, 1] == least


@pytest.mark.parametrize("code", [E4M3, I8])
@pytest.mark.parametrize("C", [20, 130, 1000, 4100, 9000, 20000])
def test_codes_with_weights_far_from_one(B, C, code):
    """y fits where weight times total does not, and is above the least scale where that product has lost bits: fp32 weights of 2^70 and 2^-60 on rows up to
    2^62 and down to 2^-75, in one row as well.  (Products of the row's own power of two are exact, so no tolerance more.)"""
    for dtype, eps in (("fp32", 1e-6), ("bf16", 1e-12), ("fp32", 2.0 ** -100)):
        x = rows_of(9, C, dtype, 1)
        for n, f in {1: 2.0 ** 50, 2: 2.0 ** 62 / math.sqrt(C), 4: 2.0 ** 80, 5: 2.0 ** -30, 6: 2.0 ** -60, 7: 2.0 ** -75}.items():
            x[n] = rows_of(1, C, dtype, n, f)[0]
        w = rows_of(1, C, "fp32", 9)[0] * 0.3 + 1.0
        for size in (2.0 ** 70, 2.0 ** 110, 2.0 ** -60, 2.0 ** -90):
            check_codes(B, x, w * size, eps, code, 0)
            check_codes(B, x, w * size, eps, code, 32)
        mixed = w.clone()
        mixed[::3], mixed[1::5] = w[::3] * 2.0 ** 70, w[1::5] * 2.0 ** -60
        check_codes(B, x, mixed, eps, code, 0)
        check_codes(B, x, mixed, eps, code, 64)
    # what y itself does not fit into makes its group NaN, as it makes the whole type's y infinite
    x, w = torch.ones(2, C, device=dev), torch.ones(C, device=dev)
    x[0, 3], w[3], w[C - 1] = 8.0, 2.0 ** 127, 2.0 ** 100
    q, s, y = torch.ones(2, C, device=dev).to(code), torch.empty(2, 1, device=dev), torch.empty_like(x)
    B.rms_norm(x, q, weight=w, scales=s)
    B.rms_norm(x, y, weight=w)
    want = torch.isinf(y).any(1)
    assert bool(want[0]) and not bool(want[1]) and torch.equal(torch.isnan(s[:, 0]), want) and not q.float()[0].any()


# ---- rows whose squares do not fit ---------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("C", [100, 1000, 2048, 4096, 8192, 16384, 32768])
def test_rows_whose_squares_hardly_fit_beside_a_large_eps(B, C, dtype):
    """eps counts on both sides of the border: a mean of 2^128 / C, where the sum no longer fits, is not far enough above 2^100 to leave it out."""
    eps, border = 2.0 ** 100, 2.0 ** 64 / math.sqrt(C)
    x, dy, w = rows_of(8, C, dtype, 1), rows_of(8, C, dtype, 2), rows_of(1, C, "fp32", 3)[0] * 0.3 + 1.0
    for n, f in {1: 0.9, 2: 0.97, 3: 1.03, 4: 1.2, 6: 8.0, 7: 2.0 ** -10}.items():
        x[n] = (torch.sign(x[n].double()) * border * f).to(x.dtype)
    h = x.cpu().double()
    fits = (h * h).sum(1) < 2.0 ** 128 * (1 - 2.0 ** -12)
    assert not bool(fits[3]) and not bool(fits[6]) and bool(fits[1]) and bool(fits[7])
    y, dres, dw = torch.empty_like(x), torch.empty_like(x), torch.empty(C, device=dev)
    B.rms_norm(x, y, weight=w, eps=eps)
    want, tol = X.norm_of(h, torch.zeros_like(h), w, eps)
    X.check(y, want, tol + X.rounding(want, tol, y.dtype), f"{C}: y")
    B.rms_norm_backward(x, dy, weight=w, eps=eps, dresidual=dres, dweight=dw)
    want, tol, want_w, tol_w = X.backward(x, dy, w, eps)
    X.check(dres, want, tol + X.rounding(want, tol, y.dtype), f"{C}: gradient")
    X.check(dw, want_w, tol_w, f"{C}: dweight")
    check_codes(B, x, w, eps, E4M3, 0)


# ---- the gradient --------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("C", [4, 100, 500, 1000, 2000, 4000, 8000, 16000, 32768])
def test_gradients_whose_products_with_the_totals_do_not_fit(B, C, dtype):
    """dy times a total passes the largest float, dy and the gradient do not.  (2^-126 and less does not occur, so no tolerance more.)"""
    N = 20
    x, dy, dt, w = rows_of(N, C, dtype, 1), rows_of(N, C, dtype, 2), rows_of(N, C, dtype, 3), rows_of(1, C, "fp32", 4)[0] * 0.3 + 1.0
    for n, (a, b) in {2: (2.0 ** 55, 2.0 ** 75), 3: (2.0 ** 55, 2.0 ** 120), 7: (1.0, 2.0 ** 118), 8: (2.0 ** 12, 2.0 ** 118), 11: (2.0 ** 56, 2.0 ** -30), 13: (2.0 ** 100, 2.0 ** 118),
                      16: (2.0 ** -20, 2.0 ** 112)}.items():
        x[n], dy[n] = rows_of(1, C, dtype, 10 + n, a)[0], rows_of(1, C, dtype, 40 + n, b)[0]
    dres, dx = torch.empty_like(x), torch.empty_like(x)
    B.rms_norm_backward(x, dy, weight=w, eps=1e-6, dtotal=dt, dresidual=dres, dx=dx)
    want, tol, _, _ = X.backward(x, dy, w, 1e-6, dt)
    X.check(dres, want, tol + X.rounding(want, tol, x.dtype), f"{C}: gradient")
    assert torch.equal(dres, dx)
    # such rows change no others, and what is no number stays none
    plain, dw = torch.empty_like(x), torch.empty(C, device=dev)
    quiet, loud = dy.clone(), dy.clone()
    for n in (2, 3, 7, 8, 13, 16):
        quiet[n] = 0.0
    loud[3, C // 2], loud[7, C - 1] = float("nan"), float("inf")
    B.rms_norm_backward(x, quiet, weight=w, eps=1e-6, dtotal=dt, dresidual=plain)
    B.rms_norm_backward(x, loud, weight=w, eps=1e-6, dtotal=dt, dresidual=dx)
    others = [n for n in range(N) if n not in (2, 3, 7, 8, 13, 16)]
    assert torch.equal(plain[others], dres[others]) and torch.equal(dx[others], dres[others])
    assert torch.isnan(dx[3]).all() and not torch.isfinite(dx[7]).any() and torch.equal(dx[[2, 8, 13, 16]], dres[[2, 8, 13, 16]])


# ---- results that the caches do not hold ---------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype,C", [(t, c) for t in ("fp32", "bf16", "fp16") for c in (120, 500, 1000, 2047, 4096, 8191)])
def test_codes_that_the_caches_do_not_hold(B, dtype, C):
    """More than 256 MB of totals and codes: some rows against the definitions, all of them against smaller calls, bit for bit."""
    N = (2 ** 28 // (C * (5 if dtype == "fp32" else 3))) * 21 // 20 + 3
    g = torch.Generator(device=dev).manual_seed(1)
    x, res = (torch.randn(N, C, generator=g, device=dev).to(X.TYPES[dtype]) for _ in range(2))
    w, p = (rows_of(1, C, "fp32", 3)[0] * 0.3 + 1.0).to(x.dtype), 0.2
    step = N // 7 + 1
    for code, group in ((E4M3, 0), (I8, 128), (E4M3, 32)):
        G = -(-C // group) if group else 1
        made = lambda n: (torch.empty(n, C, dtype=x.dtype, device=dev), torch.empty(n, C, dtype=code, device=dev), torch.empty(n, G, device=dev))
        t, q, s = made(N)
        assert t.numel() * t.element_size() + q.numel() > 2 ** 28
        B.rms_norm(x, q, weight=w, residual=res, total=t, p=p, seed=1, scales=s, group=group)
        for a in range(0, N, step):
            t2, q2, s2 = made(len(x[a:a + step]))
            B.rms_norm(x[a:a + step], q2, weight=w, residual=res[a:a + step], total=t2, p=p, seed=1, row0=a, scales=s2, group=group)
            assert torch.equal(t[a:a + step], t2) and torch.equal(q[a:a + step].view(torch.uint8), q2.view(torch.uint8)) and torch.equal(s[a:a + step], s2), (code, group, a)
        Q = 448.0 if code is E4M3 else 127.0
        for a in (0, N // 2, N - 5):
            h, tol = X.total_of(x[a:a + 5], res[a:a + 5], X.kept(5, C, p, seed=1, row0=a), p)
            y, tol_y = X.norm_of(h, tol, w, 1e-6)
            want_s, tol_s, spread = X.scales_of(y, tol_y, group, Q)
            X.check(s[a:a + 5], want_s, tol_s, "scales")
            v = y / spread
            t_v = 1.01 * (tol_y / spread + v.abs() * (tol_s / want_s).repeat_interleave(group or C, 1)[:, :C] + 3 * X.U * v.abs())
            X.check(q[a:a + 5].float(), v, t_v + (torch.full_like(v, 0.5) if code is I8 else X.rounding(v, t_v, code)), "codes")
            X.check(t[a:a + 5], h, tol + X.rounding(h, tol, t.dtype), "total")


@pytest.mark.parametrize("N,C,dtype,past", [(70000, 2048, "bf16", True), (16500, 8200, "fp16", True), (17000, 4099, "bf16", True), (300000, 513, "bf16", True), (1100000, 127, "fp16", True),
                                            (600000, 127, "fp32", True), (33000, 2100, "fp32", True), (8300, 8200, "fp32", True), (4200, 16390, "fp32", True), (8300, 16400, "bf16", True),
                                            (600, 16384, "fp32", False), (300, 32768, "fp32", False)])
def test_the_weights_gradient_of_large_calls(B, N, C, dtype, past):
    """Against the sum in 64 bits.  A term's roundings: the root's SUM / 2 + 3, the product with the total, that with dy: SUM / 2 + 6; its sums: at most
    ceil(N / 256) rows one after the other (there are at least 256 blocks), then 16 groups of a block and the blocks, 112 steps."""
    g = torch.Generator(device=dev).manual_seed(2)
    h, dy = (torch.randn(N, C, generator=g, device=dev).to(X.TYPES[dtype]) for _ in range(2))
    w = (rows_of(1, C, "fp32", 3)[0] * 0.3 + 1.0).to(h.dtype)
    dres, dx, dw = torch.empty_like(h), torch.empty_like(h), torch.empty(C, device=dev)
    assert (2 * h.numel() * h.element_size() > 2 ** 28) == past
    B.rms_norm_backward(h, dy, weight=w, eps=1e-5, dresidual=dres, dx=dx, dweight=dw)
    assert torch.equal(dres, dx)
    want, size = torch.zeros(C, dtype=torch.float64, device=dev), torch.zeros(C, dtype=torch.float64, device=dev)
    step = max(1, 2 ** 25 // C)
    for a in range(0, N, step):
        k = h[a:a + step].double()
        terms = dy[a:a + step].double() * k / torch.sqrt((k * k).mean(1, keepdim=True) + 1e-5)
        want += terms.sum(0)
        size += terms.abs().sum(0)
    X.check(dw, want.cpu(), (X.U * (X.SUM / 2 + 6 + math.ceil(N / 256) + 112) * size).cpu(), f"{N} x {C}")


# ---- where the training harness uses them --------------------------------------------------------------------------------------
def test_a_run_that_goes_on_or_is_repeated_has_the_same_gradients():
    from paper_1906_02367_amd import algorithm1 as A
    data = A.SoftmaxProblem(seed=4, n_per_worker=20, R=3)
    new = lambda: A.RegularisedProblem(data, p=0.3, seed=11)
    w = 0.1 * torch.randn(3, A.D, generator=torch.Generator().manual_seed(2)).to(dev)
    first, whole, states = new(), [], []
    for _ in range(6):
        states.append((first.step, first.gen.get_state()))
        whole.append(first.minibatch_grads(w, 5))
    again = new()
    assert all(torch.equal(again.minibatch_grads(w, 5), g) for g in whole)
    later = new()
    later.step = states[4][0]
    later.gen.set_state(states[4][1])
    assert all(torch.equal(later.minibatch_grads(w, 5), g) for g in whole[4:])
    # the mask belongs to the place: the same sample at every place of a mini-batch has another mask at each
    rows = first.features(data.x[0, :1].expand(15, -1).contiguous(), p=0.3, seed=11, round=0)
    assert all(not torch.equal(rows[i] == 0, rows[j] == 0) for i in range(15) for j in range(i))
