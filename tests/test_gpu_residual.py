"""The operators on a residual stream on the GPU against their definitions in 64 bits (residual_util), at the sizes, masks, layouts and calls
where they can go wrong."""
import math

import pytest
import torch

import residual_util as X

pytestmark = pytest.mark.gpu

INF, NAN = float("inf"), float("nan")
dev = torch.device("cuda")
COLS = [1, 2, 7, 8, 9, 63, 64, 120, 127, 128, 129, 511, 512, 513, 785, 1000, 1024, 1025, 2047, 2048, 2056, 4096, 4099, 8191, 8192, 8200, 12289, 16384, 16390, 32761, 32768]


@pytest.fixture(scope="module")
def B():
    from paper_1906_02367_amd import binding
    return binding


def rows_of(N, C, dtype, seed=0, pad=0, spread=1.0):
    """Rows of values, with NaN in the padding behind them."""
    g = torch.Generator().manual_seed(seed * 1009 + 7 * C + N)
    held = torch.full((N, C + pad), NAN, dtype=X.TYPES.get(dtype, dtype))
    held[:, :C] = (spread * torch.randn(N, C, generator=g)).to(held.dtype)
    return held.to(dev)[:, :C]


def room(N, C, dtype, pad=0):
    """Where a result goes, and the whole of the memory, of ones everywhere."""
    dtype = X.TYPES.get(dtype, dtype)
    held = torch.ones(N, C + pad, dtype=torch.float32, device=dev).to(dtype)
    return held[:, :C], held


def untouched(held, C):
    return bool((held[:, C:].float() == 1.0).all())


def weight_of(C, kind, dtype):
    if kind == "none":
        return None
    w = 1.0 + 0.3 * torch.randn(C, generator=torch.Generator().manual_seed(C))
    return w.to(torch.float32 if kind == "fp32" else X.TYPES[dtype]).to(dev)


def rows_for(C):
    return 21 if C <= 128 else 9 if C <= 1024 else 3


# ---- dropout -------------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("C", [1, 7, 8, 9, 64, 785, 2051, 4096, 40001])
def test_dropout(B, C, dtype):
    for N, pad, p, with_res, row0 in ((1, 0, 0.1, False, 0), (5, 3, 0.5, True, 11), (130, 1, 0.2, True, 2 ** 32 - 130), (64, 8, 1e-6, True, 0), (33, 0, 0.999, False, 5)):
        x, res = rows_of(N, C, dtype, 1, pad), rows_of(N, C, dtype, 2, (2 * pad) % 5) if with_res else None
        y, held = room(N, C, dtype, pad)
        B.dropout(x, y, p, seed=2 ** 40 + 9, round=2 ** 33 + 3, row0=row0, residual=res)
        keep = X.kept(N, C, p, seed=2 ** 40 + 9, round=2 ** 33 + 3, row0=row0)
        want, tol = X.total_of(x, res, keep, p)
        X.check(y, want, tol + X.rounding(want, tol, y.dtype), f"{N} x {C}, p = {p}")
        assert untouched(held, C)


def test_the_dropped_are_zero_and_nothing_else(B):
    """Ones: 0 or the factor, whose rounding is the only one; the mask value by value."""
    N, C = 257, 1003
    for p in (0.0, 0.05, 0.37, 1.0 - 2.0 ** -16, 1.0 - 2.0 ** -18, 1.0):
        y, _ = room(N, C, "fp32")
        B.dropout(torch.ones(N, C, device=dev), y, p, seed=3)
        keep, T = X.kept(N, C, p, seed=3), X.threshold(p)
        factor = torch.tensor(65536.0 / T if T else 0.0, dtype=torch.float32)
        assert torch.equal(y.cpu(), torch.where(keep, factor, torch.tensor(0.0))), p


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
def test_what_stands_in_dropped_places_does_not_matter(B, dtype):
    N, C, p = 40, 803, 0.4
    keep = X.kept(N, C, p, seed=8).to(dev)
    x, res = rows_of(N, C, dtype, 3), rows_of(N, C, dtype, 4)
    y, y2, t, t2, n, n2 = (room(N, C, dtype)[0] for _ in range(6))
    B.dropout(x, y, p, seed=8, residual=res)
    B.rms_norm(x, n, residual=res, total=t, p=p, seed=8)
    bad = x.clone()
    bad[~keep] = torch.tensor([NAN, INF, -INF, torch.finfo(x.dtype).min], device=dev, dtype=x.dtype).repeat(N * C)[: int((~keep).sum())]
    B.dropout(bad, y2, p, seed=8, residual=res)
    B.rms_norm(bad, n2, residual=res, total=t2, p=p, seed=8)
    assert torch.equal(y, y2) and torch.equal(t, t2) and torch.equal(n, n2)
    # where it is kept it does
    bad = x.clone()
    bad[5, int(keep[5].nonzero()[0])] = NAN
    B.dropout(bad, y2, p, seed=8, residual=res)
    B.rms_norm(bad, n2, residual=res, total=t2, p=p, seed=8)
    assert int(torch.isnan(y2).sum()) == 1 and int(torch.isnan(t2).sum()) == 1 and torch.isnan(n2[5]).all() and int(torch.isnan(n2).sum()) == C


def test_everything_dropped(B):
    """p = 1: the residual alone; without one, rows of zeros, whose norm and gradient are zeros."""
    N, C = 19, 300
    x, res = rows_of(N, C, "bf16", 1), rows_of(N, C, "bf16", 2)
    x[3] = NAN
    y, t = (room(N, C, "bf16")[0] for _ in range(2))
    B.dropout(x, y, 1.0, residual=res)
    assert torch.equal(y, res)
    B.rms_norm(x, y, total=t, p=1.0)
    assert not y.any() and not t.any()
    dres, dx, dw = room(N, C, "bf16")[0], room(N, C, "bf16")[0], torch.ones(C, device=dev)
    B.rms_norm_backward(t, res, dresidual=dres, dx=dx, dweight=dw, p=1.0, eps=1.0)
    assert torch.equal(dres, res) and not dx.any() and not dw.any()      # eps = 1: r = 1, u = 0


def test_parts_of_a_batch_have_the_masks_of_the_whole(B):
    N, C, p = 50, 777, 0.3
    x, dy = rows_of(N, C, "fp32", 1), rows_of(N, C, "fp32", 2)
    whole = [room(N, C, "fp32")[0] for _ in range(4)]
    parts = [room(N, C, "fp32")[0] for _ in range(4)]
    for out, cuts in ((whole, [0, N]), (parts, [0, 1, 18, 49, N])):
        for a, b in zip(cuts, cuts[1:]):
            kw = dict(p=p, seed=4, round=9, row0=1000 + a)
            B.dropout(x[a:b], out[0][a:b], **kw)
            B.rms_norm(x[a:b], out[1][a:b], total=out[2][a:b], **kw)
            B.rms_norm_backward(out[2][a:b], dy[a:b], dx=out[3][a:b], **kw)
    assert all(torch.equal(a, b) for a, b in zip(whole, parts))
    assert torch.equal(whole[0], whole[2])


def test_the_round_on_the_device(B):
    N, C = 12, 500
    x = rows_of(N, C, "bf16", 1)
    a, b, n, m = (room(N, C, "bf16")[0] for _ in range(4))
    for at, r, total in ((5, 7, 12), (2 ** 33, 1, 2 ** 33 + 1), (-3, 10, 7), (2 ** 62, 6, 6)):      # modulo 2^62
        B.dropout(x, a, 0.5, seed=1, round=r, round_at=torch.tensor([at], device=dev))
        B.dropout(x, b, 0.5, seed=1, round=total)
        B.rms_norm(x, n, p=0.5, seed=1, round=r, round_at=torch.tensor(at, device=dev))
        B.rms_norm(x, m, p=0.5, seed=1, round=total)
        assert torch.equal(a, b) and torch.equal(n, m), at


# ---- the norm ------------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("C", COLS)
def test_rms_norm(B, C, dtype):
    N = rows_for(C)
    for k, (pad, with_res, p, wk, eps) in enumerate(((0, True, 0.0, "same", 1e-5), (1, False, 0.0, "none", 1e-6), (3, True, 0.3, "fp32", 1e-2))):
        x, res, w = rows_of(N, C, dtype, k, pad), rows_of(N, C, dtype, 5 + k, 2 * pad, 3.0) if with_res else None, weight_of(C, wk, dtype)
        y, held = room(N, C, dtype, pad)
        t, held_t = room(N, C, dtype, 4 * pad)
        B.rms_norm(x, y, weight=w, eps=eps, residual=res, total=t if k else None, p=p, seed=11, round=k)
        h, tol = X.total_of(x, res, X.kept(N, C, p, seed=11, round=k) if p else None, p)
        want, tol_y = X.norm_of(h, tol, w, eps)
        X.check(y, want, tol_y + X.rounding(want, tol_y, y.dtype), f"{C}: y, {k}")
        if k:
            X.check(t, h, tol + X.rounding(h, tol, t.dtype), f"{C}: total, {k}")
        assert untouched(held, C) and untouched(held_t, C)


def check_8_bits(B, C, code, dtype, pad, group, wk, p, x, res):
    N, Q = x.shape[0], 448.0 if code is torch.float8_e4m3fn else 127.0
    w = weight_of(C, wk, dtype)
    G = -(-C // group) if group else 1
    q, held = room(N, C, code, pad)
    t, s = room(N, C, dtype)[0], torch.full((N, G), 77.0, device=dev)
    B.rms_norm(x, q, weight=w, residual=res, total=t, p=p, seed=2, scales=s, group=group)
    h, tol = X.total_of(x, res, X.kept(N, C, p, seed=2) if p else None, p)
    y, tol_y = X.norm_of(h, tol, w, 1e-6)
    want_s, tol_s, spread = X.scales_of(y, tol_y, group, Q)
    X.check(s, want_s, tol_s, f"{C}: scales, group {group}")
    v = y / spread
    t_v = 1.01 * (tol_y / spread + v.abs() * (tol_s / want_s).repeat_interleave(group or C, 1)[:, :C] + 3 * X.U * v.abs())
    half = torch.full_like(v, 0.5) if code is torch.int8 else X.rounding(v, t_v, code)
    X.check(q.float(), v, half + t_v, f"{C}: codes, group {group}")
    X.check(t, h, tol + X.rounding(h, tol, t.dtype), f"{C}: total")
    assert float(q.float().abs().max()) <= Q and untouched(held, C)


@pytest.mark.parametrize("code", [torch.float8_e4m3fn, torch.int8])
@pytest.mark.parametrize("C", [1, 8, 9, 31, 32, 33, 128, 130, 500, 512, 785, 1024, 1100, 2048, 3000, 4096, 8192, 9001, 16384, 20000, 32768])
def test_rms_norm_in_8_bits(B, C, code):
    """Every code is nearest to y / scale: half a step of e4m3 is 2^-4 of the value or 2^-10, of whole numbers 1/2; y and the scale are off by their
    tolerances (the scale's moves a value by as much relative), and Q / a, its product and the division for the scale by 3 u."""
    N = rows_for(C)
    for k, (dtype, pad, group, wk, p) in enumerate((("bf16", 0, 0, "same", 0.0), ("fp32", 3, 32, "none", 0.2), ("fp16", 1, 64, "fp32", 0.0), ("bf16", 5, 128, "fp32", 0.1))):
        check_8_bits(B, C, code, dtype, pad, group, wk, p, rows_of(N, C, dtype, k, pad), rows_of(N, C, dtype, 9, 0, 2.0))


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("C", [3, 20, 64, 65, 100, 127, 128, 129, 200, 512, 1000, 2047, 4096, 5001])
def test_groups_of_every_type(B, C, dtype):
    """Every size of a group with every type, by the same tolerances."""
    N = rows_for(C)
    for code in (torch.float8_e4m3fn, torch.int8):
        for group in (0, 32, 64, 128):
            check_8_bits(B, C, code, dtype, 0, group, "same", 0.0, rows_of(N, C, dtype, group), None)


def test_codes_of_known_values(B):
    """Rows whose y is known exactly: plus and minus one, weights that are multiples of the scale.  r is a power of two: sum h^2 / C + eps = 1."""
    C = 64
    x = torch.full((3, C), 0.5, device=dev)
    x[1] = -0.5
    x[2, ::2] = -0.5
    w = torch.arange(C, dtype=torch.float32, device=dev) * 2.0          # y = w x, x = 0.5: 0, 1, ..., 63
    for code, Q in ((torch.int8, 127.0), (torch.float8_e4m3fn, 448.0)):
        w2 = torch.where(torch.arange(C, device=dev) == 5, 2.0 * Q, w)   # the largest y is Q: scale 1
        q, s = room(3, C, code)[0], torch.empty(3, 1, device=dev)
        B.rms_norm(x, q, weight=w2, eps=0.75, scales=s)
        want = (x * w2).to(code).float()
        assert torch.equal(s, torch.ones_like(s)) and torch.equal(q.float(), want), code


# ---- rows with special values --------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("C", [5, 100, 300, 900, 2000, 4000, 8000, 16000, 30000])
def test_rows_of_zeros_nan_and_infinities(B, C, dtype):
    """They change no other row, those that share a wave or a block with them among them."""
    N = 20
    x, w = rows_of(N, C, dtype, 1, 1), weight_of(C, "same", dtype)
    dy = rows_of(N, C, dtype, 2)
    clean = special_outputs(B, x, w, dy)
    z = x.clone()
    z[2], z[7, C // 2], z[9, C - 1], z[12, 0] = 0.0, NAN, INF, -INF
    got = special_outputs(B, z, w, dy)
    others = [n for n in range(N) if n not in (2, 7, 9, 12)]
    for name in ("y", "q", "scales", "codes", "group_scales", "dresidual"):
        assert torch.equal(got[name][others], clean[name][others]), name
    assert not got["y"][2].any() and not got["q"][2].any() and got["scales"][2] == torch.tensor(2.0 ** -100 / 448)
    assert torch.isnan(got["y"][7]).all() and torch.isnan(got["scales"][7]) and torch.isnan(got["group_scales"][7]).all()
    for n, i in ((9, C - 1), (12, 0)):
        rest = torch.arange(C, device=dev) != i
        assert torch.isnan(got["y"][n, i]) and not got["y"][n][rest].any()
        assert torch.isnan(got["scales"][n])
        assert torch.isnan(got["group_scales"][n, i // 32]) and int(torch.isnan(got["group_scales"][n]).sum()) == 1
    assert not got["q"][[7, 9, 12]].any() and not got["codes"][[7, 9, 12]].any()
    assert torch.isnan(got["dresidual"][[7, 9, 12]]).all()
    want, tol, _, _ = X.backward(z[2:3], dy[2:3], w, 1e-5)
    if dtype != "fp16":                                              # (r = 316: g r may pass the largest fp16)
        X.check(got["dresidual"][2:3], want, tol + X.rounding(want, tol, x.dtype), "gradient of a row of zeros")
    assert torch.isnan(got["dweight"]).all() == (C >= 1)


def special_outputs(B, x, w, dy):
    N, C = x.shape
    o = dict(y=room(N, C, x.dtype)[0], q=torch.ones(N, C, device=dev).to(torch.float8_e4m3fn), scales=torch.empty(N, 1, device=dev), codes=torch.ones(N, C, dtype=torch.int8, device=dev),
             group_scales=torch.empty(N, -(-C // 32), device=dev), dresidual=room(N, C, x.dtype)[0], dweight=torch.empty(C, device=dev))
    B.rms_norm(x, o["y"], weight=w, eps=1e-5)
    B.rms_norm(x, o["q"], weight=w, eps=1e-5, scales=o["scales"])
    B.rms_norm(x, o["codes"], weight=w, eps=1e-5, scales=o["group_scales"], group=32)
    B.rms_norm_backward(x, dy, weight=w, eps=1e-5, dresidual=o["dresidual"], dweight=o["dweight"])
    return {n: v.float() if v.dtype is torch.float8_e4m3fn else v for n, v in o.items()}


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("C", [3, 100, 500, 1000, 2000, 4000, 8000, 16000, 32768])
def test_totals_whose_squares_do_not_fit(B, C, dtype):
    """Values up to 2^127 and down to 2^-80 beside ordinary rows.  The factor of such rows is a power of two: no tolerance more; a gradient below
    2^-126 has steps of 2^-149, and 1 / rms is below it, which puts 2^-149 / 2^-127 = 2^-22 relative on it."""
    N = 20
    x, w, dy = rows_of(N, C, dtype, 1), weight_of(C, "fp32", dtype), rows_of(N, C, dtype, 2)
    big = {1: 2.0 ** 70, 4: 2.0 ** 100, 8: 2.0 ** 124, 9: 2.0 ** 64, 13: 2.0 ** 62, 15: 2.0 ** -80, 18: 2.0 ** -130}
    for n, f in big.items():
        x[n] = (x[n].double() * f).to(x.dtype)
    x[5], x[6] = torch.finfo(x.dtype).max, torch.finfo(x.dtype).min
    y, dres, dx, dw = room(N, C, dtype)[0], room(N, C, dtype)[0], room(N, C, dtype)[0], torch.empty(C, device=dev)
    B.rms_norm(x, y, weight=w, eps=1e-6)
    h = x.cpu().double()
    want, tol = X.norm_of(h, torch.zeros_like(h), w, 1e-6)
    X.check(y, want, tol + X.rounding(want, tol, y.dtype), f"{C}: y")
    B.rms_norm_backward(x, dy, weight=w, eps=1e-6, dresidual=dres, dx=dx, dweight=dw)
    want, tol, want_w, tol_w = X.backward(x, dy, w, 1e-6)
    tol = tol + 2.0 ** -22 * want.abs() + 2.0 ** -148
    X.check(dres, want, tol + X.rounding(want, tol, y.dtype), f"{C}: gradient")
    X.check(dw, want_w, tol_w, f"{C}: dweight")
    assert torch.equal(dres, dx)


# ---- the gradient --------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("C", COLS)
def test_rms_norm_backward(B, C, dtype):
    N = rows_for(C)
    for k, (pad, with_dt, p, wk, eps) in enumerate(((0, True, 0.2, "same", 1e-5), (1, False, 0.0, "none", 1e-6), (3, True, 0.0, "fp32", 1e-2))):
        h, dy, dt, w = rows_of(N, C, dtype, k, pad, 2.0), rows_of(N, C, dtype, 5 + k, 2 * pad), rows_of(N, C, dtype, 9, pad) if with_dt else None, weight_of(C, wk, dtype)
        dres, held = room(N, C, dtype, pad)
        dx, held_x = room(N, C, dtype, 4 * pad)
        dw = torch.full((C,), 77.0, device=dev)
        B.rms_norm_backward(h, dy, weight=w, eps=eps, dtotal=dt, dresidual=dres, dx=dx, dweight=dw, p=p, seed=3, round=k, row0=6)
        want, tol, want_w, tol_w = X.backward(h, dy, w, eps, dt)
        X.check(dres, want, tol + X.rounding(want, tol, dres.dtype), f"{C}: dresidual, {k}")
        if p:
            keep = X.kept(N, C, p, seed=3, round=k, row0=6)
            want, t2 = X.dropped(want, keep, p)
            tol = torch.where(keep, tol * (65536 / X.threshold(p)) * 1.01 + t2, 0.0)
        X.check(dx, want, tol + X.rounding(want, tol, dx.dtype), f"{C}: dx, {k}")
        X.check(dw, want_w, tol_w, f"{C}: dweight, {k}")
        assert untouched(held, C) and untouched(held_x, C)


@pytest.mark.parametrize("N,C,dtype", [(1, 4096, "bf16"), (700, 100, "fp32"), (17000, 64, "bf16"), (5000, 300, "fp16"), (4500, 1000, "bf16"), (3000, 2001, "fp32"), (2600, 4096, "bf16"), (1100, 8192, "fp32"), (600, 16384, "fp16"),
                                       (300, 32768, "bf16")])
def test_the_weights_gradient_over_many_rows(B, N, C, dtype):
    """More rows than blocks; dweight alone, and beside the others, with a workspace of one's own."""
    h, dy, w = rows_of(N, C, dtype, 1, 0, 1.5), rows_of(N, C, dtype, 2), weight_of(C, "same", dtype)
    dw, dw2, dres = torch.empty(C, device=dev), torch.empty(C, device=dev), torch.empty_like(h)
    B.rms_norm_backward(h, dy, weight=w, eps=1e-5, dweight=dw)
    space = torch.empty(B.rms_norm_workspace_bytes(h) + 256, dtype=torch.uint8, device=dev)
    space[-256:] = 7
    B.rms_norm_backward(h, dy, weight=w, eps=1e-5, dweight=dw2, dresidual=dres, workspace=space)
    want, tol, want_w, tol_w = X.backward(h, dy, w, 1e-5)
    X.check(dw, want_w, tol_w, "dweight")
    X.check(dres, want, tol + X.rounding(want, tol, dres.dtype), "dresidual")
    assert torch.equal(dw, dw2) and (space[-256:] == 7).all()


@pytest.mark.parametrize("C", [5, 100, 400, 1000, 2000, 4000, 8000, 16000, 32768])
def test_the_weights_gradient_of_few_rows(B, C):
    """Where one block has all rows its sum is dweight, without a workspace; and the numbers of rows around that border."""
    per = 16 if C <= 128 else 4 if C <= 1024 else 1
    for N in (1, 2, 2 * per, 2 * per + 1):
        h, dy = rows_of(N, C, "fp32", N), rows_of(N, C, "fp32", 50 + N)
        dw = torch.full((C,), 77.0, device=dev)
        assert (B.rms_norm_workspace_bytes(h) == 0) == (N <= 2 * per)
        B.rms_norm_backward(h, dy, dweight=dw)
        _, _, want, tol = X.backward(h, dy, None, 1e-6)
        X.check(dw, want, tol, f"{N} x {C}")


@pytest.mark.parametrize("N,C,dtype", [(70000, 2048, "bf16"), (16500, 8200, "fp16"), (17000, 4099, "bf16"), (300000, 513, "bf16"), (1100000, 127, "fp16"),
                                        (600000, 127, "fp32"), (33000, 2100, "fp32"), (8300, 8200, "fp32"), (4200, 16390, "fp32"), (8300, 16400, "bf16")])
def test_results_that_the_caches_do_not_hold(B, N, C, dtype):
    """More than 256 MB written: the first and the last rows, and rows between, against the definitions; all of them against smaller calls."""
    g = torch.Generator(device=dev).manual_seed(1)
    x, res, dy = (torch.randn(N, C, generator=g, device=dev).to(X.TYPES[dtype]) for _ in range(3))
    w, p = weight_of(C, "same", dtype), 0.2
    y, t, dres, dx, d, dw = (torch.empty_like(x) for _ in range(6))
    dw = torch.empty(C, device=dev)
    B.rms_norm(x, y, weight=w, residual=res, total=t, p=p, seed=1)
    B.rms_norm_backward(t, dy, weight=w, dtotal=res, dresidual=dres, dx=dx, dweight=dw, p=p, seed=1)
    B.dropout(x, d, p, seed=1, residual=res)
    assert torch.equal(d, t)
    for a in (0, N // 2, N - 7):
        keep = X.kept(7, C, p, seed=1, row0=a)
        h, tol = X.total_of(x[a:a + 7], res[a:a + 7], keep, p)
        want, tol_y = X.norm_of(h, tol, w, 1e-6)
        X.check(t[a:a + 7], h, tol + X.rounding(h, tol, t.dtype), "total")
        X.check(y[a:a + 7], want, tol_y + X.rounding(want, tol_y, y.dtype), "y")
        want, tol, _, _ = X.backward(t[a:a + 7], dy[a:a + 7], w, 1e-6, res[a:a + 7])
        X.check(dres[a:a + 7], want, tol + X.rounding(want, tol, y.dtype), "dresidual")
    step = N // 7 + 1
    for a in range(0, N, step):
        part = [torch.empty_like(v[a:a + step]) for v in (y, t, dres, dx)]
        kw = dict(p=p, seed=1, row0=a)
        B.rms_norm(x[a:a + step], part[0], weight=w, residual=res[a:a + step], total=part[1], **kw)
        B.rms_norm_backward(t[a:a + step], dy[a:a + step], weight=w, dtotal=res[a:a + step], dresidual=part[2], dx=part[3], **kw)
        assert all(torch.equal(v[a:a + step], q) for v, q in zip((y, t, dres, dx), part)), a


def test_no_rows(B):
    x, w = torch.empty(0, 100, device=dev), torch.ones(100, device=dev)
    dw = torch.full((100,), 5.0, device=dev)
    B.dropout(x, x, 0.5)
    B.rms_norm(x, x, weight=w)
    B.rms_norm_backward(x, x, weight=w, dresidual=x, dweight=dw)
    assert not dw.any()


def test_the_gradient_by_differences(B):
    """Central differences of sum(dy y) + sum(dt total) in x and the residual, step e = 2^-6 at single places: the norm's third derivative, below 6 / rms^3
    times the values, times e^2 / 6, and the roundings of the two sums of y, 2 u 40 each, over 2 e, stay below 2e-3 here."""
    N, C, p, eps = 2, 40, 0.25, 0.3
    x, res, w = rows_of(N, C, "fp32", 1), rows_of(N, C, "fp32", 2), weight_of(C, "same", "fp32")
    dy, dt = rows_of(N, C, "fp32", 3), rows_of(N, C, "fp32", 4)
    y, t, dres, dx, dw = (torch.empty_like(x) for _ in range(5))
    dw = torch.empty(C, device=dev)

    def value(x, res, w):
        B.rms_norm(x, y, weight=w, eps=eps, residual=res, total=t, p=p, seed=1)
        return float((dy.double() * y.double()).sum() + (dt.double() * t.double()).sum())

    value(x, res, w)
    B.rms_norm_backward(t, dy, weight=w, eps=eps, dtotal=dt, dresidual=dres, dx=dx, dweight=dw, p=p, seed=1)
    e = 2.0 ** -6
    for arg, grad in ((x, dx), (res, dres), (w, dw)):
        flat, g = arg.view(-1), grad.view(-1)
        for i in range(0, flat.numel(), 7):
            was = flat[i].clone()
            flat[i] = was + e
            up = value(x, res, w)
            flat[i] = was - e
            down = value(x, res, w)
            flat[i] = was
            assert abs((up - down) / (2 * e) - float(g[i])) < 2e-3, i


# ---- a run of them together ----------------------------------------------------------------------------------------------------
def test_two_layers_forward_and_backward(B):
    """x -> norm -> times a matrix -> dropout onto the stream -> norm -> ... -> dropout onto the stream: values and gradients against autograd in 64
    bits.  fp32: the products of 96 terms are off by at most 96 u relative to the terms' sizes; all values here are of size 1 to 10 and pass four
    such products forward and four back, and the norms and sums by less: 8 * 96 * 2^-24 * 10 * sqrt(96) < 5e-3; roundings of random sign are a
    hundredth of that."""
    N, C, p, eps = 33, 96, 0.2, 1e-3
    g = torch.Generator().manual_seed(5)
    mats = [torch.randn(C, C, generator=g).div_(math.sqrt(C)).to(dev) for _ in range(2)]
    ws = [weight_of(C, "same", "fp32").mul(1 + 0.1 * k) for k in range(3)]
    x, dy = rows_of(N, C, "fp32", 1), rows_of(N, C, "fp32", 2)
    new = lambda: torch.empty(N, C, device=dev)
    # forward: stream, normed, layer's output by turns
    streams, normed = [x], [new()]
    B.rms_norm(x, normed[0], weight=ws[0], eps=eps)
    for k in range(2):
        out = normed[k] @ mats[k]
        streams.append(new()); normed.append(new())
        B.rms_norm(out, normed[-1], weight=ws[k + 1], eps=eps, residual=streams[k], total=streams[-1], p=p, seed=6, round=k)
    # backward
    dws, dnorm, dstream = [torch.empty(C, device=dev) for _ in range(3)], dy, None
    for k in (1, 0):
        dres, dout = new(), new()
        B.rms_norm_backward(streams[k + 1], dnorm, weight=ws[k + 1], eps=eps, dtotal=dstream, dresidual=dres, dx=dout, dweight=dws[k + 1], p=p, seed=6, round=k)
        dnorm, dstream = dout @ mats[k].t().contiguous(), dres
    dx = new()
    B.rms_norm_backward(x, dnorm, weight=ws[0], eps=eps, dtotal=dstream, dresidual=dx, dweight=dws[0])
    # the same by autograd on the CPU
    leaf = lambda v: v.cpu().double().requires_grad_(True)
    x64, w64 = leaf(x), [leaf(w) for w in ws]
    m64 = [m.cpu().double() for m in mats]
    norm = lambda h, w: h / torch.sqrt((h * h).mean(1, keepdim=True) + eps) * w
    h = x64
    n = norm(h, w64[0])
    for k in range(2):
        keep = X.kept(N, C, p, seed=6, round=k)
        h = h + torch.where(keep, (n @ m64[k]) * (65536 / X.threshold(p)), 0.0)
        n = norm(h, w64[k + 1])
    grads = torch.autograd.grad((n * dy.cpu().double()).sum(), [x64] + w64)
    assert float((normed[-1].cpu().double() - n.detach()).abs().max()) < 5e-3
    for got, want in zip([dx] + dws, grads):
        assert float((got.cpu().double() - want).abs().max()) < 5e-3 * max(1.0, float(want.abs().max()))


# ---- layouts and calls ---------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("C", [100, 785, 4096])
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_results_in_the_place_of_what_is_read(B, C, dtype):
    N, p = 37, 0.3
    kw = dict(p=p, seed=1)
    x, res, w, dy, dt = rows_of(N, C, dtype, 1, 2), rows_of(N, C, dtype, 2, 3), weight_of(C, "same", dtype), rows_of(N, C, dtype, 3), rows_of(N, C, dtype, 4, 1)
    copy = lambda v: torch.empty_strided(v.shape, v.stride(), dtype=v.dtype, device=dev).copy_(v)
    y, t, n, a, b = (room(N, C, dtype)[0] for _ in range(5))
    B.dropout(x, y, residual=res, **kw)
    for over in ("x", "res"):
        v = dict(x=copy(x), res=copy(res))
        B.dropout(v["x"], v[over], residual=v["res"], **kw)
        assert torch.equal(v[over], y), over
    B.rms_norm(x, n, weight=w, residual=res, total=t, **kw)
    for total, out in (("x", "n"), ("res", "n"), ("x", "res"), ("res", "x"), ("t", "x"), ("t", "res")):
        v = dict(x=copy(x), res=copy(res), n=torch.empty_like(n), t=torch.empty_like(n))
        B.rms_norm(v["x"], v[out], weight=w, residual=v["res"], total=v[total], **kw)
        assert torch.equal(v[total], t) and torch.equal(v[out], n), (total, out)
    B.rms_norm_backward(t, dy, weight=w, dtotal=dt, dresidual=a, dx=b, **kw)
    for first, second in (("t", "dy"), ("dy", "dt"), ("dt", "t"), ("dt", "b"), ("a", "dt")):
        v = dict(t=copy(t), dy=copy(dy), dt=copy(dt), a=torch.empty_like(a), b=torch.empty_like(b))
        B.rms_norm_backward(v["t"], v["dy"], weight=w, dtotal=v["dt"], dresidual=v[first], dx=v[second], **kw)
        assert torch.equal(v[first], a) and torch.equal(v[second], b), (first, second)


@pytest.mark.parametrize("C", [1, 13, 129, 785, 2001, 4100])
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_rows_that_stand_in_turn(B, C, dtype):
    """Every array's rows among the others', at all offsets an element's alignment allows; what lies between stays as it was."""
    N, p = 17, 0.3
    parts = [rows_of(N, C, dtype, k) for k in range(5)]
    w = weight_of(C, "same", dtype)
    apart = [room(N, C, dtype)[0] for _ in range(5)]
    B.rms_norm(parts[0], apart[0], weight=w, residual=parts[1], total=apart[1], p=p, seed=1)
    B.rms_norm_backward(apart[1], parts[2], weight=w, dtotal=parts[3], dresidual=apart[2], dx=apart[3], p=p, seed=1)
    B.dropout(parts[0], apart[4], p, seed=2, residual=parts[4])
    held = torch.full((N, 11 * (C + 1) + 1), 7.0, dtype=X.TYPES[dtype], device=dev)
    place = [held[:, 1 + k * (C + 1): 1 + k * (C + 1) + C] for k in range(10)]
    for v, q in zip(place, parts):
        v.copy_(q)
    x, res, dy, dt, res2, y, t, dres, dx, d = place
    wide = torch.full((C + 1,), 7.0, dtype=w.dtype, device=dev)
    w2 = wide[1:].copy_(w)
    B.rms_norm(x, y, weight=w2, residual=res, total=t, p=p, seed=1)
    B.rms_norm_backward(t, dy, weight=w2, dtotal=dt, dresidual=dres, dx=dx, p=p, seed=1)
    B.dropout(x, d, p, seed=2, residual=res2)
    assert all(torch.equal(a, b) for a, b in zip((y, t, dres, dx, d), apart)) and all(torch.equal(a, b) for a, b in zip(place, parts))
    between = held.clone()
    for v in (between[:, 1 + k * (C + 1): 1 + k * (C + 1) + C] for k in range(10)):
        v.fill_(7.0)
    assert (between == 7.0).all()
    # codes in turn with codes, at every byte
    q, s = room(N, C, torch.int8)[0], torch.empty(N, 1, device=dev)
    B.rms_norm(x, q, weight=w2, residual=res, p=p, seed=1, scales=s)
    bytes_ = torch.full((N, 3 * C + 5), 9, dtype=torch.int8, device=dev)
    for k in (0, C + 2):
        B.rms_norm(x, bytes_[:, k:k + C], weight=w2, residual=res, p=p, seed=1, scales=s)
        assert torch.equal(bytes_[:, k:k + C], q)
    assert (bytes_[:, C:C + 2] == 9).all() and (bytes_[:, 2 * C + 2:] == 9).all()


def test_two_host_threads_at_once(B):
    import threading
    N, C = 300, 1500
    xs = [rows_of(N, C, "bf16", s) for s in (1, 2)]
    dy = rows_of(N, C, "bf16", 3)

    def calls(x, o):
        for _ in range(20):
            B.rms_norm(x, o[0], p=0.1, seed=1, total=o[1])
            B.rms_norm_backward(o[1], dy, dx=o[2], dweight=o[3], p=0.1, seed=1)
            B.dropout(x, o[4], 0.1, seed=1)

    outputs = lambda: [torch.zeros_like(dy) for _ in range(3)] + [torch.zeros(C, device=dev), torch.zeros_like(dy)]
    want, got = [outputs() for _ in xs], [outputs() for _ in xs]
    for x, o in zip(xs, want):
        calls(x, o)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in xs]

    def run(x, o, s):
        with torch.cuda.stream(s):
            calls(x, o)

    threads = [threading.Thread(target=run, args=a) for a in zip(xs, got, streams)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for w, g in zip(want, got) for a, b in zip(w, g))


def test_one_array_read_twice(B):
    x = rows_of(9, 300, "bf16", 1)
    y, t = (room(9, 300, "bf16")[0] for _ in range(2))
    B.rms_norm(x, y, residual=x, total=t)
    assert torch.equal(t, x + x)
    dres = room(9, 300, "bf16")[0]
    B.rms_norm_backward(x, x, dtotal=x, dresidual=dres)
    want, tol, _, _ = X.backward(x, x, None, 1e-6, x)
    X.check(dres, want, tol + X.rounding(want, tol, x.dtype), "one array for all")


@pytest.mark.parametrize("dtype,far", [("bf16", 2 ** 31 + 11), ("fp32", 2 ** 30 + 5)])
def test_offsets_that_pass_32_bits(B, dtype, far):
    """Three rows, the later ones beyond 4 GB and 8 GB."""
    C = 4100
    buf = torch.empty(2 * far + C, dtype=X.TYPES[dtype], device=dev)
    away = torch.as_strided(buf, (3, C), (far, 1))
    x, near = rows_of(3, C, dtype, 1), [room(3, C, dtype)[0] for _ in range(4)]
    away.copy_(x)
    kw = dict(p=0.4, seed=2)
    B.dropout(x, near[0], **kw)
    B.dropout(away, near[1], **kw)
    assert torch.equal(near[0], near[1])
    B.dropout(away, away, **kw)
    assert torch.equal(away, near[0])
    away.copy_(x)
    B.rms_norm(x, near[0], total=near[1], **kw)
    B.rms_norm(away, near[2], total=away, **kw)
    assert torch.equal(near[2], near[0]) and torch.equal(away, near[1])
    B.rms_norm_backward(near[1], x, dx=near[2], **kw)
    B.rms_norm_backward(away, x, dx=away, **kw)
    assert torch.equal(away, near[2])


def test_more_blocks_than_a_grids_row(B):
    """17.5 million rows of 8: 1.1 million blocks of the norm."""
    N, C = 17_500_001, 8
    x = torch.empty(N, C, dtype=torch.bfloat16, device=dev).normal_()
    y, t, d = torch.empty_like(x), torch.empty_like(x), torch.empty_like(x)
    B.dropout(x, d, 0.5, seed=1, row0=3)
    B.rms_norm(x, y, eps=1e-5, total=t, p=0.5, seed=1, row0=3)
    assert torch.equal(d, t)
    for a, b in ((0, 1000), (2 ** 24 - 500, 2 ** 24 + 500), (N - 1000, N)):
        keep = X.kept(b - a, C, 0.5, seed=1, row0=3 + a)
        h, tol = X.total_of(x[a:b], None, keep, 0.5)
        X.check(t[a:b], h, tol + X.rounding(h, tol, t.dtype), "total")
        want, tol_y = X.norm_of(h, tol, None, 1e-5)
        X.check(y[a:b], want, tol_y + X.rounding(want, tol_y, y.dtype), "y")
    dw, dres = torch.empty(C, device=dev), torch.empty_like(x)
    B.rms_norm_backward(t, x, eps=1e-5, dresidual=dres, dweight=dw)
    h = t.double()
    u = h / torch.sqrt((h * h).mean(1, keepdim=True) + 1e-5)
    terms = x.double() * u
    tol = X.U * (40 + math.ceil(N / 1024) + 112) * terms.abs().sum(0)      # (a row group has at most a 1,024th of the rows: 16 groups a block, 64 blocks at least)
    X.check(dw, terms.sum(0).cpu(), tol.cpu(), "dweight")


def test_the_same_call_gives_the_same_bits(B):
    N, C = 3000, 1500
    x, dy, w = rows_of(N, C, "bf16", 1), rows_of(N, C, "bf16", 2), weight_of(C, "fp32", "bf16")
    first = None
    for _ in range(4):
        y, t, dx, dw = torch.empty_like(x), torch.empty_like(x), torch.empty_like(x), torch.empty(C, device=dev)
        B.rms_norm(x, y, weight=w, total=t, p=0.1, seed=3)
        B.rms_norm_backward(t, dy, weight=w, dx=dx, dweight=dw, p=0.1, seed=3)
        now = [y, t, dx, dw]
        first = first or now
        assert all(torch.equal(a, b) for a, b in zip(first, now))


def test_a_captured_step_with_a_round_of_its_own(B):
    """Dropout, norm and gradient in one graph; the round is counted up in it: every replay has the next mask."""
    N, C, p = 260, 1030, 0.25
    x, res, dy, w = rows_of(N, C, "bf16", 1), rows_of(N, C, "bf16", 2), rows_of(N, C, "bf16", 3), weight_of(C, "same", "bf16")
    at = torch.zeros(1, dtype=torch.int64, device=dev)
    outputs = lambda: [torch.empty_like(x) for _ in range(5)] + [torch.empty(C, device=dev)]

    def calls(o, **kw):
        B.dropout(x, o[0], p, seed=5, residual=res, **kw)
        B.rms_norm(o[0], o[1], weight=w, residual=res, total=o[2], p=p, seed=6, **kw)
        B.rms_norm_backward(o[2], dy, weight=w, dresidual=o[3], dx=o[4], dweight=o[5], p=p, seed=6, **kw)

    a, b = outputs(), outputs()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        calls(a, round_at=at)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls(a, round=3, round_at=at)
        at.add_(1)
    at.zero_()
    masks = []
    for k in range(5):
        x.copy_(rows_of(N, C, "bf16", 20 + k))
        graph.replay()
        calls(b, round=3 + k)
        torch.cuda.synchronize()
        assert all(torch.equal(p_, q) for p_, q in zip(a, b)), k
        assert int(at) == k + 1
        masks.append((a[4] == 0).clone())
    assert not any(torch.equal(masks[0], m) for m in masks[1:])


def test_two_graphs_and_two_streams_at_once(B):
    N, C = 2000, 2000
    xs = [rows_of(N, C, "bf16", s) for s in (1, 2)]
    dy = rows_of(N, C, "bf16", 3)

    def calls(x, o):
        B.rms_norm(x, o[0], p=0.1, seed=1, total=o[1])
        B.rms_norm_backward(o[1], dy, dx=o[2], dweight=o[3], p=0.1, seed=1)

    outputs = lambda: [torch.zeros_like(dy) for _ in range(3)] + [torch.zeros(C, device=dev)]
    want = [outputs() for _ in xs]
    for x, o in zip(xs, want):
        calls(x, o)
    streams = [torch.cuda.Stream() for _ in xs]
    torch.cuda.synchronize()
    graphs, outs = [], []
    for x, s in zip(xs, streams):
        o = outputs()
        torch.cuda.synchronize()
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr, stream=s):
            calls(x, o)
        graphs.append(gr); outs.append(o)
    for k in range(4):
        for o in outs:
            for v in o:
                v.zero_()
        torch.cuda.synchronize()
        for gr, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                gr.replay()
        direct = [outputs() for _ in xs]
        torch.cuda.synchronize()
        for x, s, o in zip(xs, reversed(streams), direct):
            with torch.cuda.stream(s):
                calls(x, o)
        torch.cuda.synchronize()
        for w, o, d in zip(want, outs, direct):
            assert all(torch.equal(a, b) and torch.equal(a, c) for a, b, c in zip(w, o, d)), k


def test_refusals_through_the_binding(B):
    x, y = rows_of(40, 64, "bf16", 1), room(40, 64, "bf16")[0]
    for call in (lambda: B.dropout(x, y, 1.5), lambda: B.dropout(x, y, -0.1), lambda: B.rms_norm(x, y, eps=0.0), lambda: B.rms_norm(x, y, total=y), lambda: B.rms_norm(x, y, group=32),
                 lambda: B.rms_norm(x, torch.empty(40, 64, dtype=torch.int8, device=dev)), lambda: B.rms_norm_backward(x, y), lambda: B.rms_norm_backward(x, y, dresidual=x, dx=x),
                 lambda: B.rms_norm_backward(x, y, dweight=torch.empty(64, device=dev), workspace=torch.empty(256, dtype=torch.uint8, device=dev)[:0]),
                 lambda: B.rms_norm(rows_of(1, 32769, "bf16"), room(1, 32769, "bf16")[0])):
        with pytest.raises(B.QslError):
            call()
    torch.cuda.synchronize()
