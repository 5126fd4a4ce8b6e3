"""Operators on logits on the GPU: rows in which one side has nothing or NaN, statistics that are kept, layouts that lie close together.
Against the definitions in 64 bits (logits_util) where a value is computed."""
import pytest
import torch

import logits_util as X

pytestmark = pytest.mark.gpu

INF, NAN = float("inf"), float("nan")
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
dev = torch.device("cuda")
# rows that a wave holds, that a block holds in one and in several vectors a thread, and that are split
HELD_AND_SPLIT = [(5, 12, "fp32"), (5, 500, "bf16"), (6, 30000, "bf16"), (5, 65536, "fp16"), (5, 100001, "fp32"), (5, 200000, "fp32")]


@pytest.fixture(scope="module")
def B():
    from paper_1906_02367_amd import binding
    return binding


def new(*shape, dtype=torch.float32):
    return torch.full(shape, 77, dtype=dtype, device=dev)


def logits_of(N, V, dtype, seed=0):
    return (2.0 * torch.randn(N, V, generator=torch.Generator().manual_seed(seed * 1009 + V))).to(TYPES[dtype]).to(dev)


def taught_by(B, teacher, K):
    """A teacher's table: classes, log probabilities, and the logarithm of all classes' sum."""
    N = teacher.shape[0]
    index, value, lse = new(N, K, dtype=torch.int32), new(N, K), new(N)
    B.token_logprobs(teacher, lse=lse, top_index=index, top_logprob=value)
    return index, value, lse


def three_ways(B, z, index, value, **kw):
    """loss and gradient: formed at once, the loss alone with the statistics, the gradient from them."""
    N = z.shape[0]
    g = torch.linspace(0.5, 1.5, N, device=dev)
    loss, loss2, stats, dz, dz2 = new(N), new(N), new(N, 8), torch.empty_like(z), torch.empty_like(z)
    B.distill_backward(z, index, value, dz, grad_loss=g, loss=loss, **kw)
    B.distill(z, index, value, loss=loss2, stats=stats, **kw)
    B.distill_backward(z, index, value, dz2, grad_loss=g, stats=stats, **kw)
    return g, loss, loss2, dz, dz2


@pytest.mark.parametrize("N,V,dtype", HELD_AND_SPLIT)
def test_a_teacher_whose_row_has_no_class(B, N, V, dtype):
    """What token_logprobs hands out for a row of -inf, handed on: it teaches nothing, with the rest as a class and without."""
    K = 6
    teacher = logits_of(N, V, dtype, seed=1)
    teacher[0] = -INF
    teacher[3] = -INF
    z = logits_of(N, V, dtype)
    z[3] = -INF                                                        # nor has the student's
    index, value, lse = taught_by(B, teacher, K)
    assert lse[0] == -INF and (value[0] == -INF).all()
    kept = torch.where(lse == -INF, lse, 0.0)                          # of log probabilities the sum is 1
    r = X.rows_of(z, 1.0)
    for l in (None, kept):
        g, loss, loss2, dz, dz2 = three_ways(B, z, index, value, teacher_lse=l)
        some = torch.tensor([n for n in range(N) if n not in (0, 3)])
        rows = {k: v[some] if torch.is_tensor(v) and v.dim() else v for k, v in r.items()}
        want, tol_loss, want_dz, tol = X.distill(rows, index.cpu()[some], value.cpu()[some], 1.0, None if l is None else l.cpu()[some], g.cpu()[some], TYPES[dtype])
        for a, b in ((loss, dz), (loss2, dz2)):
            assert a[[0, 3]].tolist() == [0.0, 0.0] and not b[[0, 3]].any(), (V, l is None)
            X.check(a[some], want, tol_loss, f"{V}: loss")
            X.check(b[some], want_dz, tol, f"{V}: gradient")
    # the teacher's logits instead of their logarithms, and its lse as it is
    raw = teacher.float().gather(1, index.long())
    g, loss, loss2, dz, dz2 = three_ways(B, z, index, raw, teacher_lse=lse)
    assert loss[[0, 3]].tolist() == [0.0, 0.0] and not dz[[0, 3]].any() and not dz2[[0, 3]].any() and torch.equal(loss, loss2)
    # a NaN in the table or among the student's logits is one in the results, whatever the teacher has
    raw[0, 2] = NAN
    z[3, V // 2] = NAN
    g, loss, loss2, dz, dz2 = three_ways(B, z, index, raw, teacher_lse=lse)
    assert torch.isnan(loss[[0, 3]]).all() and torch.isnan(loss2[[0, 3]]).all() and torch.isnan(dz[[0, 3]]).all() and torch.isnan(dz2[[0, 3]]).all()
    assert torch.isfinite(dz[1]).all() and torch.isfinite(loss[1])


@pytest.mark.parametrize("N,V,dtype", HELD_AND_SPLIT)
def test_nan_among_the_entries_with_nothing_outside(B, N, V, dtype):
    """Only the entries' classes are left, one of them NaN or +inf: the row's results are NaN, at the classes outside too."""
    K = 5
    index, value, lse = taught_by(B, logits_of(N, V, dtype, seed=2), K)
    lse = torch.zeros(N, device=dev)
    z = torch.full((N, V), -INF, dtype=TYPES[dtype], device=dev)
    z.scatter_(1, index.long(), 0.25)
    z[0, index[0, 2].long()] = NAN
    z[1, index[1, 4].long()] = INF
    z[3, index[3, 0].long()] = NAN
    value[3] = -INF                                                    # entries without mass: every term is 0
    z[4, :] = 0.5
    z[4, V - 1] = NAN
    index[4] = -1                                                      # no entries
    for l in (None, lse):
        g, loss, loss2, dz, dz2 = three_ways(B, z, index, value, teacher_lse=l)
        for n in (0, 1, 3, 4):
            assert torch.isnan(loss[n]) and torch.isnan(loss2[n]), (n, l is None)
            assert torch.isnan(dz[n]).all() and torch.isnan(dz2[n]).all(), (n, l is None)
        assert torch.isfinite(loss[2]) and torch.isfinite(dz[2]).all() and torch.isfinite(dz2[2]).all()


@pytest.mark.parametrize("N,V,dtype", HELD_AND_SPLIT)
def test_nan_in_a_teachers_table(B, N, V, dtype):
    """One NaN among a row's values: loss and gradient of the row are NaN at every class, other rows are as without it."""
    index, value, lse = taught_by(B, logits_of(N, V, dtype, seed=2), 5)
    z = logits_of(N, V, dtype)
    for l in (None, torch.full((N,), 0.125, device=dev)):
        clean = three_ways(B, z, index, value, teacher_lse=l)[1:]
        broken = value.clone()
        broken[1, 3] = NAN
        for a, b in zip(three_ways(B, z, index, broken, teacher_lse=l)[1:], clean):
            assert torch.isnan(a[1]).all() and torch.equal(a[[0, 2, 3, 4]], b[[0, 2, 3, 4]]), (V, l is None)


@pytest.mark.parametrize("rest", [False, True])
@pytest.mark.parametrize("N,V,dtype", HELD_AND_SPLIT)
def test_kept_statistics_of_a_distillation_lose_nothing(B, N, V, dtype, rest):
    """The row's sums are kept in the precision that the gradient takes them in: from them it comes out with the same bits."""
    index, value, lse = taught_by(B, logits_of(N, V, dtype, seed=3), min(V, 64))
    z = logits_of(N, V, dtype, seed=4)
    if rest:
        value -= 0.25                                                  # something is left over
    g, loss, loss2, dz, dz2 = three_ways(B, z, index, value, teacher_lse=torch.zeros(N, device=dev) if rest else None)
    assert torch.equal(loss, loss2) and torch.equal(dz, dz2)


@pytest.mark.parametrize("N,V,dtype", HELD_AND_SPLIT + [(700, 90, "fp32"), (300, 100001, "fp32")])
def test_the_loss_where_its_weights_stood(B, N, V, dtype):
    """The one array of qsl_distill_backward that may hold an input and an output."""
    index, value, lse = taught_by(B, logits_of(N, V, dtype, seed=3), 5)
    z = logits_of(N, V, dtype)
    for l in (None, torch.full((N,), 0.125, device=dev)):
        g, loss, loss2, dz, dz2 = three_ways(B, z, index, value, teacher_lse=l)
        both, dz3 = g.clone(), torch.empty_like(z)
        B.distill_backward(z, index, value, dz3, grad_loss=both, loss=both, teacher_lse=l)
        assert torch.equal(both, loss) and torch.equal(dz3, dz), (V, l is None)


@pytest.mark.parametrize("V", [40, 150001])
def test_arrays_between_rows_and_beside_the_workspace(B, V):
    """What lies in the gaps between rows, or right behind what it could be taken to overlap, is apart."""
    N, K = 6, 5
    held = torch.full((N, V + 60), 77.0, device=dev)
    z = held[:, :V]
    z.copy_(logits_of(N, V, "fp32"))
    t = torch.randint(0, V, (N,), generator=torch.Generator().manual_seed(1)).to(dev)
    gap = [held[n, V + (-V) % 4:][: 4 * N] for n in range(N)]             # 16-byte aligned if the row is
    need = B.logits_workspace_bytes(z, K)
    arena = torch.empty(need + 4096, dtype=torch.uint8, device=dev)
    behind = arena[need:].view(torch.float32)
    want = dict(logprob=new(N), entropy=new(N), lse=new(N), top_index=new(N, K, dtype=torch.int32), top_logprob=new(N, K), stats=new(N, 4))
    B.token_logprobs(z, t, **want)
    got = dict(logprob=gap[0][:N], entropy=gap[0][N:2 * N], lse=gap[1][:N], stats=behind[: 4 * N].view(N, 4), top_index=new(N, K, dtype=torch.int32),
               top_logprob=behind[4 * N:4 * N + N * K].view(N, K))
    B.token_logprobs(z, t, workspace=arena, **got)                        # larger than needed: only its first part is used
    for k in want:
        assert torch.equal(got[k], want[k]), k
    g = gap[2][:N].copy_(torch.linspace(-1, 1, N, device=dev))
    dz, dz2 = torch.empty(N, V, device=dev), torch.empty(N, V, device=dev)
    lp = gap[4][:N]
    B.token_logprobs_backward(z, t, dz, grad_logprob=g, logprob=lp)
    B.token_logprobs_backward(z, t, dz2, grad_logprob=g.clone(), logprob=want["logprob"])
    assert torch.equal(dz, dz2) and torch.equal(lp, want["logprob"])
    bad = [lambda: B.token_logprobs(z, t, logprob=z[1, :N]), lambda: B.token_logprobs_backward(z, t, dz, grad_logprob=g, logprob=g),
           lambda: B.token_logprobs_backward(z, t, dz, grad_logprob=dz[3, :N]), lambda: B.token_logprobs(z, t, logprob=lp, entropy=lp)]
    for f in bad:
        with pytest.raises(B.QslError):
            f()


@pytest.mark.parametrize("first", [True, False])
@pytest.mark.parametrize("gap", [0, 1])
@pytest.mark.parametrize("N,V,dtype", HELD_AND_SPLIT + [(200, 33, "fp16"), (130, 100003, "bf16")])
def test_gradient_rows_between_the_logits_rows(B, N, V, dtype, gap, first):
    """Two halves of one array: rows in turn, none of which shares an element with another."""
    held = torch.full((N, 2 * V + 2 * gap), 77.0, dtype=TYPES[dtype], device=dev)
    a, b = held[:, :V], held[:, V + gap:2 * V + gap]
    z, dz = (a, b) if first else (b, a)
    z.copy_(logits_of(N, V, dtype))
    before = z.clone()
    t, g = torch.randint(0, V, (N,), generator=torch.Generator().manual_seed(1)).to(dev), torch.linspace(-1, 1, N, device=dev)
    r = X.rows_of(z, 1.0)
    lp, stats = new(N), new(N, 4)
    B.token_logprobs(z, t, logprob=lp, stats=stats)
    for kw in ({}, dict(stats=stats)):
        dz.fill_(55.0)
        B.token_logprobs_backward(z, t, dz, grad_logprob=g, **kw)
        X.check(dz, *X.logprob_gradient(r, t, g, None, TYPES[dtype]), f"{N} x {V}")
        assert torch.equal(z, before)
    if N < 100:
        index, value, lse = taught_by(B, logits_of(N, V, dtype, seed=3), 5)
        apart = torch.empty_like(before)
        B.distill_backward(before, index, value, apart, grad_loss=g)
        B.distill_backward(z, index, value, dz, grad_loss=g)
        want, tol_loss, want_dz, tol = X.distill(r, index.cpu(), value.cpu(), 1.0, None, g.cpu(), TYPES[dtype])
        X.check(dz, want_dz, tol, f"{N} x {V}: distillation")
        assert torch.equal(z, before)
    if gap:
        assert (held[:, V] == 77).all() and (held[:, 2 * V + 1] == 77).all()


@pytest.mark.parametrize("N,V", [(140, 100003), (600, 140001), (3, 140001)])
def test_calls_that_need_no_workspace_take_none(B, N, V):
    """Straight through the C entry points, without the binding's allocation."""
    z, t = logits_of(N, V, "bf16"), torch.randint(0, V, (N,), generator=torch.Generator().manual_seed(1)).to(dev)
    index, value, lse = taught_by(B, z, 5)
    stats, want, dz = new(N, 4), torch.empty_like(z), torch.empty_like(z)
    lp, g, loss, want_loss = new(N), torch.linspace(-1, 1, N, device=dev), new(N), new(N)
    B.token_logprobs(z, t, logprob=lp, stats=stats)
    B.token_logprobs_backward(z, t, want, grad_logprob=g, stats=stats, workspace=torch.empty(B.logits_workspace_bytes(z), dtype=torch.uint8, device=dev))
    rows = B.C.byref(B._Logits(z.data_ptr(), V, N, V, 1, 1.0))
    stream = torch.cuda.current_stream().cuda_stream
    st = B._lib.qsl_token_logprobs_backward(rows, t.data_ptr(), g.data_ptr(), None, stats.data_ptr(), None, None, dz.data_ptr(), V, None, 0, stream)
    assert st == B.OK and torch.equal(dz, want)
    teacher = B.C.byref(B._Teacher(index.data_ptr(), value.data_ptr(), None, 5, 1.0))
    B.distill(z, index, value, loss=want_loss)
    st = B._lib.qsl_distill(rows, teacher, loss.data_ptr(), None, None, 0, stream)
    if B.logits_workspace_bytes(z) == 0:
        assert st == B.OK and torch.equal(loss, want_loss)
    else:
        assert st == B.ERR_INVALID_ARG
    st = B._lib.qsl_token_logprobs(rows, t.data_ptr(), 0, loss.data_ptr(), None, None, None, None, None, None, 0, stream)
    if N >= 512 or B.logits_workspace_bytes(z) == 0:                   # many rows: a block walks along each
        assert st == B.OK and torch.equal(loss, lp)
    else:
        assert st == B.ERR_INVALID_ARG


@pytest.mark.parametrize("N,V,dtype", HELD_AND_SPLIT)
def test_weights_that_are_no_numbers_on_rows_without_a_gradient(B, N, V, dtype):
    """A row of -inf has gradient 0, and so has one that nothing is taught in, whatever weight the caller's arithmetic made of them."""
    z = logits_of(N, V, dtype)
    z[0], z[1] = -INF, -INF
    t = torch.zeros(N, dtype=torch.int64, device=dev)
    t[1] = V - 1
    lp, stats = new(N), new(N, 4)
    B.token_logprobs(z, t, logprob=lp, stats=stats)
    for g0, g1 in ((NAN, INF), (INF, NAN), (-INF, 1.0)):
        g = torch.ones(N, device=dev)
        g[0], g[1] = g0, g1
        r = X.rows_of(z, 1.0)
        for h in (None, g):
            for kw in ({}, dict(stats=stats)):
                dz = torch.full_like(z, 55.0)
                B.token_logprobs_backward(z, t, dz, grad_logprob=g, grad_entropy=h, **kw)
                assert not dz[:2].any(), (V, g0, h is None)
                clean = torch.where(torch.isfinite(g), g, 0.0)
                X.check(dz, *X.logprob_gradient(r, t, clean, None if h is None else clean, TYPES[dtype]), f"{V}")
    index, value, lse = taught_by(B, logits_of(N, V, dtype, seed=3), 5)
    z = logits_of(N, V, dtype)
    value[0], lse[0] = -INF, -INF                                      # an empty teacher's row
    index[1] = -1                                                      # no entries
    z[2] = -INF                                                        # an empty student's
    for l in (None, torch.where(lse == -INF, lse, 0.0)):
        g = torch.ones(N, device=dev)
        g[0], g[1], g[2] = NAN, INF if l is None else 1.0, INF
        dz = torch.full_like(z, 55.0)
        B.distill_backward(z, index, value, dz, grad_loss=g, teacher_lse=l)
        assert not dz[[0, 2]].any() and (l is not None or not dz[1].any()) and torch.isfinite(dz).all(), (V, l is None)
