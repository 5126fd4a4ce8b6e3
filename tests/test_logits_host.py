"""The operators on logits without a GPU: the definitions that the GPU tests compare with, against differences and autograd in 64 bits,
and the refusals of the C entry points, which come before any GPU work."""
import ctypes as C
import math
import os
import subprocess
import sys

import pytest
import torch

import logits_util as X
from paper_1906_02367_amd.build import LIB_PATH

INVALID, TOO_SMALL = 1, 2


class Logits(C.Structure):
    _fields_ = [("data", C.c_void_p), ("stride", C.c_uint64), ("rows", C.c_uint32), ("vocab", C.c_uint32), ("dtype", C.c_uint32), ("scale", C.c_float)]


class Teacher(C.Structure):
    _fields_ = [("index", C.c_void_p), ("value", C.c_void_p), ("lse", C.c_void_p), ("top", C.c_uint32), ("scale", C.c_float)]


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(LIB_PATH):
        from paper_1906_02367_amd import build
        build.build()
    l = C.CDLL(LIB_PATH)
    vp, u32, u64, sz = C.c_void_p, C.c_uint32, C.c_uint64, C.c_size_t
    l.qsl_logits_workspace_bytes.argtypes = [C.POINTER(Logits), u32]; l.qsl_logits_workspace_bytes.restype = sz
    l.qsl_token_logprobs.argtypes = [C.POINTER(Logits), vp, u32, vp, vp, vp, vp, vp, vp, vp, sz, vp]
    l.qsl_token_logprobs_backward.argtypes = [C.POINTER(Logits), vp, vp, vp, vp, vp, vp, vp, u64, vp, sz, vp]
    l.qsl_distill.argtypes = [C.POINTER(Logits), C.POINTER(Teacher), vp, vp, vp, sz, vp]
    l.qsl_distill_backward.argtypes = [C.POINTER(Logits), C.POINTER(Teacher), vp, vp, vp, vp, u64, vp, sz, vp]
    return l


A = 1 << 20                                    # an address that is never looked at: every call here is refused first


def rows(**kw):
    d = dict(data=A, stride=1000, rows=4, vocab=1000, dtype=0, scale=1.0)
    d.update(kw)
    return Logits(**d)


BAD_ROWS = [dict(data=None), dict(data=A + 2), dict(data=A + 1, dtype=1), dict(stride=999), dict(stride=1 << 48), dict(stride=1 << 40, rows=1 << 30), dict(vocab=0), dict(vocab=1 << 31, stride=1 << 32),
            dict(rows=1 << 31), dict(dtype=3), dict(scale=0.0), dict(scale=-1.0), dict(scale=float("inf")), dict(scale=float("nan")), dict(scale=1e-38)]


@pytest.mark.parametrize("kw", BAD_ROWS)
def test_rows_that_are_refused(lib, kw):
    z = C.byref(rows(**kw))
    t = C.byref(Teacher(A, A, None, 4, 1.0))
    assert lib.qsl_token_logprobs(z, A, 0, A, None, None, None, None, None, None, 0, None) == INVALID
    assert lib.qsl_token_logprobs_backward(z, A, A, None, None, None, None, 1 << 36, 1000, None, 0, None) == INVALID
    assert lib.qsl_distill(z, t, A, None, None, 0, None) == INVALID
    assert lib.qsl_distill_backward(z, t, None, None, None, 1 << 36, 1000, None, 0, None) == INVALID
    assert lib.qsl_logits_workspace_bytes(z, 0) == 0


def test_log_probability_arguments_that_are_refused(lib):
    z = C.byref(rows())
    call = lambda target=A, top=0, lp=A, H=None, lse=None, ti=None, tl=None, stats=None, ws=None, n=0: \
        lib.qsl_token_logprobs(z, target, top, lp, H, lse, ti, tl, stats, ws, n, None)
    assert lib.qsl_token_logprobs(None, A, 0, A, None, None, None, None, None, None, 0, None) == INVALID
    assert call(target=None) == INVALID                                   # a log probability of nothing
    assert call(lp=None) == INVALID                                       # nothing asked for
    assert call(top=129, ti=A) == INVALID                                 # too many alternatives
    assert call(top=5) == INVALID and call(ti=A) == INVALID               # alternatives without a place, a place without alternatives
    assert lib.qsl_token_logprobs(C.byref(rows(vocab=4)), None, 5, None, None, None, A, None, None, None, 0, None) == INVALID     # more than classes
    for kw in (dict(target=A + 4), dict(lp=A + 2), dict(H=A + 2), dict(lse=A + 1), dict(top=2, ti=A + 2), dict(top=2, tl=A + 2), dict(stats=A + 4)):
        assert call(**kw) == INVALID, kw


def test_gradient_arguments_that_are_refused(lib):
    z = C.byref(rows())
    far = 1 << 36
    call = lambda target=A, g=A, h=None, stats=None, lp=None, H=None, dz=far, ds=1000: \
        lib.qsl_token_logprobs_backward(z, target, g, h, stats, lp, H, dz, ds, None, 0, None)
    assert call(g=None) == INVALID and call(target=None) == INVALID and call(target=None, g=None, h=A, lp=A) == INVALID
    assert call(stats=A, lp=A) == INVALID and call(stats=A, H=A) == INVALID
    assert call(dz=None) == INVALID and call(ds=999) == INVALID and call(dz=far + 2) == INVALID
    assert call(dz=A, ds=1001) == INVALID                                 # the logits with another stride
    assert call(dz=A + 4) == INVALID and call(dz=A + 4 * 3999) == INVALID and call(dz=A - 4 * 3999) == INVALID     # overlapping them
    assert call(stats=A + 8) == INVALID and call(g=A + 2) == INVALID and call(h=A + 2) == INVALID


def test_workspaces_that_are_refused(lib):
    """Long rows are split, and the parts' results meet in the caller's workspace."""
    z = C.byref(rows(vocab=200_000, stride=200_000, rows=2))
    need = [lib.qsl_logits_workspace_bytes(z, top) for top in (0, 5, 128, 256)]
    assert 0 < need[0] < need[1] < need[2] and all(n % 256 == 0 for n in need)
    assert lib.qsl_logits_workspace_bytes(z, 257) == 0
    t = C.byref(Teacher(A, A, None, 5, 1.0))
    calls = [lambda top, ws, n: lib.qsl_token_logprobs(z, A, top, A, None, None, A if top else None, None, None, ws, n, None),
             lambda top, ws, n: lib.qsl_token_logprobs_backward(z, A, A, None, None, None, None, 1 << 36, 200_000, ws, n, None),
             lambda top, ws, n: lib.qsl_distill(z, t, A, None, ws, n, None),
             lambda top, ws, n: lib.qsl_distill_backward(z, t, None, None, None, 1 << 36, 200_000, ws, n, None)]
    for k, call in enumerate(calls):
        top = 5 if k != 1 else 0
        n = need[1] if k != 1 else need[0]
        assert call(top, None, n) == INVALID and call(top, A + 128, n) == INVALID and call(top, A, n - 1) == TOO_SMALL, k
    assert lib.qsl_logits_workspace_bytes(C.byref(rows(vocab=10, stride=10, rows=6000)), 5) == 0        # short rows need none
    assert lib.qsl_logits_workspace_bytes(None, 0) == 0


def test_no_rows_is_no_work(lib):
    """Pointers that nothing is read from may be null; what says how rows look is checked all the same."""
    z = C.byref(rows(rows=0, data=None))
    assert lib.qsl_token_logprobs(z, None, 0, None, None, None, None, None, None, None, 0, None) == 0
    assert lib.qsl_token_logprobs_backward(z, None, None, None, None, None, None, None, 1000, None, 0, None) == 0
    t = C.byref(Teacher(None, None, None, 4, 1.0))
    assert lib.qsl_distill(z, t, None, None, None, 0, None) == 0
    assert lib.qsl_distill_backward(z, t, None, None, None, None, 1000, None, 0, None) == 0
    assert lib.qsl_token_logprobs(z, None, 129, None, None, None, None, None, None, None, 0, None) == INVALID
    assert lib.qsl_distill(z, C.byref(Teacher(None, None, None, 0, 1.0)), None, None, None, 0, None) == INVALID
    assert lib.qsl_token_logprobs_backward(z, None, None, None, None, None, None, None, 999, None, 0, None) == INVALID


def test_teachers_that_are_refused(lib):
    z = C.byref(rows())
    for t in (None, Teacher(None, A, None, 4, 1.0), Teacher(A, None, None, 4, 1.0), Teacher(A, A, None, 0, 1.0), Teacher(A, A, None, 257, 1.0), Teacher(A, A, None, 4, 0.0),
              Teacher(A, A, None, 4, float("nan")), Teacher(A + 2, A, None, 4, 1.0), Teacher(A, A + 2, None, 4, 1.0), Teacher(A, A, A + 2, 4, 1.0)):
        t = C.byref(t) if t else None
        assert lib.qsl_distill(z, t, A, None, None, 0, None) == INVALID
        assert lib.qsl_distill_backward(z, t, None, None, None, 1 << 36, 1000, None, 0, None) == INVALID
    t = C.byref(Teacher(A, A, None, 4, 1.0))
    assert lib.qsl_distill(z, t, None, None, None, 0, None) == INVALID
    assert lib.qsl_distill(z, t, A, A + 4, None, 0, None) == INVALID
    assert lib.qsl_distill_backward(z, t, None, A, A, 1 << 36, 1000, None, 0, None) == INVALID
    assert lib.qsl_distill_backward(z, t, None, None, None, A + 4, 1000, None, 0, None) == INVALID


def _definitions(z, t, index, value, lse, c):
    """The losses as written, for autograd."""
    logp = torch.log_softmax(c * z, 1)
    H = -(logp.exp() * logp).sum(1)
    u = c * value
    q = torch.exp(u - lse[:, None]) if lse is not None else torch.softmax(u, 1)
    at = logp.gather(1, index)
    kl = (q * (q.log() - at)).sum(1)
    if lse is not None:
        left, p_r = 1 - q.sum(1), 1 - at.exp().sum(1)
        kl = kl + left * (left.log() - p_r.log())
    return logp.gather(1, t[:, None]).squeeze(1), H, kl


@pytest.mark.parametrize("V,K,c", [(5, 2, 1.0), (40, 7, 0.5), (300, 64, 1.25)])
def test_definitions_against_autograd_and_differences(V, K, c):
    """The gradients that the kernels are held to are those of the losses: by autograd in 64 bits, and by central differences."""
    gen = torch.Generator().manual_seed(V)
    N = 4
    z = (1.5 * torch.randn(N, V, generator=gen)).float().double().requires_grad_(True)
    t = torch.randint(0, V, (N,), generator=gen)
    teach = 1.5 * torch.randn(N, V, generator=gen)
    value, index = torch.topk(teach, K, dim=1)
    lse = torch.logsumexp(c * teach.double(), 1).float()
    g, h = torch.randn(N, generator=gen).double(), torch.randn(N, generator=gen).double()
    r = X.rows_of(z, c)
    for rest in (None, lse):
        lp, H, kl = _definitions(z, t, index, value.double(), None if rest is None else rest.double(), c)
        d1, = torch.autograd.grad((g * lp + h * H).sum(), z, retain_graph=True)
        d2, = torch.autograd.grad((g * kl).sum(), z)
        mine1, _ = X.logprob_gradient(r, t, g, h, torch.float32)
        loss, _, mine2, _ = X.distill(r, index, value, c, rest, g, torch.float32)
        assert torch.allclose(mine1, d1, rtol=1e-9, atol=1e-11) and torch.allclose(mine2, d2, rtol=1e-7, atol=1e-9)
        assert torch.allclose(X.entropy(r)[0].squeeze(1), H.detach(), rtol=1e-12) and torch.allclose(loss, kl.detach(), rtol=1e-7, atol=1e-10)
        e = 1e-5
        d = torch.randn(N, V, generator=gen).double()
        up, dn = (_definitions(z.detach() + s * e * d, t, index, value.double(), None if rest is None else rest.double(), c) for s in (1, -1))
        for mine, f in ((mine1, lambda o: g * o[0] + h * o[1]), (mine2, lambda o: g * o[2])):
            diff = (f(up) - f(dn)) / (2 * e)
            assert torch.allclose((mine * d).sum(1), diff, rtol=1e-5, atol=1e-7)


def test_definitions_of_special_rows():
    z = torch.tensor([[-math.inf] * 4, [0.0, -math.inf, -math.inf, -math.inf], [1.0, 1.0, -0.0, 0.0]])
    r = X.rows_of(z, 1.0)
    H, _ = X.entropy(r)
    assert H.squeeze(1)[:2].tolist() == [0.0, 0.0]
    assert X.lse(r)[0].tolist()[:2] == [-math.inf, 0.0]
    assert X.target_logprob(r, torch.tensor([1, 1, -1]))[0].tolist() == [-math.inf, -math.inf, 0.0]
    index, lp, _ = X.top(r, 4)
    assert index.tolist() == [[0, 1, 2, 3], [0, 1, 2, 3], [0, 1, 2, 3]] and lp[0].tolist() == [-math.inf] * 4
    dz, _ = X.logprob_gradient(r, torch.tensor([0, 0, 0]), torch.ones(3), None, torch.float32)
    assert dz[0].tolist() == [0.0] * 4 and dz[1].tolist() == [0.0] * 4


def test_binding_without_a_library_raises_not_falls_back():
    """The binding has no other way to compute these: without the library its import fails."""
    src = ("import paper_1906_02367_amd.build as b; b.LIB_PATH = '/nonexistent/libqsl.so'\n"
           "try:\n    import paper_1906_02367_amd.binding\nexcept ImportError:\n    print('refused')\n")
    out = subprocess.run([sys.executable, "-c", src], capture_output=True, text=True, cwd=os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
    assert out.stdout.strip() == "refused", out.stdout + out.stderr
