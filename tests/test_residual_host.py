"""The operators on a residual stream without a GPU: the definitions that the GPU tests compare with, the refusals of the C entry points, which
come before any GPU work, and the binding's checks."""
import ctypes as C
import os

import numpy as np
import pytest
import torch
from torch._subclasses.fake_tensor import FakeTensorMode

import residual_util as X
from paper_1906_02367_amd.build import LIB_PATH

INVALID, TOO_SMALL = 1, 2
pytestmark = pytest.mark.filterwarnings("ignore:Accessing the data pointer of FakeTensor")      # the address of no memory is 0


class Rows(C.Structure):
    _fields_ = [("data", C.c_void_p), ("stride", C.c_uint64)]


class Drop(C.Structure):
    _fields_ = [("p", C.c_double), ("seed", C.c_uint64), ("round", C.c_uint64), ("round_at", C.c_void_p), ("row0", C.c_uint32)]


class Norm(C.Structure):
    _fields_ = [("rows", C.c_uint32), ("cols", C.c_uint32), ("dtype", C.c_uint32), ("weight_dtype", C.c_uint32), ("weight", C.c_void_p),
                ("eps", C.c_float)]


class DropoutArgs(C.Structure):
    _fields_ = [("rows", C.c_uint32), ("cols", C.c_uint32), ("dtype", C.c_uint32), ("x", Rows), ("residual", Rows), ("y", Rows), ("drop", Drop)]


class NormArgs(C.Structure):
    _fields_ = [("norm", Norm), ("x", Rows), ("residual", Rows), ("total", Rows), ("y", Rows), ("drop", Drop), ("out_dtype", C.c_uint32), ("group", C.c_uint32),
                ("scales", C.c_void_p)]


class BackArgs(C.Structure):
    _fields_ = [("norm", Norm), ("total", Rows), ("dy", Rows), ("dtotal", Rows), ("dresidual", Rows), ("dx", Rows), ("drop", Drop), ("dweight", C.c_void_p),
                ("workspace", C.c_void_p), ("workspace_bytes", C.c_size_t)]


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(LIB_PATH):
        from paper_1906_02367_amd import build
        build.build()
    l = C.CDLL(LIB_PATH)
    l.qsl_dropout.argtypes = [C.POINTER(DropoutArgs), C.c_void_p]
    l.qsl_rms_norm.argtypes = [C.POINTER(NormArgs), C.c_void_p]
    l.qsl_rms_norm_workspace_bytes.argtypes = [C.POINTER(Norm)]; l.qsl_rms_norm_workspace_bytes.restype = C.c_size_t
    l.qsl_rms_norm_backward.argtypes = [C.POINTER(BackArgs), C.c_void_p]
    return l


N, W, PITCH = 40, 1000, 1008                     # rows, columns, stride


def at(k):                                       # addresses that are never looked at, far apart
    return (1 << 40) + k * (1 << 24)


def a_drop(**kw):
    d = dict(p=0.1, seed=1, round=2, round_at=None, row0=0)
    d.update(kw)
    return Drop(**d)


def a_norm(**kw):
    d = dict(rows=N, cols=W, dtype=0, weight_dtype=0, weight=at(50), eps=1e-5)
    d.update(kw)
    return Norm(**d)


def drop_call(lib, n=N, cols=W, dtype=0, x=at(1), res=at(2), drop=None, y=at(3), **st):
    s = lambda k: st.get("s" + k, PITCH)
    return lib.qsl_dropout(C.byref(DropoutArgs(n, cols, dtype, Rows(x, s("x")), Rows(res, s("res")), Rows(y, s("y")), drop or a_drop())), None)


def norm_call(lib, norm=None, x=at(1), res=at(2), drop=None, total=at(3), y=at(4), out=0, group=0, scales=None, **st):
    s = lambda k: st.get("s" + k, PITCH)
    return lib.qsl_rms_norm(C.byref(NormArgs(norm or a_norm(), Rows(x, s("x")), Rows(res, s("res")), Rows(total, s("total")), Rows(y, s("y")), drop or a_drop(), out, group, scales)),
                            None)


def back_call(lib, norm=None, total=at(1), dy=at(2), dtotal=at(3), drop=None, dres=at(4), dx=at(5), dw=at(6), ws=at(7), n=1 << 20, **st):
    s = lambda k: st.get("s" + k, PITCH)
    return lib.qsl_rms_norm_backward(C.byref(BackArgs(norm or a_norm(), Rows(total, s("total")), Rows(dy, s("dy")), Rows(dtotal, s("dtotal")), Rows(dres, s("dres")), Rows(dx, s("dx")),
                                                      drop or a_drop(), dw, ws, n)), None)


def test_the_words_are_those_of_the_known_answers():
    for line in open(os.path.join(os.path.dirname(__file__), "golden", "philox4x32_10_kat.txt")):
        if not line.startswith("#"):
            v = [int(x, 16) for x in line.split()]
            assert [int(x) for x in X.philox(*v[:6])] == v[6:]


def test_the_masks_share_and_parts():
    k = X.kept(400, 1000, 0.3, seed=9, round=5)
    share = 400 * 1000
    assert abs(float(k.double().mean()) - X.threshold(0.3) / 65536) < 5 * (0.3 * 0.7 / share) ** 0.5
    assert torch.equal(X.kept(100, 1000, 0.3, seed=9, round=5, row0=300), k[300:])
    assert not torch.equal(X.kept(100, 1000, 0.3, seed=9, round=6, row0=300), k[300:])
    assert X.kept(3, 9, 0.0).all() and not X.kept(3, 9, 1.0).any()


def test_the_gradient_of_the_definition():
    g = torch.Generator().manual_seed(1)
    h = torch.randn(5, 37, generator=g, dtype=torch.float64, requires_grad=True)
    w = torch.randn(37, generator=g, dtype=torch.float64, requires_grad=True)
    dy, dt = torch.randn(5, 37, generator=g, dtype=torch.float64), torch.randn(5, 37, generator=g, dtype=torch.float64)
    y, _ = X.norm_of(h, torch.zeros_like(h), None, 1e-3)
    dh, dw = torch.autograd.grad((y * w * dy).sum() + (h * dt).sum(), (h, w))
    got, _, got_w, _ = X.backward(h, dy, w, 1e-3, dt)
    assert torch.allclose(got, dh, rtol=1e-12, atol=1e-12) and torch.allclose(got_w, dw, rtol=1e-12, atol=1e-12)


def test_drops_that_are_refused(lib):
    for kw in (dict(p=-0.1), dict(p=-1e-300), dict(p=1.0001), dict(p=float("nan")), dict(p=float("inf")), dict(round=1 << 62), dict(round_at=at(9) + 4), dict(row0=2 ** 32 - N + 1)):
        d = a_drop(**kw)
        assert drop_call(lib, drop=d) == INVALID and norm_call(lib, drop=d) == INVALID and back_call(lib, drop=d) == INVALID, kw


def test_dropout_arguments_that_are_refused(lib):
    for kw in (dict(x=None), dict(y=None), dict(dtype=3), dict(dtype=4), dict(n=1 << 31), dict(cols=0), dict(cols=1 << 31, sx=1 << 32, sres=1 << 32, sy=1 << 32), dict(x=at(1) + 2),
               dict(res=at(2) + 1), dict(y=at(3) + 2), dict(x=at(1) + 1, dtype=1), dict(sx=999), dict(sy=999), dict(sres=0), dict(sx=1 << 48)):
        assert drop_call(lib, **kw) == INVALID, kw
    assert lib.qsl_dropout(None, None) == INVALID and lib.qsl_rms_norm(None, None) == INVALID and lib.qsl_rms_norm_backward(None, None) == INVALID
    # y over a part of x or of the residual, or over them with another stride, or over the round
    for kw in (dict(y=at(1) + 4), dict(y=at(2) - 4 * PITCH), dict(y=at(1), sy=PITCH + 1), dict(y=at(2), sy=PITCH - 1), dict(drop=a_drop(round_at=at(3) + 4 * PITCH + 8))):
        assert drop_call(lib, **kw) == INVALID, kw
    assert drop_call(lib, n=0) == 0 and drop_call(lib, n=0, x=None, y=None, res=None) == 0


BAD_NORMS = [dict(rows=1 << 31), dict(cols=0), dict(cols=32769), dict(dtype=3), dict(weight_dtype=1), dict(dtype=1, weight_dtype=2), dict(weight=at(50) + 2), dict(eps=0.0), dict(eps=-1e-5),
             dict(eps=float("nan")), dict(eps=float("inf")), dict(eps=1e-31)]


@pytest.mark.parametrize("kw", BAD_NORMS)
def test_norms_that_are_refused(lib, kw):
    n = a_norm(**kw)
    wide = dict(sx=1 << 16, sres=1 << 16, stotal=1 << 16, sy=1 << 16)
    assert norm_call(lib, norm=n, **wide) == INVALID
    assert back_call(lib, norm=n, n=1 << 40, stotal=1 << 16, sdy=1 << 16, sdtotal=1 << 16, sdres=1 << 16, sdx=1 << 16) == INVALID
    assert lib.qsl_rms_norm_workspace_bytes(n) == 0
    assert lib.qsl_rms_norm_workspace_bytes(None) == 0


def test_norm_arguments_that_are_refused(lib):
    for kw in (dict(x=None), dict(y=None), dict(x=at(1) + 2), dict(res=at(2) + 2), dict(total=at(3) + 1), dict(y=at(4) + 2), dict(sx=W - 1), dict(sres=W - 1), dict(stotal=W - 1),
               dict(sy=W - 1), dict(out=1), dict(out=2), dict(out=5), dict(group=32), dict(scales=at(9)),                     # scales and groups of no codes
               dict(out=3), dict(out=4), dict(out=3, scales=at(9) + 2), dict(out=3, scales=at(9), group=16), dict(out=3, scales=at(9), group=96), dict(out=4, scales=at(9), group=256)):
        assert norm_call(lib, **kw) == INVALID, kw
    n0 = a_norm(rows=0)
    assert norm_call(lib, norm=n0) == 0 and norm_call(lib, norm=n0, x=None, y=None, res=None, total=None) == 0 and norm_call(lib, norm=n0, out=3) == 0


def test_norm_arrays_that_share_memory(lib):
    span = 4 * ((N - 1) * PITCH + W)
    clashes = [dict(total=at(1) + 4), dict(total=at(2) + 4 * PITCH), dict(total=at(1), stotal=PITCH + 1), dict(y=at(1), sy=PITCH + 1), dict(y=at(2) - 4), dict(total=at(4)), dict(y=at(3) + span - 4),
               dict(total=at(1), y=at(1)), dict(y=at(50)), dict(total=at(50) - span + 4), dict(drop=a_drop(round_at=at(4))), dict(drop=a_drop(round_at=at(3) + 8))]
    codes = [dict(y=at(1)), dict(y=at(2) + 100), dict(y=at(3) + span - 1), dict(scales=at(1)), dict(scales=at(2) + span - 4), dict(scales=at(3)), dict(scales=at(4) + 996), dict(scales=at(50) + 4 * W - 4),
             dict(scales=at(9), drop=a_drop(round_at=at(9) + 8))]
    for kw in clashes:
        assert norm_call(lib, **kw) == INVALID, kw
    for kw in codes:
        assert norm_call(lib, **{"out": 3, "scales": at(9), **kw}) == INVALID, kw


def test_gradient_arguments_that_are_refused(lib):
    for kw in (dict(total=None), dict(dy=None), dict(dres=None, dx=None, dw=None), dict(total=at(1) + 2), dict(dy=at(2) + 2), dict(dtotal=at(3) + 2), dict(dres=at(4) + 2), dict(dx=at(5) + 2),
               dict(dw=at(6) + 2), dict(stotal=W - 1), dict(sdy=W - 1), dict(sdtotal=W - 1), dict(sdres=W - 1), dict(sdx=W - 1), dict(ws=None), dict(ws=at(7) + 128)):
        assert back_call(lib, **kw) == INVALID, kw
    need = lib.qsl_rms_norm_workspace_bytes(a_norm())
    assert need >= 4 * W and need % 256 == 0
    assert back_call(lib, n=need - 1) == TOO_SMALL
    assert [lib.qsl_rms_norm_workspace_bytes(a_norm(rows=n)) for n in (0, 1, 2)] == [0, 0, 0]      # one block, whose sum is dweight
    assert back_call(lib, norm=a_norm(rows=0), dw=None, ws=None, n=0, total=None, dy=None) == 0


def test_gradient_arrays_that_share_memory(lib):
    need, span = lib.qsl_rms_norm_workspace_bytes(a_norm()), 4 * ((N - 1) * PITCH + W)
    clashes = [dict(dres=at(1) + 4), dict(dres=at(2), sdres=PITCH + 1), dict(dx=at(3) - 4 * PITCH), dict(dres=at(5)), dict(dx=at(4) + 4), dict(dres=at(1), dx=at(1)), dict(dres=at(50)), dict(dx=at(50) - span + 4),
               dict(dw=at(1)), dict(dw=at(2) - 4 * W + 4), dict(dw=at(3) + span - 4), dict(dw=at(4)), dict(dw=at(5) + 8), dict(dw=at(50)), dict(dw=at(7) + need - 512), dict(ws=at(1)), dict(ws=at(2) - 256),
               dict(ws=at(3)), dict(ws=at(4)), dict(ws=at(5)), dict(ws=at(50)), dict(ws=at(6)), dict(drop=a_drop(round_at=at(4))), dict(drop=a_drop(round_at=at(5) + 16)), dict(drop=a_drop(round_at=at(6))),
               dict(drop=a_drop(round_at=at(7)))]
    for kw in clashes:
        assert back_call(lib, **kw) == INVALID, kw


# ---- the binding ---------------------------------------------------------------------------------------------------------------
def test_the_bindings_structures_have_the_headers_layout(B):
    """What the binding packs, read back field by field by ctypes."""
    norm, drop = (3, 5, 1, 0, 1 << 40, 0.25), (0.5, 7, 9, 1 << 41, 11)
    m = [(k << 20, 100 + k) for k in range(1, 6)]
    flat = [v for pair in m for v in pair]

    def fields(s):
        return [x for f, _ in s._fields_ for x in (fields(getattr(s, f)) if isinstance(getattr(s, f), C.Structure) else [getattr(s, f)])]

    for cls, pack, values in ((Norm, B._PACK_NORM, [*norm]), (DropoutArgs, B._PACK_DROPOUT, [3, 5, 1, *flat[:6], *drop]), (NormArgs, B._PACK_RMS_NORM, [*norm, *flat[:8], *drop, 3, 64, 1 << 42]),
                              (BackArgs, B._PACK_RMS_NORM_BACKWARD, [*norm, *flat, *drop, 1 << 43, 1 << 44, 1 << 33])):
        raw = pack(*values)
        assert len(raw) == C.sizeof(cls) and fields(cls.from_buffer_copy(raw)) == values, cls


@pytest.fixture(scope="module")
def B():
    from paper_1906_02367_amd import binding
    return binding


def fake(*shape, dtype=torch.float32):
    return torch.empty(*shape, dtype=dtype, device="cuda")


def test_sizes_that_32_bits_do_not_hold_are_refused(B):
    with FakeTensorMode():
        for n, c in ((2 ** 31, 4), (2 ** 32 + 5, 8), (1, 2 ** 32 + 8), (1, 2 ** 31)):
            x, y = fake(n, c, dtype=torch.bfloat16), fake(n, c, dtype=torch.bfloat16)
            for call in (lambda: B.dropout(x, y, 0.5), lambda: B.rms_norm(x, y), lambda: B.rms_norm_backward(x, y, dresidual=y), lambda: B.rms_norm_workspace_bytes(x)):
                with pytest.raises(ValueError, match="2\\^31"):
                    call()


def test_numbers_of_the_random_words_that_are_refused(B):
    with FakeTensorMode():
        x, y = fake(4, 8), fake(4, 8)
        for kw in (dict(seed=2 ** 64), dict(seed=-1), dict(round=2 ** 62), dict(round=-1), dict(row0=2 ** 32), dict(row0=-1)):
            for call in (lambda: B.dropout(x, y, 0.5, **kw), lambda: B.rms_norm(x, y, p=0.5, **kw), lambda: B.rms_norm_backward(x, y, dresidual=x, p=0.5, **kw)):
                with pytest.raises(ValueError, match="2\\^64"):
                    call()
        with pytest.raises(ValueError, match="round_at"):
            B.dropout(x, y, 0.5, round_at=fake(2, dtype=torch.int64))
        with pytest.raises(ValueError, match="round_at"):
            B.dropout(x, y, 0.5, round_at=fake(1, dtype=torch.int32))


def test_tensors_that_are_refused(B):
    with FakeTensorMode():
        x, y, h = fake(4, 8), fake(4, 8), fake(4, 8, dtype=torch.bfloat16)
        for other in (h, fake(4, 9), fake(5, 8), fake(8), torch.empty(4, 8), fake(8, 4).t(), fake(1, 8).expand(4, 8), fake(4, 16)[:, ::2]):
            for call in (lambda: B.dropout(x, other, 0.5), lambda: B.dropout(x, y, 0.5, residual=other), lambda: B.rms_norm(x, other), lambda: B.rms_norm(x, y, residual=other),
                         lambda: B.rms_norm(x, y, total=other), lambda: B.rms_norm_backward(x, other, dresidual=y), lambda: B.rms_norm_backward(x, y, dresidual=other),
                         lambda: B.rms_norm_backward(x, y, dx=other), lambda: B.rms_norm_backward(x, y, dtotal=other, dx=y)):
                with pytest.raises(ValueError):
                    call()
        for other in (fake(9), fake(8, dtype=torch.float16), fake(8, dtype=torch.float64), fake(16)[::2], torch.empty(8)):
            for call in (lambda: B.rms_norm(h, h, weight=other), lambda: B.rms_norm_backward(h, h, weight=other, dresidual=h)):
                with pytest.raises(ValueError):
                    call()
        q = fake(4, 8, dtype=torch.float8_e4m3fn)
        for kw in (dict(scales=fake(4)), dict(scales=fake(4, 2)), dict(scales=fake(4, 1), group=-32), dict(scales=fake(4, 1), group=2 ** 32), dict(scales=fake(4, 1, dtype=torch.float16))):
            with pytest.raises(ValueError):
                B.rms_norm(x, q, **kw)
        for call in (lambda: B.dropout(fake(4, 8, dtype=torch.float64), y, 0.5), lambda: B.rms_norm(fake(2, 4, 8), fake(2, 4, 8)), lambda: B.dropout(torch.empty(4, 8), y, 0.5),
                     lambda: B.rms_norm_backward(x, y, dweight=fake(8, dtype=torch.bfloat16)), lambda: B.rms_norm_backward(x, y, dweight=fake(8), workspace=fake(100))):
            with pytest.raises(ValueError):
                call()
