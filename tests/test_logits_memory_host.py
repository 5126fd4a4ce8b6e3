"""Arrays that a call on logits writes and that share memory with what it reads, or with one another: refused before any GPU work."""
import ctypes as C
import os

import pytest

from test_logits_host import INVALID, Logits, Teacher, lib  # noqa: F401

# addresses that are never looked at: 4 rows of 200,000 (split) or 1,000 floats, everything else far apart
Z, DZ, FAR = 1 << 40, 1 << 41, 1 << 42


def at(k):
    return FAR + k * (1 << 24)


@pytest.fixture(params=[1000, 200_000])
def calls(request, lib):  # noqa: F811
    """Each call with arguments of its own, by name; those that are given replace them."""
    V = request.param
    z = lambda a: C.byref(Logits(a["z"], V + 8, 4, V, 0, 1.0))
    ws = 1 << 20

    def score(**kw):
        a = dict(z=Z, target=at(1), logprob=at(2), entropy=at(3), lse=at(4), top_index=at(5), top_logprob=at(6), stats=at(7), workspace=at(8), **{})
        a.update(kw)
        return lib.qsl_token_logprobs(z(a), a["target"], 5, a["logprob"], a["entropy"], a["lse"], a["top_index"], a["top_logprob"], a["stats"], a["workspace"], ws, None)

    def step(**kw):
        a = dict(z=Z, target=at(1), g=at(2), h=at(3), stats=None, logprob=at(4), entropy=at(5), dz=DZ, workspace=at(8))
        a.update(kw)
        return lib.qsl_token_logprobs_backward(z(a), a["target"], a["g"], a["h"], a["stats"], a["logprob"], a["entropy"], a["dz"], V + 8, a["workspace"], ws, None)

    def loss(**kw):
        a = dict(z=Z, index=at(1), value=at(2), tlse=at(3), loss=at(4), stats=at(5), workspace=at(8))
        a.update(kw)
        return lib.qsl_distill(z(a), C.byref(Teacher(a["index"], a["value"], a["tlse"], 5, 1.0)), a["loss"], a["stats"], a["workspace"], ws, None)

    def taught(**kw):
        a = dict(z=Z, index=at(1), value=at(2), tlse=at(3), g=at(6), stats=None, loss=at(4), dz=DZ, workspace=at(8))
        a.update(kw)
        return lib.qsl_distill_backward(z(a), C.byref(Teacher(a["index"], a["value"], a["tlse"], 5, 1.0)), a["g"], a["stats"], a["loss"], a["dz"], V + 8, a["workspace"], ws, None)

    return dict(score=score, step=step, loss=loss, taught=taught, split=V > 1000, V=V)


def test_an_output_over_an_input(calls):
    """Where rows are split, one block writes a row's log probability while others still read its weight."""
    V = calls["V"]
    row = lambda n, i: Z + 4 * (n * (V + 8) + i)
    for name, clashes in {
        "score": [dict(logprob=at(1)), dict(lse=at(1) + 28), dict(stats=at(1) - 48), dict(top_index=at(1) - 76), dict(entropy=Z), dict(lse=row(3, V - 1)),
                  dict(top_logprob=row(1, 0) - 76), dict(logprob=row(2, 0) - 12), dict(logprob=row(0, V + 5))],
        "step": [dict(logprob=at(2)), dict(entropy=at(3)), dict(logprob=at(3)), dict(entropy=at(2)), dict(logprob=at(2) + 12), dict(entropy=at(3) - 12), dict(logprob=at(1) + 28),
                 dict(logprob=row(1, 5)), dict(entropy=Z), dict(dz=at(2)), dict(dz=at(3) - 4 * V + 4), dict(dz=at(1)), dict(logprob=DZ), dict(logprob=DZ + 4 * (V + 5)),
                 dict(stats=DZ, logprob=None, entropy=None), dict(stats=DZ - 48, logprob=None, entropy=None), dict(dz=Z, g=row(1, 0)), dict(dz=Z, logprob=row(2, V - 1))],
        "loss": [dict(loss=at(1)), dict(loss=at(2) + 76), dict(loss=at(3)), dict(stats=at(3) - 112), dict(loss=row(0, 0)), dict(stats=row(2, 8) - row(2, 8) % 16)],
        "taught": [dict(loss=at(1)), dict(loss=at(2)), dict(loss=at(3)), dict(loss=at(6) + 4), dict(loss=at(6) - 4), dict(dz=at(1)), dict(dz=at(2)), dict(dz=at(3)), dict(dz=at(6)),
                   dict(stats=DZ, loss=None), dict(loss=row(1, 1)), dict(loss=DZ + 8)],
    }.items():
        for kw in clashes:
            assert calls[name](**kw) == INVALID, (name, kw)


def test_an_output_over_another(calls):
    for name, clashes in {
        "score": [dict(logprob=at(3)), dict(entropy=at(4) + 12), dict(top_index=at(6) - 76), dict(stats=at(2) - 48), dict(lse=at(7) + 60)],
        "step": [dict(logprob=at(5)), dict(entropy=at(4) - 12)],
        "loss": [dict(loss=at(5) + 124), dict(loss=at(5))],
    }.items():
        for kw in clashes:
            assert calls[name](**kw) == INVALID, (name, kw)


def test_the_workspace_over_others(calls):
    if not calls["split"]:
        return                                                         # short rows: it is not looked at
    for name, clashes in {
        "score": [dict(workspace=at(1)), dict(workspace=at(7) - 256), dict(workspace=Z + 256), dict(workspace=at(2))],
        "step": [dict(workspace=at(k)) for k in range(1, 6)] + [dict(workspace=Z), dict(workspace=DZ + 1024)],
        "loss": [dict(workspace=at(k)) for k in range(1, 6)] + [dict(workspace=Z)],
        "taught": [dict(workspace=at(k)) for k in (1, 2, 3, 4, 6)] + [dict(workspace=Z), dict(workspace=DZ)],
    }.items():
        for kw in clashes:
            assert calls[name](**kw) == INVALID, (name, kw)


@pytest.mark.parametrize("dtype,es", [(0, 4), (1, 2), (2, 2)])
def test_gradient_rows_that_share_elements_with_the_logits_rows(lib, dtype, es):  # noqa: F811
    """Rows of 1,000 with 2,000 from one to the next: the second array's may begin 1,000 elements behind or before the first's, nowhere else."""
    N, V, stride = 5, 1000, 2000
    t = C.byref(Teacher(at(1), at(2), None, 5, 1.0))
    for d in (1, 999, 1001, 1999, 2000, 2001, 2999, 3001, 4 * stride, 4 * stride + 999):
        for dz, ds in ((Z + es * d, stride), (Z - es * d, stride)):
            z = C.byref(Logits(Z, stride, N, V, dtype, 1.0))
            assert lib.qsl_token_logprobs_backward(z, at(3), at(4), None, None, None, None, dz, ds, None, 0, None) == INVALID, (d, dz < Z)
            assert lib.qsl_distill_backward(z, t, None, None, None, dz, ds, None, 0, None) == INVALID, (d, dz < Z)
    for dz, ds in ((Z + es * 1000, 2001), (Z + es * 1000, 1999), (Z, 2001)):                    # of another stride: not looked at so closely
        assert lib.qsl_token_logprobs_backward(C.byref(Logits(Z, stride, N, V, dtype, 1.0)), at(3), at(4), None, None, None, None, dz, ds, None, 0, None) == INVALID


def test_workspaces_that_no_call_needs(lib):  # noqa: F811
    """Rows of 128 to 256 KB, not few: only alternatives split them, and of those a call has at most 128."""
    z = C.byref(Logits(Z, 131072, 4096, 131072, 1, 1.0))
    need = [lib.qsl_logits_workspace_bytes(z, top) for top in (0, 1, 128, 129, 256)]
    assert need[0] == 0 and 0 < need[1] < need[2] and need[3:] == [0, 0]
    few = C.byref(Logits(Z, 131072, 100, 131072, 1, 1.0))               # few: split for gradients too
    need = [lib.qsl_logits_workspace_bytes(few, top) for top in (0, 1, 256)]
    assert 0 < need[0] < need[1] and need[0] < need[2]
