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
