"""The binding's checks of the operators on logits, without a GPU: tensors that have a device, a type and a shape, but no memory."""
import pytest
import torch
from torch._subclasses.fake_tensor import FakeTensorMode

pytestmark = pytest.mark.filterwarnings("ignore:Accessing the data pointer of FakeTensor")      # the address of no memory is 0


@pytest.fixture(scope="module")
def B():
    from paper_1906_02367_amd import binding
    return binding


def fake(*shape, dtype=torch.float32):
    return torch.empty(*shape, dtype=dtype, device="cuda")


@pytest.mark.parametrize("N,V", [(1, 2 ** 32 + 10), (2 ** 32 + 5, 10), (2 ** 31, 4), (1, 2 ** 31), (0, 2 ** 32 + 1)])
def test_more_rows_or_classes_than_32_bits_count_are_refused(B, N, V):
    """A size of 2^32 + 10 would be 10 in the structure that the library is handed."""
    with FakeTensorMode():
        z, dz, t, one = fake(N, V, dtype=torch.bfloat16), fake(N, V, dtype=torch.bfloat16), fake(N, dtype=torch.int64), fake(N)
        index, value = fake(N, 3, dtype=torch.int32), fake(N, 3)
        for call in (lambda: B.logits_workspace_bytes(z), lambda: B.token_logprobs(z, t, logprob=one), lambda: B.token_logprobs_backward(z, t, dz, grad_logprob=one),
                     lambda: B.distill(z, index, value, loss=one), lambda: B.distill_backward(z, index, value, dz)):
            with pytest.raises(ValueError, match="2\\^31"):
                call()


def test_more_alternatives_or_entries_than_32_bits_count_are_refused(B):
    K = 2 ** 32 + 4
    with FakeTensorMode():
        z, dz = fake(1, 50), fake(1, 50)
        index, value = fake(1, K, dtype=torch.int32), fake(1, K)
        for call in (lambda: B.token_logprobs(z, top_index=index), lambda: B.token_logprobs(z, top_logprob=value),
                     lambda: B.distill(z, index, value, loss=fake(1)), lambda: B.distill_backward(z, index, value, dz)):
            with pytest.raises(ValueError, match=str(K)):
                call()


def test_the_workspace_of_a_number_that_32_bits_do_not_hold(B, monkeypatch):
    monkeypatch.setattr(B, "_rows_of", lambda t, what: (1 << 20, t.shape[1]))      # an address that is never looked at
    with FakeTensorMode():
        z = fake(2, 200_000)
        assert B.logits_workspace_bytes(z, 4) > 0
        assert [B.logits_workspace_bytes(z, top) for top in (2 ** 32 + 4, 2 ** 32, -1, -2 ** 32)] == [0] * 4


@pytest.mark.parametrize("N,V,few", [(4096, 131072, False), (100, 131072, True), (64, 50, None)])
def test_workspaces_that_the_binding_allocates(B, monkeypatch, N, V, few):
    """Only for calls that look at one."""
    given = {}

    def seen(name, at):
        def call(*args):
            given[name] = args[at]
            return B.OK
        return call

    monkeypatch.setattr(B, "_rows_of", lambda t, what: (1 << 20, t.shape[1]))      # an address that is never looked at
    monkeypatch.setattr(B, "_current_device", lambda: 0)
    monkeypatch.setattr(B, "_raw_stream", lambda device: None)
    for name in ("qsl_token_logprobs", "qsl_token_logprobs_backward", "qsl_distill", "qsl_distill_backward"):
        monkeypatch.setattr(B._lib, name, seen(name, -2))
    with FakeTensorMode():
        z, dz, t, one = fake(N, V, dtype=torch.bfloat16), fake(N, V, dtype=torch.bfloat16), fake(N, dtype=torch.int64), fake(N)
        index, value = fake(N, 64, dtype=torch.int32), fake(N, 64)
        need = [B.logits_workspace_bytes(z, top) for top in (0, 64)]
        B.token_logprobs(z, t, logprob=one, top_index=index)
        B.token_logprobs_backward(z, t, dz, grad_logprob=one)
        B.distill(z, index, value, loss=one)
        B.distill_backward(z, index, value, dz, stats=fake(N, 8))
        assert need[1] >= need[0] and (need[0] > 0) == bool(few) and (need[1] > 0) == (few is not None)
        assert given == {"qsl_token_logprobs": need[1], "qsl_token_logprobs_backward": need[0], "qsl_distill": need[1] if few else 0,
                         "qsl_distill_backward": need[1] if few else 0}
        B.token_logprobs_backward(z, t, dz, grad_logprob=one, stats=fake(N, 4))
        assert given["qsl_token_logprobs_backward"] == 0
