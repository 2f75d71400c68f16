"""The attention over the state store has no gradient: its answers can be used forwards, and a backward pass that reaches them raises instead of leaving gradients out."""
import pytest
import torch


@pytest.fixture(params=["stand-in", pytest.param("gpu", marks=pytest.mark.gpu)])
def attend(request, monkeypatch):
    """(device, attend_chunk and attend_passages of a small store).  Stand-in: the binding's own work on the CPU, with a library that computes nothing."""
    from paper_2410_18926_amd import states
    device = "cuda" if request.param == "gpu" else "cpu"
    if request.param == "stand-in":
        class Library:
            lorann_attend_workspace = lorann_attend_chunk = lorann_attend_passages = staticmethod(lambda *_: 0)
        monkeypatch.setattr(states, "lib", lambda: Library)
    st = states.States.empty(4, 2, 16, 64, device=device)
    tables, lengths = torch.tensor([[0, 1]], dtype=torch.int32, device=device), torch.tensor([20], dtype=torch.int32, device=device)
    ids = torch.zeros((1, 1), dtype=torch.int64, device=device)
    return device, [lambda q, scores=None, **k: st.attend_chunk(q, tables, lengths, **k),
                    lambda q, scores=None, **k: st.attend_passages(q, ids, tables, lengths, scores=scores, **k)]


def queries(device, grad):
    return torch.ones((1, 4, 64), dtype=torch.bfloat16, device=device, requires_grad=grad)


def test_a_backward_pass_raises(attend):
    device, calls = attend
    for call in calls:
        x = torch.ones((), device=device, requires_grad=True)
        y = call(queries(device, True)) * x           # a loss with another way to its inputs
        with pytest.raises(NotImplementedError, match="no gradient"):
            y.float().sum().backward()
        whole = torch.zeros((1, 6, 64), dtype=torch.bfloat16, device=device)
        out = whole[:, 1:5]
        y = call(queries(device, True), out=out)
        assert y is out
        with pytest.raises(NotImplementedError, match="no gradient"):
            whole.float().sum().backward()
    scores = torch.ones((1, 1), device=device, requires_grad=True)
    with pytest.raises(NotImplementedError, match="no gradient"):
        calls[1](queries(device, False), scores=scores).float().sum().backward()


def test_forward_use_is_left_alone(attend):
    device, calls = attend
    for call in calls:
        assert not call(queries(device, False)).requires_grad
        with torch.no_grad():
            assert not call(queries(device, True)).requires_grad
        out = torch.empty((1, 4, 64), dtype=torch.bfloat16, device=device)
        assert call(queries(device, False), out=out) is out


def test_a_buffer_used_again_grows_no_chain(attend):
    device, calls = attend
    for call in calls:
        out = torch.empty((1, 4, 64), dtype=torch.bfloat16, device=device)
        for _ in range(5):
            y = call(queries(device, True), out=out)
            assert y is out and all(f is None or f.name().endswith("AccumulateGrad") for f, _ in y.grad_fn.next_functions)
        with pytest.raises(NotImplementedError, match="no gradient"):
            y.float().sum().backward()
