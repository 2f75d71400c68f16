"""Sums of weights, kept sums and buffers of the caller's have no gradient: a backward pass that reaches one raises, and a leaf that requires a gradient is refused before it is written to."""
import pytest
import torch


@pytest.fixture(params=["stand-in", pytest.param("gpu", marks=pytest.mark.gpu)])
def store(request, monkeypatch):
    """A small store.  Stand-in: the binding's own work on the CPU, with a library that notes its calls and computes nothing."""
    from paper_2410_18926_amd import states
    device, called = "cuda" if request.param == "gpu" else "cpu", []
    if request.param == "stand-in":
        class Library:
            def __getattr__(self, name):
                return lambda *_: 0 if name.endswith("workspace") else called.append(name) or 0
        monkeypatch.setattr(states, "lib", lambda: Library())
    st = states.States.empty(8, 2, 16, 64, device=device)
    st.called, st.on = called, device
    return st


def tables(st):
    return torch.tensor([[0, 1]], dtype=torch.int32, device=st.on), torch.tensor([20], dtype=torch.int32, device=st.on)


def calls(st):
    """Every call that answers with numbers, as functions of (what its answer follows from, the buffer to write to), and such a buffer's shape and type."""
    t, n = tables(st)
    q = torch.ones((1, 4, 64), dtype=torch.bfloat16, device=st.on)
    slots, ids = torch.arange(3, device=st.on), torch.zeros((1, 1), dtype=torch.int64, device=st.on)
    sums, to = torch.ones((1, 2, 32), device=st.on), torch.tensor([[4, 5]], dtype=torch.int32, device=st.on)
    ints = lambda: (torch.empty((1, 2, 20), dtype=torch.int32, device=st.on), torch.empty(1, dtype=torch.int32, device=st.on))  # noqa: E731
    return {
        "chunk": (q, lambda x, out: st.attend_chunk(x, t, n, out=out), q),
        "passages": (q, lambda x, out: st.attend_passages(x, ids, t, n, out=out), q),
        "weights of queries": (q, lambda x, out: st.attend_weights(x, t, n, out=out), sums),
        "weights on sums": (sums, lambda x, out: st.attend_weights(q, t, n, before=x, out=out), sums),
        "evict": (sums, lambda x, out: st.evict(t, n, x, 20, to, out=None if out is None else (*ints(), out))[2], sums),
        "read": (None, lambda x, out: st.read(slots, torch.float32, out=None if out is None else (out, torch.empty_like(out)))[0], torch.ones((3, 2, 64), device=st.on)),
    }


NAMES = ["chunk", "passages", "weights of queries", "weights on sums", "evict", "read"]


@pytest.mark.parametrize("name", NAMES)
def test_a_backward_pass_raises(store, name):
    given, call, like = calls(store)[name]
    if given is None:
        return
    x = given.clone().requires_grad_()
    y = call(x, None)
    assert y.requires_grad
    with pytest.raises(NotImplementedError, match="no gradient"):
        (y.float().sum() + x.float().sum()).backward()
    with torch.no_grad():
        assert not call(x, None).requires_grad
    assert not call(given, None).requires_grad


@pytest.mark.parametrize("name", NAMES)
def test_a_leaf_is_refused_before_it_is_written(store, name):
    given, call, like = calls(store)[name]
    for grad in (False, True):
        x = None if given is None else given.clone().requires_grad_(grad)
        wide = torch.full((2, *like.shape), 7.0, dtype=like.dtype, device=store.on, requires_grad=True)
        leaf = torch.full_like(like, 7.0).requires_grad_()
        for out in (leaf, wide[1]):
            before = len(store.called)
            with pytest.raises(ValueError, match="leaf"):
                call(x, out)
            assert (out == 7).all() and len(store.called) == before
        with torch.no_grad():
            call(x, leaf)


def test_sums_that_are_added_to_in_place(store):
    """before and out the same leaf: refused; the same result of another operation: written, and a backward pass raises."""
    t, n = tables(store)
    q = torch.ones((1, 4, 64), dtype=torch.bfloat16, device=store.on)
    leaf = torch.full((1, 2, 32), 7.0, device=store.on, requires_grad=True)
    with pytest.raises(ValueError, match="leaf"):
        store.attend_weights(q, t, n, before=leaf, out=leaf)
    assert (leaf == 7).all()
    sums = leaf * 1
    assert store.attend_weights(q, t, n, before=sums, out=sums) is sums
    with pytest.raises(NotImplementedError, match="no gradient"):
        sums.sum().backward()


@pytest.mark.parametrize("name", NAMES)
def test_a_buffer_with_a_graph_of_its_own(store, name):
    """What stood in the buffer is gone: the gradient of what was there before must not be taken for the answer's."""
    given, call, like = calls(store)[name]
    leaf = torch.full_like(like, 2.0).requires_grad_()
    out = leaf * 1
    y = call(given, out)
    with pytest.raises(NotImplementedError, match="no gradient"):
        y.float().sum().backward()
