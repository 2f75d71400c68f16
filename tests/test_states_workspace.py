"""A workspace handed to the binding is taken at its size in memory: one whose elements share memory (or lie apart) is refused, the library would write past its end."""
import pytest
import torch


def test_a_workspace_that_is_not_contiguous_is_refused(monkeypatch):
    from paper_2410_18926_amd import states
    given = []

    class Library:                            # notes what it is given, computes nothing
        @staticmethod
        def lorann_attend_chunk(*a):
            given.append(a[5:7])
            return 0

        @staticmethod
        def lorann_attend_passages(*a):
            given.append(a[10:12])
            return 0

    monkeypatch.setattr(states, "lib", lambda: Library)
    st = states.States.empty(4, 2, 16, 64, device="cpu")
    q = torch.zeros((1, 4, 64), dtype=torch.bfloat16)
    tables, lengths, ids = torch.tensor([[0, 1]], dtype=torch.int32), torch.tensor([20], dtype=torch.int32), torch.zeros((1, 1), dtype=torch.int64)
    good = torch.empty(1024, dtype=torch.float32)
    calls = [lambda w: st.attend_chunk(q, tables, lengths, workspace=w), lambda w: st.attend_passages(q, ids, tables, lengths, workspace=w)]
    for call in calls:
        for bad in (torch.empty(1).expand(1 << 20), torch.empty(16).view(16, 1).expand(16, 64), torch.empty(64, 64)[:, ::2]):
            with pytest.raises(ValueError, match="workspace must be contiguous"):
                call(bad)
        call(good)
    assert given == [(good.data_ptr(), 4096)] * 2
