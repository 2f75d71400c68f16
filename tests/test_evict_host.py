"""Host-side checks of the sums of weights and of eviction that need no GPU: exported symbols, refusals before anything is enqueued, the binding's own checks."""
import pathlib
import re

import pytest
import torch

from test_states4_host import questions

ROOT = pathlib.Path(__file__).resolve().parent.parent
HEADER = (ROOT / "include" / "lorann_evict.h").read_text()


@pytest.fixture(scope="module")
def S():
    from paper_2410_18926_amd import binding, build, states
    if not binding.LIB_PATH.exists():
        build.build()
    states.lib()
    return states


def test_exports(S):
    declared = set(re.findall(r"^(?:int|int64_t) (lorann_[a-z0-9_]+)\(", HEADER, re.M))
    assert declared == set(S.EVICT_EXPORTS)
    for name in declared:
        assert getattr(S.lib(), name) is not None


@pytest.fixture(params=["", "4"])
def A(S, request):
    """(weights, its workspace, evict) of one of the stores, as functions of what changes in a good call."""
    L, bits = S.lib(), request.param
    make = S.CStates4 if bits else S.CStates

    def store(at=16, **change):
        f = {n: at for n, _ in make._fields_ if n not in ("pages", "heads", "page_size", "dim")}
        f.update(dict(pages=10, heads=2, page_size=16, dim=64), **change)
        return make(**f)

    def weights(st=None, qs=None, tables=16, width=1, lengths=16, before=16, sums=16, ws=None, size=0):
        return getattr(L, f"lorann_attend{bits}_weights")(store() if st is None else st, questions(S) if qs is None else qs, tables, width, lengths, before, sums, ws, size, None)

    def room(st=None, qs=None, width=1):
        return getattr(L, f"lorann_attend{bits}_weights_workspace")(store() if st is None else st, questions(S) if qs is None else qs, width)

    def evict(st=None, tables=16, width=4, lengths=16, sequences=2, sums=16, budget=20, recent=5, to=16, to_width=2, kept=16, left=16, kept_sums=16):
        return getattr(L, f"lorann_states{bits}_evict")(store() if st is None else st, tables, width, lengths, sequences, sums, budget, recent, to, to_width, kept, left, kept_sums, None, 0, None)

    return L, store, weights, room, evict


def refused(L, code, word, rc):
    assert rc == code and word.encode() in L.lorann_last_error(), L.lorann_last_error()


@pytest.mark.parametrize("change,code,word", [
    (dict(pages=0), -1, "page"), (dict(heads=0), -1, "head"), (dict(page_size=24), -1, "power of two"), (dict(page_size=8), -4, "page_size"), (dict(dim=80), -4, "dim"),
    (dict(dim=160), -4, "dim"), (dict(pages=2 ** 31), -4, "pages"),
])
def test_stores_that_are_refused(A, change, code, word):
    L, store, weights, room, evict = A
    for call in (weights, room, evict):
        refused(L, code, word, call(st=store(**change)))


def test_other_refusals(S, A):
    L, store, weights, room, evict = A
    for call in (weights, room):
        refused(L, -1, "multiple", call(qs=questions(S, heads=3)))
        refused(L, -4, "F16", call(qs=questions(S, type=0)))
        refused(L, -1, "scale", call(qs=questions(S, scale=float("inf"))))
        refused(L, -1, "width", call(width=-1))
        refused(L, -4, "longer", call(width=2 ** 27))
        refused(L, -1, "tokens", call(qs=questions(S, tokens=-1)))
        refused(L, -4, "sequences", call(qs=questions(S, tokens=70000, sequences=70000)))
    refused(L, -1, "divide", weights(qs=questions(S, tokens=7, sequences=3)))
    refused(L, -1, "newest", evict(recent=-1))
    refused(L, -1, "newest", evict(recent=21))
    refused(L, -1, "budget", evict(budget=-1, recent=0))
    refused(L, -1, "hold no", evict(budget=33))
    refused(L, -1, "width", evict(width=-1))
    refused(L, -1, "width", evict(to_width=-1, budget=0, recent=0))
    refused(L, -4, "longer", evict(width=2 ** 27))
    refused(L, -4, "sequences", evict(sequences=70000))
    refused(L, -1, "sequences", evict(sequences=-1))
    refused(L, -1, "NULL", evict(st=store(k_codes=None)))
    refused(L, -1, "aligned", evict(st=store(k_codes=24)))
    # host memory where device memory is asked for
    host = torch.zeros(64, dtype=torch.float32)
    at = host.data_ptr() + (-host.data_ptr()) % 16
    refused(L, -1, "device pointer", weights(st=store(at)))
    refused(L, -1, "device pointer", evict(st=store(at)))
    assert L.lorann_evict_workspace(0, 16, 1) == -1 and L.lorann_evict_workspace(1, -1, 1) == -1 and L.lorann_evict_workspace(1, 16, -1) == -1


def test_calls_without_work_do_nothing(S, A):
    L, store, weights, room, evict = A
    assert weights(qs=questions(S, tokens=0, sequences=0), tables=None, lengths=None, before=None, sums=None) == 0
    assert weights(width=0, tables=None, lengths=None, before=None, sums=None) == 0
    assert evict(sequences=0, tables=None, lengths=None, sums=None, to=None, kept=None, left=None, kept_sums=None) == 0
    assert room(qs=questions(S, tokens=0)) == 0 and room(width=0) == 0


def test_workspace_stays_within_its_limits(S, A):
    """Scores are kept for few rows and 1 GiB at most; otherwise the operands of the queries and three or four numbers of a row."""
    L, store, weights, room, evict = A
    st = store(pages=10 ** 6, heads=8, dim=128)
    for tokens, sequences, width in ((1, 1, 250), (64, 64, 512), (64, 64, 8192), (1, 1, 8192), (4096, 1, 2048), (300, 3, 60000), (5000, 5000, 4)):
        need = room(st=st, qs=questions(S, heads=32, tokens=tokens, sequences=sequences), width=width)
        rows = 32 * tokens
        splits = max(512, -(-width * 16 // 16384))
        assert 0 < need <= max(min(rows * (width * 16 + 64) * 4, 2 ** 30), (rows + 64 * 8 * (sequences + 1)) * (256 + 12)) + 8 * splits * (rows + 8 * 64 * (sequences + 1)), (tokens, sequences, width, need)


def test_the_bindings_own_checks(S):
    from paper_2410_18926_amd.states4 import States4
    for Store in (S.States, States4):
        st = Store.empty(8, 2, 16, 64, device="cpu")
        q, tables, lengths = torch.zeros((2, 4, 64), dtype=torch.float16), torch.zeros((2, 3), dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
        sums, to = torch.zeros((2, 2, 48)), torch.zeros((2, 2), dtype=torch.int32)
        for bad in (sums[:, :, :40], sums.double(), sums[:1], torch.zeros((2, 48, 2)).transpose(1, 2)):
            with pytest.raises(ValueError, match="before"):
                st.attend_weights(q, tables, lengths, before=bad)
            with pytest.raises(ValueError, match="out"):
                st.attend_weights(q, tables, lengths, out=bad)
            with pytest.raises(ValueError, match="sums"):
                st.evict(tables, lengths, bad, 20, to)
        with pytest.raises(ValueError, match="q must be"):
            st.attend_weights(q[:, :, :32], tables, lengths)
        with pytest.raises(ValueError, match="tables"):
            st.attend_weights(q, tables.long(), lengths)
        with pytest.raises(ValueError, match="lengths"):
            st.evict(tables, lengths[:1], sums, 20, to)
        with pytest.raises(ValueError, match="to_tables"):
            st.evict(tables, lengths, sums, 20, to.long())
        with pytest.raises(ValueError, match="to_tables"):
            st.evict(tables, lengths, sums, 20, to[:1])
        with pytest.raises(ValueError, match="workspace must be contiguous"):
            st.attend_weights(q, tables, lengths, workspace=torch.empty(1).expand(1 << 20))
        with pytest.raises(S.LorannError, match="budget"):
            st.evict(tables, lengths, sums, 20, to, recent=30)
        with pytest.raises(S.LorannError, match="device pointer"):
            st.attend_weights(q, tables, lengths)
        with pytest.raises(S.LorannError, match="device pointer"):
            st.evict(tables, lengths, sums, 20, to)
