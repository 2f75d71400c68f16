"""Host-side checks of the state store's entry points that need no GPU: exported symbols, constants, structures, refusals before anything is enqueued."""
import ctypes as C
import pathlib
import re
import subprocess

import pytest
import torch

ROOT = pathlib.Path(__file__).resolve().parent.parent
HEADER = (ROOT / "include" / "lorann_states.h").read_text()


@pytest.fixture(scope="module")
def S():
    from paper_2410_18926_amd import binding, build, states
    if not binding.LIB_PATH.exists():
        build.build()
    states.lib()
    return states


def test_exports_and_constants(S):
    declared = set(re.findall(r"^(?:int|int64_t) (lorann_[a-z_]+)\(", HEADER, re.M))
    assert declared == set(S.EXPORTS)
    for name in declared:
        assert getattr(S.lib(), name) is not None
    for name, value in (("MIN_PAGE", S.MIN_PAGE), ("MAX_PAGE", S.MAX_PAGE), ("MAX_DIM", S.MAX_DIM), ("MAX_HEADS", S.MAX_HEADS), ("MAX_FOUND", S.MAX_FOUND)):
        assert int(re.search(rf"#define LORANN_{name} (\d+)", HEADER).group(1)) == value
    assert re.search(r"LORANN_F32 = 0, LORANN_F16 = 1, LORANN_BF16 = 2", HEADER) and (S.F32, S.F16, S.BF16) == (0, 1, 2)


def test_structures_have_the_headers_layout(S, tmp_path):
    """Offsets of every field, as a C compiler sees the header (which also shows that it is plain C)."""
    fields = [("lorann_states", n) for n, _ in S.CStates._fields_] + [("lorann_questions", n) for n, _ in S.CQuestions._fields_]
    src = tmp_path / "offsets.c"
    src.write_text('#include <stddef.h>\n#include <stdio.h>\n#include "lorann_states.h"\nint main(void) {\n' +
                   "".join(f'  printf("%zu\\n", offsetof({s}, {n}));\n' for s, n in fields) +
                   '  printf("%zu %zu\\n", sizeof(lorann_states), sizeof(lorann_questions));\n  return 0;\n}\n')
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Werror", "-I", str(ROOT / "include"), "-o", str(tmp_path / "offsets"), str(src)], check=True)
    said = subprocess.run([str(tmp_path / "offsets")], check=True, capture_output=True, text=True).stdout.split()
    mine = [getattr(S.CStates, n).offset for n, _ in S.CStates._fields_] + [getattr(S.CQuestions, n).offset for n, _ in S.CQuestions._fields_]
    assert [int(x) for x in said] == mine + [C.sizeof(S.CStates), C.sizeof(S.CQuestions)]


def store(S, **change):
    f = dict(k_codes=16, v_codes=16, k_scales=16, v_scales=16, pages=10, heads=2, page_size=16, dim=64)
    f.update(change)
    return S.CStates(**f)


def questions(S, **change):
    f = dict(q=16, out=16, type=S.BF16, heads=4, tokens=6, sequences=3, q_token=256, q_head=64, out_token=256, out_head=64, q_start=None, scale=0.125)
    f.update(change)
    return S.CQuestions(**f)


@pytest.mark.parametrize("change,code,word", [
    (dict(pages=0), -1, "page"), (dict(heads=0), -1, "head"), (dict(page_size=24), -1, "power of two"), (dict(page_size=8), -4, "page_size"),
    (dict(page_size=512), -4, "page_size"), (dict(dim=0), -1, "dim"), (dict(dim=80), -4, "dim"), (dict(dim=160), -4, "dim"), (dict(heads=2000), -4, "heads"),
    (dict(pages=2 ** 31), -4, "pages"),
])
def test_stores_that_are_refused(S, change, code, word):
    L, st, qs = S.lib(), store(S, **change), questions(S, heads=4000 if change.get("heads", 0) > 4 else 4)
    calls = [lambda: L.lorann_states_write(st, 16, 16, S.F32, 1, 64, 64, 64, 64, 16, None),
             lambda: L.lorann_states_read(st, 16, 1, 16, 16, S.F32, 64, 64, 64, 64, None),
             lambda: L.lorann_attend_chunk(st, qs, 16, 1, 16, None, 0, None),
             lambda: L.lorann_attend_passages(st, qs, 16, 1, None, 1.0, 16, 1, 16, 1, None, 0, None),
             lambda: L.lorann_attend_workspace(st, qs, 0, 1)]
    for call in calls:
        assert call() == code
        assert word.encode() in L.lorann_last_error()


@pytest.mark.parametrize("change,code,word", [
    (dict(type=0), -4, "F16"), (dict(type=9), -1, "type"), (dict(tokens=-1), -1, "tokens"), (dict(sequences=-1), -1, "sequences"), (dict(heads=3), -1, "multiple"),
    (dict(heads=0), -1, "multiple"), (dict(heads=2048), -4, "heads"), (dict(scale=float("inf")), -1, "scale"), (dict(scale=float("nan")), -1, "scale"), (dict(tokens=2 ** 40), -4, "tokens"),
])
def test_questions_that_are_refused(S, change, code, word):
    L, st, qs = S.lib(), store(S), questions(S, **change)
    for call in (lambda: L.lorann_attend_chunk(st, qs, 16, 1, 16, None, 0, None),
                 lambda: L.lorann_attend_passages(st, qs, 16, 1, None, 1.0, 16, 1, 16, 1, None, 0, None),
                 lambda: L.lorann_attend_workspace(st, qs, 2, 1)):
        assert call() == code
        assert word.encode() in L.lorann_last_error()


def test_other_refusals(S):
    L, st, qs = S.lib(), store(S), questions(S)

    def refused(code, word, rc):
        assert rc == code and word.encode() in L.lorann_last_error(), L.lorann_last_error()

    refused(-1, "NULL", L.lorann_attend_chunk(None, qs, 16, 1, 16, None, 0, None))
    refused(-1, "NULL", L.lorann_attend_chunk(st, None, 16, 1, 16, None, 0, None))
    refused(-1, "NULL", L.lorann_attend_workspace(None, qs, 0, 1))
    refused(-1, "NULL", L.lorann_states_write(None, 16, 16, 0, 1, 1, 1, 1, 1, 16, None))
    refused(-1, "NULL", L.lorann_states_write(store(S, v_scales=None), 16, 16, 0, 1, 1, 1, 1, 1, 16, None))
    refused(-1, "aligned", L.lorann_states_write(store(S, v_codes=24), 16, 16, 0, 1, 1, 1, 1, 1, 16, None))
    refused(-1, "type", L.lorann_states_write(st, 16, 16, 7, 1, 1, 1, 1, 1, 16, None))
    refused(-1, "tokens", L.lorann_states_read(st, 16, -1, 16, 16, 0, 1, 1, 1, 1, None))
    refused(-4, "tokens", L.lorann_states_read(st, 16, 2 ** 31, 16, 16, 0, 1, 1, 1, 1, None))
    refused(-1, "width", L.lorann_attend_chunk(st, qs, 16, -1, 16, None, 0, None))
    refused(-4, "longer", L.lorann_attend_chunk(st, qs, 16, 2 ** 30, 16, None, 0, None))
    refused(-1, "passages", L.lorann_attend_passages(st, qs, 16, 0, None, 1.0, 16, 1, 16, 1, None, 0, None))
    refused(-4, "passages", L.lorann_attend_passages(st, qs, 16, 5000, None, 1.0, 16, 1, 16, 1, None, 0, None))
    refused(-1, "passages", L.lorann_attend_passages(st, qs, 16, 1, None, 1.0, 16, 1, 16, -1, None, 0, None))
    refused(-1, "weight", L.lorann_attend_passages(st, qs, 16, 1, None, float("nan"), 16, 1, 16, 1, None, 0, None))
    refused(-4, "tokens", L.lorann_states_write(store(S, heads=1), 16, 16, 0, 2 ** 30, 1, 1, 1, 1, 16, None))
    refused(-4, "passages", L.lorann_attend_passages(st, qs, 16, 1, None, 1.0, 16, 1, 16, 2 ** 31, None, 0, None))
    # host memory where device memory is asked for
    host = torch.zeros(64, dtype=torch.float32)
    at = host.data_ptr() + (-host.data_ptr()) % 16
    here = store(S, k_codes=at, v_codes=at, k_scales=at, v_scales=at)
    refused(-1, "device pointer", L.lorann_states_write(here, at, at, 0, 1, 64, 64, 64, 64, at, None))
    refused(-1, "device pointer", L.lorann_attend_chunk(here, qs, at, 1, at, None, 0, None))


def test_calls_without_work_do_nothing(S):
    L, st = S.lib(), store(S)
    assert L.lorann_states_write(st, None, None, S.F16, 0, 64, 64, 64, 64, None, None) == 0
    assert L.lorann_states_read(st, None, 0, None, None, S.F16, 64, 64, 64, 64, None) == 0
    assert L.lorann_attend_chunk(st, questions(S, tokens=0), None, 1, None, None, 0, None) == 0
    assert L.lorann_attend_chunk(st, questions(S, tokens=0, sequences=0), None, 1, None, None, 0, None) == 0
    assert L.lorann_attend_passages(st, questions(S, tokens=0), None, 3, None, 1.0, None, 1, None, 1, None, 0, None) == 0


def test_workspace_grows_with_the_split_only(S):
    """One sequence with many keys is split over the GPU and joined; a call that fills it needs no workspace, and no plan asks for more than the
    joined pieces of a few thousand blocks."""
    L = S.lib()
    st = store(S, pages=10 ** 6, heads=8, dim=128)
    one = questions(S, heads=32, tokens=1, sequences=1)
    assert L.lorann_attend_workspace(st, one, 0, 1) == 0
    assert L.lorann_attend_workspace(st, one, 0, 8192) > 0
    assert L.lorann_attend_workspace(st, questions(S, heads=32, tokens=4096, sequences=1), 0, 64) == 0
    for tokens, sequences, found, width in ((1, 1, 0, 8192), (64, 64, 0, 512), (7, 7, 10, 100), (3000, 1, 0, 60000), (1, 1, 4096, 60000)):
        need = L.lorann_attend_workspace(st, questions(S, heads=32, tokens=tokens, sequences=sequences), found, width)
        assert 0 <= need <= 4096 * 32 * 130 * 4 + 4096 * 130 * 4, (tokens, sequences, found, width, need)
