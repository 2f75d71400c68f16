"""Host-side checks of the 4-bit state store's entry points that need no GPU: exported symbols, structure, refusals before anything is enqueued; and of its reference."""
import ctypes as C
import pathlib
import re
import subprocess

import numpy as np
import pytest
import torch

import states4_reference as R4

ROOT = pathlib.Path(__file__).resolve().parent.parent
HEADER = (ROOT / "include" / "lorann_states4.h").read_text()


@pytest.fixture(scope="module")
def S():
    from paper_2410_18926_amd import binding, build, states
    if not binding.LIB_PATH.exists():
        build.build()
    states.lib()
    return states


def test_exports(S):
    from paper_2410_18926_amd import states4
    declared = set(re.findall(r"^(?:int|int64_t) (lorann_[a-z0-9_]+)\(", HEADER, re.M))
    assert declared == set(states4.EXPORTS)
    for name in declared:
        assert getattr(S.lib(), name) is not None


def test_structure_has_the_headers_layout(S, tmp_path):
    fields = [n for n, _ in S.CStates4._fields_]
    src = tmp_path / "offsets.c"
    src.write_text('#include <stddef.h>\n#include <stdio.h>\n#include "lorann_states4.h"\nint main(void) {\n' +
                   "".join(f'  printf("%zu\\n", offsetof(lorann_states4, {n}));\n' for n in fields) + '  printf("%zu\\n", sizeof(lorann_states4));\n  return 0;\n}\n')
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Werror", "-I", str(ROOT / "include"), "-o", str(tmp_path / "offsets"), str(src)], check=True)
    said = subprocess.run([str(tmp_path / "offsets")], check=True, capture_output=True, text=True).stdout.split()
    assert [int(x) for x in said] == [getattr(S.CStates4, n).offset for n in fields] + [C.sizeof(S.CStates4)]


def store(S, **change):
    f = dict(k_codes=16, v_codes=16, k_factors=16, v_factors=16, k_scales=16, v_scales=16, pages=10, heads=2, page_size=16, dim=64)
    f.update(change)
    return S.CStates4(**f)


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
    calls = [lambda: L.lorann_states4_write(st, 16, 16, S.F32, 1, 64, 64, 64, 64, 16, None),
             lambda: L.lorann_states4_read(st, 16, 1, 16, 16, S.F32, 64, 64, 64, 64, None),
             lambda: L.lorann_attend4_chunk(st, qs, 16, 1, 16, None, 0, None),
             lambda: L.lorann_attend4_passages(st, qs, 16, 1, None, 1.0, 16, 1, 16, 1, None, 0, None),
             lambda: L.lorann_attend4_workspace(st, qs, 0, 1)]
    for call in calls:
        assert call() == code
        assert word.encode() in L.lorann_last_error()


def test_other_refusals(S):
    L, st, qs = S.lib(), store(S), questions(S)

    def refused(code, word, rc):
        assert rc == code and word.encode() in L.lorann_last_error(), L.lorann_last_error()

    for name in ("k_codes", "v_codes", "k_factors", "v_factors", "k_scales", "v_scales"):
        refused(-1, "NULL", L.lorann_states4_write(store(S, **{name: None}), 16, 16, 0, 1, 1, 1, 1, 1, 16, None))
        refused(-1, "aligned", L.lorann_states4_write(store(S, **{name: 24 if "codes" in name else 18}), 16, 16, 0, 1, 1, 1, 1, 1, 16, None))
    refused(-1, "NULL", L.lorann_attend4_chunk(None, qs, 16, 1, 16, None, 0, None))
    refused(-1, "NULL", L.lorann_attend4_chunk(st, None, 16, 1, 16, None, 0, None))
    refused(-1, "NULL", L.lorann_attend4_workspace(None, qs, 0, 1))
    refused(-1, "type", L.lorann_states4_write(st, 16, 16, 7, 1, 1, 1, 1, 1, 16, None))
    refused(-1, "tokens", L.lorann_states4_read(st, 16, -1, 16, 16, 0, 1, 1, 1, 1, None))
    refused(-4, "F16", L.lorann_attend4_chunk(st, questions(S, type=0), 16, 1, 16, None, 0, None))
    refused(-1, "scale", L.lorann_attend4_chunk(st, questions(S, scale=float("nan")), 16, 1, 16, None, 0, None))
    refused(-1, "width", L.lorann_attend4_chunk(st, qs, 16, -1, 16, None, 0, None))
    refused(-1, "passages", L.lorann_attend4_passages(st, qs, 16, 0, None, 1.0, 16, 1, 16, 1, None, 0, None))
    refused(-1, "weight", L.lorann_attend4_passages(st, qs, 16, 1, None, float("nan"), 16, 1, 16, 1, None, 0, None))
    host = torch.zeros(64, dtype=torch.float32)
    at = host.data_ptr() + (-host.data_ptr()) % 16
    here = store(S, **{n: at for n in ("k_codes", "v_codes", "k_factors", "v_factors", "k_scales", "v_scales")})
    refused(-1, "device pointer", L.lorann_states4_write(here, at, at, 0, 1, 64, 64, 64, 64, at, None))
    refused(-1, "device pointer", L.lorann_attend4_chunk(here, qs, at, 1, at, None, 0, None))


def test_calls_without_work_do_nothing(S):
    L, st = S.lib(), store(S)
    assert L.lorann_states4_write(st, None, None, S.F16, 0, 64, 64, 64, 64, None, None) == 0
    assert L.lorann_states4_read(st, None, 0, None, None, S.F16, 64, 64, 64, 64, None) == 0
    assert L.lorann_attend4_chunk(st, questions(S, tokens=0), None, 1, None, None, 0, None) == 0
    assert L.lorann_attend4_passages(st, questions(S, tokens=0), None, 3, None, 1.0, None, 1, None, 1, None, 0, None) == 0


def test_the_bindings_own_checks(S):
    from paper_2410_18926_amd.states4 import States4
    st = States4.empty(4, 2, 16, 64, device="cpu")
    assert (st.pages, st.heads, st.page_size, st.dim) == (4, 2, 16, 64)
    good = {n: getattr(st, n) for n in R4.NAMES}
    for name, t in good.items():
        for bad in (t.to(torch.float64), t[:3], t.transpose(0, 1).contiguous().transpose(0, 1)):
            with pytest.raises(ValueError, match="codes|factors|scales"):
                States4(**dict(good, **{name: bad}))
    with pytest.raises(ValueError, match="odd"):
        States4.empty(4, 2, 16, 33, device="cpu")
    slots, x = torch.zeros(3, dtype=torch.int64), torch.zeros((3, 2, 64))
    with pytest.raises(ValueError, match="k must be"):
        st.write(x[:, :1], x, slots)
    with pytest.raises(ValueError, match="both"):
        st.write(x, x.half(), slots)
    with pytest.raises(ValueError, match="consecutive"):
        st.write(torch.zeros((3, 64, 2)).transpose(1, 2), x, slots)
    with pytest.raises(S.LorannError, match="device pointer"):
        st.write(x, x, slots)                                    # host memory: the library's refusal


def test_what_rows_are_held_as():
    """Nearest of the held values, halfway to the even code, nothing cut off; groups far below the row's largest keep factors of their own."""
    rng = np.random.default_rng(0)
    x = rng.normal(size=(300, 96)).astype(np.float32)
    x[:, 32:64] *= np.exp2(rng.integers(-16, 1, (300, 1))).astype(np.float32)
    code, byte, step = R4.quantise(x)
    back = R4.values(code, byte, step).astype(np.float64)
    unit = R4.factor_of(byte).repeat(32, 1) * step[:, None].astype(np.float64)
    grid = np.concatenate([R4.LEVELS, -R4.LEVELS]) * unit[..., None]
    best = np.abs(grid - x[..., None]).min(-1)
    assert (np.abs(back - x) <= best + 1e-6 * np.abs(x)).all()
    top = np.abs(x).reshape(300, 3, 32).max(-1)
    r = R4.factor_of(byte)
    assert (r * np.abs(x).max(1)[:, None] >= top).all() and (r <= np.maximum(1.125 * top / np.abs(x).max(1)[:, None], 2.0 ** -13) * (1 + 1e-12)).all()
    # exactly halfway: a = 6 makes the unit 1
    row = np.zeros((1, 32), np.float32)
    row[0, :9] = [6, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5, -5]
    assert (R4.quantise(row)[0][0, :9] == [7, 0, 2, 2, 4, 4, 6, 6, 14]).all()
