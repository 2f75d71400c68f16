"""Memory of another GPU is refused, each array by its name.  The HIP runtime's two answers that the checks rest on - which device memory is on, which device is current - come from a
stand-in, so no GPU is needed; every call here is refused before anything is enqueued."""
import os
import pathlib
import shutil
import subprocess
import sys

import pytest

ROOT = pathlib.Path(__file__).resolve().parent.parent

STAND_IN = r"""
#include <hip/hip_runtime_api.h>
static void* other = nullptr;                 // the one address that is memory of GPU 1; all below 64 KiB are of GPU 0
extern "C" void on_other_gpu(void* p) { other = p; }
extern "C" hipError_t hipGetDevice(int* device) { *device = 0; return hipSuccess; }
extern "C" hipError_t hipPointerGetAttributes(hipPointerAttribute_t* at, const void* p) {
    if ((size_t)p >= 65536) return hipErrorInvalidValue;
    *at = hipPointerAttribute_t{};
    at->type = hipMemoryTypeDevice;
    at->device = p == other;
    return hipSuccess;
}
"""

CHILD = r"""
import ctypes as C, sys
stand_in = C.CDLL(sys.argv[1], mode=C.RTLD_GLOBAL)         # (before the library: its symbols are found first)
stand_in.on_other_gpu.argtypes = [C.c_void_p]
from paper_2410_18926_amd import states as S
L = S.lib()
at = {n: 4096 + 256 * i for i, n in enumerate(("k_codes", "v_codes", "k_scales", "v_scales", "q", "out", "q_start", "tables", "lengths", "ids", "scores", "workspace", "k", "v", "slots"))}
st = S.CStates(at["k_codes"], at["v_codes"], at["k_scales"], at["v_scales"], 100000, 2, 16, 64)
qs = S.CQuestions(at["q"], at["out"], S.BF16, 4, 1, 1, 256, 64, 256, 64, at["q_start"], 0.125)
width = 8192
need = max(L.lorann_attend_workspace(st, qs, 0, width), L.lorann_attend_workspace(st, qs, 3, width))
assert need > 0
store = ["k_codes", "v_codes", "k_scales", "v_scales"]
calls = {
    "write": (lambda: L.lorann_states_write(st, at["k"], at["v"], S.BF16, 5, 128, 64, 128, 64, at["slots"], None), store + ["k", "v", "slots"]),
    "read": (lambda: L.lorann_states_read(st, at["slots"], 5, at["k"], at["v"], S.BF16, 128, 64, 128, 64, None), store + ["k", "v", "slots"]),
    "chunk": (lambda: L.lorann_attend_chunk(st, qs, at["tables"], width, at["lengths"], at["workspace"], need, None),
              store + ["q", "out", "q_start", "tables", "lengths", "workspace"]),
    "passages": (lambda: L.lorann_attend_passages(st, qs, at["ids"], 3, at["scores"], 1.0, at["tables"], width, at["lengths"], 7, at["workspace"], need, None),
                 store + ["q", "out", "q_start", "tables", "lengths", "ids", "scores", "workspace"]),
}
for call, (run, names) in calls.items():
    for name in names:
        stand_in.on_other_gpu(at[name])
        rc, said = run(), L.lorann_last_error().decode()
        assert rc == -1 and said.startswith(name + " ") and "GPU 1" in said, (call, name, rc, said)
        print(call, name, "refused", flush=True)
print("done")
"""


def test_memory_of_another_gpu_is_refused(tmp_path):
    from paper_2410_18926_amd import binding, build
    if not binding.LIB_PATH.exists():
        build.build()
    cxx = shutil.which("g++") or shutil.which("clang++")
    include = pathlib.Path(os.environ.get("ROCM_PATH", "/opt/rocm")) / "include"
    if cxx is None or not (include / "hip" / "hip_runtime_api.h").exists():
        pytest.skip("no C++ compiler or no HIP headers")
    src, lib = tmp_path / "stand_in.cpp", tmp_path / "stand_in.so"
    src.write_text(STAND_IN)
    subprocess.run([cxx, "-std=c++17", "-shared", "-fPIC", "-D__HIP_PLATFORM_AMD__", "-I", str(include), "-o", str(lib), str(src)], check=True)
    env = dict(os.environ, HIP_VISIBLE_DEVICES="-1", ROCR_VISIBLE_DEVICES="-1")          # (addresses made up here must never reach a GPU)
    res = subprocess.run([sys.executable, "-c", CHILD, str(lib)], cwd=ROOT, env=env, capture_output=True, text=True, timeout=600)
    assert res.returncode == 0 and res.stdout.endswith("done\n"), res.stdout[-2000:] + res.stderr[-4000:]
