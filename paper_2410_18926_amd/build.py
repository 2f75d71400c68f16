"""Build the HIP library: hipcc for gfx950 -> paper_2410_18926_amd/liblorann.so (in-tree)."""
from __future__ import annotations

import pathlib
import shutil
import subprocess
import tempfile

HERE = pathlib.Path(__file__).resolve().parent
SRCS = [HERE / "csrc" / n for n in ("lorann.hip", "states.hip", "states4.hip", "evict.hip")]      # the search; the state stores of 8 and 4 bits and their attention; eviction from them
LIB = HERE / "liblorann.so"

FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC",
    # packed fp32 instructions are kept off: some of their forms have produced wrong results on the test machines
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    # matrix-core results go to ordinary vector registers: the epilogues read every result register once, and
    # from the accumulation registers each read costs an extra move
    "-mllvm", "-amdgpu-mfma-vgpr-form=1",
    "-Wall", "-Wno-unused-function",
]


SAN_LIB = HERE / "liblorann_san.so"


def _compile_and_link(hipcc: str, flags: list, out: pathlib.Path, link=(), verbose: bool = False) -> str:
    """One object per source, compiled side by side, linked into `out`; the compiler's messages."""
    with tempfile.TemporaryDirectory() as tmp:
        objs = [str(pathlib.Path(tmp) / (src.stem + ".o")) for src in SRCS]
        cmds = [[hipcc, *flags, "-c", "-o", obj, str(src)] for src, obj in zip(SRCS, objs)]
        runs = []
        for cmd in cmds:
            if verbose:
                print(" ".join(cmd))
            runs.append(subprocess.Popen(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True))
        said = "".join(r.communicate()[0] for r in runs)
        ok = all(r.returncode == 0 for r in runs)
        if ok:
            res = subprocess.run([hipcc, "--offload-arch=gfx950", "-shared", "-fPIC", *link, "-o", str(out), *objs], capture_output=True, text=True)
            said, ok = said + res.stderr, res.returncode == 0
    said = "\n".join(l for l in said.splitlines() if "packed-fp32-ops" not in l)
    if not ok:
        raise RuntimeError(f"hipcc failed:\n{said}")
    return said


def build_sanitized() -> pathlib.Path:
    """The same library with AddressSanitizer and UndefinedBehaviorSanitizer in its HOST code (argument checks, index
    loading, workspace planning; device code is compiled as usual).  Load it with LORANN_LIB=<path> and clang's
    sanitizer runtime first in the process (sanitizer_runtime())."""
    hipcc = shutil.which("hipcc") or "/opt/rocm/bin/hipcc"
    checks = ["-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined"]
    flags = [f for f in FLAGS if f != "-O3"] + ["-O1", "-g", *checks, "-Xarch_host", "-fno-sanitize-recover=all", "-Xarch_host", "-fno-omit-frame-pointer"]
    _compile_and_link(hipcc, flags, SAN_LIB, link=checks)
    return SAN_LIB


def sanitizer_runtime() -> str:
    clang = pathlib.Path(shutil.which("hipcc") or "/opt/rocm/bin/hipcc").resolve().parent.parent / "llvm" / "bin" / "clang"
    if not clang.exists():
        clang = pathlib.Path("/opt/rocm/llvm/bin/clang")
    return subprocess.run([str(clang), "--print-file-name=libclang_rt.asan-x86_64.so"], check=True, capture_output=True, text=True).stdout.strip()


def sources():
    return SRCS + sorted((HERE / "csrc").glob("*.hpp")) + sorted((HERE.parent / "include").glob("*.h"))


def build(force: bool = True, verbose: bool = False) -> pathlib.Path:
    hipcc = shutil.which("hipcc") or "/opt/rocm/bin/hipcc"
    if not force and LIB.exists() and all(LIB.stat().st_mtime >= s.stat().st_mtime for s in sources()):
        return LIB
    err = _compile_and_link(hipcc, FLAGS, LIB, verbose=verbose)
    if verbose and err.strip():
        print(err)
    return LIB


if __name__ == "__main__":
    print(build(verbose=True))
