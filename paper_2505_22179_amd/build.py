"""Compile the HIP sources for gfx950 (hipcc cross-compiles without a GPU): csrc/*.hip into lib/libw4a16.so, csrc/w8a8/*.hip into
lib/libw8a8.so.  `python -m paper_2505_22179_amd.build` rebuilds unconditionally."""
from __future__ import annotations

import glob
import os
import subprocess
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIBDIR = os.path.join(HERE, "lib")
LIB = os.path.join(LIBDIR, "libw4a16.so")
LIB_W8A8 = os.path.join(LIBDIR, "libw8a8.so")
INCLUDE = os.path.join(os.path.dirname(HERE), "include")

# packed fp32 VALU instructions are switched off for every kernel in these libraries
HIPCC_FLAGS = ["-O3", "--offload-arch=gfx950", "-fPIC", "-std=c++17",
               "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
               "-mllvm", "-amdgpu-mfma-vgpr-form",   # MFMA results feed VALU scale folds: keep them in VGPRs
               "-Wall", "-Wno-unused-function", "-I" + INCLUDE]
NOISE = "is not a recognized feature for this target"


def sources() -> list[str]:
    return sorted(glob.glob(os.path.join(CSRC, "*.hip")))


def sources_w8a8() -> list[str]:
    return sorted(glob.glob(os.path.join(CSRC, "w8a8", "*.hip")))


def _headers() -> list[str]:
    return [f for d, ext in ((CSRC, "*.h"), (CSRC, "*.inc"), (INCLUDE, "*.h"), (os.path.join(CSRC, "w8a8"), "*.h")) for f in glob.glob(os.path.join(d, ext))]


def _older(path: str, deps: list[str]) -> bool:
    return not os.path.exists(path) or any(os.path.getmtime(d) > os.path.getmtime(path) for d in deps)


def stale() -> bool:
    return _older(LIB, sources() + _headers())


def stale_w8a8() -> bool:
    return _older(LIB_W8A8, sources_w8a8() + _headers())


def _run(cmd: list[str]) -> None:
    proc = subprocess.run(cmd, capture_output=True, text=True)
    err = "\n".join(ln for ln in proc.stderr.splitlines() if NOISE not in ln)
    if proc.returncode != 0:
        raise RuntimeError("hipcc failed:\n" + err)
    if err.strip():
        print(err)


def _library(lib: str, files: list[str], force: bool, extra_flags: list[str] | None) -> str:
    """the objects (those that are out of date, or all), a few at a time, and the library of them"""
    os.makedirs(LIBDIR, exist_ok=True)
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    flags, headers = HIPCC_FLAGS + (extra_flags or []), _headers()
    objects = {f: os.path.join(LIBDIR, os.path.basename(lib)[3:-3] + "_" + os.path.basename(f)[:-4] + ".o") for f in files}
    todo = [f for f in files if force or extra_flags or _older(objects[f], [f] + headers)]
    with ThreadPoolExecutor(max_workers=max(1, min(8, len(todo)))) as pool:
        list(pool.map(lambda f: _run([hipcc] + flags + ["-c", "-o", objects[f], f]), sorted(todo, key=os.path.getsize, reverse=True)))
    _run([hipcc, "--offload-arch=gfx950", "-fPIC", "-shared", "-o", lib] + [objects[f] for f in files])
    return lib


def build(force: bool = True, extra_flags: list[str] | None = None) -> str:
    if not force and not stale():
        return LIB
    return _library(LIB, sources(), force, extra_flags)


def build_w8a8(force: bool = True, extra_flags: list[str] | None = None) -> str:
    if not force and not stale_w8a8():
        return LIB_W8A8
    return _library(LIB_W8A8, sources_w8a8(), force, extra_flags)


if __name__ == "__main__":
    print(build())
    print(build_w8a8())
