"""Compile the HIP sources for gfx950 (hipcc cross-compiles without a GPU): csrc/*.hip into lib/libw4a16.so, csrc/w8a8/*.hip into
lib/libw8a8.so.  `python -m paper_2505_22179_amd.build` rebuilds unconditionally."""
from __future__ import annotations

import glob
import hashlib
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


def _hipcc() -> str:
    return os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")


def _made_by(extra_flags: list[str] | None) -> str:
    """names the compiler and the flags: objects of one kind lie in a directory of that name, and a library is linked of one kind"""
    return hashlib.sha256("\0".join([_hipcc()] + HIPCC_FLAGS + (extra_flags or [])).encode()).hexdigest()[:16]


def _stamp(lib: str) -> str:
    """holds _made_by() of the library's objects; a library without it is judged by its time alone"""
    return os.path.join(os.path.dirname(lib), "_build", os.path.basename(lib) + ".made_by")


def _stale(lib: str, files: list[str], extra_flags: list[str] | None) -> bool:
    if _older(lib, files + _headers()):
        return True
    if not os.path.exists(_stamp(lib)):
        return False
    with open(_stamp(lib)) as f:
        return f.read() != _made_by(extra_flags)


def stale(extra_flags: list[str] | None = None) -> bool:
    return _stale(LIB, sources(), extra_flags)


def stale_w8a8(extra_flags: list[str] | None = None) -> bool:
    return _stale(LIB_W8A8, sources_w8a8(), extra_flags)


def _run(cmd: list[str]) -> None:
    proc = subprocess.run(cmd, capture_output=True, text=True)
    err = "\n".join(ln for ln in proc.stderr.splitlines() if NOISE not in ln)
    if proc.returncode != 0:
        raise RuntimeError("hipcc failed:\n" + err)
    if err.strip():
        print(err)


def _library(lib: str, files: list[str], force: bool, extra_flags: list[str] | None) -> str:
    """the objects (those that are out of date, or all), a few at a time, and the library of them"""
    flags, headers, made_by = HIPCC_FLAGS + (extra_flags or []), _headers(), _made_by(extra_flags)
    kept = os.path.join(os.path.dirname(lib), "_build", made_by)
    os.makedirs(kept, exist_ok=True)
    objects = {f: os.path.join(kept, os.path.basename(lib)[3:-3] + "_" + os.path.basename(f)[:-4] + ".o") for f in files}
    todo = [f for f in files if force or _older(objects[f], [f] + headers)]
    with ThreadPoolExecutor(max_workers=max(1, min(8, len(todo)))) as pool:
        list(pool.map(lambda f: _run([_hipcc()] + flags + ["-c", "-o", objects[f], f]), sorted(todo, key=os.path.getsize, reverse=True)))
    _run([_hipcc(), "--offload-arch=gfx950", "-fPIC", "-shared", "-o", lib] + [objects[f] for f in files])
    with open(_stamp(lib), "w") as f:
        f.write(made_by)
    return lib


def build(force: bool = True, extra_flags: list[str] | None = None) -> str:
    if not force and not stale(extra_flags):
        return LIB
    return _library(LIB, sources(), force, extra_flags)


def build_w8a8(force: bool = True, extra_flags: list[str] | None = None) -> str:
    if not force and not stale_w8a8(extra_flags):
        return LIB_W8A8
    return _library(LIB_W8A8, sources_w8a8(), force, extra_flags)


if __name__ == "__main__":
    print(build())
    print(build_w8a8())
