"""Compile the HIP sources of this package into ``libkurtail.so`` for gfx950."""
import hashlib
import os
import subprocess
import tempfile
from concurrent.futures import ThreadPoolExecutor

_HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(_HERE, "csrc")
LIB = os.path.join(_HERE, "libkurtail.so")

HIPCC_FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC",
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wall", "-Wno-unused-function",
]


def sources():
    return [os.path.join(CSRC, f) for f in sorted(os.listdir(CSRC)) if f.endswith(".hip")]


def source_id():
    """16 hex digits over the contents of every file the library is compiled from (csrc/ and the C header).
    The library carries the id it was built from (kt_build_id()), so that the binding can tell a library that no
    longer matches its sources, whatever the files' time stamps say."""
    h = hashlib.sha256()
    files = [os.path.join(CSRC, f) for f in sorted(os.listdir(CSRC)) if f.endswith((".hip", ".h"))]
    files.append(os.path.join(os.path.dirname(_HERE), "include", "kt.h"))
    for f in files:
        h.update(os.path.basename(f).encode())
        with open(f, "rb") as fh:
            h.update(fh.read())
    return h.hexdigest()[:16]


def _hipcc(args):
    res = subprocess.run(["hipcc", *args], capture_output=True, text=True)
    noise = "is not a recognized feature for this target"
    err = "\n".join(l for l in res.stderr.splitlines() if noise not in l)
    if res.returncode != 0:
        raise RuntimeError("hipcc failed:\n" + err)
    return err


def compile_object(source, out):
    """One source file to an object; returns the compiler's warnings."""
    extra = os.environ.get("KT_HIPCC_EXTRA", "").split()  # developer knob: extra hipcc flags
    return _hipcc([*HIPCC_FLAGS, f'-DKT_BUILD_ID="{source_id()}"', *extra, "-c", source, "-o", out])


def link_library(objects):
    _hipcc(["--offload-arch=gfx950", "-shared", "-fPIC", *objects, "-o", LIB])
    return LIB


def build_library(verbose=False):
    """Always recompiles every source, side by side (cross-compiles without a GPU). Returns the library path."""
    with tempfile.TemporaryDirectory() as tmp:
        objects = [os.path.join(tmp, os.path.basename(s) + ".o") for s in sources()]
        with ThreadPoolExecutor(len(objects)) as pool:
            warnings = list(pool.map(compile_object, sources(), objects))
        link_library(objects)
    if verbose and any(w.strip() for w in warnings):
        print("\n".join(w for w in warnings if w.strip()))
    return LIB


if __name__ == "__main__":
    print(build_library(verbose=True))
