"""Builds the CPU run of the 8-bit operators and the block norm (test infrastructure;
block_main.cpp says what it is) into tests/cpu_kernels/_build; reused while no source
changed."""
from __future__ import annotations

import concurrent.futures
import hashlib
import os
import shutil
import subprocess

from . import build as B

OUT = os.path.join(B.OUT, "block")
EXE = os.path.join(OUT, "cpu_block_kernels")
OWN = ["main.cpp", "block_main.cpp", "run_dense.cpp", "run_int8.cpp", "hip_runtime.h", "int8_runtime.h", "block_lds_load.hpp"]
AS = {"hip_runtime.h": "hip/hip_runtime.h", "block_lds_load.hpp": "lds_load.hpp"}  # names in the build
TAKEN = B.TAKEN + ["ff_block_api.cpp", "quantize.hip", "dense_int8.hip", "block_norm.hip"]
UNITS = ["block_main.cpp", "run_dense.cpp", "run_int8.cpp", "quantize.hip", "block_norm.hip", "norm.hip", "dropout.hip",
         "ff_api.cpp", "ff_block_api.cpp"]


def build() -> str:
    include = os.path.join(B.ROOT, "include")
    paths = [os.path.join(B.HERE, f) for f in OWN] + [os.path.join(B.CSRC, f) for f in TAKEN] + \
        [os.path.join(include, f) for f in ("cliffconv.h", "cliffconv_ff.h")]
    h = hashlib.sha256(" ".join(B.FLAGS).encode())
    for p in paths:
        with open(p, "rb") as f:
            h.update(f.read())
    stamp = os.path.join(OUT, "digest")
    if os.path.exists(EXE) and os.path.exists(stamp):
        with open(stamp) as f:
            if f.read() == h.hexdigest():
                return EXE
    src = os.path.join(OUT, "src")
    os.makedirs(os.path.join(src, "hip"), exist_ok=True)
    for f in TAKEN:
        shutil.copy(os.path.join(B.CSRC, f), src)
    for f in OWN:
        shutil.copy(os.path.join(B.HERE, f), os.path.join(src, AS.get(f, f)))

    def compile_one(unit):
        obj = os.path.join(OUT, unit + ".o")
        r = subprocess.run([B.CLANG, *B.FLAGS, "-I" + src, "-I" + include, "-include", "int8_runtime.h", "-c",
                            os.path.join(src, unit), "-o", obj], capture_output=True, text=True)
        if r.returncode:
            raise RuntimeError("%s: %s" % (unit, r.stderr[-4000:]))
        return obj
    with concurrent.futures.ThreadPoolExecutor(len(UNITS)) as ex:
        objs = list(ex.map(compile_one, UNITS))
    r = subprocess.run([B.CLANG, "-fsanitize=address,undefined", *objs, "-o", EXE], capture_output=True, text=True)
    if r.returncode:
        raise RuntimeError(r.stderr[-4000:])
    with open(stamp, "w") as f:
        f.write(h.hexdigest())
    return EXE


def run(cases, timeout=900, processes=4):
    """[(result line, launches' lines)] of the cases (dicts)."""
    exe = build()
    n = max(1, min(processes, len(cases) // 4))
    with concurrent.futures.ThreadPoolExecutor(n) as ex:
        parts = list(ex.map(lambda i: B._run(exe, cases[i::n], timeout), range(n)))
    return [parts[i % n][i // n] for i in range(len(cases))]
