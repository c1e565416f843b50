"""Builds the CPU run of the feed-forward kernels (test infrastructure; main.cpp
says what it is) into tests/cpu_kernels/_build; reused while no source changed."""
from __future__ import annotations

import concurrent.futures
import hashlib
import os
import shutil
import subprocess

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(os.path.dirname(HERE))
CSRC = os.path.join(ROOT, "paper_2507_01040_amd", "csrc")
OUT = os.path.join(HERE, "_build")
EXE = os.path.join(OUT, "cpu_kernels")
CLANG = os.environ.get("CPU_CLANG", "/opt/rocm/llvm/bin/clang++")
OWN = ["main.cpp", "run_dense.cpp", "hip_runtime.h", "lds_load.hpp"]
TAKEN = ["common.hpp", "dense.hip", "dense_geom.hpp", "dropout.hip", "ff_api.cpp", "ff_common.hpp", "norm.hip",
         "rows.hpp", "split.hpp"]
UNITS = ["main.cpp", "run_dense.cpp", "norm.hip", "dropout.hip", "ff_api.cpp"]
# products fused with sums as on the GPU; pointers of tensors that are absent may be
# offset, as long as nothing is read there
FLAGS = ["-x", "c++", "-std=c++17", "-O2", "-g1", "-march=x86-64-v3", "-ffp-contract=fast", "-fno-omit-frame-pointer",
         "-fsanitize=address,undefined", "-fno-sanitize=pointer-overflow,alignment,vptr",
         "-fno-sanitize-recover=undefined", "-Wno-unknown-attributes", "-Wno-psabi"]


def build() -> str:
    include = os.path.join(ROOT, "include")
    paths = [os.path.join(HERE, f) for f in OWN] + [os.path.join(CSRC, f) for f in TAKEN] + \
        [os.path.join(include, f) for f in ("cliffconv.h", "cliffconv_ff.h")]
    h = hashlib.sha256(" ".join(FLAGS).encode())
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
        shutil.copy(os.path.join(CSRC, f), src)
    for f in OWN:
        shutil.copy(os.path.join(HERE, f), os.path.join(src, "hip") if f == "hip_runtime.h" else src)

    def compile_one(unit):
        obj = os.path.join(OUT, unit + ".o")
        r = subprocess.run([CLANG, *FLAGS, "-I" + src, "-I" + include, "-include", "hip/hip_runtime.h", "-c", os.path.join(src, unit), "-o", obj],
                           capture_output=True, text=True)
        if r.returncode:
            raise RuntimeError("%s: %s" % (unit, r.stderr[-4000:]))
        return obj
    with concurrent.futures.ThreadPoolExecutor(len(UNITS)) as ex:
        objs = list(ex.map(compile_one, UNITS))
    r = subprocess.run([CLANG, "-fsanitize=address,undefined", *objs, "-o", EXE], capture_output=True, text=True)
    if r.returncode:
        raise RuntimeError(r.stderr[-4000:])
    with open(stamp, "w") as f:
        f.write(h.hexdigest())
    return EXE


def _run(exe, cases, timeout):
    lines = [" ".join("%s=%s" % kv for kv in c.items()) for c in cases]
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=0:detect_stack_use_after_return=0:abort_on_error=1",
               UBSAN_OPTIONS="print_stacktrace=1:halt_on_error=1")
    r = subprocess.run([exe], input="\n".join(lines) + "\n", capture_output=True, text=True, env=env,
                       timeout=timeout)
    if r.returncode:
        at = ("\n" + r.stderr).count("\ncase ") - 1
        raise RuntimeError("case %s\n%s" % (lines[min(at, len(lines) - 1)], r.stderr[-6000:]))
    launches = [[s for s in part.split("\n")[1:] if s] for part in ("\n" + r.stderr).split("\ncase ")[1:]]
    return list(zip(r.stdout.strip().split("\n"), launches))


def run(cases, timeout=900, processes=4):
    """[(result line, launches' lines)] of the cases (dicts)."""
    exe = build()
    n = max(1, min(processes, len(cases) // 4))
    with concurrent.futures.ThreadPoolExecutor(n) as ex:
        parts = list(ex.map(lambda i: _run(exe, cases[i::n], timeout), range(n)))
    return [parts[i % n][i // n] for i in range(len(cases))]
