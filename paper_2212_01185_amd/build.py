"""Build libpcc.so (HIP, gfx950) in-tree next to the package."""
from __future__ import annotations

import os
import subprocess
import sys
import tempfile

_HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(_HERE)
SRC = os.path.join(_HERE, "csrc", "pcc.hip")                # the codec
TRAIN_SRC = os.path.join(_HERE, "csrc", "pcc_train.hip")    # the operators of a training step
ROUTED_SRC = os.path.join(_HERE, "csrc", "pcc_routed.hip")  # the operators round the grouped products
LIB = os.path.join(_HERE, "libpcc.so")

HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-shared",
    # encoder and decoder must round identically: no contraction the source does not spell out
    "-ffp-contract=off",
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    # MFMA results land in vector registers proper (the vector ALU reads them without a copy per register); the
    # decoder's resident weights, which only the matrix cores read, go to the accumulation registers instead
    "-mllvm", "-amdgpu-mfma-vgpr-form",
    "-Wall", "-Wno-unused-function",
    "-I" + os.path.join(ROOT, "include"),
    "-I" + os.path.join(_HERE, "csrc"),
]


def _start(cmd, verbose: bool):
    if verbose:
        print(" ".join(cmd), flush=True)
    return subprocess.Popen(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)


def _finish(process):
    out, _ = process.communicate()
    return process.returncode, "\n".join(l for l in out.splitlines() if "packed-fp32-ops" not in l)


def build(verbose: bool = False, extra=(), lib: str = LIB, src=(SRC, TRAIN_SRC, ROUTED_SRC)) -> str:
    """Compile the library to `lib` (default: libpcc.so next to the package).  `extra` are more hipcc flags, e.g.
    -DPCC_PHASE_TIMING for the measurement build that counts the decode step's cycles per phase.  `src` is another HIP
    source, or several, to compile with the library's flags."""
    LIB = lib
    os.makedirs(os.path.dirname(os.path.abspath(LIB)), exist_ok=True)
    tmp = LIB + ".tmp%d" % os.getpid()
    sources = [src] if isinstance(src, str) else list(src)
    # each source by itself, side by side, then all together
    with tempfile.TemporaryDirectory(dir=os.path.dirname(os.path.abspath(LIB))) as d:
        objects = [os.path.join(d, "%d.o" % i) for i in range(len(sources))]
        running = [_start([HIPCC] + [f for f in FLAGS if f != "-shared"] + list(extra) + ["-c", "-o", o, s], verbose) for o, s in zip(objects, sources)]
        out = [_finish(p) for p in running]
        if all(rc == 0 for rc, _ in out):
            out.append(_finish(_start([HIPCC, "--offload-arch=gfx950", "-fPIC", "-shared"] + list(extra) + ["-o", tmp] + objects, verbose)))
    text = "\n".join(t for _, t in out if t)
    if any(rc != 0 for rc, _ in out):
        raise RuntimeError("hipcc failed:\n" + text)
    if verbose and text.strip():
        print(text)
    os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    # python -m paper_2212_01185_amd.build [--out PATH] [hipcc flags ...]
    argv = sys.argv[1:]
    out = LIB
    if argv[:1] == ["--out"]:
        out, argv = os.path.abspath(argv[1]), argv[2:]
    print(build(verbose=True, extra=argv, lib=out))
