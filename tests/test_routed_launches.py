"""The launches of the operators round the grouped products, written down on the CPU instead of made: LDS that is asked for.

The host side of csrc/pcc_routed.hip is compiled alone and linked with tests/host_checks/recorded_launches.cpp in the place of
HIP's runtime, so nothing here can reach a GPU; the kernels' static LDS is what the compiler says of them.
"""
import ctypes as C
import functools
import os
import subprocess
import tempfile

import pytest

import test_kernel_hazards as hazards
import test_routed_kernel_hazards as routed
from paper_2212_01185_amd import build as pcc_build

HERE = os.path.dirname(os.path.abspath(__file__))
PLAIN_LIMIT, CARD_LIMIT = 64 * 1024, 160 * 1024
# stand for device pointers, far from each other
A, B, D, E, F, G, H, I = (0x100000000000 * i for i in range(1, 9))


@functools.lru_cache(maxsize=None)
def _library():
    with tempfile.TemporaryDirectory() as d:
        objects = [os.path.join(d, "host.o"), os.path.join(d, "runtime.o")]
        flags = [f for f in pcc_build.FLAGS if f != "-shared"]
        for cmd in ([pcc_build.HIPCC] + flags + ["--cuda-host-only", "-fuse-cuid=none", "-c", "-o", objects[0], pcc_build.ROUTED_SRC],
                    ["g++", "-std=c++17", "-O2", "-fPIC", "-c", "-o", objects[1], os.path.join(HERE, "host_checks", "recorded_launches.cpp")]):
            subprocess.run(cmd, check=True, stdout=subprocess.PIPE, stderr=subprocess.STDOUT)
        lib = os.path.join(d, "launches.so")
        subprocess.run(["g++", "-shared", "-Wl,-Bsymbolic", "-Wl,-z,defs", "-o", lib] + objects, check=True, stdout=subprocess.PIPE, stderr=subprocess.STDOUT)
        # symbols of its own before any others of the process
        L = C.CDLL(lib, mode=os.RTLD_LOCAL | os.RTLD_NOW | os.RTLD_DEEPBIND)
    L.recorded.restype = C.c_char_p
    return L


@functools.lru_cache(maxsize=None)
def _static():
    return hazards.static_lds(routed._assembly())


def _launches():
    """(kernel, dynamic LDS, limit asked for, workgroups, threads) of the launches since the last call."""
    return [(w[0],) + tuple(int(v) for v in w[1:]) for w in (line.split() for line in _library().recorded().decode().splitlines())]


def _check(what):
    found = _launches()
    assert found, what
    for name, dynamic, limit, _, _ in found:
        all_of_it = dynamic + _static()[name]
        assert all_of_it <= CARD_LIMIT, (what, name, all_of_it)
        assert dynamic == 0 or _static()[name] <= 1024      # what the library counts with
        assert all_of_it <= PLAIN_LIMIT or limit >= dynamic, (what, name, dynamic, _static()[name])


# every width round the borders of a row's shapes and of 64 KB of weights, and some between them
WIDTHS = sorted({w for c in (64, 200, 264, 520, 1032, 2056, 4096, 8192, 16384) for w in range(max(1, c - 24), c + 17)} | set(range(1, 17000, 331)) | {20000, 65536})


@hazards.needs_hipcc
@pytest.mark.parametrize("x_type,y_type", [(0, 0), (1, 1), (2, 2), (2, 0), (2, 1)])
def test_layer_norms_ask_for_the_lds_that_they_have(x_type, y_type):
    L, sz = _library(), C.c_size_t
    for f in WIDTHS:
        _launches()
        assert L.pcc_layer_norm(C.c_void_p(A), sz(f), C.c_void_p(B), C.c_void_p(D), C.c_void_p(E), 2, sz(300), f, C.c_float(1e-5), x_type, C.c_void_p(F), y_type, sz(f), C.c_void_p(G), None) == 0
        _check(("forward", f))
        assert L.pcc_layer_norm_grad(C.c_void_p(A), y_type, sz(f), C.c_void_p(B), sz(f), C.c_void_p(D), C.c_void_p(E), C.c_void_p(F), 2, sz(300), f, x_type, C.c_void_p(G), sz(f), C.c_void_p(H),
                                     C.c_void_p(H + (1 << 32)), C.c_void_p(I), sz(1 << 40), None) == 0
        _check(("backward", f))


@hazards.needs_hipcc
def test_sorts_ask_for_the_lds_that_they_have():
    L, sz = _library(), C.c_size_t
    for experts in range(1, 1025):
        for tokens in (100, 100000):
            _launches()
            assert L.pcc_expert_sort(C.c_void_p(A), sz(tokens), 2, experts, C.c_void_p(B), C.c_void_p(D), C.c_void_p(E), sz(1 << 40), None) == 0
            _check((experts, tokens))
