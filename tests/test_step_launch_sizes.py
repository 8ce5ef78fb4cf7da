"""How many work items the launches of the optimizer's step, the norm and the loss have at
their largest sizes (a launch of 2^32 and more runs their number modulo 2^32, without an
error).  A child process loads the library over a stand-in for the runtime's launch, so
nothing runs and no GPU is needed."""
import ctypes
import json
import os
import subprocess
import sys

import pytest

from paper_2501_04266_amd import _lib

HERE = os.path.dirname(os.path.abspath(__file__))
ITEMS = 1 << 32
CHILD = r"""
import ctypes, json, sys
launches = ctypes.CDLL(sys.argv[1], mode=ctypes.RTLD_GLOBAL)
L = ctypes.CDLL(sys.argv[2])
out = []
buf = (ctypes.c_uint64 * (6 * 8192))()
for name, types, args in json.load(sys.stdin):
    fn = getattr(L, name)
    fn.argtypes = [getattr(ctypes, t) for t in types]
    held = [ctypes.create_string_buffer(bytes.fromhex(a)) if isinstance(a, str) else a for a in args]
    rc = fn(*[ctypes.cast(a, ctypes.c_void_p) if isinstance(a, ctypes.Array) else a for a in held])
    n = launches.take_launches(buf, 8192)
    out.append([rc, [list(buf[6 * i:6 * i + 6]) for i in range(min(n, 8192))], n])
print(json.dumps(out))
"""
P, I, Q, D, F = "c_void_p", "c_int", "c_int64", "c_double", "c_float"
A, B, C, E, G, H, W = (k << 52 for k in range(1, 8))


@pytest.fixture(scope="module")
def run(tmp_path_factory):
    if not os.path.exists(_lib.LIB_PATH):
        from paper_2501_04266_amd import build
        build.build()
    so = str(tmp_path_factory.mktemp("launches") / "launches.so")
    subprocess.run(["g++", "-std=c++17", "-O2", "-Wall", "-Wextra", "-Werror", "-shared", "-fPIC",
                    os.path.join(HERE, "c", "launches.cpp"), "-o", so], check=True)

    def ask(name, types, *args):
        r = subprocess.run([sys.executable, "-c", CHILD, so, _lib.LIB_PATH], input=json.dumps([[name, types, list(args)]]),
                           capture_output=True, text=True)
        assert r.returncode == 0, r.stderr
        rc, launches, n = json.loads(r.stdout)[0]
        assert n == len(launches)
        return rc, launches
    return ask


def parts(launches, groups, threads):
    """The launches are one kernel's, one part after the other, `groups` workgroups in all."""
    done = 0
    for kernel, x, y, z, block, first in launches:
        assert kernel == launches[0][0] and y == z == 1 and block == threads and x * block < ITEMS and first == done
        done += x
    assert done == groups


RMS = [P, P, I, P, I, Q, Q, D, P, P, I, P, P]
GRAD = [P, I, P, I, P, I, P, P, Q, Q, P, I, P, I, P, Q, P]


@pytest.mark.parametrize("T,D,groups,threads", [((1 << 31) - 1, 128, 1 << 27, 256), ((1 << 31) - 1, 64, 1 << 27, 256),
                                                (1 << 30, 500, 1 << 28, 256), ((1 << 31) - 1, 2048, (1 << 31) - 1, 256),
                                                (1 << 27, 16384, 1 << 27, 1024), (1 << 24, 1 << 24, 1 << 24, 1024)])
def test_norm(run, T, D, groups, threads):
    rc, launches = run("zq_rms_norm", RMS, A, None, 2, None, 0, T, D, 1e-6, None, B, 2, None, None)
    assert rc == 0
    parts(launches, groups, threads)


@pytest.mark.parametrize("T,D", [((1 << 31) - 1, 64), ((1 << 31) - 1, 6144), (1 << 26, 16384)])
def test_gradient(run, T, D):
    need = _lib.lib().zq_rms_norm_grad_bytes(T, D)
    rc, launches = run("zq_rms_norm_grad", GRAD, A, 2, B, 2, None, 0, C, None, T, D, E, 0, G, 0, W, need, None)
    assert rc == 0 and len(launches) == 2 and all(x * block < ITEMS for _, x, _, _, block, _ in launches)


def test_gradient_of_long_rows(run):
    T, D = 1 << 23, 1 << 20
    need = _lib.lib().zq_rms_norm_grad_bytes(T, D)
    rc, launches = run("zq_rms_norm_grad", GRAD, A, 2, B, 2, None, 0, C, None, T, D, E, 0, G, 0, W, need, None)
    assert rc == 0
    kernels = list(dict.fromkeys(e[0] for e in launches))
    assert len(kernels) == 3
    parts([e for e in launches if e[0] == kernels[0]], T, 1024)
    parts([e for e in launches if e[0] == kernels[1]], need // (4 * D) * (D // 2048), 256)


@pytest.mark.parametrize("T,V,threads", [(1 << 30, 1000, 64), (1 << 30, 50000, 1024), (1 << 28, 1 << 24, 1024)])
def test_logp(run, T, V, threads):
    rc, launches = run("zq_token_logp", [P, I, Q, Q, Q, P, I, F, P, P], A, 2, T, V, V, B, 4, 1.0, C, None)
    assert rc == 0
    parts(launches, T, threads)


def test_step(run):
    pieces = (1 << 31) - 1
    plan = _lib._AdamWPlan(1 << 40, pieces, 0, 1, 0)
    args = _lib._AdamWArgs(1e-3, 0.9, 0.99, 1e-8, 1, 1.0, 1.0)
    text = [ctypes.string_at(ctypes.byref(s), ctypes.sizeof(s)).hex() for s in (plan, args)]
    rc, launches = run("zq_adamw_step", [P] * 7, text[0], A, text[1], None, None, None, None)
    assert rc == 0
    parts(launches, pieces, 256)
    # the count on the device: one more launch before
    rc, launches = run("zq_adamw_step", [P] * 7, text[0], A, text[1], B, None, None, None)
    assert rc == 0 and launches[0][4] == 64 and launches[0][0] != launches[1][0]
    parts(launches[1:], pieces, 256)
    # tensors of both kinds: a kernel each
    plan.block_pieces = 1 << 30
    text[0] = ctypes.string_at(ctypes.byref(plan), ctypes.sizeof(plan)).hex()
    rc, launches = run("zq_adamw_step", [P] * 7, text[0], A, text[1], None, None, None, None)
    kernels = list(dict.fromkeys(e[0] for e in launches))
    assert rc == 0 and len(kernels) == 2
    parts([e for e in launches if e[0] == kernels[0]], pieces, 256)
    parts([e for e in launches if e[0] == kernels[1]], 1 << 30, 256)
