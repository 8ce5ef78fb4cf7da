"""How many work items the library's launches have, at sizes around and beyond the 2^32
that a launch can have (the runtime launches more of them modulo 2^32, without an
error, which leaves the end of the result unwritten).  A child process loads the library
over a stand-in for the runtime's launch, so nothing runs and no GPU is needed: the
addresses are made up, far apart."""
import json
import os
import subprocess
import sys

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
SIZE = -5
ITEMS = 1 << 32

CHILD = r"""
import ctypes, json, sys
launches = ctypes.CDLL(sys.argv[1], mode=ctypes.RTLD_GLOBAL)
L = ctypes.CDLL(sys.argv[2])
out = []
buf = (ctypes.c_uint64 * (6 * 4096))()
for name, types, args in json.load(sys.stdin):
    fn = getattr(L, name)
    fn.argtypes = [getattr(ctypes, t) for t in types]
    rc = fn(*args)
    n = launches.take_launches(buf, 4096)
    out.append([rc, [list(buf[6 * i:6 * i + 6]) for i in range(n)]])
print(json.dumps(out))
"""
P, I, Q, F = "c_void_p", "c_int", "c_int64", "c_float"
TYPES = {
    "zq_embedding": [P, I, Q, P, I, Q, Q, F, P, I, P],
    "qwz_embedding": [P, I, Q, P, P, Q, Q, I, F, P, I, P],
    "zq_embedding_grad": [P, I, Q, P, I, Q, Q, F, I, P, I, P, Q, P],
    "zq_int4_dequant_gemm": [P, I, P, P, Q, Q, Q, I, P, P, Q, P],
    "qwz_quantize": [P, I, Q, I, P, P, P],
    "qwz_dequantize": [P, P, Q, I, P, I, P],
    "qgz_quantize": [P, I, Q, I, P, P, P],
    "qgz_dequantize": [P, P, Q, I, P, I, P],
    "qgz_reduce_level": [P, P, I, Q, I, P, P, P],
    "qgz_reduce_dequantize": [P, P, I, Q, I, P, I, P, P, P],
    "qwz_dequant_gemm": [P, I, P, P, Q, Q, Q, I, P, P],
}
# made-up addresses
A, B, C, SC, WS = (k << 52 for k in range(1, 6))


@pytest.fixture(scope="module")
def run(tmp_path_factory):
    from paper_2501_04266_amd import _lib
    if not os.path.exists(_lib.LIB_PATH):
        from paper_2501_04266_amd import build
        build.build()
    so = str(tmp_path_factory.mktemp("launches") / "launches.so")
    subprocess.run(["g++", "-std=c++17", "-O2", "-Wall", "-Wextra", "-Werror", "-shared", "-fPIC",
                    os.path.join(HERE, "c", "launches.cpp"), "-o", so], check=True)

    def ask(calls, child=CHILD, *more):
        if child is not CHILD:
            r = subprocess.run([sys.executable, "-c", child, so, _lib.LIB_PATH, *more], capture_output=True, text=True)
            assert r.returncode == 0, r.stderr
            return json.loads(r.stdout)
        text = json.dumps([[name, TYPES.get(name) or types, args] for name, types, args in calls])
        r = subprocess.run([sys.executable, "-c", CHILD, so, _lib.LIB_PATH], input=text, capture_output=True, text=True)
        assert r.returncode == 0, r.stderr
        return json.loads(r.stdout)
    return ask


def one(run, name, *args):
    return run([(name, None, list(args))])[0]


def check(rc, launches, groups, threads):
    """Launches of one kernel after another, each with its number of workgroups in all."""
    assert rc == 0
    at = 0
    for want in groups:
        done = 0
        while done < want:
            kernel, x, y, z, block, first = launches[at]
            assert x * block < ITEMS and block == threads and (y, z) == (1, 1)
            if want * threads >= ITEMS:
                assert first == done
            done += x
            at += 1
        assert done == want
    assert at == len(launches)


@pytest.mark.parametrize("T,D", [(1000, 64), ((ITEMS - 256) // 7, 7), (ITEMS // 7, 7), (ITEMS // 7 + 1000, 7),
                                 (3 << 30, 8), (3 << 31, 24), (1 << 35, 64)])
def test_lookup(run, T, D):
    pieces = T * (D if D < 8 else D // 8)
    check(*one(run, "zq_embedding", A, 4, T, B, 2, 1000, D, 1.0, C, 2, None), [-(-pieces // 256)], 256)
    check(*one(run, "qwz_embedding", A, 4, T, B, SC, 1000, D, 256, 1.0, C, 2, None), [-(-pieces // 256)], 256)


@pytest.mark.parametrize("T,V,D", [(600, 1 << 26, 1), (600, (1 << 26) - 4, 1), (600, 70_000_000, 1), (600, 70_000_000, 64),
                                   (600, 3_000_000, 6144), (1 << 20, 3_000_000, 6144), (600, 1 << 30, 1),
                                   (40, 1 << 30, 8), (1 << 20, 4, 1 << 24)])
def test_gradient(run, T, V, D):
    per = -(-(D if D < 8 else -(-D // 4)) // 64)
    segs = -(-T // 64) if T >= 64 else 0
    rc, launches = one(run, "zq_embedding_grad", A, 4, T, B, 2, V, D, 1.0, 0, C, 0, WS, 1 << 51, None)
    assert rc == 0
    sort, rest = launches[0], launches[1:]
    assert sort[1] * sort[4] < ITEMS and sort[4] == 1024
    seg_groups = -(-segs * per // 4)
    check(rc, rest, [-(-V * per // 4) + seg_groups] + ([seg_groups] if segs else []), 256)


def test_more_workgroups_than_a_call_numbers(run):
    """Refused before anything is launched."""
    assert one(run, "zq_embedding", A, 4, 1 << 40, B, 2, 1000, 8, 1.0, C, 2, None) == [SIZE, []]
    assert one(run, "zq_embedding_grad", A, 4, 600, B, 2, 1 << 30, 1 << 20, 1.0, 0, C, 0, WS, 1 << 51, None) == [SIZE, []]


CLIP = r"""
import ctypes, json, sys
launches = ctypes.CDLL(sys.argv[1], mode=ctypes.RTLD_GLOBAL)
L = ctypes.CDLL(sys.argv[2])
class Grad(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("scales", ctypes.c_void_p), ("out", ctypes.c_void_p), ("n", ctypes.c_int64),
                ("dtype", ctypes.c_int32), ("out_dtype", ctypes.c_int32), ("block", ctypes.c_int32), ("r", ctypes.c_int32)]
class Plan(ctypes.Structure):
    _fields_ = [("bytes", ctypes.c_int64), ("norm", ctypes.c_int64), ("clip", ctypes.c_int64), ("count", ctypes.c_int32),
                ("r", ctypes.c_int32)]
g, p = (Grad * 1)(Grad(1 << 50, 0, 0, int(sys.argv[3]), 2, 0, 0, 0)), Plan()
assert L.zq_grad_plan_make(g, 1, ctypes.byref(p)) == 0
F, P = ctypes.c_float, ctypes.c_void_p
out = [p.clip]
buf = (ctypes.c_uint64 * (6 * 64))()
for rc in (lambda: L.zq_grad_norm(ctypes.byref(p), P(1 << 52), F(1), P(1 << 53), None),
           lambda: L.zq_grad_clip(ctypes.byref(p), P(1 << 52), P(1 << 53), F(1), F(1), None)):
    rc = rc()
    n = launches.take_launches(buf, 64)
    out.append([rc, [list(buf[6 * i:6 * i + 6]) for i in range(n)]])
print(json.dumps(out))
"""


@pytest.mark.parametrize("n", [5000, ((1 << 24) - 1) * 4096, (1 << 24) * 4096, (1 << 26) * 4096 + 3])
def test_norm_and_clip(run, n):
    pieces, norm, clip = run([], CLIP, str(n))
    assert pieces == -(-n // 4096)
    assert norm[0] == 0 and all(x * b < ITEMS for _, x, _, _, b, _ in norm[1])
    check(*clip, [pieces], 256)


# more than 16 rows: where a tile a wave would need 2^32 items; up to 4: the join of slices
@pytest.mark.parametrize("M,N,K", [(64, (1 << 30) - 1024, 64), (64, (1 << 30) + 16, 64), (20, 3 << 30, 128), (4, 1 << 28, 65536),
                                   (4, 1 << 30, 65536), (16, 1 << 29, 1 << 17), (1, 1 << 32, 64)])
def test_int4_product(run, M, N, K):
    rc, launches = one(run, "zq_int4_dequant_gemm", A, 2, B, C, M, N, K, 128, SC, WS, 1 << 51, None)
    assert rc == 0 and 1 <= len(launches)
    kernel, x, y, z, block, first = launches[0]
    assert block == 512 and x * block < ITEMS
    check(rc, launches[1:], [-(-M * N // 256)] if z > 1 else [], 256)


PATH = [
    ("qwz_quantize", lambda n: (A, 0, n, 32, B, C, None)), ("qwz_quantize", lambda n: (A, 2, n, 1024, B, C, None)),
    ("qgz_quantize", lambda n: (A, 0, n, 32, B, C, None)), ("qgz_quantize", lambda n: (A, 1, n, 1024, B, C, None)),
    ("qwz_dequantize", lambda n: (A, B, n, 256, C, 0, None)), ("qwz_dequantize", lambda n: (A, B, n, 256, C, 2, None)),
    ("qgz_dequantize", lambda n: (A, B, n, 256, C, 0, None)), ("qgz_dequantize", lambda n: (A, B, n, 256, C, 2, None)),
    ("qgz_reduce_level", lambda n: (A, B, 2, n, 128, C, SC, None)), ("qgz_reduce_level", lambda n: (A, B, 48, n, 32, C, SC, None)),
    ("qgz_reduce_dequantize", lambda n: (A, B, 3, n, 1024, C, 0, None, None, None)),
]


@pytest.mark.parametrize("k", range(len(PATH)))
def test_path_calls(run, k):
    """Whole, in one launch that has room for it, or refused with nothing launched."""
    name, args = PATH[k]
    sizes = [1 << e for e in range(20, 43)] + [(1 << e) + 33 for e in range(30, 43)]
    got = run([(name, None, list(args(n))) for n in sizes])
    refused = []
    for n, (rc, launches) in zip(sizes, got):
        if rc == SIZE:
            assert launches == [], n
            refused.append(n)
        else:
            assert rc == 0 and len(launches) == 1 and launches[0][1] * launches[0][4] < ITEMS, n
    assert refused and min(refused) > 1 << 33, "a size that memory holds many times is refused"
    assert all(n in refused for n in sizes if n >= min(refused))
