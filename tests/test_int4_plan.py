"""The INT4 product's plan (csrc/zq_int4_plan.h, host arithmetic), compiled with the host
compiler and asked without a GPU: which kernel runs the shapes of the GPU tests, that
these name every kernel that the plan chooses at all, that no plan exceeds what its
kernels can hold, and that slices and tiles cover the product."""
import os
import random
import subprocess

import pytest

from tests.int4_routes import ROUTES

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(os.path.dirname(HERE), "paper_2501_04266_amd", "csrc")


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    exe = str(tmp_path_factory.mktemp("plan") / "int4_plan")
    subprocess.run(["g++", "-std=c++17", "-O2", "-Wall", "-Wextra", "-Werror", "-I", CSRC,
                    os.path.join(HERE, "c", "int4_plan.cpp"), "-o", exe], check=True)

    def ask(shapes):
        text = "".join(f"{M} {N} {K} {B}\n" for M, N, K, B in shapes)
        out = subprocess.run([exe], input=text, capture_output=True, text=True, check=True).stdout.splitlines()
        rows = [(f[0], *(int(v) for v in f[1:])) for f in (line.split() for line in out)]
        assert len(rows) == len(shapes)
        return rows
    return ask


def shapes(count, seed):
    rng = random.Random(seed)
    return [(int(2 ** rng.uniform(0, 9)), int(2 ** rng.uniform(0, 18)), 64 * int(2 ** rng.uniform(0, 14)),
             rng.choice([32, 64, 128, 256, 512, 1024])) for _ in range(count)]


def test_gpu_shapes_run_the_kernels_they_name(plan):
    got = plan([r[1:] for r in ROUTES])
    wrong = [(want, g[0], s) for (want, *s), g in zip(ROUTES, got) if want != g[0]]
    assert not wrong, wrong


def test_gpu_shapes_name_every_kernel(plan):
    named = {r[0] for r in ROUTES}
    for shape, p in zip(*(lambda s: (s, plan(s)))(shapes(200000, 3))):
        assert p[0] in named, (p[0], shape)


# hidden 2,048 and 6,144 layers and larger ones, 1 to 64 rows
LAYERS = [(M, N, K, 128) for M in (1, 5, 16, 17, 32, 48, 49, 64) for N, K in
          [(6144, 2048), (2048, 8192), (6144, 6144), (18432, 6144), (24576, 6144), (6144, 24576), (20000, 12288),
           (50001, 6144), (65536, 2048)]]


def test_layers_take_kernels_that_are_tested(plan):
    named = {r[0] for r in ROUTES}
    got = plan(LAYERS)
    assert {p[0] for p in got} <= named
    # 49 to 64 rows with K in slices, a tile a wave
    names = {s: p[0] for s, p in zip(LAYERS, got)}
    for N, K in ((6144, 6144), (18432, 6144), (6144, 24576), (20000, 12288)):
        assert names[64, N, K, 128] == "wide:4,G128,slices"


EDGES = [(M, N, 64 * k, 32) for M in (1, 2, 3, 4, 5, 16, 17, 32, 33, 48, 49, 64, 65, 64 * 65535) for N in (1, 16, 8192, 8193)
         for k in (0, 1, 1 << 10, (1 << 16) - 1, 1 << 16)]
EDGES += [(M, N, 64, 32) for M in (1, 5, 17, 64) for N in ((1 << 30) - 16, (1 << 30) - 15, (1 << 34) - 16)]


def test_plans_fit_their_kernels(plan):
    every = shapes(40000, 5) + LAYERS + EDGES
    for (M, N, K, B), (name, grid, mgroups, slices, each, groups, lds, ws, ok) in zip(every, plan(every)):
        what = (M, N, K, B, name, slices)
        tiles = -(-N // 16)
        assert ok, what
        assert each % 256 == 0 and each * slices >= K and (slices == 1 or each * (slices - 1) < K), what
        assert ws == (4 * M * N * slices if slices > 1 else 0) and ("slices" in name) == (slices > 1), what
        assert 0 < grid * 512 < 1 << 32 and 0 < mgroups <= 65535 and 0 < slices <= 65535 and groups < 1 << 31, what
        assert 0 <= lds <= 160 * 1024, what
        # byte offsets stay below the mark of a load outside
        assert 48 * K // 2 < 0x7fff0000 and 2 * 64 * K < 0x7fff0000, what
        kind = name.split(",")[0]
        if kind.startswith("few"):
            rows = int(kind[4:])
            assert M <= rows <= 4 and mgroups == 1 and groups == tiles and grid <= groups, what
            # x with one unit more a row, and two groups' sums of 8 waves
            assert lds >= M * (each // 8 + 1) * 16 + 2 * 8 * 4 * (4 * rows * 16), what
        elif kind == "lds":
            assert 4 < M <= 16 and mgroups == 1 and groups == tiles and grid <= groups, what
            assert lds >= M * (each // 8 + 1) * 16 + 2 * 8 * 4 * 16 * M, what
        elif kind.startswith("regs"):
            mt, gb = (int(v) for v in kind[5:].split("x"))
            assert mgroups * 16 * mt >= M and groups * gb >= tiles and grid <= groups, what
            assert lds >= 8 * 16 * 4 * min(M, 16 * mt) * gb, what
        else:
            mt = int(kind[5:])
            assert M > 16 and mgroups * 16 * mt >= M and grid * 8 >= tiles and groups == tiles and lds == 0, what


def test_codes_under_one_scale(plan):
    """128 at a time only where rows start at multiples of 128 and blocks have as many."""
    for K in range(64, 1025, 64):
        for B in (32, 64, 128, 256, 512, 1024):
            name = plan([(20, 100, K, B)])[0][0]
            G = int(name.split("G")[1].split(",")[0])
            assert all((r * K + k) // B == (r * K + min(k + G, K) - 1) // B for r in range(40) for k in range(0, K, G)), (K, B, G)
