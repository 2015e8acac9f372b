"""How the gated feed-forward block's products are laid out (csrc/gdr2_gatedff_plan.hpp), on the CPU.

The header is host arithmetic alone; it is compiled here as it is, behind one function."""

import ctypes
import os
import random
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CXX = shutil.which("g++") or shutil.which("c++")

pytestmark = pytest.mark.skipif(CXX is None, reason="no host compiler")

STORE, GATE, GRAD = 0, 1, 2
SHIM = """
#include "gdr2_gatedff_plan.hpp"
extern "C" void plan(int end, const int64_t* z, int pairs, int E, int64_t* out) {
  const gdr2::FfPlan q = gdr2::ff_choose(end, {{z[0], z[1]}, {z[2], z[3]}, z[4], pairs}, E);
  const int64_t left = q.tiles - q.full;
  const int64_t all[] = {q.bm, q.bn, q.tiles, q.full, q.split, (q.full + left * q.split) * gdr2::ff_threads(q.bm)};
  for (int i = 0; i < 6; ++i) out[i] = all[i];
}
extern "C" int thin(int64_t M, int64_t N, int64_t K, int E) { return gdr2::ff_thin_rows(M, N, K, E); }
"""


@pytest.fixture(scope="module")
def shim(tmp_path_factory):
    at = tmp_path_factory.mktemp("plan")
    (at / "shim.cpp").write_text(SHIM)
    subprocess.run([CXX, "-std=c++17", "-O1", "-fPIC", "-shared", "-I", os.path.join(ROOT, "paper_2605_22791_amd", "csrc"),
                    str(at / "shim.cpp"), "-o", str(at / "shim.so")], check=True)
    return ctypes.CDLL(str(at / "shim.so"))


def products(rows, D, F):
    """name -> (end, M of one or two products, N of them, K, pairs)"""
    return {"gate": (GATE, (rows, 0), (F, 0), D, 1), "down": (STORE, (rows, 0), (D, 0), F, 1),
            "grad": (GRAD, (rows, 0), (F, 0), D, 1), "dx": (STORE, (rows, 0), (D, 0), F, 2),
            "dw": (STORE, (2 * F, D), (D, F), rows, 1)}


def plan(shim, product, E):
    """(tile, its columns, tiles, whole ones, parts of the others, threads)"""
    end, M, N, K, pairs = product
    out = (ctypes.c_int64 * 6)()
    shim.plan(end, (ctypes.c_int64 * 5)(*M, *N, K), pairs, E, out)
    return tuple(out)


def test_every_launch_of_the_documented_range_has_less_than_2_32_threads(shim):
    """rows up to 2^24, D and F multiples of 8 up to 65536, rows D and rows F below 2^36."""
    r = random.Random(1)
    sizes = [(1 << 24, 8, 2056), (1 << 24, 2056, 8), (1 << 24, 4088, 4088), ((1 << 20) - 1, 65536, 65536), (1, 65536, 65536),
             ((1 << 24) - 77, 8, 2104), (1 << 24, 4088, 2056), (9000001, 7632, 7624), (0, 65536, 65536)]
    while len(sizes) < 20000:
        rows, D, F = (1 << 24) - r.randrange(1 << r.randrange(1, 24)), 8 * r.randint(1, 8192), 8 * r.randint(1, 8192)
        most = (1 << 36) - 1
        sizes.append((rows, max(8, min(D, most // rows // 8 * 8)), max(8, min(F, most // rows // 8 * 8))))
    for rows, D, F in sizes:
        assert rows * D < 1 << 36 and rows * F < 1 << 36
        for name, p in products(rows, D, F).items():
            for E in (2, 4):
                threads = plan(shim, p, E)[-1]
                assert threads < 1 << 32, (rows, D, F, name, E, threads)


def _combinations(shim, rows, D, F, E):
    """The forms of the product kernel that a problem runs: (bytes of a value, product, tile, whole or cut)"""
    out = set()
    for name, p in products(rows, D, F).items():
        tile, _, tiles, whole, _, _ = plan(shim, p, E)
        out |= {(E, name, tile, "whole")} if whole else set()
        out |= {(E, name, tile, "cut")} if whole < tiles else set()
    return out


def test_the_gpu_tests_have_every_tile_that_is_chosen(shim):
    from tests.test_gpu_gatedff_sizes import SHAPES
    r = random.Random(2)
    spread = lambda lo, hi: int(lo * (hi / lo) ** r.random())  # noqa: E731
    found = {E: set() for E in (2, 4)}
    for _ in range(60000):
        rows, D, F = spread(1, 1 << 18), spread(1, 8192) * 8, spread(1, 8192) * 8
        if rows * max(D, F) < 1 << 36:
            E = r.choice((2, 4))
            found[E] |= _combinations(shim, rows, D, F, E)
    for dtype, E in (("bf16", 2), ("fp32", 4)):
        tested = set().union(*(_combinations(shim, rows, D, F, E) for rows, D, F, t, _ in SHAPES if t == dtype))
        assert not found[E] - tested, found[E] - tested
    assert len(found[2]) == 30 and len(found[4]) == 20  # five products, three tiles or two, whole and cut
