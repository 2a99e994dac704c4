"""Which kernel a product of 8-bit rows runs on: the planner's header compiled for the host (no GPU needed).  Tiles differ in code, so the GPU tests' sizes have to
reach all of them with every epilogue."""
import ctypes
import itertools
import os
import subprocess

import pytest

from paper_2510_15620_amd import binding as B
from tests import test_gpu_q8 as G

HEADER = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2510_15620_amd", "csrc", "gemm_q8_plan.h")
SOURCE = """
#include "%s"
using namespace prism;
extern "C" int tiles() { return kQ8Tiles; }
extern "C" void plan(int M, int cols, int slices, int epi, int *out) {
  const Q8Plan p = q8_plan(M, cols, slices, (Q8Epilogue)epi);
  out[0] = p.rows_first; out[1] = p.first; out[2] = p.kind; out[3] = kQ8Tile[p.first].bm; out[4] = kQ8Tile[p.kind].bn;
}
extern "C" int few(int M, int N, int K) { return q8_few_rows(M, N, K); }
extern "C" int turn(int M, long long stride) { return q8_turn(M, stride); }
extern "C" int columns(int kind, int glu) { return glu ? kQ8Tile[kind].bn / 2 : kQ8Tile[kind].bn; }
"""


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    d = tmp_path_factory.mktemp("q8")
    (d / "plan.cpp").write_text(SOURCE % HEADER)
    subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-o", str(d / "plan.so"), str(d / "plan.cpp")], check=True)
    return ctypes.CDLL(str(d / "plan.so"))


def kinds(lib, M, N, K, epilogue):
    """Tiles of a launch; none where the kernel of few rows takes it."""
    if lib.few(M, N, K):
        return []
    out = (ctypes.c_int * 5)()
    glu = epilogue == B.EPI_SWIGLU
    lib.plan(M, N // 2 if glu else N, -(-K // 128), 2 if glu else 1 if epilogue == B.EPI_RESIDUAL else 0, out)
    assert 0 <= out[0] < M and out[0] % out[3] == 0 and not (glu and out[4] == 32)
    return ([out[1]] if out[0] else []) + [out[2]]


def test_the_gpu_tests_reach_every_tile(plan):
    for epilogue, _ in G.EPILOGUES:
        seen = set(itertools.chain(*(kinds(plan, *size, epilogue) for size in G.SIZES)))
        ragged = set(itertools.chain(*(kinds(plan, M, N * (2 if epilogue == B.EPI_SWIGLU else 1), K, epilogue) for M, N, K in G.ODD_SIZES)))
        want = set(range(plan.tiles())) - ({11, 12} if epilogue == B.EPI_SWIGLU else set())
        assert seen | ragged == want, (epilogue, want - seen - ragged)


def test_the_gpu_tests_turn_every_tile(plan):
    """Loops that begin elsewhere than at K's start, at different places in the tiles of a launch."""
    for epilogue, _ in G.EPILOGUES:
        glu, seen = epilogue == B.EPI_SWIGLU, set()
        for M, N, K in G.TURN_SIZES:
            turn, slices = plan.turn(M, ctypes.c_longlong(-(-K // 4096) * 4096)), -(-K // 128)
            assert turn and not plan.turn(M, ctypes.c_longlong(-(-K // 4096) * 4096 + 128))
            for kind in kinds(plan, M, N, K, epilogue):
                tiles = -(-(N // 2 if glu else N) // plan.columns(kind, glu))
                if len({i * turn % slices for i in range(tiles)}) >= min(slices, 3):
                    seen.add(kind)
        assert seen == set(range(plan.tiles())) - ({11, 12} if glu else set()), (epilogue, seen)


def test_plans_of_all_sizes_are_possible(plan):
    for M, N, K in itertools.product((17, 65, 300, 1000, 4097, 20000, 1048576), (2, 130, 1026, 24576, 300000), (1, 129, 4096, 131071)):
        for epilogue in (B.EPI_STORE, B.EPI_RESIDUAL, B.EPI_SWIGLU):
            kinds(plan, M, N, K, epilogue)


def test_generated_loops_are_in_sync_with_their_generator():
    import sys
    csrc = os.path.dirname(HEADER)
    out = subprocess.run([sys.executable, os.path.join(csrc, "gen_gemm_kloop.py"), "q8"], capture_output=True, text=True, check=True).stdout
    assert out == open(os.path.join(csrc, "gemm_q8_kloop.inc")).read()
