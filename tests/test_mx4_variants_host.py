"""The sizes of tests/mx4_variants.py reach every variant that the choice of kernel can take, and the query's refusals, on the CPU."""
import ctypes
import random

import pytest

import mx4_variants as v
from paper_2405_01943_b200 import binding as b
from paper_2405_01943_b200 import build

OK, NULL, SHAPE, UNSUPPORTED = 0, 1, 2, 5


@pytest.fixture(scope="module")
def lib():
    build.build()
    return b.load()


def test_every_variant_that_sizes_reach_is_among_the_cases(lib):
    """The kernel is chosen by a time model: a change of its constants may reach variants that no case compares."""
    compared = {v.variant(*size, both4, glu) for both4, glu, *size in v.CASES}
    rng = random.Random(20)
    log = lambda lo, hi: round(lo * (hi / lo) ** rng.random())                                                     # noqa: E731
    missing = {}
    for _ in range(60000):
        groups = 0 if rng.random() < 0.5 else log(1, 64)
        size = (log(1, 8192 if groups else 4096), log(8, 16384), log(8, 32768), groups)
        form = (rng.random() < 0.5, rng.random() < 0.5)
        key = v.variant(*size, *form)
        if key not in compared:
            missing[key] = size
    assert not missing, missing


def test_the_kernel_of_a_call(lib):
    plan = (ctypes.c_int32 * 5)()
    f = lambda T=5, K=4096, N=14336, G=1, off=0, up=1, x4=0, out=plan: lib.dass_linear_mx4_plan(T, K, N, G, off, up, x4, out)          # noqa: E731
    assert f(out=None) == NULL
    assert f(T=0) == SHAPE and f(K=0) == SHAPE and f(N=0) == SHAPE and f(G=0) == SHAPE and f(G=2) == SHAPE
    assert f(T=1 << 29) == UNSUPPORTED and f(off=1, G=1025) == UNSUPPORTED and f(K=1 << 31) == UNSUPPORTED
    assert f() == OK and plan[0] == 1                                  # rows that are split: the one kernel with a workspace
    for both4, glu, T, K, N, groups in v.CASES:
        kernel, tile, sixteens, split, warps = v.plan(T, K, N, groups, both4, glu)
        assert (b.linear_mx4_workspace_bytes(T, K, N, groups or 1, groups > 0, glu, both4) > 0) == (kernel == 1 and not both4)
        if kernel == 0:
            assert tile in (1, 2, 4) and sixteens in (1, 2) and split in (1, 2, 4, 8) and warps in (8, 16)
        else:
            assert (sixteens, split, warps) == (0, 0, 0)
            assert tile in {1: (32, 64, 128) if both4 else (4, 8, 10), 2: (128, 256), 3: (64, 128, 256)}[kernel]
            assert both4 if kernel == 2 else kernel != 3 or not both4
