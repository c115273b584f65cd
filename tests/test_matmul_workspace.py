"""Workspaces of the products: one for T tokens serves every call with fewer.  No call is launched: a workspace that is large enough and not aligned is
refused for that, and for its size before that."""
import ctypes as C
import random

import pytest

ALIGN, WORKSPACE = 6, 9
P = C.c_void_p(0x1000)
ODD = C.c_void_p(0x1008)
INT4, ASYM, INT8 = 0, 4, 5
FORMATS = [(INT4, INT4), (ASYM, INT4), (INT8, INT4), (INT4, INT8), (ASYM, INT8), (INT8, INT8)]


@pytest.fixture(scope="module")
def lib():
    from paper_2601_22347_b200 import binding, build
    build.build()
    return binding.load()


def dense_bytes(lib, T, N, d, af, wf):
    n = C.c_size_t(0)
    assert lib.perq_matmul_i8_workspace_bytes(T, N, d, af, wf, C.byref(n)) == 0
    return n.value


def dense(lib, T, N, d, af, wf, have):
    return lib.perq_matmul_i8(P, P, af, P, P, wf, P, T, N, d, P, 0, ODD, have, None)


def grouped_bytes(lib, T, E, N, d, af, wf):
    n = C.c_size_t(0)
    assert lib.perq_grouped_matmul_i8_workspace_bytes(T, E, N, d, af, wf, C.byref(n)) == 0
    return n.value


def grouped(lib, T, E, N, d, af, wf, have):
    return lib.perq_grouped_matmul_i8(P, P, af, P, P, wf, P, P, T, E, N, d, P, 0, ODD, have, None)


SHAPES = [(4096, 4096), (1024, 4096), (8192, 2048), (257, 9728), (14336, 4096), (100, 32), (1000, 32768), (2048, 14336)]


@pytest.mark.parametrize("af,wf", FORMATS)
@pytest.mark.parametrize("N,d", SHAPES)
def test_a_workspace_serves_every_smaller_call(lib, af, wf, N, d):
    """At both sides of every tile's border, and between; the sizes of larger calls are no smaller."""
    rng = random.Random(N + d + 10 * af + wf)
    tokens = sorted({1, 2, 64, 65, 66} | {128 * k + i for k in range(1, 60) for i in (-1, 0, 1, 2)} | {rng.randint(1, 20000) for _ in range(200)})
    sizes = [dense_bytes(lib, T, N, d, af, wf) for T in tokens]
    assert sizes == sorted(sizes)
    if (af, wf) == (INT8, INT8):
        assert sizes[-1] == 0
    for i, T in enumerate(tokens):
        for j in {i, min(i + 1, len(tokens) - 1), rng.randrange(i, len(tokens)), len(tokens) - 1}:
            assert dense(lib, T, N, d, af, wf, sizes[j]) == ALIGN, "%d of %d tokens" % (T, tokens[j])


def test_sizes_of_this_kind(lib):
    """(1024 tokens want 20 MB and 1025 .. 1152 want none, by the times of both kernels; a caller with one buffer for 1152 has room for all.)"""
    for T in (1024, 1025, 1100, 1152):
        assert dense(lib, T, 4096, 4096, INT4, INT4, dense_bytes(lib, 1152, 4096, 4096, INT4, INT4)) == ALIGN
    assert dense(lib, 4608, 1024, 4096, INT8, INT4, dense_bytes(lib, 4609, 1024, 4096, INT8, INT4)) == ALIGN


def test_too_small_is_still_refused(lib):
    n = dense_bytes(lib, 8000, 2064, 160, INT4, INT4)
    assert n > 0 and dense(lib, 8000, 2064, 160, INT4, INT4, n) == ALIGN and dense(lib, 8000, 2064, 160, INT4, INT4, n - 1) == WORKSPACE


@pytest.mark.parametrize("af,wf", FORMATS)
def test_grouped_calls(lib, af, wf):
    for E, N, d in ((1, 260, 544), (8, 4096, 2048), (60, 100, 96)):
        tokens = sorted({1, 63, 64, 65} | {E * k + i for k in (64, 96, 768) for i in (-1, 0, 1)} | {5000, 60000})
        sizes = [grouped_bytes(lib, T, E, N, d, af, wf) for T in tokens]
        assert sizes == sorted(sizes)
        for i, T in enumerate(tokens):
            for have in sizes[i:]:
                assert grouped(lib, T, E, N, d, af, wf, have) == ALIGN


def test_the_largest_question_is_answered(lib):
    """2^30 tokens, where the search for a smaller call that wants one has the most to look at."""
    assert dense_bytes(lib, 2 ** 30, 1, 32, INT4, INT4) >= 0
    assert dense_bytes(lib, 2 ** 30, 4096, 4096, INT4, INT4) >= 2 ** 42
