"""The interpreter's own entry to the 8-bit calls: same status as through ctypes, the same refusals, and ctypes in its place."""
import ctypes
import os

import numpy as np
import pytest


@pytest.fixture(scope="module")
def B():
    from paper_2601_22347_b200 import binding, build
    build.build()
    binding._lib = None                          # (another test may have loaded it without the entry)
    binding.load()
    if not os.path.exists(build.CALL_PATH):
        pytest.skip("no interpreter headers")
    return binding


ROWS = [16, None, 4, 2048, 16, 16, 16, 0]
DENSE = [16, 16, 5, 16, 16, 5, None, 4, 128, 256, 16, 0, None, 0, None]
GROUPED = [16, 16, 5, 16, 16, 5, None, 16, 4, 8, 128, 256, 16, 0, None, 0, None]


def changed(args, at, value):
    return args[:at] + [value] + args[at + 1:]


# (all of these are decided before anything is launched: one change each, in every place of the arguments)
@pytest.mark.parametrize("at,value", [(0, None), (0, 8), (0, 2 ** 64 - 8), (1, 8), (2, -1), (2, -2 ** 40), (3, 40), (3, 2 ** 32 + 2048), (4, 24), (4, 8), (4, 2 ** 32 + 17), (5, None),
                                      (5, 24), (6, None), (6, 8)])
def test_rows(B, at, value):
    args = changed(ROWS, at, value)
    if (at, value) == (3, 2 ** 32 + 2048):
        args[2] = 0                              # (cut to 2048, as ctypes does, and no rows)
    assert B._rotate_quantize_i8(*args) == B._lib.perq_rotate_quantize_i8(*args)


@pytest.mark.parametrize("at,value", [(0, None), (0, 8), (1, 8), (2, 2), (2, 2 ** 32 + 1), (3, None), (3, 8), (4, 2 ** 64 - 8), (5, 4), (5, -1), (7, -1), (7, 2 ** 31), (8, 0),
                                      (8, 2 ** 20 + 1), (9, 48), (10, None), (10, 8), (11, 3), (12, 8)])
def test_products(B, at, value):
    assert B._matmul_i8(*changed(DENSE, at, value)) == B._lib.perq_matmul_i8(*changed(DENSE, at, value)) != 0
    to = at + (at >= 7) + (at >= 8)
    args = changed(GROUPED, to, value)
    assert B._grouped_matmul_i8(*args) == B._lib.perq_grouped_matmul_i8(*args) != 0


@pytest.mark.parametrize("at,value", [(7, None), (7, 8), (9, 0), (9, 1025), (9, -1)])
def test_experts(B, at, value):
    assert B._grouped_matmul_i8(*changed(GROUPED, at, value)) == B._lib.perq_grouped_matmul_i8(*changed(GROUPED, at, value)) != 0


def test_no_rows(B):
    assert B._rotate_quantize_i8(*changed(ROWS, 2, 0)) == B._matmul_i8(*changed(DENSE, 7, 0)) == B._grouped_matmul_i8(*changed(GROUPED, 8, 0)) == 0


@pytest.mark.parametrize("bad", [1.5, "16", None, np.float32(16), ctypes.c_int(16)])
def test_refusals(B, bad):
    for call, args, at in ((B._rotate_quantize_i8, ROWS, 4), (B._matmul_i8, DENSE, 8), (B._matmul_i8, DENSE, 13), (B._grouped_matmul_i8, GROUPED, 9), (B._grouped_matmul_i8, GROUPED, 15)):
        with pytest.raises(TypeError):
            call(*changed(args, at, bad))
    for call, args in ((B._rotate_quantize_i8, ROWS), (B._matmul_i8, DENSE), (B._grouped_matmul_i8, GROUPED)):
        with pytest.raises(TypeError):
            call(*args[:-1])
        with pytest.raises(TypeError):
            call(*args, 0)


def test_without_the_entry_ctypes_takes_the_calls(B, monkeypatch, tmp_path):
    from paper_2601_22347_b200 import build
    for name in ("_lib", "_rotate_quantize", "_swiglu_rotate_quantize", "_rotate_quantize_i8", "_matmul_i8", "_grouped_matmul_i8"):
        monkeypatch.setattr(B, name, None)
    monkeypatch.setattr(build, "CALL_PATH", str(tmp_path / "_perq_call.so"))
    lib = B.load()
    assert B._rotate_quantize_i8 is lib.perq_rotate_quantize_i8 and B._matmul_i8 is lib.perq_matmul_i8 and B._grouped_matmul_i8 is lib.perq_grouped_matmul_i8
    assert B._matmul_i8(*changed(DENSE, 0, None)) == 1       # PERQ_ERR_NULL
