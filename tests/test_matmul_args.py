"""Refusals of the products of codes: all of them come before the library touches the CUDA runtime, so they run without a GPU."""
import ctypes as C

import pytest

OK, NULL, SHAPE, FMT, ALIGN, WORKSPACE = 0, 1, 2, 5, 6, 9
P = C.c_void_p(0x1000)
ODD = C.c_void_p(0x1008)
DENSE = dict(a=P, sa=P, af=5, w=P, sw=P, wf=5, ws=None, T=4, N=128, d=256, out=P, ot=0, wk=None, wb=0)


@pytest.fixture(scope="module")
def lib():
    from paper_2601_22347_b200 import binding, build
    build.build()
    return binding.load()


def dense(lib, **change):
    v = dict(DENSE, **change)
    return lib.perq_matmul_i8(v["a"], v["sa"], v["af"], v["w"], v["sw"], v["wf"], v["ws"], v["T"], v["N"], v["d"], v["out"], v["ot"], v["wk"], v["wb"], None)


def grouped(lib, **change):
    v = dict(DENSE, off=P, E=4, **change)
    return lib.perq_grouped_matmul_i8(v["a"], v["sa"], v["af"], v["w"], v["sw"], v["wf"], v["ws"], v["off"], v["T"], v["E"], v["N"], v["d"], v["out"], v["ot"],
                                      v["wk"], v["wb"], None)


REFUSED = [(dict(T=-1), SHAPE), (dict(T=2 ** 30 + 1), SHAPE), (dict(N=0), SHAPE), (dict(N=2 ** 20 + 1), SHAPE), (dict(d=0), SHAPE), (dict(d=48), SHAPE),
           (dict(d=32768 + 32), SHAPE), (dict(af=1), FMT), (dict(af=2), FMT), (dict(af=3), FMT), (dict(af=9), FMT), (dict(wf=4), FMT), (dict(wf=1), FMT),
           (dict(ot=3), FMT), (dict(ot=-1), FMT), (dict(a=None), NULL), (dict(sa=None), NULL), (dict(w=None), NULL), (dict(sw=None), NULL),
           (dict(out=None), NULL), (dict(af=4), NULL), (dict(a=ODD), ALIGN), (dict(sa=ODD), ALIGN), (dict(w=ODD), ALIGN), (dict(sw=ODD), ALIGN),
           (dict(out=ODD), ALIGN), (dict(af=4, ws=ODD), ALIGN), (dict(wk=ODD), ALIGN)]


@pytest.mark.parametrize("call", [dense, grouped])
@pytest.mark.parametrize("change,status", REFUSED, ids=[",".join("%s=%s" % (k, getattr(v, "value", v)) for k, v in c.items()) for c, _ in REFUSED])
def test_refused(lib, call, change, status):
    assert call(lib, **change) == status


@pytest.mark.parametrize("call", [dense, grouped])
def test_no_rows(lib, call):
    """Nothing to read or write: pointers may be anything, sizes are still looked at."""
    assert call(lib, T=0, a=None, sa=None, w=None, out=None) == OK
    assert call(lib, T=0, d=48) == SHAPE


def test_grouped_refused(lib):
    def call(**change):
        v = dict(DENSE, off=P, E=4)
        v.update(change)
        return lib.perq_grouped_matmul_i8(v["a"], v["sa"], v["af"], v["w"], v["sw"], v["wf"], v["ws"], v["off"], v["T"], v["E"], v["N"], v["d"], v["out"],
                                          v["ot"], v["wk"], v["wb"], None)
    assert call(off=None) == NULL
    assert call(off=ODD) == ALIGN
    assert call(E=0) == SHAPE
    assert call(E=1025) == SHAPE
    assert call(E=1024, N=2 ** 20 + 1) == SHAPE
    assert call(E=1024, N=2 ** 20, T=0) == OK
    assert call(E=4, T=0, off=None) == OK


def test_workspace_bytes(lib):
    n = C.c_size_t(1)
    assert lib.perq_matmul_i8_workspace_bytes(1, 4096, 4096, 0, 0, C.byref(n)) == OK and n.value == 0
    assert lib.perq_matmul_i8_workspace_bytes(1, 4096, 4096, 1, 0, C.byref(n)) == FMT
    assert lib.perq_matmul_i8_workspace_bytes(1, 4096, 4100, 0, 0, C.byref(n)) == SHAPE
    assert lib.perq_matmul_i8_workspace_bytes(1, 4096, 4096, 0, 0, None) == NULL
    assert lib.perq_grouped_matmul_i8_workspace_bytes(1, 8, 4096, 4096, 0, 0, C.byref(n)) == OK and n.value == 0
    assert lib.perq_grouped_matmul_i8_workspace_bytes(1, 0, 4096, 4096, 0, 0, C.byref(n)) == SHAPE
    assert lib.perq_grouped_matmul_i8_workspace_bytes(1, 8, 4096, 4096, 0, 0, None) == NULL


@pytest.mark.parametrize("change,status", [(dict(T=-1), SHAPE), (dict(d=40), SHAPE), (dict(d=0), SHAPE), (dict(d=65536), SHAPE), (dict(b=8), 3), (dict(b=24), 3),
                                           (dict(b=0), 3), (dict(d=96, b=64), 3), (dict(b=512, d=256), 3), (dict(b=1024), 10), (dict(b=4096), 10),
                                           (dict(x=None), NULL), (dict(oc=None), NULL), (dict(os=None), NULL), (dict(x=ODD), ALIGN), (dict(perm=ODD), ALIGN),
                                           (dict(oc=ODD), ALIGN), (dict(os=ODD), ALIGN), (dict(T=0, x=None), OK)])
def test_rows_to_8_bit_codes_refused(lib, change, status):
    v = dict(dict(x=P, perm=None, T=4, d=4096, b=32, oc=P, os=P), **change)
    assert lib.perq_rotate_quantize_i8(v["x"], v["perm"], v["T"], v["d"], v["b"], v["oc"], v["os"], None) == status


def test_code_sums_refused(lib):
    def call(codes=P, fmt=5, rows=4, d=256, sums=P):
        return lib.perq_code_sums(codes, fmt, rows, d, sums, None)
    assert call(fmt=4) == FMT and call(fmt=1) == FMT
    assert call(rows=-1) == SHAPE and call(d=100) == SHAPE and call(d=40000) == SHAPE
    assert call(codes=None) == NULL and call(sums=None) == NULL
    assert call(codes=ODD) == ALIGN and call(sums=ODD) == ALIGN
    assert call(rows=0, codes=None) == OK


def test_8_bit_codes_are_not_a_format_of_the_4_bit_path(lib):
    assert lib.perq_rotate_quantize(P, None, 4, 4096, 32, 5, 0, P, P, None) == FMT
    assert lib.perq_out_sizes(4, 4096, 5, 0, None, None) == FMT
