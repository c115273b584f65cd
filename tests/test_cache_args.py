"""Refusals of the calls on the 8-bit cache: all of them come before the library touches the CUDA runtime, so they run without a GPU."""
import ctypes as C

import pytest

OK, NULL, SHAPE, BLOCK, FMT, ALIGN, WORKSPACE = 0, 1, 2, 3, 5, 6, 9
P = C.c_void_p(0x1000)
ODD = C.c_void_p(0x1008)
BASE = dict(T=4, S=2, H=4, D=64, b=16, page=32, pages=10, width=5, kc=P, ks=P, vc=P, vs=P, off=P, len=P, tab=P, type=0)


@pytest.fixture(scope="module")
def lib():
    from paper_2601_22347_b200 import binding, build
    build.build()
    return binding.load()


def write(lib, **change):
    v = dict(BASE, k=P, v=P, k_stride=256, v_stride=256, **change)
    return lib.perq_cache_write_i8(v["k"], v["v"], v["type"], v["k_stride"], v["v_stride"], v["off"], v["len"], v["tab"], v["T"], v["S"], v["H"], v["D"], v["b"], v["page"],
                                   v["pages"], v["width"], v["kc"], v["ks"], v["vc"], v["vs"], None)


def read(lib, **change):
    v = dict(BASE, k=P, v=P, **change)
    return lib.perq_cache_read_i8(v["kc"], v["ks"], v["vc"], v["vs"], v["off"], v["len"], v["tab"], v["T"], v["S"], v["H"], v["D"], v["b"], v["page"], v["pages"],
                                  v["width"], v["k"], v["v"], v["type"], None)


def attend(lib, **change):
    v = dict(dict(BASE, q=P, stride=512, g=2, most=4, scale=0.1, window=0, sinks=0, out=P, ot=0, wk=P, wb=1 << 30), **change)
    return lib.perq_attention_i8(v["q"], v["type"], v["stride"], v["kc"], v["ks"], v["vc"], v["vs"], v["off"], v["len"], v["tab"], v["T"], v["S"], v["H"], v["g"], v["D"],
                                 v["b"], v["page"], v["pages"], v["width"], v["most"], v["scale"], v["window"], v["sinks"], v["out"], v["ot"], v["wk"], v["wb"], None)


REFUSED = [(dict(T=-1), SHAPE), (dict(T=2 ** 30 + 1), SHAPE), (dict(S=-1), SHAPE), (dict(S=65537), SHAPE), (dict(H=0), SHAPE), (dict(H=1025), SHAPE), (dict(D=32), SHAPE),
           (dict(D=96), SHAPE), (dict(D=256), SHAPE), (dict(page=8), SHAPE), (dict(page=48), SHAPE), (dict(page=256), SHAPE), (dict(page=0), SHAPE), (dict(pages=0), SHAPE),
           (dict(pages=2 ** 31), SHAPE), (dict(width=0), SHAPE), (dict(width=2 ** 25 + 1), SHAPE), (dict(b=0), BLOCK), (dict(b=8), BLOCK), (dict(b=48), BLOCK),
           (dict(b=128), BLOCK), (dict(type=3), FMT), (dict(type=-1), FMT)]
REFUSED += [({name: None}, NULL) for name in ("kc", "ks", "vc", "vs", "off", "len", "tab")] + [({name: ODD}, ALIGN) for name in ("kc", "ks", "vc", "vs", "off", "len", "tab")]


@pytest.mark.parametrize("call", [write, read, attend])
@pytest.mark.parametrize("change,status", REFUSED, ids=[",".join("%s=%s" % (k, getattr(v, "value", v)) for k, v in c.items()) for c, _ in REFUSED])
def test_refused(lib, call, change, status):
    assert call(lib, **change) == status


@pytest.mark.parametrize("call", [write, read, attend])
def test_no_rows(lib, call):
    """Nothing to read or write: pointers may be anything, sizes are still looked at."""
    nothing = dict.fromkeys(("kc", "ks", "vc", "vs", "off", "len", "tab"))
    assert call(lib, T=0, **nothing) == OK and call(lib, S=0, **nothing) == OK
    assert call(lib, T=0, D=48) == SHAPE


@pytest.mark.parametrize("change,status", [(dict(k_stride=255), SHAPE), (dict(k_stride=260), SHAPE), (dict(k_stride=248), SHAPE), (dict(v_stride=-256), SHAPE), (dict(k=None), NULL),
                                           (dict(v=None), NULL), (dict(k=ODD), ALIGN), (dict(v=ODD), ALIGN), (dict(type=2), FMT)])
def test_write_refused(lib, change, status):
    v = dict(BASE, k=P, v=P, k_stride=256, v_stride=256)
    v.update(change)
    assert lib.perq_cache_write_i8(v["k"], v["v"], v["type"], v["k_stride"], v["v_stride"], v["off"], v["len"], v["tab"], v["T"], v["S"], v["H"], v["D"], v["b"], v["page"],
                                   v["pages"], v["width"], v["kc"], v["ks"], v["vc"], v["vs"], None) == status


def test_read_refused(lib):
    for name, value, status in (("k", None, NULL), ("v", None, NULL), ("k", ODD, ALIGN), ("v", ODD, ALIGN)):
        v = dict(BASE, k=P, v=P)
        v[name] = value
        assert lib.perq_cache_read_i8(v["kc"], v["ks"], v["vc"], v["vs"], v["off"], v["len"], v["tab"], v["T"], v["S"], v["H"], v["D"], v["b"], v["page"], v["pages"],
                                      v["width"], v["k"], v["v"], v["type"], None) == status


@pytest.mark.parametrize("change,status", [(dict(g=0), SHAPE), (dict(g=257, stride=1 << 20), SHAPE), (dict(stride=504), SHAPE), (dict(stride=513), SHAPE), (dict(most=0), SHAPE),
                                           (dict(window=-1), SHAPE), (dict(sinks=-1), SHAPE), (dict(type=2), FMT), (dict(ot=3), FMT), (dict(ot=-1), FMT), (dict(q=None), NULL),
                                           (dict(out=None), NULL), (dict(q=ODD), ALIGN), (dict(out=ODD), ALIGN), (dict(wk=None), WORKSPACE), (dict(wb=16), WORKSPACE),
                                           (dict(wk=ODD), ALIGN)])
def test_attend_refused(lib, change, status):
    assert attend(lib, **change) == status


def test_workspace(lib):
    """Enough for a call is enough for fewer rows, sequences and rows of the longest."""
    def need(T, S, H, g, D, most):
        n = C.c_size_t(0)
        assert lib.perq_attention_i8_workspace_bytes(T, S, H, g, D, most, C.byref(n)) == OK
        return n.value

    assert need(0, 4, 8, 4, 128, 1) == 0 and need(8, 0, 8, 4, 128, 1) == 0
    for H, g, D in ((8, 4, 128), (1, 1, 64), (4, 16, 64), (32, 1, 128)):
        sizes = [(T, S, most) for T in (1, 2, 5, 64, 700, 4096) for S in (1, 2, 64, 300) for most in (1, 2, 8, 100, 5000)]
        for T, S, most in sizes:
            for T2, S2, most2 in sizes:
                if T2 <= T and S2 <= S and most2 <= most:
                    assert need(T2, S2, H, g, D, most2) <= need(T, S, H, g, D, most)
    n = C.c_size_t(0)
    assert lib.perq_attention_i8_workspace_bytes(1, 1, 8, 4, 96, 1, C.byref(n)) == SHAPE
    assert lib.perq_attention_i8_workspace_bytes(1, 1, 8, 0, 64, 1, C.byref(n)) == SHAPE
    assert lib.perq_attention_i8_workspace_bytes(1, 1, 8, 4, 64, 0, C.byref(n)) == SHAPE
    assert lib.perq_attention_i8_workspace_bytes(1, 1, 8, 4, 64, 1, None) == NULL


@pytest.mark.parametrize("scale", [float("nan"), float("inf"), -float("inf"), 1e39])
def test_scales_that_are_not_finite(lib, scale):
    assert attend(lib, scale=scale) == SHAPE
