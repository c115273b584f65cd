"""The interpreter's own entry to the calls on the cache: same status as through ctypes, the same refusals, and ctypes in its place."""
import os

import numpy as np
import pytest

from test_call_products import B, changed  # noqa: F401  (the fixture)

WRITE = [16, 16, 0, 256, 256, 16, 16, 16, 4, 2, 4, 64, 16, 32, 10, 5, 16, 16, 16, 16, 0]
READ = [16, 16, 16, 16, 16, 16, 16, 4, 2, 4, 64, 16, 32, 10, 5, 16, 16, 0, 0]
ATTEND = [16, 0, 512, 16, 16, 16, 16, 16, 16, 16, 4, 2, 4, 2, 64, 16, 32, 10, 5, 4, 0.125, 0, 0, 16, 0, 16, 1 << 30, 0]
# (T is 0 where a call that nothing is wrong with would begin work: a change that is refused is refused all the same, unless it is a pointer)
NUMBERS = {"write": (WRITE, (2, 3, 4, 9, 10, 11, 12, 13, 14, 15), 8), "read": (READ, (8, 9, 10, 11, 12, 13, 14, 17), 7),
           "attend": (ATTEND, (1, 2, 11, 12, 13, 14, 15, 16, 17, 18, 19, 21, 22, 24), 10)}
ADDRESSES = {"write": (WRITE, (0, 1, 5, 6, 7, 16, 17, 18, 19)), "read": (READ, (0, 1, 2, 3, 4, 5, 6, 15, 16)), "attend": (ATTEND, (0, 3, 4, 5, 6, 7, 8, 9, 23, 25))}


def both(B, name, args):
    own, plain = {"write": (B._cache_write_i8, B._lib.perq_cache_write_i8), "read": (B._cache_read_i8, B._lib.perq_cache_read_i8),
                  "attend": (B._attention_i8, B._lib.perq_attention_i8)}[name]
    return own(*args), plain(*args)


@pytest.mark.parametrize("name", list(NUMBERS))
@pytest.mark.parametrize("value", [-1, 0, 3, 2 ** 31, 2 ** 32 + 1, -2 ** 40])
def test_numbers(B, name, value):  # noqa: F811
    args, places, rows = NUMBERS[name]
    seen = set()
    for at in places:
        own, plain = both(B, name, changed(changed(args, at, value), rows, 0))
        assert own == plain, at
        seen.add(own)
    assert seen - {0}


@pytest.mark.parametrize("name", list(ADDRESSES))
@pytest.mark.parametrize("value", [None, 8, 2 ** 64 - 8])
def test_addresses(B, name, value):  # noqa: F811
    for at in ADDRESSES[name][1]:
        own, plain = both(B, name, changed(ADDRESSES[name][0], at, value))
        assert own == plain != 0, at


def test_what_is_no_plain_integer(B):  # noqa: F811
    """A TypeError, upon which the binding takes ctypes."""
    for call, args, floats in ((B._cache_write_i8, WRITE, ()), (B._cache_read_i8, READ, ()), (B._attention_i8, ATTEND, (20,))):
        for at in range(len(args)):
            with pytest.raises(TypeError):
                call(*changed(args, at, np.float32(1.0) if at in floats else 1.5))
        for wrong in (args[:-1], args + [0]):
            with pytest.raises(TypeError):
                call(*wrong)


def test_without_the_entry(B, monkeypatch):  # noqa: F811
    from paper_2601_22347_b200 import build
    monkeypatch.setattr(build, "CALL_PATH", os.path.join(os.path.dirname(build.CALL_PATH), "no_such_file.so"))
    B._lib = None
    try:
        lib = B.load()
        assert B._cache_write_i8 is lib.perq_cache_write_i8 and B._cache_read_i8 is lib.perq_cache_read_i8 and B._attention_i8 is lib.perq_attention_i8
    finally:
        monkeypatch.undo()
        B._lib = None
        B.load()
    assert B._attention_i8 is not B._lib.perq_attention_i8
