"""Numbers beyond 32 bits are refused by the calls on the 8-bit cache before anything else is looked at, so without a GPU too."""
import pytest

from paper_2601_22347_b200 import binding as B

SHAPE, BLOCK = 2, 3
PAST = [2 ** 31, 2 ** 32, 2 ** 32 + 1, 2 ** 40 + 16, -2 ** 31 - 1, -2 ** 32 + 4, 2 ** 64 + 64]


@pytest.mark.parametrize("value", PAST)
@pytest.mark.parametrize("name,status", [("most", SHAPE), ("window", SHAPE), ("sinks", SHAPE), ("b", BLOCK)])
def test_attention(name, status, value):
    with pytest.raises(B.PerqError) as error:
        B.perq_attention_i8(*[None] * 8, **{name: value})
    assert error.value.status == status


@pytest.mark.parametrize("value", PAST)
def test_write_and_read(value):
    for call in (lambda: B.perq_cache_write_i8(*[None] * 9, b=value), lambda: B.perq_cache_read_i8(*[None] * 7, 4, b=value)):
        with pytest.raises(B.PerqError) as error:
            call()
        assert error.value.status == BLOCK


@pytest.mark.parametrize("value", PAST)
@pytest.mark.parametrize("at", (1, 2, 3, 4, 5))
def test_workspace(at, value):
    args = [4, 2, 8, 4, 64, 4]
    args[at] = value
    with pytest.raises(B.PerqError) as error:
        B.perq_attention_i8_workspace_bytes(*args)
    assert error.value.status == SHAPE
