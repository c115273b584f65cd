"""Rows to 8-bit codes at the ends of the range, against the definition in 64 bits."""
import pytest
import torch

from test_quant8_gpu import B, check  # noqa: F401 (the fixture)

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def no_device_error(B):  # noqa: F811
    B.perq_device_error_clear()
    yield
    torch.cuda.synchronize()
    assert B.perq_device_error() == 0


def rows(T, d, b, top, seed):
    """Small whole numbers times a power of two, some of them where quotients lie on borders, so that sqrt(b) |y| of every row is between top / 2 and top."""
    g = torch.Generator().manual_seed(seed)
    x = torch.randint(-127, 128, (T, d), generator=g).double()
    x[T // 2:] = torch.randn(T - T // 2, d, generator=g).double() * 40
    x = x.to(torch.bfloat16).double()
    h = torch.ones(1, 1, dtype=torch.float64)
    while h.shape[0] < b:
        h = torch.cat((torch.cat((h, h), 1), torch.cat((h, -h), 1)), 0)
    most = (x.reshape(-1, b) @ h).reshape(T, d).abs().amax(1, keepdim=True)
    return (x * torch.exp2(torch.floor(torch.log2(top * (1 - 2.0 ** -20) / most)))).to(torch.bfloat16).cuda()


@pytest.mark.parametrize("b", [1, 16, 32, 128, 512])
@pytest.mark.parametrize("d", [512, 2048, 9728])
@pytest.mark.parametrize("permuted", [False, True])
def test_rows_of_the_largest_numbers(B, b, d, permuted):  # noqa: F811
    """sqrt(b) |y| up to 2^128, on either side of 2^126, where the reciprocal of a row's maximum is no normal number any more."""
    perm = torch.randperm(d, generator=torch.Generator().manual_seed(d)).to(torch.int32).cuda() if permuted else None
    y = torch.cat([rows(20, d, b, 2.0 ** e, 10 * e + b) for e in (125, 126, 127, 128)])
    assert torch.isfinite(y).all()
    x = torch.empty_like(y)
    x[:, torch.arange(d, device="cuda") if perm is None else perm.long()] = y
    check(B, x, perm, b)
    check(B, x[torch.randperm(80, generator=torch.Generator().manual_seed(b))].contiguous(), perm, b)


@pytest.mark.parametrize("e", [126, 127])
def test_maxima_of_a_binade(B, e):  # noqa: F811
    """Without a rotation: every maximum that bf16 has between 2^e and twice that, and every number below it as a channel."""
    m = torch.arange(128, 256).double() * 2.0 ** (e - 7)
    below = torch.cat([torch.arange(128, 256).double() * 2.0 ** (e - 7 - k) for k in range(9)])
    x = below.clamp(max=1.0 * m[0]).repeat(128, 1)
    x = torch.where(below[None] <= m[:, None], below[None], m[:, None])
    x[:, 0] = m
    x[:, 1::2] *= -1
    check(B, x.to(torch.bfloat16).cuda(), None, 1)
