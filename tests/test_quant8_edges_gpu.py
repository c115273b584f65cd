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


def want(x, perm, b):
    """(largest |u| of each row, NaN where one is) in 64 bits."""
    y = (x if perm is None else x[:, perm.long()]).double()
    u = torch.zeros_like(y)
    h = torch.ones(1, 1, dtype=torch.float64)
    while h.shape[0] < b:
        h = torch.cat((torch.cat((h, h), 1), torch.cat((h, -h), 1)), 0)
    for r in range(len(y)):                                     # (as sums of single terms: products of whole blocks may meet infinities of both signs)
        u[r] = (y[r].reshape(-1, 1, b) * h.cuda()[None]).sum(2).flatten()
    return u.abs().amax(1, keepdim=True)


NAN, INF = float("nan"), float("inf")


@pytest.mark.parametrize("b,d", [(1, 32), (32, 32), (16, 64), (1, 512), (32, 544), (64, 2048), (512, 2048), (128, 9728), (32, 16384)])
@pytest.mark.parametrize("permuted", [False, True])
def test_rows_that_are_not_finite_say_so(B, b, d, permuted):  # noqa: F811
    """Their scale is what 64 bits make of the largest output, their codes are 0, and the rows between them are as they are without them."""
    perm = torch.randperm(d, generator=torch.Generator().manual_seed(d)).to(torch.int32).cuda() if permuted else None
    g = torch.Generator().manual_seed(b + d)
    clean = torch.randn(50, d, generator=g).to(torch.bfloat16).cuda()
    x, at = clean.clone(), lambda: int(torch.randint(d, (1,), generator=g))
    x[0, at()], x[3, at()], x[6, at()] = NAN, INF, -INF
    x[7] = NAN
    x[9, at()], x[9, at()] = NAN, INF
    x[12] = INF
    x[20, 0], x[20, 1] = INF, -INF
    x[21, :] = torch.where(torch.arange(d, device="cuda") % 3 == 0, INF, -INF)
    x[30] = 0
    x[30, at()] = NAN
    x[31] = x[31] * 2.0 ** -130
    x[31, at()] = NAN
    x[32, d - 1] = -NAN
    x[49, 0] = NAN
    codes, scales = B.perq_rotate_quantize_i8(x, perm, b)
    top = want(x, perm, b)
    wrong = ~torch.isfinite(top).flatten()
    assert wrong.sum() == 12
    assert torch.equal(torch.isnan(scales[wrong]), torch.isnan(top[wrong])) and torch.equal(torch.isposinf(scales[wrong]), torch.isposinf(top[wrong]))
    assert (codes[wrong] == 0).all()
    alone = x.clone()
    alone[wrong] = 0
    others = B.perq_rotate_quantize_i8(alone, perm, b)
    assert torch.equal(codes[~wrong], others[0][~wrong]) and torch.equal(scales[~wrong], others[1][~wrong])


def test_a_layer_does_not_hide_them(B):  # noqa: F811
    x = torch.randn(5, 1024, generator=torch.Generator().manual_seed(1)).to(torch.bfloat16).cuda()
    x[1], x[3, 700] = NAN, NAN
    w, sw = B.perq_rotate_quantize_i8(torch.randn(64, 1024, generator=torch.Generator().manual_seed(2)).to(torch.bfloat16).cuda(), None, 32)
    out = B.perq_matmul_i8(*B.perq_rotate_quantize_i8(x, None, 32), B.PERQ_FMT_INT8, w, sw, B.PERQ_FMT_INT8)
    assert torch.equal(torch.isnan(out).all(1), torch.tensor([False, True, False, True, False], device="cuda")) and torch.isfinite(out[::2]).all()


@pytest.mark.parametrize("b", [1, 16, 32, 128, 512])
@pytest.mark.parametrize("d", [512, 2048, 9728])
def test_finite_rows_whose_sums_pass_fp32(B, b, d):  # noqa: F811
    """sqrt(b) |y| from 2^128 on: every finite row has its codes and scale."""
    g = torch.Generator().manual_seed(b + d)
    largest = 255.0 * 2.0 ** 120
    x = torch.randn(30, d, generator=g).to(torch.bfloat16)
    x[0] = largest
    x[1] = torch.where(torch.randint(0, 2, (d,), generator=g) > 0, largest, -largest)
    x[5, d // 2:] = -largest
    x[9] = torch.randint(-255, 256, (d,), generator=g) * 2.0 ** 120
    x[10, :2] = largest
    x[29] = torch.randint(100, 256, (d,), generator=g) * 2.0 ** 120
    check(B, x.cuda(), None, b)
