"""Writing the 8-bit cache and reading it back, against the definition in 64 bits: codes and steps are equal."""
import math

import pytest
import torch

import cache as C

pytestmark = pytest.mark.gpu
BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32


@pytest.fixture(scope="module")
def B():
    from paper_2601_22347_b200 import binding
    return binding


def tokens(T, heads, D, dtype, gen, spread=1.0):
    """Gaussian rows with a few larger channels, some rows zero."""
    x = torch.randn((T, heads, D), generator=gen) * spread
    x[..., torch.randperm(D, generator=gen)[:max(1, D // 32)]] *= 10.0
    x[torch.rand(T, generator=gen) < 0.1] = 0.0
    return x.to(dtype)


def check_write(B, steps, heads, D, page, b, dtype, seed, strided=False, spread=lambda step: 1.0, **kw):
    """steps: for each call the new rows of every sequence.  Codes and steps equal the definition's after each."""
    gen = torch.Generator()
    gen.manual_seed(seed)
    S, total = len(steps[0]), [sum(rows) for rows in zip(*steps)]
    n_pages = sum(-(-n // page) for n in total) + 2
    pages = C.table(total, page, n_pages, gen)
    cache = C.Cache(n_pages, heads, page, D, gen)
    device = cache.on_gpu()
    lengths = [0] * S
    for step, rows in enumerate(steps):
        lengths = [l + n for l, n in zip(lengths, rows)]
        offsets = C.starts(rows)
        k, v = (tokens(offsets[-1], heads, D, dtype, gen, spread(step)) for _ in range(2))
        if strided:                                    # as parts of a longer row
            row = torch.full((len(k), 3 * heads + 1, D), math.nan, dtype=dtype).cuda()
            row[:, heads:2 * heads], row[:, 2 * heads:3 * heads] = k.cuda(), v.cuda()
            kd, vd = row[:, heads:2 * heads], row[:, 2 * heads:3 * heads]
        else:
            kd, vd = k.cuda(), v.cuda()
        B.perq_cache_write_i8(kd, vd, *device, C.ints(offsets), C.ints(lengths), pages.cuda(), b=b, **kw)
        cache.write(k, v, offsets, lengths, pages, b)
        for got, want, name in zip(device, (cache.codes[0], cache.steps[0], cache.codes[1], cache.steps[1]), ("k codes", "k steps", "v codes", "v steps")):
            got = got.cpu()
            assert torch.equal(got, want), "%s differ in call %d: %d of %d" % (name, step, int((got != want).sum()), want.numel())
    return cache, device, pages, lengths


@pytest.mark.parametrize("dtype", (BF16, F16), ids=("bf16", "f16"))
@pytest.mark.parametrize("page", (16, 32, 64, 128))
@pytest.mark.parametrize("D,b", [(64, 1), (64, 16), (64, 64), (128, 1), (128, 32), (128, 128)])
def test_prompts_then_tokens(B, D, b, page, dtype):
    """Prompts of any length, then single tokens, then several: every form of the kernel, pages that are opened, filled and passed."""
    check_write(B, [[page * 2 + 3, 1, page, 0, page - 1], [1] * 5, [1, 0, 1, 1, 1], [3, 2, 1, 0, 5], [page + 1, 0, 1, 2, 3 * page]], 3, D, page, b, dtype, 7 * page + D + b)


@pytest.mark.parametrize("D,page,b", [(64, 16, 64), (128, 64, 128), (128, 128, 16), (64, 128, 32)])
def test_steps_that_grow(B, D, page, b):
    """Every call's tokens are larger than the last one's, so that earlier codes are rounded again, some by a little and some to nothing."""
    check_write(B, [[5, 1]] + [[1, 2]] * 6, 2, D, page, b, BF16, 3, spread=lambda step: 1.07 ** step)
    check_write(B, [[5, 1]] + [[1, 2]] * 6, 2, D, page, b, BF16, 4, spread=lambda step: 3.0 ** step)
    check_write(B, [[page - 3, 2], [2, page], [40, 1]], 2, D, page, b, F16, 5, spread=lambda step: 1.5 ** step)


@pytest.mark.parametrize("heads", (1, 5, 8, 40))
def test_heads_and_parts_of_rows(B, heads):
    check_write(B, [[70, 3], [1, 1], [9, 30]], heads, 64, 32, 16, BF16, heads, strided=True)


def test_many_sequences(B):
    """More sequences than a CTA looks at once."""
    gen = torch.Generator()
    gen.manual_seed(11)
    rows = [int(n) for n in torch.randint(0, 4, (700,), generator=gen)]
    check_write(B, [rows, [1] * 700], 1, 64, 16, 16, BF16, 12)


@pytest.mark.parametrize("value", (1.0, -2.5, 3.0))
@pytest.mark.parametrize("b", (1, 16, 64))
def test_equal_values_and_ties(B, value, b):
    """Constant rows; whole numbers whose quotients lie on borders between codes."""
    gen = torch.Generator()
    gen.manual_seed(2)
    page, D, heads = 32, 64, 2
    cache = C.Cache(4, heads, page, D, gen)
    device, pages = cache.on_gpu(), C.table([60], page, 4, gen)
    constant = torch.full((30, heads, D), value).to(BF16)
    # 127 in each row makes the step a power of two: 0.5, 1.5, .. are ties
    whole = torch.randint(-254, 255, (30, heads, D), generator=gen).float() / 2
    whole[..., 0] = 127.0
    for at, x in ((30, constant), (60, whole.to(BF16))):
        B.perq_cache_write_i8(x.cuda(), x.cuda(), *device, C.ints([0, 30]), C.ints([at]), pages.cuda(), b=b)
        cache.write(x, x, [0, 30], [at], pages, b)
        for got, want in zip(device, (cache.codes[0], cache.steps[0], cache.codes[1], cache.steps[1])):
            assert torch.equal(got.cpu(), want)


@pytest.mark.parametrize("scale", (2.0 ** -133, 2.0 ** -120, 2.0 ** -90, 2.0 ** 90, 2.0 ** 118))
def test_ends_of_the_range(B, scale):
    """bf16 from subnormals to its largest; a step that fp32 rounds to 0 makes codes 0."""
    gen = torch.Generator()
    gen.manual_seed(8)
    page, D, heads, b = 16, 128, 2, 128
    cache = C.Cache(3, heads, page, D, gen)
    device, pages = cache.on_gpu(), C.table([20], page, 3, gen)
    for at, n in ((18, 18), (20, 2)):
        x = (torch.randn((n, heads, D), generator=gen).double() * scale).to(BF16)
        B.perq_cache_write_i8(x.cuda(), x.cuda(), *device, C.ints([0, n]), C.ints([at]), pages.cuda(), b=b)
        cache.write(x, x, [0, n], [at], pages, b)
        for got, want in zip(device, (cache.codes[0], cache.steps[0], cache.codes[1], cache.steps[1])):
            assert torch.equal(got.cpu(), want)


@pytest.mark.parametrize("bad", (math.inf, -math.inf, math.nan))
@pytest.mark.parametrize("b", (1, 64))
def test_values_that_are_not_finite(B, bad, b):
    """The page and head that one is written to has codes 0 and a step that is not finite, until it starts anew; nothing else changes."""
    gen = torch.Generator()
    gen.manual_seed(9)
    page, D, heads = 32, 64, 3
    cache = C.Cache(4, heads, page, D, gen)
    device, pages = cache.on_gpu(), C.table([40], page, 4, gen)
    at = 0
    for step, n in enumerate((10, 5, 3, 20)):
        at += n
        x = tokens(n, heads, D, BF16, gen)
        clean = x.clone()
        if step == 1:
            x[2, 1, 17] = bad
        B.perq_cache_write_i8(x.cuda(), x.cuda(), *device, C.ints([0, n]), C.ints([at]), pages.cuda(), b=b)
        cache.write(clean, clean, [0, n], [at], pages, b)
    first = int(pages[0, 0])
    for kind in range(2):
        codes, steps = device[2 * kind].cpu(), device[2 * kind + 1].cpu()
        assert not torch.isfinite(steps[first, 1]) and (codes[first, 1] == 0).all()
        steps[first, 1], codes[first, 1] = cache.steps[kind][first, 1], cache.codes[kind][first, 1]
        assert torch.equal(codes, cache.codes[kind]) and torch.equal(steps, cache.steps[kind])


def test_what_is_no_page_is_not_written(B):
    """Pages outside the pool, sequences longer than their table, rows at positions below 0, rows of no sequence."""
    gen = torch.Generator()
    gen.manual_seed(10)
    page, D, heads, b = 16, 64, 2, 16
    cache = C.Cache(6, heads, page, D, gen)
    device = cache.on_gpu()
    pages = torch.tensor([[0, -1, 2], [9, 3, 4], [5, 1, 1 << 30]], dtype=torch.int32)
    x = tokens(100, heads, D, BF16, gen)
    offsets, lengths = [3, 40, 60, 70], [37, 20, 4]            # the third has ten rows and four tokens
    B.perq_cache_write_i8(x.cuda(), x.cuda(), *device, C.ints(offsets), C.ints(lengths), pages.cuda(), b=b)
    cache.write(x, x, offsets, lengths, pages, b)
    for got, want in zip(device, (cache.codes[0], cache.steps[0], cache.codes[1], cache.steps[1])):
        assert torch.equal(got.cpu(), want)
    # more tokens than the table has places for, offsets out of range: some pages of the pool change, nothing else happens
    B.perq_cache_write_i8(x.cuda(), x.cuda(), *device, C.ints([-5, 40, 20, 1 << 30]), C.ints([1 << 30, -7, 3 * page]), pages.cuda(), b=b)
    torch.cuda.synchronize()


# ------------------------------------------------------------------------------------------------------ reading back
def back_tolerance(y, dtype):
    """fp32: the factor's and the product's two roundings, then the result's."""
    return 4 * 2.0 ** -24 * y.abs() + C.half_step(y, dtype) + 2.0 ** -149


@pytest.mark.parametrize("dtype", (BF16, F16, F32), ids=("bf16", "f16", "f32"))
@pytest.mark.parametrize("D,b,page,heads", [(64, 1, 16, 1), (64, 64, 64, 3), (128, 16, 128, 8), (128, 128, 32, 5)])
def test_read(B, D, b, page, heads, dtype):
    gen = torch.Generator()
    gen.manual_seed(D + b + page)
    lengths = [5 * page + 3, 0, 1, page, 40]
    cache, device, pages, _ = check_write(B, [lengths], heads, D, page, b, BF16, 21)
    for rows in (lengths, [1, 0, 1, 1, 1], [page + 2, 0, 1, 7, 33]):
        offsets = [4 + n for n in C.starts(rows)]
        T = offsets[-1] + 3
        k, v = torch.full((T, heads, D), 77.0, dtype=dtype).cuda(), torch.full((T, heads, D), 77.0, dtype=dtype).cuda()
        got = B.perq_cache_read_i8(*device, C.ints(offsets), C.ints(lengths), pages.cuda(), T, b=b, k=k, v=v)
        assert got[0] is k and got[1] is v
        for kind, out in enumerate((k.cpu(), v.cpu())):
            for i, n in enumerate(rows):
                y = cache.tokens(kind, i, lengths[i], pages)[lengths[i] - n:]
                y = C.rotated(y, b) if kind == 0 else y
                at = out[offsets[i]:offsets[i + 1]].double()
                assert ((at - y).abs() <= back_tolerance(y, dtype)).all()
            assert (out[:4] == 77.0).all() and (out[offsets[-1]:] == 77.0).all()


def test_read_is_near_what_was_written(B):
    """Half a step a channel, in the rotated basis, so as much in 2-norm in the other; the keys' outlier channels cost less with the rotation than without."""
    gen = torch.Generator()
    gen.manual_seed(31)
    D, page, heads, n = 128, 64, 4, 300
    x = tokens(n, heads, D, BF16, gen)
    off = {}
    for b in (1, 128):
        device = C.Cache(8, heads, page, D, gen).on_gpu()
        pages = C.table([n], page, 8, gen).cuda()
        B.perq_cache_write_i8(x.cuda(), x.cuda(), *device, C.ints([0, n]), C.ints([n]), pages, b=b)
        k, v = B.perq_cache_read_i8(*device, C.ints([0, n]), C.ints([n]), pages, n, b=b, out_dtype=F32)
        off[b] = float((k.cpu() - x.float()).norm())
        most = float(device[1].max()) / 2 * math.sqrt(D) * math.sqrt(n * heads)
        assert off[b] <= 1.001 * most and float((v.cpu() - x.float()).abs().max()) <= 1.001 * float(device[3].max()) / 2
    assert off[128] < off[1]


def test_read_of_what_is_no_page(B):
    gen = torch.Generator()
    gen.manual_seed(32)
    cache = C.Cache(3, 2, 16, 64, gen)
    device = cache.on_gpu()
    pages = torch.tensor([[-4, 1, 3]], dtype=torch.int32)
    k, v = B.perq_cache_read_i8(*device, C.ints([0, 50]), C.ints([45]), pages.cuda(), 50, out_dtype=F32)
    for kind, out in enumerate((k.cpu(), v.cpu())):
        # five rows at positions below 0, then a page that is none, one that is, one that is none
        assert (out[:21] == 0).all() and (out[37:] == 0).all()
        y = cache.codes[kind][1].double().transpose(0, 1) * cache.steps[kind][1].double()[:, None]
        assert ((out[21:37].double() - y).abs() <= back_tolerance(y, F32)).all()
