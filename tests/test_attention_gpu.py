"""Attention over the 8-bit cache against the definition in 64 bits."""
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


def filled(lengths, heads, D, page, gen, spread=0.35, spare=2):
    """A cache of gaussian codes, whose pages' steps differ by a factor of up to about ten."""
    n_pages = sum(-(-max(n, 0) // page) for n in lengths) + spare
    cache = C.Cache(n_pages, heads, page, D, gen)
    for kind in range(2):
        cache.codes[kind] = torch.clamp(torch.round(40 * torch.randn((n_pages, heads, page, D), generator=gen)), -127, 127).to(torch.int8)
        cache.steps[kind] = torch.exp(0.6 * torch.randn((n_pages, heads), generator=gen)) * spread / 40
    return cache, C.table(lengths, page, n_pages, gen)


def queries(T, Hq, D, dtype, gen, spread=3.0):
    return (torch.randn((T, Hq, D), generator=gen) * spread).to(dtype)


def check(B, rows, lengths, heads, group, D, page, b, dtype, seed, window=0, sinks=0, out_dtype=None, scale=None, most=None, spare_rows=(0, 0), **kw):
    gen = torch.Generator()
    gen.manual_seed(seed)
    cache, pages = filled(lengths, heads, D, page, gen)
    offsets = [spare_rows[0] + n for n in C.starts(rows)]
    T = offsets[-1] + spare_rows[1]
    q = queries(T, heads * group, D, dtype, gen)
    out = torch.full((T, heads * group, D), 55.0, dtype=out_dtype or dtype).cuda()
    got = B.perq_attention_i8(q.cuda(), *cache.on_gpu(), C.ints(offsets), C.ints(lengths), pages.cuda(), most=most, b=b, scale=scale, window=window, sinks=sinks, out=out, **kw)
    assert got is out
    y, tolerance = C.attention(cache, q, offsets, lengths, pages, b, D ** -0.5 if scale is None else scale, window, sinks)
    there = slice(offsets[0], offsets[-1])
    C.compare(out[there], y[there], tolerance[there])
    assert (out[:offsets[0]] == 55.0).all() and (out[offsets[-1]:] == 55.0).all()


@pytest.mark.parametrize("page", (16, 32, 64, 128))
@pytest.mark.parametrize("D,b", [(64, 1), (64, 64), (128, 16), (128, 128)])
@pytest.mark.parametrize("group", (1, 3, 4, 8))
def test_one_token(B, D, b, page, group):
    """Decode steps: lengths from one token on, around pages and units, some sequences without rows."""
    check(B, [1, 1, 0, 1, 1, 1], [1, page + 1, 5, 300, 16, 129], 2, group, D, page, b, BF16, page + D + group)


@pytest.mark.parametrize("dtype", (BF16, F16), ids=("bf16", "f16"))
@pytest.mark.parametrize("out_dtype", (BF16, F16, F32), ids=("to_bf16", "to_f16", "to_f32"))
def test_types(B, dtype, out_dtype):
    check(B, [1, 2, 3], [70, 33, 200], 2, 4, 128, 32, 32, dtype, 5, out_dtype=out_dtype)


@pytest.mark.parametrize("rows,group", [(2, 4), (3, 5), (5, 8), (8, 2), (7, 1), (12, 4), (16, 1), (1, 40)])
def test_drafted_tokens(B, rows, group):
    """Several rows to a sequence, each seeing itself and what lies before it; tiles of rows that are not full."""
    check(B, [rows, 1, rows - 1], [150, 40, rows - 1], 2, group, 64, 16, 16, BF16, rows + group)


@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (7, 4), (16, 16), (50, 0), (50, 4), (100, 33), (1000, 4), (3, 1000)])
@pytest.mark.parametrize("rows", (1, 6))
def test_window_and_first_tokens(B, window, sinks, rows):
    check(B, [rows, rows, rows, 1], [333, rows, 64, 1], 2, 4, 64, 32, 64, BF16, window + sinks + rows, window=window, sinks=sinks)
    check(B, [rows, rows, rows], [200, rows + 1, 17], 1, 2, 128, 16, 1, F16, window + sinks + rows, window=window, sinks=sinks)


@pytest.mark.parametrize("rows", (1, 3))
def test_rows_that_see_nothing_are_zero(B, rows):
    """No tokens, and fewer tokens than rows."""
    check(B, [rows, 4, rows], [0, 2, 30], 2, 4, 64, 16, 16, BF16, rows)
    check(B, [rows, 4, rows], [0, 2, 30], 2, 4, 128, 16, 16, BF16, rows, window=3, sinks=2)


def test_rows_of_no_sequence_stay(B):
    check(B, [1, 0, 2], [50, 9, 60], 2, 4, 64, 16, 16, BF16, 1, spare_rows=(3, 5))


def test_long_and_short_sequences(B):
    """Shares of CTAs that begin and end inside tiles, tiles that many share."""
    check(B, [1, 1, 1, 1], [9000, 1, 700, 3000], 2, 4, 128, 64, 32, BF16, 2, most=1)
    check(B, [1, 4, 1], [5000, 6000, 17], 1, 3, 64, 128, 64, F16, 3, most=4)
    check(B, [1] * 40, [int(37 * (i % 7) ** 2 + 1) for i in range(40)], 2, 2, 64, 16, 16, BF16, 4, most=1)


def test_many_sequences(B):
    """More than a CTA looks at once."""
    check(B, [1 if i % 5 else 0 for i in range(600)], [1 + i % 40 for i in range(600)], 1, 2, 64, 16, 1, BF16, 6, most=1)


@pytest.mark.parametrize("scale", (0.0, 1.0, -0.2, 5.0))
def test_scales(B, scale):
    check(B, [1, 2], [100, 60], 2, 4, 64, 32, 16, BF16, 8, scale=scale)


def test_parts_of_longer_rows(B):
    gen = torch.Generator()
    gen.manual_seed(12)
    cache, pages = filled([90, 40], 2, 64, 16, gen)
    q = queries(5, 8, 64, BF16, gen)
    row = torch.full((5, 12, 64), math.nan, dtype=BF16).cuda()
    row[:, 2:10] = q.cuda()
    out = B.perq_attention_i8(row[:, 2:10], *cache.on_gpu(), C.ints([0, 2, 5]), C.ints([90, 40]), pages.cuda(), b=16)
    y, tolerance = C.attention(cache, q, [0, 2, 5], [90, 40], pages, 16, 64 ** -0.5)
    C.compare(out, y, tolerance)


@pytest.mark.parametrize("rows", (1, 5))
def test_steps_of_every_size(B, rows):
    """Pages of zeros among others (a step of 0), pages whose values are a million times larger or smaller, keys of step 0."""
    gen = torch.Generator()
    gen.manual_seed(13)
    for case in range(4):
        cache, pages = filled([200, 100], 2, 64, 16, gen)
        at = pages[0, :5].long()
        if case == 0:
            cache.codes[1][at[0]], cache.steps[1][at[0]] = 0, 0.0
            cache.codes[0][at[3]], cache.steps[0][at[3]] = 0, 0.0
        elif case == 1:
            cache.steps[1][at[1]] *= 2.0 ** -20
            cache.steps[1][at[2]] *= 2.0 ** 20
        elif case == 2:
            cache.codes[1][pages[0].long().clamp_max(cache.n_pages - 1)] = 0
            cache.steps[1][pages[0].long().clamp_max(cache.n_pages - 1)] = 0.0
        else:
            cache.codes[1][at[2]], cache.steps[1][at[2]] = 0, 0.0
            cache.steps[1][:] *= 2.0 ** -30
        q = queries(2 * rows, 8, 64, BF16, gen)
        args = ([0, rows, 2 * rows], [200, 100])
        out = B.perq_attention_i8(q.cuda(), *cache.on_gpu(), C.ints(args[0]), C.ints(args[1]), pages.cuda(), b=64, out_dtype=F32)
        y, tolerance = C.attention(cache, q, *args, pages, 64, 64 ** -0.5)
        C.compare(out, y, tolerance)


@pytest.mark.parametrize("bad", (math.inf, math.nan))
@pytest.mark.parametrize("kind", (0, 1))
@pytest.mark.parametrize("rows", (1, 6))
def test_pages_that_are_not_finite(B, bad, kind, rows):
    """What sees such a page is not finite; what does not see it is as it was, and so are the others' heads."""
    gen = torch.Generator()
    gen.manual_seed(14)
    cache, pages = filled([100, 100], 2, 64, 16, gen)
    q = queries(2 * rows, 4, 64, BF16, gen)
    args = ([0, rows, 2 * rows], [100, 100])
    y, tolerance = C.attention(cache, q, *args, pages, 16, 64 ** -0.5, 20, 4)
    for place, hidden in ((int(pages[0, 0]), False), (int(pages[0, 2]), True)):
        device = cache.on_gpu()
        device[2 * kind][place, 1], device[2 * kind + 1][place, 1] = 0, bad
        out = B.perq_attention_i8(q.cuda(), *device, C.ints(args[0]), C.ints(args[1]), pages.cuda(), b=16, window=20, sinks=4).cpu()
        if hidden:
            C.compare(out, y, tolerance)
        else:
            assert not torch.isfinite(out[:rows, 2:]).any()
            C.compare(out[:rows, :2], y[:rows, :2], tolerance[:rows, :2])
            C.compare(out[rows:], y[rows:], tolerance[rows:])


def test_what_is_out_of_range_is_no_fault(B):
    """Pages outside the pool, lengths beyond the table, offsets in any order: wrong numbers, nothing else."""
    gen = torch.Generator()
    gen.manual_seed(15)
    cache, pages = filled([64, 64], 2, 64, 16, gen)
    device, q = cache.on_gpu(), queries(12, 4, 64, BF16, gen).cuda()
    wild = torch.tensor([[-1, 1 << 30, 2, 99], [5, -(1 << 31), 1, 0]], dtype=torch.int32).cuda()
    for offsets, lengths in (([0, 6, 12], [64, 64]), ([-9, 1 << 30, 5], [1 << 30, -5]), ([12, 6, 0], [64, 64]), ([0, 12, 12], [2 ** 31 - 1, 2 ** 31 - 1])):
        for window, sinks in ((0, 0), (2 ** 31 - 1, 2 ** 31 - 1), (5, 3)):
            for most in (1, 3, None):
                B.perq_attention_i8(q, *device, C.ints(offsets), C.ints(lengths), wild, most=most, b=16, window=window, sinks=sinks)
    torch.cuda.synchronize()


def test_fewer_rows_than_a_sequence_has(B):
    """Rows from `most` on stay as they are."""
    gen = torch.Generator()
    gen.manual_seed(16)
    cache, pages = filled([50, 60], 2, 64, 16, gen)
    q, args = queries(9, 4, 64, BF16, gen), ([0, 6, 9], [50, 60])
    out = torch.full((9, 4, 64), 55.0, dtype=BF16).cuda()
    B.perq_attention_i8(q.cuda(), *cache.on_gpu(), C.ints(args[0]), C.ints(args[1]), pages.cuda(), most=4, b=16, out=out)
    y, tolerance = C.attention(cache, q, *args, pages, 16, 64 ** -0.5)
    for part in (slice(0, 4), slice(6, 9)):
        C.compare(out[part], y[part], tolerance[part])
    assert (out[4:6] == 55.0).all()


# ------------------------------------------------------------------------------------------------------ many rows to a sequence
@pytest.mark.parametrize("page", (16, 32, 64, 128))
@pytest.mark.parametrize("D,b", [(64, 1), (64, 64), (128, 32), (128, 128)])
@pytest.mark.parametrize("group", (1, 4))
def test_prompts(B, D, b, page, group):
    """Ragged prompts beside short ones: tiles of one and two parts, not full, keys that end inside a tile and a page."""
    check(B, [300 // group, 1, 70, 0, 513 // group, 129], [300 // group, 40, 70, 9, 513 // group, 129], 2, group, D, page, b, BF16, page + D + group)


@pytest.mark.parametrize("rows,length", [(65, 65), (128, 128), (129, 129), (256, 256), (257, 257), (100, 700), (65, 1000), (300, 1111)])
@pytest.mark.parametrize("D", (64, 128))
def test_one_sequence(B, rows, length, D):
    """Few tiles of rows behind long contexts: keys split over CTAs."""
    check(B, [rows], [length], 2, 1, D, 32, 16, F16, rows + D)
    check(B, [rows], [length], 1, 3, D, 16, 16, BF16, rows + D)


@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (7, 4), (128, 128), (50, 0), (100, 4), (200, 133), (1000, 4), (3, 1000)])
@pytest.mark.parametrize("D,page", [(64, 16), (128, 64)])
def test_prompts_with_a_window(B, window, sinks, D, page):
    check(B, [200, 90, 3, 333], [700, 90, 50, 400], 2, 2, D, page, D, BF16, window + sinks, window=window, sinks=sinks)
    check(B, [260], [900], 1, 1, D, page, 1, BF16, window + sinks, window=window, sinks=sinks)


@pytest.mark.parametrize("dtype", (BF16, F16), ids=("bf16", "f16"))
@pytest.mark.parametrize("out_dtype", (BF16, F16, F32), ids=("to_bf16", "to_f16", "to_f32"))
def test_types_of_prompts(B, dtype, out_dtype):
    check(B, [100, 70], [100, 200], 2, 3, 128, 32, 32, dtype, 5, out_dtype=out_dtype, spare_rows=(2, 7))


@pytest.mark.parametrize("length", (0, 3, 100))
def test_prompts_of_more_rows_than_tokens(B, length):
    """Rows at positions below 0 see nothing."""
    check(B, [150], [length], 2, 2, 64, 16, 16, BF16, 1)
    check(B, [150, 80], [length, 0], 2, 2, 128, 64, 16, BF16, 2)
    check(B, [150, 80], [length, 0], 2, 2, 64, 64, 16, BF16, 2, window=5, sinks=3)


@pytest.mark.parametrize("scale", (0.0, -0.2, 3.0))
def test_scales_of_prompts(B, scale):
    check(B, [100, 70], [150, 70], 2, 4, 64, 32, 16, BF16, 8, scale=scale)


def test_fewer_prompt_rows_than_a_sequence_has(B):
    gen = torch.Generator()
    gen.manual_seed(16)
    cache, pages = filled([250, 100], 2, 64, 16, gen)
    q, args = queries(300, 4, 64, BF16, gen), ([0, 200, 300], [250, 100])
    out = torch.full((300, 4, 64), 55.0, dtype=BF16).cuda()
    B.perq_attention_i8(q.cuda(), *cache.on_gpu(), C.ints(args[0]), C.ints(args[1]), pages.cuda(), most=130, b=16, out=out)
    y, tolerance = C.attention(cache, q, *args, pages, 16, 64 ** -0.5)
    for part in (slice(0, 130), slice(200, 300)):
        C.compare(out[part], y[part], tolerance[part])
    assert (out[130:200] == 55.0).all()


@pytest.mark.parametrize("page", (16, 64))
def test_steps_of_every_size_before_prompts(B, page):
    gen = torch.Generator()
    gen.manual_seed(13)
    for case in range(4):
        cache, pages = filled([400, 100], 2, 64, page, gen)
        at = pages[0, :5].long()
        if case == 0:
            cache.codes[1][at[0]], cache.steps[1][at[0]] = 0, 0.0
            cache.codes[0][at[3]], cache.steps[0][at[3]] = 0, 0.0
        elif case == 1:
            cache.steps[1][at[1]] *= 2.0 ** -20
            cache.steps[1][at[2]] *= 2.0 ** 20
        elif case == 2:
            every = pages[0][pages[0] < cache.n_pages].long()
            cache.codes[1][every], cache.steps[1][every] = 0, 0.0
        else:
            cache.codes[1][at[2]], cache.steps[1][at[2]] = 0, 0.0
            cache.steps[1][:] *= 2.0 ** -30
        q, args = queries(200, 8, 64, BF16, gen), ([0, 110, 200], [400, 100])
        out = B.perq_attention_i8(q.cuda(), *cache.on_gpu(), C.ints(args[0]), C.ints(args[1]), pages.cuda(), b=64, out_dtype=F32)
        y, tolerance = C.attention(cache, q, *args, pages, 64, 64 ** -0.5)
        C.compare(out, y, tolerance)


@pytest.mark.parametrize("bad", (math.inf, math.nan))
@pytest.mark.parametrize("kind", (0, 1))
@pytest.mark.parametrize("page", (16, 32))
def test_pages_that_are_not_finite_before_prompts(B, bad, kind, page):
    """Rows that see such a page are not finite; those that do not, for the window, are as they were, and so are the others' heads."""
    gen = torch.Generator()
    gen.manual_seed(14)
    cache, pages = filled([300, 100], 2, 64, page, gen)
    q, args = queries(350, 4, 64, BF16, gen), ([0, 250, 350], [300, 100])
    window, sinks, index = 40, 4, 3
    y, tolerance = C.attention(cache, q, *args, pages, 16, 64 ** -0.5, window, sinks)
    device = cache.on_gpu()
    place = int(pages[0, index])
    device[2 * kind][place, 1], device[2 * kind + 1][place, 1] = 0, bad
    out = B.perq_attention_i8(q.cuda(), *device, C.ints(args[0]), C.ints(args[1]), pages.cuda(), b=16, window=window, sinks=sinks).cpu()
    sees = C.visible(torch.arange(50, 300), 300, window, sinks)[:, index * page:(index + 1) * page].any(1)
    assert sees.any() and not sees.all() and not torch.isfinite(out[:250, 2:][sees]).any()
    C.compare(out[:250, :2], y[:250, :2], tolerance[:250, :2])
    C.compare(out[:250, 2:][~sees], y[:250, 2:][~sees], tolerance[:250, 2:][~sees])
    C.compare(out[250:], y[250:], tolerance[250:])


def test_what_is_out_of_range_is_no_fault_for_prompts(B):
    gen = torch.Generator()
    gen.manual_seed(15)
    cache, pages = filled([64, 64], 2, 64, 16, gen)
    device, q = cache.on_gpu(), queries(120, 4, 64, BF16, gen).cuda()
    wild = torch.tensor([[-1, 1 << 30, 2, 99], [5, -(1 << 31), 1, 0]], dtype=torch.int32).cuda()
    for offsets, lengths in (([0, 60, 120], [64, 64]), ([-9, 1 << 30, 5], [1 << 30, -5]), ([120, 6, 0], [64, 64]), ([0, 120, 120], [2 ** 31 - 1, 2 ** 31 - 1])):
        for window, sinks in ((0, 0), (2 ** 31 - 1, 2 ** 31 - 1), (5, 3)):
            for most in (50, None, 2 ** 31 - 1):
                B.perq_attention_i8(q, *device, C.ints(offsets), C.ints(lengths), wild, most=most, b=16, window=window, sinks=sinks)
    torch.cuda.synchronize()
