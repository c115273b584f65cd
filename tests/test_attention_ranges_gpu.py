"""Attention over the 8-bit cache with numbers far from 1."""
import pytest
import torch

import cache as C
from test_attention_gpu import filled, queries

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def B():
    from paper_2601_22347_b200 import binding
    return binding


@pytest.mark.parametrize("rows", (1, 7, 40, 90))
@pytest.mark.parametrize("D", (64, 128))
@pytest.mark.parametrize("sign", (1.0, -1.0))
@pytest.mark.parametrize("size", (2.0 ** 10, 2.0 ** 20, 2.0 ** 26, 2.0 ** 34, 2.0 ** 60))
def test_large_logits(B, size, sign, D, rows):
    """Logits of up to 127 D times `size`, D of it apart at least, so that a row has the value of the largest that it sees."""
    gen = torch.Generator()
    gen.manual_seed(rows + D)
    length, page = 120, 16
    pages = torch.randperm(9, generator=gen)[None, :8].to(torch.int32)
    cache = C.Cache(9, 1, page, D, gen)
    j = torch.arange(length)
    place, slot = pages[0, j // page].long(), j % page
    level = torch.randperm(length, generator=gen) + 8
    cache.codes[0][place, 0, slot] = (sign * level[:, None] * torch.ones(D)).to(torch.int8)
    cache.steps[0][:], cache.steps[1][:] = size, 0.25
    q = torch.ones((rows, 1, D), dtype=BF16)
    out = B.perq_attention_i8(q.cuda(), *cache.on_gpu(), C.ints([0, rows]), C.ints([length]), pages.cuda(), scale=1.0, out_dtype=F32)
    seen = C.visible(torch.arange(length - rows, length), length, 0, 0)
    best = (torch.where(seen, sign * level, -1000)).argmax(1)
    y = cache.tokens(1, 0, length, pages)[best]
    # (the next one has at most e^-65536 of its probability.  That one number is rounded to fp16, by 2^-11, where it is added to the values, and not where it is divided by)
    C.compare(out, y, (2.0 ** -11 + 2.0 ** -20) * y.abs())


def run(B, rows, D, b, of_queries, of_scale, of_steps, spread=3.0):
    gen = torch.Generator()
    gen.manual_seed(rows + D + b)
    lengths = [rows + 90, 700]
    cache, pages = filled(lengths, 2, D, 32, gen)
    cache.steps[0] *= of_steps
    offsets = [0, rows, 2 * rows]
    q = (queries(2 * rows, 4, D, BF16, gen, spread).double() * of_queries).to(BF16)
    scale = D ** -0.5 * of_scale
    out = B.perq_attention_i8(q.cuda(), *cache.on_gpu(), C.ints(offsets), C.ints(lengths), pages.cuda(), b=b, scale=scale, out_dtype=F32)
    y, tolerance = C.attention(cache, q, offsets, lengths, pages, b, scale)
    C.compare(out, y, tolerance)


@pytest.mark.parametrize("rows", (1, 7, 90))
@pytest.mark.parametrize("D,b", [(64, 1), (64, 64), (128, 128)])
@pytest.mark.parametrize("q,scale,step", [(-40, -40, 80), (-20, -60, 80), (0, 75, -75), (60, 40, -100), (-100, 0, 100), (0, -100, 100)])
def test_products_of_far_factors(B, q, scale, step, rows, D, b):
    run(B, rows, D, b, 2.0 ** q, 2.0 ** scale, 2.0 ** step)


@pytest.mark.parametrize("rows", (1, 7, 90))
@pytest.mark.parametrize("D,b", [(64, 64), (128, 128)])
def test_queries_near_the_largest(B, rows, D, b):
    """Whose rotation passes fp32's largest (bf16's is 2^128)."""
    run(B, rows, D, b, 2.0 ** 125, 2.0 ** -100, 2.0 ** -25, spread=1.0)
