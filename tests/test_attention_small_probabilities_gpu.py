"""Attention over the 8-bit cache where few keys have nearly all of the probability and a value of zero, so that results are what small probabilities make of the others."""
import pytest
import torch

import cache as C

pytestmark = pytest.mark.gpu
F16, F32 = torch.float16, torch.float32


@pytest.fixture(scope="module")
def B():
    from paper_2601_22347_b200 import binding
    return binding


def some_dominate(length, every, bits, D, page, gen):
    """One head whose keys have one channel: 127 for every `every`-th token (0: the first alone), 0 for the others, which are 2^-bits as probable.  Queries of 1 in that channel.
    Values of the former are 0, of the others 60 to 127 steps of 1 / 64."""
    n_pages = -(-length // page)
    cache, pages = C.Cache(n_pages, 1, page, D, gen), torch.randperm(n_pages, generator=gen).to(torch.int32)[None]
    j = torch.arange(length)
    place, slot = pages[0, j // page].long(), j % page
    first = j % every == 0 if every else j == 0
    cache.codes[0][:], cache.codes[1][:] = 0, 0
    cache.codes[0][place, 0, slot, 3] = torch.where(first, 127, 0).to(torch.int8)
    cache.codes[1][place, 0, slot] = torch.where(first[:, None], 0, torch.randint(60, 128, (length, D), generator=gen)).to(torch.int8)
    cache.steps[0][:], cache.steps[1][:] = bits * 0.6931471805599453 / 127, 1 / 64
    return cache, pages


def expected(cache, pages, rows, length):
    """(out, tolerance) of one head's rows in 64 bits.

    A probability's exponent is off by its logit's and its sums' roundings, (64 + 2 |x|) 2^-22 in all (a query of one channel is kept exactly); as a fp16 number by 2^-11 of it, or by half of
    fp16's smallest step, 2^-25, where 2^7 stands for a probability of at most the largest: 2^-32 of that.  Sums are of the same probabilities in fp32."""
    k, v = (cache.tokens(kind, 0, length, pages)[:, 0] for kind in (0, 1))
    seen = C.visible(torch.arange(length - rows, length), length, 0, 0)
    x = k[:, 3].expand(rows, length).masked_fill(~seen, -torch.inf)
    p = torch.softmax(x, 1)
    d = (64 + 2 * torch.where(seen, x.abs(), 0.0)) * 2.0 ** -22
    y = p @ v
    return y, 1.05 * ((p * (d + 2.0 ** -11) + 2.0 ** -32 * p.amax(1, keepdim=True) * seen) @ v.abs() + y.abs() * (p * d).sum(1, keepdim=True))


@pytest.mark.parametrize("D", (64, 128))
@pytest.mark.parametrize("rows", (1, 7, 40, 90))
@pytest.mark.parametrize("length,every,bits", [(700, 16, 20.4), (3000, 16, 22.4), (3000, 0, 21.3), (9000, 0, 24.3), (2000, 16, 27.7), (130, 0, 16.2)])
def test_small_probabilities(B, length, every, bits, rows, D):
    gen = torch.Generator()
    gen.manual_seed(length + rows)
    cache, pages = some_dominate(length, every, bits, D, 32, gen)
    q = torch.zeros((rows, 1, D), dtype=F16)
    q[..., 3] = 1.0
    out = B.perq_attention_i8(q.cuda(), *cache.on_gpu(), C.ints([0, rows]), C.ints([length]), pages.cuda(), scale=1.0, out_dtype=F32)
    y, tolerance = expected(cache, pages, rows, length)
    C.compare(out[:, 0], y, tolerance)


@pytest.mark.parametrize("D", (64, 128))
def test_a_long_context_behind_a_first_token(B, D):
    """130000 keys, each 2^-22.7 of the first one's probability: 2 % of it together."""
    gen = torch.Generator()
    gen.manual_seed(D)
    cache, pages = some_dominate(130000, 0, 22.7, D, 128, gen)
    for rows in (1, 70):
        q = torch.zeros((rows, 1, D), dtype=F16)
        q[..., 3] = 1.0
        out = B.perq_attention_i8(q.cuda(), *cache.on_gpu(), C.ints([0, rows]), C.ints([130000]), pages.cuda(), scale=1.0, out_dtype=F32)
        y, tolerance = expected(cache, pages, rows, 130000)
        C.compare(out[:, 0], y, tolerance)
