"""The 8-bit cache and the attention over it in large and mixed batches: more sequences with many rows than a warp or a CTA looks at once, prompts beside decode steps."""
import math

import pytest
import torch

import cache as C
from test_attention_gpu import check, filled, queries
from test_cache_gpu import check_write

pytestmark = pytest.mark.gpu
BF16, F16 = torch.bfloat16, torch.float16


@pytest.fixture(scope="module")
def B():
    from paper_2601_22347_b200 import binding
    return binding


def some(n, low, high, seed):
    gen = torch.Generator()
    gen.manual_seed(seed)
    return [int(v) for v in torch.randint(low, high, (n,), generator=gen)]


@pytest.mark.parametrize("D,page", [(64, 64), (64, 128), (128, 64), (128, 128)])
@pytest.mark.parametrize("sequences", (33, 70))
def test_prompts_of_many_sequences(B, D, page, sequences):
    """Eight and sixteen warps to a block, found by the whole CTA; then prompts that begin inside blocks."""
    check_write(B, [some(sequences, 0, 300, page + D), some(sequences, 9, 40, page)], 1, D, page, 64, BF16, sequences)


def test_prompts_of_more_sequences_than_threads(B):
    check_write(B, [[0 if i % 3 else 20 + i % 7 for i in range(1100)]], 1, 64, 128, 16, F16, 3)


@pytest.mark.parametrize("D,page,group", [(64, 16, 1), (128, 64, 4)])
@pytest.mark.parametrize("window,sinks", [(0, 0), (40, 4)])
def test_many_rows_of_many_sequences(B, D, page, group, window, sinks):
    """Over 32 sequences the tiles come in the sequences' order; some have none, some few rows."""
    rows = some(45, 0, 2, D) + [100, 65, 300, 1, 0, 129] + some(20, 60, 90, page)
    lengths = [n + 37 * (i % 11) for i, n in enumerate(rows)]
    check(B, rows, lengths, 1, group, D, page, 16, BF16, 7, window=window, sinks=sinks)


def test_many_rows_of_more_sequences_than_a_pass(B):
    rows = [70 if i in (0, 255, 256, 300, 599) else i % 2 for i in range(600)]
    check(B, rows, [n + i % 50 for i, n in enumerate(rows)], 1, 2, 64, 16, 16, F16, 8)


@pytest.mark.parametrize("D", (64, 128))
@pytest.mark.parametrize("window,sinks", [(0, 0), (500, 4)])
def test_a_prompt_beside_decode_steps(B, D, window, sinks):
    """Both kernels of a call, keys split among CTAs in both; parts of a window's keys that a row does not see."""
    check(B, [1, 400, 1, 3, 0, 90], [6000, 4000, 20, 2500, 100, 90], 2, 4, D, 32, 32, BF16, 9, window=window, sinks=sinks)


def test_the_parts_of_a_batch_are_its_sequences(B):
    """A batch gives each sequence what a call of its own gives, up to how its keys are split."""
    gen = torch.Generator()
    gen.manual_seed(5)
    rows, lengths = [80, 1, 200], [900, 1300, 200]
    n_pages = sum(-(-n // 32) for n in lengths)
    cache = C.Cache(n_pages, 2, 32, 64, gen)
    device, pages = cache.on_gpu(), C.table(lengths, 32, n_pages, gen)
    offsets = C.starts(rows)
    k, v = (torch.randn((sum(lengths), 2, 64), generator=gen).to(BF16) for _ in range(2))
    B.perq_cache_write_i8(k.cuda(), v.cuda(), *device, C.ints(C.starts(lengths)), C.ints(lengths), pages.cuda(), b=64)
    q = torch.randn((offsets[-1], 8, 64), generator=gen).to(BF16).cuda()
    largest = float(v.abs().max()) * (1 + 0.5 / 127)
    whole = B.perq_attention_i8(q, *device, C.ints(offsets), C.ints(lengths), pages.cuda(), b=64)
    for i in range(3):
        alone = B.perq_attention_i8(q[offsets[i]:offsets[i + 1]], *device, C.ints([0, rows[i]]), C.ints([lengths[i]]), pages[i:i + 1].contiguous().cuda(), b=64)
        # two results, of values up to the largest and half a code: rounded to bf16, of probabilities off by 2^-11
        assert (whole[offsets[i]:offsets[i + 1]].float() - alone.float()).abs().max() <= 2 * largest * (2.0 ** -8 + 2.0 ** -10)


@pytest.mark.parametrize("bad", (math.nan, math.inf, -math.inf))
@pytest.mark.parametrize("D,b", [(64, 1), (64, 16), (128, 128)])
@pytest.mark.parametrize("rows,window", [(3, 0), (3, 1), (90, 0), (90, 1)])
def test_queries_that_are_not_finite(B, bad, D, b, rows, window):
    """Their rows are NaN, wherever the keys that they see lie; the others stay what they are, and what sees nothing is 0."""
    gen = torch.Generator()
    gen.manual_seed(D + rows)
    lengths = [rows + 70, rows - 2]
    cache, pages = filled(lengths, 1, D, 16, gen)
    offsets = C.starts([rows, rows])
    q = queries(2 * rows, 2, D, BF16, gen)
    hit = torch.zeros((2 * rows, 2), dtype=torch.bool)
    hit[::2, 1] = True
    hit[-1] = hit[rows] = True
    clean = q.clone()
    q[hit.nonzero()[:, 0], hit.nonzero()[:, 1], torch.randint(0, D, (int(hit.sum()),), generator=gen)] = bad
    out = B.perq_attention_i8(q.cuda(), *cache.on_gpu(), C.ints(offsets), C.ints(lengths), pages.cuda(), b=b, window=window).cpu()
    y, tolerance = C.attention(cache, clean, offsets, lengths, pages, b, D ** -0.5, window)
    C.compare(out[~hit], y[~hit], tolerance[~hit])
    unseen = torch.zeros_like(hit)
    unseen[rows:rows + 2] = True                       # (two rows more than the sequence has tokens)
    assert out[hit & ~unseen].isnan().all() and (out[unseen] == 0).all()


@pytest.mark.parametrize("rows", (1, 70))
def test_a_padded_batch(B, rows):
    """Sequences without rows before, between and behind those that have some."""
    taken = {3: 900, 40: 80, 41: 133, 300: 2000, 411: 70}
    check(B, [rows if i in taken else 0 for i in range(500)], [taken.get(i, 0) for i in range(500)], 2, 4, 64, 16, 16, BF16, 11)


@pytest.mark.parametrize("rows,group", [([9, 9, 9], 4), ([8, 8], 8), ([16, 2, 15, 14], 4), ([5, 5, 1, 5, 5], 8), ([1, 1, 1], 40)])
@pytest.mark.parametrize("D", (64, 128))
@pytest.mark.parametrize("window,sinks", [(0, 0), (200, 5)])
def test_one_kernel_for_all(B, rows, group, D, window, sinks):
    """33 to 64 rows to the longest sequence."""
    check(B, rows, [n + 113 * i * i for i, n in enumerate(rows)], 2, group, D, 32, 16, BF16, group, window=window, sinks=sinks)


@pytest.mark.parametrize("dtype", (BF16, torch.float32), ids=("bf16", "f32"))
def test_read_into_what_is_aligned_to_16_bytes(B, dtype):
    gen = torch.Generator()
    gen.manual_seed(1)
    cache, pages = filled([50, 90], 3, 64, 16, gen)
    device, tables = cache.on_gpu(), (C.ints([0, 50, 140]), C.ints([50, 90]), pages.cuda())
    k, v = B.perq_cache_read_i8(*device, *tables, T=140, b=32, out_dtype=dtype)
    room = torch.full((2, 140 * 3 * 64 + 16), 7.0, dtype=dtype).cuda()
    at = 16 // dtype.itemsize
    parts = [r[at:at + k.numel()].view(k.shape) for r in room]
    assert parts[0].data_ptr() % 32 == 16
    B.perq_cache_read_i8(*device, *tables, T=140, b=32, k=parts[0], v=parts[1])
    assert torch.equal(parts[0], k) and torch.equal(parts[1], v)
    assert (room[:, :at] == 7).all() and (room[:, at + k.numel():] == 7).all()
