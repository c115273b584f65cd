"""The calls on the cache as a program makes them: a prompt and decode steps behind it, between the 8-bit linear layers, captured and replayed, on other streams, at places past 32 bits."""
import math

import pytest
import torch

import cache as C
from test_attention_gpu import filled, queries
from test_cache_gpu import tokens

pytestmark = pytest.mark.gpu
BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32


@pytest.fixture(scope="module")
def B():
    from paper_2601_22347_b200 import binding
    return binding


def near(out, cache, q, offsets, lengths, pages, b, D, **kw):
    y, tolerance = C.attention(cache, q, offsets, lengths, pages, b, D ** -0.5, **kw)
    there = slice(offsets[0], offsets[-1])
    C.compare(out[there], y[there], tolerance[there])


@pytest.mark.parametrize("D,page,b,heads,group", [(128, 32, 128, 2, 4), (64, 16, 16, 3, 2)])
def test_a_prompt_and_steps_behind_it(B, D, page, b, heads, group):
    """What is written by a call is what the next one attends to: a ragged prefill, single tokens, a few drafted ones that are taken back, and others in their place."""
    gen = torch.Generator()
    gen.manual_seed(D)
    prompt, most = [page * 3 + 5, 7, 90], 40
    n_pages = sum(-(-(n + most) // page) for n in prompt)
    pages = C.table([n + most for n in prompt], page, n_pages, gen)
    cache = C.Cache(n_pages, heads, page, D, gen)
    device, table = cache.on_gpu(), pages.cuda()
    lengths = [0] * 3
    for rows in (prompt, [1, 1, 1], [1, 0, 1], [5, 5, 5], [-3, -3, -3], [2, 1, 2], [1, 1, 1]):
        if rows[0] < 0:                                # tokens are taken back: their places are written again
            lengths = [l + n for l, n in zip(lengths, rows)]
            continue
        lengths = [l + n for l, n in zip(lengths, rows)]
        offsets = C.starts(rows)
        qkv = tokens(offsets[-1], heads * (group + 2), D, BF16, gen)
        q, k, v = qkv[:, :heads * group], qkv[:, heads * group:heads * (group + 1)], qkv[:, heads * (group + 1):]
        on, at, n = qkv.cuda(), C.ints(offsets), C.ints(lengths)
        B.perq_cache_write_i8(on[:, heads * group:heads * (group + 1)], on[:, heads * (group + 1):], *device, at, n, table, b=b)
        cache.write(k, v, offsets, lengths, pages, b)
        for got, want in zip(device, (cache.codes[0], cache.steps[0], cache.codes[1], cache.steps[1])):
            assert torch.equal(got.cpu(), want)
        out = B.perq_attention_i8(on[:, :heads * group], *device, at, n, table, most=max(rows), b=b)
        near(out, cache, q, offsets, lengths, pages, b, D)


def test_between_linear_layers(B):
    """Hidden states to 8-bit codes, one product to queries, keys and values side by side, the cache, attention, codes again and the product behind it: each stage
    is what its definition makes of what the one before it returned."""
    gen = torch.Generator()
    gen.manual_seed(5)
    T, hidden, heads, group, D, page, b = 150, 512, 2, 2, 64, 16, 64
    wide = (heads * (group + 2)) * D
    x = torch.randn((T, hidden), generator=gen).to(BF16).cuda()
    w, w_out = (torch.randn(shape, generator=gen).to(BF16).cuda() * 0.05 for shape in ((wide, hidden), (hidden, heads * group * D)))
    codes, scales = B.perq_rotate_quantize_i8(x, None, 32)
    w_codes, w_scales = B.perq_rotate_quantize_i8(w, None, 32)
    row = B.perq_matmul_i8(codes, scales, B.PERQ_FMT_INT8, w_codes, w_scales, B.PERQ_FMT_INT8).reshape(T, heads * (group + 2), D)
    y = x.double() @ w.double().T
    assert (row.reshape(T, -1).double() - y).norm() <= 0.02 * y.norm()
    q, k, v = row[:, :heads * group], row[:, heads * group:heads * (group + 1)], row[:, heads * (group + 1):]
    lengths, offsets = [100, 50], [0, 100, 150]
    pages = C.table(lengths, page, 12, gen)
    cache = C.Cache(12, heads, page, D, gen)
    device, args = cache.on_gpu(), (C.ints(offsets), C.ints(lengths), pages.cuda())
    B.perq_cache_write_i8(k, v, *device, *args, b=b)
    cache.write(k.cpu(), v.cpu(), offsets, lengths, pages, b)
    out = B.perq_attention_i8(q, *device, *args, b=b)
    near(out, cache, q.cpu(), offsets, lengths, pages, b, D)
    codes, scales = B.perq_rotate_quantize_i8(out.reshape(T, -1), None, 32)
    w_codes, w_scales = B.perq_rotate_quantize_i8(w_out, None, 32)
    last = B.perq_matmul_i8(codes, scales, B.PERQ_FMT_INT8, w_codes, w_scales, B.PERQ_FMT_INT8)
    y = out.reshape(T, -1).double() @ w_out.double().T
    assert (last.double() - y).norm() <= 0.02 * y.norm()


@pytest.mark.parametrize("rows,lengths", [([1, 1, 1], [700, 30, 2000]), ([200, 3, 100], [900, 40, 100]), ([300], [5000])])
def test_the_same_bits_again(B, rows, lengths):
    gen = torch.Generator()
    gen.manual_seed(1)
    cache, pages = filled(lengths, 2, 64, 16, gen)
    offsets = C.starts(rows)
    q, device, args = queries(offsets[-1], 8, 64, BF16, gen).cuda(), cache.on_gpu(), (C.ints(offsets), C.ints(lengths), pages.cuda())
    first = B.perq_attention_i8(q, *device, *args, b=16, out_dtype=F32)
    for _ in range(20):
        assert torch.equal(B.perq_attention_i8(q, *device, *args, b=16, out_dtype=F32), first)


def test_captured_and_replayed_with_other_sequences(B):
    """A step of writing and attending, captured once; what the sequences are changes between replays, and two such graphs have one workspace in turn."""
    gen = torch.Generator()
    gen.manual_seed(2)
    heads, group, D, page, b, S, T = 2, 4, 64, 16, 16, 4, 160
    n_pages, width = 120, 30
    cache = C.Cache(n_pages, heads, page, D, gen)
    pages = torch.randperm(n_pages, generator=gen)[:S * width].reshape(S, width).to(torch.int32)
    device, table = cache.on_gpu(), pages.cuda()
    offsets, lengths = C.ints([0] * (S + 1)), C.ints([0] * S)
    row = torch.zeros((T, heads * (group + 2), D), dtype=BF16).cuda()
    q, k, v = row[:, :heads * group], row[:, heads * group:heads * (group + 1)], row[:, heads * (group + 1):]
    outs = [torch.zeros((T, heads * group, D), dtype=BF16).cuda() for _ in range(2)]
    space = torch.zeros(B.perq_attention_i8_workspace_bytes(T, S, heads, group, D, T), dtype=torch.uint8).cuda()

    def step(out, window):
        B.perq_cache_write_i8(k, v, *device, offsets, lengths, table, b=b)
        B.perq_attention_i8(q, *device, offsets, lengths, table, most=T, b=b, window=window, sinks=3 if window else 0, out=out, workspace=space)

    graphs = []
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for i in range(2):
            step(outs[i], 50 * i)
    torch.cuda.current_stream().wait_stream(side)
    for i in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            step(outs[i], 50 * i)
        graphs.append(g)
    held = [0] * S
    for turn, rows in enumerate(([70, 1, 0, 33], [1, 1, 1, 1], [0, 80, 1, 20], [1, 2, 3, 4])):
        held = [h + n for h, n in zip(held, rows)]
        at = C.starts(rows)
        x = tokens(at[-1], heads * (group + 2), D, BF16, gen)
        row[:at[-1]] = x.cuda()
        offsets.copy_(torch.tensor(at, dtype=torch.int32))
        lengths.copy_(torch.tensor(held, dtype=torch.int32))
        graphs[turn % 2].replay()
        cache.write(x[:, heads * group:heads * (group + 1)], x[:, heads * (group + 1):], at, held, pages, b)
        near(outs[turn % 2], cache, x[:, :heads * group], at, held, pages, b, D, **({"window": 50, "sinks": 3} if turn % 2 else {}))


def test_two_streams_at_once(B):
    """Calls that overlap, each on its stream with a workspace of its own (made here by one, given to the other)."""
    gen = torch.Generator()
    gen.manual_seed(3)
    jobs = []
    for rows, lengths, given in (([1, 1], [3000, 100], True), ([150, 70], [400, 70], False)):
        cache, pages = filled(lengths, 2, 128, 32, gen)
        offsets = C.starts(rows)
        q = queries(offsets[-1], 8, 128, BF16, gen)
        stream = torch.cuda.Stream()
        jobs.append((cache, q, offsets, lengths, pages, stream, given, (q.cuda(), *cache.on_gpu(), C.ints(offsets), C.ints(lengths), pages.cuda())))
    torch.cuda.synchronize()
    for _ in range(5):
        outs = []
        for cache, q, offsets, lengths, pages, stream, given, args in jobs:
            if given:
                space = torch.empty(B.perq_attention_i8_workspace_bytes(offsets[-1], 2, 2, 4, 128, offsets[-1]), dtype=torch.uint8, device="cuda")
                out = torch.empty(args[0].shape, dtype=BF16, device="cuda")
                stream.wait_stream(torch.cuda.current_stream())
                B.perq_attention_i8(*args, b=128, out=out, workspace=space, stream=stream)
                space.record_stream(stream)
            else:
                with torch.cuda.stream(stream):
                    out = B.perq_attention_i8(*args, b=128)
            outs.append(out)
        torch.cuda.synchronize()
        for out, (cache, q, offsets, lengths, pages, *_) in zip(outs, jobs):
            near(out, cache, q, offsets, lengths, pages, 128, 128)


def test_a_stream_by_its_handle(B):
    """Tensors that a call makes are the given stream's memory; the caller's stream waits before it reads them."""
    gen = torch.Generator()
    gen.manual_seed(4)
    cache, pages = filled([60], 2, 64, 16, gen)
    q = queries(2, 4, 64, BF16, gen)
    args = (C.ints([0, 2]), C.ints([60]), pages.cuda())
    device, on = cache.on_gpu(), q.cuda()
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    out = B.perq_attention_i8(on, *device, *args, b=16, stream=stream.cuda_stream)
    k, v = B.perq_cache_read_i8(*device, *args, 2, b=16, out_dtype=F32, stream=stream)
    torch.cuda.current_stream().wait_stream(stream)
    near(out, cache, q, [0, 2], [60], pages, 16, 64)
    y = cache.tokens(1, 0, 60, pages)[58:]
    assert (v.cpu().double() - y).abs().max() <= 1e-6 * y.abs().max()
    assert (k.cpu().double() - C.rotated(cache.tokens(0, 0, 60, pages)[58:], 16)).abs().max() <= 1e-6 * k.abs().max().cpu()


def test_places_past_32_bits(B):
    """Pages whose codes lie more than 2^32 bytes into the pool: written, read back and attended to by one row and by many."""
    gen = torch.Generator()
    gen.manual_seed(6)
    heads, page, D, b, n = 8, 128, 128, 32, 300
    n_pages = (1 << 32) // (heads * page * D) + 9
    device = tuple(torch.zeros(shape, dtype=t, device="cuda") for shape, t in (((n_pages, heads, page, D), torch.int8), ((n_pages, heads), F32)) * 2)
    high = [n_pages - 1, n_pages - 8, n_pages - 3]
    pages = torch.tensor([high], dtype=torch.int32)
    k, v, q = (tokens(n, heads, D, BF16, gen) for _ in range(3))
    args = (C.ints([0, n]), C.ints([n]), pages.cuda())
    B.perq_cache_write_i8(k.cuda(), v.cuda(), *device, *args, b=b)
    cache = C.Cache(3, heads, page, D, gen)
    low = torch.tensor([[0, 1, 2]], dtype=torch.int32)
    cache.write(k, v, [0, n], [n], low, b)
    there = torch.arange(page)[None, None, :, None] + torch.arange(3)[:, None, None, None] * page < n
    for kind in range(2):
        got, steps = device[2 * kind][high].cpu(), device[2 * kind + 1][high].cpu()
        assert torch.equal(torch.where(there, got, 0), torch.where(there, cache.codes[kind], 0)) and torch.equal(steps, cache.steps[kind])
    out = B.perq_attention_i8(q.cuda(), *device, *args, b=b)
    near(out, cache, q, [0, n], [n], low, b, D)
    one = B.perq_attention_i8(q[-1:].contiguous().cuda(), *device, C.ints([0, 1]), args[1], args[2], b=b)
    near(one, cache, q[-1:], [0, 1], [n], low, b, D)
    _, back = B.perq_cache_read_i8(*device, *args, n, b=b, out_dtype=F32)
    y = cache.tokens(1, 0, n, low)
    assert (back.cpu().double() - y).abs().max() <= 1e-6 * y.abs().max()


def test_shared_pages_that_are_only_read(B):
    """Two sequences behind the same prefix."""
    gen = torch.Generator()
    gen.manual_seed(7)
    cache, pages = filled([64 + 20, 0], 2, 64, 32, gen, spare=2)
    both = torch.tensor([[pages[0, 0], pages[0, 1], pages[0, 2]], [pages[0, 0], pages[0, 1], (set(range(cache.n_pages)) - set(pages[0].tolist())).pop()]], dtype=torch.int32)
    q = queries(12, 4, 64, BF16, gen)
    for rows in ([1, 1], [5, 7]):
        offsets = C.starts(rows)
        out = B.perq_attention_i8(q[:offsets[-1]].cuda(), *cache.on_gpu(), C.ints(offsets), C.ints([84, 70]), both.cuda(), b=64)
        near(out, cache, q[:offsets[-1]], offsets, [84, 70], both, 64, 64)


def test_tensors_the_call_refuses(B):
    gen = torch.Generator()
    gen.manual_seed(8)
    cache, pages = filled([40], 2, 64, 16, gen)
    device, args = cache.on_gpu(), (C.ints([0, 3]), C.ints([40]), pages.cuda())
    q = queries(3, 4, 64, BF16, gen).cuda()
    k = q[:, :2].contiguous()
    bad_caches = [(device[0].cpu(),) + device[1:], (device[0].to(torch.int32),) + device[1:], (device[0], device[1].double()) + device[2:], device[:2] + (device[2][:-1], device[3]),
                  (device[0].transpose(1, 2),) + device[1:]]
    for bad in bad_caches:
        with pytest.raises((AssertionError, RuntimeError)):
            B.perq_attention_i8(q, *bad, *args)
        with pytest.raises((AssertionError, RuntimeError)):
            B.perq_cache_write_i8(k, k, *bad, *args)
        with pytest.raises((AssertionError, RuntimeError)):
            B.perq_cache_read_i8(*bad, *args, 3)
    for bad in ((args[0].long(), args[1], args[2]), (args[0], C.ints([40, 40]), args[2]), (args[0], args[1], args[2].cpu())):
        with pytest.raises((AssertionError, RuntimeError)):
            B.perq_attention_i8(q, *device, *bad)
    for bad in (q.float(), q[:, :3], q[..., :32], q.cpu(), q.transpose(0, 1)):
        with pytest.raises((AssertionError, RuntimeError)):
            B.perq_attention_i8(bad, *device, *args)
    for bad in (q, k.float(), k[:, :1], k[..., ::2]):
        with pytest.raises((AssertionError, RuntimeError)):
            B.perq_cache_write_i8(bad, bad, *device, *args)
    with pytest.raises(B.PerqError):
        B.perq_attention_i8(q, *device, *args, b=24)
    with pytest.raises(B.PerqError):
        B.perq_attention_i8(q, *device, *args, workspace=torch.empty(16, dtype=torch.uint8, device="cuda"))
    with pytest.raises(B.PerqError):
        B.perq_attention_i8(q, *device, *args, window=-1)
    odd = torch.empty(3 * 6 * 64 + 4, dtype=BF16, device="cuda")[4:].reshape(3, 6, 64)
    with pytest.raises(B.PerqError):
        B.perq_cache_write_i8(odd[:, :2], odd[:, 2:4], *device, *args)
