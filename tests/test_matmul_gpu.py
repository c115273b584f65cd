"""Products of codes, dense and grouped by expert, against sums in 64 bits (tests/products.py has them and the tolerance)."""
import pytest
import torch

import products as P
from products import ASYM, INT4, INT8

pytestmark = pytest.mark.gpu
FORMATS = [(INT8, INT8), (INT4, INT4), (INT8, INT4), (INT4, INT8), (ASYM, INT4), (ASYM, INT8)]
BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32


@pytest.fixture(scope="module")
def B():
    from paper_2601_22347_b200 import binding, build
    build.build()
    binding.load()
    return binding


@pytest.fixture(autouse=True)
def no_device_error(B):
    B.perq_device_error_clear()
    yield
    torch.cuda.synchronize()
    assert B.perq_device_error() == 0


def operands(a_fmt, w_fmt, T, N, d, seed, E=1):
    gen = torch.Generator().manual_seed(seed)
    a, sa = P.random_codes(a_fmt, T, d, gen)
    w, sw = P.random_codes(w_fmt, E * N, d, gen)
    return a, sa, w, sw.reshape(-1), P.code_sums(w_fmt, w) if a_fmt == ASYM else None


def dense(B, a_fmt, w_fmt, T, N, d, dtype, seed=0):
    a, sa, w, sw, cs = operands(a_fmt, w_fmt, T, N, d, 1000 * T + 10 * N + d + seed)
    out = B.perq_matmul_i8(a, sa, B.FMT_BY_NAME[a_fmt], w, sw, B.FMT_BY_NAME[w_fmt], cs, out_dtype=dtype)
    assert out.shape == (T, N) and out.dtype == dtype
    P.compare(out, *P.product(a_fmt, a, sa, w_fmt, w, sw))


# one token, one channel, the shortest rows; a k-step and a tile more or less; every number of columns; rows that end inside a
# k-step; split sums; several tiles of tokens; enough tiles that a CTA takes several
SHAPES = [(1, 1, 32), (1, 128, 256), (16, 128, 128), (17, 129, 160), (7, 130, 4096), (33, 257, 96), (64, 100, 288), (128, 128, 512), (129, 1001, 2048),
          (300, 4096, 1056), (5, 4096, 14336), (2, 70, 32768), (600, 4100, 224),
          # many tokens: ragged tiles of both sides, rows shorter than a k-step and longer than the ring, bands of tiles, several tiles to a CTA
          (1024, 256, 128), (1500, 1001, 96), (1025, 2064, 1056), (5000, 129, 32), (2600, 5000, 160)]


@pytest.mark.parametrize("a_fmt,w_fmt", FORMATS)
@pytest.mark.parametrize("T,N,d", SHAPES)
def test_dense(B, a_fmt, w_fmt, T, N, d):
    dense(B, a_fmt, w_fmt, T, N, d, F32)


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("a_fmt,w_fmt", [(INT8, INT8), (ASYM, INT4)])
@pytest.mark.parametrize("T,N,d", [(1, 1, 32), (20, 300, 512), (20, 301, 512), (150, 258, 64), (150, 4096, 64), (9, 2048, 4096), (1100, 272, 64), (1100, 280, 64), (1100, 257, 64)])
def test_result_types(B, a_fmt, w_fmt, T, N, d, dtype):
    dense(B, a_fmt, w_fmt, T, N, d, dtype)


def grouped(B, a_fmt, w_fmt, offsets, T, N, d, dtype=F32):
    E = len(offsets) - 1
    a, sa, w, sw, cs = operands(a_fmt, w_fmt, T, N, d, 77 * T + N + d + E, E)
    out = torch.full((T, N), 77.0, dtype=dtype, device="cuda")
    B.perq_grouped_matmul_i8(a, sa, B.FMT_BY_NAME[a_fmt], w.reshape(E, N, -1), sw.reshape(E, N), B.FMT_BY_NAME[w_fmt],
                             torch.tensor(offsets, dtype=torch.int32, device="cuda"), None if cs is None else cs.reshape(E, N), out=out)
    for e in range(E):
        r, c = slice(offsets[e], offsets[e + 1]), slice(e * N, (e + 1) * N)
        if offsets[e] < offsets[e + 1]:
            P.compare(out[r], *P.product(a_fmt, a[r], sa[r], w_fmt, w[c], sw[c]))
    # rows of no expert are as they were
    assert (out[:offsets[0]] == 77).all() and (out[offsets[-1]:] == 77).all()


OFFSETS = [([0, 1], 1), ([0, 0, 5, 5, 18], 20), ([3, 130, 130, 131, 400, 690], 700), ([0, 1, 10, 64], 64), ([0] * 40 + [7] * 25, 9), ([5, 5, 5], 6),
           ([0, 500, 500, 501, 502], 502), (list(range(0, 130)), 129), ([7, 7, 3000, 3001, 3001, 4000], 4005), ([0, 1, 257, 513, 2000], 2000),
           ([0, 0, 0, 0], 800), ([0, 900], 1024)]


@pytest.mark.parametrize("a_fmt,w_fmt", FORMATS)
@pytest.mark.parametrize("offsets,T", OFFSETS, ids=[str(len(o) - 1) + "x" + str(t) for o, t in OFFSETS])
def test_grouped(B, a_fmt, w_fmt, offsets, T):
    grouped(B, a_fmt, w_fmt, offsets, T, 260, 544)


@pytest.mark.parametrize("N,d", [(1, 32), (2048, 4096), (129, 32768)])
def test_grouped_widths(B, N, d):
    grouped(B, INT4, INT4, [0, 1, 10, 40], 40, N, d)


def test_many_experts(B):
    gen = torch.Generator().manual_seed(3)
    counts = torch.randint(0, 4, (1024,), generator=gen)
    grouped(B, INT8, INT8, [0] + counts.cumsum(0).tolist(), int(counts.sum()) + 3, 40, 64, BF16)


def test_bad_offsets_do_not_write_past_the_rows(B):
    """Wrong numbers, never a fault: entries outside the rows, and entries that decrease."""
    a, sa, w, sw, _ = operands(INT8, INT8, 50, 64, 128, 5, 4)
    room = torch.full((150, 64), 77.0, device="cuda")
    for bad in ([-5, 20, 10, 60, 2 ** 31 - 1], [50, 40, 30, 20, 10], [-2 ** 31, -1, 0, 200, 100], [0, 50, 0, 50, 0]):
        B.perq_grouped_matmul_i8(a, sa, B.PERQ_FMT_INT8, w.reshape(4, 64, -1), sw.reshape(4, 64), B.PERQ_FMT_INT8,
                                 torch.tensor(bad, dtype=torch.int32, device="cuda"), out=room[50:100])
        torch.cuda.synchronize()
        assert (room[:50] == 77).all() and (room[100:] == 77).all()


def test_offsets_that_go_back_and_forth_keep_their_first_rows(B):
    """An entry below an earlier one counts as that one, however many there are: no row belongs to two experts, no tile is counted twice."""
    E, T, N, d = 1024, 3000, 40, 64
    for T in (300, 90000):
        a, sa, w, sw, _ = operands(INT8, INT8, T, N, d, 6, E)
        room = torch.full((T + 200, N), 77.0, device="cuda")
        offsets = torch.tensor([0, T] * 512 + [5], dtype=torch.int32, device="cuda")
        B.perq_grouped_matmul_i8(a, sa, B.PERQ_FMT_INT8, w.reshape(E, N, -1), sw.reshape(E, N), B.PERQ_FMT_INT8, offsets, out=room[100:T + 100])
        P.compare(room[100:T + 100], *P.product(INT8, a, sa, INT8, w[:N], sw[:N]))
        assert (room[:100] == 77).all() and (room[T + 100:] == 77).all()


@pytest.mark.parametrize("T", [3, 1500, 5000])
def test_a_stream_given_to_the_call(B, T):
    """The call's own workspace outlives it on a stream that is not the current one."""
    a, sa, w, sw, cs = operands(ASYM, INT4, T, 1000, 2048, 51)
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    outs = []
    for _ in range(6):
        outs.append(B.perq_matmul_i8(a, sa, B.PERQ_FMT_INT4_ASYM, w, sw, B.PERQ_FMT_INT4, cs, out_dtype=F32, stream=stream))
        torch.full((T * 2048 + 1000 * 2048 + 4096,), 255, dtype=torch.uint8, device="cuda")      # (would take the workspace's memory)
    torch.cuda.synchronize()
    for out in outs:
        P.compare(out, *P.product(ASYM, a, sa, INT4, w, sw))


def test_results_do_not_depend_on_the_run_or_the_batch(B):
    """The sums are exact, so a row's results are the same bits alone, in a batch and grouped."""
    a, sa, w, sw, _ = operands(INT4, INT4, 300, 512, 2048, 11)
    f = B.PERQ_FMT_INT4
    full = B.perq_matmul_i8(a, sa, f, w, sw, f)
    for _ in range(3):
        assert torch.equal(B.perq_matmul_i8(a, sa, f, w, sw, f), full)
    for t in (0, 17, 299):
        assert torch.equal(B.perq_matmul_i8(a[t:t + 1].clone(), sa[t:t + 1].clone(), f, w, sw, f), full[t:t + 1])
    offsets = torch.tensor([0, 300], dtype=torch.int32, device="cuda")
    assert torch.equal(B.perq_grouped_matmul_i8(a, sa, f, w[None], sw[None], f, offsets), full)


def test_extreme_codes_reach_the_ends_of_the_range(B):
    """Rows of the lowest and highest codes: sums of 2^29 (d = 32768, both -128), and of unsigned codes 15."""
    d = 32768
    a = torch.full((2, d), -128, dtype=torch.int8, device="cuda")
    a[1] = 127
    one = torch.ones(2, 1, device="cuda")
    out = B.perq_matmul_i8(a, one, B.PERQ_FMT_INT8, a, one, B.PERQ_FMT_INT8, out_dtype=F32)
    assert out.tolist() == [[128.0 * 128 * d, -128.0 * 127 * d], [-128.0 * 127 * d, 127.0 * 127 * d]]
    p = torch.full((1, d // 2), 0xff, dtype=torch.uint8, device="cuda")              # 15 without a sign, -1 with one
    z = torch.tensor([[1.0, -3.0]], device="cuda")
    low = torch.full((1, d // 2), 0x88, dtype=torch.uint8, device="cuda")            # -8
    sums = torch.tensor([-8 * d], dtype=torch.int32, device="cuda")
    out = B.perq_matmul_i8(p, z, B.PERQ_FMT_INT4_ASYM, low, one[:1], B.PERQ_FMT_INT4, sums, out_dtype=F32)
    assert out.item() == -8.0 * d * (15 - 3)
    sums = torch.tensor([-128 * d], dtype=torch.int32, device="cuda")
    out = B.perq_matmul_i8(p, z, B.PERQ_FMT_INT4_ASYM, a[:1], one[:1], B.PERQ_FMT_INT8, sums, out_dtype=F32)
    assert out.item() == -128.0 * d * (15 - 3)


def test_scales_that_are_not_finite_stay_in_their_row_and_channel(B):
    a, sa, w, sw, _ = operands(INT8, INT8, 40, 200, 256, 9)
    sa[3, 0], sa[5, 0], sw[7] = float("nan"), float("inf"), float("nan")
    out = B.perq_matmul_i8(a, sa, B.PERQ_FMT_INT8, w, sw, B.PERQ_FMT_INT8, out_dtype=F32)
    y, acc = P.product(INT8, a, sa, INT8, w, sw)
    assert torch.equal(torch.isnan(out), torch.isnan(y)) and torch.equal(torch.isinf(out), torch.isinf(y))
    rows = [t for t in range(40) if t not in (3, 5)]
    keep = [n for n in range(200) if n != 7]
    P.compare(out[rows][:, keep], y[rows][:, keep], acc[rows][:, keep])


def test_another_stream_and_a_captured_graph(B):
    """A grouped call replayed with other offsets, tokens and weights, on another stream than the default one."""
    E, N, d, T = 4, 200, 512, 64
    a, sa, w, sw, _ = operands(INT4, INT4, T, N, d, 21, E)
    offsets = torch.tensor([0, 10, 10, 30, 64], dtype=torch.int32, device="cuda")
    out = torch.zeros(T, N, device="cuda")
    stream = torch.cuda.Stream()
    f = B.PERQ_FMT_INT4

    def call():
        B.perq_grouped_matmul_i8(a, sa, f, w.reshape(E, N, -1), sw.reshape(E, N), f, offsets, out=out)

    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        call()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            call()
        for k, at in enumerate(([0, 10, 10, 30, 64], [0, 64, 64, 64, 64], [0, 0, 1, 2, 50])):
            b, sb, v, sv, _ = operands(INT4, INT4, T, N, d, 30 + k, E)
            a.copy_(b), sa.copy_(sb), w.copy_(v), sw.copy_(sv), out.fill_(77)
            offsets.copy_(torch.tensor(at, dtype=torch.int32))
            graph.replay()
            stream.synchronize()
            for e in range(E):
                r, c = slice(at[e], at[e + 1]), slice(e * N, (e + 1) * N)
                if at[e] < at[e + 1]:
                    P.compare(out[r], *P.product(INT4, a[r], sa[r], INT4, w[c], sw[c]))
            assert (out[at[-1]:] == 77).all()
    del graph


def test_two_calls_at_once(B):
    """On two streams, with nothing between them: no call keeps anything that another uses."""
    x, y = operands(INT4, INT8, 40, 3000, 4096, 41), operands(ASYM, INT4, 700, 1000, 2048, 42)
    fx, fy = (B.PERQ_FMT_INT4, B.PERQ_FMT_INT8), (B.PERQ_FMT_INT4_ASYM, B.PERQ_FMT_INT4)
    streams = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    outs = ([], [])
    for _ in range(10):
        for k, (o, f) in enumerate(((x, fx), (y, fy))):
            with torch.cuda.stream(streams[k]):
                outs[k].append(B.perq_matmul_i8(o[0], o[1], f[0], o[2], o[3], f[1], o[4], out_dtype=F32))
    torch.cuda.synchronize()
    for k, (o, f) in enumerate(((x, (INT4, INT8)), (y, (ASYM, INT4)))):
        P.compare(outs[k][0], *P.product(f[0], o[0], o[1], f[1], o[2], o[3]))
        assert all(torch.equal(v, outs[k][0]) for v in outs[k])


@pytest.mark.parametrize("skip", [0, 16, 32, 48])
@pytest.mark.parametrize("a_fmt,w_fmt", [(INT4, INT4), (ASYM, INT8), (INT8, INT4)])
def test_a_workspace_aligned_to_16_bytes(B, a_fmt, w_fmt, skip):
    """And nothing is written outside it."""
    T, N, d = 8000, 2064, 96
    a, sa, w, sw, cs = operands(a_fmt, w_fmt, T, N, d, 77 + skip)
    af, wf = B.FMT_BY_NAME[a_fmt], B.FMT_BY_NAME[w_fmt]
    n = B.perq_matmul_i8_workspace_bytes(T, N, d, af, wf)
    assert n > 0
    room = torch.full((n + 4096,), 0xa5, dtype=torch.uint8, device="cuda")
    begin = 1024 + skip
    assert room.data_ptr() % 64 == 0
    out = B.perq_matmul_i8(a, sa, af, w, sw, wf, cs, out_dtype=F32, workspace=room[begin:begin + n])
    P.compare(out, *P.product(a_fmt, a, sa, w_fmt, w, sw))
    assert (room[:begin] == 0xa5).all() and (room[begin + n:] == 0xa5).all()


# sizes that the kernel for many tokens serves whatever the formats: ragged tiles of both sides, rows shorter than a k-step and longer than the ring, tiles
# split along k over pairs, bands of tiles, several tiles to a pair
MANY = [(1500, 1001, 9728), (1025, 1500, 8224), (5000, 2001, 2080), (8000, 2064, 160), (40000, 300, 32), (2600, 5000, 1056)]


@pytest.mark.parametrize("a_fmt,w_fmt", FORMATS)
@pytest.mark.parametrize("T,N,d", MANY)
def test_many_tokens(B, a_fmt, w_fmt, T, N, d):
    packed = (a_fmt != INT8) or (w_fmt != INT8)
    assert (B.perq_matmul_i8_workspace_bytes(T, N, d, B.FMT_BY_NAME[a_fmt], B.FMT_BY_NAME[w_fmt]) > 0) == packed
    dense(B, a_fmt, w_fmt, T, N, d, F32)


# rows on every alignment, and the last channel alone or with one, in words and between two
@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("a_fmt,w_fmt", [(INT8, INT8), (ASYM, INT4)])
@pytest.mark.parametrize("T,N,d", [(60001, n, 64) for n in (257, 258, 263, 264, 270, 271, 272, 273, 287)] + [(1531, n, 9728) for n in (1001, 1002, 1008, 1020)])
def test_many_tokens_result_types(B, a_fmt, w_fmt, T, N, d, dtype):
    if a_fmt != INT8:
        assert B.perq_matmul_i8_workspace_bytes(T, N, d, B.FMT_BY_NAME[a_fmt], B.FMT_BY_NAME[w_fmt]) > 0
    dense(B, a_fmt, w_fmt, T, N, d, dtype)


@pytest.mark.parametrize("a_fmt,w_fmt", FORMATS)
@pytest.mark.parametrize("N,d,dtype", [(260, 544, F32), (257, 96, BF16), (302, 2080, F16)])
@pytest.mark.parametrize("offsets,T", [([0, 500, 500, 2501, 2502], 3200), ([3, 1600], 1600), ([0, 0, 0, 2305], 2311), ([7, 7, 3000, 3001, 3001, 4000], 4005)],
                         ids=["4x3200", "1x1600", "3x2311", "5x4005"])
def test_many_rows_of_experts(B, a_fmt, w_fmt, offsets, T, N, d, dtype):
    packed = (a_fmt != INT8) or (w_fmt != INT8)
    assert (B.perq_grouped_matmul_i8_workspace_bytes(T, len(offsets) - 1, N, d, B.FMT_BY_NAME[a_fmt], B.FMT_BY_NAME[w_fmt]) > 0) == packed
    grouped(B, a_fmt, w_fmt, offsets, T, N, d, dtype)


def test_results_do_not_depend_on_the_kernel(B):
    """A row of a large batch has the bits that it has alone."""
    a, sa, w, sw, _ = operands(INT4, INT4, 8000, 2064, 160, 12)
    f = B.PERQ_FMT_INT4
    assert B.perq_matmul_i8_workspace_bytes(8000, 2064, 160, f, f) > 0 and B.perq_matmul_i8_workspace_bytes(7, 2064, 160, f, f) == 0
    full = B.perq_matmul_i8(a, sa, f, w, sw, f)
    for t in (0, 4000, 7993):
        assert torch.equal(B.perq_matmul_i8(a[t:t + 7].clone(), sa[t:t + 7].clone(), f, w, sw, f), full[t:t + 7])


def test_calls_of_every_kernel_at_once(B):
    """Few and many tokens, split along k and not, grouped, and the online path, each on a stream of its own with nothing between them."""
    calls, wants = [], []

    def product(a_fmt, w_fmt, T, N, d, seed):
        a, sa, w, sw, cs = operands(a_fmt, w_fmt, T, N, d, seed)
        calls.append(lambda: B.perq_matmul_i8(a, sa, B.FMT_BY_NAME[a_fmt], w, sw, B.FMT_BY_NAME[w_fmt], cs, out_dtype=F32))
        wants.append(lambda out: P.compare(out, *P.product(a_fmt, a, sa, w_fmt, w, sw)))

    product(ASYM, INT4, 8000, 2064, 160, 61)
    product(INT8, INT8, 1531, 1001, 9728, 62)
    product(INT4, INT4, 3, 4096, 4096, 63)
    product(INT8, INT4, 100, 2000, 2048, 64)
    a, sa, w, sw, _ = operands(INT4, INT8, 1000, 300, 1024, 65, 3)
    offsets = torch.tensor([0, 400, 401, 1000], dtype=torch.int32, device="cuda")
    calls.append(lambda: B.perq_grouped_matmul_i8(a, sa, B.PERQ_FMT_INT4, w.reshape(3, 300, -1), sw.reshape(3, 300), B.PERQ_FMT_INT8, offsets, out_dtype=F32))
    wants.append(lambda out: [P.compare(out[r], *P.product(INT4, a[r], sa[r], INT8, w[c], sw[c]))
                              for r, c in ((slice(0, 400), slice(0, 300)), (slice(400, 401), slice(300, 600)), (slice(401, 1000), slice(600, 900)))])
    x = torch.randn(16384, 4096, generator=torch.Generator(device="cuda").manual_seed(66), device="cuda").to(BF16)
    alone = [B.perq_rotate_quantize(x, None, 32, B.FMT_BY_NAME["mxfp4"])[0].clone(), B.perq_rotate_quantize_i8(x, None, 32)[0].clone()]
    calls += [lambda: B.perq_rotate_quantize(x, None, 32, B.FMT_BY_NAME["mxfp4"])[0], lambda: B.perq_rotate_quantize_i8(x, None, 32)[0]]
    wants += [lambda out: None, lambda out: None]
    streams = [torch.cuda.Stream() for _ in calls]
    torch.cuda.synchronize()
    outs = [[] for _ in calls]
    for _ in range(12):
        for k, call in enumerate(calls):
            with torch.cuda.stream(streams[k]):
                outs[k].append(call())
    torch.cuda.synchronize()
    for k, want in enumerate(wants):
        want(outs[k][0])
        assert all(torch.equal(v, outs[k][0]) for v in outs[k])
    assert torch.equal(outs[-2][0], alone[0]) and torch.equal(outs[-1][0], alone[1])


def test_a_captured_graph_of_many_tokens(B):
    """Two graphs, each with the workspace that its capture made, replayed in turn with other tokens and weights."""
    sizes = (5000, 1000, 2048), (1531, 1001, 9728)
    states, graphs, outs = [], [], []
    for k, (T, N, d) in enumerate(sizes):
        a, sa, w, sw, _ = operands(INT4, INT4, T, N, d, 70 + k)
        states.append((a, sa, w, sw))
        outs.append(torch.zeros(T, N, device="cuda"))

    def call(k):
        a, sa, w, sw = states[k]
        B.perq_matmul_i8(a, sa, B.PERQ_FMT_INT4, w, sw, B.PERQ_FMT_INT4, out=outs[k])

    for k in range(2):
        call(k)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            call(k)
        graphs.append(graph)
    for turn in range(3):
        for k, (T, N, d) in enumerate(sizes):
            for to, new in zip(states[k], operands(INT4, INT4, T, N, d, 80 + 2 * turn + k)):
                to.copy_(new)
            outs[k].fill_(77)
        for _ in range(3):
            for graph in graphs:
                graph.replay()
        torch.cuda.synchronize()
        for k in range(2):
            a, sa, w, sw = states[k]
            P.compare(outs[k], *P.product(INT4, a, sa, INT4, w, sw))
    del graphs
