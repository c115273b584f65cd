"""Rows to 8-bit codes against the definition in 64 bits: codes are equal, scales one rounding away; sums of codes are equal."""
import pytest
import torch

import products as P

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2601_22347_b200 import binding, build
    build.build()
    binding.load()
    return binding


def hadamard(b):
    h = torch.ones(1, 1, dtype=torch.float64)
    while h.shape[0] < b:
        h = torch.cat((torch.cat((h, h), 1), torch.cat((h, -h), 1)), 0)
    return h.cuda()


def check(B, x, perm, b):
    codes, scales = B.perq_rotate_quantize_i8(x, perm, b)
    T, d = x.shape
    y = (x if perm is None else x[:, perm.long()]).double()
    # sums of up to 512 values of 8 bits whose exponents span less than 2^36: 64-bit floats hold them exactly
    u = (y.reshape(-1, b) @ hadamard(b)).reshape(T, d)
    top = u.abs().amax(1, keepdim=True)
    want = torch.round(127 * u / torch.where(top > 0, top, 1.0)).to(torch.int8)
    assert torch.equal(codes, want), "%d codes differ" % int((codes != want).sum())
    exact = top / (127 * b ** 0.5)
    # two roundings in 64 bits of the constant and the product, then one to fp32 (below 2^-126: half its smallest step)
    assert ((scales.double() - exact).abs() <= exact * (2.0 ** -24 + 2.0 ** -51) + 2.0 ** -150).all()


def gaussian(T, d, seed, outliers=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    v = torch.randn(T, d, generator=g, device="cuda")
    if outliers:
        v[:, torch.randperm(d, generator=g, device="cuda")[:outliers]] *= 200
    return v.to(torch.bfloat16)


# one row and many, rows of one lane pair, ragged pieces and warps, every block size, one and two pieces to a lane
CASES = [(1, 32, 1), (1, 32, 32), (3, 64, 16), (5, 96, 32), (2, 512, 512), (7, 544, 32), (9, 1024, 256), (40, 2048, 128), (1, 4096, 32), (300, 4096, 64),
         (1500, 4096, 32), (17, 9728, 128), (3, 14336, 512), (2, 16384, 16), (3, 16416, 32), (3, 32768, 512), (1, 32736, 32), (700, 160, 1), (4000, 32, 16)]


@pytest.mark.parametrize("T,d,b", CASES)
@pytest.mark.parametrize("permuted", [False, True])
def test_gaussian_rows(B, T, d, b, permuted):
    perm = torch.randperm(d, generator=torch.Generator().manual_seed(d)).to(torch.int32).cuda() if permuted else None
    check(B, gaussian(T, d, T + d + b), perm, b)
    check(B, gaussian(T, d, T + d + b + 1, max(1, d // 1000)), perm, b)


@pytest.mark.parametrize("b", [1, 16, 32, 64, 128, 256, 512])
def test_rows_with_many_borders(B, b):
    """Small whole numbers: quotients lie on borders between codes, maxima are met many times."""
    g = torch.Generator(device="cuda").manual_seed(b)
    for low, high in ((-1, 2), (-2, 3), (0, 2), (-127, 128)):
        check(B, torch.randint(low, high, (64, 2048), generator=g, device="cuda").to(torch.bfloat16), None, b)
    # every other code is a border: maxima 254, odd numbers
    odd = 2 * torch.randint(-126, 126, (64, 2048), generator=g, device="cuda") + 1
    odd[:, 0] = 254
    check(B, odd.to(torch.bfloat16), None, 1)


@pytest.mark.parametrize("b", [1, 16, 128, 512])
def test_special_rows(B, b):
    d = 1024
    x = torch.zeros(12, d)
    x[1, 5] = 3.0                                     # one channel
    x[2] = 7.0                                        # equal channels
    x[3] = torch.arange(d) % 2 * 2.0 - 1              # all but one output of a block cancel
    x[4, :512], x[4, 512:] = 1e-3, 1.0                # a small block beside a large one
    x[5] = torch.randn(d, generator=torch.Generator().manual_seed(b)) * 2.0 ** -133      # subnormal
    x[6, 0] = 2.0 ** -133                             # the smallest number
    x[7, 9] = 2.0 ** 118                              # sqrt(b) |y| = 2^118
    x[8] = -2.0 ** 110
    x[9] = torch.randn(d, generator=torch.Generator().manual_seed(b + 1)) * 2.0 ** -120
    x[10, 1::2] = -0.0
    x[11] = torch.where(torch.arange(d) == 3, 1.0, 2.0 ** -17)
    check(B, x.to(torch.bfloat16).cuda(), None, b)


def test_wide_ranges_in_a_block(B):
    """Exponents spread over 28 binades in every block: sums round in fp32, codes do not."""
    g = torch.Generator(device="cuda").manual_seed(5)
    x = torch.randn(200, 2048, generator=g, device="cuda") * torch.exp2(torch.randint(-14, 14, (200, 2048), generator=g, device="cuda").float())
    for b in (16, 64, 512):
        check(B, x.to(torch.bfloat16), None, b)


def test_values_that_are_not_finite_do_not_fault(B):
    x = gaussian(6, 2048, 1)
    x[0, 3], x[1, 4], x[2, 5], x[3] = float("nan"), float("inf"), -float("inf"), float("nan")
    codes, scales = B.perq_rotate_quantize_i8(x, None, 64)
    torch.cuda.synchronize()
    want, s = B.perq_rotate_quantize_i8(x[4:].clone(), None, 64)
    assert torch.equal(codes[4:], want) and torch.equal(scales[4:], s)


def test_bad_permutations_are_clamped(B):
    x = gaussian(3, 512, 2)
    perm = torch.full((512,), 2 ** 31 - 1, dtype=torch.int32, device="cuda")
    perm[::2] = -7
    check(B, x, perm.clamp(0, 511), 1)
    a, b = B.perq_rotate_quantize_i8(x, perm, 1), B.perq_rotate_quantize_i8(x, perm.clamp(0, 511), 1)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_captured_on_another_stream(B):
    x, stream = gaussian(100, 4096, 1), torch.cuda.Stream()
    codes, scales = torch.empty(100, 4096, dtype=torch.int8, device="cuda"), torch.empty(100, device="cuda")
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        B.perq_rotate_quantize_i8(x, None, 32, codes, scales)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            B.perq_rotate_quantize_i8(x, None, 32, codes, scales)
        for seed in (2, 3):
            x.copy_(gaussian(100, 4096, seed))
            graph.replay()
            stream.synchronize()
            want = B.perq_rotate_quantize_i8(x, None, 32)
            assert torch.equal(codes, want[0]) and torch.equal(scales, want[1].flatten())
    del graph


@pytest.mark.parametrize("rows,d", [(1, 32), (7, 96), (100, 4096), (3, 32768), (5000, 64)])
def test_code_sums(B, rows, d):
    gen = torch.Generator().manual_seed(rows + d)
    for fmt in (P.INT8, P.INT4):
        codes, _ = P.random_codes(fmt, rows, d, gen)
        assert torch.equal(B.perq_code_sums(codes, B.FMT_BY_NAME[fmt]), P.code_sums(fmt, codes))
    low = torch.full((2, d), -128, dtype=torch.int8, device="cuda")
    assert B.perq_code_sums(low, B.PERQ_FMT_INT8).tolist() == [-128 * d] * 2
    assert B.perq_code_sums(torch.full((2, d // 2), 0x88, dtype=torch.uint8, device="cuda"), B.PERQ_FMT_INT4).tolist() == [-8 * d] * 2
