"""The 8-bit layers where places in a tensor pass 31 and 32 bits: rows and channels around those places against sums in 64 bits."""
import pytest
import torch

import products as P
from products import INT4, INT8

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2601_22347_b200 import binding, build
    build.build()
    binding.load()
    return binding


@pytest.fixture(autouse=True)
def around(B):
    B.perq_device_error_clear()
    yield
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    assert B.perq_device_error() == 0


def codes(rows, bytes_, seed, dtype):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randint(0, 256, (rows, bytes_), generator=g, device="cuda", dtype=torch.uint8).view(dtype)


def scales(rows, seed):
    return torch.exp(torch.randn(rows, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda")) * 0.01


def borders(n, width):
    """Of n rows of `width` elements or bytes: the ends, and those where places pass 2^31 and 2^32."""
    rows = {0, 1, n // 2, n - 2, n - 1}
    for at in (1 << 31, 1 << 32):
        rows |= {r for r in (at // width - 1, at // width, at // width + 1) if r < n}
    return torch.tensor(sorted(rows), device="cuda")


@pytest.mark.parametrize("permuted", [False, True])
def test_rows_to_codes(B, permuted):
    T, d, b = (1 << 18) + 37, 16384, 64
    x = torch.empty(T, d, dtype=torch.bfloat16, device="cuda")
    for i in range(0, T, 1 << 16):
        x[i:i + (1 << 16)].normal_(generator=torch.Generator(device="cuda").manual_seed(i))
    perm = torch.randperm(d, generator=torch.Generator().manual_seed(3)).to(torch.int32).cuda() if permuted else None
    got, s = B.perq_rotate_quantize_i8(x, perm, b)
    rows = borders(T, d)
    want, ws = B.perq_rotate_quantize_i8(x[rows].contiguous(), perm, b)
    assert torch.equal(got[rows], want) and torch.equal(s[rows], ws)


def test_code_sums(B):
    rows, d = (1 << 17) + 5, 32768
    c = codes(rows, d, 1, torch.int8)
    at = borders(rows, d)
    assert torch.equal(B.perq_code_sums(c, B.PERQ_FMT_INT8)[at], P.code_sums(INT8, c[at]))


@pytest.mark.parametrize("T,N,d", [((1 << 20) + 300, 4099, 32), ((1 << 20) + 300, 4112, 64), ((1 << 17) + 300, 256, 32768)])
def test_results_and_tokens_behind_32_bits(B, T, N, d):
    a, w, sa, sw = codes(T, d, 2, torch.int8), codes(N, d, 3, torch.int8), scales(T, 4), scales(N, 5)
    out = B.perq_matmul_i8(a, sa, B.PERQ_FMT_INT8, w, sw, B.PERQ_FMT_INT8)
    rows = torch.unique(torch.cat((borders(T, N), borders(T, d))))
    P.compare(out[rows], *P.product(INT8, a[rows], sa[rows, None], INT8, w, sw))


def experts(B, T, E, N, d, a_fmt, w_fmt, seed):
    per = {INT8: (d, torch.int8), INT4: (d // 2, torch.uint8)}
    a, w = codes(T, per[a_fmt][0], seed, per[a_fmt][1]), codes(E * N, per[w_fmt][0], seed + 1, per[w_fmt][1])
    sa, sw = scales(T, seed + 2), scales(E * N, seed + 3)
    offsets = (torch.arange(E + 1) * T // E).to(torch.int32).cuda()
    out = B.perq_grouped_matmul_i8(a, sa, B.FMT_BY_NAME[a_fmt], w.view(E, N, -1), sw.view(E, N), B.FMT_BY_NAME[w_fmt], offsets)
    g = torch.Generator(device="cuda").manual_seed(seed + 4)
    channels = torch.unique(torch.cat((torch.arange(min(N, 200), device="cuda"), torch.arange(max(0, N - 200), N, device="cuda"),
                                       torch.randint(0, N, (500,), generator=g, device="cuda"))))
    for e in torch.unique(torch.cat((borders(E, N * d), borders(E, N * per[w_fmt][0]), borders(E, N * T // E)))).tolist():
        t0, t1 = int(offsets[e]), int(offsets[e + 1])
        rows = torch.unique(torch.tensor([t0, (t0 + t1) // 2, t1 - 1], device="cuda"))
        P.compare(out[rows][:, channels], *P.product(a_fmt, a[rows], sa[rows, None], w_fmt, w[e * N + channels], sw[e * N + channels]))


def test_few_rows_of_many_experts(B):
    """(The weights are 2^30 channels, the results 2^32.)"""
    experts(B, 4100, 1024, 1 << 20, 32, INT4, INT4, 10)


def test_many_rows_of_experts_whose_weights_are_spread(B):
    experts(B, 40 * 512, 40, 4096, 32768, INT8, INT4, 20)


def test_tokens_that_are_spread(B):
    T, N, d = (1 << 17) + 300, 512, 32768
    a, w, sa, sw = codes(T, d // 2, 30, torch.uint8), codes(N, d, 31, torch.int8), scales(T, 32), scales(N, 33)
    out = B.perq_matmul_i8(a, sa, B.PERQ_FMT_INT4, w, sw, B.PERQ_FMT_INT8)
    rows = torch.unique(torch.cat((borders(T, d), borders(T, d // 2))))
    P.compare(out[rows], *P.product(INT4, a[rows], sa[rows, None], INT8, w, sw))
