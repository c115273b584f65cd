"""The entry points of a quantised feedforward block one after another, as they would be used: weights rotated, quantised and summed once, tokens
rotated and quantised in each of the formats, the products, dense and grouped by expert, on one stream with nothing between them."""
import pytest
import torch

import products as P
from products import ASYM, INT4, INT8

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2601_22347_b200 import binding, build
    build.build()
    binding.load()
    return binding


def rows(B, fmt, x, b, perm=None):
    if fmt == INT8:
        return B.perq_rotate_quantize_i8(x, perm, b)
    return B.perq_rotate_quantize(x, perm, b, B.FMT_BY_NAME[fmt])


def normal(shape, seed, scale=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (scale * torch.randn(*shape, generator=g, device="cuda")).to(torch.bfloat16)


def step(a_fmt, d):
    """Largest relative error of a row's values: half a step of 1/7, 1/15 of twice, or 1/127 of its maximum, against a gaussian row's norm."""
    most = 5.5                        # sigma of the largest of 2^14 values, at most
    return {INT4: most / 14, ASYM: most / 15, INT8: most / 254}[a_fmt]


@pytest.mark.parametrize("T", [1, 40, 1300])
@pytest.mark.parametrize("a_fmt,w_fmt", [(INT4, INT4), (ASYM, INT4), (INT8, INT8), (INT8, INT4), (ASYM, INT8)])
def test_a_down_projection(B, a_fmt, w_fmt, T):
    """(X P R)(W P R)^T is X W^T but for what the codes lose; the product itself is exact for these codes."""
    N, d, b = 768, 2048, 32
    x, w = normal((T, d), T), normal((N, d), 3, 0.02)
    perm = torch.randperm(d, generator=torch.Generator().manual_seed(9)).to(torch.int32).cuda()
    w_codes, w_scales = rows(B, w_fmt, w, b, perm)
    w_sums = B.perq_code_sums(w_codes, B.FMT_BY_NAME[w_fmt])
    codes, scales = rows(B, a_fmt, x, b, perm)
    out = B.perq_matmul_i8(codes, scales, B.FMT_BY_NAME[a_fmt], w_codes, w_scales, B.FMT_BY_NAME[w_fmt], w_sums)
    y, acc = P.product(a_fmt, codes, scales, w_fmt, w_codes, w_scales)
    P.compare(out, y, acc)
    # the layer without codes: errors of rows and channels, uniform in a step of their own, add up like norms; six of their standard deviations
    plain = x.double() @ w.double().t()
    sigma = 0.02 * d ** 0.5 * ((step(a_fmt, d) ** 2 + step(w_fmt, d) ** 2) / 3) ** 0.5
    assert (out.double() - plain).abs().max() < 6 * sigma + plain.abs().max() * 2 ** -8


def test_experts(B):
    """Rows sorted by expert, a buffer with rows to spare; weights of all experts quantised in one call."""
    E, N, d, b, T = 6, 320, 1024, 64, 500
    counts = torch.tensor([0, 100, 3, 0, 257, 128])
    offsets = torch.cat((torch.zeros(1, dtype=torch.int64), counts.cumsum(0))).to(torch.int32)
    x, w = normal((T, d), 1), normal((E * N, d), 2, 0.05)
    for a_fmt, w_fmt in ((INT4, INT4), (ASYM, INT4), (INT8, INT8)):
        w_codes, w_scales = rows(B, w_fmt, w, b)
        sums = B.perq_code_sums(w_codes.reshape(E, N, -1), B.FMT_BY_NAME[w_fmt])
        codes, scales = rows(B, a_fmt, x, b)
        out = torch.full((T, N), 5.0, dtype=torch.float16, device="cuda")
        B.perq_grouped_matmul_i8(codes, scales, B.FMT_BY_NAME[a_fmt], w_codes.reshape(E, N, -1), w_scales, B.FMT_BY_NAME[w_fmt], offsets.cuda(), sums, out=out)
        assert sums.shape == (E, N)
        at = offsets.tolist()
        for e in range(E):
            r, c = slice(at[e], at[e + 1]), slice(e * N, (e + 1) * N)
            if at[e] < at[e + 1]:
                P.compare(out[r], *P.product(a_fmt, codes[r], scales[r], w_fmt, w_codes[c], w_scales[c]))
        assert (out[at[-1]:] == 5).all()


def test_a_captured_layer(B):
    """Quantisation and product in one graph, replayed on new tokens: what the first kernel writes the second one reads."""
    N, d, b = 1024, 4096, 32
    for T in (4, 700):
        w = normal((N, d), 5, 0.02)
        w_codes, w_scales = rows(B, INT4, w, b)
        x = normal((T, d), 6)
        codes, scales = torch.empty(T, d // 2, dtype=torch.uint8, device="cuda"), torch.empty(T, 1, device="cuda")
        out = torch.empty(T, N, device="cuda")
        space = torch.empty(max(16, B.perq_matmul_i8_workspace_bytes(T, N, d, B.PERQ_FMT_INT4, B.PERQ_FMT_INT4)), dtype=torch.uint8, device="cuda")

        def layer():
            B.perq_rotate_quantize(x, None, b, B.PERQ_FMT_INT4, 0, codes, scales)
            B.perq_matmul_i8(codes, scales, B.PERQ_FMT_INT4, w_codes, w_scales, B.PERQ_FMT_INT4, out=out, workspace=space)

        stream = torch.cuda.Stream()
        stream.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(stream):
            layer()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=stream):
                layer()
            for seed in (7, 8, 9):
                x.copy_(normal((T, d), seed))
                graph.replay()
                stream.synchronize()
                c, s = B.perq_rotate_quantize(x, None, b, B.PERQ_FMT_INT4)
                P.compare(out, *P.product(INT4, c, s, INT4, w_codes, w_scales))
        del graph
