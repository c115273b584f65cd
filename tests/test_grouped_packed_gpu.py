"""Grouped products of packed codes with many rows to an expert: operands are spread to bytes before the product, for the experts that have rows, which
two kernels find out each for itself from the offsets on the device."""
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


def operands(a_fmt, w_fmt, T, E, N, d, seed):
    gen = torch.Generator().manual_seed(seed)
    a, sa = P.random_codes(a_fmt, T, d, gen)
    w, sw = P.random_codes(w_fmt, E * N, d, gen)
    return a, sa, w, sw.reshape(-1), P.code_sums(w_fmt, w)


def call(B, a_fmt, w_fmt, E, N, ops, offsets, out, workspace=None):
    a, sa, w, sw, cs = ops
    B.perq_grouped_matmul_i8(a, sa, B.FMT_BY_NAME[a_fmt], w.reshape(E, N, -1), sw.reshape(E, N), B.FMT_BY_NAME[w_fmt], offsets, cs.reshape(E, N), out=out,
                             workspace=workspace)


def compare(a_fmt, w_fmt, T, N, ops, settled, out):
    """settled: offsets that do not decrease and lie in 0 .. T."""
    a, sa, w, sw, _ = ops
    for e in range(len(settled) - 1):
        r, c = slice(settled[e], settled[e + 1]), slice(e * N, (e + 1) * N)
        if settled[e] < settled[e + 1]:
            P.compare(out[r], *P.product(a_fmt, a[r], sa[r], w_fmt, w[c], sw[c]))
    assert (out[:settled[0]] == 77).all() and (out[settled[-1]:] == 77).all()


@pytest.mark.parametrize("a_fmt,w_fmt", [(INT4, INT4), (ASYM, INT4), (INT8, INT4), (INT4, INT8)])
def test_a_captured_call_replayed_with_other_experts(B, a_fmt, w_fmt):
    """Experts that were empty get rows and the others lose them; the workspace holds what earlier replays spread."""
    E, N, d, T = 4, 260, 544, 4000
    ops = operands(a_fmt, w_fmt, T, E, N, d, 1)
    offsets = torch.tensor([0, T, T, T, T], dtype=torch.int32, device="cuda")
    out = torch.zeros(T, N, device="cuda")
    space = torch.full((B.perq_grouped_matmul_i8_workspace_bytes(T, E, N, d, B.FMT_BY_NAME[a_fmt], B.FMT_BY_NAME[w_fmt]),), 0x5a, dtype=torch.uint8, device="cuda")
    assert space.numel() > 0
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        call(B, a_fmt, w_fmt, E, N, ops, offsets, out, space)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            call(B, a_fmt, w_fmt, E, N, ops, offsets, out, space)
        for k, at in enumerate(([0, T, T, T, T], [0, 0, 0, 0, T], [0, 1, 2000, 2000, 3999], [5, 5, 5, 2005, 2006], [7, 7, 7, 7, 7], [0, 1000, 2000, 3000, 4000])):
            for to, new in zip(ops, operands(a_fmt, w_fmt, T, E, N, d, 10 + k)):
                to.copy_(new)
            out.fill_(77)
            offsets.copy_(torch.tensor(at, dtype=torch.int32))
            graph.replay()
            stream.synchronize()
            compare(a_fmt, w_fmt, T, N, ops, at, out)
    del graph


@pytest.mark.parametrize("a_fmt,w_fmt", [(INT4, INT4), (ASYM, INT4), (INT8, INT4), (INT4, INT8)])
@pytest.mark.parametrize("bad", [[0, 3000, 100, 3500, 200], [-5, 2000, 1000, 2 ** 31 - 1, 0], [4000, 0, 4000, 0, 4000], [2000, 1000, 2500, -2 ** 31, 2600], [9, 4, 9, 8, 9]])
def test_offsets_that_decrease(B, a_fmt, w_fmt, bad):
    """An entry below an earlier one counts as that one, one outside the rows as their end; nothing else is written."""
    E, N, d, T = 4, 200, 288, 4000
    ops = operands(a_fmt, w_fmt, T, E, N, d, 2)
    assert B.perq_grouped_matmul_i8_workspace_bytes(T, E, N, d, B.FMT_BY_NAME[a_fmt], B.FMT_BY_NAME[w_fmt]) > 0
    room = torch.full((T + 600, N), 77.0, device="cuda")
    settled = []
    for v in bad:
        settled.append(max([min(max(v, 0), T)] + settled[-1:]))
    # (workspace of 0xff: what is not spread and read all the same is not what it should be)
    space = torch.full((B.perq_grouped_matmul_i8_workspace_bytes(T, E, N, d, B.FMT_BY_NAME[a_fmt], B.FMT_BY_NAME[w_fmt]),), 0xff, dtype=torch.uint8, device="cuda")
    call(B, a_fmt, w_fmt, E, N, ops, torch.tensor(bad, dtype=torch.int32, device="cuda"), room[300:T + 300], space)
    assert (room[:300] == 77).all() and (room[T + 300:] == 77).all()
    compare(a_fmt, w_fmt, T, N, ops, settled, room[300:T + 300])
