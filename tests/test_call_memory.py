"""Whose memory a call's own tensors are: with a stream given, they belong to that stream and not to the current one, whose freed blocks kernels that
are still queued there may use.  On the CPU, with stand-ins for tensors, streams and the library."""
import contextlib
import types

import pytest
import torch

CURRENT, GIVEN = 0x4000, 0x5000


class Memory:
    """A contiguous tensor on device 0; `pool`: the stream that was the current one when it was made."""
    is_cuda = True

    def __init__(self, torch_, shape, dtype):
        self.torch, self.shape, self.dtype, self.pool, self.recorded = torch_, tuple(shape) if isinstance(shape, (tuple, list)) else (shape,), dtype, torch_.current, []
        torch_.made.append(self)

    device = "cuda:0"

    def get_device(self):
        return 0

    def is_contiguous(self):
        return True

    def dim(self):
        return len(self.shape)

    def numel(self):
        n = 1
        for s in self.shape:
            n *= s
        return n

    def element_size(self):
        return self.dtype.itemsize

    def data_ptr(self):
        return 0x10000

    def new_empty(self, shape, dtype):
        return Memory(self.torch, shape, dtype)

    def record_stream(self, stream):
        self.recorded.append(stream.cuda_stream)


class Torch:
    """torch with a current stream that is a number, and a list of the tensors made."""

    def __init__(self):
        self.current, self.made = CURRENT, []
        self._C = types.SimpleNamespace(_cuda_getDevice=lambda: 0, _cuda_getCurrentRawStream=lambda device: self.current)
        self.cuda = types.SimpleNamespace(stream=self.stream, ExternalStream=self.external, default_stream=lambda device=None: types.SimpleNamespace(cuda_stream=0),
                                          current_stream=lambda device=None: types.SimpleNamespace(cuda_stream=self.current))

    def __getattr__(self, name):
        return getattr(torch, name)

    def empty(self, shape, dtype=None, device=None):
        return Memory(self, shape, dtype)

    @staticmethod
    def external(handle, device=None):
        assert handle > 1, "0 makes a new stream, and 1 is not taken for a handle"
        return types.SimpleNamespace(cuda_stream=handle)

    @contextlib.contextmanager
    def stream(self, stream):
        before, self.current = self.current, stream.cuda_stream
        yield
        self.current = before


class Library:
    """Every call succeeds, but that the products want a workspace."""

    def __init__(self):
        self.streams = []

    def __getattr__(self, name):
        def call(*args):
            if name.endswith("_workspace_bytes"):
                args[-1]._obj.value = 4096
                return 0
            self.streams.append(args[-1])
            return 9 if "matmul" in name and args[-3] is None else 0
        return call


@pytest.fixture
def world(monkeypatch):
    from paper_2601_22347_b200 import binding as B
    t, lib = Torch(), Library()
    monkeypatch.setattr(B, "torch", t)
    monkeypatch.setattr(B, "_lib", lib)
    monkeypatch.setattr(B, "_rotate_quantize", lib.perq_rotate_quantize)
    monkeypatch.setattr(B, "_swiglu_rotate_quantize", lib.perq_swiglu_rotate_quantize)
    monkeypatch.setattr(B, "_rotate_quantize_i8", lib.perq_rotate_quantize_i8)
    monkeypatch.setattr(B, "_matmul_i8", lib.perq_matmul_i8)
    monkeypatch.setattr(B, "_grouped_matmul_i8", lib.perq_grouped_matmul_i8)
    return B, t, lib


CALLS = {
    "int4": lambda B, m, s: B.perq_rotate_quantize(m((8, 256), torch.bfloat16), None, 32, B.PERQ_FMT_INT4, stream=s),
    "int4_asym": lambda B, m, s: B.perq_rotate_quantize(m((8, 256), torch.bfloat16), None, 32, B.PERQ_FMT_INT4_ASYM, stream=s),
    "fp4": lambda B, m, s: B.perq_rotate_quantize(m((8, 256), torch.bfloat16), None, 32, B.PERQ_FMT_FP4, stream=s),
    "mxfp4": lambda B, m, s: B.perq_rotate_quantize(m((8, 256), torch.bfloat16), None, 32, B.PERQ_FMT_MXFP4, stream=s),
    "f32": lambda B, m, s: B.perq_rotate_quantize(m((8, 256), torch.bfloat16), None, 32, B.PERQ_FMT_F32_DEBUG, stream=s),
    "swiglu": lambda B, m, s: B.perq_swiglu_rotate_quantize(m((8, 256), torch.bfloat16), m((8, 256), torch.bfloat16), None, 32, B.PERQ_FMT_INT4, stream=s),
    "statistic": lambda B, m, s: B.perq_block_l1_stats(m((8, 256), torch.bfloat16), None, 32, stream=s),
    "diagnostics": lambda B, m, s: B.perq_token_diagnostics(m((8, 256), torch.bfloat16), None, 32, stream=s),
    "validate": lambda B, m, s: B.perq_validate_perm(m((256,), torch.int32), stream=s),
    "massdiff": lambda B, m, s: B.perq_massdiff_perm_device(m((256,), torch.float32), 32, stream=s),
    "maxima": lambda B, m, s: B.perq_chan_abs_max(m((8, 256), torch.bfloat16), stream=s),
    "int8": lambda B, m, s: B.perq_rotate_quantize_i8(m((8, 256), torch.bfloat16), None, 32, stream=s),
    "sums": lambda B, m, s: B.perq_code_sums(m((8, 256), torch.int8), B.PERQ_FMT_INT8, stream=s),
    "product": lambda B, m, s: B.perq_matmul_i8(m((8, 256), torch.int8), m((8, 1), torch.float32), B.PERQ_FMT_INT8, m((64, 256), torch.int8), m((64,), torch.float32),
                                                B.PERQ_FMT_INT8, stream=s),
    "experts": lambda B, m, s: B.perq_grouped_matmul_i8(m((8, 256), torch.int8), m((8, 1), torch.float32), B.PERQ_FMT_INT8, m((2, 64, 256), torch.int8),
                                                        m((2, 64), torch.float32), B.PERQ_FMT_INT8, m((3,), torch.int32), stream=s),
}


def tensors(results):
    return [t for t in (results if isinstance(results, tuple) else (results,)) if t is not None]


@pytest.mark.parametrize("handle", [GIVEN, 0], ids=["given", "default"])
@pytest.mark.parametrize("as_object", [False, True], ids=["number", "object"])
@pytest.mark.parametrize("name", sorted(CALLS))
def test_with_a_stream_given(world, name, as_object, handle):
    B, t, lib = world
    inputs = []

    def make(shape, dtype):
        inputs.append(Memory(t, shape, dtype))
        return inputs[-1]

    out = tensors(CALLS[name](B, make, types.SimpleNamespace(cuda_stream=handle) if as_object else handle))
    assert set(lib.streams) == {handle} and t.current == CURRENT
    own = [m for m in t.made if not any(m is i for i in inputs)]
    assert own and all(m.pool == handle for m in own)
    # what the caller gets is read on the current stream, and may be let go there before that is done
    assert all(m.recorded == [CURRENT] for m in out)


@pytest.mark.parametrize("name", sorted(CALLS))
def test_on_the_current_stream(world, name):
    B, t, lib = world
    for stream in (None, CURRENT):
        out = tensors(CALLS[name](B, lambda shape, dtype: Memory(t, shape, dtype), stream))
        assert all(m.pool == CURRENT and m.recorded == [] for m in t.made) and out
    assert set(lib.streams) == {CURRENT}


@pytest.mark.gpu
def test_blocks_let_go_on_the_current_stream_are_left_alone():
    """The current stream still has to fill blocks that were let go when calls on another stream, which does not wait for it, make their tensors."""
    import products as P
    from paper_2601_22347_b200 import binding as B, build
    build.build()
    T, N, d = 5000, 1000, 2048
    gen = torch.Generator().manual_seed(3)
    a, sa = P.random_codes(P.INT4, T, d, gen)
    w, sw = P.random_codes(P.INT4, N, d, gen)
    x = torch.randn(T, d, generator=torch.Generator(device="cuda").manual_seed(4), device="cuda").to(torch.bfloat16)
    f, space = B.PERQ_FMT_INT4, B.perq_matmul_i8_workspace_bytes(T, N, d, B.PERQ_FMT_INT4, B.PERQ_FMT_INT4)
    assert space > 0
    want = B.perq_rotate_quantize_i8(x, None, 32), B.perq_rotate_quantize(x, None, 32, f), B.perq_chan_abs_max(x)
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    torch.cuda._sleep(100_000_000)                           # (50 ms of the current stream)
    blocks = [torch.full((n,), 255, dtype=torch.uint8, device="cuda") for n in (space, T * N * 4, T * d, T * d // 2, T * 4, d * 4)]
    taken = {(t.data_ptr(), t.data_ptr() + t.numel()) for t in blocks}
    del blocks
    out = B.perq_matmul_i8(a, sa, f, w, sw, f, out_dtype=torch.float32, stream=stream)
    got = (B.perq_rotate_quantize_i8(x, None, 32, stream=stream), B.perq_rotate_quantize(x, None, 32, f, stream=stream.cuda_stream),
           B.perq_chan_abs_max(x, stream=stream))
    for t in (out, *got[0], *got[1], got[2]):
        assert all(t.data_ptr() >= end or t.data_ptr() + t.numel() * t.element_size() <= begin for begin, end in taken)
    stream.synchronize()
    result = out.clone()                                     # (on the current stream, behind its fills)
    torch.cuda.synchronize()
    P.compare(result, *P.product(P.INT4, a, sa, P.INT4, w, sw))
    for g, v in zip((*got[0], *got[1], got[2]), (*want[0], *want[1], want[2])):
        assert torch.equal(g, v)


@pytest.mark.gpu
@pytest.mark.parametrize("handle", [0, 1])
def test_the_default_stream_given_on_another_one(handle):
    """By its handles, as a number."""
    from paper_2601_22347_b200 import binding as B, build
    build.build()
    x = torch.randn(300, 2048, generator=torch.Generator(device="cuda").manual_seed(5), device="cuda").to(torch.bfloat16)
    want = B.perq_rotate_quantize_i8(x, None, 32) + B.perq_block_l1_stats(x, None, 32)
    torch.cuda.synchronize()
    with torch.cuda.stream(torch.cuda.Stream()):
        got = B.perq_rotate_quantize_i8(x, None, 32, stream=handle) + B.perq_block_l1_stats(x, None, 32, stream=handle)
        empty = B.perq_rotate_quantize_i8(x[:0], None, 32, stream=handle)
    torch.cuda.synchronize()
    assert all(torch.equal(g, w) for g, w in zip(got, want)) and empty[0].shape == (0, 2048)


@pytest.mark.gpu
def test_captured_on_a_stream_that_joined_the_capture():
    """Results and workspace of a call on a second stream of a graph, replayed."""
    import products as P
    from paper_2601_22347_b200 import binding as B, build
    build.build()
    T, N, d, f = 5000, 1000, 2048, B.PERQ_FMT_INT4
    assert B.perq_matmul_i8_workspace_bytes(T, N, d, f, f) > 0
    ops = [t for k in range(2) for t in P.random_codes(P.INT4, (T, N)[k], d, torch.Generator().manual_seed(7 + k))]
    side, fork, join = torch.cuda.Stream(), torch.cuda.Event(), torch.cuda.Event()
    B.perq_matmul_i8(ops[0], ops[1], f, ops[2], ops[3], f, out_dtype=torch.float32)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        fork.record()
        side.wait_event(fork)
        out = B.perq_matmul_i8(ops[0], ops[1], f, ops[2], ops[3], f, out_dtype=torch.float32, stream=side)
        join.record(side)
        torch.cuda.current_stream().wait_event(join)
        twice = out * 2
    for seed in (20, 30):
        for k in range(2):
            for to, new in zip(ops[2 * k:2 * k + 2], P.random_codes(P.INT4, (T, N)[k], d, torch.Generator().manual_seed(seed + k))):
                to.copy_(new)
        graph.replay()
        torch.cuda.synchronize()
        P.compare(out, *P.product(P.INT4, ops[0], ops[1], P.INT4, ops[2], ops[3]))
        assert torch.equal(twice, 2 * out)
    del graph
