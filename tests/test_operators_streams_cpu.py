"""The conveniences around the layer on an explicit stream: which stream owns the memory that
they allocate, on the host (no GPU, the library's calls replaced)."""
import contextlib

import pytest

torch = pytest.importorskip("torch")
sa = pytest.importorskip("paper_2406_05981_amd.shiftadd",
                         reason="libshiftadd.so not built (python -m paper_2406_05981_amd.build)")

CALLER, SIDE = 100, 7


class Stream:
    def __init__(self, handle):
        self.cuda_stream = handle


class Tensor(torch.Tensor):
    """A host tensor that notes which streams it is recorded on."""

    def record_stream(self, stream):
        self.recorded = getattr(self, "recorded", []) + [stream.cuda_stream]

    def cpu(self):
        World.read_on.append(torch.cuda.current_stream().cuda_stream)
        return self.zero_()


class World:
    read_on = []   # stream of every copy to the host

    def __init__(self, monkeypatch):
        World.read_on.clear()
        self.current = Stream(CALLER)
        self.allocated = []   # stream of every allocation
        self.calls = []       # stream of every library call
        empty = torch.empty

        @contextlib.contextmanager
        def on(stream):
            before, self.current = self.current, stream
            try:
                yield
            finally:
                self.current = before

        def new(*args, **kw):
            self.allocated.append(self.current.cuda_stream)
            return empty(*args, **kw).as_subclass(Tensor)

        def call(*args):
            self.calls.append(args[-1])
            return 0

        monkeypatch.setattr(torch.cuda, "current_stream", lambda *a: self.current)
        monkeypatch.setattr(torch.cuda, "stream", on)
        monkeypatch.setattr(torch.cuda, "ExternalStream", Stream)
        monkeypatch.setattr(torch, "empty", new)
        monkeypatch.setattr(sa, "_raw_stream", None)
        monkeypatch.setattr(sa, "_dev", lambda t, *a, **kw: t.data_ptr())
        monkeypatch.setattr(sa, "_here", lambda: None)
        for name in self.LIBRARY:
            monkeypatch.setattr(sa.lib, name, call)

    LIBRARY = ("sa_shiftadd_gemm_epilogue", "sa_shiftadd_gemm_experts", "sa_route_experts",
               "sa_combine_experts", "sa_pack_weights", "sa_shiftadd_gemm",
               "sa_shiftadd_gemm_colwise", "sa_shiftadd_gemm_blockwise", "sa_quantize_bcq",
               "sa_quantize_bcq_terms", "sa_gram_f16", "sa_inverse_cholesky_diag",
               "sa_importance_criterion")


@pytest.fixture
def world(monkeypatch):
    return World(monkeypatch)


def linear(out=None, **kw):
    x, p, e = torch.zeros(3, 256).half(), torch.zeros(64, dtype=torch.uint8), torch.zeros(64).char()
    return sa.shiftadd_linear(x, p, e, 1, 16, 256, 128, out=out, **kw)


def route(**kw):
    return sa.route_experts(torch.zeros(100, 8), 2, **kw)


def moe(**kw):
    layer = (torch.zeros(8, dtype=torch.uint8), torch.zeros(8).char(), 1)
    return sa.shiftadd_moe(torch.zeros(100, 128).half(), torch.zeros(100, 8), 2, layer, layer, layer,
                           256, 128, 128, **kw)


def pack(**kw):
    return sa.pack_weights(torch.zeros(1, 16, 128).char(), **kw)


def plain(out=None, **kw):
    return sa.shiftadd_gemm(torch.zeros(2, 128).half(), torch.zeros(8), torch.zeros(8), 1, 16, 128,
                            128, out=out, **kw)


def colwise(out=None, **kw):
    return sa.shiftadd_gemm_colwise(torch.zeros(2, 128).half(), torch.zeros(8), torch.zeros(8), 1, 16,
                                    128, out=out, **kw)


def blockwise(out=None, **kw):
    return sa.shiftadd_gemm_blockwise(torch.zeros(2, 128).half(), torch.zeros(8), torch.zeros(8), 1,
                                      16, 128, 2, out=out, **kw)


def quantize(**kw):
    return sa.quantize_bcq(torch.zeros(16, 128), 2, 128, 3, **kw)


def quantize_terms(**kw):
    return sa.quantize_bcq_terms(torch.zeros(16, 128), 2, 128, 3, 2, **kw)


def criterion(**kw):
    return sa.bit_criterion(torch.zeros(16, 128), torch.zeros(128, 64).half(), **kw)[3:]


CONVENIENCES = [linear, route, moe, pack, plain, colwise, blockwise, quantize, quantize_terms,
                criterion]


@pytest.mark.parametrize("f", CONVENIENCES)
def test_memory_belongs_to_the_stream_that_writes_it(world, f):
    """Temporaries freed while the stream's work is queued go back to that stream alone, and no
    block that the caller's stream still uses is written; what is returned waits for the caller's
    stream too before its memory is used again."""
    out = f(stream=SIDE)
    assert world.allocated and set(world.allocated) == {SIDE}
    assert world.calls and set(world.calls) == {SIDE}
    assert world.current.cuda_stream == CALLER
    for t in out if isinstance(out, tuple) else (out,):
        assert CALLER in t.recorded


@pytest.mark.parametrize("f", CONVENIENCES)
@pytest.mark.parametrize("kw", [{}, {"stream": CALLER}])
def test_the_current_stream_needs_nothing(world, f, kw):
    out = f(**kw)
    assert set(world.allocated) == {CALLER} and set(world.calls) == {CALLER}
    for t in out if isinstance(out, tuple) else (out,):
        assert not hasattr(t, "recorded")


@pytest.mark.parametrize("f", [linear, plain, colwise, blockwise])
def test_a_given_output_is_the_callers(world, f):
    y = torch.zeros(3, 16).half()
    assert f(out=y, stream=SIDE) is y
    assert world.allocated == [] and world.calls == [SIDE]


def test_the_criterion_is_read_on_its_stream(world):
    sa.bit_criterion(torch.zeros(16, 128), torch.zeros(128, 64).half(), stream=SIDE)
    assert World.read_on == [SIDE]
