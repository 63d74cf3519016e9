"""Refusals of the operators' binding, on the host: tensors and streams of another device than
the current one, activations that do not match the router's logits."""
import pytest

torch = pytest.importorskip("torch")
sa = pytest.importorskip("paper_2406_05981_amd.shiftadd",
                         reason="libshiftadd.so not built (python -m paper_2406_05981_amd.build)")


class Tensor(torch.Tensor):
    """A host tensor that says it lies on device `where`."""
    where = 0

    @property
    def is_cuda(self):
        return True

    def get_device(self):
        return self.where


def on(t, where=0):
    t = t.as_subclass(Tensor)
    t.where = where
    return t


class Stream:
    def __init__(self, device):
        self.cuda_stream, self.device_index = 100 + device, device


@pytest.fixture
def calls(monkeypatch):
    """Library calls made with device 0 current (none of them runs)."""
    made = []
    monkeypatch.setattr(sa, "_here", lambda: 0)
    monkeypatch.setattr(sa, "_raw_stream", lambda device: 100 + device)
    monkeypatch.setattr(torch.cuda, "is_initialized", lambda: True)
    monkeypatch.setattr(torch.cuda, "Stream", Stream)
    for name in ("sa_shiftadd_gemm_epilogue", "sa_shiftadd_gemm_experts", "sa_route_experts",
                 "sa_combine_experts"):
        monkeypatch.setattr(sa.lib, name, lambda *a: made.append(a[-1]) or 0)
    return made


E, T, K_, N_ = 4, 3, 128, 16


def half(*s):
    return on(torch.zeros(s, dtype=torch.float16))


def ints(*s):
    return on(torch.zeros(s, dtype=torch.int32))


def floats(*s):
    return on(torch.zeros(s))


def layers(n):
    return (on(torch.zeros(n * N_ * K_ // 8, dtype=torch.uint8)),
            on(torch.zeros(n * N_, dtype=torch.int8)))


def epilogue():
    p, e = layers(1)
    return sa.sa_shiftadd_gemm_epilogue, dict(
        x=half(T, K_), packed_bits=p, exps=e, q=1, N=N_, K=K_, group=128, rows=T, bias=floats(N_),
        activation="none", multiplier=half(T, N_), residual=half(T, N_), y=half(T, N_))


def experts():
    p, e = layers(E)
    return sa.sa_shiftadd_gemm_experts, dict(
        x=half(T, K_), row_of=ints(2 * T), offsets=ints(E + 1), packed_bits=p, exps=e, q=1, N=N_,
        K=K_, group=128, experts=E, slots=2 * T, bias=floats(E, N_), activation="none",
        multiplier=half(2 * T, N_), y=half(2 * T, N_))


def route():
    return sa.sa_route_experts, dict(
        logits=floats(T, E), tokens=T, experts=E, k=2, normalize=True, ids=ints(T, 2),
        weights=floats(T, 2), offsets=ints(E + 1), row_of=ints(2 * T), slot_of=ints(T, 2),
        workspace=on(torch.zeros(64, dtype=torch.uint8)))


def combine():
    return sa.sa_combine_experts, dict(
        h=half(2 * T, N_), slot_of=ints(T, 2), weights=floats(T, 2), tokens=T, k=2, N=N_,
        residual=half(T, N_), y=half(T, N_))


OPERATORS = [epilogue, experts, route, combine]


@pytest.mark.parametrize("operator", OPERATORS)
def test_tensors_of_another_device_are_refused(calls, operator):
    f, kw = operator()
    f(**kw)
    f(**kw, stream=Stream(0))
    f(**kw, stream=55)
    assert calls == [100, 100, 55]
    for name, t in kw.items():
        if isinstance(t, torch.Tensor):
            with pytest.raises(ValueError, match=f"{name} must be on the current device"):
                f(**{**kw, name: on(t.clone(), 1)})
    assert len(calls) == 3


@pytest.mark.parametrize("operator", OPERATORS)
def test_a_stream_of_another_device_is_refused(calls, operator):
    f, kw = operator()
    with pytest.raises(ValueError, match="stream must be of the current device"):
        f(**kw, stream=Stream(1))
    assert calls == []


@pytest.mark.parametrize("operator", OPERATORS)
def test_host_tensors_are_refused(calls, operator):
    f, kw = operator()
    for name, t in kw.items():
        if isinstance(t, torch.Tensor):
            with pytest.raises(ValueError, match=f"{name} must be on the GPU"):
                f(**{**kw, name: t.as_subclass(torch.Tensor).clone()})
    assert calls == []


def test_moe_refuses_activations_that_do_not_match_the_logits(calls):
    """With fewer rows of x than of logits some slots had no row, and their outputs were summed
    as they were found in memory."""
    layer = (*layers(E), 1)
    down = (on(torch.zeros(E * N_ * K_ // 8, dtype=torch.uint8)), None, 1)
    for rows in (T - 1, T + 1, 0):
        with pytest.raises(ValueError, match="x must have"):
            sa.shiftadd_moe(half(rows, K_), floats(T, E), 2, layer, layer, down, N_, K_, 128)
    assert calls == []
