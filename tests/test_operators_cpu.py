"""Refusals of the operators around the layer (epilogue, experts, router, combination),
on the host before any HIP call."""
import pytest

sa = pytest.importorskip("paper_2406_05981_amd.shiftadd",
                         reason="libshiftadd.so not built (python -m paper_2406_05981_amd.build)")

A = 1 << 20  # a non-null, 16-byte aligned fake address; never dereferenced here
NULL, SHAPE, Q, GROUP, ALIGN = -1, -2, -3, -4, -5


def epilogue(x=A, p=A, e=A, q=3, N=64, K=256, G=128, rows=1, bias=None, act=0, mul=None, res=None,
             half=1, y=A):
    return sa.lib.sa_shiftadd_gemm_epilogue(x, p, e, q, N, K, G, rows, bias, act, mul, res, half,
                                            y, None)


def experts(x=A, x_rows=8, row_of=None, off=A, p=A, e=A, q=3, N=64, K=256, G=128, E=4, slots=8,
            bias=None, act=0, mul=None, half=1, y=A):
    return sa.lib.sa_shiftadd_gemm_experts(x, x_rows, row_of, off, p, e, q, N, K, G, E, slots, bias,
                                           act, mul, half, y, None)


@pytest.mark.parametrize("kw,status", [
    (dict(x=None), NULL), (dict(p=None), NULL), (dict(e=None), NULL), (dict(y=None), NULL),
    (dict(q=0), Q), (dict(q=9), Q), (dict(N=0), SHAPE), (dict(K=12), SHAPE), (dict(K=0), SHAPE),
    (dict(rows=-1), SHAPE), (dict(rows=sa.SA_MAX_ROWS + 1), SHAPE),
    (dict(rows=sa.SA_MAX_ROWS, N=1 << 15), SHAPE),   # 2^35 outputs
    (dict(rows=1, N=1 << 28, K=8, G=8), SHAPE),       # 2^23 columns of tiles
    (dict(rows=sa.SA_MAX_ROWS, K=1 << 16), SHAPE),    # 2^36 activations
    (dict(act=-1), SHAPE), (dict(act=5), SHAPE),
    (dict(G=0), GROUP), (dict(G=12), GROUP), (dict(G=96), GROUP),
    (dict(x=A + 8), ALIGN), (dict(p=A + 4), ALIGN), (dict(y=A + 8), ALIGN),
    (dict(mul=A + 8), ALIGN), (dict(res=A + 2), ALIGN), (dict(bias=A + 2), ALIGN)])
def test_epilogue_refusals(kw, status):
    assert epilogue(**kw) == status


def test_no_rows_is_no_work():
    assert epilogue(rows=0, x=None, p=None, e=None, y=None) == 0
    assert epilogue(rows=0, q=9) == Q   # sizes are checked all the same
    assert experts(slots=0, x_rows=0, x=None, off=None, p=None, e=None, y=None) == 0
    assert experts(x_rows=0, x=None, row_of=A) == 0   # no slot has a row
    assert sa.lib.sa_combine_experts(None, None, None, 0, 0, 2, 64, None, 1, None, None) == 0


@pytest.mark.parametrize("kw,status", [
    (dict(x=None), NULL), (dict(off=None), NULL), (dict(p=None), NULL), (dict(e=None), NULL),
    (dict(y=None), NULL), (dict(q=9), Q), (dict(N=0), SHAPE), (dict(E=0), SHAPE),
    (dict(E=sa.SA_MAX_EXPERTS + 1), SHAPE), (dict(slots=-1), SHAPE), (dict(x_rows=-1), SHAPE),
    (dict(x_rows=sa.SA_MAX_ROWS + 1), SHAPE),
    (dict(x_rows=7), SHAPE),                          # slot 7 has no row
    (dict(slots=sa.SA_MAX_ROWS + 1, x_rows=1, row_of=A), SHAPE), (dict(act=5), SHAPE),
    (dict(G=96), GROUP), (dict(off=A + 2), ALIGN), (dict(row_of=A + 1), ALIGN),
    (dict(x=A + 8), ALIGN), (dict(mul=A + 4), ALIGN), (dict(y=A + 4), ALIGN)])
def test_experts_refusals(kw, status):
    assert experts(**kw) == status


def route(logits=A, T=100, E=8, k=2, norm=1, ids=A, w=A, off=A, row=A, slot=A, ws=A, n=1 << 20):
    return sa.lib.sa_route_experts(logits, T, E, k, norm, ids, w, off, row, slot, ws, n, None)


@pytest.mark.parametrize("kw,status", [
    (dict(logits=None), NULL), (dict(ids=None), NULL), (dict(w=None), NULL), (dict(off=None), NULL),
    (dict(row=None), NULL), (dict(slot=None), NULL), (dict(ws=None, T=5000), NULL),
    (dict(T=-1), SHAPE), (dict(T=sa.SA_MAX_ROWS + 1), SHAPE), (dict(E=0), SHAPE),
    (dict(E=sa.SA_MAX_EXPERTS + 1), SHAPE), (dict(k=0), SHAPE), (dict(k=9), SHAPE),
    (dict(E=64, k=sa.SA_MAX_CHOICES + 1), SHAPE),
    (dict(T=5000, n=sa.sa_route_workspace_bytes(5000, 8, 2) - 1), SHAPE),
    (dict(off=A + 2), ALIGN), (dict(ws=A + 8, T=5000), ALIGN)])
def test_route_refusals(kw, status):
    assert route(**kw) == status


def test_route_workspace():
    size = sa.sa_route_workspace_bytes
    assert size(-1, 8, 2) == 0 and size(5000, 0, 1) == 0 and size(5000, 8, 9) == 0
    assert size(0, 8, 2) == 0 and size(1, 8, 2) == 0
    assert size(5000, 8, 2) > 0
    assert size(sa.SA_MAX_ROWS, sa.SA_MAX_EXPERTS, 8) <= 1 << 24


@pytest.mark.parametrize("kw,status", [
    (dict(h=None), NULL), (dict(slot=None), NULL), (dict(w=None), NULL), (dict(y=None), NULL),
    (dict(T=-1), SHAPE), (dict(T=sa.SA_MAX_ROWS + 1), SHAPE), (dict(slots=-1), SHAPE),
    (dict(k=0), SHAPE), (dict(k=sa.SA_MAX_CHOICES + 1), SHAPE), (dict(N=0), SHAPE),
    (dict(T=sa.SA_MAX_ROWS, N=1 << 15), SHAPE), (dict(slots=sa.SA_MAX_ROWS, N=1 << 15), SHAPE),
    (dict(h=A + 8), ALIGN), (dict(y=A + 2), ALIGN), (dict(res=A + 8), ALIGN),
    (dict(slot=A + 2), ALIGN), (dict(w=A + 1), ALIGN)])
def test_combine_refusals(kw, status):
    a = dict(h=A, slot=A, w=A, slots=16, T=8, k=2, N=64, res=None, half=1, y=A)
    a.update(kw)
    assert sa.lib.sa_combine_experts(a["h"], a["slot"], a["w"], a["slots"], a["T"], a["k"], a["N"],
                                     a["res"], a["half"], a["y"], None) == status


def test_binding_names_the_activations():
    with pytest.raises(ValueError, match="activation"):
        sa._activation("swish")
    assert [sa._activation(a) for a in ("none", "relu", "gelu", "gelu_tanh", "silu")] == [0, 1, 2, 3, 4]
