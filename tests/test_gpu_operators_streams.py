"""The conveniences around the layer on a stream that is not the current one."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():  # pragma: no cover - CPU-only environment
    pytest.skip("no GPU", allow_module_level=True)
sa = pytest.importorskip("paper_2406_05981_amd.shiftadd")

from tests.test_gpu_operators import gen, make_layer, moe_case  # noqa: E402


def busy(stream):
    """Work of some ms in front of what follows on the stream."""
    a = torch.ones((4096, 4096), device="cuda")
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        for _ in range(8):
            a = torch.mm(a, a).clamp_(max=1.0)


@pytest.mark.parametrize("raw", [False, True])
def test_moe_on_a_side_stream(raw):
    """The block is queued behind other work on a side stream while the current stream
    allocates and fills tensors of every size that the block used for itself."""
    tokens, E, k, N, K, q = 300, 6, 2, 512, 256, 3
    gate, up, down, x, logits, res = moe_case(tokens, E, k, N, K, q, seed=11)
    layers = [(a[0], a[1], q) for a in (gate, up, down)]
    call = lambda **kw: sa.shiftadd_moe(x, logits, k, *layers, N, K, 128, residual=res, **kw)  # noqa: E731
    want = call()
    sizes = [2 * tokens * k * N, 2 * tokens * k * K, 2 * tokens * K, 4 * tokens * k, 4 * (E + 1),
             sa.sa_route_workspace_bytes(tokens, E, k)]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for _ in range(3):
        busy(side)
        y = call(stream=side.cuda_stream if raw else side)
        filled = [torch.full((n,), 0x7F, dtype=torch.uint8, device="cuda") for n in sizes * 4]
        torch.cuda.current_stream().wait_stream(side)
        got = y.clone()
        del y
        with torch.cuda.stream(side):
            again = [torch.full((n,), 0x55, dtype=torch.uint8, device="cuda") for n in sizes]
        torch.cuda.synchronize()
        assert torch.equal(got, want)
        assert all((f == 0x7F).all() for f in filled) and all((f == 0x55).all() for f in again)


def test_linear_and_router_on_a_side_stream():
    q, N, K, G, rows = 3, 200, 640, 128, 90
    packed, exps, _, _ = make_layer(q, N, K, G)
    x = torch.randn((rows, K), device="cuda", generator=gen(1)).half()
    logits = torch.randn((rows, 9), device="cuda", generator=gen(2))
    want = sa.shiftadd_linear(x, packed, exps, q, N, K, G, activation="silu")
    routed = sa.route_experts(logits, 3)
    side = torch.cuda.Stream()
    busy(side)
    y = sa.shiftadd_linear(x, packed, exps, q, N, K, G, activation="silu", stream=side)
    r = sa.route_experts(logits, 3, stream=side)
    given = torch.zeros_like(want)
    torch.cuda.synchronize()
    busy(side)
    assert sa.shiftadd_linear(x, packed, exps, q, N, K, G, activation="silu", out=given,
                              stream=side) is given
    torch.cuda.synchronize()
    assert torch.equal(y, want) and torch.equal(given, want)
    assert all(torch.equal(a, b) for a, b in zip(r, routed))


def test_layer_and_quantizer_on_a_side_stream():
    q, N, K, G, rows = 2, 100, 512, 128, 12
    w = torch.randn((N, K), device="cuda", generator=gen(3))
    x = torch.randn((rows, K), device="cuda", generator=gen(4)).half()
    calib = torch.randn((K, 1024), device="cuda", generator=gen(5)).half()
    signs, exps = sa.quantize_bcq(w, q, G, 5)
    packed = sa.pack_weights(signs)
    want = sa.shiftadd_gemm(x, packed, exps, q, N, K, G)
    criterion = sa.bit_criterion(w, calib)
    side = torch.cuda.Stream()
    busy(side)
    s, e = sa.quantize_bcq(w, q, G, 5, stream=side)
    p = sa.pack_weights(s, stream=side)
    y = sa.shiftadd_gemm(x, p, e, q, N, K, G, stream=side)
    torch.cuda.synchronize()
    assert torch.equal(s, signs) and torch.equal(e, exps) and torch.equal(p, packed)
    assert torch.equal(y, want)
    busy(side)
    c = sa.bit_criterion(w, calib, stream=side)
    assert c[:3] == criterion[:3]
    torch.cuda.synchronize()
    assert torch.equal(c[3], criterion[3])
