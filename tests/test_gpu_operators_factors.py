"""The operators around the layer with factors at the ends of int8.  Bounds as in
test_gpu_operators.py."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():  # pragma: no cover - CPU-only environment
    pytest.skip("no GPU", allow_module_level=True)
sa = pytest.importorskip("paper_2406_05981_amd.shiftadd")

from tests.test_gpu_operators import check, expected, gen, make_layer  # noqa: E402


def cancelling_case(q, N, K, G, rows, seed, layers=1):
    """Planes and activations whose groups sum to +-1 although |x| goes up to 64, and factors
    above 2^100 in every third row, down to 2^-128 in every third, ordinary in the others.
    Every group's sum times its factor is far inside fp32, a single product of the first rows
    is not."""
    g = gen(seed)
    signs = torch.randint(0, 2, (1, 1, K), dtype=torch.int8, device="cuda", generator=g) * 2 - 1
    signs = signs.expand(q, N, K).contiguous()
    s = signs[0, 0].double()
    x = torch.randint(-64, 65, (rows, K // 2), device="cuda", generator=g).double()
    x = torch.stack([x, -x * s[0::2] * s[1::2]], 2).reshape(rows, K)
    x[:, 0::G] = 1.0
    x[:, 1::G] = 0.0
    packed, exps, W, F = [], [], [], []
    for _ in range(layers):
        e = torch.randint(-10, -2, (q, N, K // G), dtype=torch.int8, device="cuda", generator=g)
        e[:, 0::3] = torch.randint(101, 124, e[:, 0::3].shape, dtype=torch.int8, device="cuda",
                                   generator=g)
        e[:, 1::3] = torch.randint(-128, -119, e[:, 1::3].shape, dtype=torch.int8, device="cuda",
                                   generator=g)
        f = torch.ldexp(torch.ones((), dtype=torch.float64, device="cuda"),
                        e.int().repeat_interleave(G, 2))
        packed.append(sa.pack_weights(signs))
        exps.append(e)
        W.append((f * signs).sum(0))
        F.append(f.sum(0))
    return x.half(), torch.cat(packed), torch.stack(exps), W, F


END_LAYERS = [(1, 70, 512, 128), (3, 100, 256, 128), (2, 70, 256, 256), (4, 70, 640, 128),
              (2, 70, 256, 64), (3, 70, 256, 8), (2, 70, 264, 88), (5, 70, 256, 128), (8, 40, 256, 32)]


@pytest.mark.parametrize("rows", [1, 3, 8, 16, 40, 64, 100, 300])
def test_factors_whose_products_leave_fp32(rows):
    """What the sum of a group times its factor is finite for stays finite.  Subnormal results
    round by 2^-149 at each of the q K / G additions."""
    for q, N, K, G in END_LAYERS:
        x, packed, exps, W, F = cancelling_case(q, N, K, G, rows, rows + q)
        y = torch.empty((rows, N), device="cuda")
        sa.sa_shiftadd_gemm_epilogue(x, packed, exps, q, N, K, G, rows, None, "none", None, None, y)
        torch.cuda.synchronize()
        want, bound = expected(x, W[0], F[0], q, None, "none", None, None, 0)
        check(y, want, bound + q * (K // G) * 2.0 ** -149, f"q={q} K={K} G={G} rows={rows}")


@pytest.mark.parametrize("N,K,rows", [(4096, 512, 1300), (2048, 512, 700), (1024, 1024, 300)])
@pytest.mark.parametrize("q", [1, 2, 3, 4])
def test_factors_whose_products_leave_fp32_in_larger_tiles(N, K, rows, q):
    x, packed, exps, W, F = cancelling_case(q, N, K, 128, rows, rows + q)
    y = torch.empty((rows, N), device="cuda")
    sa.sa_shiftadd_gemm_epilogue(x, packed, exps, q, N, K, 128, rows, None, "none", None, None, y)
    want, bound = expected(x, W[0], F[0], q, None, "none", None, None, 0)
    check(y, want, bound + q * (K // 128) * 2.0 ** -149, f"q={q} N={N} K={K} rows={rows}")


@pytest.mark.parametrize("counts", [[3, 0, 8, 1], [40, 0, 70, 9]])
def test_experts_factors_whose_products_leave_fp32(counts):
    E, slots = len(counts), sum(counts)
    ends = [0]
    for n in counts:
        ends.append(ends[-1] + n)
    offsets = torch.tensor(ends, dtype=torch.int32, device="cuda")
    for q, N, K, G in END_LAYERS + [(3, 70, 1152, 128)]:
        x, packed, exps, W, F = cancelling_case(q, N, K, G, slots, q, layers=E)
        y = torch.empty((slots, N), device="cuda")
        sa.sa_shiftadd_gemm_experts(x, None, offsets, packed, exps, q, N, K, G, E, slots, None,
                                    "none", None, y)
        torch.cuda.synchronize()
        for e in range(E):
            a, b = ends[e], ends[e + 1]
            if a == b:
                continue
            want, bound = expected(x[a:b], W[e], F[e], q, None, "none", None, None, 0)
            check(y[a:b], want, bound + q * (K // G) * 2.0 ** -149, f"q={q} K={K} G={G} expert {e}")


@pytest.mark.parametrize("e", [-126, -127, -128])
@pytest.mark.parametrize("rows", [1, 4, 16, 40, 300])
def test_smallest_factors(rows, e):
    """Factors that are subnormal as bfloat16 (-128 is what a zero scale quantizes to)."""
    for q, N, K, G in [(1, 70, 1024, 128), (2, 70, 1024, 64), (3, 70, 1056, 88), (5, 40, 1024, 128)]:
        packed, exps, W, F = make_layer(q, N, K, G, e, e)
        x = torch.randn((rows, K), device="cuda", generator=gen(rows)).half()
        y = sa.shiftadd_linear(x, packed, exps, q, N, K, G, out_dtype=torch.float32)
        want, bound = expected(x, W[0], F[0], q, None, "none", None, None, 0)
        check(y, want, bound + q * K * 2.0 ** -149, f"q={q} G={G} rows={rows}")
