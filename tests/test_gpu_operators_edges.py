"""The operators around the layer at their edges: every tile shape with groups that are not
whole blocks of 128 columns, experts whose columns are shared by waves, infinities and NaN
among experts, subnormal activations.  Bounds as in
test_gpu_operators.py."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():  # pragma: no cover - CPU-only environment
    pytest.skip("no GPU", allow_module_level=True)
sa = pytest.importorskip("paper_2406_05981_amd.shiftadd")

from tests.test_gpu_operators import (INF, check, expected, gen, make_layer,  # noqa: E402
                                      run_epilogue, run_experts)

# ------------------------------------------------------------------ groups and tile shapes

# N, rows: tiles of 128 rows that end after 72, 2 and 48; of 64 that end after 32, 36 and 2; of 32
SHAPES = [(8200, 200), (8200, 258), (4100, 1200), (8200, 160), (4100, 100), (2050, 258), (8200, 70)]


@pytest.mark.parametrize("q", [1, 2, 3, 4, 5, 8])
@pytest.mark.parametrize("G,K", [(64, 576), (32, 544), (8, 520), (88, 528), (208, 624), (64, 512)])
def test_tile_shapes_of_other_groups(G, K, q):
    """Columns end inside a block but for the last; planes summed, and some blocks plane by
    plane."""
    for i, (N, rows) in enumerate(SHAPES):
        lo, hi = ((-8, -2), (-20, 3))[(i + q) % 2]
        run_epilogue(q, N, K, G, rows, "silu", 1, i % 2, 1 - i % 2, (i + q) % 2, lo, hi)


@pytest.mark.parametrize("q", [2, 3, 5])
@pytest.mark.parametrize("N,K,G,counts", [
    (2050, 576, 64, [150, 0, 70, 260]), (4100, 576, 64, [300, 33, 1, 466]),
    (4100, 520, 8, [130, 800, 40]), (2050, 528, 88, [150, 0, 70, 260]),
    (4100, 624, 208, [100, 120, 131, 129])])
def test_experts_of_other_groups(N, K, G, counts, q):
    run_experts(q, N, K, G, counts, 200, 1, "gelu", 1, 1, q % 2, lead=2, tail=3, seed=q)
    run_experts(q, N, K, G, counts, 200, 0, "none", 0, 0, 0, seed=q, lo=-20, hi=3)


@pytest.mark.parametrize("G,K", [(64, 8192), (88, 8184)])
def test_far_activations_of_other_groups(G, K):
    """Rows of x beyond 4 GiB, by a list and in order."""
    q, N, rows, slots = 2, 33, 262144 + 300, 300
    assert rows * K >= 1 << 31
    packed, exps, W, F = make_layer(q, N, K, G)
    x = torch.zeros((rows, K), dtype=torch.float16, device="cuda")
    x[-slots:] = torch.randn((slots, K), device="cuda", generator=gen(4)).half()
    row_of = torch.arange(rows - 1, rows - 1 - slots, -1, dtype=torch.int32, device="cuda")
    offsets = torch.tensor([0, slots], dtype=torch.int32, device="cuda")
    y = torch.empty((slots, N), device="cuda")
    sa.sa_shiftadd_gemm_experts(x, row_of, offsets, packed, exps, q, N, K, G, 1, slots, None, "none",
                                None, y)
    want, bound = expected(x[row_of.long()], W[0], F[0], q, None, "none", None, None, 0)
    check(y, want, bound, "far rows by a list")
    full = sa.shiftadd_linear(x, packed, exps, q, N, K, G, out_dtype=torch.float32)
    check(full[-slots:].flip(0), want, bound, "far rows in order")
    assert (full[:-slots] == 0).all()


# ------------------------------------------------------------------ experts of a few rows

@pytest.mark.parametrize("K", [640, 1152, 2048, 4096])
@pytest.mark.parametrize("q", [1, 2, 3, 4])
def test_experts_of_shared_columns(q, K):
    """Two waves share more than 512 columns, four more than 1024."""
    for gather in (0, 1):
        run_experts(q, 133, K, 128, [3, 0, 8, 1, 5, 2], 11, gather, "silu", 1, gather, gather, lead=1,
                    tail=2, seed=K + q)
    run_experts(q, 80, K, K, [0, 1, 7, 4], 9, 1, "none", 0, 0, 0, seed=K + q, lo=-30, hi=30)


def test_experts_of_several_tiles_a_wave():
    run_experts(2, 12300, 640, 128, [4, 1, 8, 2, 6, 3], 30, 1, "gelu", 1, 1, 1, seed=5)


LAYERS = [(3, 130, 640, 128), (2, 65, 1152, 128), (2, 65, 136, 8), (3, 70, 264, 88), (5, 40, 256, 128)]


@pytest.mark.parametrize("value", [INF, -INF, float("nan")])
@pytest.mark.parametrize("counts", [[3, 0, 6, 1], [40, 0, 70, 9], [0, 2, 150, 0, 0]])
def test_experts_not_finite_rows_keep_to_themselves(counts, value):
    """Two tokens that are not finite: one in several slots, and row 0, which slots without a
    row must not take anything from."""
    E, slots = len(counts), sum(counts)
    ends = [0]
    for n in counts:
        ends.append(ends[-1] + n)
    offsets = torch.tensor(ends, dtype=torch.int32, device="cuda")
    for q, N, K, G in LAYERS:
        g = gen(slots)
        packed, exps, W, F = make_layer(q, N, K, G, layers=E)
        tokens = 12
        x = torch.randn((tokens, K), device="cuda", generator=g).half()
        x[0, K - 1] = value
        x[5, K // 3] = value
        row_of = torch.randint(1, tokens, (slots,), dtype=torch.int32, device="cuda", generator=g)
        row_of[slots // 2] = 5
        row_of[slots - 1] = 7
        row_of[0] = -1
        row_of[slots // 3] = tokens
        y = torch.full((slots, N), 3.0, device="cuda")
        sa.sa_shiftadd_gemm_experts(x, row_of, offsets, packed, exps, q, N, K, G, E, slots, None,
                                    "none", None, y)
        torch.cuda.synchronize()
        for e in range(E):
            s = torch.arange(ends[e], ends[e + 1], device="cuda")
            r = row_of[s].long()
            none = (r < 0) | (r >= tokens)
            assert (y[s[none]] == 3.0).all()
            assert not torch.isfinite(y[s[r == 5]]).any()
            keep = ~none & (r != 5)
            if keep.any():
                want, bound = expected(x[r[keep]], W[e], F[e], q, None, "none", None, None, 0)
                check(y[s[keep]], want, bound, f"q={q} K={K} G={G} expert {e}")


# ------------------------------------------------------------------ subnormal activations

@pytest.mark.parametrize("rows", [1, 4, 16, 40, 300])
def test_subnormal_activations(rows):
    """x of at most 3 steps of 2^-24 and factors in 2^-10..2^-3: every partial sum is a
    multiple of 2^-34 below q K 3 2^-24 2^-3 < 2^-13, so fp32 holds it and the result is exact."""
    for q, N, K, G in [(3, 130, 256, 128), (2, 70, 512, 64), (3, 70, 264, 88), (5, 40, 256, 128)]:
        packed, exps, _, _ = make_layer(q, N, K, G, -10, -3)
        # factors as whole numbers of 2^-10: torch.ldexp is off by an ulp of fp64
        signs = torch.empty((q, N, K), dtype=torch.int8, device="cuda")
        sa.sa_unpack_weights(packed, q, N, K, signs)
        factors = (1 << (exps[0].int() + 10)).repeat_interleave(G, 2)
        W = (factors * signs).sum(0).double() / 1024
        k = torch.randint(-3, 4, (rows, K), device="cuda", generator=gen(rows))
        x = (k.double() * 2.0 ** -24).half()
        y = sa.shiftadd_linear(x, packed, exps, q, N, K, G, out_dtype=torch.float32)
        assert torch.equal(y.double(), torch.mm(x.double(), W.t().contiguous())), (q, G, rows)
