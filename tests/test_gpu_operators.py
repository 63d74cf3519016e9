"""The operators around the layer against their formulas in 64 bits.

Bounds.  A product's fp32 additions form chains of at most q * K / 32 + 64 terms,
each off by 2^-24 of a partial sum, which sum|terms| bounds.  The activations' slope
is at most 1.13 and their own evaluation takes a few fp32 roundings of v (16 * 2^-24
allowed); the product with the multiplier, the sum with the residual and the store in
fp32 round once each; a binary16 store is off by 2^-11 of the value, or 2^-25 among
subnormals."""
import sys

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():  # pragma: no cover - CPU-only environment
    pytest.skip("no GPU", allow_module_level=True)
sa = pytest.importorskip("paper_2406_05981_amd.shiftadd")

U = 2.0 ** -24
INF = float("inf")


def say(*a):
    print(*a, file=sys.stderr, flush=True)


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def make_layer(q, N, K, G, lo=-8, hi=-2, seed=0, layers=1):
    """(packed [layers * bytes], exps, W fp64 [layers][N][K], sum of factors fp64)."""
    g = gen(seed)
    packed, ws, factors, es = [], [], [], []
    for _ in range(layers):
        signs = torch.randint(0, 2, (q, N, K), dtype=torch.int8, device="cuda", generator=g) * 2 - 1
        exps = torch.randint(lo, hi + 1, (q, N, K // G), dtype=torch.int8, device="cuda",
                             generator=g)
        f = torch.ldexp(torch.ones((), dtype=torch.float64, device="cuda"),
                        exps.int().repeat_interleave(G, 2))
        packed.append(sa.pack_weights(signs))
        ws.append((f * signs).sum(0))
        factors.append(f.sum(0))
        es.append(exps)
    return torch.cat(packed), torch.stack(es), torch.stack(ws), torch.stack(factors)


def activate64(v, act):
    if act == "relu":
        return torch.where(v < 0, torch.zeros_like(v), v)
    if act == "gelu":
        return 0.5 * v * torch.special.erfc(-v * 0.5 ** 0.5)
    if act == "gelu_tanh":
        return v / (1 + torch.exp(-2 * (2 / torch.pi) ** 0.5 * (v + 0.044715 * v ** 3)))
    if act == "silu":
        return v / (1 + torch.exp(-v))
    return v


def expected(x, W, F, q, bias, act, mul, res, half):
    """(value, bound) of every output in fp64."""
    K = W.shape[1]
    xd = x.double()
    v = torch.mm(xd, W.t().contiguous())
    off = (q * K / 32 + 64) * U * torch.mm(xd.abs(), F.t().contiguous())
    if bias is not None:
        v = v + bias.double()
        off = off + U * v.abs()
    if act != "none":
        off = 1.13 * off + 16 * U * v.abs()
        v = activate64(v, act)
    if mul is not None:
        v = v * mul.double()
        off = off * mul.double().abs() + 2 * U * v.abs()
    if res is not None:
        v = v + res.double()
        off = off + 2 * U * v.abs()
    off = off * 1.01
    return v, off + ((2.0 ** -11) * v.abs() + 2.0 ** -25 if half else U * v.abs())


def check(got, want, bound, what):
    d = (got.double() - want).abs()
    worst = float((d / bound.clamp(min=1e-300)).max()) if d.numel() else 0.0
    say(f"  {what}: worst error / bound {worst:.3f}")
    assert torch.isfinite(got).all(), what
    assert worst <= 1.0, what


def guarded(rows, N, dtype):
    """An output buffer with 64 elements behind it that must not change."""
    buf = torch.full((rows * N + 64,), float("nan"), dtype=dtype, device="cuda")
    buf[rows * N:] = 7.0
    return buf, buf[:rows * N].view(rows, N)


def run_epilogue(q, N, K, G, rows, act, bias, mul, res, half, lo=-8, hi=-2, seed=1):
    g = gen(seed)
    packed, exps, W, F = make_layer(q, N, K, G, lo, hi, seed)
    out = torch.float16 if half else torch.float32
    x = torch.randn((rows, K), device="cuda", generator=g).half()
    r = lambda *s: torch.randn(s, device="cuda", generator=g)  # noqa: E731
    b = r(N) if bias else None
    m = r(rows, N).to(out) if mul else None
    e = (4 * r(rows, N)).to(out) if res else None
    buf, y = guarded(rows, N, out)
    sa.sa_shiftadd_gemm_epilogue(x, packed, exps, q, N, K, G, rows, b, act, m, e, y)
    again = torch.empty_like(y)
    sa.sa_shiftadd_gemm_epilogue(x, packed, exps, q, N, K, G, rows, b, act, m, e, again)
    torch.cuda.synchronize()
    want, bound = expected(x, W[0], F[0], q, b, act, m, e, half)
    check(y, want, bound, f"q={q} N={N} K={K} G={G} rows={rows} {act}")
    assert torch.equal(y, again)
    assert (buf[rows * N:] == 7.0).all()


ACTS = ("none", "relu", "gelu", "gelu_tanh", "silu")
# layers: whole and partial 16-, 32- and 64-row tiles; 1 to 9 blocks of 128 columns; every
# plane count; groups of one and several blocks, of a part of one, of no whole one; columns
# that end inside a block
LAYERS = [(3, 64, 128, 128), (3, 130, 256, 128), (2, 1509, 128, 128), (1, 16, 512, 256),
          (4, 100, 640, 128), (3, 257, 1152, 384), (5, 70, 384, 128), (8, 33, 256, 128),
          (3, 130, 256, 8), (2, 65, 136, 8), (3, 77, 264, 88), (3, 50, 192, 64), (1, 1, 8, 8),
          (6, 48, 1040, 208), (2, 300, 4096, 128), (4, 45, 160, 32), (7, 40, 304, 16),
          (2, 300, 960, 64), (1, 3, 64, 64), (3, 66, 2048, 64)]
ROWS = [1, 2, 3, 8, 9, 16, 17, 33, 64, 65, 129, 250, 257, 300, 513]


@pytest.mark.parametrize("rows", ROWS)
def test_epilogue_over_layers(rows):
    for i, (q, N, K, G) in enumerate(LAYERS):
        flags = (rows + i) % 8
        run_epilogue(q, N, K, G, rows, ACTS[(rows + i) % 5], flags & 1, flags & 2, flags & 4,
                     half=(i // 2 + rows) % 2, seed=rows + i)


@pytest.mark.parametrize("rows", [1, 4, 7, 16, 40, 128, 300])
@pytest.mark.parametrize("act", ACTS)
def test_epilogue_terms(rows, act):
    """Each part alone and all of them, for both types."""
    for half in (0, 1):
        for flags in (0, 1, 2, 4, 7):
            run_epilogue(3, 136, 256, 128, rows, act, flags & 1, flags & 2, flags & 4, half)


@pytest.mark.parametrize("lo,hi", [(-30, 30), (-24, 0), (-40, -28), (0, 12), (-3, -3), (-14, -3)])
@pytest.mark.parametrize("rows", [1, 8, 17, 64, 300])
def test_epilogue_exponent_ranges(rows, lo, hi):
    """Exponents far apart within a group and outside binary16's range."""
    for q, N, K, G in [(3, 70, 512, 128), (4, 40, 256, 256), (2, 33, 384, 128), (5, 40, 256, 128),
                       (3, 40, 160, 32), (1, 64, 128, 128), (2, 40, 256, 8), (3, 40, 264, 88)]:
        run_epilogue(q, N, K, G, rows, "none", 0, 0, 0, 0, lo, hi)


# sizes at which each tile shape of the panel kernel has the least estimate, with rows that
# end inside a tile: 256 rows; 128 with and without column shares; 64; 32
@pytest.mark.parametrize("q", [1, 2, 3, 4, 5, 8])
@pytest.mark.parametrize("N,K,rows", [(4096, 4096, 4010), (4096, 1024, 1200), (4096, 1024, 600),
                                      (2048, 512, 700), (2048, 1024, 300), (512, 2048, 200),
                                      (1024, 1024, 100)])
def test_epilogue_tile_shapes(N, K, rows, q):
    for lo, hi in ((-8, -2), (-20, 3)):   # planes summed; some blocks plane by plane
        run_epilogue(q, N, K, 128, rows, "silu", 1, 1, 1, q % 2, lo, hi)


def test_epilogue_extreme_exponents():
    """Factors near the ends of fp32's range."""
    q, N, K, G = 2, 64, 256, 128
    for rows in (1, 5, 40, 300):
        packed, exps, _, _ = make_layer(q, N, K, G, seed=3)
        x = torch.zeros((rows, K), dtype=torch.float16, device="cuda")
        x[:, 0] = 0.5
        exps[:] = -120
        exps[:, :, N // 2:] = 120
        y = torch.empty((rows, N), device="cuda")
        sa.sa_shiftadd_gemm_epilogue(x, packed, exps, q, N, K, G, rows, None, "none", None, None, y)
        s = torch.empty((q, N, K), dtype=torch.int8, device="cuda")
        sa.sa_unpack_weights(packed, q, N, K, s)
        f = torch.ldexp(torch.ones((), dtype=torch.float64, device="cuda"),
                        exps[0].int().repeat_interleave(G, 2))
        want = torch.mm(x.double(), (f * s).sum(0).t().contiguous())
        assert torch.equal(y.double(), want), rows


@pytest.mark.parametrize("rows", [2, 5, 12, 70, 300])
@pytest.mark.parametrize("value", [INF, -INF, float("nan")])
def test_not_finite_rows_keep_to_themselves(rows, value):
    for q, N, K, G in [(3, 130, 256, 128), (2, 65, 136, 8), (3, 70, 1152, 128)]:
        packed, exps, W, F = make_layer(q, N, K, G)
        x = torch.randn((rows, K), device="cuda", generator=gen(5)).half()
        x[rows // 2, K // 3] = value
        y = torch.empty((rows, N), device="cuda")
        sa.sa_shiftadd_gemm_epilogue(x, packed, exps, q, N, K, G, rows, None, "none", None, None, y)
        torch.cuda.synchronize()
        assert not torch.isfinite(y[rows // 2]).any()
        keep = torch.arange(rows, device="cuda") != rows // 2
        want, bound = expected(x[keep], W[0], F[0], q, None, "none", None, None, 0)
        check(y[keep], want, bound, f"rows={rows} {value}")


def test_activations_at_the_ends():
    """Infinite, NaN and huge sums: bias carries them through a zero product."""
    N, K = 16, 128
    packed, exps, _, _ = make_layer(1, N, K, 128)
    bias = torch.zeros(N, device="cuda")
    ends = [INF, -INF, float("nan"), 1e30, -1e30, 200.0, -200.0, 0.0]
    bias[:8] = torch.tensor(ends, device="cuda")
    for rows in (1, 4, 20, 300):
        x = torch.zeros((rows, K), dtype=torch.float16, device="cuda")
        for act, want in [("relu", [INF, 0.0, None, 1e30, 0.0, 200.0, 0.0, 0.0]),
                          ("silu", [INF, None, None, 1e30, 0.0, 200.0, 0.0, 0.0]),
                          ("gelu", [INF, None, None, 1e30, 0.0, 200.0, 0.0, 0.0]),
                          ("gelu_tanh", [INF, None, None, 1e30, 0.0, 200.0, 0.0, 0.0])]:
            y = sa.shiftadd_linear(x, packed, exps, 1, N, K, 128, bias, act,
                                   out_dtype=torch.float32)
            for j, w in enumerate(want):
                col = y[:, j]
                assert torch.isnan(col).all() if w is None else (col == torch.tensor(
                    w, device="cuda")).all(), (rows, act, ends[j], col[0])


def test_in_place_residual_and_multiplier():
    q, N, K, G = 3, 203, 384, 128
    packed, exps, W, F = make_layer(q, N, K, G)
    for rows in (1, 6, 30, 270):
        for out in (torch.float16, torch.float32):
            g = gen(rows)
            x = torch.randn((rows, K), device="cuda", generator=g).half()
            y = torch.randn((rows, N), device="cuda", generator=g).to(out)
            before = y.clone()
            sa.sa_shiftadd_gemm_epilogue(x, packed, exps, q, N, K, G, rows, None, "none", None, y, y)
            check(y, *expected(x, W[0], F[0], q, None, "none", None, before, out == torch.float16),
                  "residual in place")
            y.copy_(before)
            sa.sa_shiftadd_gemm_epilogue(x, packed, exps, q, N, K, G, rows, None, "silu", y, None, y)
            check(y, *expected(x, W[0], F[0], q, None, "silu", before, None, out == torch.float16),
                  "multiplier in place")


def test_batch_agrees_with_the_plain_layer():
    q, N, K, G = 3, 1000, 1024, 128
    packed, exps, W, F = make_layer(q, N, K, G)
    for rows in (1, 5, 48, 256):
        x = torch.randn((rows, K), device="cuda", generator=gen(rows)).half()
        a = sa.shiftadd_gemm(x, packed, exps, q, N, K, G)
        b = sa.shiftadd_linear(x, packed, exps, q, N, K, G, out_dtype=torch.float32)
        _, bound = expected(x, W[0], F[0], q, None, "none", None, None, 0)
        assert ((a - b).abs() <= 2 * bound).all()


def test_outputs_past_32_bit_offsets():
    """70001 x 32769 outputs: element offsets past 2^31."""
    q, N, K, G, rows = 1, 32769, 128, 128, 70001
    packed, exps, W, F = make_layer(q, N, K, G)
    x = torch.randn((rows, K), device="cuda", generator=gen(9)).half()
    y = sa.shiftadd_linear(x, packed, exps, q, N, K, G, residual=None)
    pick = torch.tensor([0, 1, 65535, 65536, 65537, 70000], device="cuda")
    want, bound = expected(x[pick], W[0], F[0], q, None, "none", None, None, 1)
    check(y[pick], want, bound, "far rows")


def test_most_rows():
    q, N, K, G, rows = 2, 40, 64, 64, sa.SA_MAX_ROWS
    packed, exps, W, F = make_layer(q, N, K, G)
    x = torch.randn((rows, K), device="cuda", generator=gen(2)).half()
    y = sa.shiftadd_linear(x, packed, exps, q, N, K, G, activation="relu")
    check(y, *expected(x, W[0], F[0], q, None, "relu", None, None, 1), "2^20 rows")


def test_long_rows():
    """2^22 + 128 columns: past the bound of the kernels that divide by multiplication."""
    q, N, K, G = 1, 17, (1 << 22) + 128, 128
    packed, exps, W, F = make_layer(q, N, K, G)
    for rows in (1, 3, 40):
        x = torch.randn((rows, K), device="cuda", generator=gen(rows)).half()
        y = sa.shiftadd_linear(x, packed, exps, q, N, K, G, out_dtype=torch.float32)
        check(y, *expected(x, W[0], F[0], q, None, "none", None, None, 0), f"{rows} long rows")


def test_activations_past_32_bit_offsets():
    """Rows of x beyond 4 GiB, by a list and in order."""
    q, N, K, G, rows = 2, 33, 8192, 128, 262144 + 300
    packed, exps, W, F = make_layer(q, N, K, G)
    x = torch.zeros((rows, K), dtype=torch.float16, device="cuda")
    x[-300:] = torch.randn((300, K), device="cuda", generator=gen(4)).half()
    slots = 300
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


@pytest.mark.parametrize("rows", [1, 6, 20, 90, 300])
def test_epilogue_captured_and_replayed(rows):
    q, N, K, G = 3, 200, 640, 128
    packed, exps, _, _ = make_layer(q, N, K, G)
    x = torch.zeros((rows, K), dtype=torch.float16, device="cuda")
    res = torch.zeros((rows, N), dtype=torch.float16, device="cuda")
    y = torch.empty_like(res)
    call = lambda out: sa.sa_shiftadd_gemm_epilogue(  # noqa: E731
        x, packed, exps, q, N, K, G, rows, None, "gelu", None, res, out)
    call(y)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(y)
    for seed in range(3):
        x.copy_(torch.randn((rows, K), device="cuda", generator=gen(seed)))
        res.copy_(torch.randn((rows, N), device="cuda", generator=gen(seed + 9)))
        graph.replay()
        eager = torch.empty_like(y)
        call(eager)
        torch.cuda.synchronize()
        assert torch.equal(y, eager)


def test_calls_on_two_streams():
    """Different calls in flight at once share nothing."""
    q, N, K, G = 3, 1024, 1024, 128
    packed, exps, W, F = make_layer(q, N, K, G)
    streams = [torch.cuda.Stream() for _ in range(2)]
    xs = [torch.randn((r, K), device="cuda", generator=gen(r)).half() for r in (5, 500)]
    ys = [torch.empty((x.shape[0], N), device="cuda") for x in xs]
    torch.cuda.synchronize()
    for _ in range(5):
        for st, x, y in zip(streams, xs, ys):
            sa.sa_shiftadd_gemm_epilogue(x, packed, exps, q, N, K, G, x.shape[0], None, "silu", None,
                                         None, y, stream=st)
    torch.cuda.synchronize()
    for x, y in zip(xs, ys):
        check(y, *expected(x, W[0], F[0], q, None, "silu", None, None, 0), "two streams")


# ------------------------------------------------------------------ experts

def run_experts(q, N, K, G, counts, tokens, gather, act, bias, mul, half, lead=0, tail=0, seed=0,
                lo=-8, hi=-2):
    g = gen(seed)
    E, used = len(counts), sum(counts)
    slots = lead + used + tail
    packed, exps, W, F = make_layer(q, N, K, G, lo, hi, seed, layers=E)
    out = torch.float16 if half else torch.float32
    ends = [lead]
    for n in counts:
        ends.append(ends[-1] + n)
    offsets = torch.tensor(ends, dtype=torch.int32, device="cuda")
    x = torch.randn((tokens if gather else slots, K), device="cuda", generator=g).half()
    row_of = None
    skipped = []
    if gather:
        row_of = torch.randint(0, tokens, (slots,), dtype=torch.int32, device="cuda", generator=g)
        if used > 2:  # two slots without a row
            skipped = [lead, lead + used // 2]
            row_of[skipped[0]] = -1
            row_of[skipped[1]] = tokens
    b = torch.randn((E, N), device="cuda", generator=g) if bias else None
    m = torch.randn((slots, N), device="cuda", generator=g).to(out) if mul else None
    buf, y = guarded(slots, N, out)
    y.fill_(3.0)
    sa.sa_shiftadd_gemm_experts(x, row_of, offsets, packed, exps, q, N, K, G, E, slots, b, act, m, y)
    torch.cuda.synchronize()
    left = torch.ones(slots, dtype=torch.bool, device="cuda")
    for e, n in enumerate(counts):
        s = [i for i in range(ends[e], ends[e + 1]) if i not in skipped]
        if not s:
            continue
        s = torch.tensor(s, device="cuda")
        left[s] = False
        xe = x[row_of[s].long()] if gather else x[s]
        want, bound = expected(xe, W[e], F[e], q, b[e] if bias else None, act,
                               m[s] if mul else None, None, half)
        check(y[s], want, bound, f"expert {e} rows {n}")
    assert (y[left] == 3.0).all()
    assert (buf[slots * N:] == 7.0).all()


COUNTS = [[1], [0], [0, 0, 3], [5, 0, 1, 2], [8, 1, 0, 0, 9, 16], [17, 0, 64, 1], [0, 130, 3, 33],
          [300, 0, 1], [1] * 40, [0] * 70 + [4] + [0] * 10 + [11]]


@pytest.mark.parametrize("counts", COUNTS, ids=lambda c: "-".join(map(str, c[:6])) + f"-of{len(c)}")
@pytest.mark.parametrize("gather", [0, 1])
def test_experts(counts, gather):
    layers = [(3, 64, 256, 128), (2, 133, 384, 128), (3, 65, 136, 8), (5, 48, 128, 128),
              (1, 33, 192, 64)]
    for i, (q, N, K, G) in enumerate(layers):
        run_experts(q, N, K, G, counts, tokens=max(sum(counts), 7), gather=gather,
                    act=ACTS[(i + len(counts)) % 5], bias=i % 2, mul=(i + gather) % 2,
                    half=(i + len(counts)) % 2, lead=3 * (i % 2), tail=5 * (i // 2), seed=i)


@pytest.mark.parametrize("q", [1, 2, 3, 4])
def test_experts_tile_heights(q):
    """Tiles of 256 rows that end after 40, 100, 170 and 250 rows."""
    run_experts(q, 8192, 2048, 128, [296, 356, 426, 762], 500, 1, "silu", 1, 1, q % 2, tail=3)


def test_most_experts():
    counts = [(7 * e) % 5 for e in range(sa.SA_MAX_EXPERTS)]
    run_experts(2, 16, 128, 128, counts, 50, 1, "silu", 1, 1, 1, lead=2, tail=3)


@pytest.mark.parametrize("q,K,G", [(7, 256, 128), (6, 384, 128), (8, 192, 32), (4, 320, 16)])
def test_experts_of_many_planes(q, K, G):
    run_experts(q, 70, K, G, [3, 0, 70, 9], 60, 1, "relu", 1, 0, 0)


@pytest.mark.parametrize("counts", [[3, 0, 12], [100, 40, 0, 5]])
def test_experts_exponent_ranges(counts):
    for lo, hi in [(-30, 30), (-40, -28), (0, 12)]:
        run_experts(3, 70, 256, 128, counts, 160, 1, "none", 0, 0, 0, lo=lo, hi=hi)


def test_experts_with_offsets_out_of_range():
    """Offsets beyond the buffer or descending reach no memory outside it."""
    q, N, K, G, E, slots = 2, 64, 128, 128, 4, 10
    packed, exps, _, _ = make_layer(q, N, K, G, layers=E)
    x = torch.randn((slots, K), device="cuda").half()
    for off in ([0, 1 << 30, 5, -7, 1 << 30], [-5, -3, 2, 2, 400], [50, 60, 70, 80, 90]):
        buf, y = guarded(slots, N, torch.float32)
        y.fill_(0.0)
        offsets = torch.tensor(off, dtype=torch.int32, device="cuda")
        sa.sa_shiftadd_gemm_experts(x, None, offsets, packed, exps, q, N, K, G, E, slots, None,
                                    "none", None, y)
        torch.cuda.synchronize()
        assert (buf[slots * N:] == 7.0).all() and torch.isfinite(y).all()


# ------------------------------------------------------------------ router

def route_reference(logits, k, normalize):
    T, E = logits.shape
    ids = torch.full((T, k), -1, dtype=torch.int32)
    w = torch.zeros((T, k), dtype=torch.float64)
    for t in range(T):
        row = logits[t].double()
        # a NaN counts as -inf; -0 as 0
        row = torch.where(torch.isnan(row), torch.full_like(row, -INF), row) + 0.0
        v = row.tolist()
        order = sorted((e for e in range(E) if v[e] > -INF), key=lambda e: (-v[e], e))[:k]
        if not order:
            continue
        p = torch.exp(row - row[order[0]])
        total = p[order].sum() if normalize else p.sum()
        for j, e in enumerate(order):
            ids[t, j] = e
            w[t, j] = p[e] / total
    pairs = sorted((int(ids[t, j]), t, j) for t in range(T) for j in range(k) if ids[t, j] >= 0)
    slot_of = torch.full((T, k), -1, dtype=torch.int32)
    row_of = torch.full((T * k,), -1, dtype=torch.int32)
    offsets = torch.zeros(E + 1, dtype=torch.int32)
    for s, (e, t, j) in enumerate(pairs):
        slot_of[t, j] = s
        row_of[s] = t
        offsets[e + 1] += 1
    return ids, w, offsets.cumsum(0).to(torch.int32), row_of, slot_of


def check_route(logits, k, normalize):
    ids, w, offsets, row_of, slot_of = sa.route_experts(logits.cuda(), k, normalize)
    torch.cuda.synchronize()
    r = route_reference(logits, k, normalize)
    assert torch.equal(ids.cpu(), r[0])
    assert torch.equal(offsets.cpu(), r[2])
    assert torch.equal(row_of.cpu(), r[3])
    assert torch.equal(slot_of.cpu(), r[4])
    # an exponential of an fp32 difference d (off by 2^-24 |d|), a sum of up to 1024 terms in
    # chains of at most 22, a division: relative to the weight
    d = (logits.double().nan_to_num(0, 0, 0).abs().amax() * 2 + 32) * U
    assert ((w.cpu().double() - r[1]).abs() <= d * r[1] + 1e-38).all()


@pytest.mark.parametrize("E,k", [(1, 1), (2, 2), (8, 2), (64, 8), (65, 3), (128, 8), (200, 16),
                                 (300, 1), (1000, 6)])
@pytest.mark.parametrize("tokens", [1, 3, 64, 65, 300])
def test_route(tokens, E, k):
    g = torch.Generator().manual_seed(tokens * E + k)
    logits = (torch.randn((tokens, E), generator=g) * 2).bfloat16().float()
    check_route(logits, k, True)
    logits[torch.rand((tokens, E), generator=g) < 0.3] = -INF
    logits[tokens // 2] = -INF
    check_route(logits, k, False)
    check_route(logits, k, True)


def test_route_long():
    """More tokens than one 64-token step a workgroup."""
    g = torch.Generator().manual_seed(1)
    check_route(torch.randint(-3, 4, (17001, 6), generator=g).float(), 2, True)


def test_route_ties_and_odd_values():
    logits = torch.tensor([[0.0, -0.0, 0.0, -0.0], [1.0, float("nan"), 1.0, 1.0],
                           [float("nan")] * 4, [-INF, -INF, -3e38, -INF],
                           [3e38, -3e38, 3e38, 0.0], [5.0, 5.0, 5.0, 5.0]])
    for k in (1, 2, 4):
        for normalize in (True, False):
            check_route(logits, k, normalize)


def test_route_infinite_logit():
    logits = torch.tensor([[0.0, INF, 1.0], [0.0, 1.0, 2.0]], device="cuda")
    ids, w, *_ = sa.route_experts(logits, 2)
    assert ids.tolist() == [[1, 2], [2, 1]]
    assert torch.isnan(w[0]).all() and torch.isfinite(w[1]).all()


def test_route_no_tokens():
    offsets = torch.full((9,), 5, dtype=torch.int32, device="cuda")
    none = torch.empty(0, dtype=torch.int32, device="cuda")
    sa.sa_route_experts(none.float(), 0, 8, 2, True, none, none.float(), offsets, none, none)
    assert (offsets == 0).all()


# ------------------------------------------------------------------ combination

@pytest.mark.parametrize("N", [1, 7, 64, 130, 2048, 2056, 4100])
@pytest.mark.parametrize("tokens,k", [(1, 1), (3, 2), (65, 4), (40, 16)])
def test_combine(tokens, k, N):
    g = gen(N + k)
    slots = tokens * k
    for half in (0, 1):
        out = torch.float16 if half else torch.float32
        for res in (0, 1, 2):   # none, a tensor, y itself
            h = torch.randn((slots, N), device="cuda", generator=g).to(out)
            slot_of = torch.randperm(slots, device="cuda", generator=g).int().view(tokens, k)
            slot_of[torch.rand((tokens, k), device="cuda", generator=g) < 0.2] = -1
            slot_of[0, 0] = slots          # none either
            w = torch.rand((tokens, k), device="cuda", generator=g)
            w[slot_of < 0] = float("nan")  # of no slot: not used
            w[0, 0] = INF
            buf, y = guarded(tokens, N, out)
            r = torch.randn((tokens, N), device="cuda", generator=g).to(out) if res else None
            want = r.double() if res else torch.zeros((tokens, N), dtype=torch.float64, device="cuda")
            if res == 2:
                y.copy_(r)
            size = want.abs()
            for j in range(k):
                live = (slot_of[:, j] >= 0) & (slot_of[:, j] < slots)
                term = h[slot_of[:, j].long().clamp(0, slots - 1)].double() * w[:, j:j + 1].double()
                term = torch.where(live[:, None], term, torch.zeros_like(term))
                want = want + term
                size = size + term.abs()
            sa.sa_combine_experts(h, slot_of, w, tokens, k, N, y if res == 2 else r, y)
            torch.cuda.synchronize()
            bound = (k + 1) * U * size + (2.0 ** -11 * want.abs() + 2.0 ** -25 if half else 0)
            check(y, want, bound + 1e-30, f"combine half={half} res={res}")
            assert (buf[tokens * N:] == 7.0).all()


# ------------------------------------------------------------------ together

def moe_case(tokens, E, k, N, K, q, seed):
    G = 128
    g = gen(seed)
    gate, up = make_layer(q, N, K, G, seed=seed, layers=E), make_layer(q, N, K, G, seed=seed + 1, layers=E)
    down = make_layer(q, K, N, G, seed=seed + 2, layers=E)
    x = torch.randn((tokens, K), device="cuda", generator=g).half()
    logits = torch.randn((tokens, E), device="cuda", generator=g)
    res = torch.randn((tokens, K), device="cuda", generator=g).half()
    return gate, up, down, x, logits, res


def moe_reference(gate, up, down, x, logits, k, res):
    """fp64 with the block's binary16 roundings between its calls left out, and the size
    of the terms."""
    ids, w, *_ = route_reference(logits.cpu(), k, True)
    y, size = res.double(), res.double().abs()
    for t in range(x.shape[0]):
        for j in range(k):
            e = int(ids[t, j])
            xt = x[t].double()
            a = activate64((gate[2][e] * xt).sum(1), "silu")
            u = (up[2][e] * xt).sum(1)
            y[t] += w[t, j].item() * (down[2][e] * (a * u)).sum(1)
            size[t] += w[t, j].item() * (down[3][e] * (a * u).abs()).sum(1)
    return y, size


@pytest.mark.parametrize("tokens,E,k", [(1, 4, 2), (5, 8, 2), (40, 4, 3), (150, 6, 2)])
def test_moe_block(tokens, E, k):
    """Router, experts and combination as a block uses them.  The three binary16 tensors
    between the calls round by 2^-11 of their values each, and the last store by 2^-11;
    fp32 sums are far below."""
    N, K, q = 256, 128, 3
    gate, up, down, x, logits, res = moe_case(tokens, E, k, N, K, q, seed=tokens)
    layers = [(a[0], a[1], q) for a in (gate, up, down)]
    y = sa.shiftadd_moe(x, logits, k, *layers, N, K, 128, residual=res)
    torch.cuda.synchronize()
    want, size = moe_reference(gate, up, down, x, logits, k, res)
    check(y, want, 5 * 2.0 ** -11 * size + 2.0 ** -20, "moe block")


def test_moe_block_captured_and_replayed():
    """One graph, replayed on new inputs with eager work between; on a stream of its own."""
    tokens, E, k, N, K, q = 70, 6, 2, 256, 128, 3
    gate, up, down, x, logits, _ = moe_case(tokens, E, k, N, K, q, seed=3)
    layers = [(a[0], a[1], q) for a in (gate, up, down)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        sa.shiftadd_moe(x, logits, k, *layers, N, K, 128)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = sa.shiftadd_moe(x, logits, k, *layers, N, K, 128)
    for seed in range(4):
        g = gen(100 + seed)
        x.copy_(torch.randn((tokens, K), device="cuda", generator=g))
        logits.copy_(torch.randn((tokens, E), device="cuda", generator=g))
        graph.replay()
        eager = sa.shiftadd_moe(x, logits, k, *layers, N, K, 128)
        torch.cuda.synchronize()
        assert torch.equal(y, eager)


def test_binding_refuses_wrong_tensors():
    q, N, K, G = 1, 16, 128, 128
    packed, exps, _, _ = make_layer(q, N, K, G)
    x = torch.zeros((2, K), dtype=torch.float16, device="cuda")
    y = torch.zeros((2, N), dtype=torch.float16, device="cuda")
    call = lambda **kw: sa.sa_shiftadd_gemm_epilogue(*{**dict(  # noqa: E731
        x=x, packed_bits=packed, exps=exps, q=q, N=N, K=K, group=G, rows=2, bias=None,
        activation="none", multiplier=None, residual=None, y=y), **kw}.values())
    call()
    for kw in (dict(x=x.float()), dict(x=x.cpu()), dict(x=x[:, ::2]), dict(rows=3),
               dict(y=y.bfloat16()), dict(residual=y.float()), dict(multiplier=y[:1]),
               dict(bias=torch.zeros(N, dtype=torch.float16, device="cuda")),
               dict(activation="swish"), dict(packed_bits=packed[:-1])):
        with pytest.raises(ValueError):
            call(**kw)
    with pytest.raises(sa.SaError):
        call(group=96)
