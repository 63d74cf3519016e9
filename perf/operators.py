"""The layer's operators around the plain product, as cases that are timed and checked.

Four operators, on the public binding ``paper_2406_05981_amd.shiftadd``:

* ``linear``: y = act(x W^T + bias) * multiplier + residual on packed planes, any
  number of rows (``sa_shiftadd_gemm_epilogue``);
* ``experts``: the same product for experts with ragged sizes, rows gathered by a
  device-side list (``sa_shiftadd_gemm_experts``);
* ``route``: a router's top-k choice with its weights and the expert-sorted lists
  (``sa_route_experts``);
* ``combine``: the weighted sum of each token's expert rows (``sa_combine_experts``).

``run`` computes them with elementary torch operations where ``own`` is false and
with the library's calls where it is true.

Inputs follow the synthetic layers of ``workloads``: fair-coin planes (the packed
layout is a permutation of the keys, so packed planes are uniform bytes),
exponents uniform over a range, N(0, 1) activations with 1% of the channels x20.
"""
import math

import torch

own = False
DEV = "cuda"

ACTS = ("none", "relu", "gelu", "gelu_tanh", "silu")


# ------------------------------------------------------------------ cases

def _linear(name, N, K, q, rows, act="none", bias=False, mul=False, res=False, f16=True, G=128,
            lo=-10, hi=-3):
    return dict(name=name, kind="linear", N=N, K=K, q=q, rows=rows, act=act, bias=bias, mul=mul,
                res=res, f16=f16, G=G, lo=lo, hi=hi)


def _experts(name, E, tokens, slots, N, K, q, act="none", bias=False, mul=False, gather=True,
             f16=True, tail=0, skew=0.5, G=128, lo=-10, hi=-3):
    return dict(name=name, kind="experts", E=E, tokens=tokens, slots=slots, N=N, K=K, q=q, act=act,
                bias=bias, mul=mul, gather=gather, f16=f16, tail=tail, skew=skew, G=G, lo=lo,
                hi=hi)


def listed():
    return [
        # a token step of the 125M projection, with its bias and the residual
        # stream: a launch's latency
        _linear("proj_768_row1", 768, 768, 3, 1, bias=True, res=True, lo=-8, hi=-2),
        # a token step of a 7B model: the gate projection, SiLU, times the up branch
        _linear("gate_7b_row1", 11008, 4096, 3, 1, act="silu", mul=True),
        # eight sequences decoded together, the 70B down projection into an fp32
        # residual stream
        _linear("down_70b_rows8", 8192, 28672, 3, 8, res=True, f16=False, lo=-12),
        # a chunk of a prompt, rows and outputs of odd sizes
        _linear("chunk_rows250", 11003, 4096, 3, 250, act="gelu", bias=True, f16=False),
        # a prompt of 4096 tokens through the gate projection
        _linear("prompt_rows4096", 11008, 4096, 3, 4096, act="silu", mul=True),
        # four tokens of a decoding batch, two of eight experts each
        _experts("experts_decode", 8, 4, 8, 11008, 4096, 3, act="silu", mul=True),
        # the down projections of sixteen experts, 96 tokens with four each, in a
        # buffer with a tail that belongs to no expert
        _experts("experts_ragged", 16, 96, 384, 4096, 11008, 2, gather=False, f16=False, tail=37,
                 skew=1.0),
        # a prompt of 2048 tokens, two of eight experts each
        _experts("experts_prompt", 8, 2048, 4096, 11008, 4096, 3, act="silu", mul=True),
        # the router of a decoding batch
        dict(name="route_decode", kind="route", tokens=4, E=8, k=2, norm=True, masked=0.0),
        # the router of a long prompt over many experts, some of them masked
        dict(name="route_prompt", kind="route", tokens=8192, E=128, k=8, norm=True, masked=0.05),
        # the sum of the experts' rows for a decoding batch and for a prompt
        dict(name="combine_decode", kind="combine", tokens=4, k=2, N=4096, res=True, f16=True,
             dropped=0.0),
        dict(name="combine_prompt", kind="combine", tokens=4095, k=4, N=4096, res=True, f16=True,
             dropped=0.05),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _draw_layer(rng, weights):
    """(N, K, G, lo, hi, q) of a layer of at most ``weights`` weights."""
    G = rng.choice([128] * 6 + [256, 64, 32, 8])
    while True:
        N, K = _log(rng, 64, 28672), G * _log(rng, max(1, 256 // G), 28672 // G)
        if N * K <= weights:
            break
    if rng.random() < 0.5:
        N = 16 * max(N // 16, 1)
    return N, K, G, rng.choice([-8, -10, -12]), -3, rng.choice([1, 2, 2, 3, 3, 3, 4, 5])


def draw(rng):
    kind = rng.choice(["linear"] * 4 + ["experts"] * 3 + ["route", "combine"])
    if kind == "route":
        E = _log(rng, 4, 256)
        return dict(kind=kind, tokens=_log(rng, 1, 16384), E=E, k=min(E, rng.randint(1, 8)),
                    norm=rng.random() < 0.7, masked=rng.choice([0.0, 0.1]))
    if kind == "combine":
        tokens, N = _log(rng, 1, 8192), _log(rng, 64, 8192)
        return dict(kind=kind, tokens=tokens, k=rng.randint(1, 8), N=N, res=rng.random() < 0.7,
                    f16=rng.random() < 0.7, dropped=rng.choice([0.0, 0.1]))
    act = rng.choice(ACTS)
    bias, mul, f16 = rng.random() < 0.5, rng.random() < 0.4, rng.random() < 0.6
    if kind == "linear":
        N, K, G, lo, hi, q = _draw_layer(rng, 8192 * 28672)
        rows = rng.choice([1, _log(rng, 2, 16), _log(rng, 17, 256), _log(rng, 257, 8192)])
        # the sizes that are not a multiple of 128 columns a group are less common and smaller
        limit = 11008 * 4096 * 4096 // (16 if G % 128 else 1)
        while rows > 16 and N * K * rows * max(q, 3) // 3 > limit:
            rows //= 2
        c = _linear("", N, K, q, rows, act, bias, mul, rng.random() < 0.5, f16, G, lo, hi)
    else:
        E = _log(rng, 2, 64)
        N, K, G, lo, hi, q = _draw_layer(rng, min(8192 * 8192, 16 * 4096 * 11008 // E))
        tokens = rng.choice([_log(rng, 1, 16), _log(rng, 17, 256), _log(rng, 257, 2048)])
        k = min(E, rng.choice([1, 2, 4, 8]))
        limit = 11008 * 4096 * 4096 // (16 if G % 128 else 1)
        while tokens > 16 and N * K * tokens * k * max(q, 3) // 3 > limit:
            tokens //= 2
        c = _experts("", E, tokens, tokens * k, N, K, q, act, bias, mul, rng.random() < 0.6, f16,
                     rng.choice([0, 0, rng.randint(1, 64)]), rng.choice([0.0, 0.5, 1.0]), G, lo, hi)
    del c["name"]
    return c


# ------------------------------------------------------------------ inputs

def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(0x0E9A + int(seed))
    return g


def _counts(c):
    """Rows of each expert: shares falling with its rank, none above the tokens."""
    E, S = c["E"], c["slots"]
    share = [(e + 1.0) ** -c["skew"] for e in range(E)]
    total = sum(share)
    counts = [min(c["tokens"], int(S * s / total)) for s in share]
    e = 0
    while sum(counts) < S:
        if counts[e % E] < c["tokens"]:
            counts[e % E] += 1
        e += 1
    # the ranks are spread over the experts' numbers
    step = next(s for s in (5, 3, 7, 11, 1) if math.gcd(s, E) == 1)
    return [counts[(step * e + 1) % E] for e in range(E)]


def _uniform(g, shape, lo, hi, dtype):
    return torch.randint(lo, hi + 1, shape, dtype=dtype, device=DEV, generator=g)


def _normal(g, shape, dtype=torch.float32, scale=1.0):
    return torch.randn(shape, device=DEV, generator=g).mul_(scale).to(dtype)


def _activations(g, rows, K):
    x = torch.randn((rows, K), device=DEV, generator=g)
    x[:, torch.randperm(K, device=DEV, generator=g)[:round(0.01 * K)]] *= 20.0
    return x.to(torch.float16)


def prepare(case, seed):
    c, g = case, _gen(seed)
    s = dict(c)
    if c["kind"] in ("linear", "experts"):
        E = c.get("E", 1)
        N, K, q = c["N"], c["K"], c["q"]
        out = torch.float16 if c["f16"] else torch.float32
        s["packed"] = _uniform(g, (E, q * N * K // 8), 0, 255, torch.uint8)
        s["exps"] = _uniform(g, (E, q, N, K // c["G"]), c["lo"], c["hi"], torch.int8)
        s["bias"] = _normal(g, (E, N)) if c["bias"] else None
        if c["kind"] == "linear":
            rows = c["rows"]
            s["x"] = _activations(g, rows, K)
            s["residual"] = _normal(g, (rows, N), out, 4.0) if c["res"] else None
        else:
            rows = c["slots"] + c["tail"]
            s["counts"] = _counts(c)
            ends = [0]
            for n in s["counts"]:
                ends.append(ends[-1] + n)
            s["offsets"] = torch.tensor(ends, dtype=torch.int32, device=DEV)
            s["x"] = _activations(g, c["tokens"] if c["gather"] else rows, K)
            s["row_of"] = None
            if c["gather"]:
                # each expert's rows are distinct tokens in ascending order
                s["row_of"] = torch.cat(
                    [torch.randperm(c["tokens"], device=DEV, generator=g)[:n].sort().values
                     for n in s["counts"]] +
                    [torch.zeros(c["tail"], dtype=torch.int64, device=DEV)]).to(torch.int32)
        s["multiplier"] = _normal(g, (rows, N), out) if c["mul"] else None
        s["y"] = torch.zeros((rows, N), dtype=out, device=DEV)
    elif c["kind"] == "route":
        T, E, k = c["tokens"], c["E"], c["k"]
        # logits with 8 significant bits, as a router in bf16 gives them: ties occur
        logits = _normal(g, (T, E), scale=2.0) + _normal(g, (1, E))
        logits = logits.to(torch.bfloat16).float()
        if c["masked"]:
            logits[torch.rand((T, E), device=DEV, generator=g) < c["masked"]] = -math.inf
            logits[T // 2] = -math.inf  # a padded token
        s["logits"] = logits
        s["ids"] = torch.empty((T, k), dtype=torch.int32, device=DEV)
        s["weights"] = torch.empty((T, k), dtype=torch.float32, device=DEV)
        s["offsets"] = torch.empty(E + 1, dtype=torch.int32, device=DEV)
        s["row_of"] = torch.empty(T * k, dtype=torch.int32, device=DEV)
        s["slot_of"] = torch.empty((T, k), dtype=torch.int32, device=DEV)
        s["workspace"] = None
        if own:
            import paper_2406_05981_amd.shiftadd as sa
            s["workspace"] = torch.empty(sa.sa_route_workspace_bytes(T, E, k), dtype=torch.uint8,
                                         device=DEV)
    else:
        T, k, N = c["tokens"], c["k"], c["N"]
        out = torch.float16 if c["f16"] else torch.float32
        s["h"] = _normal(g, (T * k, N), out)
        s["slot_of"] = torch.randperm(T * k, device=DEV, generator=g).reshape(T, k).to(torch.int32)
        if c["dropped"]:
            s["slot_of"][torch.rand((T, k), device=DEV, generator=g) < c["dropped"]] = -1
        s["weights"] = torch.rand((T, k), device=DEV, generator=g)
        s["residual"] = _normal(g, (T, N), out, 4.0) if c["res"] else None
        s["y"] = torch.empty((T, N), dtype=out, device=DEV)
    return s


# ------------------------------------------------------------------ the plain form

def _weight(packed, exps, q, N, K, G, n0, n1):
    """fp32 rows n0..n1 of W = sum_i 2^e_i s_i from the packed planes.

    Rows lie in tiles of 64 and chunks of 8 columns in blocks of 16; inside a full
    block the keys of row r are rotated by r."""
    C = K // 8
    n = torch.arange(n0, n1, device=DEV)[:, None]
    c = torch.arange(C, device=DEV)[None, :]
    r, J, u = n % 64, c // 16, c % 16
    R = (N - (n - r)).clamp(max=64)
    U = (C - 16 * J).clamp(max=16)
    p = torch.where(U == 16, (u - r) % 16, u)
    at = (n - r) * C + 16 * J * R + r * U + p
    bit = torch.arange(8, device=DEV, dtype=torch.uint8)
    w = torch.zeros((n1 - n0, K), device=DEV)
    for i in range(q):
        keys = packed[i * N * C:(i + 1) * N * C][at]
        signs = (((keys[:, :, None] >> bit) & 1).float() * 2 - 1).reshape(n1 - n0, K // G, G)
        w += (signs * torch.exp2(exps[i, n0:n1].float())[:, :, None]).reshape(n1 - n0, K)
    return w


def _activate(v, act):
    if act == "relu":
        return torch.where(v < 0, torch.zeros_like(v), v)
    if act == "gelu":
        return 0.5 * v * (1 + torch.erf(v * math.sqrt(0.5)))
    if act == "gelu_tanh":
        return 0.5 * v * (1 + torch.tanh(math.sqrt(2 / math.pi) * (v + 0.044715 * v * v * v)))
    if act == "silu":
        return v / (1 + torch.exp(-v))
    return v


def _plain_product(x, packed, exps, s, bias, multiplier, residual):
    """fp32 [rows][N]; weights are expanded in slices of rows."""
    N, K = s["N"], s["K"]
    step = 64 * max(1, (1 << 25) // (64 * K))
    y = torch.cat([x @ _weight(packed, exps, s["q"], N, K, s["G"], n, min(n + step, N)).t()
                   for n in range(0, N, step)], 1)
    if bias is not None:
        y = y + bias
    y = _activate(y, s["act"])
    if multiplier is not None:
        y = y * multiplier.float()
    if residual is not None:
        y = y + residual.float()
    return y


def _plain_route(s):
    logits, k, E = s["logits"], s["k"], s["E"]
    T = logits.shape[0]
    order = torch.sort(logits, dim=1, descending=True, stable=True)
    top, ids = order.values[:, :k], order.indices[:, :k]
    live = top > -math.inf
    peak = torch.where(live[:, :1], top[:, :1], torch.zeros_like(top[:, :1]))
    weights = torch.exp(top - peak)
    total = weights.sum(1, keepdim=True) if s["norm"] else torch.exp(logits - peak).sum(
        1, keepdim=True)
    weights = torch.where(live, weights / total, torch.zeros_like(weights))
    # slots by expert, then by token and choice; choices of no expert come last
    key = torch.where(live, ids, torch.full_like(ids, E)).reshape(-1)
    by_expert = torch.sort(key, stable=True)
    offsets = torch.searchsorted(by_expert.values, torch.arange(E + 1, device=DEV))
    slot = torch.empty_like(key)
    slot[by_expert.indices] = torch.arange(T * k, device=DEV)
    slot = torch.where(key < E, slot, torch.full_like(slot, -1)).reshape(T, k)
    row_of = torch.where(by_expert.values < E, by_expert.indices // k,
                         torch.full_like(by_expert.indices, -1))
    return {"ids": torch.where(live, ids, torch.full_like(ids, -1)).to(torch.int32),
            "weights": weights, "offsets": offsets.to(torch.int32),
            "row_of": row_of.to(torch.int32), "slot_of": slot.to(torch.int32)}


def _run_plain(s):
    if s["kind"] == "linear":
        bias = s["bias"][0] if s["bias"] is not None else None
        return _plain_product(s["x"].float(), s["packed"][0], s["exps"][0], s, bias,
                              s["multiplier"], s["residual"]).to(s["y"].dtype)
    if s["kind"] == "experts":
        y = torch.zeros_like(s["y"])
        a = 0
        for e, n in enumerate(s["counts"]):
            if n == 0:
                continue
            x = s["x"][s["row_of"][a:a + n]] if s["gather"] else s["x"][a:a + n]
            y[a:a + n] = _plain_product(
                x.float(), s["packed"][e], s["exps"][e], s,
                s["bias"][e] if s["bias"] is not None else None,
                s["multiplier"][a:a + n] if s["mul"] else None, None).to(y.dtype)
            a += n
        return y
    if s["kind"] == "route":
        return _plain_route(s)
    slot, h = s["slot_of"].long(), s["h"]
    y = s["residual"].float() if s["residual"] is not None else torch.zeros(
        (s["tokens"], s["N"]), device=DEV)
    for j in range(s["k"]):
        live = slot[:, j:j + 1] >= 0
        rows = h[slot[:, j].clamp(min=0)].float() * s["weights"][:, j:j + 1]
        y = y + torch.where(live, rows, torch.zeros_like(rows))
    return y.to(s["y"].dtype)


# ------------------------------------------------------------------ the library's calls

def _run_own(s):
    import paper_2406_05981_amd.shiftadd as sa
    if s["kind"] == "linear":
        sa.sa_shiftadd_gemm_epilogue(
            s["x"], s["packed"], s["exps"], s["q"], s["N"], s["K"], s["G"], s["rows"], s["bias"],
            s["act"], s["multiplier"], s["residual"], s["y"])
        return s["y"]
    if s["kind"] == "experts":
        sa.sa_shiftadd_gemm_experts(
            s["x"], s["row_of"], s["offsets"], s["packed"], s["exps"], s["q"], s["N"], s["K"],
            s["G"], s["E"], s["slots"] + s["tail"], s["bias"], s["act"], s["multiplier"], s["y"])
        return s["y"]
    if s["kind"] == "route":
        sa.sa_route_experts(s["logits"], s["tokens"], s["E"], s["k"], s["norm"], s["ids"],
                            s["weights"], s["offsets"], s["row_of"], s["slot_of"], s["workspace"])
        return {n: s[n] for n in ("ids", "weights", "offsets", "row_of", "slot_of")}
    sa.sa_combine_experts(s["h"], s["slot_of"], s["weights"], s["tokens"], s["k"], s["N"],
                          s["residual"], s["y"])
    return s["y"]


def run(state):
    return _run_own(state) if own else _run_plain(state)


# ------------------------------------------------------------------ what a pass cannot do without

def work(case):
    c = case
    if c["kind"] == "route":
        T, E, k = c["tokens"], c["E"], c["k"]
        return {"bytes": 4 * T * E + 16 * T * k + 4 * (E + 1), "flops": 4 * T * E}
    out = 2 if c["f16"] else 4
    if c["kind"] == "combine":
        T, k, N = c["tokens"], c["k"], c["N"]
        live = T * k - int(T * k * c["dropped"])
        return {"bytes": out * N * (live + T * (2 if c["res"] else 1)) + 8 * T * k,
                "flops": 2 * live * N}
    N, K, q = c["N"], c["K"], c["q"]
    if c["kind"] == "linear":
        layers, rows, x_rows, extra = 1, c["rows"], c["rows"], 0
    else:
        layers, rows = sum(1 for n in _counts(c) if n), c["slots"]
        x_rows = min(c["tokens"], rows) if c["gather"] else rows
        extra = 4 * (c["E"] + 1) + (4 * rows if c["gather"] else 0)
    streams = 1 + int(c["mul"]) + int(c.get("res", False))
    return {"bytes": layers * q * N * (K // 8 + K // c["G"]) + 2 * x_rows * K
            + (4 * N * layers if c["bias"] else 0) + out * rows * N * streams + extra,
            "flops": 2 * rows * N * K}


# ------------------------------------------------------------------ the definition in 64 bits

def _weight64(packed, exps, q, N, K, G, t0, t1):
    """fp64 rows of the 64-row tiles t0..t1, tile by tile as they are stored."""
    C = K // 8
    full, rest = C // 16, C % 16
    out = []
    for t in range(t0, t1):
        R = min(64, N - 64 * t)
        turn = (torch.arange(16, device=DEV)[None, :] - torch.arange(R, device=DEV)[:, None]) & 15
        w = torch.zeros((R, K // G, G), dtype=torch.float64, device=DEV)
        for i in range(q):
            a = (i * N + 64 * t) * C
            tile = packed[a:a + R * C]
            blocks = tile[:16 * R * full].reshape(full, R, 16)
            keys = torch.gather(blocks, 2, turn.expand(full, R, 16)).transpose(0, 1).reshape(R, -1)
            keys = torch.cat([keys, tile[16 * R * full:].reshape(R, rest)], 1).to(torch.int32)
            for j in range(8):
                bit = torch.bitwise_and(torch.bitwise_right_shift(keys, j), 1).double()
                w.view(R, C, 8)[:, :, j] += torch.ldexp(
                    2.0 * bit - 1.0,
                    exps[i, 64 * t:64 * t + R].int().repeat_interleave(G // 8, 1))
        out.append(w.reshape(R, K))
    return torch.cat(out)


def _activate64(v, act):
    if act == "relu":
        return v.clamp(min=0.0)
    if act == "gelu":
        return v * 0.5 * torch.special.erfc(-v * math.sqrt(0.5))
    if act == "gelu_tanh":
        return v / (1.0 + torch.exp(-2.0 * math.sqrt(2.0 / math.pi) * (v + 0.044715 * v ** 3)))
    if act == "silu":
        return v / (1.0 + torch.exp(-v))
    return v


def _product64(x, packed, exps, s, bias, multiplier, residual):
    N, K = s["N"], s["K"]
    tiles = (N + 63) // 64
    step = max(1, (1 << 26) // (64 * K))
    y = torch.empty((x.shape[0], N), dtype=torch.float64, device=DEV)
    for t in range(0, tiles, step):
        w = _weight64(packed, exps, s["q"], N, K, s["G"], t, min(t + step, tiles))
        y[:, 64 * t:64 * t + w.shape[0]] = torch.mm(x, w.t().contiguous())
    if bias is not None:
        y += bias.double()
    y = _activate64(y, s["act"])
    if multiplier is not None:
        y *= multiplier.double()
    if residual is not None:
        y += residual.double()
    return y


def _route64(s):
    """Token by token on the host's arrays, from the definition."""
    import numpy as np
    logits = s["logits"].double().cpu().numpy()
    T, E, k = s["tokens"], s["E"], s["k"]
    # descending logits, equal ones by ascending number; -inf is no choice
    rank = np.lexsort((np.broadcast_to(np.arange(E), (T, E)), -logits), axis=1)[:, :k]
    top = np.take_along_axis(logits, rank, 1)
    live = np.isfinite(top)
    with np.errstate(invalid="ignore", divide="ignore"):
        p = np.exp(logits - logits.max(1, keepdims=True))
        p /= p.sum(1, keepdims=True)
        w = np.where(live, np.take_along_axis(p, rank, 1), 0.0)
        if s["norm"]:
            w = np.where(live, w / w.sum(1, keepdims=True), 0.0)
    ids = np.where(live, rank, -1)
    slot_of = np.full((T, k), -1, dtype=np.int32)
    row_of = np.full(T * k, -1, dtype=np.int32)
    offsets = np.zeros(E + 1, dtype=np.int32)
    at = 0
    for e in range(E):
        t, j = np.nonzero(ids == e)
        slot_of[t, j] = at + np.arange(len(t))
        row_of[at:at + len(t)] = t
        at += len(t)
        offsets[e + 1] = at
    t = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to(DEV)  # noqa: E731
    return {"ids": t(ids.astype(np.int32)), "weights": t(w), "offsets": t(offsets),
            "row_of": t(row_of), "slot_of": t(slot_of)}


def exact(case, seed):
    s = prepare(case, seed)
    if s["kind"] == "linear":
        return _product64(s["x"].double(), s["packed"][0], s["exps"][0], s,
                          s["bias"][0] if s["bias"] is not None else None, s["multiplier"],
                          s["residual"])
    if s["kind"] == "experts":
        y = torch.zeros(s["y"].shape, dtype=torch.float64, device=DEV)
        ends = s["offsets"].tolist()
        for e in range(s["E"]):
            a, b = ends[e], ends[e + 1]
            if a == b:
                continue
            x = s["x"].index_select(0, s["row_of"][a:b]) if s["gather"] else s["x"][a:b]
            y[a:b] = _product64(x.double(), s["packed"][e], s["exps"][e], s,
                                s["bias"][e] if s["bias"] is not None else None,
                                s["multiplier"][a:b] if s["multiplier"] is not None else None, None)
        return y
    if s["kind"] == "route":
        return _route64(s)
    y = torch.zeros((s["tokens"], s["N"]), dtype=torch.float64, device=DEV)
    if s["residual"] is not None:
        y += s["residual"].double()
    t, j = torch.nonzero(s["slot_of"] >= 0, as_tuple=True)
    rows = s["h"].double().index_select(0, s["slot_of"][t, j].long())
    y.index_add_(0, t, rows * s["weights"][t, j].double()[:, None])
    return y
