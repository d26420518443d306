"""Performance cases of the mixture-of-experts layer and of block-scaled 8-bit weights.

Four operators, each in its plain form (torch operations in 32 bits, the router's sums in 64) and,
where ``own`` is true, as the calls a user makes of ``paper_2607_18081_amd``:

``quant``  e4m3 codes and one float32 scale for each block of 1 x 128 (activations) or 128 x 128
           (weights): a = max |x| of the block (at least 2^-60), scale a / 448, code x * (448 / a)
``matmul`` y[m][n] = sum over the blocks b of 128 columns of xs[m][b] * ws[n // 128][b] * (the
           product of the codes of block b), x quantised by rows and w by 128 x 128
``route``  the k experts of each token by their router logits, ties to the lower expert, and their
           weights (softmax over the chosen, or sigmoid scores with a choice bias)
``layer``  the whole layer: router, gate and up products, SiLU(g) * u, down product, weighted sum
"""
import math

import torch

own = False

DEV = "cuda:0"
W_STD = 0.02
BLK = 128
E4M3_MAX = 448.0
AMAX_MIN = 2.0 ** -60
DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


def listed():
    return [
        # activations of a decode batch of 16 before a product: latency
        dict(name="quant_rows_16", op="quant", G=1, R=16, C=4096, br=1, dt="bf16"),
        # activations of a long prompt, an odd number of tokens
        dict(name="quant_rows_8191", op="quant", G=1, R=8191, C=5120, br=1, dt="bf16"),
        # the gate and up matrices of four experts, laid out once after loading
        dict(name="quant_weights", op="quant", G=8, R=11008, C=4096, br=128, dt="bf16"),
        # one token through a dense projection of the 8B-shape layer
        dict(name="matmul_1", op="matmul", M=1, N=14336, K=4096, out="bf16"),
        # a small serving batch, odd, with a ragged last tile of 128 rows
        dict(name="matmul_13", op="matmul", M=13, N=11000, K=4096, out="bf16"),
        # a short ragged prompt through the 7B-shape down projection, summed on in 32 bits
        dict(name="matmul_200", op="matmul", M=200, N=4096, K=11008, out="f32"),
        # a long prompt through the 8B-shape gate projection: the matrix cores' rate
        dict(name="matmul_4096", op="matmul", M=4096, N=14336, K=4096, out="bf16"),
        # the router of one token
        dict(name="route_1", op="route", T=1, E=128, k=8, d=2048, dt="bf16", score="softmax"),
        # the router of a batch with a choice bias (sigmoid scores)
        dict(name="route_200", op="route", T=200, E=256, k=8, d=5120, dt="bf16",
             score="sigmoid"),
        # one token through a layer of many small experts
        dict(name="layer_1", op="layer", T=1, E=128, k=8, d=2048, I=768, dt="bf16", w="same",
             out="bf16"),
        # an odd decode batch over 8-bit experts
        dict(name="layer_13_fp8", op="layer", T=13, E=64, k=6, d=4096, I=1408, dt="bf16",
             w="fp8", out="bf16"),
        # a larger batch over a few large experts
        dict(name="layer_48", op="layer", T=48, E=8, k=2, d=4096, I=14336, dt="bf16", w="same",
             out="bf16"),
    ]


def _log_int(rng, lo, hi, step=1):
    v = math.exp(rng.uniform(math.log(lo), math.log(hi)))
    return max(lo, min(hi // step * step, int(round(v / step)) * step))


def draw(rng):
    op = rng.choice(["quant", "matmul", "matmul", "route", "layer", "layer"])
    dt = rng.choice(["bf16", "bf16", "f16"])
    if op == "quant":
        R, C = _log_int(rng, 1, 16384), _log_int(rng, 256, 16384, 16)
        G = rng.randint(1, max(1, min(16, (8 * 11008 * 4096) // (R * C))))
        return dict(op=op, G=G, R=R, C=C, br=rng.choice([1, 128]),
                    dt=rng.choice(["bf16", "f16", "f32"]))
    if op == "matmul":
        N, K = _log_int(rng, 512, 16384), _log_int(rng, 512, 16384, 16)
        M = _log_int(rng, 1, 8192)
        M = max(1, min(M, 4096 * 14336 * 4096 // (N * K)))
        return dict(op=op, M=M, N=N, K=K, out=rng.choice(["bf16", "bf16", "f16", "f32"]))
    E = rng.choice([8, 16, 40, 64, 128, 256])
    k = rng.randint(1, min(10, E // 4))
    dt = rng.choice([dt, dt, dt, "f32"])
    if op == "route":
        return dict(op=op, T=_log_int(rng, 1, 512), E=E, k=k, d=_log_int(rng, 512, 8192, 8),
                    dt=dt, score=rng.choice(["softmax", "sigmoid"]))
    w = "same" if dt == "f32" else rng.choice(["same", "fp8"])
    most = 8 * 4096 * 14336 // (2 if dt == "f32" else 1)    # the largest listed layer's bytes
    d = _log_int(rng, 512, min(8192, most // (256 * E)), 16)
    inter = _log_int(rng, 256, min(16384, most // (E * d)), 16)
    return dict(op=op, T=_log_int(rng, 1, 256), E=E, k=k, d=d, I=inter, dt=dt, w=w,
                out=rng.choice([dt, dt, "f32"]))


# ---- inputs ------------------------------------------------------------------------------------

def _normal(g, dtype, std, *shape):
    return torch.empty(shape, dtype=dtype, device=DEV).normal_(0.0, std, generator=g)


def _blocks(n):
    return -(-n // BLK)


def _codes(g, *shape):
    """Codes of N(0, 1) values scaled so that a block's largest is near 448."""
    x = torch.empty(shape, dtype=torch.bfloat16, device=DEV).normal_(0.0, 120.0, generator=g)
    return x.clamp_(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn)


def _scales(g, std, *shape):
    """Block scales of values of that deviation, a few per cent apart as blocks' maxima are."""
    u = torch.rand(shape, dtype=torch.float32, device=DEV, generator=g)
    return (std / 120.0) * (0.85 + 0.3 * u)


def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(int(seed))
    op = case["op"]
    s = {"case": case}
    if op == "quant":
        std = 1.0 if case["br"] == 1 else W_STD
        s["x"] = _normal(g, DTYPES[case["dt"]], std, case["G"], case["R"], case["C"])
        return s
    if op == "matmul":
        M, N, K = case["M"], case["N"], case["K"]
        s["x"], s["xs"] = _codes(g, M, K), _scales(g, 1.0, M, _blocks(K))
        s["w"], s["ws"] = _codes(g, N, K), _scales(g, W_STD, _blocks(N), _blocks(K))
        return s
    dt, d, E = DTYPES[case["dt"]], case["d"], case["E"]
    s["x"] = _normal(g, dt, 1.0, case["T"], d)
    s["router"] = _normal(g, dt, 1.0 / math.sqrt(d), E, d)
    if op == "route":
        s["bias"] = None
        if case["score"] == "sigmoid":
            s["bias"] = _normal(g, torch.float32, 0.1, E)
        return s
    inter = case["I"]
    if case["w"] == "fp8":
        s["gate_up"], s["down"] = _codes(g, E, 2, inter, d), _codes(g, E, d, inter)
        s["gus"] = _scales(g, W_STD, E, 2, _blocks(inter), _blocks(d))
        s["dns"] = _scales(g, W_STD, E, _blocks(d), _blocks(inter))
    else:
        s["gate_up"] = _normal(g, dt, W_STD, E, 2, inter, d)
        s["down"] = _normal(g, dt, W_STD, E, d, inter)
        s["gus"] = s["dns"] = None
    return s


# ---- the plain forms -----------------------------------------------------------------------------

def _pad_blocks(x, br):
    G, R, C = x.shape
    pr, pc = -R % br, -C % BLK
    x = torch.nn.functional.pad(x, (0, pc, 0, pr))
    return x.view(G, (R + pr) // br, br, (C + pc) // BLK, BLK)


def _quant(s):
    case = s["case"]
    G, R, C, br = case["G"], case["R"], case["C"], case["br"]
    x = _pad_blocks(s["x"].float(), br)
    a = x.abs().amax(dim=(2, 4)).clamp_min(AMAX_MIN)
    q = x * (E4M3_MAX / a)[:, :, None, :, None]
    q = q.reshape(G, x.shape[1] * br, x.shape[3] * BLK)[:, :R, :C]
    return {"codes": q.to(torch.float8_e4m3fn), "scales": a / E4M3_MAX}


def _spread(scales, rows, cols, br):
    """Block scales [..., R/br, C/128] at every element [..., R, C]."""
    s = scales.repeat_interleave(BLK, dim=-1)[..., :cols]
    return s if br == 1 else s.repeat_interleave(br, dim=-2)[..., :rows, :]


def _matmul(s):
    M, N, K = s["case"]["M"], s["case"]["N"], s["case"]["K"]
    x = s["x"].float() * _spread(s["xs"], M, K, 1)
    w = s["w"].float() * _spread(s["ws"], N, K, BLK)
    return (x @ w.t()).to(DTYPES[s["case"]["out"]])


def _route(s):
    case = s["case"]
    z = s["x"].double() @ s["router"].double().t()
    sig = case.get("score", "softmax") == "sigmoid"
    p = torch.sigmoid(z) if sig else torch.softmax(z, dim=1)
    key = p + s["bias"].double() if sig else z
    # a stable sort: equal keys to the lower expert
    ids = torch.sort(key, dim=1, descending=True, stable=True).indices[:, : case["k"]]
    w = torch.gather(p, 1, ids)
    w = w / w.sum(dim=1, keepdim=True)
    return ids.to(torch.int32), w.float()


def _weights32(q, scales, dt):
    if scales is None:
        return q.float()
    return q.float() * _spread(scales, q.shape[-2], q.shape[-1], BLK)


def _layer(s):
    case = s["case"]
    T, E, k = case["T"], case["E"], case["k"]
    ids, w = _route(s)
    x, gu, dn, gus, dns = s["x"].float(), s["gate_up"], s["down"], s["gus"], s["dns"]
    fp8 = gus is not None
    if T * k < E:
        # few tokens: the chosen experts of each token, one (token, expert) pair a batch entry
        pick = ids.reshape(-1).long()
        raw = lambda t: (t.view(torch.uint8)[pick].view(t.dtype) if fp8 else t[pick])  # noqa: E731
        gup = _weights32(raw(gu), gus[pick] if fp8 else None, fp8)
        dnp = _weights32(raw(dn), dns[pick] if fp8 else None, fp8)
        xp = x.repeat_interleave(k, dim=0)[:, None, :, None]
        z = torch.matmul(gup, xp).squeeze(-1)                       # [T k][2][I]
        h = torch.nn.functional.silu(z[:, 0]) * z[:, 1]
        y = torch.bmm(dnp, h.unsqueeze(-1)).squeeze(-1)             # [T k][d]
        y = (y.view(T, k, -1) * w.unsqueeze(-1)).sum(dim=1)
    else:
        # many: every expert on every token, weighted by its share
        share = torch.zeros((T, E), device=x.device).scatter_(1, ids.long(), w)
        g32, d32 = _weights32(gu, gus, fp8), _weights32(dn, dns, fp8)
        z = (x @ g32.view(-1, x.shape[1]).t()).view(T, E, 2, -1)
        h = torch.nn.functional.silu(z[:, :, 0]) * z[:, :, 1] * share.unsqueeze(-1)
        y = torch.bmm(d32, h.permute(1, 2, 0).contiguous()).sum(dim=0).t()
    return {"y": y.to(DTYPES[case["out"]]).contiguous(), "ids": ids, "weights": w}


# ---- one pass ----------------------------------------------------------------------------------

def run(s):
    case = s["case"]
    op = case["op"]
    if not own:
        if op == "route":
            ids, w = _route(s)
            return {"ids": ids, "weights": w}
        return {"quant": _quant, "matmul": _matmul, "layer": _layer}[op](s)
    import paper_2607_18081_amd as si

    if op == "quant":
        codes, scales = si.quantize_fp8(s["x"], block_rows=case["br"])
        return {"codes": codes, "scales": scales}
    if op == "matmul":
        return si.matmul_fp8(s["x"], s["xs"], s["w"], s["ws"], out_dtype=DTYPES[case["out"]])
    if op == "route":
        ids, w = si.moe_route(s["x"], s["router"], case["k"], bias=s["bias"],
                              score=case["score"])
        return {"ids": ids, "weights": w}
    y, ids, w = si.moe_layer(s["x"], s["router"], s["gate_up"], s["down"], case["k"],
                             gate_up_scales=s["gus"], down_scales=s["dns"],
                             out_dtype=DTYPES[case["out"]])
    return {"y": y, "ids": ids, "weights": w}


# ---- what a pass cannot do without ---------------------------------------------------------------

def work(case):
    op = case["op"]
    size = {"bf16": 2, "f16": 2, "f32": 4}
    if op == "quant":
        n = case["G"] * case["R"] * case["C"]
        blocks = case["G"] * -(-case["R"] // case["br"]) * _blocks(case["C"])
        return {"bytes": n * (size[case["dt"]] + 1) + 4 * blocks, "flops": 0}
    if op == "matmul":
        M, N, K = case["M"], case["N"], case["K"]
        scales = 4 * _blocks(K) * (M + _blocks(N))
        return {"bytes": M * K + N * K + scales + M * N * size[case["out"]],
                "flops": 2.0 * M * N * K}
    T, E, k, d = case["T"], case["E"], case["k"], case["d"]
    es = size[case["dt"]]
    route = {"bytes": (T + E) * d * es + 8 * T * k, "flops": 2.0 * T * E * d}
    if op == "route":
        return route
    inter = case["I"]
    # distinct experts of T tokens that choose k of E each, expected
    experts = E * (1.0 - (1.0 - k / E) ** T)
    if case["w"] == "fp8":
        expert = 3 * d * inter + 4 * 3 * _blocks(d) * _blocks(inter)
    else:
        expert = 3 * d * inter * es
    return {"bytes": route["bytes"] + experts * expert + T * d * size[case["out"]],
            "flops": route["flops"] + 6.0 * T * k * d * inter}


# ---- the same in 64 bits -------------------------------------------------------------------------

def _exact_quant(x, br):
    G, R, C = x.shape
    nr, nc = -(-R // br), _blocks(C)
    scales = torch.empty((G, nr, nc), dtype=torch.float64, device=DEV)
    vals = torch.empty((G, R, C), dtype=torch.float64, device=DEV)
    for g in range(G):
        xg = torch.zeros((nr * br, nc * BLK), dtype=torch.float64, device=DEV)
        xg[:R, :C] = x[g].double()
        xb = xg.view(nr, br, nc, BLK).permute(0, 2, 1, 3)
        a = torch.clamp(xb.reshape(nr, nc, -1).abs().max(dim=2).values, min=AMAX_MIN)
        scales[g] = a / E4M3_MAX
        v = (xb / scales[g][:, :, None, None]).permute(0, 2, 1, 3).reshape(nr * br, nc * BLK)
        v = v[:R, :C]
        # e4m3: steps of 2^(e - 3) from 2^-6 up, of 2^-9 below
        e = torch.floor(torch.log2(v.abs().clamp_min(2.0 ** -6)))
        step = torch.exp2(e - 3.0)
        vals[g] = torch.round(v / step) * step
    return {"codes": vals, "scales": scales}


def _exact_matmul(s):
    x, w, K = s["x"].double(), s["w"].double(), s["case"]["K"]
    y = torch.zeros((x.shape[0], w.shape[0]), dtype=torch.float64, device=DEV)
    for b in range(_blocks(K)):
        lo, hi = b * BLK, min(K, (b + 1) * BLK)
        row = s["ws"][:, b].double()[torch.arange(w.shape[0], device=DEV) // BLK]
        y += (x[:, lo:hi] @ w[:, lo:hi].t()) * s["xs"][:, b].double()[:, None] * row[None, :]
    return y


def _exact_weights(s):
    """Weights of the chosen experts; the choice itself is whole numbers and stays out."""
    case = s["case"]
    z = s["x"].double() @ s["router"].double().t()
    if case.get("score") == "sigmoid":
        p = 1.0 / (1.0 + torch.exp(-z))
        key = p + s["bias"].double()
    else:
        p = torch.exp(z - z.max(dim=1, keepdim=True).values)
        key = z
    order = torch.argsort(key, dim=1, descending=True, stable=True)[:, : case["k"]]
    chosen = torch.gather(p, 1, order)
    return order, chosen / chosen.sum(dim=1, keepdim=True)


def _expert64(t, scales, e):
    if scales is None:
        return t[e].double()
    w = t[e].to(torch.float32).double()
    r = torch.arange(w.shape[-2], device=DEV) // BLK
    c = torch.arange(w.shape[-1], device=DEV) // BLK
    return w * scales[e].double()[..., r, :][..., c]


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "quant":
        return _exact_quant(s["x"], case["br"])
    if op == "matmul":
        return _exact_matmul(s)
    order, w = _exact_weights(s)
    if op == "route":
        return {"ids": None, "weights": w}
    x = s["x"].double()
    y = torch.zeros((case["T"], case["d"]), dtype=torch.float64, device=DEV)
    for e in range(case["E"]):
        tok, rank = torch.nonzero(order == e, as_tuple=True)
        if tok.numel():
            gu = _expert64(s["gate_up"], s["gus"], e)
            g, u = x[tok] @ gu[0].t(), x[tok] @ gu[1].t()
            h = g / (1.0 + torch.exp(-g)) * u
            y[tok] += w[tok, rank][:, None] * (h @ _expert64(s["down"], s["dns"], e).t())
    return {"y": y, "ids": None, "weights": w}
