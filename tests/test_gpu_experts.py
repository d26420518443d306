"""The mixture-of-experts router and layer against the float64 oracle.

Router: a logit is off by at most 33 2^-23 sum |x| |w| (float32 sums of up to 32 products, float64
beyond), so the key of the expert at each rank lies within twice that of the sorted key there; on
data whose sums are exact in float32 the choice is compared exactly, ties included.
Layer: the oracle carries the bound of float32 arithmetic through (oracle.moe_ffn), h entering the
down product with 2^-16 of its value (bf16 pair), 2^-24 (three bf16 parts, float32) or 2^-22 and
2^-28 absolutely (half pair), and the output half a step of its type.
"""
import math

import numpy as np
import pytest
import torch

import oracle
import paper_2607_18081_amd as si
from tests.gpu_util import say

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
HALF_STEP = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
DT = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def _np(t):
    return t.double().cpu().numpy()


# ---- router ----------------------------------------------------------------------------------

def _check_route(x, w, k, ids, weights, **kw):
    n = kw.get("n_valid")
    ref_ids, ref_w, keys = oracle.moe_route(_np(x), _np(w), k, **kw)
    slack = 2 * 33 * 2.0 ** -23 * np.max(np.abs(_np(x)) @ np.abs(_np(w)).T, axis=1)
    ids, weights = ids.cpu().numpy(), _np(weights)
    for t in range(x.shape[0]):
        if n is not None and t >= n:
            assert np.all(ids[t] == -1) and np.all(weights[t] == 0)
            continue
        assert len(set(ids[t])) == k and ids[t].min() >= 0 and ids[t].max() < w.shape[0]
        # sigmoid and softmax have slopes of at most 1
        assert np.all(np.abs(keys[t][ids[t]] - keys[t][ref_ids[t]]) <= slack[t])
        if np.array_equal(ids[t], ref_ids[t]):
            # d ln p and d ln of a sum of p are at most twice the largest logit error each
            tol = np.abs(ref_w[t]) * (4 * slack[t] + 2.0 ** -23)
            assert np.all(np.abs(weights[t] - ref_w[t]) <= tol)


@pytest.mark.parametrize("T,E,k,d,xdt,wdt", [
    (1, 1, 1, 8, "bf16", "bf16"), (1, 8, 2, 264, "bf16", "f32"), (1, 128, 8, 2048, "bf16", "bf16"),
    (3, 40, 6, 520, "f16", "f16"), (7, 64, 6, 4096, "f16", "f32"), (16, 256, 8, 1032, "bf16", "bf16"),
    (17, 65, 10, 516, "f32", "f32"), (33, 1024, 32, 136, "bf16", "bf16"), (70, 17, 17, 72, "f32", "f32"),
    (130, 100, 4, 640, "bf16", "f32"), (600, 16, 2, 64, "f16", "f16"),
])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
def test_route(T, E, k, d, xdt, wdt, score):
    say(f"route T={T} E={E} k={k} d={d} {xdt} {wdt} {score}")
    g = torch.Generator().manual_seed(T + E + d)
    x = torch.randn(T, d, generator=g).to(DT[xdt]).to(DEV)
    w = (torch.randn(E, d, generator=g) / d ** 0.5).to(DT[wdt]).to(DEV)
    bias = None if score == "softmax" else (0.2 * torch.randn(E, generator=g)).to(DEV)
    b = None if bias is None else bias.cpu().numpy()
    ids, weights = si.moe_route(x, w, k, bias=bias, score=score)
    _check_route(x, w, k, ids, weights, bias=b, score=score)
    ids2, weights2 = si.moe_route(x, w, k, bias=bias, score=score, renorm=False, scale=2.5)
    assert torch.equal(ids2, ids)
    _check_route(x, w, k, ids2, weights2, bias=b, score=score, renorm=False, scale=2.5)


@pytest.mark.parametrize("T,E,k", [(1, 24, 3), (9, 300, 5)])
@pytest.mark.parametrize("score,biased", [("softmax", True), ("sigmoid", False)])
def test_route_modes(T, E, k, score, biased):
    """A choice bias on softmax scores, sigmoid scores without one; weights with and without their
    sum, and scaled; the same from the whole layer, which makes the choice elsewhere."""
    say(f"route modes T={T} E={E} {score} bias={biased}")
    g = torch.Generator().manual_seed(E)
    x = torch.randn(T, 64, generator=g).to(torch.bfloat16).to(DEV)
    w = (torch.randn(E, 64, generator=g) / 8).to(DEV)
    bias = (0.3 * torch.randn(E, generator=g)).to(DEV) if biased else None
    gu = torch.zeros(E, 2, 16, 64, dtype=torch.bfloat16, device=DEV)
    dn = torch.zeros(E, 64, 16, dtype=torch.bfloat16, device=DEV)
    for renorm, scale in ((True, 1.0), (True, -2.0), (False, 0.5)):
        kw = dict(bias=bias, score=score, renorm=renorm, scale=scale)
        ids, weights = si.moe_route(x, w, k, **kw)
        ref = dict(kw, bias=None if bias is None else bias.cpu().numpy())
        _check_route(x, w, k, ids, weights, **ref)
        _, ids2, weights2 = si.moe_layer(x, w, gu, dn, k, **kw)
        assert torch.equal(ids2, ids) and torch.equal(weights2, weights)


@pytest.mark.parametrize("xdt", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("T,E,k,d", [(1, 16, 4, 64), (5, 200, 20, 320), (40, 1000, 32, 1040)])
def test_route_ties(T, E, k, d, xdt):
    """Small whole numbers: every sum is exact, many logits are equal, the lower expert wins."""
    say(f"route ties T={T} E={E} {xdt}")
    rng = np.random.default_rng(E)
    x = torch.from_numpy(rng.integers(-1, 2, (T, d)).astype(np.float32)).to(DT[xdt]).to(DEV)
    w = torch.from_numpy(rng.integers(-1, 2, (E, d)).astype(np.float32))
    w[E // 2:] = w[: E - E // 2]                              # every row at least twice
    w = w.to(DT[xdt]).to(DEV)
    ids, _ = si.moe_route(x, w, k)
    want, _, _ = oracle.moe_route(_np(x), _np(w), k)
    assert np.array_equal(ids.cpu().numpy(), want)
    ids, weights = si.moe_route(torch.zeros_like(x), w, k)    # all logits equal
    assert np.array_equal(ids.cpu().numpy(), np.tile(np.arange(k), (T, 1)))
    assert torch.equal(weights, torch.full_like(weights, 1.0 / k))


def test_route_values_out_of_range():
    """NaN logits rank last, infinite ones first or last; the padded rows of a batch are left
    alone whatever they hold."""
    say("route NaN, infinities and padding")
    w = torch.zeros(6, 8, device=DEV)
    w[:, 0] = torch.tensor([0.0, 3.0, float("nan"), -1.0, 3.0, float("inf")])
    x = torch.zeros(4, 8, device=DEV)
    x[:, 0] = torch.tensor([1.0, -1.0, float("nan"), 1.0])
    ids, weights = si.moe_route(x, w, 6, score="sigmoid", renorm=False)
    ids, weights = ids.cpu().numpy(), weights.cpu().numpy()
    assert ids[0].tolist() == [5, 1, 4, 0, 3, 2] and weights[0, 0] == 1.0
    assert ids[1].tolist() == [3, 0, 1, 4, 5, 2] and weights[1, 4] == 0.0
    assert ids[2].tolist() == [0, 1, 2, 3, 4, 5] and np.all(np.isnan(weights[2]))
    assert np.isnan(weights[0, 5]) and not np.any(np.isnan(weights[0, :5]))
    x[2:] = float("nan")
    wf = torch.randn(6, 8, device=DEV)
    n = torch.tensor([2], dtype=torch.int32, device=DEV)
    ids, weights = si.moe_route(x, wf, 2, n_valid=n)
    _check_route(torch.nan_to_num(x), wf, 2, ids, weights, n_valid=2)
    n.fill_(0)
    ids, weights = si.moe_route(x, wf, 2, n_valid=n)
    assert torch.all(ids == -1) and torch.all(weights == 0)


# ---- experts ---------------------------------------------------------------------------------

def _experts(E, d, inter, dt, wkind, seed):
    """Device weights and what they stand for in float64."""
    g = torch.Generator().manual_seed(seed)
    gu = torch.randn(E, 2, inter, d, generator=g) / d ** 0.5
    dn = torch.randn(E, d, inter, generator=g) / inter ** 0.5
    if wkind != "fp8":
        gu, dn = gu.to(DT[dt]), dn.to(DT[dt])
        return (gu.to(DEV), dn.to(DEV), None, None), gu.double().numpy(), dn.double().numpy()
    dev, ref = [], []
    for w in (gu, dn):
        q, s = si.quantize_fp8(w.to(DEV), block_rows=128)
        dev.append((q, s))
        R, C = w.shape[-2:]
        full = np.stack([oracle.spread(m, R, C, 128) for m in
                         s.cpu().numpy().reshape(-1, *s.shape[-2:])]).reshape(w.shape)
        ref.append(oracle.decode_e4m3(q.view(torch.uint8).cpu().numpy()) * full)
    return (dev[0][0], dev[1][0], dev[0][1], dev[1][1]), ref[0], ref[1]


def _h_err(dt, wkind, out):
    if dt == "f32":
        return 2.0 ** -24, 0.0
    if dt == "f16" and wkind != "fp8":
        return 2.0 ** -22, 2.0 ** -28
    return (2.0 ** -24 if out == torch.float32 else 2.0 ** -16), 0.0


def _check_layer(y, x, ids, weights, gu, dn, dt, wkind):
    rel, ab = _h_err(dt, wkind, y.dtype)
    want, bound = oracle.moe_ffn(_np(x), ids.cpu().numpy(), _np(weights), gu, dn, rel, ab)
    tol = bound + HALF_STEP[y.dtype] * (np.abs(want) + bound)
    if y.dtype == torch.float16:
        tol = tol + 2.0 ** -25
    err = np.abs(_np(y) - want)
    assert np.all(err <= tol), float(np.max(err / np.maximum(tol, 1e-300)))


LAYERS = [
    # T, E, k, d, I
    (1, 8, 2, 64, 48), (1, 4, 4, 272, 16), (2, 16, 3, 128, 400), (5, 6, 6, 144, 144),
    (13, 64, 6, 256, 208), (16, 2, 1, 528, 336), (17, 1, 1, 64, 32), (40, 3, 2, 160, 272),
    (70, 2, 2, 96, 64), (130, 5, 1, 64, 128),
    # one token: a choice of its own launch, h past the LDS kept for it, x past it, many ranks
    (1, 300, 3, 64, 48), (1, 200, 6, 64, 2064), (1, 16, 10, 4368, 32), (1, 256, 32, 256, 16),
    # long rows; the most tokens and pairs
    (3, 4, 2, 8208, 16), (3, 4, 2, 48, 8208), (512, 20, 16, 64, 32),
    (480, 16, 16, 64, 32),
    # many tokens an expert, over several lines of both products: one, two and more passes, the
    # last of up to 32 tokens and of more
    (90, 2, 2, 400, 272), (200, 3, 1, 1040, 528), (100, 3, 1, 144, 1552), (170, 2, 1, 784, 144),
    (45, 3, 1, 656, 400), (33, 4, 2, 272, 80),
]


@pytest.mark.parametrize("dt,wkind", [("bf16", "same"), ("f16", "same"), ("f32", "same"),
                                      ("bf16", "fp8"), ("f16", "fp8")])
@pytest.mark.parametrize("T,E,k,d,inter", LAYERS)
def test_layer(T, E, k, d, inter, dt, wkind):
    say(f"layer T={T} E={E} k={k} d={d} I={inter} {dt} {wkind}")
    dev, gu, dn = _experts(E, d, inter, dt, wkind, T + d)
    g = torch.Generator().manual_seed(T * 3 + E)
    x = torch.randn(T, d, generator=g).to(DT[dt]).to(DEV)
    w = (torch.randn(E, d, generator=g) / d ** 0.5).to(DT[dt]).to(DEV)
    for out in {torch.float32, DT[dt]}:
        y = torch.full((T, d), float("nan"), dtype=out, device=DEV)
        y, ids, weights = si.moe_layer(x, w, dev[0], dev[1], k, gate_up_scales=dev[2],
                                       down_scales=dev[3], y=y, out_dtype=out)
        _check_route(x, w, k, ids, weights)
        _check_layer(y, x, ids, weights, gu, dn, dt, wkind)
        # the two calls on their own give the same bits, and again the same
        ids2, weights2 = si.moe_route(x, w, k)
        assert torch.equal(ids2, ids) and torch.equal(weights2, weights)
        y2 = si.moe_ffn(x, ids, weights, dev[0], dev[1], gate_up_scales=dev[2],
                        down_scales=dev[3], out_dtype=out)
        assert torch.equal(y2, y)


@pytest.mark.parametrize("dt,wkind", [("bf16", "same"), ("f16", "same"), ("f32", "same"),
                                      ("bf16", "fp8")])
@pytest.mark.parametrize("T", [1, 4, 33, 100])
def test_caller_ids(T, dt, wkind):
    """Ids of the caller's own: none, outside [0, E), one expert twice for a token, every token on
    one expert (more than one pass over its weights), weights that are NaN where the id is not."""
    say(f"ids of the caller T={T} {dt} {wkind}")
    E, d, inter, k = 5, 96, 80, 4
    dev, gu, dn = _experts(E, d, inter, dt, wkind, T)
    rng = np.random.default_rng(T)
    x = torch.randn(T, d, generator=torch.Generator().manual_seed(T)).to(DT[dt]).to(DEV)
    ids = rng.integers(-2, E + 2, (T, k)).astype(np.int32)
    ids[0] = [-1, E, 2 ** 31 - 1, -2 ** 31]                   # a token without an expert
    if T > 1:
        ids[1] = [3, 3, 3, -1]
        ids[2:] = np.where(rng.random((T - 2, k)) < 0.5, 3, ids[2:])
    weights = rng.normal(0, 1, (T, k)).astype(np.float32)
    weights[(ids < 0) | (ids >= E)] = np.nan
    run = lambda i, w: si.moe_ffn(x, torch.from_numpy(i).to(DEV), torch.from_numpy(w).to(DEV),  # noqa: E731
                                  dev[0], dev[1], gate_up_scales=dev[2], down_scales=dev[3])
    y = run(ids, weights)
    assert torch.all(y[0] == 0)
    _check_layer(y, x, torch.from_numpy(ids), torch.from_numpy(weights), gu, dn, dt, wkind)
    none = np.full_like(ids, -1)
    assert torch.all(run(none, weights) == 0)
    one = np.full((T, k), -1, dtype=np.int32)
    one[:, 1] = 4
    _check_layer(run(one, weights), x, torch.from_numpy(one), torch.from_numpy(
        np.where(one < 0, 0, weights)), gu, dn, dt, wkind) if not np.isnan(weights[:, 1]).any() \
        else None


@pytest.mark.parametrize("T", [20, 150])
def test_values_stay_in_their_token(T):
    """NaN and infinities of a token, or of an expert, reach only the tokens that use them."""
    say(f"layer: NaN and infinities T={T}")
    E, d, inter, k = 4, 64, 48, 1
    dev, gu, dn = _experts(E, d, inter, "bf16", "same", 1)
    x = torch.randn(T, d, generator=torch.Generator().manual_seed(1)).to(torch.bfloat16).to(DEV)
    ids = (torch.arange(T, dtype=torch.int32, device=DEV) % E).view(T, 1)
    weights = torch.ones(T, 1, device=DEV)
    clean = si.moe_ffn(x, ids, weights, dev[0], dev[1])
    x[3], x[8, 5] = float("nan"), float("inf")
    dev[0][2, 1, 7, 9] = float("nan")
    y = si.moe_ffn(x, ids, weights, dev[0], dev[1])
    touched = torch.zeros(T, dtype=torch.bool, device=DEV)
    touched[3], touched[8] = True, True
    touched |= ids[:, 0] == 2
    assert torch.equal(y[~touched], clean[~touched])
    assert torch.all(torch.isnan(y[3])) and torch.all(torch.isnan(y[ids[:, 0] == 2]))
    assert not torch.any(torch.isfinite(y[8]))


@pytest.mark.parametrize("T", [1, 5, 70])
def test_nan_codes(T):
    """A NaN code, or a NaN scale, of an 8-bit expert reaches the tokens that use it and no other."""
    say(f"layer: NaN codes T={T}")
    E, d, inter = 3, 64, 48
    dev, _, _ = _experts(E, d, inter, "bf16", "fp8", 9)
    x = torch.randn(T, d, generator=torch.Generator().manual_seed(T)).to(torch.bfloat16).to(DEV)
    run = lambda e: si.moe_ffn(x, torch.full((T, 1), e, dtype=torch.int32, device=DEV),  # noqa: E731
                               torch.ones(T, 1, device=DEV), dev[0], dev[1], dev[2], dev[3])
    clean = run(0)
    dev[0].view(torch.uint8)[1, 0, 3, 5] = 0x7f
    dev[3][2, 0, 0] = float("nan")
    assert torch.equal(run(0), clean)
    assert torch.all(torch.isnan(run(1))) and torch.all(torch.isnan(run(2)))


@pytest.mark.parametrize("dt,T", [("f16", 9), ("bf16", 9), ("f16", 75), ("bf16", 75)])
def test_large_and_small_h(dt, T):
    """h from 2^-20 to 2^20: beyond what one half value holds at either end."""
    say(f"layer: large and small h {dt} T={T}")
    E, d, inter = 1, 64, 64
    g = torch.Generator().manual_seed(2)
    gu = torch.randn(E, 2, inter, d, generator=g).to(DT[dt])
    dn = (torch.randn(E, d, inter, generator=g) / 8).to(DT[dt])
    x = torch.randn(T, d, generator=g)
    x = (x * torch.exp2(torch.linspace(-14, 8, T)).view(T, 1)).to(DT[dt])
    ids = torch.zeros(T, 1, dtype=torch.int32)
    weights = torch.ones(T, 1)
    y = si.moe_ffn(x.to(DEV), ids.to(DEV), weights.to(DEV), gu.to(DEV), dn.to(DEV))
    # half weights promise |h| < 2^24 (one token of the 75 lies past it, at 2^24.2)
    G, U = (x.double() @ gu[0, i].double().t() for i in (0, 1))
    ok = (G / (1 + torch.exp(-G)) * U).abs().amax(dim=1) < (2.0 ** 24 if dt == "f16" else math.inf)
    assert int((~ok).sum()) == (1 if (dt, T) == ("f16", 75) else 0)
    assert torch.all(torch.isfinite(y[ok.to(DEV)]))
    _check_layer(y[ok.to(DEV)], x[ok], ids[ok], weights[ok], gu.double().numpy(),
                 dn.double().numpy(), dt, "same")


@pytest.mark.parametrize("T,dt,wkind", [(1, "bf16", "same"), (6, "bf16", "fp8"), (90, "f16", "same")])
def test_graph_and_streams(T, dt, wkind):
    """A captured layer replayed with eager work between gives the eager bits; two captured layers
    and two streams at once share nothing."""
    say(f"layer in graphs and on streams T={T} {dt} {wkind}")
    E, d, inter, k = 8, 256, 144, 2
    dev, _, _ = _experts(E, d, inter, dt, wkind, T)
    g = torch.Generator().manual_seed(T)
    xs = [torch.randn(T, d, generator=g).to(DT[dt]).to(DEV) for _ in range(2)]
    w = (torch.randn(E, d, generator=g) / d ** 0.5).to(DT[dt]).to(DEV)
    run = lambda x, y=None: si.moe_layer(x, w, dev[0], dev[1], k, gate_up_scales=dev[2],  # noqa: E731
                                         down_scales=dev[3], y=y)[0]
    want = [run(x) for x in xs]
    torch.cuda.synchronize()
    graphs, outs = [], []
    for x in xs:
        y = torch.empty_like(want[0])
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            run(x, y)
        graphs.append(graph)
        outs.append(y)
    side = [torch.cuda.Stream() for _ in range(2)]
    for rep in range(3):
        for y in outs:
            y.fill_(float("nan"))
        torch.cuda.synchronize()
        for s, graph in zip(side, graphs):
            with torch.cuda.stream(s):
                graph.replay()
        torch.cuda.synchronize()
        for y, ref in zip(outs, want):
            assert torch.equal(y, ref), rep
        eager = []
        for s, x in zip(side, xs):
            with torch.cuda.stream(s):
                eager.append([run(x) for _ in range(3)])
        torch.cuda.synchronize()
        assert all(torch.equal(y, ref) for ys, ref in zip(eager, want) for y in ys)


def test_padded_batch():
    """A batch padded to a captured size: n_valid on the device says how many rows count, and may
    change between replays."""
    say("layer: padded batch")
    T, E, d, inter, k = 12, 8, 128, 64, 2
    dev, gu, dn = _experts(E, d, inter, "bf16", "same", 4)
    g = torch.Generator().manual_seed(4)
    x = torch.randn(T, d, generator=g).to(torch.bfloat16).to(DEV)
    w = (torch.randn(E, d, generator=g) / 11).to(torch.bfloat16).to(DEV)
    whole, _, _ = si.moe_layer(x, w, dev[0], dev[1], k)
    n = torch.tensor([T], dtype=torch.int32, device=DEV)
    y = torch.empty(T, d, device=DEV)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        _, ids, weights = si.moe_layer(x, w, dev[0], dev[1], k, n_valid=n, y=y)
    for valid in (12, 5, 0, 1):
        n.fill_(valid)
        y.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y[:valid], whole[:valid]) and torch.all(y[valid:] == 0)
        assert torch.all(ids[valid:] == -1)


def test_beside_the_selective_ffn():
    """A layer stack's step with both: an expert layer whose one expert holds a compacted layer's
    neurons equals the selective FFN over all of them, then the residual norm feeds the next."""
    say("experts beside the selective FFN")
    N, d, L, T = 96, 128, 64, 3
    g = torch.Generator().manual_seed(8)
    wg, wu = (torch.randn(N, d, generator=g).to(torch.bfloat16).to(DEV) / 11 for _ in range(2))
    wd = torch.randn(d, N, generator=g).to(torch.bfloat16).to(DEV) / 10
    loaded = torch.randperm(N, generator=g)[:L]
    layer = si.compact_ffn(wg, wu, wd, loaded)
    x = torch.randn(T, d, generator=g).to(torch.bfloat16).to(DEV)
    off = torch.arange(0, (T + 1) * L, L, dtype=torch.int32, device=DEV)
    idx = torch.arange(L, dtype=torch.int32, device=DEV).repeat(T)
    a = si.selective_ffn(x, off, idx, layer.gate_up_c, layer.down_c)
    gate_up = layer.gate_up_c.transpose(0, 1).contiguous().unsqueeze(0)
    down = layer.down_c.t().contiguous().unsqueeze(0)
    ids = torch.zeros(T, 1, dtype=torch.int32, device=DEV)
    b = si.moe_ffn(x, ids, torch.ones(T, 1, device=DEV), gate_up, down)
    _check_layer(b, x, ids, torch.ones(T, 1), _np(gate_up), _np(down), "bf16", "same")
    _check_layer(a, x, ids, torch.ones(T, 1), _np(gate_up), _np(down), "bf16", "same")
    xn = si.residual_rmsnorm(x, b)
    wr = torch.randn(1, d, generator=g).to(torch.bfloat16).to(DEV)
    y, ids, weights = si.moe_layer(xn, wr, gate_up, down, 1)
    assert torch.all(weights == 1)
    _check_layer(y, xn, ids, weights, _np(gate_up), _np(down), "bf16", "same")


def test_binding_refusals():
    say("experts: binding refusals")
    dev, _, _ = _experts(4, 64, 48, "bf16", "same", 0)
    q, _, _ = _experts(4, 64, 48, "bf16", "fp8", 0)
    x = torch.zeros(3, 64, dtype=torch.bfloat16, device=DEV)
    w = torch.zeros(4, 64, dtype=torch.bfloat16, device=DEV)
    ids = torch.zeros(3, 2, dtype=torch.int32, device=DEV)
    wt = torch.zeros(3, 2, device=DEV)
    bad = ValueError
    for call, err in (
            (lambda: si.moe_route(x, w, 5), si.SelectInferError),
            (lambda: si.moe_route(x, w, 0), si.SelectInferError),
            (lambda: si.moe_route(x, w.half(), 2), bad),
            (lambda: si.moe_route(x.t(), w, 2), bad),
            (lambda: si.moe_route(x, w, 2, score="tanh"), KeyError),
            (lambda: si.moe_route(x, w, 2, bias=torch.zeros(3, device=DEV)), bad),
            (lambda: si.moe_route(x, w, 2, n_valid=torch.zeros(1, device=DEV)), bad),
            (lambda: si.moe_route(x, w, 2, workspace=torch.empty(8, dtype=torch.uint8, device=DEV)),
             si.SelectInferError),
            (lambda: si.moe_ffn(x, ids.long(), wt, dev[0], dev[1]), bad),
            (lambda: si.moe_ffn(x, ids, wt.half(), dev[0], dev[1]), bad),
            (lambda: si.moe_ffn(x, ids, wt, dev[0], dev[1].transpose(1, 2)), bad),
            (lambda: si.moe_ffn(x, ids, wt, dev[0], dev[1][:3]), bad),
            (lambda: si.moe_ffn(x, ids, wt, q[0], q[1]), bad),
            (lambda: si.moe_ffn(x, ids, wt, q[0], q[1], q[2], q[3][:2]), bad),
            (lambda: si.moe_ffn(x, ids, wt, dev[0], dev[1], q[2], q[3]), bad),
            (lambda: si.moe_ffn(x, ids, wt, dev[0], dev[1], out_dtype=torch.float16),
             si.SelectInferError),
            (lambda: si.moe_ffn(x.cpu(), ids, wt, dev[0], dev[1]), bad),
            (lambda: si.moe_ffn(x, ids, wt, dev[0].cpu(), dev[1]), bad),
            (lambda: si.moe_layer(x, w[:3], dev[0], dev[1], 2), bad)):
        with pytest.raises(err):
            call()
    big = torch.zeros(513, 64, dtype=torch.bfloat16, device=DEV)
    with pytest.raises(si.SelectInferError):
        si.moe_layer(big, w, dev[0], dev[1], 2)
    y, ids, wt = si.moe_layer(x[:0], w, dev[0], dev[1], 2)
    assert y.shape == (0, 64) and ids.shape == (0, 2)
