"""Expert layers at the ends of their value range: half weights with small, large and mixed h.

h of half weights enters the down product as two half parts of h * 2^e, e by the pair's largest |h|
so that it lies in [2^14, 2^15): 22 bits of each value down to 2^-13, and below that a step of
2^-35 (the second part's subnormal step, 2^-24 / 2^11), half of it 2^-36: 2^-50 of the largest |h|.
"""
import numpy as np
import pytest
import torch

import oracle
import paper_2607_18081_amd as si
from tests.gpu_util import say
from tests.test_gpu_experts import DEV, HALF_STEP, _np

pytestmark = pytest.mark.gpu


def _largest_h(x, gate_up, ids):
    """Largest |h| of each (token, rank)."""
    out = np.zeros(ids.shape)
    for t, row in enumerate(ids):
        for r, e in enumerate(row):
            if 0 <= e < gate_up.shape[0]:
                g, u = gate_up[e, 0] @ x[t], gate_up[e, 1] @ x[t]
                with np.errstate(over="ignore"):
                    out[t, r] = np.max(np.abs(g / (1.0 + np.exp(-g)) * u))
    return out


def _check(y, x, ids, weights, gate_up, down):
    """Every token of y against the oracle, a (token, rank) at a time with its own error of h."""
    got, half = _np(y), HALF_STEP[y.dtype]
    top = _largest_h(x, gate_up, ids)
    worst = 0.0
    for t in range(len(x)):
        want, tol, size = (np.zeros(x.shape[1]) for _ in range(3))
        for r in range(ids.shape[1]):
            with np.errstate(over="ignore"):
                a, b = oracle.moe_ffn(x[t: t + 1], ids[t: t + 1, r: r + 1],
                                      weights[t: t + 1, r: r + 1], gate_up, down, 2.0 ** -22,
                                      2.0 ** -50 * top[t, r])
            want, tol, size = want + a[0], tol + b[0], size + np.abs(a[0])
        # the sum over the ranks rounds too
        tol = tol + ids.shape[1] * 2.0 ** -23 * (size + tol)
        tol = tol + half * (np.abs(want) + tol) + (2.0 ** -25 if half == 2.0 ** -11 else 2.0 ** -149)
        err = np.abs(got[t] - want)
        assert np.all(err <= tol), (t, float(np.max(err / tol)))
        worst = max(worst, float(np.max(err / tol)))
    return worst


# T, E, k, d, I: one token (h in LDS; past the LDS kept for it; x past it; fewer ranks than waves
# and more), few tokens an expert, many, and several passes of many
SHAPES = [(1, 4, 2, 64, 48), (1, 12, 10, 96, 400), (1, 3, 2, 48, 8208), (1, 3, 2, 4368, 64),
          (1, 2, 1, 64, 4112), (5, 6, 2, 128, 144), (40, 2, 1, 64, 80), (150, 1, 1, 64, 144)]


@pytest.mark.parametrize("x_std,g_std", [(1.0, 0.02), (0.1, 0.02), (0.01, 0.02), (0.001, 0.02),
                                         (0.001, 0.001), (300.0, 8.0)])
@pytest.mark.parametrize("T,E,k,d,inter", SHAPES)
def test_half_weights_keep_small_h(T, E, k, d, inter, x_std, g_std):
    """rms h from 2^-35 to past 2^24: the float32 result keeps 22 bits of h whatever its size."""
    say(f"small h T={T} E={E} k={k} d={d} I={inter} x {x_std} gate {g_std}")
    g = torch.Generator().manual_seed(T + d + inter)
    gu = (torch.randn(E, 2, inter, d, generator=g) * g_std).to(torch.float16)
    dn = (torch.randn(E, d, inter, generator=g) * 0.02).to(torch.float16)
    x = (torch.randn(T, d, generator=g) * x_std).to(torch.float16)
    ids = torch.stack([torch.randperm(E, generator=g)[:k] for _ in range(T)]).to(torch.int32)
    weights = torch.rand(T, k, generator=g) + 0.1
    y = si.moe_ffn(x.to(DEV), ids.to(DEV), weights.to(DEV), gu.to(DEV), dn.to(DEV))
    worst = _check(y, _np(x), ids.numpy(), _np(weights), _np(gu), _np(dn))
    say(f"worst error / bound {worst:.3f}")


@pytest.mark.parametrize("out", [torch.float32, torch.float16])
@pytest.mark.parametrize("T", [6, 33, 130])
def test_half_weights_mixed_sizes(T, out):
    """Tokens whose h differ by 2^38 side by side, each held to its own bound; a token whose h is
    all zero, and one without an expert."""
    say(f"mixed h T={T} {out}")
    E, d, inter, k = 2, 64, 96, 2
    g = torch.Generator().manual_seed(T)
    gu = (torch.randn(E, 2, inter, d, generator=g) * 0.25).to(torch.float16)
    dn = (torch.randn(E, d, inter, generator=g) * 2).to(torch.float16)
    size = torch.exp2(torch.linspace(-16, 3, T)).view(T, 1)
    x = (torch.randn(T, d, generator=g) * size).to(torch.float16)
    x[2] = 0.0
    ids = torch.tensor([[0, 1]], dtype=torch.int32).repeat(T, 1)
    ids[3] = torch.tensor([-1, E])
    weights = torch.rand(T, k, generator=g) + 0.1
    y = si.moe_ffn(x.to(DEV), ids.to(DEV), weights.to(DEV), gu.to(DEV), dn.to(DEV), out_dtype=out)
    assert torch.all(y[2] == 0) and torch.all(y[3] == 0)
    _check(y, _np(x), ids.numpy(), _np(weights), _np(gu), _np(dn))


@pytest.mark.parametrize("T", [1, 7, 40, 150])
def test_half_weights_infinite_h(T):
    """An infinite or NaN h reaches its own token alone, and does not cost the others a bit; one
    very large h costs its own token's others what the bound says."""
    say(f"infinite h T={T}")
    E, d, inter = 2, 64, 48
    g = torch.Generator().manual_seed(T)
    gu = (torch.randn(E, 2, inter, d, generator=g) / 8).to(torch.float16).to(DEV)
    dn = (torch.randn(E, d, inter, generator=g) / 7).to(torch.float16).to(DEV)
    x = (torch.randn(T, d, generator=g) / 512).to(torch.float16).to(DEV)
    ids = torch.zeros(T, 1, dtype=torch.int32, device=DEV)
    weights = torch.ones(T, 1, device=DEV)
    clean = si.moe_ffn(x, ids, weights, gu, dn)
    bad = x.clone()
    bad[0, 3] = float("inf")
    if T > 1:
        bad[T - 1, 5] = float("nan")
    y = si.moe_ffn(bad, ids, weights, gu, dn)
    assert not torch.any(torch.isfinite(y[0])) and not torch.any(torch.isfinite(y[T - 1]))
    assert torch.equal(y[1: T - 1], clean[1: T - 1])
    # one neuron at 2^75 beside others near 2^32
    gu[0, :, 7], x[0] = 60000.0, 60000.0
    dn[0, 11, 7] = 0.0
    y = si.moe_ffn(x, ids, weights, gu, dn)
    _check(y[:1], _np(x[:1]), ids[:1].cpu().numpy(), _np(weights[:1]), _np(gu), _np(dn))


@pytest.mark.parametrize("T,E,k,d,inter", [(1, 4, 2, 64, 48), (1, 3, 2, 48, 8208), (7, 4, 2, 64, 80),
                                           (40, 2, 2, 64, 4104), (150, 2, 1, 64, 80),
                                           (3, 1, 1, 8, 65536)])
@pytest.mark.parametrize("out", [torch.float32, torch.float16])
def test_half_weights_workspace(T, E, k, d, inter, out):
    """Nothing outside the queried bytes is written, and nothing that a call did not write is read:
    the workspace starts as NaN bits, and pairs without an expert are among the others."""
    say(f"half workspace T={T} E={E} k={k} d={d} I={inter} {out}")
    g = torch.Generator().manual_seed(T + inter)
    gu = (torch.randn(E, 2, inter, d, generator=g) / 8).to(torch.float16).to(DEV)
    dn = (torch.randn(E, d, inter, generator=g) / inter ** 0.5).to(torch.float16).to(DEV)
    x = torch.randn(T, d, generator=g).to(torch.float16).to(DEV)
    ids = torch.randint(-1, E, (T, k), generator=g).to(torch.int32).to(DEV)
    weights = torch.rand(T, k, generator=g).to(DEV)
    n = si._lib.load().si_moe_ffn_workspace(T, k, E, d, inter, si.F16, si.F16,
                                            si.F32 if out == torch.float32 else si.F16)
    space = torch.full((n + 4096,), 0xff, dtype=torch.uint8, device=DEV)
    y = si.moe_ffn(x, ids, weights, gu, dn, out_dtype=out, workspace=space[:n])
    assert torch.all(space[n:] == 0xff)
    assert torch.equal(y, si.moe_ffn(x, ids, weights, gu, dn, out_dtype=out))
    _check(y, _np(x), ids.cpu().numpy(), _np(weights), _np(gu), _np(dn))
    space.fill_(0)
    assert torch.equal(y, si.moe_ffn(x, ids, weights, gu, dn, out_dtype=out, workspace=space))


def test_silu():
    """SiLU(g) alone: unit rows make g and u = 1, and a float32 layer returns h. Error of the
    exponential: a rounding of g log2(e) (|g| 2^-23 with the constant's own) and 2^-23; of the sum,
    the reciprocal and the product: 2^-24, 2^-23 and 2^-24. Past 2^126 the reciprocal is 0."""
    say("SiLU alone")
    T, d, inter = 512, 4, 4
    g = torch.linspace(-110.0, 110.0, T, dtype=torch.float64).float()
    g[:8] = torch.tensor([0.0, -0.0, 1e-30, -1e-30, 1e30, 3e38, -1e30, -3e38])
    x = torch.zeros(T, d)
    x[:, 0], x[:, 1] = g, 1.0
    gu, dn = torch.zeros(1, 2, inter, d), torch.zeros(1, d, inter)
    gu[0, 0, :, 0], gu[0, 1, :, 1], dn[0, 2, 1] = 1.0, 1.0, 1.0
    y = si.moe_ffn(x.to(DEV), torch.zeros(T, 1, dtype=torch.int32, device=DEV),
                   torch.ones(T, 1, device=DEV), gu.to(DEV), dn.to(DEV))
    v = g.double().numpy()
    with np.errstate(over="ignore"):
        want = v / (1.0 + np.exp(-v))
    err = np.abs(_np(y[:, 2]) - want)
    assert np.all(err <= (np.minimum(np.abs(v), 120.0) + 4.0) * 2.0 ** -23 * np.abs(want) + 1e-36)
    assert torch.all(y[:, :2] == 0) and torch.all(y[:, 3] == 0)
