"""Ids of the caller's own: many tokens on one expert, among ids of no expert whose weights are NaN."""
import numpy as np
import pytest
import torch

import paper_2607_18081_amd as si
from tests.gpu_util import say
from tests.test_gpu_experts import DEV, DT, _check_layer, _experts

pytestmark = pytest.mark.gpu


# Tokens, experts and ranks by which kernels they reach: fewer pairs than experts (a slot a pair),
# fewer than 16 an expert (a slot an expert), and more (waves that share the tokens); with one pass
# over the expert's weights, and with several
@pytest.mark.parametrize("T,E,k", [(1, 5, 4), (4, 5, 4), (100, 512, 4), (100, 64, 4), (12, 64, 4),
                                   (33, 5, 4), (100, 5, 4), (300, 2, 2), (512, 3, 4)])
@pytest.mark.parametrize("dt,wkind", [("bf16", "same"), ("f16", "same"), ("f32", "same"),
                                      ("bf16", "fp8"), ("f16", "fp8")])
def test_every_token_on_one_expert(T, E, k, dt, wkind):
    say(f"one expert for all T={T} E={E} k={k} {dt} {wkind}")
    d, inter = 96, 80
    dev, gu, dn = _experts(E, d, inter, dt, wkind, T)
    rng = np.random.default_rng(T + E)
    x = torch.randn(T, d, generator=torch.Generator().manual_seed(T)).to(DT[dt]).to(DEV)
    for rank, expert in ((1, E - 1), (k - 1, 0)):
        ids = rng.choice(np.array([-1, E, 2 ** 31 - 1, -2 ** 31], dtype=np.int32), (T, k))
        ids[:, rank] = expert
        weights = np.full((T, k), np.nan, dtype=np.float32)
        weights[:, rank] = rng.normal(0, 1, T)
        args = [torch.from_numpy(v).to(DEV) for v in (ids, weights)]
        for out in {torch.float32, DT[dt]}:
            y = torch.full((T, d), float("nan"), dtype=out, device=DEV)
            y = si.moe_ffn(x, *args, dev[0], dev[1], gate_up_scales=dev[2], down_scales=dev[3],
                           out_dtype=out, y=y)
            _check_layer(y, x, args[0], args[1], gu, dn, dt, wkind)


@pytest.mark.parametrize("dt,wkind", [("bf16", "same"), ("f16", "same"), ("f32", "same"),
                                      ("bf16", "fp8")])
@pytest.mark.parametrize("T,E", [(2, 40), (60, 40), (60, 2)])
def test_one_expert_at_every_rank(T, E, dt, wkind):
    """The same expert at all of a token's ranks, added as often: k pairs a token, several passes."""
    say(f"one expert at every rank T={T} E={E} {dt} {wkind}")
    d, inter, k = 64, 48, 5
    dev, gu, dn = _experts(E, d, inter, dt, wkind, T + 1)
    rng = np.random.default_rng(T * E)
    x = torch.randn(T, d, generator=torch.Generator().manual_seed(T)).to(DT[dt]).to(DEV)
    ids = np.repeat(rng.integers(0, 2, (T, 1)), k, axis=1).astype(np.int32)
    weights = rng.normal(0, 1, (T, k)).astype(np.float32)
    args = [torch.from_numpy(v).to(DEV) for v in (ids, weights)]
    y = si.moe_ffn(x, *args, dev[0], dev[1], gate_up_scales=dev[2], down_scales=dev[3])
    _check_layer(y, x, args[0], args[1], gu, dn, dt, wkind)


@pytest.mark.parametrize("dt,wkind", [("bf16", "same"), ("f16", "same"), ("f32", "same"),
                                      ("bf16", "fp8"), ("f16", "fp8")])
@pytest.mark.parametrize("T,E", [(1, 8), (1, 300), (3, 8), (40, 2)])
def test_padding_comes_and_goes(T, E, dt, wkind):
    """A captured layer whose n_valid goes from all to none and back between replays, with eager
    work between; the rows behind are NaN in x, and 0 in y. The choice is made in a kernel of its
    own, or (one token, few experts) in the experts' first one."""
    say(f"padding comes and goes T={T} E={E} {dt} {wkind}")
    d, inter, k = 64, 80, 2
    dev, gu, dn = _experts(E, d, inter, dt, wkind, T + E)
    g = torch.Generator().manual_seed(E)
    x = torch.randn(T, d, generator=g).to(DT[dt]).to(DEV)
    w = (torch.randn(E, d, generator=g) / 8).to(DT[dt]).to(DEV)
    kw = dict(gate_up_scales=dev[2], down_scales=dev[3])
    whole, ids_w, weights_w = si.moe_layer(x, w, dev[0], dev[1], k, **kw)
    _check_layer(whole, x, ids_w, weights_w, gu, dn, dt, wkind)
    held = x.clone()
    n = torch.tensor([T], dtype=torch.int32, device=DEV)
    y = torch.empty(T, d, device=DEV)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        _, ids, weights = si.moe_layer(held, w, dev[0], dev[1], k, n_valid=n, y=y, **kw)
    for valid in (T, 0, T, T - 1, 0, 0, T):
        held.copy_(x)
        held[valid:] = float("nan")
        n.fill_(valid)
        y.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y[:valid], whole[:valid]) and torch.all(y[valid:] == 0), valid
        assert torch.equal(ids[:valid], ids_w[:valid]) and torch.all(ids[valid:] == -1)
        assert torch.equal(weights[:valid], weights_w[:valid]) and torch.all(weights[valid:] == 0)
        again, _, _ = si.moe_layer(held, w, dev[0], dev[1], k, n_valid=n, **kw)
        assert torch.equal(again, y)
