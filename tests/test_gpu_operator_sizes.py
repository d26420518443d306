"""The 8-bit and expert operators past 2^31 elements or bytes, and at the most tokens and experts: the
far end of a large call equals the same rows or experts on their own, to the bit."""
import pytest
import torch

import paper_2607_18081_amd as si
from tests.gpu_util import say
from tests.test_gpu_experts import _check_layer, _np

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _u8(t):
    return t.view(torch.uint8)


@pytest.mark.parametrize("br", [1, 128])
def test_quantize_past_32_bits(br):
    """2.3e9 values: 4.6 GB of bf16, whose last blocks lie past 2^32 bytes and 2^31 values."""
    say(f"quantise past 2^31 values br={br}")
    R, C = 70000, 32768
    x = torch.empty(R, C, dtype=torch.bfloat16, device=DEV)
    x.view(-1, 32768).normal_(0.0, 1.0, generator=torch.Generator(device=DEV).manual_seed(1))
    codes, scales = si.quantize_fp8(x, block_rows=br)
    for r0 in (0, 65536, R - R % 128):
        part = x[r0: r0 + 300].contiguous() if r0 + 300 <= R else x[r0:].contiguous()
        c, s = si.quantize_fp8(part, block_rows=br)
        n = part.shape[0] // br * br if r0 + 300 <= R else part.shape[0]    # whole blocks
        assert torch.equal(_u8(codes[r0: r0 + n]), _u8(c[:n])), r0
        b0, nb = r0 // br, -(-n // br)
        assert torch.equal(scales[b0: b0 + nb], s[:nb]), r0


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_matmul_past_32_bits(dtype):
    """2.3e9 results, of whole numbers: exact whatever the tile."""
    say(f"product past 2^31 results {dtype}")
    M, N, K = 70000, 32769, 144
    g = torch.Generator(device=DEV).manual_seed(2)
    x = torch.randint(-4, 5, (M, K), generator=g, device=DEV).float()
    w = torch.randint(-4, 5, (N, K), generator=g, device=DEV).float()
    xs = torch.ones(M, 2, device=DEV)
    ws = torch.ones(-(-N // 128), 2, device=DEV)
    y = si.matmul_fp8(x.to(torch.float8_e4m3fn), xs, w.to(torch.float8_e4m3fn), ws,
                      out_dtype=dtype)
    for r0 in (0, 65535, M - 70):
        want = (x[r0: r0 + 70].double() @ w.double().t()).to(dtype)
        assert torch.equal(y[r0: r0 + 70], want), r0


def test_route_most_tokens():
    say("route 65535 tokens")
    T, E, d, k = 65535, 72, 136, 5
    g = torch.Generator(device=DEV).manual_seed(3)
    x = torch.randn(T, d, generator=g, device=DEV).to(torch.bfloat16)
    w = torch.randn(E, d, generator=g, device=DEV)
    ids, weights = si.moe_route(x, w, k)
    for t0 in (0, 32768, T - 31):
        i, v = si.moe_route(x[t0: t0 + 31], w, k)
        assert torch.equal(ids[t0: t0 + 31], i) and torch.equal(weights[t0: t0 + 31], v), t0


@pytest.mark.parametrize("T", [1, 3, 480])
@pytest.mark.parametrize("wkind", ["bf16", "fp8"])
def test_far_experts(T, wkind):
    """Experts past 2^32 bytes: 11 GB of bf16 gate and up rows (6.9 GB of codes), each token on the
    first, a middle or the last of them; against the same three alone, by kernels of the same kind
    (one token, few tokens an expert, 16 and more), whose sums have the same order."""
    say(f"far experts T={T} {wkind}")
    d, inter = 4096, 14336
    E = 48 if wkind == "bf16" else 59
    g = torch.Generator(device=DEV).manual_seed(4)
    at = torch.tensor([0, E // 2 + 1, E - 1], device=DEV)
    kw, few = {}, {}
    if wkind == "bf16":
        gu = torch.empty(E, 2, inter, d, dtype=torch.bfloat16, device=DEV).normal_(0, 0.02, generator=g)
        dn = torch.empty(E, d, inter, dtype=torch.bfloat16, device=DEV).normal_(0, 0.02, generator=g)
        gu3, dn3 = gu[at], dn[at]
    else:
        # codes of random bytes without NaN
        gu = torch.randint(0, 127, (E, 2, inter, d), dtype=torch.uint8, device=DEV, generator=g)
        dn = torch.randint(128, 255, (E, d, inter), dtype=torch.uint8, device=DEV, generator=g)
        gu3, dn3 = gu[at], dn[at]
        s = [torch.rand(E, 2, inter // 128, d // 128, generator=g, device=DEV) * 1e-4,
             torch.rand(E, d // 128, inter // 128, generator=g, device=DEV) * 1e-4]
        kw = dict(gate_up_scales=s[0], down_scales=s[1])
        few = dict(gate_up_scales=s[0][at], down_scales=s[1][at])
    x = torch.randn(T, d, generator=g, device=DEV).to(torch.bfloat16)
    pick = torch.randint(0, 3, (T, 2), generator=g, device=DEV)
    weights = torch.rand(T, 2, generator=g, device=DEV)
    y = si.moe_ffn(x, at[pick].to(torch.int32), weights, gu, dn, **kw)
    assert torch.all(torch.isfinite(y)) and float(y.abs().max()) > 0
    assert torch.equal(y, si.moe_ffn(x, pick.to(torch.int32), weights, gu3, dn3, **few))


def test_most_experts_and_pairs():
    """65535 experts, 8192 pairs: a slot a pair; and the last expert's weights."""
    say("65535 experts")
    T, k, E, d, inter = 512, 16, 65535, 16, 16
    g = torch.Generator(device=DEV).manual_seed(5)
    gu = torch.randn(E, 2, inter, d, generator=g, device=DEV).to(torch.bfloat16)
    dn = torch.randn(E, d, inter, generator=g, device=DEV).to(torch.bfloat16)
    x = torch.randn(T, d, generator=g, device=DEV).to(torch.bfloat16)
    ids = torch.randint(0, E, (T, k), generator=g, device=DEV).to(torch.int32)
    ids[:, 3], ids[7, 7] = E - 1, 0
    weights = torch.rand(T, k, generator=g, device=DEV)
    y = si.moe_ffn(x, ids, weights, gu, dn)
    some = torch.tensor([0, 7, 100, 511], device=DEV)
    _check_layer(y[some], x[some], ids[some], weights[some], _np(gu), _np(dn), "bf16", "same")
    # and every token against the experts it names, laid out one after the other
    for t0 in range(0, T, 128):
        rows = slice(t0, t0 + 128)
        near, place = torch.unique(ids[rows], return_inverse=True)
        z = si.moe_ffn(x[rows].contiguous(), place.to(torch.int32), weights[rows].contiguous(),
                       gu[near.long()], dn[near.long()])
        assert torch.equal(y[rows], z), t0
