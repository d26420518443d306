"""Block quantisation and the product of block-scaled 8-bit matrices against the float64 oracle.

Quantisation is compared bit for bit (its definition is in float32). The product is a float32 sum
of at most 128 products a block and one scaled addition a block: with each step rounded or
truncated, an output is off by at most (128 + blocks + 4) 2^-23 sum |x| |w|, and by half a step of
its type (2^-8 of the value for bf16, 2^-11 for half) after its one rounding. Outputs of 16 bits
come from the 8-bit matrix instruction, which drops what lies 2^-14 below a block's largest
product: at most 128 times that, with the largest product at most max |x| max |w| of the block.
"""
import numpy as np
import pytest
import torch

import oracle
import paper_2607_18081_amd as si
from tests.gpu_util import say

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
HALF_STEP = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}


def _u8(t):
    return t.view(torch.uint8).cpu().numpy()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("br", [1, 128])
@pytest.mark.parametrize("G,R,C", [(1, 1, 16), (1, 1, 128), (1, 16, 4096), (2, 127, 144),
                                   (3, 128, 256), (1, 129, 400), (2, 300, 1040), (1, 5, 2064)])
def test_quantize(G, R, C, br, dtype):
    say(f"quantize G={G} R={R} C={C} br={br} {dtype}")
    g = torch.Generator().manual_seed(G * 1000 + R + C + br)
    x = torch.randn(G, R, C, generator=g) * torch.exp(3 * torch.randn(G, R, 1, generator=g))
    x[0, 0, : min(C, 128)] = 0.0                             # a block row of zeros
    x = x.to(dtype)
    codes, scales = si.quantize_fp8(x.to(DEV), block_rows=br)
    assert codes.dtype == torch.float8_e4m3fn and codes.shape == x.shape
    for i in range(G):
        c, s = oracle.quantize_fp8(x[i].float().numpy(), br)
        # a half block whose values overflowed to infinity has scale NaN on both sides
        assert np.array_equal(scales[i].cpu().numpy(), s, equal_nan=True), i
        assert np.array_equal(_u8(codes[i]), c), i


@pytest.mark.parametrize("br", [1, 128])
def test_quantize_extremes(br):
    """Blocks of zeros, of the smallest values, of the largest, with a NaN, with an infinity."""
    say(f"quantize extremes br={br}")
    R = 128 * 6
    x = torch.randn(R, 272, generator=torch.Generator().manual_seed(1))
    x[:128] = 0.0
    x[128:256] *= 1e-44
    x[256:384] *= 3e37
    x[384 + 7, 3], x[512 + 1, 130], x[640, 271] = float("nan"), float("inf"), float("-inf")
    codes, scales = si.quantize_fp8(x.to(DEV), block_rows=br)
    c, s = oracle.quantize_fp8(x.numpy(), br)
    got = scales.cpu().numpy()
    assert np.array_equal(np.isnan(got), np.isnan(s))
    assert np.array_equal(got[~np.isnan(s)], s[~np.isnan(s)])
    nan = np.isnan(oracle.decode_e4m3(c))
    assert np.array_equal(np.isnan(oracle.decode_e4m3(_u8(codes))), nan)
    assert np.array_equal(_u8(codes)[~nan], c[~nan])


def _operands(M, N, K, seed):
    rng = np.random.default_rng(seed)
    nk = -(-K // 128)
    x = oracle.encode_e4m3(np.clip(rng.normal(0, 120, (M, K)), -448, 448))
    w = oracle.encode_e4m3(np.clip(rng.normal(0, 120, (N, K)), -448, 448))
    xs = np.exp(rng.normal(-4, 1, (M, nk))).astype(np.float32)
    ws = np.exp(rng.normal(-8, 1, (-(-N // 128), nk))).astype(np.float32)
    return x, xs, w, ws


def _dev(a):
    return torch.from_numpy(a).to(DEV)


def _check(y, x, xs, w, ws, dtype):
    want, mag = oracle.matmul_fp8(x, xs, w, ws)
    nk = xs.shape[1]
    tol = (128 + nk + 4) * 2.0 ** -23 * mag
    if dtype != torch.float32:
        a, b = oracle.decode_e4m3(x), oracle.decode_e4m3(w)
        for k in range(nk):
            ax = np.max(np.abs(a[:, 128 * k: 128 * k + 128]), axis=1) * xs[:, k].astype(np.float64)
            bw = np.max(np.abs(b[:, 128 * k: 128 * k + 128]), axis=1)
            bw = bw * np.repeat(ws[:, k].astype(np.float64), 128)[: w.shape[0]]
            tol = tol + 128 * 2.0 ** -14 * np.outer(ax, bw)
    tol = tol + HALF_STEP[dtype] * (np.abs(want) + tol)
    if dtype == torch.float16:
        tol = tol + 2.0 ** -25                                # its subnormal step
    err = np.abs(y.double().cpu().numpy() - want)
    assert np.all(err <= tol), float(np.max(err / tol))


@pytest.mark.parametrize("M,N,K,dtype", [
    (1, 1, 16, torch.float32), (1, 16, 128, torch.float32), (1, 640, 2048, torch.bfloat16),
    (2, 33, 144, torch.float32), (13, 200, 1040, torch.bfloat16), (16, 130, 4112, torch.float32),
    (17, 129, 256, torch.float16), (33, 257, 400, torch.float32), (64, 64, 384, torch.bfloat16),
    (65, 127, 528, torch.float32), (100, 1000, 640, torch.bfloat16), (127, 384, 784, torch.float32),
    (128, 256, 256, torch.float32), (129, 255, 272, torch.bfloat16), (200, 513, 1408, torch.float32),
    (255, 260, 16, torch.float32), (256, 512, 512, torch.float16), (257, 300, 2064, torch.float32),
    (700, 385, 896, torch.bfloat16), (1025, 770, 400, torch.float32),
])
def test_matmul(M, N, K, dtype):
    say(f"matmul M={M} N={N} K={K} {dtype}")
    x, xs, w, ws = _operands(M, N, K, M * 7 + N + K)
    args = (_dev(x), _dev(xs), _dev(w), _dev(ws))
    out = torch.full((M, N), float("nan"), dtype=dtype, device=DEV)
    y = si.matmul_fp8(*args, out_dtype=dtype, out=out)
    _check(y, x, xs, w, ws, dtype)
    again = si.matmul_fp8(args[0].view(torch.float8_e4m3fn), *args[1:], out_dtype=dtype)
    assert torch.equal(again, y)                             # bitwise repeatable


# sizes that reach every tile, with and without K chunks, at ragged edges: 64 tokens are compared
LARGE = [
    (4010, 3401, 400, "bf16"), (2050, 3500, 272, "f16"), (1001, 4000, 5264, "bf16"),
    (1500, 3400, 144, "bf16"), (2047, 3390, 400, "f32"), (700, 3990, 5200, "bf16"),
    (1030, 3333, 272, "f32"), (900, 3333, 272, "bf16"), (511, 4095, 5136, "f32"),
    (500, 3333, 656, "bf16"), (500, 3333, 656, "f32"), (120, 6001, 5216, "bf16"),
    (1500, 5000, 5264, "bf16"), (250, 3400, 400, "bf16"), (250, 3400, 400, "f32"),
    (60, 4000, 4112, "f16"),
    (60, 4000, 2064, "f32"), (9, 10500, 272, "bf16"), (9, 10500, 400, "f32"),
    (17, 200, 5136, "f32"), (100, 3131, 10256, "bf16"), (100, 3131, 10256, "f32"),
    (130, 3131, 10256, "bf16"), (130, 3131, 10256, "f32"), (130, 4283, 5136, "bf16"),
    (130, 4283, 5136, "f32"), (1001, 4000, 5264, "f32"), (900, 3333, 10256, "bf16"),
    (260, 4155, 10256, "bf16"), (260, 4155, 10256, "f32"),
    (817, 601, 14080, "bf16"), (452, 515, 9536, "bf16"), (66, 6461, 28048, "bf16"),
    (961, 1030, 11216, "bf16"), (1190, 1733, 16896, "f16"), (18, 258, 1728, "f32"),
    (1308, 722, 7824, "f32"), (1856, 2312, 1680, "f32"), (1276, 790, 17712, "f32"),
    (1748, 1769, 23488, "f32"),
]
NAMES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


@pytest.mark.parametrize("M,N,K,dt", LARGE)
def test_matmul_tiles(M, N, K, dt):
    say(f"matmul tiles M={M} N={N} K={K} {dt} {si.matmul_fp8_plan(M, N, K, NAMES[dt])}")
    rng = np.random.default_rng(M + N + K)
    nk = -(-K // 128)
    table = oracle.encode_e4m3(np.clip(rng.normal(0, 120, 1 << 16), -448, 448))
    x, w = table[rng.integers(0, 1 << 16, (M, K))], table[rng.integers(0, 1 << 16, (N, K))]
    xs = np.exp(rng.normal(-4, 1, (M, nk))).astype(np.float32)
    ws = np.exp(rng.normal(-8, 1, (-(-N // 128), nk))).astype(np.float32)
    args = [_dev(a) for a in (x, xs, w, ws)]
    need = si._lib.load().si_matmul_fp8_workspace(M, N, K)
    space = torch.full((max(need, 16),), 0xff, dtype=torch.uint8, device=DEV)    # NaN bits
    out = torch.full((M, N), float("nan"), dtype=NAMES[dt], device=DEV)
    y = si.matmul_fp8(*args, out_dtype=NAMES[dt], out=out, workspace=space)
    rows = np.unique(np.concatenate([[0, M - 1], rng.integers(0, M, 62)]))
    _check(y[torch.from_numpy(rows).to(DEV)], x[rows], xs[rows], w, ws, NAMES[dt])
    assert torch.equal(si.matmul_fp8(*args, out_dtype=NAMES[dt]), y)


@pytest.mark.parametrize("M", [3, 70, 300])
def test_matmul_nan_stays_in_its_row(M):
    """A token quantised from a NaN is NaN, and so is a weight row; the rest is as without."""
    say(f"matmul nan M={M}")
    x, xs, w, ws = _operands(M, 300, 640, M)
    clean = si.matmul_fp8(_dev(x), _dev(xs), _dev(w), _dev(ws), out_dtype=torch.float32)
    x[1, 130], w[7, 5] = 0x7f, 0xff
    xs[2, 4] = np.nan
    y = si.matmul_fp8(_dev(x), _dev(xs), _dev(w), _dev(ws), out_dtype=torch.float32)
    bad = torch.zeros((M, 300), dtype=torch.bool, device=DEV)
    bad[1], bad[2], bad[:, 7] = True, True, True
    assert torch.equal(torch.isnan(y), bad)
    assert torch.equal(y[~bad], clean[~bad])


def test_quantize_then_multiply():
    """The two together, as a dense projection runs: within the rounding of e4m3 (2^-4 a value, or
    2^-10 of its block's step at the small end) of the unquantised product."""
    say("quantise, then multiply")
    g = torch.Generator().manual_seed(5)
    x = torch.randn(37, 1040, generator=g).to(torch.bfloat16)
    w = (torch.randn(300, 1040, generator=g) * 0.02).to(torch.bfloat16)
    xq, xs = si.quantize_fp8(x.to(DEV))
    wq, ws = si.quantize_fp8(w.to(DEV), block_rows=128)
    y = si.matmul_fp8(xq, xs, wq, ws, out_dtype=torch.float32).double().cpu().numpy()
    xf, wf = x.double().numpy(), w.double().numpy()
    sx = oracle.spread(xs.cpu().numpy(), 37, 1040, 1)
    sw = oracle.spread(ws.cpu().numpy(), 300, 1040, 128)
    # half a step of a code: 2^-4 of the value, or 2^-10 scales for subnormal codes; 2^-22 covers
    # the float32 scale and product
    ex = np.maximum((2.0 ** -4 + 2.0 ** -22) * np.abs(xf), 2.0 ** -10 * sx)
    ew = np.maximum((2.0 ** -4 + 2.0 ** -22) * np.abs(wf), 2.0 ** -10 * sw)
    tol = ex @ np.abs(wf).T + np.abs(xf) @ ew.T + ex @ ew.T
    tol = tol + 200 * 2.0 ** -23 * ((np.abs(xf) + ex) @ (np.abs(wf) + ew).T)
    assert np.all(np.abs(y - xf @ wf.T) <= tol)


def test_streams_and_graph():
    """Two streams at once, and a graph replayed with eager calls between: the eager bits."""
    say("fp8 on streams and in a graph")
    x, xs, w, ws = _operands(40, 700, 1408, 9)
    args = [_dev(a) for a in (x, xs, w, ws)]
    src = torch.randn(40, 1408, device=DEV).to(torch.bfloat16)
    want = si.matmul_fp8(*args, out_dtype=torch.float32)
    wc, wsc = si.quantize_fp8(src)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = []
    for s in streams:
        with torch.cuda.stream(s):
            got.append([si.matmul_fp8(*args, out_dtype=torch.float32) for _ in range(4)])
    torch.cuda.synchronize()
    assert all(torch.equal(y, want) for ys in got for y in ys)
    out = torch.empty_like(want)
    codes, scales = torch.empty_like(wc), torch.empty_like(wsc)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        si.quantize_fp8(src, codes=codes, scales=scales)
        si.matmul_fp8(*args, out_dtype=torch.float32, out=out)
    for _ in range(3):
        out.fill_(float("nan"))
        codes.view(torch.uint8).fill_(1)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)
        assert torch.equal(codes.view(torch.uint8), wc.view(torch.uint8))
        assert torch.equal(scales, wsc)
        si.matmul_fp8(args[0].flip(0).contiguous(), *args[1:])


def test_binding_refusals():
    say("fp8 binding refusals")
    x = torch.zeros(4, 256, dtype=torch.bfloat16, device=DEV)
    q, s = si.quantize_fp8(x)
    w, ws = si.quantize_fp8(x, block_rows=128)
    with pytest.raises(ValueError):
        si.quantize_fp8(x[:, ::2])                           # not contiguous
    with pytest.raises(ValueError):
        si.quantize_fp8(x, block_rows=64)
    with pytest.raises(TypeError):
        si.quantize_fp8(x.double())
    with pytest.raises(si.SelectInferError):
        si.quantize_fp8(x[:, :24].contiguous())              # not a multiple of 16
    with pytest.raises(ValueError):
        si.matmul_fp8(q, s[:3], w, ws)                       # scales of another shape
    with pytest.raises(ValueError):
        si.matmul_fp8(x, s, w, ws)                           # not codes
    with pytest.raises(ValueError):
        si.matmul_fp8(q, s, w, ws, out=torch.empty(4, 4, device=DEV))     # another type
    with pytest.raises(ValueError):
        si.matmul_fp8(q, s, w.cpu(), ws)
    assert si.matmul_fp8(q[:0], s[:0], w, ws).shape == (0, 4)
    assert si.quantize_fp8(x[:0])[0].shape == (0, 256)
