"""Products of block-scaled 8-bit matrices: exact sums, and what the 8-bit matrix instruction drops.

Whole numbers: codes of small whole numbers and scales that are powers of two have exact sums in
every order and in every step of either instruction, so y is the exact sum rounded once, to the bit.

Outliers: for a 16-bit y the products of 8 consecutive columns are cut, towards zero, to multiples
of 2^-13 of the largest of their powers of two (the sum of the two codes' exponents; codes below
2^-6 have the exponent -6). Of 8 products the one with that exponent is whole, so a group is off by
less than 7 such steps.
"""
import numpy as np
import pytest
import torch

import oracle
import paper_2607_18081_amd as si
from tests.gpu_util import say
from tests.test_gpu_fp8 import DEV, HALF_STEP, LARGE, NAMES

pytestmark = pytest.mark.gpu


def _codes(values):
    return torch.from_numpy(oracle.encode_e4m3(values)).to(DEV)


# the sizes of every tile, and small ones: one token and row, ragged blocks, the rows kernel
SMALL = [(1, 1, 16), (1, 130, 128), (2, 33, 144), (7, 500, 4112), (16, 129, 272), (16, 4096, 1040)]


@pytest.mark.parametrize("M,N,K,dt", LARGE + [(*s, dt) for s in SMALL for dt in NAMES])
def test_whole_numbers(M, N, K, dt):
    say(f"whole numbers M={M} N={N} K={K} {dt} {si.matmul_fp8_plan(M, N, K, NAMES[dt])}")
    g = torch.Generator(device=DEV).manual_seed(M + N + K)
    nk = -(-K // 128)
    x = torch.randint(-4, 5, (M, K), generator=g, device=DEV).to(torch.float64)
    w = torch.randint(-4, 5, (N, K), generator=g, device=DEV).to(torch.float64)
    xs = torch.exp2(torch.randint(-1, 2, (M, nk), generator=g, device=DEV).float())
    ws = torch.exp2(torch.randint(-1, 2, (-(-N // 128), nk), generator=g, device=DEV).float())
    want = torch.zeros(M, N, dtype=torch.float64, device=DEV)
    for b in range(nk):
        c = slice(128 * b, 128 * b + 128)
        row = ws[:, b].double().repeat_interleave(128)[:N]
        want += (x[:, c] @ w[:, c].t()) * xs[:, b].double()[:, None] * row
    # multiples of 1/4 that float32 holds exactly, and half does not overflow
    assert float(want.abs().max()) < 2.0 ** 15
    y = si.matmul_fp8(x.to(torch.float8_e4m3fn), xs, w.to(torch.float8_e4m3fn), ws,
                      out_dtype=NAMES[dt])
    assert torch.equal(y, want.to(NAMES[dt]))


def _exponent(v):
    """Power of two of each code's value, 2^-6 for the smallest ones and 0 for zeros."""
    with np.errstate(divide="ignore"):
        e = np.exp2(np.maximum(np.floor(np.log2(np.abs(v))), -6.0))
    return np.where(v == 0.0, 0.0, e)


def _data(kind, M, N, K, rng):
    """Codes' values of x and w."""
    x, w = rng.normal(0, 2, (M, K)), rng.normal(0, 100, (N, K))
    if kind == "outlier":                 # one a block, at the code that the quantiser gives it
        x[:, 5::128] = 448.0
    elif kind == "outlier in w":
        w[:, 77::128], x = 448.0, rng.normal(0, 100, (M, K))
        w[:, np.arange(K) % 128 != 77] *= 0.02
    elif kind == "apart":                 # outliers that cancel, in two groups of 8
        x[:, 5::128], x[:, 77::128] = 448.0, -448.0
        w[:, 77::128] = w[:, 5::128][:, : w[:, 77::128].shape[1]]
    elif kind == "together":              # in one
        x[:, 8::128], x[:, 15::128] = 448.0, -448.0
        w[:, 15::128] = w[:, 8::128][:, : w[:, 15::128].shape[1]]
    elif kind == "tiny":                  # codes at and below 2^-6, and a few large
        x, w = np.exp(rng.normal(-4, 2, (M, K))) * rng.choice([-1, 1], (M, K)), w / 100
    return (oracle.decode_e4m3(oracle.encode_e4m3(np.clip(v, -448, 448))) for v in (x, w))


@pytest.mark.parametrize("dt", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("M,N,K", [(3, 200, 640), (40, 150, 528), (300, 100, 384)])
@pytest.mark.parametrize("kind", ["outlier", "outlier in w", "apart", "together", "tiny"])
def test_outliers(kind, M, N, K, dt):
    say(f"8-bit product: {kind} M={M} N={N} K={K} {dt}")
    rng = np.random.default_rng(M + len(kind))
    x, w = _data(kind, M, N, K, rng)
    nk = -(-K // 128)
    # (half: sums stay below 65504)
    xs = np.exp2(rng.integers(-9, -6, (M, nk))).astype(np.float32)
    ws = np.exp2(rng.integers(-3, 0, (-(-N // 128), nk))).astype(np.float32)
    y = si.matmul_fp8(_codes(x), torch.from_numpy(xs).to(DEV), _codes(w),
                      torch.from_numpy(ws).to(DEV), out_dtype=NAMES[dt])
    a, b = x * oracle.spread(xs, M, K, 1), w * oracle.spread(ws, N, K, 128)
    want, mag = a @ b.T, np.abs(a) @ np.abs(b).T
    tol = (128 + nk + 4) * 2.0 ** -23 * mag       # float32 sums, each step rounded or cut
    if dt != "f32":
        ea = _exponent(x) * oracle.spread(xs, M, K, 1)
        eb = _exponent(w) * oracle.spread(ws, N, K, 128)
        for k in range(0, K, 8):
            top = np.max(ea[:, None, k: k + 8] * eb[None, :, k: k + 8], axis=2)
            tol = tol + 7 * 2.0 ** -13 * top
    tol = tol + HALF_STEP[NAMES[dt]] * (np.abs(want) + tol) + (2.0 ** -25 if dt == "f16" else 0.0)
    err = np.abs(y.double().cpu().numpy() - want)
    assert np.all(err <= tol), float(np.max(err / tol))
