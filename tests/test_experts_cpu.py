"""Block-scaled 8-bit matrices and experts, the parts that need no GPU: the oracle against library
conversions and brute force, workspace queries, and every refusal that the host makes (each returns
before anything is enqueued)."""
import ctypes
import math

import numpy as np
import pytest
import torch

import oracle
from tests.test_lib_cpu import lib  # noqa: F401  (fixture)

F32, BF16, F16, E4M3 = 0, 1, 2, 3
OK, INVALID, UNSUPPORTED, WORKSPACE = 0, 1, 5, 7
SOFT, SIG, RENORM = 1, 2, 4


# ---- oracle ----------------------------------------------------------------------------------

def test_e4m3_codes_agree_with_torch():
    codes = np.arange(256, dtype=np.uint8)
    want = torch.from_numpy(codes).view(torch.float8_e4m3fn).double().numpy()
    got = oracle.decode_e4m3(codes)
    assert np.array_equal(np.isnan(got), np.isnan(want))
    assert np.array_equal(got[~np.isnan(got)], want[~np.isnan(want)])
    rng = np.random.default_rng(0)
    pos = got[:127]
    x = np.concatenate([got[~np.isnan(got)], (pos[1:] + pos[:-1]) / 2, -(pos[1:] + pos[:-1]) / 2,
                        rng.normal(0, 100, 4000), rng.normal(0, 0.01, 4000)]).astype(np.float32)
    x = x[np.abs(x) <= 448.0]
    want = torch.from_numpy(x).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert np.array_equal(oracle.encode_e4m3(x), want)


def test_quantize_by_hand():
    x = np.zeros((2, 144), dtype=np.float32)
    x[0, 3], x[0, 5], x[0, 130] = 448.0, -224.0, 1.0
    x[1, 0] = np.inf
    codes, scales = oracle.quantize_fp8(x, 1)
    assert scales.shape == (2, 2) and scales[0, 0] == 1.0
    assert scales[0, 1] == np.float32(1.0) / np.float32(448.0)
    assert oracle.decode_e4m3(codes[0, [3, 5, 130]]).tolist() == [448.0, -224.0, 448.0]
    assert np.isnan(scales[1, 0]) and np.all(codes[1, :128] == 0x7f)
    assert np.all(codes[1, 128:] == 0) and scales[1, 1] == np.float32(2.0 ** -60 / 448.0)
    codes, scales = oracle.quantize_fp8(x[:1], 128)
    assert scales.shape == (1, 2)


def test_oracle_layer_against_torch():
    g = torch.Generator().manual_seed(3)
    T, d, E, inter, k = 5, 24, 6, 20, 3
    x = torch.randn(T, d, dtype=torch.float64, generator=g)
    wr = torch.randn(E, d, dtype=torch.float64, generator=g)
    gu = torch.randn(E, 2, inter, d, dtype=torch.float64, generator=g)
    dn = torch.randn(E, d, inter, dtype=torch.float64, generator=g)
    p = torch.softmax(x @ wr.t(), dim=1)
    top = torch.topk(p, k, dim=1)
    w = top.values / top.values.sum(dim=1, keepdim=True)
    ids, weights, _ = oracle.moe_route(x.numpy(), wr.numpy(), k)
    assert np.array_equal(ids, top.indices.numpy())
    assert np.allclose(weights, w.numpy(), rtol=1e-13, atol=0)
    want = torch.zeros(T, d, dtype=torch.float64)
    for t in range(T):
        for r in range(k):
            e = int(ids[t, r])
            h = torch.nn.functional.silu(gu[e, 0] @ x[t]) * (gu[e, 1] @ x[t])
            want[t] += w[t, r] * (dn[e] @ h)
    got, bound = oracle.moe_ffn(x.numpy(), ids, weights, gu.numpy(), dn.numpy())
    assert np.allclose(got, want.numpy(), rtol=1e-12, atol=1e-12)
    assert np.all(bound > 0)
    ids[0] = -1
    assert not np.any(oracle.moe_ffn(x.numpy(), ids, weights, gu.numpy(), dn.numpy())[0][0])


def test_oracle_route_order():
    x = np.array([[1.0, 0.0]])
    w = np.array([[0.0, 0], [2.0, 0], [-0.0, 0], [2.0, 0], [np.nan, 0], [-1.0, 0]])
    ids, _, _ = oracle.moe_route(x, w, 6)
    assert ids[0].tolist() == [1, 3, 0, 2, 5, 4]
    ids, weights, _ = oracle.moe_route(x, w[:4], 2, bias=[5.0, 0, 0, 0], score="sigmoid")
    assert ids[0].tolist() == [0, 1]                 # the bias chooses, the score weighs
    s2 = 1.0 / (1.0 + math.exp(-2.0))
    assert np.allclose(weights[0], [0.5 / (0.5 + s2), s2 / (0.5 + s2)])


# ---- workspaces ------------------------------------------------------------------------------

def test_workspace_queries(lib):  # noqa: F811
    assert lib.si_moe_route_workspace(0, 8, 64) == 0
    for T, E, d in ((1, 128, 2048), (200, 256, 5120), (65535, 8, 64)):
        n = lib.si_moe_route_workspace(T, E, d)
        assert n >= T * E * 8 and n % (T * E * 8) == 0
    for xdt, wdt, ydt, per in ((BF16, BF16, BF16, 4), (BF16, BF16, F32, 6), (F16, F16, F32, 4),
                               (F16, E4M3, F16, 4), (BF16, E4M3, F32, 6), (F32, F32, F32, 4)):
        n = lib.si_moe_ffn_workspace(3, 2, 8, 64, 48, xdt, wdt, ydt)
        assert n >= 6 * 48 * per + 6 * 64 * 4
        assert lib.si_moe_layer_workspace(3, 2, 8, 64, 48, xdt, wdt, ydt) >= \
            n + lib.si_moe_route_workspace(3, 8, 64)
    assert lib.si_moe_ffn_workspace(3, 2, 8, 64, 48, BF16, F32, F32) == 0    # refused types
    assert lib.si_moe_layer_workspace(0, 2, 8, 64, 48, BF16, BF16, F32) == 0


def test_queries_out_of_range(lib):  # noqa: F811
    """Sizes past every limit are answered, not computed with: no division by a wrapped zero."""
    plan = (ctypes.c_int32 * 3)()
    for M, N, K in ((17, 17, 1 << 39), (1 << 40, 1 << 40, 64), (1 << 62, 1 << 62, 1 << 62),
                    (1 << 24, 1 << 24, 64), (17, 1 << 25, 64)):
        assert lib.si_matmul_fp8_workspace(M, N, K) == 0
        assert lib.si_matmul_fp8_plan(M, N, K, BF16, plan) == UNSUPPORTED
    assert lib.si_matmul_fp8_plan(1 << 20, 1 << 20, 64, BF16, plan) == OK
    for T, E, d in ((1 << 34, 1 << 38, 64), (65536, 8, 64), (4, 1025, 64), (4, 8, 1 << 62)):
        assert lib.si_moe_route_workspace(T, E, d) == 0
    assert lib.si_moe_ffn_workspace(1 << 62, 1 << 62, 8, 64, 48, BF16, BF16, F32) == 0
    assert lib.si_moe_layer_workspace(4, 2, 8, 1 << 62, 1 << 62, BF16, BF16, F32) == 0


def test_every_tile_is_value_checked(lib):  # noqa: F811
    """The sizes of the GPU tests reach every tile of the 8-bit product, for float32 and 16-bit
    results, with K whole and in chunks."""
    import paper_2607_18081_amd as si
    from tests.test_gpu_fp8 import LARGE, NAMES
    seen = {(dt == "f32", *si.matmul_fp8_plan(M, N, K, NAMES[dt])) for M, N, K, dt in LARGE}
    seen = {(*s[:3], s[3] > 1) for s in seen}
    for exact in (False, True):
        for t in [(256, 256), (256, 128), (128, 128), (128, 64), (64, 64)][exact:]:
            assert {(exact, *t, False), (exact, *t, True)} <= seen, (exact, t)
    assert not any(s[:2] == (True, 256) and s[2] == 256 for s in seen)
    for M in (17, 64, 100, 260, 700, 1500, 4096):
        for N in range(64, 20000, 320):
            for K in (400, 2560, 10240, 28672):
                assert si.matmul_fp8_plan(M, N, K, torch.float32)[:2] != (256, 256)
    assert si.matmul_fp8_plan(1, 4096, 4096)[0] == 0
    for M in (1, 5, 17, 64, 200, 1000, 5000):
        for N in (1, 100, 3000, 20000):
            for K in (16, 1000 * 16, 128 * 37):
                for dt in NAMES.values():
                    ks = si.matmul_fp8_plan(M, N, K, dt)[2]
                    assert 1 <= ks <= 4
                    assert lib.si_matmul_fp8_workspace(M, N, K) >= (ks > 1) * ks * M * N * 4


# ---- refusals --------------------------------------------------------------------------------

@pytest.fixture(scope="module")
def mem():
    """An address that is 16-byte aligned and never dereferenced by a refused call."""
    buf = ctypes.create_string_buffer(256)
    p = (ctypes.addressof(buf) + 15) & ~15
    yield p
    del buf


def _call(fn, args, **change):
    a = dict(args)
    a.update(change)
    return fn(*a.values())


def test_quantize_refusals(lib, mem):  # noqa: F811
    ok = dict(x=mem, xdt=BF16, G=1, R=4, C=64, br=1, codes=mem, scales=mem, s=None)
    f = lambda **c: _call(lib.si_quantize_fp8, ok, **c)  # noqa: E731
    assert f(G=-1) == f(R=-1) == f(C=0) == f(br=0) == f(br=64) == INVALID
    assert f(xdt=E4M3) == f(xdt=7) == f(C=24) == UNSUPPORTED
    assert f(x=None) == f(codes=None) == f(scales=None) == INVALID
    assert f(x=mem + 8) == f(codes=mem + 8) == INVALID
    assert f(R=0, x=None, codes=None, scales=None) == f(G=0, x=None) == OK
    assert f(R=1 << 31, C=1 << 20) == f(G=1 << 33, R=1 << 33) == UNSUPPORTED
    # block counts that would wrap 64 bits, or a launch of 2^32 threads
    assert f(G=1 << 20, R=1 << 20, C=1 << 31) == f(G=1 << 20, R=1 << 20, C=1 << 31, br=128) \
        == UNSUPPORTED
    assert f(R=1 << 28) == f(R=1 << 20, C=128 << 8) == UNSUPPORTED
    assert f(R=1 << 30, br=128) == UNSUPPORTED


def test_matmul_refusals(lib, mem):  # noqa: F811
    ok = dict(x=mem, xs=mem, M=4, K=64, w=mem, ws=mem, N=8, y=mem, ydt=BF16, wk=None, n=0, s=None)
    f = lambda **c: _call(lib.si_matmul_fp8, ok, **c)  # noqa: E731
    assert f(M=-1) == f(N=0) == f(K=0) == INVALID
    assert f(ydt=E4M3) == f(K=72) == f(K=1 << 21) == f(M=1 << 25) == f(N=1 << 25) == UNSUPPORTED
    for name in ("x", "xs", "w", "ws", "y"):
        assert f(**{name: None}) == INVALID
    for name in ("x", "w", "y"):
        assert f(**{name: mem + 4}) == INVALID
    assert f(M=0, x=None, w=None, y=None) == OK


def test_route_refusals(lib, mem):  # noqa: F811
    ok = dict(x=mem, xdt=BF16, T=4, d=64, w=mem, wdt=BF16, E=8, bias=None, k=2, mode=SOFT,
              scale=ctypes.c_float(1.0), nv=None, ids=mem, wt=mem, ws=mem, n=1 << 20, s=None)
    f = lambda **c: _call(lib.si_moe_route, ok, **c)  # noqa: E731
    assert f(T=-1) == f(d=0) == f(E=0) == f(k=0) == f(k=9) == INVALID
    assert f(mode=0) == f(mode=3) == f(mode=RENORM) == f(mode=8 | SOFT) == INVALID
    assert f(scale=ctypes.c_float(math.inf)) == f(scale=ctypes.c_float(math.nan)) == INVALID
    assert f(xdt=E4M3) == f(wdt=F16) == f(xdt=F32) == UNSUPPORTED
    assert f(T=65536) == f(E=1025) == f(E=64, k=33) == f(d=60) == f(d=1 << 17) == UNSUPPORTED
    for name in ("x", "w", "ids", "wt"):
        assert f(**{name: None}) == INVALID
    assert f(x=mem + 8) == f(w=mem + 8) == INVALID
    assert f(ws=None) == f(n=64) == f(ws=mem + 4) == WORKSPACE
    assert f(T=0, x=None, ids=None, ws=None) == OK


FFN = dict(x=0, xdt=BF16, T=4, d=64, ids=0, wt=0, k=2, gu=0, gus=None, dn=0, dns=None, E=8, I=48,
           wdt=BF16, y=0, ydt=BF16, ws=0, n=1 << 20, s=None)


def test_ffn_refusals(lib, mem):  # noqa: F811
    ok = {n: (mem if v == 0 and n in ("x", "ids", "wt", "gu", "dn", "y", "ws") else v)
          for n, v in FFN.items()}
    f = lambda **c: _call(lib.si_moe_ffn, ok, **c)  # noqa: E731
    assert f(T=-1) == f(d=0) == f(k=0) == f(E=0) == f(I=0) == INVALID
    assert f(wdt=F16) == f(wdt=F32) == f(xdt=E4M3, wdt=E4M3) == f(xdt=F32, wdt=E4M3) == UNSUPPORTED
    assert f(ydt=F16) == f(ydt=E4M3) == UNSUPPORTED
    assert f(T=513) == f(k=33) == f(T=512, k=32) == f(E=65536) == UNSUPPORTED
    assert f(d=60) == f(I=44) == f(I=1 << 17) == f(d=1 << 17) == UNSUPPORTED
    assert f(d=32768, I=32768) == UNSUPPORTED            # an expert past 32-bit offsets
    assert f(wdt=E4M3, gus=mem, dns=mem, I=56) == UNSUPPORTED      # codes: multiples of 16
    assert f(wdt=E4M3) == f(wdt=E4M3, gus=mem) == f(wdt=E4M3, dns=mem) == INVALID
    for name in ("x", "ids", "wt", "gu", "dn", "y"):
        assert f(**{name: None}) == INVALID
    for name in ("x", "gu", "dn", "y"):
        assert f(**{name: mem + 8}) == INVALID
    assert f(ws=None) == f(n=64) == f(ws=mem + 8) == WORKSPACE
    assert f(T=0, x=None, ids=None, ws=None) == OK


def test_layer_refusals(lib, mem):  # noqa: F811
    ok = dict(x=mem, xdt=BF16, T=4, d=64, w=mem, rdt=BF16, bias=None, k=2, mode=SOFT,
              scale=ctypes.c_float(1.0), nv=None, gu=mem, gus=None, dn=mem, dns=None, E=8, I=48,
              wdt=BF16, ids=mem, wt=mem, y=mem, ydt=BF16, ws=mem, n=1 << 20, s=None)
    f = lambda **c: _call(lib.si_moe_layer, ok, **c)  # noqa: E731
    assert f(T=-1) == f(k=9) == f(I=0) == f(mode=0) == INVALID
    assert f(T=513) == f(rdt=F16) == f(wdt=F16) == f(ydt=F16) == f(E=1025) == UNSUPPORTED
    for name in ("x", "w", "gu", "dn", "y", "ids", "wt"):
        assert f(**{name: None}) == INVALID
    assert f(w=mem + 8) == f(y=mem + 8) == INVALID
    need = lib.si_moe_layer_workspace(4, 2, 8, 64, 48, BF16, BF16, BF16)
    assert f(ws=None) == f(n=need - 1) == f(ws=mem + 4) == WORKSPACE
    assert f(T=0, x=None, y=None, ws=None) == OK


def test_binding_refuses_host_tensors():
    import paper_2607_18081_amd as si
    x = torch.zeros(2, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        si.quantize_fp8(x)
    with pytest.raises(ValueError):
        si.moe_route(x, torch.zeros(4, 64, dtype=torch.bfloat16), 2)
    with pytest.raises(ValueError):
        si.matmul_fp8(x.view(torch.uint8), x, x, x)
