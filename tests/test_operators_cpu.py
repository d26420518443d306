"""Limits of the block-scaled 8-bit matrices and the expert layers that the host answers for."""
from tests.test_experts_cpu import BF16, INVALID, UNSUPPORTED, _call, mem  # noqa: F401  (fixture)
from tests.test_lib_cpu import lib  # noqa: F401  (fixture)


def test_quantize_block_limit(lib, mem):  # noqa: F811
    """16 blocks of 1 x 128 a work-group of 256 threads, and a launch holds fewer than 2^32 threads:
    2^24 work-groups are one too many. (An accepted size reaches the check of the addresses.)"""
    ok = dict(x=mem, xdt=BF16, G=1, R=4, C=64, br=1, codes=mem, scales=mem, s=None)
    f = lambda **c: _call(lib.si_quantize_fp8, ok, **c)  # noqa: E731
    top = (1 << 28) - 16
    assert f(R=top, x=None) == f(G=16, R=top // 16, x=None) == INVALID
    for n in (top + 1, top + 15, 1 << 28):
        assert f(R=n) == f(R=n, x=None) == UNSUPPORTED
    assert f(R=(1 << 26) - 4, C=512, x=None) == INVALID
    assert f(R=(1 << 26) - 3, C=512) == f(R=(1 << 26) - 1, C=400) == UNSUPPORTED
    # 128 x 128 blocks: one work-group of 512 threads each
    assert f(R=((1 << 23) - 1) * 128, br=128, x=None) == INVALID
    assert f(R=((1 << 23) - 1) * 128 + 1, br=128) == UNSUPPORTED
