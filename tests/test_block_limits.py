"""Sizes beyond what a launch takes (2^32 - 1 threads along a dimension) are refused as shapes by the operators around the melded layer, before
anything is launched: nothing is read at these addresses.  Numbers of double precision that fp32 does not hold are refused, too."""
import ctypes as c

import pytest

from test_block_abi import OK, SHAPE, L, NormBwd, NormFwd  # noqa: F401


def norm_fwd(L, **kw):  # noqa: F811
    a = dict(x=OK, b=OK, w=OK, scale=1.0, eps=1e-5, xt=0, T=4, d=64, ld_x=64, ld_b=64, s=OK, h=OK, rstd=OK)
    return L.falqon_norm_fwd(c.byref(NormFwd(**{**a, **kw})), None)


def norm_bwd(L, **kw):  # noqa: F811
    a = dict(dh=OK, ds=OK, s=OK, b=OK, w=OK, rstd=OK, xt=0, T=4, d=64, ld_dh=64, ld_ds=64, ld_s=64, ld_b=64, dx=OK, db=OK, scale=1.0)
    return L.falqon_norm_bwd(c.byref(NormBwd(**{**a, **kw})), None)


def test_passes_over_a_matrix(L):  # noqa: F811
    fwd = lambda T, m, xt: L.falqon_swiglu_fwd(OK, OK, xt, T, m, m, m, OK, None, None, None, None, None)  # noqa: E731
    bwd = lambda T, m, xt: L.falqon_swiglu_bwd(OK, m, OK, OK, None, None, m, m, xt, T, m, OK, OK, None)  # noqa: E731
    quantize = lambda T, m, xt, fmt: L.falqon_mx_quantize(OK, xt, T, m, m, fmt, OK, OK, None)  # noqa: E731
    values = lambda T, m, xt, fmt: L.falqon_mx_dequantize(OK, OK, fmt, T, m, OK, xt, m, None)  # noqa: E731
    for T, m, xt in ((1 << 20, 1 << 15, 0), (1 << 24, 1 << 15, 0), (1 << 20, 1 << 14, 1), (1 << 24, 1 << 12, 1), (1 << 24, 2048, 0), ((1 << 24) - 1, 2064, 0)):
        assert fwd(T, m, xt) == SHAPE and bwd(T, m, xt) == SHAPE, (T, m, xt)
        assert quantize(T, m, xt, 0) == SHAPE and values(T, m, xt, 0) == SHAPE, (T, m, xt)
        if m % 32 == 0:
            assert quantize(T, m, xt, 1) == SHAPE and values(T, m, xt, 1) == SHAPE, (T, m, xt)


def test_rows(L):  # noqa: F811
    for T, d, xt in ((1 << 24, 2048, 0), (1 << 24, 16384, 0), (1 << 22, 16384, 1), (1 << 24, 1024, 1), (1 << 22, 16384, 0)):
        assert norm_fwd(L, T=T, d=d, ld_x=d, ld_b=d, xt=xt) == SHAPE, (T, d, xt)
    assert L.falqon_token_logprob(OK, 0, 1 << 24, 8, 8, OK, OK, OK, OK, 1 << 40, None) == SHAPE
    assert L.falqon_token_logprob_bwd(OK, OK, 0, 1 << 24, 8, 8, OK, OK, OK + 64, 8, None) == SHAPE


def test_products(L):  # noqa: F811
    f = lambda T, n, m, x=None: L.falqon_mx4_linear(x, OK, OK, T, n, m, OK, OK, OK, 0, None)  # noqa: E731
    assert f(1 << 24, 32, 1 << 20) == SHAPE                                     # 2^44 outputs
    assert f(1 << 24, 32, 1 << 16) == SHAPE                                     # 2^24 tiles of 256 x 256
    assert f(1 << 20, 1 << 15, 64, OK) == SHAPE                                 # the quantizer's pass over x
    assert f(1 << 24, 32, (1 << 16) - 16) == SHAPE                              # a tile more by its last columns


@pytest.mark.parametrize("value", [1e39, -1e39, 1e300])
def test_numbers_beyond_fp32(L, value):  # noqa: F811
    assert norm_fwd(L, scale=value) == SHAPE and norm_bwd(L, scale=value) == SHAPE
    assert L.falqon_preference_loss(OK, OK, OK, 4, 2, value, 0.0, OK, OK, OK, OK, 64, None) == SHAPE
