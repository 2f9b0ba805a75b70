"""What the 8-bit entry points refuse, through the C ABI and without a GPU: nothing is launched when a call returns
MOE_ERR_INVALID_ARG or MOE_ERR_UNSUPPORTED_SHAPE, so pointers that no call may touch stand in for tensors."""
import ctypes as C

import pytest

INVALID, UNSUPPORTED = -1, -2
P = C.c_void_p(64)           # never read: every call below is refused
NULL = C.c_void_p(0)


@pytest.fixture(scope="module")
def lib():
    import os
    from paper_2605_17889_amd import build
    if not os.path.exists(build.LIB):
        build.build()
    return C.CDLL(build.LIB)


def norm(lib, x=P, stride=64, residual=P, kind=0, weight=P, eps=1e-6, T=4, d=64, out=P, y=P, q=P, scale=P):
    return lib.moe_rmsnorm_i8(x, C.c_int64(stride), residual, C.c_int(kind), weight, C.c_float(eps), C.c_int32(T),
                              C.c_int32(d), out, y, q, scale, NULL)


@pytest.mark.parametrize("change", [
    dict(x=NULL), dict(weight=NULL), dict(stride=63), dict(stride=-64), dict(kind=2), dict(kind=-1), dict(eps=0.0),
    dict(eps=-1e-6), dict(eps=float("nan")), dict(eps=float("inf")), dict(T=-1), dict(d=0), dict(d=-8), dict(q=NULL),
    dict(scale=NULL), dict(out=NULL, y=NULL, q=NULL, scale=NULL)])
def test_norm_refuses(lib, change):
    assert norm(lib, **change) == INVALID


def test_norm_refuses_rows_too_long(lib):
    assert norm(lib, d=65537, stride=65537) == UNSUPPORTED


def test_norm_of_no_rows_needs_no_pointers(lib):
    assert norm(lib, T=0, x=NULL, residual=NULL, weight=NULL, out=NULL, y=NULL, q=NULL, scale=NULL) == 0


def quantize(lib, x=P, stride=64, T=4, d=64, q=P, scale=P):
    return lib.moe_quantize_i8(x, C.c_int64(stride), C.c_int32(T), C.c_int32(d), q, scale, NULL)


@pytest.mark.parametrize("change", [dict(x=NULL), dict(q=NULL), dict(scale=NULL), dict(T=-1), dict(d=0), dict(stride=1)])
def test_quantize_refuses(lib, change):
    assert quantize(lib, **change) == INVALID


def test_quantize_refuses_rows_too_long(lib):
    assert quantize(lib, d=65537, stride=70000) == UNSUPPORTED
    assert quantize(lib, T=0, x=NULL, q=NULL, scale=NULL) == 0


def gemm(lib, ctx=NULL, x=P, xs=P, offsets=NULL, R=4, E=1, N=64, K=256, w=P, ws=P, out=P, kind=0):
    return lib.moe_gemm_i8(ctx, x, xs, offsets, C.c_int32(R), C.c_int32(E), C.c_int32(N), C.c_int32(K), w, ws, out,
                           C.c_int(kind), NULL)


def test_products_without_a_context_are_refused(lib):
    assert gemm(lib) == INVALID
    assert lib.moe_expert_ffn_i8(NULL, P, P, P, C.c_int32(4), P, P, P, P, P, P, P, NULL) == INVALID
    assert lib.moe_layer_forward_i8(NULL, P, P, P, P, NULL, P, P, P, P, P, P, C.c_int32(4), P, NULL) == INVALID
