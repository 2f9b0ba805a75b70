"""What the 4-bit entry points and the routers by scores refuse, through the C ABI and the binding, without a GPU: nothing is
launched when a call is refused, so pointers that no call may touch stand in for tensors."""
import ctypes as C
from types import SimpleNamespace

import pytest

from test_i8_refusals import Stream, Tensor, calls, lib  # noqa: F401

INVALID, UNSUPPORTED = -1, -2
P, NULL = C.c_void_p(64), C.c_void_p(0)


def quantize(lib, x=P, stride=64, T=4, d=64, q=P, scale=P):
    return lib.moe_quantize_mx4(x, C.c_int64(stride), C.c_int32(T), C.c_int32(d), q, scale, NULL)


def dequantize(lib, q=P, scale=P, T=4, d=64, y=P):
    return lib.moe_dequantize_mx4(q, scale, C.c_int32(T), C.c_int32(d), y, NULL)


@pytest.mark.parametrize("change", [dict(x=NULL), dict(q=NULL), dict(scale=NULL), dict(T=-1), dict(d=0), dict(d=-32), dict(stride=63)])
def test_rows_to_4_bits_refuse(lib, change):  # noqa: F811
    assert quantize(lib, **change) == INVALID


@pytest.mark.parametrize("change", [dict(q=NULL), dict(scale=NULL), dict(y=NULL), dict(T=-1), dict(d=0)])
def test_rows_from_4_bits_refuse(lib, change):  # noqa: F811
    assert dequantize(lib, **change) == INVALID


def test_widths_that_are_no_blocks_or_too_long(lib):  # noqa: F811
    for d in (1, 31, 33, 48, (1 << 22) + 32):
        assert quantize(lib, d=d, stride=d) == UNSUPPORTED
        assert dequantize(lib, d=d) == UNSUPPORTED
    assert quantize(lib, T=0, x=NULL, q=NULL, scale=NULL) == 0 and dequantize(lib, T=0, q=NULL, scale=NULL, y=NULL) == 0


def test_more_rows_than_a_launch_holds(lib):  # noqa: F811
    """A launch of 256 threads for 16 rows of one run holds fewer than 2^32 threads."""
    for T, d in ((2**31 - 1, 32), (2**28 - 15, 32), (2**31 - 1, 512), (2**27 - 15, 512), (2**20, 1 << 17)):
        assert quantize(lib, T=T, d=d, stride=d) == UNSUPPORTED
        assert dequantize(lib, T=T, d=d) == UNSUPPORTED


def test_calls_without_a_context_are_refused(lib):  # noqa: F811
    i = C.c_int32
    assert lib.moe_gemm_mx4(NULL, P, P, NULL, i(4), i(1), i(64), i(256), P, P, P, i(0), NULL) == INVALID
    assert lib.moe_expert_ffn_mx4(NULL, P, P, P, i(4), P, P, P, P, P, P, P, NULL) == INVALID
    assert lib.moe_layer_forward_mx4(NULL, P, P, NULL, NULL, NULL, P, P, P, P, P, P, i(4), P, NULL) == INVALID
    assert lib.moe_route_scored(NULL, P, P, NULL, NULL, P, i(4), P, P, NULL, NULL) == INVALID
    assert lib.moe_route_scored_from_logits(NULL, P, NULL, P, i(4), P, P, NULL) == INVALID


def test_scores_that_there_are_not():
    from paper_2605_17889_amd import binding
    with pytest.raises(binding.MoeError):
        binding.MoeScoring("tanh")
    sc = binding.MoeScoring("softmax", 4, 2, 1, False, 2.5)
    assert (sc.score, sc.groups, sc.top_groups, sc.group_best, sc.renormalise, sc.scale) == (0, 4, 2, 1, 0, 2.5)
    assert C.sizeof(sc) == 24


def arguments_of(name):
    import torch
    from paper_2605_17889_amd import binding
    bf, u8, f32, i32 = torch.bfloat16, torch.uint8, torch.float32, torch.int32
    T, sc = Tensor, binding.MoeScoring("sigmoid")
    matrices = lambda: [t for n, k in ((128, 512), (128, 512), (512, 128))
                        for t in (T(u8, 2, n, k // 2), T(u8, 2, -(-k // 256), n, 8))]
    return {
        "moe_quantize_mx4": lambda: [T(bf, 4, 64), T(u8, 4, 32), T(u8, 1, 4, 8)],
        "moe_dequantize_mx4": lambda: [T(u8, 4, 32), T(u8, 1, 4, 8), T(bf, 4, 64)],
        "moe_gemm_mx4": lambda: [T(u8, 4, 144), T(u8, 2, 4, 8), T(i32, 2), 4, 1, 64, 288, T(u8, 64, 144), T(u8, 2, 64, 8), T(bf, 4, 64)],
        "moe_expert_ffn_mx4": lambda: [T(u8, 4, 256), T(u8, 2, 4, 8), T(i32, 3), 4, *matrices(), T(bf, 4, 512)],
        "moe_layer_forward_mx4": lambda: [T(bf, 4, 512), T(f32, 512, 2), T(f32, 2), T(f32, 2), sc, *matrices(), 4, T(bf, 4, 512)],
        "moe_route_scored": lambda: [T(bf, 4, 512), T(f32, 512, 2), T(f32, 2), T(f32, 2), sc, 4, T(i32, 4, 2), T(f32, 4, 2), T(f32, 4, 2)],
        "moe_route_scored_from_logits": lambda: [T(f32, 4, 2), T(f32, 2), sc, 4, T(i32, 4, 2), T(f32, 4, 2)],
    }[name]()


NAMES = ["moe_quantize_mx4", "moe_dequantize_mx4", "moe_gemm_mx4", "moe_expert_ffn_mx4", "moe_layer_forward_mx4", "moe_route_scored",
         "moe_route_scored_from_logits"]


def context_of(name):
    return [] if "quant" in name else [SimpleNamespace(_h=None, device=0, d_model=512, d_ff=128, E=2, k=2)]


@pytest.mark.parametrize("name", NAMES)
def test_tensors_and_streams_of_another_gpu_or_shape_are_refused(calls, name):  # noqa: F811
    import torch
    from paper_2605_17889_amd import binding
    call = getattr(binding, name)
    call(*context_of(name), *arguments_of(name))
    call(*context_of(name), *arguments_of(name), stream=Stream(0))
    assert calls == [name] * 2
    for i, a in enumerate(arguments_of(name)):
        if isinstance(a, Tensor):
            longer = (a.shape[0] + 1, *a.shape[1:])
            for t in (Tensor(a.dtype, *a.shape, device=1), Tensor(torch.float64, *a.shape), Tensor(a.dtype, *longer)):
                other = arguments_of(name)
                other[i] = t
                with pytest.raises(binding.MoeError):
                    call(*context_of(name), *other)
    with pytest.raises(binding.MoeError):
        call(*context_of(name), *arguments_of(name), stream=Stream(1))
    assert calls == [name] * 2


def test_scoring_has_to_be_one(calls):  # noqa: F811
    from paper_2605_17889_amd import binding
    for name in ("moe_layer_forward_mx4", "moe_route_scored", "moe_route_scored_from_logits"):
        other = [("sigmoid" if isinstance(a, binding.MoeScoring) else a) for a in arguments_of(name)]
        with pytest.raises(binding.MoeError):
            getattr(binding, name)(*context_of(name), *other)
    assert not calls


def test_rows_that_are_missing_are_refused(calls):  # noqa: F811
    from paper_2605_17889_amd import binding
    with pytest.raises(binding.MoeError):
        binding.moe_quantize_mx4(None, *arguments_of("moe_quantize_mx4")[1:])
    with pytest.raises(binding.MoeError):
        binding.moe_dequantize_mx4(*arguments_of("moe_dequantize_mx4")[:2], None)
    assert not calls
