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


class Tensor:
    """What the binding asks of a tensor, for a GPU that this machine need not have."""

    def __init__(self, dtype, *shape, device=0):
        import torch
        self.dtype, self.shape, self.device = dtype, torch.Size(shape), torch.device("cuda", device)
        self.is_cuda = True

    def get_device(self): return self.device.index
    def is_contiguous(self): return True
    def data_ptr(self): return 64
    def dim(self): return len(self.shape)
    def stride(self, dim=None):
        strides = [1] * len(self.shape)
        for i in reversed(range(len(strides) - 1)):
            strides[i] = strides[i + 1] * self.shape[i + 1]
        return strides if dim is None else strides[dim]


class Stream:
    def __init__(self, device): self.device_index, self.cuda_stream = device, 0


@pytest.fixture
def calls(monkeypatch):
    """Names of the calls that got through the binding's checks; the current device is 0."""
    import torch
    from paper_2605_17889_amd import binding

    class Library:
        def __getattr__(self, name):
            return lambda *arguments: made.append(name) or 0

    made = []
    monkeypatch.setattr(binding, "lib", Library)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0, raising=False)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda device: 0, raising=False)
    return made


def arguments_of(name):
    """Arguments of a complete call, the context apart, and how many of its first ones are tensors' places."""
    import torch
    bf, i8, f32, i32 = torch.bfloat16, torch.int8, torch.float32, torch.int32
    T = Tensor
    matrices = lambda: [t for n, k in ((128, 512), (128, 512), (512, 128)) for t in (T(i8, 2, n, k), T(f32, 2, n))]
    return {
        "moe_rmsnorm_i8": lambda: [T(bf, 4, 64), T(bf, 4, 64), T(bf, 64), 1e-6, T(bf, 4, 64), T(bf, 4, 64), T(i8, 4, 64), T(f32, 4)],
        "moe_quantize_i8": lambda: [T(bf, 4, 64), T(i8, 4, 64), T(f32, 4)],
        "moe_gemm_i8": lambda: [T(i8, 4, 256), T(f32, 4), T(i32, 2), 4, 1, 64, 256, T(i8, 64, 256), T(f32, 64), T(bf, 4, 64)],
        "moe_expert_ffn_i8": lambda: [T(i8, 4, 512), T(f32, 4), T(i32, 3), 4, *matrices(), T(bf, 4, 512)],
        "moe_layer_forward_i8": lambda: [T(bf, 4, 512), T(i8, 4, 512), T(f32, 4), T(f32, 512, 2), T(f32, 2), *matrices(), 4,
                                         T(bf, 4, 512)],
    }[name]()


@pytest.mark.parametrize("name", ["moe_rmsnorm_i8", "moe_quantize_i8", "moe_gemm_i8", "moe_expert_ffn_i8", "moe_layer_forward_i8"])
def test_tensors_and_streams_of_another_gpu_are_refused(calls, name):
    """Kernels run on the current GPU, the context's: memory of another one need not be mapped there."""
    from types import SimpleNamespace
    from paper_2605_17889_amd import binding
    context = [SimpleNamespace(_h=None, device=0, d_model=512, d_ff=128, E=2)] if "norm" not in name and "quant" not in name else []
    call = getattr(binding, name)
    call(*context, *arguments_of(name))
    call(*context, *arguments_of(name), stream=Stream(0))
    assert calls == [name] * 2
    for i, a in enumerate(arguments_of(name)):
        if isinstance(a, Tensor):
            other = arguments_of(name)
            other[i] = Tensor(a.dtype, *a.shape, device=1)
            with pytest.raises(binding.MoeError):
                call(*context, *other)
    with pytest.raises(binding.MoeError):
        call(*context, *arguments_of(name), stream=Stream(1))
    assert calls == [name] * 2


def test_rows_that_are_missing_are_refused(calls):
    from paper_2605_17889_amd import binding
    for name in ("moe_rmsnorm_i8", "moe_quantize_i8"):
        with pytest.raises(binding.MoeError):
            getattr(binding, name)(None, *arguments_of(name)[1:])
    assert not calls
