"""The entry points of the 8-bit path refuse what they do not take, before any device work."""
import pytest
import torch

from paper_2410_09615_b200 import binding as K, build

INVALID, SHAPE = K.SLIM_ERR_INVALID_ARG, K.SLIM_ERR_UNSUPPORTED_SHAPE
P = 64                    # a fake, aligned, never dereferenced address
Q = 128


@pytest.fixture(scope="module")
def lib():
    build.build()
    return K.lib()


def norm(lib, **kw):
    a = dict(X=P, residual=Q, gamma=P, eps=1e-5, b=1, d=64, H=None, Y=256) | kw
    return lib.slim_rmsnorm(a["X"], a["residual"], a["gamma"], a["eps"], a["b"], a["d"], a["H"], a["Y"], None)


def norm8(lib, **kw):
    a = dict(X=P, residual=Q, gamma=P, eps=1e-5, b=1, d=64, format=0, H=None, codes=256, scales=P) | kw
    return lib.slim_rmsnorm_fp8(a["X"], a["residual"], a["gamma"], a["eps"], a["b"], a["d"], a["format"], a["H"], a["codes"], a["scales"], None)


def quant(lib, **kw):
    a = dict(X=P, b=1, d=64, format=0, codes=Q, scales=P) | kw
    return lib.slim_quant_fp8(a["X"], a["b"], a["d"], a["format"], a["codes"], a["scales"], None)


def pack(lib, **kw):
    a = dict(W=P, type=0, d_out=1, d_in=64, format=0, codes=Q, scales=P) | kw
    return lib.slim_pack_fp8(a["W"], a["type"], a["d_out"], a["d_in"], a["format"], a["codes"], a["scales"], None)


def linear(lib, **kw):
    a = dict(Xq=P, Xs=P, xf=0, b=1, Wq=P, Ws=P, wf=0, d_out=16, d_in=64, Y=256, status=None) | kw
    return lib.slim_linear_fwd_fp8(a["Xq"], a["Xs"], a["xf"], a["b"], a["Wq"], a["Ws"], a["wf"], a["d_out"], a["d_in"], a["Y"], a["status"], None)


@pytest.mark.parametrize("call, name", [(norm, "X"), (norm, "gamma"), (norm, "Y"), (norm8, "X"), (norm8, "gamma"), (norm8, "codes"), (norm8, "scales"),
                                        (quant, "X"), (quant, "codes"), (quant, "scales"), (pack, "W"), (pack, "codes"), (pack, "scales"),
                                        (linear, "Xq"), (linear, "Xs"), (linear, "Wq"), (linear, "Ws"), (linear, "Y")])
def test_null_and_misaligned_pointers(lib, call, name):
    assert call(lib, **{name: None}) == INVALID
    assert call(lib, **{name: P + (2 if name in ("scales", "Xs", "Ws") else 8)}) == INVALID


@pytest.mark.parametrize("call, name", [(norm, "residual"), (norm, "H"), (norm8, "residual"), (norm8, "H"), (linear, "status")])
def test_misaligned_optional_pointers(lib, call, name):
    assert call(lib, **{name: P + 2}) == INVALID


@pytest.mark.parametrize("call, rows, cols", [(norm, "b", "d"), (norm8, "b", "d"), (quant, "b", "d"), (pack, "d_out", "d_in"), (linear, "b", "d_in")])
def test_sizes(lib, call, rows, cols):
    for n in (0, -1, -(1 << 31)):
        assert call(lib, **{rows: n}) == INVALID and call(lib, **{cols: n}) == INVALID
    for n in (1, 8, 17, 120):
        assert call(lib, **{cols: n}) == SHAPE


def test_more_of_each(lib):
    assert linear(lib, d_out=0) == INVALID and linear(lib, d_out=-5) == INVALID
    for call in (norm, norm8):
        assert call(lib, d=32768 + 16) == SHAPE
        for eps in (0.0, -1e-5, float("nan"), float("inf")):
            assert call(lib, eps=eps) == INVALID
    for f in (-1, 2):
        assert norm8(lib, format=f) == INVALID and quant(lib, format=f) == INVALID and pack(lib, format=f) == INVALID
        assert linear(lib, xf=f) == INVALID and linear(lib, wf=f) == INVALID and pack(lib, type=f) == INVALID
    assert norm(lib, Y=P) == INVALID and norm(lib, Y=Q) == INVALID and norm(lib, Y=256, H=256) == INVALID      # an output in place of an input


@pytest.mark.parametrize("call, name", [(quant, "d"), (pack, "d_out"), (pack, "d_in"), (linear, "b"), (linear, "d_out"), (linear, "d_in")])
def test_sizes_whose_tiles_pass_31_bits(lib, call, name):
    for n in ((1 << 31) - 496, (1 << 31) - 16):
        assert call(lib, **{name: n}) == INVALID


def test_a_missing_device_is_an_error_not_a_fall_back(lib):
    if torch.cuda.is_available():
        pytest.skip("there is a device")
    assert linear(lib) in (K.SLIM_ERR_CUDA, K.SLIM_ERR_ARCH)


def test_binding_takes_cuda_tensors_only(lib):
    x = torch.zeros(2, 64, dtype=torch.bfloat16)
    with pytest.raises(TypeError):
        K.slim_rmsnorm(x, x[0], 1e-5)
    with pytest.raises(TypeError):
        K.slim_rmsnorm_fp8(x, x[0], 1e-5)
    with pytest.raises(TypeError):
        K.slim_quant_fp8(x)
    with pytest.raises(TypeError):
        K.slim_pack_fp8(x)
    with pytest.raises(TypeError):
        K.slim_linear_fwd_fp8(x, x, x, x)
    with pytest.raises(TypeError):
        K.slim_rmsnorm_fp8(x, x[0], 1e-5, dtype=torch.int8)
