"""The 8-bit calls without a GPU: what they refuse, and what the binding refuses before them."""
import ctypes
import os
import subprocess

import pytest
import torch

from tests import host_lib as H

MOST = (1 << 31) - (1 << 16)
A, B, C, D, E, F = (i << 24 for i in range(1, 7))   # addresses; nothing is launched, nothing read


@pytest.fixture(scope="module")
def S():
    from paper_2509_11628_b200 import build, binding
    build.build()
    binding._lib()
    return binding


@pytest.fixture(scope="module")
def lib(S, tmp_path_factory):
    from paper_2509_11628_b200 import build
    cuda = os.path.join(os.path.dirname(os.path.dirname(os.path.realpath(build._nvcc()))), "include")
    so = os.path.join(str(tmp_path_factory.mktemp("host8")), "libspeca_host8.so")
    here = os.path.join(H.ROOT, "tests", "c_abi")
    srcs = [os.path.join(build.CSRC, n) for n in ("speca_layer.cpp", "speca_layer8.cpp", "speca_api.cpp")]
    srcs += [os.path.join(here, n) for n in ("host_runtime.cpp", "host_runtime8.cpp")]
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-fPIC", "-shared", "-Wl,-Bsymbolic", "-I", cuda, "-I", os.path.join(H.ROOT, "include"),
                           "-I", build.CSRC, "-o", so] + srcs)
    libdl = ctypes.CDLL(None)
    libdl.dlopen.restype = ctypes.c_void_p
    handle = libdl.dlopen(so.encode(), os.RTLD_LAZY)
    assert handle
    lib = ctypes.CDLL(so, handle=handle)
    vp, i32, i64, m8 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.POINTER(S.Matrix8Desc)
    lib.speca_quantize8.argtypes = [i64, i32, vp, i64, i32, m8, i32, vp]
    lib.speca_layer_quantize8.argtypes = [vp, i32, vp, i64, vp, m8, vp]
    lib.speca_layer_norm8.argtypes = [vp, i32, i32, vp, i64, vp, i64, vp, vp, vp, i64, vp, vp, vp, i64, m8, vp]
    lib.speca_layer_matmul8.argtypes = [vp, i32, i32, m8, m8, vp, i32, vp, i64, vp, i64, vp, vp, i64, m8, vp]
    lib.speca_layer_last_error.restype = ctypes.c_char_p
    return lib


def matrix(S, codes, code_stride, scales, scale_stride):
    return S.Matrix8Desc(codes, code_stride, scales, scale_stride)


ROWS, DIM = 6, 1152   # three groups of scales


def quantize(S, lib, layer, **kw):
    a = dict(dim=DIM, x=A, x_stride=DIM, out=(B, DIM, C, 4 * ROWS))
    a.update(kw)
    out = None if a["out"] is None else ctypes.byref(matrix(S, *a["out"]))
    return lib.speca_layer_quantize8(layer, a["dim"], a["x"], a["x_stride"], None, out, None)


def norm(S, lib, layer, **kw):
    a = dict(kind=1, dim=DIM, x=A, x_stride=DIM, branch=None, branch_stride=0, gate=None, scale=None, shift=None, mod_stride=DIM, weight=None,
             x_out=None, x_out_stride=0, out=(B, DIM, C, 4 * ROWS))
    a.update(kw)
    return lib.speca_layer_norm8(layer, a["kind"], a["dim"], a["x"], a["x_stride"], a["branch"], a["branch_stride"], a["gate"], a["scale"],
                                 a["shift"], a["mod_stride"], a["weight"], None, a["x_out"], a["x_out_stride"],
                                 ctypes.byref(matrix(S, *a["out"])), None)


def product(S, lib, layer, **kw):
    a = dict(n=256, k=DIM, a=(A, DIM, B, 4 * ROWS), w=(C, DIM, D, 4 * 256), bias=None, act=0, residual=None, residual_stride=256, gate=None,
             gate_stride=256, out=E, out_stride=256, eight=None)
    a.update(kw)
    ref = lambda m: None if m is None else ctypes.byref(matrix(S, *m))
    return lib.speca_layer_matmul8(layer, a["n"], a["k"], ref(a["a"]), ref(a["w"]), a["bias"], a["act"], a["residual"], a["residual_stride"],
                                   a["gate"], a["gate_stride"], None, a["out"], a["out_stride"], ref(a["eight"]), None)


@pytest.mark.parametrize("dtype", [0, 1])
def test_quantize_and_norm_refuse(S, lib, dtype):
    layer, _mem = H.layer(S, lib, [0, 2, ROWS], dtype)
    size = 4 if dtype == 0 else 2
    bad = [
        (dict(dim=0), "SHAPE"), (dict(dim=MOST + 1), "SHAPE"), (dict(dim=-5), "SHAPE"), (dict(x=None), "INVALID_ARG"), (dict(x_stride=-1), "SHAPE"),
        (dict(x=A + 1), "ALIGNMENT"), (dict(out=(None, DIM, C, 4 * ROWS)), "INVALID_ARG"), (dict(out=(B, DIM, None, 4 * ROWS)), "INVALID_ARG"),
        (dict(out=(B, DIM - 1, C, 4 * ROWS)), "SHAPE"), (dict(out=(B, DIM, C, 4 * ROWS - 4)), "SHAPE"), (dict(out=(B, DIM, C, 0)), "SHAPE"),
        (dict(out=(B, DIM, C + 2, 4 * ROWS)), "ALIGNMENT"), (dict(out=(B, DIM, C, 4 * ROWS + 2)), "ALIGNMENT"),
        (dict(out=(A, DIM, C, 4 * ROWS)), "INVALID_ARG"), (dict(out=(B, DIM, A, 4 * ROWS)), "INVALID_ARG"), (dict(out=(B, DIM, B, 4 * ROWS)), "INVALID_ARG"),
    ]
    before = lib.host_norms()
    for kw, status in bad:
        assert quantize(S, lib, layer, **kw) == getattr(S, "SPECA_ERR_" + status), kw
        assert norm(S, lib, layer, **kw) == getattr(S, "SPECA_ERR_" + status), kw
    assert quantize(S, lib, layer, out=None) == S.SPECA_ERR_INVALID_ARG
    for kw, status in [
        (dict(kind=2), "INVALID_ARG"), (dict(gate=D), "INVALID_ARG"), (dict(branch=D, branch_stride=-8), "SHAPE"), (dict(scale=D, mod_stride=-8), "SHAPE"),
        (dict(x_out=D, x_out_stride=DIM - 1), "SHAPE"), (dict(x_out=A, x_out_stride=DIM + 8), "INVALID_ARG"),
        (dict(branch=D, branch_stride=DIM, x_out=D, x_out_stride=DIM + 8), "INVALID_ARG"), (dict(x_out=B, x_out_stride=DIM), "INVALID_ARG"),
        (dict(x_out=C, x_out_stride=DIM), "INVALID_ARG"), (dict(branch=B, branch_stride=DIM), "INVALID_ARG"), (dict(weight=C), "INVALID_ARG"),
        (dict(weight=D, x_out=D, x_out_stride=DIM), "INVALID_ARG"), (dict(scale=D, x_out=D, x_out_stride=DIM), "INVALID_ARG"),
        (dict(shift=D, x_out=D, x_out_stride=DIM), "INVALID_ARG"),
        (dict(branch=E, branch_stride=DIM, gate=D, x_out=D, x_out_stride=DIM), "INVALID_ARG"),
        (dict(weight=D + 1), "ALIGNMENT"), (dict(shift=D + 1), "ALIGNMENT"), (dict(x_out=D + 1, x_out_stride=DIM), "ALIGNMENT"),
    ]:
        assert norm(S, lib, layer, **kw) == getattr(S, "SPECA_ERR_" + status), kw
        assert b"norm8" in lib.speca_layer_last_error(layer)
    assert lib.host_norms() == before
    # and what is fine: which rows take 16 bytes at once
    for kw, vectors in [({}, 1), (dict(x=A + size), 0), (dict(out=(B + 4, DIM, C, 4 * ROWS)), 0), (dict(out=(B, DIM + 4, C, 4 * ROWS)), 0),
                        (dict(dim=DIM - 8, out=(B, DIM, C, 4 * ROWS)), 0), (dict(x_stride=0), 1), (dict(out=(B, DIM, C, 4 * ROWS + 64)), 1)]:
        assert quantize(S, lib, layer, **kw) == S.SPECA_OK and lib.host_vectors() == vectors, kw
        assert norm(S, lib, layer, **kw) == S.SPECA_OK and lib.host_vectors() == vectors, kw
    assert norm(S, lib, layer, weight=D + size) == S.SPECA_OK and lib.host_vectors() == 0
    assert norm(S, lib, layer, branch=D, branch_stride=DIM, gate=E, x_out=A, x_out_stride=DIM) == S.SPECA_OK and lib.host_vectors() == 1
    # one row, one group of scales: those strides say nothing
    one, _m = H.layer(S, lib, [0, 1], dtype)
    assert quantize(S, lib, one, dim=512, x_stride=0, out=(B, 0, C, 0)) == S.SPECA_OK
    # none
    none, _m = H.layer(S, lib, [0, 0], dtype)
    assert quantize(S, lib, none, x=None, out=(None, 0, None, 0)) == S.SPECA_OK


def test_quantize_without_a_handle_refuses(S, lib):
    out = matrix(S, B, DIM, C, 4 * ROWS)
    call = lambda rows=ROWS, dim=DIM, x=A, dtype=1, device=0: lib.speca_quantize8(rows, dim, x, DIM, dtype, ctypes.byref(out), device, None)
    assert call() == S.SPECA_OK
    assert call(dtype=2) == S.SPECA_ERR_INVALID_ARG and call(device=2) == S.SPECA_ERR_INVALID_ARG and call(device=-1) == S.SPECA_ERR_INVALID_ARG
    assert call(rows=-1) == S.SPECA_ERR_SHAPE and call(rows=MOST + 1) == S.SPECA_ERR_SHAPE and call(dim=0) == S.SPECA_ERR_SHAPE
    assert call(x=None) == S.SPECA_ERR_INVALID_ARG
    assert lib.speca_quantize8(ROWS, DIM, A, DIM, 1, None, 0, None) == S.SPECA_ERR_INVALID_ARG
    assert lib.speca_quantize8(0, DIM, None, DIM, 1, ctypes.byref(matrix(S, None, 0, None, 0)), 0, None) == S.SPECA_OK


@pytest.mark.parametrize("dtype", [0, 1])
def test_product_refuses(S, lib, dtype):
    layer, _mem = H.layer(S, lib, [0, 2, ROWS], dtype)
    before = lib.host_products()
    for kw, status in [
        (dict(n=0), "SHAPE"), (dict(n=MOST + 1), "SHAPE"), (dict(k=0), "SHAPE"), (dict(k=MOST + 1), "SHAPE"), (dict(act=3), "INVALID_ARG"),
        (dict(a=None), "INVALID_ARG"), (dict(w=None), "INVALID_ARG"), (dict(a=(None, DIM, B, 4 * ROWS)), "INVALID_ARG"),
        (dict(w=(C, DIM, None, 1024)), "INVALID_ARG"), (dict(a=(A, DIM - 16, B, 4 * ROWS)), "SHAPE"), (dict(w=(C, DIM - 16, D, 1024)), "SHAPE"),
        (dict(a=(A, DIM, B, 4 * ROWS - 4)), "SHAPE"), (dict(w=(C, DIM, D, 1020)), "SHAPE"),
        (dict(a=(A + 8, DIM, B, 4 * ROWS)), "ALIGNMENT"), (dict(w=(C + 8, DIM, D, 1024)), "ALIGNMENT"), (dict(a=(A, DIM + 8, B, 4 * ROWS)), "ALIGNMENT"),
        (dict(w=(C, DIM + 8, D, 1024)), "ALIGNMENT"), (dict(w=(C, DIM, D + 2, 1024)), "ALIGNMENT"), (dict(a=(A, DIM, B, 4 * ROWS + 2)), "ALIGNMENT"),
        (dict(out=None), "INVALID_ARG"), (dict(eight=(F, 256, F + (1 << 20), 4 * ROWS)), "INVALID_ARG"),
        (dict(out=None, eight=(F, 256, F + (1 << 20), 4 * ROWS), residual=D), "INVALID_ARG"),
        (dict(out=None, eight=(F, 256, F + (1 << 20), 4 * ROWS), gate=D), "INVALID_ARG"),
        (dict(out=None, eight=(F, 255, F + (1 << 20), 4 * ROWS)), "SHAPE"), (dict(out=None, eight=(F, 256, F + 2, 4 * ROWS)), "ALIGNMENT"),
        (dict(out=None, eight=(A, 256, F, 4 * ROWS)), "INVALID_ARG"), (dict(out=None, eight=(F, 256, D, 4 * ROWS)), "INVALID_ARG"),
        (dict(out=None, eight=(F, 256, F, 4 * ROWS)), "INVALID_ARG"),
        (dict(out_stride=255), "SHAPE"), (dict(residual=F, residual_stride=-256), "SHAPE"), (dict(gate=F, gate_stride=-256), "SHAPE"),
        (dict(residual=E, residual_stride=264), "INVALID_ARG"), (dict(bias=E), "INVALID_ARG"), (dict(gate=E), "INVALID_ARG"), (dict(out=A), "INVALID_ARG"),
        (dict(out=D), "INVALID_ARG"), (dict(out=E + 1), "ALIGNMENT"), (dict(bias=F + 1), "ALIGNMENT"), (dict(residual=F + 1), "ALIGNMENT"),
        (dict(gate=F + 1), "ALIGNMENT"),
    ]:
        assert product(S, lib, layer, **kw) == getattr(S, "SPECA_ERR_" + status), kw
        assert b"matmul8" in lib.speca_layer_last_error(layer)
    assert lib.host_products() == before
    size = 4 if dtype == 0 else 2
    for kw, vectors in [({}, 1), (dict(residual=E), 1), (dict(residual=F, residual_stride=0), 1), (dict(out=E + size), 0), (dict(bias=F + size), 0),
                        (dict(gate=F, gate_stride=257), 0), (dict(out=None, eight=(F, 256, F + (1 << 20), 4 * ROWS)), 1),
                        (dict(out=None, eight=(F + 8, 256, F + (1 << 20), 4 * ROWS)), 0), (dict(n=250), 1)]:
        assert product(S, lib, layer, **kw) == S.SPECA_OK, (kw, lib.speca_layer_last_error(layer))
        assert lib.host_vectors() == vectors, kw
    none, _m = H.layer(S, lib, [0, 0], dtype)
    assert product(S, lib, none, a=(None, 0, None, 24), out=None) == S.SPECA_OK
    assert product(S, lib, none, a=(None, 0, None, 24), out=E, eight=(F, 256, F + 4, 0)) == S.SPECA_ERR_INVALID_ARG
    assert lib.speca_layer_matmul8(None, 1, 1, None, None, None, 0, None, 0, None, 0, None, None, 0, None, None) == S.SPECA_ERR_INVALID_ARG


def test_product_of_the_longest_rows(S, lib):
    layer, _mem = H.layer(S, lib, [0, 2, ROWS], 1)
    k = S.SPECA_MAX_K8
    far = dict(a=(A, k + 16, B, 4 * ROWS), w=(C, k + 16, D, 1024))
    assert product(S, lib, layer, k=k, **far) == S.SPECA_OK
    assert product(S, lib, layer, k=k + 1, **far) == S.SPECA_ERR_SHAPE and b"262144" in lib.speca_layer_last_error(layer)


def test_the_binding_refuses_what_it_cannot_marshal(S):
    codes = torch.zeros(4, 600, dtype=torch.uint8).view(torch.float8_e4m3fn)
    scales = torch.zeros(2, 4, 4, dtype=torch.uint8).view(torch.float8_e8m0fnu)
    m = S.Matrix8(codes, scales)
    assert m.shape == (4, 600)
    S.Matrix8(codes[:, :513], scales)
    with pytest.raises(TypeError):
        S.Matrix8(codes.view(torch.uint8), scales)
    with pytest.raises(TypeError):
        S.Matrix8(codes, scales.view(torch.uint8))
    for bad in (scales[:1], scales[:, :3], scales[:, :, :3], scales.reshape(-1)):
        with pytest.raises(ValueError):
            S.Matrix8(codes, bad)
    with pytest.raises(ValueError):
        S.Matrix8(codes[:, :512], scales)
    with pytest.raises(ValueError):
        S.Matrix8(codes.reshape(2, 2, 600), scales)
    with pytest.raises(TypeError):
        S.Matrix8(codes.T.contiguous().T, scales)
    with pytest.raises(TypeError):
        S.Matrix8(codes, scales.transpose(0, 1).contiguous().transpose(0, 1))
    for x in (torch.zeros(4, 600), torch.zeros(4, 600, dtype=torch.float16)):
        with pytest.raises(TypeError):
            S.quantize8(x)
    assert S.Matrix8.empty(3, 513, "cpu").codes.stride(0) == 528
