"""The library's host side compiled against tests/c_abi/host_runtime.cpp: handles and argument checks without a GPU."""
import ctypes
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def load(folder):
    """Builds it into ``folder``; returns the library."""
    from paper_2509_11628_b200 import build
    cuda = os.path.join(os.path.dirname(os.path.dirname(os.path.realpath(build._nvcc()))), "include")
    so = os.path.join(str(folder), "libspeca_host.so")
    # symbols bind inside the library: a CUDA runtime that torch has loaded stays out
    srcs = [os.path.join(build.CSRC, "speca_layer.cpp"), os.path.join(build.CSRC, "speca_api.cpp"),
            os.path.join(ROOT, "tests", "c_abi", "host_runtime.cpp")]
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-fPIC", "-shared", "-Wl,-Bsymbolic", "-I", cuda, "-I", os.path.join(ROOT, "include"),
                           "-I", build.CSRC, "-o", so] + srcs)
    # lazily: the cache's kernels are not there
    libdl = ctypes.CDLL(None)
    libdl.dlopen.restype = ctypes.c_void_p
    handle = libdl.dlopen(so.encode(), os.RTLD_LAZY)
    assert handle
    lib = ctypes.CDLL(so, handle=handle)
    lib.host_events.restype = ctypes.c_char_p
    vp, i32, i64 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64
    lib.speca_layer_modulate.argtypes = [vp, i32, vp, i64, vp, i64, vp, vp, vp, i64, vp, vp, i64, vp, i64, vp]
    lib.speca_layer_rope.argtypes = [vp] + [vp, i64, i64] * 4 + [vp] * 5
    lib.speca_layer_attention.argtypes = [vp] + [vp, i64, i64] * 4 + [vp] * 4
    return lib


class Memory:
    """Host bytes that stand for device memory, 256-byte aligned."""

    def __init__(self, nbytes):
        self.raw = ctypes.create_string_buffer(nbytes + 256)
        self.ptr = (ctypes.addressof(self.raw) + 255) // 256 * 256


def layer(S, lib, q_start, dtype, **kw):
    """(handle, its memory) of a layer on the host library."""
    args = dict(kv_start=None, n_heads=0, n_kv_heads=0, head_dim=0, causal=False, scale=0.0, norm_eps=0.0, axis_dims=(),
                theta=10000.0, pairing=0)
    args.update(kw)
    cfg = S._layer_config(q_start, dtype, **args)
    n = ctypes.c_size_t(0)
    assert lib.speca_layer_workspace_bytes(ctypes.byref(cfg), ctypes.byref(n)) == S.SPECA_OK
    mem = Memory(n.value)
    cfg.workspace, cfg.workspace_bytes, cfg.device = mem.ptr, n.value, 0
    out = ctypes.c_void_p(None)
    status = lib.speca_layer_create(ctypes.byref(cfg), ctypes.byref(out))
    assert status == S.SPECA_OK, status
    return out, mem
