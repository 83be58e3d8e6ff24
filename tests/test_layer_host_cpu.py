"""The host side of the layer calls without a GPU: what a handle asks of the device, and what the calls refuse."""
import ctypes

import pytest

from tests import host_lib as H

HEADS = dict(n_heads=8, n_kv_heads=2, head_dim=64)


@pytest.fixture(scope="module")
def S():
    from paper_2509_11628_b200 import binding
    return binding


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    return H.load(tmp_path_factory.mktemp("host"))


def test_work_pending_on_the_workspace_ends_before_it_is_written(S, lib):
    # memory that a stream's allocator hands out may still be written by kernels of that stream; one of them behind
    # the upload would leave its bytes where the work list was
    lib.host_events_clear()
    _, _ = H.layer(S, lib, [0, 4, 300], S.SPECA_BF16, kv_start=[0, 4, 9000], axis_dims=(16, 24, 24), **HEADS)
    events = lib.host_events().decode()
    assert "C" in events and "M" in events
    assert events[0] == "S", events    # and every stream finds it written
    assert events[-1] == "S", events


def test_work_pending_on_the_arena_ends_before_it_is_written(S, lib):
    cfg = S._config([(4, 8), (16, 8)], 2, 2, S.SPECA_BF16, 0, -1, 0.0, None, 0, 0, 0)
    n = ctypes.c_size_t(0)
    assert lib.speca_cache_arena_bytes(ctypes.byref(cfg), ctypes.byref(n)) == S.SPECA_OK
    mem = H.Memory(n.value)
    cfg.arena, cfg.arena_bytes = mem.ptr, n.value
    out = ctypes.c_void_p(None)
    lib.host_events_clear()
    assert lib.speca_cache_create(ctypes.byref(cfg), ctypes.byref(out)) == S.SPECA_OK
    events = lib.host_events().decode()
    assert "C" in events and events[0] == "S" and events[-1] == "S", events
