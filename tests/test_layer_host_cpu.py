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


# ---- limits: kernels round rows and keys up to their tiles in 32 bits ------------------------------------------------

MOST = (1 << 31) - (1 << 16)


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("causal", [False, True])
def test_key_rows_leave_room_to_round_up(S, lib, dtype, causal):
    kw = dict(causal=causal, n_heads=1, n_kv_heads=1, head_dim=8)
    args = lambda n: S._layer_config([0, 1], dtype, [0, n], scale=0.0, norm_eps=0.0, axis_dims=(), theta=1.0, pairing=0, **kw)
    out = ctypes.c_size_t(0)
    for n, status in ((MOST, S.SPECA_OK), (MOST + 1, S.SPECA_ERR_SHAPE), ((1 << 31) - 1, S.SPECA_ERR_SHAPE)):
        assert lib.speca_layer_workspace_bytes(ctypes.byref(args(n)), ctypes.byref(out)) == status, n


def test_packed_rows_leave_room_to_round_up(S, lib):
    # rows x heads per key head are indexed in 32 bits too: 128 heads over 2^24 rows reach 2^31
    out = ctypes.c_size_t(0)
    for n, status in ((1 << 10, S.SPECA_OK), ((1 << 24) - 511, S.SPECA_ERR_SHAPE), (1 << 24, S.SPECA_ERR_SHAPE)):
        cfg = S._layer_config([0, n], S.SPECA_BF16, [0, 1], 128, 1, 8, False, 0.0, 0.0, (), 1.0, 0)
        assert lib.speca_layer_workspace_bytes(ctypes.byref(cfg), ctypes.byref(out)) == status, n


def test_modulate_dim_leaves_room_to_round_up(S, lib):
    layer, mem = H.layer(S, lib, [0, 1], S.SPECA_F32)
    p, i64 = ctypes.c_void_p(mem.ptr), ctypes.c_int64

    def call(dim):
        return lib.speca_layer_modulate(layer, dim, p, i64(dim), None, i64(0), None, None, None, i64(0), None, None, i64(0), p, i64(dim), None)

    assert call(MOST) == S.SPECA_OK            # counted by the runtime, not run
    assert call(MOST + 1) == S.SPECA_ERR_SHAPE
    assert call((1 << 31) - 1) == S.SPECA_ERR_SHAPE


# ---- outputs that share memory: a race between blocks ---------------------------------------------------------------

A, B, C, D = (1 << 20, 2 << 20, 3 << 20, 4 << 20)   # addresses; nothing is launched, nothing read


def refused(S, lib, status, what):
    lib.host_events_clear()
    assert status() == what
    assert lib.host_events() == (b"" if what != S.SPECA_OK else b"L")


@pytest.mark.parametrize("dtype", [0, 1])
def test_outputs_that_overlap_themselves_are_refused(S, lib, dtype):
    rows, h, hd = 6, 4, 16
    layer, _mem = H.layer(S, lib, [0, rows], dtype, n_heads=h, n_kv_heads=h, head_dim=hd, axis_dims=(hd,))
    dense = (h * hd, hd)

    def attend(rs, hs):
        return lambda: lib.speca_layer_attention(layer, A, *dense, B, *dense, C, *dense, D, rs, hs, None, None, None, None)

    def rope(rs, hs):
        return lambda: lib.speca_layer_rope(layer, A, *dense, B, rs, hs, None, 0, 0, None, 0, 0, C, None, None, None, None)

    def rope_k(rs, hs):
        return lambda: lib.speca_layer_rope(layer, A, *dense, A, *dense, B, *dense, C, rs, hs, D, None, None, None, None)

    fine = [(h * hd, hd), (hd, rows * hd), (h * hd + 8, hd), (3 * hd, 18 * hd), (8 * hd, 2 * hd),
            (16 * 8, 16 * 3),            # heads of different rows in turn, without meeting: 48 h + 128 r
            (16 * 3, 16 * 20)]
    shared = [(hd, hd), (2 * hd, hd), (hd, 2 * hd), (h * hd - 8, hd), (hd, rows * hd - 8), (3 * hd, 2 * hd), (2 * hd, 3 * hd),
              (16 * 4 + 8, 16 * 4), (hd - 8, h * hd), (h * hd, hd - 8)]
    for strides in fine + shared:
        places = sorted(r * strides[0] + j * strides[1] for r in range(rows) for j in range(h))
        meets = any(b - a < hd for a, b in zip(places, places[1:]))
        assert meets == (strides in shared), strides
        for call in (attend, rope, rope_k):
            refused(S, lib, call(*strides), S.SPECA_ERR_SHAPE if meets else S.SPECA_OK)
    # one row, or one head: that stride says nothing
    one, _m = H.layer(S, lib, [0, 1], dtype, n_heads=h, n_kv_heads=h, head_dim=hd, axis_dims=(hd,))
    refused(S, lib, lambda: lib.speca_layer_attention(one, A, 0, hd, B, 0, hd, C, 0, hd, D, 0, hd, None, None, None, None), S.SPECA_OK)
    refused(S, lib, lambda: lib.speca_layer_attention(one, A, 0, hd, B, 0, hd, C, 0, hd, D, hd, hd - 8, None, None, None, None), S.SPECA_ERR_SHAPE)


def test_rope_in_place_needs_the_strides_of_its_input(S, lib):
    rows, h, hd = 6, 4, 16
    layer, _mem = H.layer(S, lib, [0, rows], S.SPECA_F32, n_heads=h, n_kv_heads=h, head_dim=hd, axis_dims=(hd,))
    dense, other = (h * hd, hd), (hd, rows * hd)

    def call(q, qs, qo, qos, k=None, ks=(0, 0), ko=None, kos=(0, 0)):
        return lambda: lib.speca_layer_rope(layer, q, *qs, qo, *qos, k, *ks, ko, *kos, 64, None, None, None, None)

    refused(S, lib, call(A, dense, A, dense), S.SPECA_OK)
    refused(S, lib, call(A, dense, A, other), S.SPECA_ERR_INVALID_ARG)
    refused(S, lib, call(A, (0, hd), A, dense), S.SPECA_ERR_INVALID_ARG)      # broadcast rows
    refused(S, lib, call(A, dense, B, other), S.SPECA_OK)
    refused(S, lib, call(A, dense, A, dense, B, dense, B, dense), S.SPECA_OK)
    refused(S, lib, call(A, dense, A, dense, B, dense, B, other), S.SPECA_ERR_INVALID_ARG)
    refused(S, lib, call(A, dense, C, dense, B, dense, C, dense), S.SPECA_ERR_INVALID_ARG)   # one place for both
    refused(S, lib, call(A, dense, B, dense, B, dense, C, dense), S.SPECA_ERR_INVALID_ARG)   # q over k
    refused(S, lib, call(A, dense, C, dense, B, dense, A, dense), S.SPECA_ERR_INVALID_ARG)   # k over q


def test_attention_does_not_write_over_its_inputs(S, lib):
    layer, _mem = H.layer(S, lib, [0, 6], S.SPECA_BF16, n_heads=4, n_kv_heads=4, head_dim=16)
    dense = (64, 16)
    for o, status in ((A, "INVALID_ARG"), (B, "INVALID_ARG"), (C, "INVALID_ARG"), (D, None)):
        refused(S, lib, lambda: lib.speca_layer_attention(layer, A, *dense, B, *dense, C, *dense, o, *dense, None, None, None, None),
                S.SPECA_OK if status is None else S.SPECA_ERR_INVALID_ARG)


def test_modulate_in_place_needs_the_strides_of_its_input(S, lib):
    layer, _mem = H.layer(S, lib, [0, 6], S.SPECA_F32)

    def call(x, xs, b, bs, xo, xos, y, ys):
        return lambda: lib.speca_layer_modulate(layer, 32, x, xs, b, bs, None, None, None, 0, None, xo, xos, y, ys, None)

    refused(S, lib, call(A, 32, None, 0, None, 0, A, 32), S.SPECA_OK)
    refused(S, lib, call(A, 32, None, 0, None, 0, A, 64), S.SPECA_ERR_INVALID_ARG)
    refused(S, lib, call(A, 0, None, 0, None, 0, A, 32), S.SPECA_ERR_INVALID_ARG)     # one row for all
    refused(S, lib, call(A, 32, B, 32, A, 32, B, 32), S.SPECA_OK)                     # both in place
    refused(S, lib, call(A, 32, B, 40, C, 32, B, 32), S.SPECA_ERR_INVALID_ARG)
    refused(S, lib, call(A, 32, B, 32, A, 40, C, 32), S.SPECA_ERR_INVALID_ARG)
    refused(S, lib, call(A, 32, B, 32, B, 32, C, 32), S.SPECA_OK)
    refused(S, lib, call(A, 32, B, 32, C, 32, C, 32), S.SPECA_ERR_INVALID_ARG)        # one place for both outputs


# ---- the device of a handle ------------------------------------------------------------------------------------------

@pytest.mark.parametrize("asked,current,index", [("cuda", 1, 1), ("cuda", 0, 0), ("cuda:1", 0, 1), ("cuda:0", 1, 0)])
def test_workspace_and_handle_are_on_one_device(S, monkeypatch, asked, current, index):
    import torch
    seen = {}

    def empty(n, dtype, device):
        device = torch.device(device)
        seen["workspace"] = current if device.index is None else device.index
        return object()

    monkeypatch.setattr(torch.cuda, "current_device", lambda: current)
    monkeypatch.setattr(S.torch, "empty", empty)
    monkeypatch.setattr(S, "speca_layer_create", lambda q, dt, ws, device=None, **kw: seen.update(handle=device) or 0)
    layer = S.SpecaLayer([0, 4], S.SPECA_BF16, device=asked, **HEADS)
    assert seen == {"workspace": index, "handle": index}
    assert layer.device == torch.device("cuda", index) and layer.index == index


def test_create_refuses_a_workspace_of_another_device(S):
    import torch

    class There(torch.Tensor):
        """A CPU tensor that says it lives on cuda:1."""
        is_cuda = True
        device = torch.device("cuda", 1)

    ws = torch.empty(1 << 16, dtype=torch.uint8).as_subclass(There)
    with pytest.raises(S.SpecaError, match="cuda:1") as e:
        S.speca_layer_create([0, 4], S.SPECA_BF16, ws, device=0)
    assert e.value.status == S.SPECA_ERR_INVALID_ARG
    with pytest.raises(TypeError):      # host memory
        S.speca_layer_create([0, 4], S.SPECA_BF16, torch.empty(1 << 16, dtype=torch.uint8), device=0)


@pytest.mark.parametrize("asked,current,index", [("cuda", 1, 1), ("cuda:1", 0, 1), ("cuda:0", 1, 0)])
def test_arena_and_cache_are_on_one_device(S, monkeypatch, asked, current, index):
    import torch
    seen = {}

    class Arena:
        def data_ptr(self):
            return 256

    def empty(n, dtype, device):
        device = torch.device(device)
        seen["arena"] = current if device.index is None else device.index
        return Arena()

    monkeypatch.setattr(torch.cuda, "current_device", lambda: current)
    monkeypatch.setattr(S.torch, "empty", empty)
    monkeypatch.setattr(S, "speca_cache_create", lambda e, b, m, dt, arena, basis, ve, eps, device, path, **kw: seen.update(handle=device) or 0)
    cache = S.SpecaCache([(4, 8)], 1, 1, S.SPECA_BF16, device=asked)
    assert seen == {"arena": index, "handle": index} and cache.device == torch.device("cuda", index)


# ---- broadcast operands of the bf16 attention ------------------------------------------------------------------------

def test_operands_that_the_copy_engine_cannot_repeat_are_refused(S, lib):
    # a tensor map steps by a multiple of 16 bytes that is not zero; heads that share one key head's memory need no step
    rows, h, hd = 6, 4, 16
    dense, one_row, one_head = (h * hd, hd), (0, hd), (hd, 0)
    for dtype in (S.SPECA_F32, S.SPECA_BF16):
        layer, _mem = H.layer(S, lib, [0, rows], dtype, n_heads=h, n_kv_heads=h, head_dim=hd)
        for q, k, v, fine in ((dense, dense, dense, True), (dense, one_head, dense, True), (dense, dense, one_head, True),
                              (dense, one_row, dense, False), (dense, dense, one_row, False), (one_row, dense, dense, False),
                              (one_head, dense, dense, False), ((0, 0), dense, dense, False), (dense, (0, 0), dense, False)):
            refused(S, lib, lambda: lib.speca_layer_attention(layer, A, *q, B, *k, C, *v, D, *dense, None, None, None, None),
                    S.SPECA_OK if fine or dtype == S.SPECA_F32 else S.SPECA_ERR_UNSUPPORTED)
        one, _m = H.layer(S, lib, [0, 1], dtype, n_heads=1, n_kv_heads=1, head_dim=hd)     # strides that say nothing
        refused(S, lib, lambda: lib.speca_layer_attention(one, A, 0, 0, B, 0, 0, C, 0, 0, D, 0, 0, None, None, None, None), S.SPECA_OK)
