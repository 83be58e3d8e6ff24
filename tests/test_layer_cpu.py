"""Host-only checks of the verification layer's handle: workspace arithmetic and refusals. No kernel runs."""
import ctypes

import pytest


@pytest.fixture(scope="module")
def S():
    from paper_2509_11628_b200 import build, binding
    build.build()
    binding._lib()
    return binding


HEADS = dict(n_heads=8, n_kv_heads=2, head_dim=64)


def test_workspace_holds_the_work_list(S):
    rows_only = S.speca_layer_workspace_bytes([0, 100], S.SPECA_BF16)
    with_heads = S.speca_layer_workspace_bytes([0, 100], S.SPECA_BF16, **HEADS)
    assert 0 < rows_only < with_heads < 1 << 20
    # nothing to do is fine
    assert S.speca_layer_workspace_bytes([0, 0], S.SPECA_BF16, **HEADS) > 0
    # few rows against many keys: shared out, so partial results need room
    few = S.speca_layer_workspace_bytes([0, 1], S.SPECA_BF16, kv_start=[0, 1 << 20], **HEADS)
    short = S.speca_layer_workspace_bytes([0, 1], S.SPECA_BF16, kv_start=[0, 64], **HEADS)
    assert few > short
    # a full-size video sequence needs no partial results: a work list and the row map
    n = 20926
    assert S.speca_layer_workspace_bytes([0, n], S.SPECA_BF16, n_heads=24, n_kv_heads=24, head_dim=128) < 4 << 20


@pytest.mark.parametrize("bad,status", [
    (dict(q_start=[1, 5]), "SHAPE"), (dict(q_start=[0, 5, 4]), "SHAPE"), (dict(q_start=[0, 1 << 31]), "SHAPE"),
    (dict(q_start=list(range(514))), "SHAPE"), (dict(q_start=[0]), "SHAPE"), (dict(dtype=7), "INVALID_ARG"),
    (dict(n_heads=3), "SHAPE"), (dict(n_kv_heads=0), "SHAPE"), (dict(n_heads=-8), "SHAPE"), (dict(n_heads=258), "SHAPE"),
    (dict(head_dim=129), "SHAPE"), (dict(head_dim=0), "SHAPE"),
    (dict(axis_dims=(32, 34)), "SHAPE"), (dict(axis_dims=(7,)), "SHAPE"), (dict(axis_dims=(0,)), "SHAPE"),
    (dict(axis_dims=(64,), theta=0.0), "INVALID_ARG"), (dict(axis_dims=(64,), theta=float("nan")), "INVALID_ARG"),
    (dict(axis_dims=(64,), pairing=5), "INVALID_ARG"), (dict(scale=float("nan")), "INVALID_ARG"),
    (dict(scale=float("inf")), "INVALID_ARG"), (dict(norm_eps=float("nan")), "INVALID_ARG"),
    (dict(n_heads=0, n_kv_heads=0, head_dim=0, axis_dims=(2,)), "SHAPE"),
    (dict(dtype=0, head_dim=35, axis_dims=(2,)), "SHAPE"),
    (dict(kv_start=[0, -1]), "SHAPE"),
])
def test_refusals(S, bad, status):
    args = dict(q_start=[0, 4], dtype=S.SPECA_BF16, **HEADS)
    args.update(bad)
    with pytest.raises(S.SpecaError) as e:
        S.speca_layer_workspace_bytes(**args)
    assert e.value.status == getattr(S, "SPECA_ERR_" + status)


def test_binding_refuses_what_it_cannot_marshal(S):
    with pytest.raises(ValueError):
        S.speca_layer_workspace_bytes([0, 4, 8], S.SPECA_BF16, kv_start=[0, 4], **HEADS)
    with pytest.raises(ValueError):
        S.speca_layer_workspace_bytes([0, 4], S.SPECA_BF16, axis_dims=(2,) * 5, **HEADS)


def test_null_arguments(S):
    lib = S._lib()
    n = ctypes.c_size_t(0)
    assert lib.speca_layer_workspace_bytes(None, ctypes.byref(n)) == S.SPECA_ERR_INVALID_ARG
    cfg = S._layer_config([0, 4], S.SPECA_BF16, None, 0, 0, 0, False, 0.0, 0.0, (), 1.0, 0)
    assert lib.speca_layer_workspace_bytes(ctypes.byref(cfg), None) == S.SPECA_ERR_INVALID_ARG
    out = ctypes.c_void_p(None)
    assert lib.speca_layer_create(ctypes.byref(cfg), ctypes.byref(out)) == S.SPECA_ERR_INVALID_ARG   # no workspace
    assert lib.speca_layer_create(ctypes.byref(cfg), None) == S.SPECA_ERR_INVALID_ARG
    assert lib.speca_layer_destroy(None) == S.SPECA_OK
    assert lib.speca_layer_check(None, None) == S.SPECA_ERR_INVALID_ARG
    assert lib.speca_layer_last_error(None) == b""
    assert lib.speca_layer_attention(*([None] + [None, 0, 0] * 4 + [None] * 4)) == S.SPECA_ERR_INVALID_ARG
    assert lib.speca_layer_rope(*([None] + [None, 0, 0] * 4 + [None] * 5)) == S.SPECA_ERR_INVALID_ARG


def test_create_fails_loudly_without_a_gpu(S):
    import torch
    if torch.cuda.is_available():
        pytest.skip("a GPU is present")
    with pytest.raises(S.SpecaError) as e:
        S.speca_layer_create([0, 4], S.SPECA_BF16, 256, workspace_bytes=1 << 20, device=0)
    assert e.value.status in (S.SPECA_ERR_CUDA, S.SPECA_ERR_UNSUPPORTED, S.SPECA_ERR_INVALID_ARG)
