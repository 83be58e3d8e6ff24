"""The host side of the layer calls without a GPU: what a handle asks of the device, and what the calls refuse."""
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
