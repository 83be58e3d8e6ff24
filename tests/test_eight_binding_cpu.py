"""What the binding hands to the library in the 8-bit calls, without a GPU: a library that writes its arguments down."""
import ctypes

import pytest
import torch


@pytest.fixture(scope="module")
def S():
    from paper_2509_11628_b200 import binding
    return binding


class Library:
    """Every call of it succeeds, and is kept."""

    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        def call(*args):
            self.calls.append((name, args))
            return 0
        return call


class Stream:
    """Stands for torch's class of streams, whose objects need a device."""

    def __init__(self, address):
        self.cuda_stream = address


def layer_of(S, monkeypatch, rows=6):
    """A layer over `rows` rows whose tensors are the host's, with a library that only listens."""
    lib = Library()
    layer = object.__new__(S.SpecaLayer)
    layer.handle, layer.lib, layer.index, layer.device = None, lib, -1, torch.device("cpu")
    layer.n_seqs, layer.rows, layer.torch_dtype = 2, rows, torch.bfloat16
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda index: 77, raising=False)
    return layer, lib


def calls(S, layer, stream):
    x = torch.zeros(6, 256, dtype=torch.bfloat16)
    out = torch.zeros(6, 32, dtype=torch.bfloat16)
    a, w = S.Matrix8.empty(6, 256, "cpu"), S.Matrix8.empty(32, 256, "cpu")
    layer.quantize8(x, a, stream=stream)
    layer.norm8(x, a, stream=stream)
    layer.matmul8(a, w, out, stream=stream)


@pytest.mark.parametrize("make,address", [(lambda: None, 77), (lambda: 4096, 4096), (lambda: Stream(4096), 4096), (lambda: Stream(0), 0)])
def test_streams_reach_the_library_as_addresses(S, monkeypatch, make, address):
    layer, lib = layer_of(S, monkeypatch)
    monkeypatch.setattr(torch.cuda, "Stream", Stream)
    calls(S, layer, make())
    assert [name for name, _ in lib.calls] == ["speca_layer_quantize8", "speca_layer_norm8", "speca_layer_matmul8"]
    for _, args in lib.calls:
        assert args[-1] == address
        ctypes.c_void_p(args[-1])   # what the library's own argument takes


def product(S, monkeypatch, break_it):
    layer, lib = layer_of(S, monkeypatch)
    codes = torch.zeros(6, 256, dtype=torch.uint8).view(torch.float8_e4m3fn)
    scales = torch.zeros(1, 6, 4, dtype=torch.uint8).view(torch.float8_e8m0fnu)
    a, w, out = S.Matrix8(codes, scales), S.Matrix8.empty(32, 256, "cpu"), torch.zeros(6, 32, dtype=torch.bfloat16)
    at = a.desc.codes, a.desc.scales
    break_it(a, codes, scales)
    try:
        layer.matmul8(a, w, out)
    finally:
        assert (a.desc.codes, a.desc.scales) == at
    return lib.calls


def other():
    return torch.zeros(6, 256, dtype=torch.uint8).view(torch.float8_e4m3fn)


def test_a_matrix_keeps_its_tensors(S, monkeypatch):
    m = S.Matrix8.empty(6, 256, "cpu")
    with pytest.raises(AttributeError):
        m.codes = other()
    with pytest.raises(AttributeError):
        m.scales = m.scales.clone()
    # what the caller does to tensors of its own is nothing to the matrix, which keeps the memory
    assert len(product(S, monkeypatch, lambda a, codes, scales: codes.set_(other()))) == 1
    assert len(product(S, monkeypatch, lambda a, codes, scales: scales.transpose_(0, 1))) == 1


@pytest.mark.parametrize("break_it", [lambda a, codes, scales: a.codes.set_(other()),
                                      lambda a, codes, scales: a.scales.set_(a.scales.clone()),
                                      lambda a, codes, scales: a.codes.untyped_storage().resize_(0),
                                      lambda a, codes, scales: scales.untyped_storage().resize_(0)])
def test_a_matrix_whose_memory_has_gone_is_refused(S, monkeypatch, break_it):
    with pytest.raises(ValueError, match="a: the matrix"):
        product(S, monkeypatch, break_it)
