"""Every tensor of an operator's call lies on the call's device; the binding refuses others before their addresses reach a
kernel.  No GPU: tensors that say where they are, and a library that notes what it is called with."""
import pytest
import torch

from paper_1805_08768_amd import binding as sbc


class On:
    """A tensor's outside, on device `index`."""
    is_cuda = True

    def __init__(self, index, *shape, dtype=torch.float32):
        self.index, self.t = index, torch.empty(*shape, dtype=dtype)
        self.device, self.dtype, self.shape = torch.device("cuda", index), dtype, self.t.shape

    def get_device(self):
        return self.index

    def __getattr__(self, name):
        return getattr(self.t, name)


class Library:
    def __init__(self):
        self.called = []

    def __getattr__(self, name):
        if name.endswith(("_bytes", "_workspace")):
            return lambda *a: 4096
        return lambda *a: self.called.append(name) or 0


@pytest.fixture
def library(monkeypatch):
    lib = Library()
    monkeypatch.setattr(sbc, "load", lambda: lib)
    monkeypatch.setattr(sbc, "_raw_stream", lambda index: 0)
    for sizes in (sbc.sbc_mxfp_bytes, sbc.sbc_mxfp_linear_workspace, sbc.sbc_top_logits_workspace, sbc.sbc_distill_workspace):
        sizes.cache_clear()
    yield lib
    for sizes in (sbc.sbc_mxfp_bytes, sbc.sbc_mxfp_linear_workspace, sbc.sbc_top_logits_workspace, sbc.sbc_distill_workspace):
        sizes.cache_clear()


def room(index):
    return On(index, 4096, dtype=torch.uint8)


def held(rows, cols):
    return lambda index: sbc.Mxfp(rows, cols, room(index))


def ints(*shape):
    return lambda index: On(index, *shape, dtype=torch.int32)


def floats(*shape):
    return lambda index: On(index, *shape)


CALLS = {
    "sbc_mxfp_quantize": dict(x=floats(4, 8), by_rows=held(4, 8), by_cols=held(8, 4)),
    "sbc_mxfp_dequantize": dict(q=held(4, 8), out=floats(4, 8)),
    "sbc_mxfp_matmul": dict(a=held(4, 8), b=held(5, 8), out=floats(4, 5)),
    "sbc_mxfp_linear": dict(x=floats(4, 8), w=held(5, 8), out=floats(4, 5), workspace=room),
    "sbc_top_logits": dict(logits=floats(4, 8), index=ints(4, 2), top=floats(4, 2), lse=floats(4), workspace=room),
    "sbc_distill_loss": dict(logits=floats(4, 8), index=ints(4, 2), top=floats(4, 2), loss=floats(4), stats=floats(4, 4), grad=floats(4, 8), teacher_lse=floats(4), weight=floats(4),
                             workspace=room),
    "sbc_distill_grad": dict(logits=floats(4, 8), index=ints(4, 2), top=floats(4, 2), stats=floats(4, 4), dloss=floats(4), grad=floats(4, 8), teacher_lse=floats(4)),
}


@pytest.mark.parametrize("name", CALLS)
def test_tensors_of_another_device(library, name):
    more = {"temperature": 1.0} if "distill" in name else {}
    for device in (0, 1):
        getattr(sbc, name)(**{a: make(device) for a, make in CALLS[name].items()}, **more)
    assert library.called == [name, name]
    for moved in CALLS[name]:
        with pytest.raises(ValueError):
            getattr(sbc, name)(**{a: make(1 if a == moved else 0) for a, make in CALLS[name].items()}, **more)
    assert library.called == [name, name]


def test_a_stream_of_another_device(library):
    class Stream:
        cuda_stream, device = 7, torch.device("cuda", 1)

    args = {a: make(0) for a, make in CALLS["sbc_mxfp_matmul"].items()}
    with pytest.raises(ValueError):
        sbc.sbc_mxfp_matmul(**args, stream=Stream())
    assert library.called == []
