"""What the operators write through pointers counts as written for autograd: a tensor that it has saved and a call has changed
since is refused in the backward pass, not used as it now is.  No GPU: a library that does nothing."""
import pytest
import torch

from paper_1805_08768_amd import binding as sbc


class Here(torch.Tensor):
    """A tensor that says it is on a device."""
    is_cuda = property(lambda self: True)

    def get_device(self):
        return 0

    device = property(lambda self: torch.device("cuda", 0))


class Library:
    def __getattr__(self, name):
        return (lambda *a: 4096) if name.endswith(("_bytes", "_workspace")) else (lambda *a: 0)


@pytest.fixture(autouse=True)
def library(monkeypatch):
    sizes = (sbc.sbc_mxfp_bytes, sbc.sbc_mxfp_linear_workspace, sbc.sbc_top_logits_workspace, sbc.sbc_distill_workspace)
    monkeypatch.setattr(sbc, "load", lambda: Library())
    monkeypatch.setattr(sbc, "_raw_stream", lambda index: 0)
    for s in sizes:
        s.cache_clear()
    yield
    for s in sizes:
        s.cache_clear()


def made(*shape, dtype=torch.float32):
    return torch.zeros(*shape, dtype=dtype).as_subclass(Here)


def test_every_output_counts_as_written():
    x, out, index, lists = made(4, 8), made(4, 5), made(4, 2, dtype=torch.int32), [made(4, 2), made(4), made(4, 4), made(4, 8), made(4)]
    top, lse, stats, grad, loss = lists
    room = made(4096, dtype=torch.uint8)
    a, b = sbc.Mxfp(4, 8, made(4096, dtype=torch.uint8)), sbc.Mxfp(8, 4, made(4096, dtype=torch.uint8))
    w = sbc.Mxfp(5, 8, made(4096, dtype=torch.uint8))
    for call, written, read in ((lambda: sbc.sbc_mxfp_quantize(x, a, b), (a.tensor, b.tensor), (x,)),
                                (lambda: sbc.sbc_mxfp_dequantize(a, x), (x,), (a.tensor,)),
                                (lambda: sbc.sbc_mxfp_matmul(a, w, out), (out,), (a.tensor, w.tensor)),
                                (lambda: sbc.sbc_mxfp_linear(x, w, out, room), (out,), (x, w.tensor)),
                                (lambda: sbc.sbc_top_logits(x, index, top, lse, 1.0, room), (index, top, lse), (x,)),
                                (lambda: sbc.sbc_top_logits(x, index, top, None, 1.0, room), (index, top), (x, lse)),
                                (lambda: sbc.sbc_distill_loss(x, index, top, 1.0, loss, stats, grad, lse, None, room), (loss, stats, grad), (x, index, top, lse)),
                                (lambda: sbc.sbc_distill_loss(x, index, top, 1.0, loss, None, x, lse, None, room), (loss, x), (index, top, lse)),
                                (lambda: sbc.sbc_distill_grad(x, index, top, 1.0, stats, loss, grad, lse), (grad,), (x, index, top, lse, stats, loss))):
        before = [t._version for t in written], [t._version for t in read]
        call()
        assert all(t._version > v for t, v in zip(written, before[0])) and [t._version for t in read] == before[1]


def test_a_gradient_in_the_place_of_saved_logits():
    """The logits' backward needs the logits: their place is taken, and autograd says so."""
    h = torch.randn(4, 8, requires_grad=True)
    logits = torch.tanh(h)
    place = logits.detach().as_subclass(Here)
    sbc.sbc_distill_loss(place, made(4, 2, dtype=torch.int32), made(4, 2), 1.0, made(4), grad=place, workspace=made(4096, dtype=torch.uint8))
    with pytest.raises(RuntimeError, match="inplace"):
        logits.backward(place.as_subclass(torch.Tensor))


def test_inference_tensors_are_taken():
    with torch.inference_mode():
        out = made(4, 5)
    sbc.sbc_mxfp_linear(made(4, 8), sbc.Mxfp(5, 8, made(4096, dtype=torch.uint8)), out, made(4096, dtype=torch.uint8))
