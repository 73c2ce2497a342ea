"""Calls of the operators on another stream than the current one, while work is queued on both: a workspace that the binding
makes shares no memory with what is still under way."""
import pytest
import torch

from paper_1805_08768_amd import binding as sbc

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def normal(*shape, seed=0):
    return torch.empty(*shape, device=DEV).normal_(generator=torch.Generator(device=DEV).manual_seed(seed))


def linear():
    x, w = normal(40, 700), normal(300, 700, seed=1)
    q, y = sbc.Mxfp(300, 700), torch.empty(40, 300, device=DEV)
    sbc.sbc_mxfp_quantize(w, q)
    return sbc.sbc_mxfp_linear_workspace(40, 700), (y,), lambda **kw: sbc.sbc_mxfp_linear(x, q, y, **kw)


def top():
    x = normal(2, 100000)
    out = torch.empty(2, 64, dtype=torch.int32, device=DEV), torch.empty(2, 64, device=DEV), torch.empty(2, device=DEV)
    return sbc.sbc_top_logits_workspace(2, 100000, 64), out, lambda **kw: sbc.sbc_top_logits(x, *out, **kw)


def distill():
    x = normal(3, 100003)
    t, index = torch.topk(x * 0.8, 16, dim=1)
    index = index.int()
    out = torch.empty(3, device=DEV), torch.empty(3, 100003, device=DEV)
    return sbc.sbc_distill_workspace(3, 100003), out, lambda **kw: sbc.sbc_distill_loss(x, index, t, 2.0, out[0], grad=out[1], **kw)


@pytest.mark.parametrize("by_handle", [False, True])
@pytest.mark.parametrize("operator", [linear, top, distill])
def test_work_queued_on_both_streams(operator, by_handle):
    room, out, call = operator()
    assert room > 0
    call()
    want = [t.clone() for t in out]
    side = torch.cuda.Stream()
    stream = side.cuda_stream if by_handle else side
    busy, other = torch.zeros(1 << 28, device=DEV), torch.zeros(1 << 28, device=DEV)
    copy = torch.empty(room, dtype=torch.uint8, device=DEV)
    for _ in range(3):
        # a block of the workspace's size, read by work queued on the current stream and freed before that has run
        block = torch.full((room,), 5, dtype=torch.uint8, device=DEV)
        copy.zero_()
        for t in out:
            t.zero_()
        torch.cuda.synchronize()
        for _ in range(20):
            busy.add_(1.0)
        copy.copy_(block)
        del block
        call(stream=stream)
        side.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want)) and bool((copy == 5).all())
        # the other way round: blocks of that size are taken and written on the current stream while the call waits on its own
        for t in out:
            t.zero_()
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            for _ in range(20):
                other.add_(1.0)
        call(stream=stream)
        blocks = [torch.full((room,), 255, dtype=torch.uint8, device=DEV) for _ in range(4)]
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want)) and all(bool((b == 255).all()) for b in blocks)


@pytest.mark.parametrize("operator", [linear, top, distill])
def test_the_null_stream_by_its_handle(operator):
    _, out, call = operator()
    call()
    want = [t.clone() for t in out]
    for t in out:
        t.zero_()
    call(stream=0)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(out, want))


@pytest.mark.parametrize("operator", [linear, top, distill])
def test_recorded_on_a_stream_with_the_calls_own_workspace(operator):
    """A workspace taken while a graph is recorded is the graph's; replays with eager calls between them."""
    _, out, call = operator()
    call()
    want = [t.clone() for t in out]
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        call(stream=side)
    for _ in range(3):
        for t in out:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want))
        call()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want))
