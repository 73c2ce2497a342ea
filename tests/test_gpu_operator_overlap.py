"""Matrices whose rows lie beside each other in one buffer: what one holds is read or written, what the other holds stays."""
import pytest
import torch

from paper_1805_08768_amd import binding as sbc

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def normal(*shape, seed=0, dtype=torch.float32):
    return torch.empty(*shape, device=DEV).normal_(generator=torch.Generator(device=DEV).manual_seed(seed)).to(dtype)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("m,n,k", [(1, 100, 60), (7, 129, 1500), (65, 300, 257), (700, 1300, 130)])
def test_a_layers_input_and_output(m, n, k, dtype):
    w = sbc.Mxfp(n, k)
    sbc.sbc_mxfp_quantize(normal(n, k, seed=1), w)
    both = torch.full((m, k + n + 3), 7.0, dtype=dtype, device=DEV)
    x, y = both[:, 1:k + 1], both[:, k + 1:k + 1 + n]
    x.copy_(normal(m, k, seed=2))
    want = torch.empty(m, n, dtype=dtype, device=DEV)
    sbc.sbc_mxfp_linear(x.clone(), w, want)
    before = x.clone()
    sbc.sbc_mxfp_linear(x, w, y)
    assert torch.equal(y, want) and torch.equal(x, before) and (both[:, 0] == 7).all() and (both[:, k + 1 + n:] == 7).all()
    if m > 1:
        with pytest.raises(sbc.SbcError):
            sbc.sbc_mxfp_linear(x, w, both[:, k:k + n])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,vocab", [(5, 2001), (3, 40001), (3, 100003)])
def test_logits_and_their_gradient(rows, vocab, dtype):
    both = torch.full((rows, 2 * vocab + 5), 7.0, dtype=dtype, device=DEV)
    x, grad = both[:, :vocab], both[:, vocab + 2:2 * vocab + 2]
    x.copy_(normal(rows, vocab) * 2)
    before = x.clone()
    top, index = torch.topk(x.float() * 0.7, 12, dim=1)
    index = index.int()
    loss, again, stats, want = torch.empty(rows, device=DEV), torch.empty(rows, device=DEV), torch.empty(rows, 4, device=DEV), torch.empty(rows, 2 * vocab + 5, dtype=dtype, device=DEV)[:, :vocab]
    sbc.sbc_distill_loss(x, index, top, 2.0, loss, grad=want)
    sbc.sbc_distill_loss(x, index, top, 2.0, again, stats=stats, grad=grad)
    assert torch.equal(loss, again) and torch.equal(grad, want) and torch.equal(x, before)
    grad.fill_(7.0)
    sbc.sbc_distill_grad(x, index, top, 2.0, stats, None, grad)
    later = torch.empty_like(want)
    sbc.sbc_distill_grad(before, index, top, 2.0, stats, None, later)
    assert torch.equal(grad, later) and torch.equal(x, before) and (both[:, vocab:vocab + 2] == 7).all() and (both[:, 2 * vocab + 2:] == 7).all()
