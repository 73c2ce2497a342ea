"""Students who can say no listed word: all of a row's listed logits are -inf, the others anything down to the type's lowest
value.  The loss is infinite, the gradient what the formula says: with q the softmax of the others, P the listed words'
shares of the teacher (and the rest's share P_rest, whose gradient vanishes as q_rest is 1), T P q_v off the list and -T p_j on it.

Tolerance: an exponent's argument has four roundings, 2^-22 of the range L = (max - min) / T of the unlisted words and
log(vocab); the sum, a tree of at most 300 terms to a lane, 2^-21; and the type's rounding."""
import numpy as np
import pytest
import torch

from oracle import operators_oracle as oracle
from paper_1805_08768_amd import binding as sbc

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
ROUNDING = {torch.float32: 2.0 ** -23, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -10}

# a row in registers, a longer one to a workgroup, a row in parts
ROUTES = [(4, 2000), (4, 40001), (3, 100003)]


@pytest.mark.parametrize("rest", [False, True])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("rows,vocab", ROUTES)
def test_no_listed_word_can_be_said(rows, vocab, dtype, rest):
    k = 7
    g = np.random.default_rng([rows, vocab])
    low = float(torch.finfo(dtype).min)
    for T, others in ((1.0, g.standard_normal((rows, vocab))), (2.0, g.standard_normal((rows, vocab)) - 2000.0), (0.1, g.standard_normal((rows, vocab)) - 90.0),
                      (2.0, g.standard_normal((rows, vocab)) + 2000.0), (1.0, np.full((rows, vocab), low)), (0.25, np.where(g.random((rows, vocab)) < 0.5, low, -800.0))):
        x = torch.from_numpy(others).to(dtype)
        index = np.stack([g.permutation(vocab)[:k] for _ in range(rows)]).astype(np.int32)
        top = g.standard_normal((rows, k)).astype(np.float32)
        x[torch.arange(rows)[:, None], torch.from_numpy(index).long()] = -torch.inf
        lse = np.array([oracle._lse(t.astype(np.float64) / T) + 0.3 for t in top], np.float32) if rest else None
        weight = np.linspace(0.5, 1.5, rows).astype(np.float32)
        want, bound = np.empty((rows, vocab)), np.empty((rows, vocab))
        for r in range(rows):
            z = x[r].double().numpy()
            fine = z > -np.inf
            base = z[fine].max()
            e = np.where(fine, np.exp((z - base) / T), 0.0)
            q = e / e.sum()
            t = top[r].astype(np.float64) / T
            p = np.exp(t - (oracle._lse(t) if lse is None else np.float64(lse[r])))
            want[r] = T * p.sum() * q
            want[r, index[r]] = -T * p
            bound[r] = np.abs(want[r]) * (2.0 ** -22 * (min(40.0, (base - z[fine].min()) / T) + np.log(vocab) + 8) + 2.0 ** -21 + ROUNDING[dtype])
            want[r] *= weight[r]
            bound[r] = bound[r] * weight[r] + (2.0 ** -25 if dtype == torch.float16 else 1e-38)      # (and e^-40 is nothing beside 2^-24)
        t = lambda a: None if a is None else torch.from_numpy(a).to(DEV)  # noqa: E731
        d, i, tp, ls, w = x.to(DEV), t(index), t(top), t(lse), t(weight)
        loss, stats = torch.empty(rows, device=DEV), torch.empty(rows, 4, device=DEV)
        for way in ("loss", "step", "grad", "place"):
            grad = d.clone() if way == "place" else torch.full_like(d, 99.0)
            if way in ("loss", "grad"):
                sbc.sbc_distill_loss(d, i, tp, T, loss, stats=stats, teacher_lse=ls, weight=w)
            else:
                sbc.sbc_distill_loss(grad if way == "place" else d, i, tp, T, loss, grad=grad, teacher_lse=ls, weight=w)
            if way == "grad":
                sbc.sbc_distill_grad(d, i, tp, T, stats, w, grad, teacher_lse=ls)
            assert (loss == torch.inf).all(), (T, others[0, :3], way, loss)
            if way != "loss":
                off = np.abs(grad.double().cpu().numpy() - want)
                assert (off <= bound).all(), (T, others[0, :3], way, np.argwhere(~(off <= bound))[:5])


@pytest.mark.parametrize("rows,vocab", ROUTES)
def test_nan_beside_words_that_cannot_be_said(rows, vocab):
    """A NaN off the list still shows in the loss and in all of its row's gradient."""
    x = torch.zeros(rows, vocab, device=DEV)
    index = torch.arange(5, device=DEV, dtype=torch.int32).repeat(rows, 1)
    x[:, :5], x[0, vocab - 3] = -torch.inf, torch.nan
    loss, stats, grad = torch.empty(rows, device=DEV), torch.empty(rows, 4, device=DEV), torch.empty_like(x)
    for way in ("step", "grad"):
        sbc.sbc_distill_loss(x, index, torch.zeros(rows, 5, device=DEV), 1.0, loss, stats=stats, grad=grad if way == "step" else None)
        if way == "grad":
            sbc.sbc_distill_grad(x, index, torch.zeros(rows, 5, device=DEV), 1.0, stats, None, grad)
        assert loss[0].isnan() and (loss[1:] == torch.inf).all() and grad[0].isnan().all() and grad[1:].isfinite().all()
