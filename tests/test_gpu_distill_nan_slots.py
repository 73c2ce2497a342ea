"""A slot counts if the teacher's logit is above -inf, so one whose logit is NaN does not: loss and gradient are those of the
other slots, and 0 where there is none."""
import numpy as np
import pytest
import torch

from oracle import operators_oracle as oracle
from paper_1805_08768_amd import binding as sbc

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("rest", [False, True])
@pytest.mark.parametrize("rows,vocab", [(5, 2000), (5, 40001), (5, 100003)])      # in registers, a longer row, in parts
def test_slots_of_nan(rows, vocab, rest):
    """Against the same call with those slots' indexes outside the vocabulary (bit for bit), and that against the oracle;
    the tolerance of a loss is T^2 (2^-22 (L + 8) + 2^-21) with L at most 40, of a gradient T times that of q and p."""
    k, T = 9, 2.0
    g = np.random.default_rng(vocab)
    x = g.standard_normal((rows, vocab)).astype(np.float32) * 2
    index = np.stack([g.permutation(vocab)[:k] for _ in range(rows)]).astype(np.int32)
    top = g.standard_normal((rows, k)).astype(np.float32) + 4
    lse = np.array([oracle._lse(t.astype(np.float64) / T) + 0.5 for t in top], np.float32) if rest else None
    bad = np.zeros((rows, k), bool)
    bad[0, 3], bad[1, [0, 8]], bad[2], bad[4, 1:] = True, True, True, True
    with_nan, without = np.where(bad, np.float32(np.nan), top), np.where(bad, -1, index).astype(np.int32)
    want_loss, want_grad = oracle.distill(x, index, with_nan, T, lse)
    assert np.isfinite(want_loss).all() and want_loss[2] == 0 and (want_loss[[0, 1, 3, 4]] != 0).all()
    t = lambda a: None if a is None else torch.from_numpy(a).to(DEV)  # noqa: E731
    d, ls = t(x), t(lse)
    eps = 2.0 ** -22 * 48 + 2.0 ** -21
    results = []
    for i, tp in ((t(index), t(with_nan)), (t(without), t(top))):
        loss, stats, step, after = torch.empty(rows, device=DEV), torch.empty(rows, 4, device=DEV), torch.empty_like(d), torch.empty_like(d)
        sbc.sbc_distill_loss(d, i, tp, T, loss, stats=stats, grad=step, teacher_lse=ls)
        sbc.sbc_distill_grad(d, i, tp, T, stats, None, after, teacher_lse=ls)
        results.append((loss, stats, step, after))
    assert all(torch.equal(a, b) for a, b in zip(*results))
    loss, _, step, after = results[0]
    assert np.abs(loss.double().cpu().numpy() - want_loss).max() <= T * T * eps
    for grad in (step, after):
        off = np.abs(grad.double().cpu().numpy() - want_grad)
        assert (off <= T * eps * (1e-3 + np.abs(want_grad)) + 2.0 ** -23 * np.abs(want_grad)).all() and not grad[2].any()
