"""Top logits of rows that hold signalling NaN, the kind that memory never written by arithmetic may hold: not listed, and no
logit beside one is lost.  (The other tests' NaN are quiet.)"""
import numpy as np
import pytest
import torch

from oracle import operators_oracle as oracle
from paper_1805_08768_amd import binding as sbc

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BITS = {torch.float32: (torch.int32, (0x7f800001, 0x7fbfffff, 0xff800001 - (1 << 32), 0xffa00000 - (1 << 32))),
        torch.bfloat16: (torch.int16, (0x7f81, 0x7fbf, 0xff81 - (1 << 16), 0xffa0 - (1 << 16))),
        torch.float16: (torch.int16, (0x7c01, 0x7dff, 0xfc01 - (1 << 16), 0xfd00 - (1 << 16)))}


def spoiled(x, where, dtype):
    """x as the type holds it, with signalling NaN of different bits and signs where `where` says so."""
    ints, patterns = BITS[dtype]
    t = torch.from_numpy(x).to(dtype).to(DEV)
    at = torch.from_numpy(where).to(DEV)
    pattern = torch.tensor(patterns, dtype=ints, device=DEV)[torch.arange(t.numel(), device=DEV).view(t.shape) % 4]
    t.view(ints).copy_(torch.where(at, pattern, t.view(ints)))
    return t


def check(t, k, rows):
    """All rows are the first `rows` again."""
    index, top, lse = torch.empty(t.shape[0], k, dtype=torch.int32, device=DEV), torch.empty(t.shape[0], k, device=DEV), torch.empty(t.shape[0], device=DEV)
    x = t[:rows].cpu().double().numpy()
    want, values, sums = oracle.top_logits(x, k, 1.0)
    for out in (lse, None):
        sbc.sbc_top_logits(t, index, top, out)
        assert np.array_equal(index[:rows].cpu().numpy(), want) and np.array_equal(top[:rows].double().cpu().numpy(), values)
        assert torch.equal(index, index[:rows].repeat(t.shape[0] // rows, 1))
    assert np.array_equal(lse[:rows].isnan().cpu().numpy(), np.isnan(sums))


@pytest.mark.parametrize("dtype", BITS)
def test_beside_the_largest(dtype):
    """Every pair of places in a vector of eight for the largest logit and the NaN, and vectors of NaN but for it."""
    pairs = [(i, j) for i in range(8) for j in range(8) if i != j]
    rows = len(pairs) + 8
    for vocab, copies in ((300, 1), (300, 40), (6000, 1)):
        g = np.random.default_rng(vocab)
        x = np.minimum(g.standard_normal((rows, vocab)), 3.0).astype(np.float32)
        where = np.zeros((rows, vocab), bool)
        for r in range(rows):
            at = 8 * int(g.integers(0, vocab // 8 - 1))
            i, j = pairs[r] if r < len(pairs) else (r - len(pairs), None)
            x[r, at + i] = 50.0
            if j is None:
                where[r, at:at + 8] = True
                where[r, at + i] = False
            else:
                where[r, at + j] = True
        t = spoiled(x, where, dtype)
        for k in (1, 5, 70):
            check(t.repeat(copies, 1), k, rows)


@pytest.mark.parametrize("dtype", BITS)
def test_everywhere(dtype):
    """A tenth and nine tenths of NaN, in rows in any order, rising, with ties by the hundred, of NaN alone; rows that start
    anywhere, in parts, and many."""
    for rows, vocab, copies in ((7, 2025, 1), (7, 2025, 300), (7, 30000, 1), (7, 90001, 1)):
        g = np.random.default_rng(vocab)
        x = g.standard_normal((7, vocab)).astype(np.float32)
        x[1] = np.arange(vocab) % 2000
        x[2] = -(np.arange(vocab) % 2000)
        x[3] = np.round(x[3])
        x[4] = 2.0
        for share in (0.1, 0.9):
            where = g.random((7, vocab)) < share
            where[5] = True
            where[6, vocab // 2:] = True
            flat = torch.zeros(7 * copies, vocab + 5, dtype=dtype, device=DEV)
            t = flat[:, 3:vocab + 3]
            ints = BITS[dtype][0]
            flat.view(ints)[:, 3:vocab + 3] = spoiled(x, where, dtype).view(ints).repeat(copies, 1)
            for k in (1, 64, 256):
                check(t, k, 7)
