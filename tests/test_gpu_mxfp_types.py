"""What the tests of 4-bit matrices leave out: products of tiles with 16-bit outputs, with rows that start anywhere and lie
apart; the extremes of each type in each form of the quantisation."""
import math

import numpy as np
import pytest
import torch

from oracle import operators_oracle as oracle
from paper_1805_08768_amd import binding as sbc

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = [torch.float32, torch.bfloat16, torch.float16]
ROUNDING = {torch.float32: 0.0, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -10}


def normal(*shape, seed=0):
    return torch.empty(*shape, device=DEV).normal_(generator=torch.Generator(device=DEV).manual_seed(seed))


def held(x):
    q, values = sbc.Mxfp(*x.shape), torch.empty(x.shape, device=DEV)
    sbc.sbc_mxfp_quantize(x, q)
    sbc.sbc_mxfp_dequantize(q, values)
    return q, values.double()


def guarded(rows, cols, dtype, ld, lead):
    flat = torch.full((lead + rows * ld + 64,), 7.0, dtype=dtype, device=DEV)
    view = flat[lead:lead + rows * ld].view(rows, ld)[:, :cols]

    def untouched():
        rest = flat.clone()
        rest[lead:lead + rows * ld].view(rows, ld)[:, :cols] = 7.0
        return bool((rest == 7.0).all())
    return view, untouched


# more than 200 panels and up to 256 tiles of 128 x 128 (steps shared by two halves of a workgroup: 1, 4, 8, 64 steps), and more
# tiles (1, 3, 5 steps); ends of rows and columns within a tile, a panel, a vector of outputs
TILES = [(700, 1300, 128), (640, 1280, 385), (897, 1027, 1000), (256, 4000, 8192), (2100, 2200, 100), (2049, 2183, 300), (2177, 2175, 513)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("m,n,k", TILES)
def test_products_of_tiles(m, n, k, dtype):
    """Every term is exact in 32 bits; (steps + 8) additions at 2^-22 of the sum of the terms' magnitudes bound their sum's error,
    and a 16-bit output adds its rounding (2^-24 is half of float16's least value).  The rows of C lie at every offset from 16
    bytes that the type has."""
    x, w = normal(m, k, seed=m).to(dtype), normal(n, k, seed=n + 1) * torch.exp(normal(n, 1, seed=2)) * 2.0 ** -4
    qx, vx = held(x)
    qw, vw = held(w)
    want = torch.matmul(vx, vw.t().contiguous())
    bound = (math.ceil(k / 128) + 8) * 2.0 ** -22 * torch.matmul(vx.abs(), vw.abs().t().contiguous()) + ROUNDING[dtype] * want.abs() + (2.0 ** -24 if dtype == torch.float16 else 0.0)
    assert want.abs().max() < 60000
    for ld, lead in ((n, 0), (n + 5, 1), (n + 3, 3), (n + 64, 8)):
        out, untouched = guarded(m, n, dtype, ld, lead)
        sbc.sbc_mxfp_matmul(qx, qw, out)
        assert ((out.double() - want).abs() <= bound).all() and untouched()
        again, untouched = guarded(m, n, dtype, ld, lead)
        sbc.sbc_mxfp_linear(x, qw, again)
        assert torch.equal(out, again) and untouched()


def test_products_of_tiles_with_bad_blocks():
    for m, n, k in ((700, 1300, 300), (2100, 2200, 300)):
        for dtype in TYPES:
            x, w = normal(m, k, seed=3).to(dtype), normal(n, k, seed=4)
            x[m // 2, 3], w[n // 3, k - 1] = math.inf, math.nan
            out, untouched = guarded(m, n, dtype, n + 7, 5)
            sbc.sbc_mxfp_linear(x, held(w)[0], out)
            bad = torch.zeros(m, n, dtype=torch.bool, device=DEV)
            bad[m // 2], bad[:, n // 3] = True, True
            assert torch.equal(torch.isnan(out), bad) and untouched()


def extremes(dtype):
    """Denormals, the least and the largest normal numbers, infinities and NaN of a type, a block each; every kind beside
    blocks that it must leave alone, and a block that ends the matrix early."""
    info = torch.finfo(dtype)
    least = {torch.float32: 2.0 ** -149, torch.bfloat16: 2.0 ** -133, torch.float16: 2.0 ** -24}[dtype]
    x = np.zeros((7, 100))
    x[0, :32] = least * np.arange(32)
    x[0, 32:64] = info.tiny * np.linspace(-2, 2, 32)
    x[0, 64:96] = -least
    x[1, :32] = info.max * np.linspace(-1, 1, 32)
    x[1, 32:64] = info.tiny
    x[1, 40] = info.max
    x[2] = 1.5
    x[2, 40] = np.inf
    x[3] = -0.75
    x[3, 95] = np.nan
    x[4] = np.linspace(-info.max / 4, info.max / 4, 100)
    x[5, 3] = -np.inf
    x[6, 96:] = [least, 0.0, -0.0, -3 * least]
    return torch.from_numpy(x).to(dtype)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("turned", [False, True])
def test_extremes_of_each_type_in_each_form(dtype, turned):
    x = extremes(dtype)
    if turned:
        x = x.t().contiguous()
    rows, cols = x.shape
    exact = x.double().numpy()
    want = torch.from_numpy(oracle.mxfp_container(exact)), torch.from_numpy(oracle.mxfp_container(exact.T))
    both = sbc.Mxfp(rows, cols), sbc.Mxfp(cols, rows)
    alone = sbc.Mxfp(rows, cols), sbc.Mxfp(cols, rows)
    x = x.to(DEV)
    sbc.sbc_mxfp_quantize(x, *both)
    sbc.sbc_mxfp_quantize(x, alone[0])
    sbc.sbc_mxfp_quantize(x, None, alone[1])
    for q in (both, alone):
        assert torch.equal(q[0].tensor.cpu(), want[0])
        assert torch.equal(q[1].tensor.cpu(), want[1])
    for out_type in TYPES:
        for q, held_as in zip(both, (exact, exact.T)):
            out = torch.empty(held_as.shape, dtype=out_type, device=DEV)
            sbc.sbc_mxfp_dequantize(q, out)
            with np.errstate(over="ignore"):
                values = torch.from_numpy(oracle.mxfp_values(held_as)).to(out_type)
            assert torch.equal(out.cpu().nan_to_num(nan=5.0), values.nan_to_num(nan=5.0)) and torch.equal(out.cpu().isnan(), values.isnan())


@pytest.mark.parametrize("dtype", TYPES)
def test_extremes_in_a_linear_layer_of_few_rows(dtype):
    """The few-row product rounds its rows itself: through a multiple of the identity its outputs are the rounded values, exactly
    (one term each).  2^40 lifts denormals out of what the matrix instruction may flush, 2^-20 keeps the largest in 32
    bits; a bad block spoils its row."""
    x = extremes(dtype)
    for power in ((40, -20) if dtype != torch.float16 else (6, -2)):
        w = torch.eye(100, device=DEV) * 2.0 ** power
        out = torch.empty(7, 100, dtype=dtype, device=DEV)
        sbc.sbc_mxfp_linear(x.to(DEV), held(w)[0], out)
        values = oracle.mxfp_values(x.double().numpy())
        bad = np.isnan(values).any(1)
        assert bad.tolist() == [False, False, True, True, False, True, False]
        want = torch.from_numpy(values * 2.0 ** power)
        got = out.cpu().double()
        assert torch.equal(got.isnan().all(1), torch.from_numpy(bad)) and torch.equal(got.isnan().any(1), torch.from_numpy(bad))
        ok = (want.abs() < torch.finfo(dtype).max) & ((want == 0) | (want.abs() >= max(torch.finfo(dtype).tiny, 2.0 ** -110)))
        ok[torch.from_numpy(bad)] = False
        assert ok[[0, 1, 4, 6]].float().mean() > 0.5
        assert torch.equal(got[ok], want[ok])
