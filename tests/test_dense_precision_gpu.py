"""How precise the dense layer's gradients are: dX has no rounding but its own, dW all of dZ in fp32, and what is infinite stays infinite."""
import numpy as np
import pytest

from paper_2405_01067_amd import binding as abt
from plain_layers import act as value_and_slope
from plain_layers import multipliers

pytestmark = pytest.mark.gpu

BF, F32 = 2.0 ** -8, 2.0 ** -24
ACT_ERR = 4e-6                                # of a slope, see test_dense_gpu.py
SMOOTH = ("gelu", "gelu_tanh", "silu")
# few rows with everything in one launch, and in several; more rows
SIZES = [(1, 8, 8), (9, 768, 768), (48, 1024, 136), (200, 520, 136), (394, 768, 768), (1500, 512, 520), (9216, 72, 136), (9217, 72, 136), (9300, 2056, 136), (12613, 264, 520)]


def d(t):
    return t.double().cpu().numpy()


def make(M, m, n, seed):
    import torch
    g = torch.Generator().manual_seed(seed)
    return [torch.randn(s, generator=g) for s in ((M, m), (M, n), (m, n), (M, m))]


def dropout(p):
    import torch
    return abt.Dropout(p, torch.tensor([77, 5], dtype=torch.int64, device="cuda"), 3) if p else None


@pytest.mark.parametrize("M,m,n", SIZES)
@pytest.mark.parametrize("act,p", [("gelu", 0.0), ("silu", 0.3)])
def test_dX_is_rounded_once(M, m, n, act, p):
    """Rows of dY with up to `terms` values that are not 0, so that the sums' own roundings do not cover those of dZ: dZ comes in two bf16 values, what lies behind the leading
    eight bits and the eight of the rest is cut off, 2^-15 of it at most; a sum of 2 `terms` products that are not 0 is off by as many roundings."""
    import torch
    terms = 12
    dY, X, W, Z = make(M, m, n, M + m)
    keep = torch.rand((M, m), generator=torch.Generator().manual_seed(3)).argsort(1).argsort(1) < terms
    dY, X, W, Z = (dY * keep).bfloat16(), X.bfloat16(), W.bfloat16(), Z.bfloat16()
    dX, _, _ = abt.lr_dense_bwd(dY.cuda(), X.cuda(), W.cuda(), Z.cuda(), act=act, dropout=dropout(p), need_dW=False, need_dbias=False)
    f = multipliers(p, 77, 5, 3, (M, m)) if p else 1.0
    dZ, w = d(dY) * f * value_and_slope(d(Z), act)[1], d(W)
    off = np.abs(d(dY)) * f * ACT_ERR + (3 * F32 + 2.0 ** -15 + (2 * terms + 2) * F32) * np.abs(dZ)
    want, err = dZ @ w, 1.01 * off @ np.abs(w)
    worst = (np.abs(d(dX) - want) / (BF * (np.abs(want) + err) + err + 1e-30)).max()
    assert worst <= 1.0, worst


@pytest.mark.parametrize("M,m,n", SIZES)
@pytest.mark.parametrize("act,p", [("gelu", 0.0), ("gelu_tanh", 0.0), ("silu", 0.3)])
def test_dW_has_all_of_dZ(M, m, n, act, p):
    """One row of dY is not 0, and its row of X are powers of two: every sum has one term, so that dW is dZ times them to the last bit, and so is dbias."""
    import torch
    dY, X, W, Z = make(M, m, n, 2 * M + m)
    for row in {0, M // 2, M - 1}:
        one = torch.zeros_like(dY)
        one[row] = dY[row]
        X[row] = 2.0 ** (torch.arange(n) % 5 - 2) * (1 - 2 * (torch.arange(n) % 2))
        _, dW, db = abt.lr_dense_bwd(one.bfloat16().cuda(), X.bfloat16().cuda(), W.bfloat16().cuda(), Z.bfloat16().cuda(), act=act, dropout=dropout(p), need_dX=False)
        assert bool((dW == db[:, None] * X[row].cuda()).all())
        f = multipliers(p, 77, 5, 3, (M, m))[row] if p else 1.0
        y = d(one.bfloat16())[row]
        want = y * f * value_and_slope(d(Z.bfloat16())[row], act)[1]
        assert (np.abs(d(db) - want) <= np.abs(y) * f * ACT_ERR + 3 * F32 * np.abs(want)).all()


@pytest.mark.parametrize("M,m,n", [(1, 8, 8), (48, 1024, 136), (200, 520, 136), (2000, 264, 520), (9300, 264, 136)])
@pytest.mark.parametrize("act", SMOOTH)
def test_infinities_stay_infinite(M, m, n, act):
    """An infinite value of X or of W, with slopes that are not 0: every sum that it is in has no other infinity, and is infinite with dZ's sign."""
    import torch
    dY, X, W, Z = (t.bfloat16() for t in make(M, m, n, 3 * M + m))
    # numbers of few bits among them, and slopes of 1: the rest behind dZ's leading bits is 0 there
    dY, Z = torch.where(dY.abs() < 0.05, 0.5, dY), torch.where(Z.abs() < 0.2, 100.0, Z).clamp(min=-0.5)
    clean = abt.lr_dense_bwd(*(t.cuda() for t in (dY, X, W, Z)), act=act)
    row, col, out, at = M // 2, n - 1, m // 3, n // 2
    X[row, col], W[out, at] = float("inf"), -float("inf")
    dX, dW, db = abt.lr_dense_bwd(*(t.cuda() for t in (dY, X, W, Z)), act=act)
    dZ = dY.double() * torch.from_numpy(value_and_slope(d(Z), act)[1])
    assert bool((dZ != 0).all())
    assert bool((dW[:, col].cpu() == float("inf") * dZ[row].sign().float()).all())
    assert bool((dX[:, at].float().cpu() == -float("inf") * dZ[:, out].sign().float()).all())
    for got, ref, hit in ((dX, clean[0], at), (dW, clean[1], col)):
        got[:, hit] = ref[:, hit]
        assert bool((got == ref).all())
    assert bool((db == clean[2]).all())
