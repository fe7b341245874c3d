"""How precise the dense layer's gradients are: dW has all of dZ in fp32."""
import numpy as np
import pytest

from paper_2405_01067_amd import binding as abt
from plain_layers import act as value_and_slope
from plain_layers import multipliers

pytestmark = pytest.mark.gpu

F32 = 2.0 ** -24
ACT_ERR = 4e-6                                # of a slope, see test_dense_gpu.py
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
