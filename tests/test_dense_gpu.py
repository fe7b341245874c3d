"""The dense layer with bias, activation, dropout and residual against its definition in 64 bits."""
import numpy as np
import pytest

from paper_2405_01067_amd import binding as abt
from plain_layers import act as value_and_slope
from plain_layers import multipliers

pytestmark = pytest.mark.gpu

BF, F32 = 2.0 ** -8, 2.0 ** -24               # a rounding's largest relative error
ACTS = ("none", "relu", "gelu", "gelu_tanh", "silu")
# The largest |act'| is 1.13 (of gelu; silu 1.10), of |act''| 0.8 (gelu, at 0: 2 / sqrt(2 pi)); the evaluation of the activation or of its slope is off by fewer than
# 4e-6: the published formula's 1.5e-7, a few roundings of numbers up to 2 and two of the transcendental unit, times |z| <= 6 where it matters.
ACT_ERR = 4e-6


def make(M, m, n, seed, residual=True, bias=True, dtype=None):
    import torch
    g = torch.Generator().manual_seed(seed)
    t = {"X": torch.randn((M, n), generator=g), "W": torch.randn((m, n), generator=g) / n ** 0.5, "dY": torch.randn((M, m), generator=g)}
    t["residual"] = torch.randn((M, m), generator=g) if residual else None
    t = {k: v.bfloat16() if v is not None else None for k, v in t.items()}
    t["bias"] = torch.randn((m,), generator=g) if bias else None
    return t


def d(t):
    return t.double().cpu().numpy()


def gpu(t):
    return {k: v.cuda() if v is not None else None for k, v in t.items()}


def rng(seed=77, offset=5):
    import torch
    return torch.tensor([seed, offset], dtype=torch.int64, device="cuda")


def within(got, want, bound, what):
    got = d(got)
    assert got.shape == want.shape
    off = np.abs(got - want) / bound
    worst = np.unravel_index(np.argmax(off), off.shape)
    assert off[worst] <= 1.0, f"{what} at {worst}: {got[worst]} for {want[worst]}, {off[worst]:.3g} times the bound"


def check_forward(t, act, p, site=3, seed=77, offset=5):
    c = gpu(t)
    drop = abt.Dropout(p, rng(seed, offset), site) if p is not None else None
    Y, Z = abt.lr_dense_fwd(c["X"], c["W"], c["bias"], act=act, dropout=drop, residual=c["residual"], save_Z=True)
    Y2, none = abt.lr_dense_fwd(c["X"], c["W"], c["bias"], act=act, dropout=drop, residual=c["residual"])
    assert none is None and bool((Y2 == Y).all())
    X, W = d(t["X"]), d(t["W"])
    K = X.shape[1]
    z = X @ W.T + (d(t["bias"]) if t["bias"] is not None else 0)
    # products of bf16 are exact in fp32; a sum of K + 1 of them is off by at most K + 1 roundings of the sum of the sizes
    zerr = (K + 1) * F32 * (np.abs(X) @ np.abs(W).T + (np.abs(d(t["bias"])) if t["bias"] is not None else 0))
    within(Z, z, BF * np.abs(z) + 1.01 * zerr + 1e-30, "Z")
    a, _ = value_and_slope(z, act)
    f = multipliers(p, seed, offset, site, z.shape) if p is not None else 1.0
    y = a * f + (d(t["residual"]) if t["residual"] is not None else 0)
    yerr = (1.13 * zerr + (ACT_ERR if act not in ("none", "relu") else 0)) * f * (1 + 4 * F32) + 4 * F32 * (np.abs(a * f) + np.abs(y))
    within(Y, y, BF * (np.abs(y) + yerr) + yerr + 1e-30, "Y")


SIZES = [(1, 8, 8), (1, 768, 768), (2, 24, 40), (16, 64, 64), (17, 136, 72), (33, 16, 520), (48, 256, 1024), (64, 72, 64), (65, 128, 64), (100, 200, 136), (129, 136, 264),
         (257, 384, 200), (300, 264, 768), (513, 520, 328), (1000, 72, 96), (48, 520, 2304), (300, 264, 1600), (2000, 520, 264)]


@pytest.mark.parametrize("M,m,n", SIZES)
@pytest.mark.parametrize("act,p", [("none", None), ("gelu", 0.1)])
def test_forward(M, m, n, act, p):
    check_forward(make(M, m, n, M + m + n), act, p)


@pytest.mark.parametrize("M", (5, 50, 200))
@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("p", (None, 0.3))
@pytest.mark.parametrize("residual,bias", [(False, False), (True, False), (False, True)])
def test_epilogues(M, act, p, residual, bias):
    check_forward(make(M, 104, 80, 3, residual, bias), act, p)


def check_backward(t, act, p, site=3, seed=77, offset=5):
    import torch
    c = gpu(t)
    Z = (t["residual"].float() * 1.5).bfloat16() if act != "none" else None        # any Z will do
    drop = abt.Dropout(p, rng(seed, offset), site) if p is not None else None
    args = (c["dY"], c["X"], c["W"], Z.cuda() if Z is not None else None)
    dX, dW, db = abt.lr_dense_bwd(*args, act=act, dropout=drop)
    again = abt.lr_dense_bwd(*args, act=act, dropout=drop)
    assert all(bool((a.view(torch.uint8) == b.view(torch.uint8)).all()) for a, b in zip((dX, dW, db), again))
    X, W, dY = d(t["X"]), d(t["W"]), d(t["dY"])
    M, m = dY.shape
    f = multipliers(p, seed, offset, site, dY.shape) if p is not None else 1.0
    s = value_and_slope(d(Z), act)[1] if Z is not None else 1.0
    dZ = dY * f * s
    smooth = act not in ("none", "relu")
    # dZ in fp32: the slope's error, and the roundings of three products
    zerr = np.abs(dY) * f * (ACT_ERR if smooth else 0) + 3 * F32 * np.abs(dZ)
    one = zerr + (BF * (1 + 2 ** -7) * np.abs(dZ) if smooth else 0)                # rounded to bf16
    two = zerr + (BF * BF * np.abs(dZ) if smooth else 0)                           # what is left of it rounded once more
    sums = lambda a, b: (a.shape[1] + 2) * F32 * (np.abs(a) @ np.abs(b))
    want = dZ @ W
    err = one @ np.abs(W) + 1.02 * sums(dZ, W)
    within(dX, want, BF * (np.abs(want) + err) + err + 1e-30, "dX")
    want = dZ.T @ X
    within(dW, want, two.T @ np.abs(X) + 1.02 * 2 * sums(dZ.T, X) + 1e-30, "dW")
    within(db, dZ.sum(0), zerr.sum(0) + 1.02 * (M + 2) * F32 * np.abs(dZ).sum(0) + 1e-30, "dbias")
    # parts of it, and on top of what is there
    for need in ((True, False, False), (False, True, False), (False, False, True)):
        part = abt.lr_dense_bwd(*args, act=act, dropout=drop, need_dX=need[0], need_dW=need[1], need_dbias=need[2])
        for got, whole, wanted in zip(part, (dX, dW, db), need):
            assert (got is None) != wanted and (got is None or bool((got == whole).all()))
    dW2, db2 = torch.full_like(dW, 2.0), torch.full_like(db, -3.0)
    abt.lr_dense_bwd(*args, act=act, dropout=drop, dW=dW2, dbias=db2, accumulate=True, need_dX=False)
    # the sum's rounding; dropout's factor may be multiplied and added in one
    assert bool(((dW2 - (dW + 2.0)).abs() <= 2 * F32 * ((dW + 2.0).abs() + dW.abs())).all()) and bool(((db2 - (db - 3.0)).abs() <= 2 * F32 * ((db - 3.0).abs() + db.abs())).all())


@pytest.mark.parametrize("M,m,n", SIZES)
@pytest.mark.parametrize("act,p", [("none", None), ("gelu", 0.1)])
def test_backward(M, m, n, act, p):
    check_backward(make(M, m, n, M + m + n + 1), act, p)


@pytest.mark.parametrize("M", (5, 50, 200))
@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("p", (None, 0.3))
def test_backward_epilogues(M, act, p):
    check_backward(make(M, 104, 80, 4), act, p)


@pytest.mark.parametrize("M", (3, 48, 200))
@pytest.mark.parametrize("act", ACTS)
def test_sums_that_are_not_finite(M, act):
    """Infinity stays infinity, minus infinity is no infinity behind the smooth activations, NaN stays NaN; the largest and smallest finite sums stay what they are, or 0."""
    import torch
    m, n = 40, 1024
    X, W = torch.zeros((M, n)), torch.zeros((m, n))
    X[:, 0] = 1.0
    special = [float("inf"), -float("inf"), float("nan"), 2.0 ** 127, -2.0 ** 127, 2.0 ** 64, -2.0 ** 64, 20.0, -200.0]
    W[:len(special), 0] = torch.tensor(special)
    Y, Z = abt.lr_dense_fwd(X.bfloat16().cuda(), W.bfloat16().cuda(), act=act, save_Z=True)
    Y, Z = Y.float().cpu(), Z.float().cpu()
    assert bool((Y == Y[0]).logical_or(Y.isnan()).all()) and bool((Z[:, 3:len(special)] == torch.tensor(special[3:])).all())
    y = Y[0]
    assert y[0] == float("inf") and bool(y[2].isnan()) and [float(v) for v in y[3:9:2]] == special[3:9:2]
    if act == "none":
        assert [float(v) for v in y[4:9:2]] == special[4:9:2] and y[1] == -float("inf")
    else:
        assert bool((y[4:9:2].abs() < 1e-30).all()) and not bool(y[1].isinf())
        if act in ("relu", "gelu"):
            assert y[1] == 0
    assert bool((y[len(special):] == 0).all())
