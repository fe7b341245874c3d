"""Dropout from a counter-based generator: the mask from the definition, element for element."""
import numpy as np
import pytest

from paper_2405_01067_amd import binding as abt
from plain_layers import mask16, multipliers

pytestmark = pytest.mark.gpu


def state(seed, offset):
    import torch
    wrap = lambda v: v - (1 << 64) if v >= 1 << 63 else v
    return torch.tensor([wrap(seed), wrap(offset)], dtype=torch.int64, device="cuda")


@pytest.mark.parametrize("count", (0, 1, 7, 8, 9, 2047, 2048, 2049, 100003))
@pytest.mark.parametrize("dtype,eps", [("bfloat16", 2.0 ** -8), ("float32", 2.0 ** -24)])
@pytest.mark.parametrize("p", (0.0, 2.0 ** -17, 0.1, 0.9, 1 - 2.0 ** -18, 1.0))
@pytest.mark.parametrize("residual", (False, True))
def test_values(count, dtype, eps, p, residual):
    import torch
    g = torch.Generator().manual_seed(count + 1)
    X = torch.randn(count, generator=g).to(getattr(torch, dtype))
    R = torch.randn(count, generator=g).to(X.dtype) if residual else None
    seed, offset, site = 0xFEDCBA9876543210, (1 << 64) - 2, 5              # the counter wraps
    Y = abt.lr_dropout(X.cuda(), abt.Dropout(p, state(seed, offset), site), residual=R.cuda() if residual else None)
    f = multipliers(p, seed, offset, site, (count,))
    want = X.double().numpy() * f + (R.double().numpy() if residual else 0)
    got = Y.double().cpu().numpy()
    assert Y.dtype == X.dtype and got.shape == want.shape
    # the factor, the product and the sum in fp32, then the result's rounding
    small = 3 * 2.0 ** -24 * (np.abs(X.double().numpy() * f) + np.abs(want))
    assert (np.abs(got - want) <= eps * (np.abs(want) + small) + small).all()
    if not residual:
        assert ((got != 0) == (f * X.double().numpy() != 0)).all()


def test_any_shape_in_place_and_backward():
    import torch
    X = torch.randn((3, 5, 7), device="cuda")
    R = torch.randn((3, 5, 7), device="cuda")
    drop = abt.Dropout(0.25, state(1, 2))
    Y = abt.lr_dropout(X, drop, residual=R)
    a, b = X.clone(), R.clone()
    assert abt.lr_dropout(a, drop, residual=R, Y=a) is a and bool((a == Y).all())
    assert abt.lr_dropout(X, drop, residual=b, Y=b) is b and bool((b == Y).all())
    # the gradient is the same call: what reaches X is what reached Y where it was kept
    dY = torch.ones_like(X)
    assert bool(((abt.lr_dropout(dY, drop) != 0) == (abt.lr_dropout(X, drop) != 0)).all())


def test_what_is_dropped_is_not_looked_at():
    import torch
    X = torch.full((4096,), float("nan"), device="cuda")
    X[::2] = float("inf")
    f = multipliers(0.5, 9, 0, 0, (4096,))
    Y = abt.lr_dropout(X, abt.Dropout(0.5, state(9, 0)), residual=torch.ones_like(X)).cpu().numpy()
    assert (Y[f == 0] == 1).all() and not np.isfinite(Y[f != 0]).any()


def test_frequencies():
    import torch
    n = 1 << 20
    keep = lambda seed, offset, site: (abt.lr_dropout(torch.ones(n, device="cuda"), abt.Dropout(0.25, state(seed, offset), site)) != 0).cpu().numpy()
    a = keep(3, 0, 0)
    others = [keep(4, 0, 0), keep(3, 1, 0), keep(3, 0, 7)]
    assert (keep(3, 0, 1) == others[1]).all()                              # the site is added to the offset
    # n draws of probability q: six standard deviations
    for x, q in [(a, 0.75)] + [(a == o, 0.75 ** 2 + 0.25 ** 2) for o in others] + [(a[1:] == a[:-1], 0.625), (a[8:] == a[:-8], 0.625)]:
        assert abs(x.mean() - q) < 6 * (q * (1 - q) / x.size) ** 0.5
    assert (mask16(3, 0, 0, 64).reshape(8, 8).max(1) > 0).all()


def test_captured_with_another_offset():
    import torch
    X, st = torch.randn(5000, device="cuda"), state(11, 0)
    drop, Y = abt.Dropout(0.5, st), torch.empty(5000, device="cuda")
    abt.lr_dropout(X, drop, Y=Y)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        abt.lr_dropout(X, drop, Y=Y)
        st[1:] += 1
    for i in range(4):
        graph.replay()
        torch.cuda.synchronize()
        assert bool((Y == abt.lr_dropout(X, abt.Dropout(0.5, state(11, i)))).all())
