"""Group norm with an activation over channels-last images against its definition in 64 bits."""
import numpy as np
import pytest

from paper_2405_01067_amd import binding as abt
from plain_layers import act as value_and_slope

pytestmark = pytest.mark.gpu

F32 = 2.0 ** -24
ACT_ERR = 4e-6                                # of an activation or its slope, see test_dense_gpu.py
ACTS = ("none", "relu", "gelu", "gelu_tanh", "silu")
# N, pixels, C, groups: everything at once (several numbers of threads and pixels per thread), in pieces; groups of one channel, of all, of 3 and 12; slabs that cut a group
SHAPES = [(1, 1, 8, 1), (1, 1, 8, 8), (2, 49, 64, 32), (3, 196, 256, 32), (2, 7, 96, 32), (5, 50, 24, 2), (1, 784, 128, 32), (2, 300, 1024, 1), (1, 600, 2048, 2), (1, 3136, 64, 32), (1, 5000, 64, 8),
          (2, 1023, 72, 24), (1, 2049, 1160, 5), (3, 33, 8, 4), (1, 9000, 16, 16), (1, 3, 65536, 64), (70, 4, 520, 13), (5000, 2, 16, 2), (40, 3000, 8, 2)]


def make(shape, dtype, seed, offset=1.0):
    import torch
    N, pixels, C, _ = shape
    g = torch.Generator().manual_seed(seed)
    X = torch.randn((N, pixels, C), generator=g) * (0.5 + torch.rand(C, generator=g)) + offset * torch.randn(C, generator=g)
    return dict(X=X.to(dtype), dY=torch.randn((N, pixels, C), generator=g).to(dtype), gain=1 + 0.1 * torch.randn(C, generator=g), shift=0.3 * torch.randn(C, generator=g))


def d(t):
    return t.double().cpu().numpy()


def grouped(a, groups):
    N, pixels, C = a.shape
    return a.reshape(N, pixels, groups, C // groups).transpose(0, 2, 1, 3).reshape(N, groups, -1)


def spread(a, shape):                         # [N, groups] -> [N, 1, C]
    N, _, C, groups = shape
    return np.repeat(a, C // groups, axis=1)[:, None, :]


def within(got, want, bound, what):
    got = d(got)
    assert got.shape == want.shape
    off = np.abs(got - want) / bound
    worst = np.unravel_index(np.argmax(off), off.shape)
    assert off[worst] <= 1.0, f"{what} at {worst}: {got[worst]} for {want[worst]}, {off[worst]:.3g} times the bound"


def check(shape, dtype, act, eps=1e-5, offset=1.0):
    import torch
    N, pixels, C, groups = shape
    dtype = getattr(torch, dtype)
    rounding = 2.0 ** -8 if dtype == torch.bfloat16 else F32
    t = make(shape, dtype, sum(shape), offset)
    c = {k: v.cuda() for k, v in t.items()}
    Y, mean, rstd = abt.lr_group_norm_fwd(c["X"], c["gain"], c["shift"], groups, eps, act)
    x, gain, shift = d(t["X"]), d(t["gain"]), d(t["shift"])
    xg = grouped(x, groups)
    n = xg.shape[2]
    # A sum of n values in fp32, over threads, lanes, waves and channels one after the other: fewer than 60 roundings deep, or 4 per pixel of a thread (at most 40 of them) with
    # running means; 200 of the mean size cover it.
    depth = 200 * F32
    m, v = xg.mean(2), xg.var(2)
    size = np.abs(xg).mean(2)
    merr = depth * size
    within(mean, m, merr + 1e-30, "mean")
    # the squares around a mean that is off by merr: merr^2 more; the differences are rounded relative to the size of x
    verr = depth * (v + np.abs(xg).max(2) * F32 * np.sqrt(v)) + merr ** 2 + 2 * F32 * np.abs(xg).max(2) * np.sqrt(v)
    r = 1 / np.sqrt(v + eps)
    rerr = r * (0.5 * verr / (v + eps) * 1.1 + 8 * F32)
    within(rstd, r, rerr, "rstd")
    unit = (x - spread(m, shape)) * spread(r, shape)
    uerr = spread(merr * r, shape) + np.abs(unit) * spread(rerr / r, shape) + 4 * F32 * (np.abs(unit) + np.abs(x) * spread(r, shape))
    pre = unit * gain + shift
    perr = np.abs(gain) * uerr + 4 * F32 * (np.abs(pre) + np.abs(unit * gain))
    smooth = ACT_ERR if act not in ("none", "relu") else 0.0
    want, slope = value_and_slope(pre, act)
    err = 1.13 * perr + smooth
    within(Y, want, rounding * (np.abs(want) + err) + err + 1e-30, "Y")

    # backward, from the statistics of the forward as they are
    out = abt.lr_group_norm_bwd(c["dY"], c["X"], c["gain"], c["shift"], mean, rstd, act)
    again = abt.lr_group_norm_bwd(c["dY"], c["X"], c["gain"], c["shift"], mean, rstd, act)
    assert all(bool((a.view(torch.uint8) == b.view(torch.uint8)).all()) for a, b in zip(out, again))
    m, r = d(mean), d(rstd)
    unit = (x - spread(m, shape)) * spread(r, shape)
    uerr = 3 * F32 * (np.abs(unit) + np.abs(x) * spread(r, shape))
    pre = unit * gain + shift
    perr = np.abs(gain) * uerr + 4 * F32 * (np.abs(pre) + np.abs(unit * gain))
    dy = d(t["dY"])
    _, slope = value_and_slope(pre, act)
    serr = smooth + 0.81 * perr if smooth else (np.abs(pre) <= perr) * (1.0 if act == "relu" else 0.0)       # at relu's corner either side is right
    dpre = dy * slope
    derr = np.abs(dy) * serr + 2 * F32 * np.abs(dpre)
    du = dpre * unit
    duerr = derr * np.abs(unit) + (np.abs(dpre) + derr) * uerr + 2 * F32 * np.abs(du)
    within(out[1], du.sum((0, 1)), duerr.sum((0, 1)) + depth * np.abs(du).sum((0, 1)) + 1e-30, "dgain")
    within(out[2], dpre.sum((0, 1)), derr.sum((0, 1)) + depth * np.abs(dpre).sum((0, 1)) + 1e-30, "dshift")
    total = lambda a: spread(grouped(a * np.abs(gain), groups).sum(2) / n, shape)
    one, two = (spread(grouped(a * gain, groups).mean(2), shape) for a in (dpre, du))
    onee, twoe = total(derr + depth * np.abs(dpre)), total(duerr + depth * np.abs(du))
    want = spread(r, shape) * (dpre * gain - one - unit * two)
    err = spread(r, shape) * (np.abs(gain) * derr + onee + np.abs(unit) * twoe + uerr * (np.abs(two) + twoe)
                              + 6 * F32 * (np.abs(dpre * gain) + np.abs(one) + np.abs(unit * two)))
    within(out[0], want, rounding * (np.abs(want) + err) + err + 1e-30, "dX")
    return t, c, out, (Y, mean, rstd)


@pytest.mark.parametrize("shape", SHAPES, ids=str)
@pytest.mark.parametrize("dtype", ("bfloat16", "float32"))
@pytest.mark.parametrize("act", ("none", "silu"))
def test_shapes(shape, dtype, act):
    check(shape, dtype, act)


@pytest.mark.parametrize("dtype", ("bfloat16", "float32"))
@pytest.mark.parametrize("shape", [(70, 1000, 64, 16), (520, 49, 256, 8), (130, 400, 96, 8), (64, 300, 264, 3), (300, 1, 16384, 64), (33, 777, 200, 25)], ids=str)
def test_more_than_a_few_megabytes(shape, dtype):
    """Where slabs, threads and vectors are chosen otherwise."""
    check(shape, dtype, "silu")


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("shape", [(2, 49, 64, 32), (1, 9000, 48, 4)], ids=str)
def test_activations(shape, act):
    check(shape, "float32", act)


@pytest.mark.parametrize("shape", [(2, 49, 64, 32), (1, 9000, 48, 4)], ids=str)
def test_means_far_from_zero(shape):
    check(shape, "float32", "none", offset=1000.0)


@pytest.mark.parametrize("shape", [(2, 49, 64, 32), (2, 5000, 24, 3)], ids=str)
def test_parts_and_places(shape):
    """Some of the gradients, on top of others, and outputs in the place of inputs."""
    import torch
    t, c, (dX, dgain, dshift), (Y, mean, rstd) = check(shape, "bfloat16", "gelu")
    args = (c["X"], c["gain"], c["shift"], mean, rstd, "gelu")
    for need in ((True, False, False), (False, True, False), (False, False, True), (True, False, True)):
        part = abt.lr_group_norm_bwd(c["dY"], *args, need_dX=need[0], need_dgain=need[1], need_dshift=need[2])
        for got, whole, wanted in zip(part, (dX, dgain, dshift), need):
            assert (got is None) != wanted and (got is None or bool((got == whole).all()))
    a, b = torch.full_like(dgain, 2.0), torch.full_like(dshift, -1.0)
    abt.lr_group_norm_bwd(c["dY"], *args, need_dX=False, dgain=a, dshift=b, accumulate=True)
    assert bool((a == dgain + 2.0).all()) and bool((b == dshift - 1.0).all())
    over = c["dY"].clone()
    assert bool((abt.lr_group_norm_bwd(over, *args, dX=over)[0] == dX).all())
    x = c["X"].clone()
    abt.lr_group_norm_bwd(c["dY"], x, *args[1:], dX=x)
    assert bool((x == dX).all())
    x = c["X"].clone()
    abt.lr_group_norm_fwd(x, c["gain"], c["shift"], shape[3], 1e-5, "gelu", Y=x)
    assert bool((x == Y).all())


@pytest.mark.parametrize("shape", [(3, 49, 64, 8), (3, 6000, 16, 2)], ids=str)
def test_not_finite_stays_in_its_group(shape):
    import torch
    N, pixels, C, groups = shape
    t = make(shape, torch.float32, 5)
    ref = abt.lr_group_norm_fwd(t["X"].cuda(), t["gain"].cuda(), t["shift"].cuda(), groups)[0]
    bad = t["X"].clone()
    bad[1, pixels // 2, C - 1] = float("nan")
    Y = abt.lr_group_norm_fwd(bad.cuda(), t["gain"].cuda(), t["shift"].cuda(), groups)[0]
    hit = torch.zeros((N, pixels, C), dtype=torch.bool, device="cuda")
    hit[1, :, C - C // groups:] = True
    assert bool(Y[hit].isnan().all()) and bool((Y[~hit] == ref[~hit]).all())


def test_channels_last_image():
    import torch
    X = torch.randn((2, 5, 6, 16), device="cuda")
    g, s = torch.ones(16, device="cuda"), torch.zeros(16, device="cuda")
    Y, mean, rstd = abt.lr_group_norm_fwd(X, g, s, 4)
    flat = abt.lr_group_norm_fwd(X.reshape(2, 30, 16), g, s, 4)[0]
    assert Y.shape == X.shape and bool((Y.reshape(2, 30, 16) == flat).all()) and mean.shape == (2, 4)
    assert abt.lr_group_norm_bwd(X, X, g, s, mean, rstd)[0].shape == X.shape


def test_more_images_than_a_launch_takes():
    """Launches of fewer than 2^32 threads: 2^21 work-groups."""
    import torch
    N, C = (1 << 21) + 777, 8
    X = torch.randn((N, 1, C), device="cuda")
    g, s = torch.full((C,), 2.0, device="cuda"), torch.full((C,), 0.5, device="cuda")
    Y, mean, rstd = abt.lr_group_norm_fwd(X, g, s, 2)
    dX, dgain, dshift = abt.lr_group_norm_bwd(X, X, g, s, mean, rstd)
    x = X.double().reshape(N, 2, 4)
    m, v = x.mean(2, keepdim=True), x.var(2, correction=0, keepdim=True)
    unit = (x - m) / (v + 1e-5).sqrt()
    assert bool(((Y.double().reshape(N, 2, 4) - (unit * 2 + 0.5)).abs() <= 1e-3 * (1 + unit.abs())).all())        # (var of four values may be next to nothing)
    assert float((mean.double() - m[:, :, 0]).abs().max()) < 1e-6
    u = x * 2
    want = (u - u.mean(2, keepdim=True) - unit * (u * unit).mean(2, keepdim=True)) / (v + 1e-5).sqrt()
    # X lies in the span of 1 and x^, so dX is what eps leaves of terms some 1e4 times its size: fp32 errors of the terms count, not dX's own.  x^ is off by the roundings of
    # mean, rstd and their product, x (P) and Q by those of their sum, eight at most of the size (|x| + |m|) rstd; u, its mean and the products by eight of their own.
    r, mean_of = 1 / (v + 1e-5).sqrt(), lambda a: a.abs().mean(2, keepdim=True)
    off = 8 * F32 * ((x.abs() + m.abs()) * r + unit.abs())
    err = r * (8 * F32 * (u.abs() + mean_of(u) + unit.abs() * mean_of(u * unit)) + off * mean_of(u * unit) + unit.abs() * mean_of(u * off) + off.amax(2, keepdim=True) * u.abs())
    assert bool(((dX.double().reshape(N, 2, 4) - want).abs() <= err + 1e-30).all())
    for got, ref in ((dgain, (x * unit).sum(0).reshape(-1)), (dshift, x.sum(0).reshape(-1))):
        assert bool(((got.double() - ref).abs() <= 1e-6 * x.abs().sum() / C + 1e-5 * ref.abs()).all())
