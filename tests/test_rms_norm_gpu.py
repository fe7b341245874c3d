"""The root-mean-square norm on the GPU against its definition in fp64, element by element.

Bounds, with u = 2^-8 (bf16) or 2^-24 (fp32) for the rounding of a result and e = 2^-24: the mean of n squares in fp32 is off by at most
(n + 2) e of itself, its inverse root by half of that and a few roundings, so Y by (u + (n / 2 + 8) e) |Y|.  With w = dY gain and s the factor,
dX = dH + s (w - H s^2 mean(w H)) is off by u |dX| + (n + 16) e (s |w| + |H| s^3 mean|w H|) + e |dH|; dgain, a sum over M rows, by
(M + n / 2 + 16) e sum |dY H s|."""
import numpy as np
import pytest
import torch

from paper_2405_01067_amd import binding as abt

pytestmark = pytest.mark.gpu

E = 2.0 ** -24
DT = {"bf16": (torch.bfloat16, 2.0 ** -8), "f32": (torch.float32, E)}
SHAPES = [(1, 8), (3, 64), (5, 504), (4, 512), (7, 520), (197, 768), (2, 1032), (1000, 1536), (9, 2048), (3, 2056), (48, 4096), (5, 6152), (2, 8200), (3, 12296), (2, 16384),
          (2100, 72), (513, 2056)]


def make(M, n, dtype, seed):
    g = torch.Generator().manual_seed(seed)
    t = lambda *s: torch.randn(s, generator=g)
    dt = DT[dtype][0]
    return dict(X=(t(M, n) * 2).to(dt), R=t(M, n).to(dt), gain=1 + 0.2 * t(n), dY=t(M, n).to(dt), dH=(t(M, n) * 0.5).to(dt))


def within(got, want, bound, what):
    err = (got.double().cpu() - want).abs()
    over = err - 1.0001 * bound - 1e-38
    assert bool((over <= 0).all()), (what, float(err.max()), float(over.max()))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("M,n", SHAPES)
def test_forward(M, n, dtype):
    c = make(M, n, dtype, M + n)
    u = DT[dtype][1]
    d = {k: v.cuda() for k, v in c.items()}
    for R in (None, c["R"]):
        H = c["X"].double() + (0 if R is None else R.double())
        want = H / torch.sqrt((H * H).mean(1, keepdim=True) + 1e-6) * c["gain"].double()
        Y, Hg, Yq, s = abt.lr_rms_norm_fwd(d["X"], d["gain"], residual=None if R is None else d["R"])
        assert Yq is None and s is None
        # (the sum of X and the residual rounds to fp32 before anything else)
        within(Y, want, (u + (n / 2 + 8) * E) * want.abs() + E * H.abs() / torch.sqrt((H * H).mean(1, keepdim=True) + 1e-6) * c["gain"].double().abs(), "Y")
        if R is None:
            assert Hg is d["X"]
        else:
            within(Hg, H, (u + E) * H.abs(), "H")
        # 8 bits: the scale is the largest value over 448; a value is off by half a step of four significant bits, or of the smallest one
        Y8, _, Yq, s = abt.lr_rms_norm_fwd(d["X"], d["gain"], residual=None if R is None else d["R"], quantize=True)
        assert torch.equal(Y8, Y)
        big = want.abs().amax(1)
        within(s, big / 448, (n / 2 + 16) * E * big / 448, "scale")
        back = Yq.cpu().double() * s.cpu().double()[:, None]
        within(back, want, 2.0 ** -4 * want.abs() * 1.001 + (2.0 ** -10 * 1.001) * (big / 448)[:, None], "Yq")
        none, _, Yq2, s2 = abt.lr_rms_norm_fwd(d["X"], d["gain"], residual=None if R is None else d["R"], quantize=True, need_Y=False)
        assert none is None and torch.equal(Yq2.view(torch.uint8), Yq.view(torch.uint8)) and torch.equal(s2, s)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("M,n", SHAPES)
def test_backward(M, n, dtype):
    c = make(M, n, dtype, 2 * M + n)
    u = DT[dtype][1]
    d = {k: v.cuda() for k, v in c.items()}
    H, dY, gain = c["X"].double(), c["dY"].double(), c["gain"].double()
    s = 1 / torch.sqrt((H * H).mean(1, keepdim=True) + 1e-6)
    w = dY * gain
    for dH in (None, c["dH"]):
        extra = 0 if dH is None else dH.double()
        want = extra + s * (w - H * s * s * (w * H).mean(1, keepdim=True))
        size = s * w.abs() + H.abs() * s ** 3 * (w * H).abs().mean(1, keepdim=True)
        dX, dg = abt.lr_rms_norm_bwd(d["dY"], d["X"], d["gain"], dH=None if dH is None else d["dH"])
        within(dX, want, u * want.abs() + (n + 16) * E * size + (0 if dH is None else E * extra.abs()), "dX")
        within(dg, (dY * H * s).sum(0), (M + n / 2 + 16) * E * (dY * H * s).abs().sum(0), "dgain")
        again = abt.lr_rms_norm_bwd(d["dY"], d["X"], d["gain"], dH=None if dH is None else d["dH"])
        assert torch.equal(dX, again[0]) and torch.equal(dg, again[1])
        only, none = abt.lr_rms_norm_bwd(d["dY"], d["X"], d["gain"], dH=None if dH is None else d["dH"], need_dgain=False)
        assert none is None and torch.equal(only, dX)
        none, only = abt.lr_rms_norm_bwd(d["dY"], d["X"], d["gain"], dH=None if dH is None else d["dH"], need_dX=False)
        assert none is None and torch.equal(only, dg)
        sum_ = torch.ones_like(dg)
        abt.lr_rms_norm_bwd(d["dY"], d["X"], d["gain"], dgain=sum_, need_dX=False, accumulate=True)
        assert torch.equal(sum_, dg + 1)


def test_gradients_against_differences():
    g = torch.Generator().manual_seed(3)
    H, gain, dY = torch.randn((6, 72), generator=g), 1 + 0.1 * torch.randn(72, generator=g), torch.randn((6, 72), generator=g)
    dX, dg = abt.lr_rms_norm_bwd(dY.cuda(), H.cuda(), gain.cuda(), eps=1e-3)
    loss = lambda h, k: float((dY.double() * h / torch.sqrt((h * h).mean(1, keepdim=True) + 1e-3) * k).sum())
    for got, base, at in ((dX, H, 0), (dg, gain, 1)):
        D = torch.randn(base.shape, generator=g).double()
        t = 1e-4
        args = lambda z: (H.double() + z * D, gain.double()) if at == 0 else (H.double(), gain.double() + z * D)
        # central difference of fourth order: off by t^4 of the fifth derivative
        want = (8 * (loss(*args(t)) - loss(*args(-t))) - (loss(*args(2 * t)) - loss(*args(-2 * t)))) / (12 * t)
        assert abs(float((got.double().cpu() * D).sum()) - want) <= 2e-5 * float((got.double().cpu() * D).abs().sum())


def test_rows_of_zeros_and_of_what_is_not_finite():
    X = torch.randn((6, 768), generator=torch.Generator().manual_seed(1))
    X[1] = 0
    X[3, 5] = float("inf")
    X[4, 700] = float("nan")
    X[5] *= 1e-36
    gain = torch.ones(768)
    Y, _, Yq, s = abt.lr_rms_norm_fwd(X.cuda(), gain.cuda(), quantize=True)
    clean = abt.lr_rms_norm_fwd(X[:1].cuda(), gain.cuda(), quantize=True)
    assert torch.equal(Y[0], clean[0][0]) and torch.equal(Yq[0].view(torch.uint8), clean[2][0].view(torch.uint8))
    assert not bool(Y[1].any()) and not bool(Yq[1].float().any()) and float(s[1]) == 0
    # infinity: the factor is 0, so 0 inf = NaN there and zeros elsewhere; NaN fills its row
    assert bool(torch.isnan(Y[3, 5])) and bool(torch.isnan(Yq[3, 5].float())) and bool(torch.isnan(Y[4]).all()) and bool(torch.isnan(Yq[4].float()).all())
    assert not bool(Yq[5].float().any()) and float(s[5]) == 0            # below what a scale can stand for
    dX, dg = abt.lr_rms_norm_bwd(torch.ones_like(Y), X.cuda(), gain.cuda())
    assert bool(torch.isfinite(dX[[0, 1, 2, 5]]).all()) and bool(torch.isnan(dg).all())


def test_in_place_and_captured():
    c = {k: v.cuda() for k, v in make(197, 768, "bf16", 4).items()}
    Y, H, _, _ = abt.lr_rms_norm_fwd(c["X"], c["gain"], residual=c["R"])
    R = c["R"].clone()
    Y1, H1, _, _ = abt.lr_rms_norm_fwd(c["X"], c["gain"], residual=R, H=R)
    assert H1 is R and torch.equal(H, R) and torch.equal(Y, Y1)
    dX, dg = abt.lr_rms_norm_bwd(c["dY"], H, c["gain"], dH=c["dH"])
    dH = c["dH"].clone()
    dX1, dg1 = abt.lr_rms_norm_bwd(c["dY"], H, c["gain"], dH=dH, dX=dH)
    assert torch.equal(dX, dH) and torch.equal(dg, dg1)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y, h, q, s = abt.lr_rms_norm_fwd(c["X"], c["gain"], residual=c["R"], quantize=True)
        got = abt.lr_rms_norm_bwd(c["dY"], h, c["gain"], dH=c["dH"])
    for k in range(3):
        c["X"].mul_(1.5)
        graph.replay()
        torch.cuda.synchronize()
        Y, H, Q, S = abt.lr_rms_norm_fwd(c["X"], c["gain"], residual=c["R"], quantize=True)
        want = abt.lr_rms_norm_bwd(c["dY"], H, c["gain"], dH=c["dH"])
        assert torch.equal(Y, y) and torch.equal(H, h) and torch.equal(S, s) and torch.equal(Q.view(torch.uint8), q.view(torch.uint8))
        assert torch.equal(want[0], got[0]) and torch.equal(want[1], got[1])


def test_refusals():
    X, gain = torch.zeros((4, 64), device="cuda"), torch.ones(64, device="cuda")
    for x, g, kw in ((X.half(), gain, {}), (X[:, :60].contiguous(), gain[:60].contiguous(), {}), (X, gain[:32].contiguous(), {}), (X.t(), gain, {}), (X, gain.bfloat16(), {}),
                     (X, gain, dict(residual=X.bfloat16())), (X, gain, dict(eps=-1.0)), (X, gain, dict(eps=float("nan"))), (X, gain, dict(need_Y=False)), (X.cpu(), gain, {})):
        with pytest.raises(abt.AbtError):
            abt.lr_rms_norm_fwd(x, g, **kw)
    wide = torch.zeros((1, 16392), device="cuda")
    with pytest.raises(abt.AbtError):
        abt.lr_rms_norm_fwd(wide, torch.ones(16392, device="cuda"))
    for kw in (dict(dH=X.bfloat16()), dict(accumulate=True), dict(dX=X[:2].contiguous()), dict(workspace=torch.empty(8, dtype=torch.uint8, device="cuda"))):
        with pytest.raises(abt.AbtError):
            abt.lr_rms_norm_bwd(X, X, gain, **kw)
