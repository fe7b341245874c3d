"""Refusals and workspace queries of the operators around a frozen layer, at the C entries: no GPU is needed, as arguments are looked at
before the device is."""
import ctypes
import os

import pytest

from paper_2405_01067_amd import binding as abt

P, ODD = 0x10000, 0x10008                     # stand for device pointers: aligned to 256, and to 8 only
BIG = 1 << 40                                 # bytes of workspace
OK, EINVAL, EDTYPE, ESHAPE, EALIGN, EWORKSPACE = 0, -1, -5, -2, -3, -4


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(abt._LIB_PATH):
        import __graft_entry__ as ge
        ge.build()
    return abt.load()


def adapters(A=P, B=P, ranks=None, scales=None, count=4, r=16):
    return abt.Adapters(A, B, ranks, scales, count, r)


BAD_STACKS = [(dict(A=None), EINVAL), (dict(B=None), EINVAL), (dict(A=ODD), EALIGN), (dict(B=ODD), EALIGN), (dict(ranks=P + 2), EALIGN), (dict(scales=P + 2), EALIGN),
              (dict(count=0), ESHAPE), (dict(count=-1), ESHAPE), (dict(count=65536), ESHAPE), (dict(r=0), ESHAPE), (dict(r=12), ESHAPE), (dict(r=136), ESHAPE), (dict(r=-8), ESHAPE)]
BAD_SIZES = [(0, 64, 64), (-1, 64, 64), ((1 << 28) + 1, 64, 64), (10, 0, 64), (10, 68, 64), (10, 64, 60), (10, (1 << 20) + 8, 64), (10, 64, (1 << 20) + 16)]


def test_forward(lib):
    def call(X=P, W=P, ad=None, rows=P, Y=P, T=None, M=10, m=64, n=64, dt=abt.ABT_BF16, ws=P, nbytes=BIG, none=False):
        ad = adapters() if ad is None else ad
        return lib.lr_adapters_fwd(X, W, None if none else ctypes.byref(ad), rows, Y, T, M, m, n, dt, ws, nbytes, None)
    assert call(dt=abt.ABT_F32) == EDTYPE and call(dt=7) == EDTYPE
    assert [call(X=None), call(W=None), call(Y=None), call(rows=None), call(none=True)] == [EINVAL] * 5
    for kw, want in BAD_STACKS:
        assert call(ad=adapters(**kw)) == want, kw
    for M, m, n in BAD_SIZES:
        assert call(M=M, m=m, n=n) == ESHAPE, (M, m, n)
    assert [call(X=ODD), call(W=ODD), call(Y=ODD), call(T=ODD), call(rows=P + 2), call(ws=P + 16)] == [EALIGN] * 6
    need = lib.lr_adapters_fwd_workspace_bytes(10, 64, 64, 16, 4)
    assert [call(ws=None), call(nbytes=need - 1), call(nbytes=0)] == [EWORKSPACE] * 3


def test_forward_from_8_bits(lib):
    def call(X=P, Xq=P, xs=P, Wq=P, ws_=P, ad=None, rows=P, Y=P, M=10, m=64, n=64, ws=P, nbytes=BIG):
        ad = adapters() if ad is None else ad
        return lib.lr_adapters_fwd_q8(X, Xq, xs, Wq, ws_, ctypes.byref(ad), rows, Y, M, m, n, ws, nbytes, None)
    assert [call(**{k: None}) for k in ("X", "Xq", "xs", "Wq", "ws_", "rows", "Y")] == [EINVAL] * 7
    for kw, want in BAD_STACKS:
        assert call(ad=adapters(**kw)) == want, kw
    for M, m, n in BAD_SIZES + [(10, 64, 72)]:
        assert call(M=M, m=m, n=n) == ESHAPE, (M, m, n)
    assert [call(**{k: ODD}) for k in ("X", "Xq", "Wq", "Y")] == [EALIGN] * 4
    assert [call(xs=P + 2), call(ws_=P + 2), call(rows=P + 1), call(ws=P + 16)] == [EALIGN] * 4
    assert [call(ws=None), call(nbytes=1)] == [EWORKSPACE] * 2


def test_backward(lib):
    def call(dY=P, X=P, T=P, W=P, ad=None, rows=P, dX=P, dA=P, dB=P, M=10, m=64, n=64, dt=abt.ABT_BF16, ws=P, nbytes=BIG):
        ad = adapters() if ad is None else ad
        return lib.lr_adapters_bwd(dY, X, T, W, ctypes.byref(ad), rows, dX, dA, dB, M, m, n, dt, 0, ws, nbytes, None)
    assert call(dt=abt.ABT_F32) == EDTYPE
    # W for dX, X for dB, X or T for dA
    assert [call(dY=None), call(W=None), call(X=None), call(X=None, T=None, dB=None), call(rows=None)] == [EINVAL] * 5
    for kw, want in BAD_STACKS:
        assert call(ad=adapters(**kw)) == want, kw
    for M, m, n in BAD_SIZES:
        assert call(M=M, m=m, n=n) == ESHAPE, (M, m, n)
    assert [call(**{k: ODD}) for k in ("dY", "X", "T", "W", "dX", "dA", "dB")] == [EALIGN] * 7
    assert call(ws=P + 16) == EALIGN and call(ws=None) == EWORKSPACE
    assert call(nbytes=lib.lr_adapters_bwd_workspace_bytes(10, 64, 64, 16, 4) - 1) == EWORKSPACE
    assert call(dX=None, dA=None, dB=None) == OK                         # nothing to do


def test_workspaces(lib):
    fwd, bwd = lib.lr_adapters_fwd_workspace_bytes, lib.lr_adapters_bwd_workspace_bytes
    for M, m, n, r, count in ((1, 8, 8, 8, 1), (128, 768, 768, 16, 4), (129, 768, 768, 16, 4), (12608, 2304, 768, 16, 7), (65536, 4096, 4096, 128, 1000)):
        f, b = fwd(M, m, n, r, count), bwd(M, m, n, r, count)
        assert f >= M * r * 2 and f % 256 == 0
        assert b >= 2 * m * n + 2 * count * n * r + 12 * M * r + 4 * (count + M) and b % 256 == 0
    for q in (fwd, bwd):
        assert [q(*a) for a in ((0, 64, 64, 16, 4), ((1 << 28) + 1, 64, 64, 16, 4), (10, 60, 64, 16, 4), (10, 64, 68, 16, 4), (10, 64, 64, 12, 4), (10, 64, 64, 136, 4),
                                (10, 64, 64, 16, 0), (10, 64, 64, 16, 65536), (10, (1 << 20) + 8, 64, 16, 4))] == [0] * 9
    norm = lib.lr_rms_norm_bwd_workspace_bytes
    for dt in (abt.ABT_BF16, abt.ABT_F32):
        assert norm(1, 8, dt) >= 32 and norm(100000, 16384, dt) >= 512 * 16384 * 4
        assert [norm(0, 8, dt), norm(1, 0, dt), norm(1, 12, dt), norm(1, 16392, dt), norm(1 << 31, 8, dt)] == [0] * 5
    assert norm(1, 8, 9) == 0
    # one for each 256 work-groups of a table of tensors
    assert lib.ab_grad_norm_workspace_bytes(0) >= 2048 and lib.ab_grad_norm_workspace_bytes(500) > lib.ab_grad_norm_workspace_bytes(1) and lib.ab_grad_norm_workspace_bytes(-1) == 0


def test_norm(lib):
    def fwd(X=P, R=None, gain=P, eps=1e-6, H=None, Y=P, Yq=None, s=None, M=4, n=64, dt=abt.ABT_BF16):
        return lib.lr_rms_norm_fwd(X, R, gain, eps, H, Y, Yq, s, M, n, dt, None)
    inf, nan = float("inf"), float("nan")
    assert fwd(dt=9) == EDTYPE
    assert [fwd(X=None), fwd(gain=None), fwd(Y=None), fwd(Yq=P), fwd(s=P), fwd(eps=-1.0), fwd(eps=inf), fwd(eps=nan)] == [EINVAL] * 8
    assert [fwd(M=0), fwd(M=1 << 31), fwd(n=0), fwd(n=12), fwd(n=16392)] == [ESHAPE] * 5
    assert [fwd(X=ODD), fwd(R=ODD), fwd(gain=ODD), fwd(H=ODD), fwd(Y=ODD), fwd(Yq=ODD, s=P), fwd(Yq=P, s=P + 2)] == [EALIGN] * 7

    def bwd(dY=P, H=P, gain=P, eps=1e-6, dH=None, dX=P, dgain=P, M=4, n=64, dt=abt.ABT_F32, ws=P, nbytes=BIG):
        return lib.lr_rms_norm_bwd(dY, H, gain, eps, dH, dX, dgain, M, n, dt, 0, ws, nbytes, None)
    assert bwd(dt=9) == EDTYPE
    assert [bwd(dY=None), bwd(H=None), bwd(gain=None), bwd(eps=-1.0), bwd(eps=nan)] == [EINVAL] * 5
    assert [bwd(M=0), bwd(M=1 << 31), bwd(n=0), bwd(n=12), bwd(n=16392)] == [ESHAPE] * 5
    assert [bwd(dY=ODD), bwd(H=ODD), bwd(gain=ODD), bwd(dH=ODD), bwd(dX=ODD), bwd(dgain=ODD), bwd(ws=P + 16)] == [EALIGN] * 7
    assert [bwd(ws=None), bwd(nbytes=lib.lr_rms_norm_bwd_workspace_bytes(4, 64, abt.ABT_F32) - 1)] == [EWORKSPACE] * 2
    assert bwd(dX=None, dgain=None) == OK and bwd(dX=None, dgain=None, ws=None) == OK


def test_clipping(lib):
    def table(**kw):
        t = dict(grad=P, out=None, count=100, dt=abt.ABT_F32)
        t.update(kw)
        a = (abt.GradTensor * 1)()
        a[0].grad, a[0].out, a[0].count, a[0].dt = t["grad"], t["out"], t["count"], t["dt"]
        return a

    def norm(a=None, n=1, out=P, ws=P, nbytes=BIG):
        return lib.ab_grad_norm(table() if a is None else a, n, out, ws, nbytes, None)

    def clip(a=None, n=1, limit=1.0, out=None, ws=P, nbytes=BIG):
        return lib.ab_clip_grads(table() if a is None else a, n, limit, out, ws, nbytes, None)
    for f in (norm, clip):
        assert [f(n=-1), f(a=table(grad=None))] == [EINVAL] * 2 and f(a=table(dt=9)) == EDTYPE
        assert [f(a=table(count=-1)), f(a=table(count=(1 << 40) + 1))] == [ESHAPE] * 2
        assert [f(a=table(grad=ODD)), f(out=P + 2), f(ws=P + 16)] == [EALIGN] * 3
        assert [f(ws=None), f(nbytes=8)] == [EWORKSPACE] * 2
    assert norm(out=None) == EINVAL and clip(a=table(out=ODD)) == EALIGN
    assert [clip(limit=x) for x in (-1.0, float("inf"), float("nan"))] == [EINVAL] * 3
    assert lib.ab_grad_norm(None, 1, P, P, BIG, None) == EINVAL

    def step(param=P, grad=P, count=100, n=1, step=1, limit=1.0, out=None, ws=P, nbytes=BIG, beta1=0.9):
        a = (abt.AdamwTensor * 1)()
        a[0].param, a[0].grad, a[0].exp_avg, a[0].exp_avg_sq, a[0].count = param, grad, P, P, count
        return lib.ab_adamw_step_clipped(a, n, step, 1e-3, 1.0, beta1, 0.999, 1e-8, 0.0, limit, out, ws, nbytes, None)
    assert [step(param=None), step(grad=None), step(n=-1), step(step=0), step(limit=-1.0), step(limit=float("nan"))] == [EINVAL] * 6
    assert step(count=-1) != OK and step(beta1=1.5) != OK and step(grad=ODD) != OK
    assert step(ws=P + 16) == EALIGN and step(ws=None) == EWORKSPACE and step(nbytes=8) == EWORKSPACE and step(out=P + 2) == EALIGN


def test_wrappers_refuse_before_the_library(lib):
    torch = pytest.importorskip("torch")
    x, w = torch.zeros(4, 16, dtype=torch.bfloat16), torch.zeros(16, 16, dtype=torch.bfloat16)
    A, B = torch.zeros(2, 16, 8, dtype=torch.bfloat16), torch.zeros(2, 8, 16, dtype=torch.bfloat16)
    ids = torch.zeros(4, dtype=torch.int32)
    for f in (lambda: abt.lr_adapters_fwd(x, w, A, B, ids), lambda: abt.lr_adapters_bwd(x, x, None, w, A, B, ids),      # tensors on the host
              lambda: abt.lr_rms_norm_fwd(x, torch.ones(16)), lambda: abt.lr_rms_norm_bwd(x, x, torch.ones(16)),
              lambda: abt.ab_clip_grads([torch.zeros(4)], 1.0)):
        with pytest.raises(abt.AbtError):
            f()
