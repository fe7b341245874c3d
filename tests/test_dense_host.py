"""Refusals and workspace queries of the dense layer, dropout and the group norm at the C entries, and the generator's published outputs: no GPU is needed, as
arguments are looked at before the device is."""
import ctypes
import os

import pytest

from paper_2405_01067_amd import binding as abt
from plain_layers import MASK, mask16, philox

P, ODD = 0x10000, 0x10008                     # stand for device pointers: aligned to 256, and to 8 only
BIG = 1 << 45                                 # bytes of workspace
OK, EINVAL, EDTYPE, ESHAPE, EALIGN, EWORKSPACE = 0, -1, -5, -2, -3, -4


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(abt._LIB_PATH):
        import __graft_entry__ as ge
        ge.build()
    return abt.load()


def drop(state=P, site=0, p=0.1):
    return ctypes.byref(abt.DropoutArgs(state, site, p))


BAD_DROPS = [(dict(state=None), EINVAL), (dict(p=-0.01), EINVAL), (dict(p=1.01), EINVAL), (dict(p=float("nan")), EINVAL), (dict(state=P + 4), EALIGN)]
BAD_SIZES = [(0, 64, 64), (-1, 64, 64), ((1 << 28) + 1, 64, 64), (10, 0, 64), (10, 68, 64), (10, 64, 60), (10, (1 << 20) + 8, 64), (10, 64, (1 << 20) + 8), (10, -8, 64)]


def test_the_generators_published_outputs():
    """Known answers of Philox4x32-10 (Salmon et al. 2011, the authors' test vectors)."""
    for counter, key, want in (((0,) * 4, (0, 0), (0x6627e8d5, 0xe169c58d, 0xbc57ac4c, 0x9b00dbd8)),
                               ((MASK,) * 4, (MASK, MASK), (0x408f276d, 0x41c83b0e, 0xa20bc7c6, 0x6d5451fd)),
                               ((0x243f6a88, 0x85a308d3, 0x13198a2e, 0x03707344), (0xa4093822, 0x299f31d0), (0xd16cfe09, 0x94fdcceb, 0x5001e420, 0x24126ea1))):
        assert tuple(philox(counter, key)) == want
    # the mask's bits are its words in order, low half first
    seed, at = 0x299f31d0a4093822, 0x0370734413198a2e
    small = philox((5, 0, at & MASK, at >> 32), (seed & MASK, seed >> 32))
    assert mask16(seed, at, 40, 8).tolist() == [w >> s & 0xffff for w in small for s in (0, 16)]
    assert mask16(seed, at, 37, 9).tolist() == mask16(seed, at, 32, 16).tolist()[5:14]


def test_dense_forward(lib):
    def call(X=P, W=P, bias=P, R=P, Y=P, Z=P, M=10, m=64, n=64, act=2, d=None, dt=abt.ABT_BF16, ws=P, nbytes=BIG):
        return lib.lr_dense_fwd(X, W, bias, R, Y, Z, M, m, n, act, d, dt, ws, nbytes, None)
    assert call(dt=abt.ABT_F32) == EDTYPE and call(dt=7) == EDTYPE
    assert [call(X=None), call(W=None), call(Y=None), call(act=-1), call(act=5)] == [EINVAL] * 5
    for kw, want in BAD_DROPS:
        assert call(d=drop(**kw)) == want, kw
    for M, m, n in BAD_SIZES:
        assert call(M=M, m=m, n=n) == ESHAPE, (M, m, n)
    assert [call(**{k: ODD}) for k in ("X", "W", "bias", "R", "Y", "Z")] == [EALIGN] * 6 and call(ws=P + 16, M=48, m=4096, n=4096) == EALIGN
    assert [call(ws=None, M=48, m=4096, n=4096), call(nbytes=lib.lr_dense_fwd_workspace_bytes(48, 4096, 4096) - 1, M=48, m=4096, n=4096)] == [EWORKSPACE] * 2


def test_dense_backward(lib):
    def call(dY=P, X=P, W=P, Z=P, dX=P, dW=P, db=P, M=10, m=64, n=64, act=2, d=None, dt=abt.ABT_BF16, ws=P, nbytes=BIG):
        return lib.lr_dense_bwd(dY, X, W, Z, dX, dW, db, M, m, n, act, d, dt, 0, ws, nbytes, None)
    assert call(dt=abt.ABT_F32) == EDTYPE
    # W for dX, X for dW, Z for an activation
    assert [call(dY=None), call(W=None), call(X=None), call(Z=None), call(act=5), call(act=-1)] == [EINVAL] * 6
    for kw, want in BAD_DROPS:
        assert call(d=drop(**kw)) == want, kw
    for M, m, n in BAD_SIZES:
        assert call(M=M, m=m, n=n) == ESHAPE, (M, m, n)
    assert [call(**{k: ODD}) for k in ("dY", "X", "W", "Z", "dX", "dW", "db")] == [EALIGN] * 7
    assert call(ws=P + 16) == EALIGN and call(ws=None) == EWORKSPACE
    assert call(nbytes=lib.lr_dense_bwd_workspace_bytes(10, 64, 64) - 1) == EWORKSPACE
    assert call(dX=None, dW=None, db=None) == OK and call(dX=None, dW=None, db=None, Z=None, act=0, W=None, X=None) == OK       # nothing to do


def test_dropout(lib):
    def call(X=P, R=None, Y=P, count=100, d=None, dt=abt.ABT_BF16, none=False):
        return lib.lr_dropout(X, R, Y, count, None if none else d or drop(), dt, None)
    assert call(dt=9) == EDTYPE
    assert [call(X=None), call(Y=None), call(none=True)] == [EINVAL] * 3
    for kw, want in BAD_DROPS:
        assert call(d=drop(**kw)) == want, kw
    assert [call(count=-1), call(count=(1 << 45) + 1)] == [ESHAPE] * 2
    assert [call(X=ODD), call(R=ODD), call(Y=ODD)] == [EALIGN] * 3
    assert call(count=0) == OK and call(count=0, X=None, Y=None) == OK


BAD_IMAGES = [(0, 4, 64, 8), (4, 0, 64, 8), (4, 4, 0, 8), (4, 4, 60, 4), (4, 4, 64, 0), (4, 4, 64, 7), (4, 4, 64, 65), (4, 4, 64, 128), (4, 4, 65544, 8), ((1 << 28) + 1, 4, 64, 8),
              (4, (1 << 28) + 1, 64, 8), (1 << 28, 1 << 20, 64, 8), (-1, 4, 64, 8), (4, 4, 64, -8)]


def test_group_norm(lib):
    inf, nan = float("inf"), float("nan")

    def fwd(X=P, gain=P, shift=P, eps=1e-5, Y=P, mean=P, rstd=P, N=4, pixels=49, C=64, G=8, act=1, dt=abt.ABT_BF16, ws=P, nbytes=BIG):
        return lib.lr_group_norm_fwd(X, gain, shift, eps, Y, mean, rstd, N, pixels, C, G, act, dt, ws, nbytes, None)

    def bwd(dY=P, X=P, gain=P, shift=P, mean=P, rstd=P, dX=P, dgain=P, dshift=P, N=4, pixels=49, C=64, G=8, act=1, dt=abt.ABT_F32, ws=P, nbytes=BIG):
        return lib.lr_group_norm_bwd(dY, X, gain, shift, mean, rstd, dX, dgain, dshift, N, pixels, C, G, act, dt, 0, ws, nbytes, None)
    assert fwd(dt=9) == EDTYPE and bwd(dt=9) == EDTYPE
    assert [fwd(**{k: None}) for k in ("X", "gain", "shift", "Y", "mean", "rstd")] + [fwd(eps=-1.0), fwd(eps=inf), fwd(eps=nan), fwd(act=5), fwd(act=-1)] == [EINVAL] * 11
    assert [bwd(**{k: None}) for k in ("dY", "X", "gain", "shift", "mean", "rstd")] + [bwd(act=5), bwd(act=-1)] == [EINVAL] * 8
    for N, pixels, C, G in BAD_IMAGES:
        assert fwd(N=N, pixels=pixels, C=C, G=G) == ESHAPE and bwd(N=N, pixels=pixels, C=C, G=G) == ESHAPE, (N, pixels, C, G)
    assert [fwd(**{k: ODD}) for k in ("X", "gain", "shift", "Y")] + [fwd(mean=P + 2), fwd(rstd=P + 2), fwd(ws=P + 16, N=1, pixels=1 << 20)] == [EALIGN] * 7
    assert [bwd(**{k: ODD}) for k in ("dY", "X", "gain", "shift", "dX", "dgain", "dshift")] + [bwd(mean=P + 2), bwd(rstd=P + 1), bwd(ws=P + 16)] == [EALIGN] * 10
    assert [fwd(ws=None, N=1, pixels=1 << 20), fwd(nbytes=0, N=1, pixels=1 << 20), bwd(ws=None), bwd(nbytes=lib.lr_group_norm_workspace_bytes(4, 49, 64, 8, abt.ABT_F32, 1) - 1)] == [EWORKSPACE] * 4
    assert bwd(dX=None, dgain=None, dshift=None) == OK


def test_workspaces(lib):
    fwd, bwd, group = lib.lr_dense_fwd_workspace_bytes, lib.lr_dense_bwd_workspace_bytes, lib.lr_group_norm_workspace_bytes
    for M, m, n in ((1, 8, 8), (48, 4096, 4096), (394, 768, 768), (12608, 2304, 768), (1 << 28, 1 << 20, 8), (1, 1 << 20, 1 << 20)):
        assert fwd(M, m, n) % 256 == 0
        assert bwd(M, m, n) >= 4 * M * m + 2 * m * n and bwd(M, m, n) % 256 == 0
    assert fwd(48, 4096, 4096) >= 2 * 4 * 48 * 4096 and fwd(1, 768, 768) == 0      # in pieces of the contraction; not
    for f in (fwd, bwd):
        assert [f(*s) for s in BAD_SIZES] == [0] * len(BAD_SIZES)
    for dt in (abt.ABT_BF16, abt.ABT_F32):
        for backward in (0, 1):
            for shape in ((1, 1 << 28, 65536, 65536), (1, 1 << 20, 64, 8), (1, 4096, 2048, 32)):         # in pieces
                assert group(*shape, dt, backward) >= 8 * shape[3] and group(*shape, dt, backward) % 256 == 0
            assert group(1, 49, 64, 8, dt, backward) == 0
            assert [group(*s, dt, backward) for s in BAD_IMAGES] == [0] * len(BAD_IMAGES)
        assert group(256, 196, 256, 32, dt, 1) >= 256 * 256 * 8
    assert group(4, 49, 64, 8, 9, 0) == 0


def test_wrappers_refuse_before_the_library(lib):
    torch = pytest.importorskip("torch")
    x, w = torch.zeros(4, 16, dtype=torch.bfloat16), torch.zeros(16, 16, dtype=torch.bfloat16)
    one = torch.ones(16)
    for f in (lambda: abt.lr_dense_fwd(x, w), lambda: abt.lr_dense_bwd(x, x, w), lambda: abt.lr_dropout(x, None), lambda: abt.Dropout(0.1, torch.zeros(2, dtype=torch.int64)),
              lambda: abt.lr_group_norm_fwd(x, one, one, 4), lambda: abt.lr_group_norm_bwd(x, x, one, one, torch.zeros(4, 4), torch.ones(4, 4))):       # tensors on the host
        with pytest.raises(abt.AbtError):
            f()


def test_native_calls_load(lib):
    pytest.importorskip("torch")
    assert abt.dense_call() is not None
