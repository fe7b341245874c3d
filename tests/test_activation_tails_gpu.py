"""gelu far below zero, where the result is the normal distribution's tail: its error relative to itself, through the group norm in fp32 and the dense layer."""
import numpy as np
import pytest

from paper_2405_01067_amd import binding as abt
from plain_layers import act as value_and_slope

pytestmark = pytest.mark.gpu

BF, F32 = 2.0 ** -8, 2.0 ** -24


def d(t):
    return t.double().cpu().numpy()


def grid():
    import torch
    return torch.linspace(-12.5, 0.0, 4097)[:4096].contiguous()


def tail_err(z):
    """Relative.  The fit's 1.7e-7 and a few roundings of its evaluation, 2.7 times those of 1 / (1 + p |z|) (its slope against R's at 0), 2^-23 of the transcendental unit each: 1.5e-6.  The
    exponent -z^2 / 2 is rounded twice, 2^-24 of it each: z^2 2^-24."""
    return 1.5e-6 + 1.1 * F32 * z * z


def test_gelu_in_fp32():
    import torch
    z = grid().cuda()
    C = z.numel()
    x = torch.randn((1, 2, C), device="cuda")
    Y, mean, rstd = abt.lr_group_norm_fwd(x, torch.zeros_like(z), z, 8, act="gelu")         # gain 0: what the activation sees is z itself
    want = value_and_slope(d(z), "gelu")[0]
    for y in d(Y[0]):
        off = np.abs(y - want) / (np.abs(want) * (tail_err(d(z)) + 2 * F32))
        assert off.max() <= 1.0, (d(z)[off.argmax()], off.max())
    # the slope Phi(z) + z phi(z), whose terms are of different signs: relative to their size
    one = torch.ones((1, 1, C), device="cuda")
    _, mean, rstd = abt.lr_group_norm_fwd(x[:, :1].contiguous(), torch.zeros_like(z), z, 8, act="gelu")
    _, _, slope = abt.lr_group_norm_bwd(one, x[:, :1].contiguous(), torch.zeros_like(z), z, mean, rstd, act="gelu", need_dX=False, need_dgain=False)
    v = d(z)
    want = value_and_slope(v, "gelu")[1]
    size = np.abs(value_and_slope(v, "gelu")[0] / v) + np.abs(v) * np.exp(-v * v / 2) / np.sqrt(2 * np.pi)
    off = np.abs(d(slope) - want) / (size * (tail_err(v) + 4 * F32))
    assert off.max() <= 1.0, (v[off.argmax()], off.max())


@pytest.mark.parametrize("M", (3, 200))
def test_gelu_of_the_dense_layer(M):
    import torch
    z = grid().cuda()
    X, W = torch.zeros((M, 64), dtype=torch.bfloat16, device="cuda"), torch.zeros((z.numel(), 64), dtype=torch.bfloat16, device="cuda")
    Y, _ = abt.lr_dense_fwd(X, W, z, act="gelu")
    want = value_and_slope(d(z), "gelu")[0]
    bound = np.abs(want) * (BF * (1 + tail_err(d(z))) + tail_err(d(z)) + 2 * F32)
    assert bool((Y == Y[0]).all()) and (np.abs(d(Y[0]) - want) <= bound).all()
