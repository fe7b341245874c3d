"""The backward of the root-mean-square norm with eps = 0, or one that is 0 in fp32, against its definition in fp64 and with the bounds of
test_rms_norm_gpu.py: rows that the last group of a work-group lacks have no part in the gain's gradient."""
import pytest
import torch

from paper_2405_01067_amd import binding as abt
from test_rms_norm_gpu import DT, E, make, within

pytestmark = pytest.mark.gpu


# one wave, a pair of waves (bf16, more than 512 rows) and a work-group per row; full and incomplete groups of rows
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("M,n", [(1, 8), (1, 768), (2, 768), (3, 768), (4, 768), (5, 768), (7, 2048), (2049, 64), (5, 2056), (513, 2056), (514, 4096), (3, 8200)])
def test_gradients_without_eps(M, n, dtype):
    c = make(M, n, dtype, 5 * M + n)
    u = DT[dtype][1]
    d = {k: v.cuda() for k, v in c.items()}
    H, dY, gain = c["X"].double(), c["dY"].double(), c["gain"].double()
    s = 1 / torch.sqrt((H * H).mean(1, keepdim=True))
    w = dY * gain
    want = s * (w - H * s * s * (w * H).mean(1, keepdim=True))
    size = s * w.abs() + H.abs() * s ** 3 * (w * H).abs().mean(1, keepdim=True)
    for eps in (0.0, 1e-60):
        dX, dg = abt.lr_rms_norm_bwd(d["dY"], d["X"], d["gain"], eps=eps)
        within(dg, (dY * H * s).sum(0), (M + n / 2 + 16) * E * (dY * H * s).abs().sum(0), "dgain")
        within(dX, want, u * want.abs() + (n + 16) * E * size, "dX")
