"""An adapter in use that holds an infinity or NaN: by Y_i = W x_i + s_a A_a T_i and dX_i = W^T dY_i + B_a^T dT_i it has a part in the results of
its own rows only, so whatever else is in their batch, tile or work-group gives the values that it gives beside a finite adapter."""
import pytest
import torch

from paper_2405_01067_amd import binding as abt
from test_adapters_gpu import gpu, make

pytestmark = pytest.mark.gpu

BAD = (float("nan"), float("inf"), float("-inf"))
# One launch, two launches, and each of the six tiles of many rows; rows in any order and in runs (-1, no adapter, among them)
SIZES = [(4, 40, 768, 8, 4, "any"), (5, 40, 768, 8, 4, "any"), (16, 24, 528, 128, 5, "any"), (40, 136, 80, 24, 5, "any"), (64, 2304, 768, 32, 9, "any"), (100, 136, 80, 24, 5, "any"),
         (128, 264, 1040, 16, 70, "any"), (700, 136, 80, 24, 5, "any"), (1000, 264, 208, 120, 9, "runs"), (2000, 136, 80, 16, 5, "any"), (3001, 2056, 80, 32, 11, "runs"), (4099, 200, 80, 64, 6, "any"),
         (9001, 72, 80, 16, 4, "runs"), (12490, 392, 80, 128, 3, "any"), (15999, 776, 80, 16, 9, "runs"), (23990, 392, 144, 24, 7, "any")]


def case(M, m, n, r, K, rows):
    c = make(M, m, n, r, K, rows, False, seed=M + 7 * m)
    c["ids"][:4] = (K - 1, -1, 0, 1)                         # one adapter, none and others side by side
    d = gpu(c)
    return d, (d["row_adapter"], d["ranks"], d["scales"]), K - 1, d["row_adapter"] == K - 1


def only(got, clean, mask, what):
    """The same bits wherever mask does not say that a value has to be infinite or NaN."""
    assert torch.equal(torch.where(mask, 0, got), torch.where(mask, 0, clean)), what
    assert bool((~torch.isfinite(got) | ~mask).all()), what


@pytest.mark.parametrize("M,m,n,r,K,rows", SIZES)
def test_forward(M, m, n, r, K, rows):
    d, of, a, mine = case(M, m, n, r, K, rows)
    f8 = torch.float8_e4m3fn
    scale = {k: d[k].float().abs().amax(1) / 448 for k in ("X", "W")}
    q = (d["X"], (d["X"].float() / scale["X"][:, None]).to(f8), scale["X"], (d["W"].float() / scale["W"][:, None]).to(f8), scale["W"])
    Y, T = abt.lr_adapters_fwd(d["X"], d["W"], d["A"], d["B"], *of)
    Y8 = abt.lr_adapters_fwd_q8(*q, d["A"], d["B"], *of)
    j = m - 3
    mask = torch.zeros_like(Y, dtype=torch.bool)
    mask[:, j] = mine
    for bad in BAD:
        A = d["A"].clone()
        A[a, j, r - 1] = bad
        got, T1 = abt.lr_adapters_fwd(d["X"], d["W"], A, d["B"], *of)
        assert torch.equal(T, T1)
        only(got, Y, mask, bad)
        only(abt.lr_adapters_fwd_q8(*q, A, d["B"], *of), Y8, mask, bad)
    B = d["B"].clone()
    B[a, 0, n // 2] = float("nan")                           # T of its own rows, and with it all of their Y
    got, T1 = abt.lr_adapters_fwd(d["X"], d["W"], d["A"], B, *of)
    column = torch.zeros_like(T, dtype=torch.bool)
    column[:, 0] = mine
    only(T1, T, column, "T")
    only(got, Y, mine[:, None].expand_as(Y), "Y")
    only(abt.lr_adapters_fwd_q8(*q, d["A"], B, *of), Y8, mine[:, None].expand_as(Y), "Y from 8 bits")


@pytest.mark.parametrize("M,m,n,r,K,rows", SIZES)
def test_backward(M, m, n, r, K, rows):
    d, of, a, mine = case(M, m, n, r, K, rows)
    _, T = abt.lr_adapters_fwd(d["X"], d["W"], d["A"], d["B"], *of)
    clean = abt.lr_adapters_bwd(d["dY"], d["X"], T, d["W"], d["A"], d["B"], *of)
    k = n - 2
    mask = torch.zeros_like(clean[0], dtype=torch.bool)
    mask[:, k] = mine
    for bad in BAD:
        B = d["B"].clone()
        B[a, r - 1, k] = bad
        dX, dA, dB = abt.lr_adapters_bwd(d["dY"], d["X"], T, d["W"], d["A"], B, *of)
        only(dX, clean[0], mask, bad)
        assert torch.equal(dA, clean[1]) and torch.equal(dB, clean[2])
    A = d["A"].clone()
    A[a, m // 2, 0] = float("nan")                           # dT of its own rows, with it all of their dX and one row of dB
    dX, dA, dB = abt.lr_adapters_bwd(d["dY"], d["X"], T, d["W"], A, d["B"], *of)
    only(dX, clean[0], mine[:, None].expand_as(dX), "dX")
    assert torch.equal(dA, clean[1])
    row = torch.zeros_like(dB, dtype=torch.bool)
    row[a, 0] = True
    only(dB, clean[2], row, "dB")


@pytest.mark.parametrize("M,m,n,r,K,rows", SIZES)
def test_all_but_one(M, m, n, r, K, rows):
    """Every adapter but the first is nothing but NaN and infinities, up to ranks that end inside a piece and past them: the first one's rows and those of
    none are what they were, the others have no finite value but where their rank is 0."""
    d, (ids, _, scales), _, _ = case(M, m, n, r, K, rows)
    ranks = torch.tensor([r if a == 0 else (r, 5, 0, r - 3)[a % 4] for a in range(K)], dtype=torch.int32, device="cuda")
    of = (ids, ranks, scales)
    broken = (ids > 0) & (ranks[ids.clamp(min=0).long()] > 0)
    A, B = d["A"].clone(), d["B"].clone()
    A[1::2], A[2::2], B[1::2], B[2::2] = float("nan"), float("inf"), float("-inf"), float("nan")
    Y, T = abt.lr_adapters_fwd(d["X"], d["W"], d["A"], d["B"], *of)
    got, T1 = abt.lr_adapters_fwd(d["X"], d["W"], A, d["B"], *of)
    assert torch.equal(T, T1)
    only(got, Y, broken[:, None].expand_as(Y), "Y, A broken")
    only(abt.lr_adapters_fwd(d["X"], d["W"], A, B, *of)[0], Y, broken[:, None].expand_as(Y), "Y, both broken")
    clean = abt.lr_adapters_bwd(d["dY"], d["X"], T, d["W"], d["A"], d["B"], *of)
    dX, dA, dB = abt.lr_adapters_bwd(d["dY"], d["X"], T, d["W"], A, B, *of)
    only(dX, clean[0], broken[:, None].expand_as(dX), "dX")
    assert torch.equal(dA, clean[1]) and torch.equal(dB[0], clean[2][0])
