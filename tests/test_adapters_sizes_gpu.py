"""The layer with adapters at the sizes where one kernel, tile or launch takes over from another, and both ways into the library, against the
definition in fp64 and with the bounds of test_adapters_gpu.py (derived there)."""
import pytest
import torch

from paper_2405_01067_amd import binding as abt
from test_adapters_gpu import E, U, gpu, make, reference, within

pytestmark = pytest.mark.gpu

# Rows, outputs and contractions for each of the six tiles of Y (of 256, 192, 128 and 64 rows), ending inside a tile; runs of one adapter and a
# new adapter in every row.
TILES = [(15999, 776, 80, 16, 9, "runs"), (23990, 392, 144, 24, 7, "runs"), (12499, 776, 80, 40, 5, "sorted"), (4101, 1544, 80, 8, 33, "runs"), (12490, 392, 80, 128, 3, "runs"),
         (9001, 72, 80, 16, 4, "runs"), (4099, 200, 80, 64, 6, "any"), (130, 72, 144, 16, 3, "any"), (3001, 2056, 80, 32, 11, "any"), (2045, 776, 400, 96, 3, "any"),
         (8200, 1032, 80, 72, 6, "outside")]


@pytest.mark.parametrize("M,m,n,r,K,rows", TILES)
def test_tiles_of_the_forward(M, m, n, r, K, rows):
    c = make(M, m, n, r, K, rows, rows != "any", seed=M + m)
    d = gpu(c)
    o, b = reference(c)
    Y, T = abt.lr_adapters_fwd(d["X"], d["W"], d["A"], d["B"], d["row_adapter"], d["ranks"], d["scales"])
    within(T, o["T"], b["T"], "T")
    within(Y, o["Y"], b["Y"], "Y")


# contractions of 16 more columns, and tiles of the 8-bit product: half the bytes in a slab
TILES_8 = [(15999, 776, 80, 16, 9, "runs"), (23990, 392, 144, 24, 7, "runs"), (15990, 520, 80, 40, 5, "sorted"), (4101, 1544, 80, 8, 33, "runs"), (12490, 392, 80, 128, 3, "runs"),
           (303, 72, 80, 16, 4, "runs"), (131, 136, 784, 64, 6, "any"), (9001, 1032, 80, 32, 3, "any"), (2045, 776, 400, 96, 3, "any")]
# The bound of test_adapters_gpu.py takes the matrix unit's sums for fp32 sums of exact products.  Of 8-bit floats they are not: a product is cut at 2^-13 of
# the largest of the eight that it is added with (the same in all three 8-bit instructions: 2^16 + 7 * 2^2 gives 2^16, in bf16 it is exact).  Where a
# row has no adapter and the sum almost cancels, that shows: 2 elements of 12 and of 6 million are off by 1.0 to 1.3 times this bound.
EXACT_8 = [pytest.param(*t, marks=pytest.mark.xfail(strict=False, reason="the matrix unit cuts 8-bit products at 2^-13 of the largest of eight")) if t[:2] in ((15999, 776), (4101, 1544))
           else t for t in TILES_8]


def forward_from_8_bits(M, m, n, r, K, rows):
    c = make(M, m, n, r, K, rows, rows != "any", seed=M + m)
    f8 = torch.float8_e4m3fn
    scale = {k: c[k].float().abs().amax(1) / 448 for k in ("X", "W")}
    q = {k: (c[k].float() / scale[k][:, None]).to(f8) for k in ("X", "W")}
    d = gpu(c)
    Y = abt.lr_adapters_fwd_q8(d["X"], q["X"].cuda(), scale["X"].cuda(), q["W"].cuda(), scale["W"].cuda(), d["A"], d["B"], d["row_adapter"], d["ranks"], d["scales"])
    o, b = reference(c)
    Xd, Wd = (q[k].double() * scale[k].double()[:, None] for k in ("X", "W"))
    X, W = c["X"].double(), c["W"].double()
    want = o["Y"] - X @ W.T + Xd @ Wd.T
    bound = b["Y"] - U * o["Y"].abs() - (n + r) * E * (X.abs() @ W.abs().T) + U * want.abs() + (n + r + 4) * E * (Xd.abs() @ Wd.abs().T)
    return Y, want, bound, Xd, Wd


@pytest.mark.parametrize("M,m,n,r,K,rows", EXACT_8)
def test_tiles_of_the_forward_from_8_bits(M, m, n, r, K, rows):
    Y, want, bound, _, _ = forward_from_8_bits(M, m, n, r, K, rows)
    within(Y, want, bound, "Y")


@pytest.mark.parametrize("M,m,n,r,K,rows", TILES_8)
def test_tiles_of_the_forward_from_8_bits_as_the_matrix_unit_adds(M, m, n, r, K, rows):
    """Every product off by up to 2^-13 of the largest that the row and the column can have; and all in all, where these cuts (some 2^-12 of a result) and
    the roundings of T and Y (2^-9 / sqrt(3) each) go either way, by less than 2^-8."""
    Y, want, bound, Xd, Wd = forward_from_8_bits(M, m, n, r, K, rows)
    within(Y, want, bound + n * 2.0 ** -13 * Xd.abs().amax(1)[:, None] * Wd.abs().amax(1)[None], "Y")
    assert float((Y.double().cpu() - want).norm() / want.norm()) < 2.0 ** -8


# One launch up to 32 values of T and 3072 bytes of a row, two launches beyond, and up to 128 rows; parts of the contraction in groups of 64 rows.
@pytest.mark.parametrize("M,m,n,r,K", [(1, 40, 1536, 32, 2), (1, 40, 1544, 32, 2), (1, 40, 1536, 40, 2), (2, 24, 768, 16, 3), (3, 24, 768, 16, 3), (4, 24, 768, 8, 3), (5, 24, 768, 8, 3),
                                       (16, 8, 136, 128, 9), (17, 8, 136, 128, 9), (63, 72, 264, 16, 5), (64, 72, 264, 16, 5), (65, 72, 264, 16, 70), (127, 72, 264, 16, 5),
                                       (128, 72, 264, 16, 5), (129, 72, 264, 16, 5), (16, 72, 4104, 16, 20), (2, 136, 8200, 8, 2)])
def test_few_rows(M, m, n, r, K):
    for rows, mixed in (("any", True), ("one", False), ("none", False)):
        c = make(M, m, n, r, K, rows, mixed, seed=M + m + r)
        d = gpu(c)
        o, b = reference(c)
        Y, T = abt.lr_adapters_fwd(d["X"], d["W"], d["A"], d["B"], d["row_adapter"], d["ranks"], d["scales"])
        within(T, o["T"], b["T"], "T")
        within(Y, o["Y"], b["Y"], "Y")


# Between the few rows' kernels and those of many: T row by row up to 24576 values and 1024 rows, by tiles beyond.
@pytest.mark.parametrize("M,m,n,r,K,rows", [(130, 40, 264, 16, 3, "any"), (160, 136, 520, 64, 30, "any"), (191, 72, 1032, 128, 5, "any"), (192, 200, 264, 8, 192, "any"), (192, 72, 2056, 24, 3, "sorted"),
                                            (193, 72, 264, 16, 5, "any"), (1024, 40, 264, 24, 3, "any"), (1025, 40, 264, 24, 3, "any"), (1024, 40, 264, 32, 30, "any"),
                                            (512, 40, 4104, 48, 6, "runs"), (513, 40, 4104, 48, 6, "runs")])
def test_rows_of_a_few_groups(M, m, n, r, K, rows):
    c = make(M, m, n, r, K, rows, True, seed=M + m + r)
    d = gpu(c)
    o, b = reference(c)
    Y, T = abt.lr_adapters_fwd(d["X"], d["W"], d["A"], d["B"], d["row_adapter"], d["ranks"], d["scales"])
    within(T, o["T"], b["T"], "T")
    within(Y, o["Y"], b["Y"], "Y")


# Gradients with dX in the same launch, before it, and beside pieces of many rows; ranks padded to 16, 32, 64 and 128; 1024 rows and one more.
@pytest.mark.parametrize("M,m,n,r,K,rows", [
    (1000, 776, 2056, 8, 4, "runs"), (1000, 776, 2056, 24, 4, "any"), (1000, 776, 2056, 40, 4, "runs"), (1000, 776, 2056, 72, 4, "runs"),
    (1023, 72, 136, 16, 5, "any"), (1024, 72, 136, 32, 5, "any"), (1024, 136, 72, 64, 5, "any"), (1024, 72, 136, 128, 5, "any"), (1025, 72, 136, 16, 5, "any"),
    (1025, 136, 72, 128, 5, "any"), (3001, 72, 2056, 16, 7, "runs"), (12499, 72, 392, 32, 5, "runs"), (12499, 72, 392, 8, 300, "any"), (3001, 72, 2056, 64, 7, "runs"),
    (5000, 136, 520, 120, 3, "sorted"), (4100, 8, 8, 16, 2, "outside")])
def test_launches_of_the_backward(M, m, n, r, K, rows):
    c = make(M, m, n, r, K, rows, rows != "any", seed=M + 3 * m + r)
    d = gpu(c)
    args = (d["W"], d["A"], d["B"], d["row_adapter"], d["ranks"], d["scales"])
    _, T = abt.lr_adapters_fwd(d["X"], *args)
    got = abt.lr_adapters_bwd(d["dY"], d["X"], T, *args)
    o, b = reference(c, T.cpu())
    for g, k in zip(got, ("dX", "dA", "dB")):
        within(g, o[k], b[k], k)


@pytest.mark.parametrize("M", [1, 2, 48, 300, 2000])
def test_both_ways_into_the_library(M):
    """The native calls and the ctypes ones give the same bits (given a workspace or an output, the wrappers take the latter)."""
    if abt.adapter_call() is None:
        pytest.skip("the native calls are not built")
    c = make(M, 136, 272, 16, 5, "any", True, seed=M)
    d = gpu(c)
    lib = abt.load()
    ws = torch.empty(max(lib.lr_adapters_fwd_workspace_bytes(M, 136, 272, 16, 5), lib.lr_adapters_bwd_workspace_bytes(M, 136, 272, 16, 5)), dtype=torch.uint8, device="cuda")
    args = (d["W"], d["A"], d["B"], d["row_adapter"])
    for more in ((d["ranks"], d["scales"]), (None, None)):
        Y, T = abt.lr_adapters_fwd(d["X"], *args, *more)
        Y1, T1 = abt.lr_adapters_fwd(d["X"], *args, *more, workspace=ws)
        assert torch.equal(Y, Y1) and torch.equal(T, T1)
        for t in (T, None):
            for x, y in zip(abt.lr_adapters_bwd(d["dY"], d["X"], t, *args, *more), abt.lr_adapters_bwd(d["dY"], d["X"], t, *args, *more, workspace=ws)):
                assert torch.equal(x, y)
        gain = torch.rand(272, device="cuda") + 0.5
        N, H, Nq, s = abt.lr_rms_norm_fwd(d["X"], gain, residual=d["X"], quantize=True)
        N1, H1, Nq1, s1 = abt.lr_rms_norm_fwd(d["X"], gain, residual=d["X"], quantize=True, Y=torch.empty_like(N))
        assert torch.equal(N, N1) and torch.equal(H, H1) and torch.equal(Nq.view(torch.uint8), Nq1.view(torch.uint8)) and torch.equal(s, s1)
        Wq = d["W"].to(torch.float8_e4m3fn)
        ones = torch.ones(136, device="cuda")
        q = (N, Nq, s, Wq, ones, *args[1:], *more)
        assert torch.equal(abt.lr_adapters_fwd_q8(*q), abt.lr_adapters_fwd_q8(*q, workspace=ws))
        dN = d["X"] * 0.5
        nws = torch.empty(lib.lr_rms_norm_bwd_workspace_bytes(M, 272, abt.ABT_BF16), dtype=torch.uint8, device="cuda")
        for x, y in zip(abt.lr_rms_norm_bwd(dN, H, gain, dH=N), abt.lr_rms_norm_bwd(dN, H, gain, dH=N, workspace=nws)):
            assert torch.equal(x, y)


@pytest.mark.parametrize("n,M", [(8, (1 << 25) + 3), (2056, 1537)])
def test_norm_of_many_rows(n, M):
    """More rows than one launch of the forward has threads for; two waves per row in the backward, and a last row alone."""
    g = torch.Generator(device="cuda").manual_seed(n)
    X = torch.randn((M, n), generator=g, device="cuda", dtype=torch.float32).bfloat16()
    gain = torch.rand(n, generator=g, device="cuda") + 0.5
    Y = abt.lr_rms_norm_fwd(X, gain)[0]
    dX, dgain = abt.lr_rms_norm_bwd(Y, X, gain)
    picked = torch.tensor([0, 1, 2, 3, M // 2, (1 << 25) - 1, 1 << 25, M - 2, M - 1]) % M
    x, dy, w = X[picked.cuda()].cpu().double(), Y[picked.cuda()].cpu().double(), gain.cpu().double()
    s = 1 / torch.sqrt((x * x).mean(1, keepdim=True) + 1e-6)
    within(Y[picked.cuda()], x * s * w, (U + (n / 2 + 8) * E) * (x * s * w).abs(), "Y")
    want = s * (dy * w - x * s * s * (dy * w * x).mean(1, keepdim=True))
    within(dX[picked.cuda()], want, U * want.abs() + (n + 16) * E * (s * (dy * w).abs() + x.abs() * s ** 3 * (dy * w * x).abs().mean(1, keepdim=True)), "dX")
    total = torch.zeros(n, dtype=torch.float64, device="cuda")
    size = torch.zeros(n, dtype=torch.float64, device="cuda")
    for i in range(0, M, 1 << 22):
        x, dy = X[i:i + (1 << 22)].double(), Y[i:i + (1 << 22)].double()
        t = dy * x / torch.sqrt((x * x).mean(1, keepdim=True) + 1e-6)
        total += t.sum(0)
        size += t.abs().sum(0)
    # a lane adds at most M / 512 rows in fp32, then waves and work-groups: far fewer than M additions in a row
    within(dgain, total.cpu(), (M / 512 + n / 2 + 544) * E * size.cpu(), "dgain")
