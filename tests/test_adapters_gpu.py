"""The layer with adapters on the GPU (lr_adapters_fwd, lr_adapters_fwd_q8, lr_adapters_bwd) against its definition in fp64,
element by element.

Bounds.  Rounding to bf16 is off by at most 2^-8 of the value.  A sum of N exact products in fp32, in any order, is off by at most
N 2^-23 times the sum of their sizes (2^-24 per addition if every one rounds to nearest; twice that allows for truncation).  So
    T    n 2^-23 sum |b x|
    Y    2^-8 |Y| + 2^-8 s sum |a T| (T is rounded once) + (n + r) 2^-23 (sum |w x| + s sum |a T|) + what T is off
    dT   (m + 2) 2^-23 s sum |dY a|
    dX   2^-8 |dX| + 2^-8 sum |dT b| + (m + r) 2^-23 (..) + what dT is off
    dA   (N + 16) 2^-23 sum |s dY T| for N rows;  dB likewise, and what dT is off
(the second factors of dA and dB are fp32 values in three bf16 pieces, exact to 2^-24)."""
import numpy as np
import pytest
import torch

from paper_2405_01067_amd import binding as abt

pytestmark = pytest.mark.gpu

BF, U, E = torch.bfloat16, 2.0 ** -8, 2.0 ** -23


def rows_of(kind, M, K, rs):
    """Adapter ids of the rows: runs of one adapter, any order, sorted, one alone, none at all, ids outside the stack."""
    if kind == "runs":
        ids = np.repeat(rs.randint(-1, K, M), rs.randint(1, 40, M))[:M]
    elif kind == "sorted":
        ids = np.sort(rs.randint(0, K, M))
    elif kind == "one":
        ids = np.full(M, K - 1)
    elif kind == "none":
        ids = np.full(M, -1)
    elif kind == "outside":
        ids = rs.choice([-1, -7, 0, K - 1, K, K + 5, 2 ** 31 - 1, -2 ** 31], M)
    else:
        ids = rs.randint(-1, K, M)
    return ids.astype(np.int64)


def make(M, m, n, r, K, kind, mixed, seed):
    rs = np.random.RandomState(seed)
    g = torch.Generator().manual_seed(seed)
    t = lambda *s: torch.randn(s, generator=g)
    c = dict(X=t(M, n).to(BF), W=(t(m, n) * n ** -0.5).to(BF), A=(t(K, m, r) * r ** -0.5).to(BF), B=(t(K, r, n) * n ** -0.5).to(BF),
             dY=(t(M, m) * 1e-2).to(BF), scales=torch.rand((K,), generator=g) + 0.5)
    c["ids"] = rows_of(kind, M, K, rs)
    c["ranks"] = rs.randint(0, r + 1, K) if mixed else np.full(K, r)
    return c


def gpu(c):
    o = {k: c[k].cuda() for k in ("X", "W", "A", "B", "dY", "scales")}
    o["row_adapter"] = torch.from_numpy(c["ids"].astype(np.int32)).cuda()
    o["ranks"] = torch.from_numpy(c["ranks"].astype(np.int32)).cuda()
    return o


def reference(c, T=None):
    """fp64: results, and the sums of sizes that the bounds need."""
    X, W, dY = (c[k].double() for k in ("X", "W", "dY"))
    M, n = X.shape
    m, r = c["A"].shape[1:]
    o = dict(T=torch.zeros(M, r).double(), Y=X @ W.T, dX=dY @ W, dA=torch.zeros(c["A"].shape).double(), dB=torch.zeros(c["B"].shape).double())
    b = dict(T=torch.zeros(M, r).double(), Y=(n + r) * E * (X.abs() @ W.abs().T), dX=(m + r) * E * (dY.abs() @ W.abs()),
             dA=torch.zeros(c["A"].shape).double(), dB=torch.zeros(c["B"].shape).double())
    for a in range(c["A"].shape[0]):
        i, k, s = torch.from_numpy(np.flatnonzero(c["ids"] == a)), int(c["ranks"][a]), float(c["scales"][a])
        if len(i) == 0 or k == 0:
            continue
        A, B, x, dy = c["A"][a, :, :k].double(), c["B"][a, :k].double(), X[i], dY[i]
        t, terr = x @ B.T, n * E * (x.abs() @ B.abs().T)
        o["T"][i, :k], b["T"][i, :k] = t, terr
        size = s * t.abs() @ A.abs().T
        o["Y"][i] += s * t @ A.T
        b["Y"][i] += (U + (n + r) * E) * size + s * terr @ A.abs().T * (1 + U)
        used = t if T is None else T[i, :k].double()
        dt, dterr = s * dy @ A, (m + 2) * E * s * (dy.abs() @ A.abs())
        o["dX"][i] += dt @ B
        b["dX"][i] += (U + (m + r) * E) * (dt.abs() @ B.abs()) + dterr @ B.abs() * (1 + U)
        o["dA"][a, :, :k] = s * dy.T @ used
        b["dA"][a, :, :k] = (len(i) + 16) * E * s * (dy.abs().T @ used.abs()) + (s * dy.abs().T @ terr if T is None else 0)
        o["dB"][a, :k] = dt.T @ x
        b["dB"][a, :k] = (len(i) + 16) * E * (dt.abs().T @ x.abs()) + dterr.T @ x.abs()
    for k in ("Y", "dX"):
        b[k] += U * o[k].abs()
    return o, b


def within(got, want, bound, what):
    err = (got.double().cpu() - want).abs()
    over = err - bound * 1.0001 - 1e-38
    assert bool((over <= 0).all()), (what, float(err.max()), float(over.max()), int((over > 0).sum()), np.unravel_index(int(over.argmax()), tuple(over.shape)))


FWD = [  # M, m, n, r, K, rows, mixed ranks: rows around the limits of the kernels and their tiles, widths that end inside one
    (1, 8, 8, 8, 1, "one", False), (1, 768, 768, 8, 4, "any", False), (3, 64, 72, 24, 3, "any", True), (16, 24, 520, 128, 5, "any", True),
    (17, 136, 64, 16, 17, "any", True), (48, 264, 1032, 40, 24, "any", True), (64, 2304, 768, 32, 9, "any", True), (64, 40, 256, 16, 2, "outside", False),
    (65, 72, 136, 16, 3, "any", True), (100, 768, 192, 64, 5, "runs", False), (128, 96, 200, 72, 4, "none", False), (129, 200, 104, 8, 2, "any", True),
    (197, 768, 768, 96, 3, "runs", True), (300, 264, 200, 120, 40, "any", True), (513, 320, 64, 128, 2, "sorted", False), (777, 520, 392, 56, 6, "outside", True),
    (2048, 1000, 72, 16, 7, "runs", True), (4100, 1032, 200, 32, 5, "runs", True), (12500, 1160, 136, 16, 3, "runs", False),
    (12700, 1288, 72, 40, 70, "sorted", True)]


@pytest.mark.parametrize("M,m,n,r,K,rows,mixed", FWD)
def test_forward(M, m, n, r, K, rows, mixed):
    c = make(M, m, n, r, K, rows, mixed, seed=M + m)
    d = gpu(c)
    o, b = reference(c)
    Y, T = abt.lr_adapters_fwd(d["X"], d["W"], d["A"], d["B"], d["row_adapter"], d["ranks"], d["scales"])
    within(T, o["T"], b["T"], "T")
    within(Y, o["Y"], b["Y"], "Y")
    Y1, T1 = abt.lr_adapters_fwd(d["X"], d["W"], d["A"], d["B"], d["row_adapter"], d["ranks"], d["scales"], save_T=False)
    assert T1 is None and torch.equal(Y, Y1)


@pytest.mark.parametrize("M,m,n,r,K,rows,mixed", [
    (1, 8, 16, 8, 1, "one", False), (5, 72, 144, 24, 3, "any", True), (33, 264, 1040, 16, 24, "any", True), (64, 136, 4096, 128, 3, "any", True),
    (65, 72, 144, 16, 3, "any", True), (300, 264, 208, 120, 40, "any", True), (2048, 1000, 80, 16, 7, "runs", True), (12500, 1160, 144, 16, 3, "runs", False)])
def test_forward_from_8_bits(M, m, n, r, K, rows, mixed):
    c = make(M, m, n, r, K, rows, mixed, seed=M + m)
    f8 = torch.float8_e4m3fn
    scale = {k: c[k].float().abs().amax(1) / 448 for k in ("X", "W")}
    q = {k: (c[k].float() / scale[k][:, None]).to(f8) for k in ("X", "W")}
    d = gpu(c)
    Y = abt.lr_adapters_fwd_q8(d["X"], q["X"].cuda(), scale["X"].cuda(), q["W"].cuda(), scale["W"].cuda(), d["A"], d["B"], d["row_adapter"], d["ranks"], d["scales"])
    o, b = reference(c)
    Xd, Wd = (q[k].double() * scale[k].double()[:, None] for k in ("X", "W"))
    X, W = c["X"].double(), c["W"].double()
    want = o["Y"] - X @ W.T + Xd @ Wd.T
    # the dense part of the bound from the 8-bit values (the product of the scales rounds once or twice more)
    bound = b["Y"] - U * o["Y"].abs() - (n + r) * E * (X.abs() @ W.abs().T) + U * want.abs() + (n + r + 4) * E * (Xd.abs() @ Wd.abs().T)
    within(Y, want, bound, "Y")


BWD = [
    (1, 8, 8, 8, 1, "one", False), (2, 72, 136, 16, 3, "any", True), (63, 64, 264, 24, 4, "any", True), (65, 136, 72, 32, 5, "outside", True),
    (130, 200, 128, 40, 3, "none", False), (394, 768, 768, 8, 2, "runs", False), (333, 264, 200, 64, 70, "any", True), (500, 128, 520, 72, 3, "sorted", True),
    (900, 392, 256, 128, 6, "runs", True), (3000, 136, 264, 16, 9, "any", True), (12608, 264, 136, 48, 5, "runs", True), (9000, 8, 16, 104, 2, "sorted", False)]


@pytest.mark.parametrize("M,m,n,r,K,rows,mixed", BWD)
def test_backward(M, m, n, r, K, rows, mixed):
    c = make(M, m, n, r, K, rows, mixed, seed=M + 3 * m)
    d = gpu(c)
    args = (d["W"], d["A"], d["B"], d["row_adapter"], d["ranks"], d["scales"])
    _, T = abt.lr_adapters_fwd(d["X"], *args)
    got = abt.lr_adapters_bwd(d["dY"], d["X"], T, *args)
    o, b = reference(c, T.cpu())
    for g, k in zip(got, ("dX", "dA", "dB")):
        within(g, o[k], b[k], k)
    # the same bits again, each gradient alone too; into what is there
    again = abt.lr_adapters_bwd(d["dY"], d["X"], T, *args)
    assert all(torch.equal(x, y) for x, y in zip(got, again))
    for i, k in enumerate(("need_dX", "need_dA", "need_dB")):
        alone = abt.lr_adapters_bwd(d["dY"], d["X"], T, *args, **{q: q == k for q in ("need_dX", "need_dA", "need_dB")})
        assert torch.equal(alone[i], got[i]) and all(x is None for j, x in enumerate(alone) if j != i)
    dA, dB = torch.ones_like(got[1]), torch.ones_like(got[2])
    abt.lr_adapters_bwd(d["dY"], d["X"], T, *args, dA=dA, dB=dB, accumulate=True)
    assert torch.equal(dA, got[1] + 1) and torch.equal(dB, got[2] + 1)
    # T computed again
    o, b = reference(c)
    within(abt.lr_adapters_bwd(d["dY"], d["X"], None, *args)[1], o["dA"], b["dA"], "dA")


def test_gradients_against_differences():
    """Of the loss sum(dY Y), which is linear in A and in B alone: a difference along a direction is the derivative, in fp64."""
    c = make(200, 40, 48, 16, 3, "any", True, seed=5)
    d = gpu(c)
    args = (d["W"], d["A"], d["B"], d["row_adapter"], d["ranks"], d["scales"])
    _, T = abt.lr_adapters_fwd(d["X"], *args)
    got = dict(zip(("X", "A", "B"), abt.lr_adapters_bwd(d["dY"], d["X"], T, *args)))
    g = torch.Generator().manual_seed(1)
    for k in ("X", "A", "B"):
        D = torch.randn(c[k].shape, generator=g)
        loss = []
        for sign in (1, -1):
            moved = dict(c, **{k: c[k].double() + 0.25 * sign * D.double()})
            loss.append(float((reference(moved)[0]["Y"] * c["dY"].double()).sum()))
        want = (loss[0] - loss[1]) / 0.5
        have = float((got[k].double().cpu() * D.double()).sum())
        _, b = reference(c)
        assert abs(want - have) <= float((b["d" + k] * D.double().abs()).sum()) + 1e-9 * abs(want), k


def test_what_no_row_asks_for_is_not_looked_at():
    """NaN and infinities in adapters without rows, in columns and rows past a rank, and in the rows of others stay where they are."""
    for M in (40, 100, 700):
        c = make(M, 136, 72, 24, 5, "any", False, seed=M)
        c["ids"] = np.where(c["ids"] == 2, 3, c["ids"])
        c["ranks"] = np.array([24, 5, 24, 0, 13])
        dirty = {k: c[k].clone() for k in ("A", "B", "X", "dY", "scales")}
        for a, k in enumerate(c["ranks"]):
            dirty["A"][a, :, k:] = float("nan")
            dirty["B"][a, k:] = float("inf")
        dirty["A"][2], dirty["B"][2], dirty["scales"][2], dirty["scales"][3] = float("nan"), float("-inf"), float("nan"), float("inf")
        d, clean = gpu(dict(c, **dirty)), gpu(c)
        of = lambda s: (s["W"], s["A"], s["B"], s["row_adapter"], s["ranks"], s["scales"])
        Y, T = abt.lr_adapters_fwd(clean["X"], *of(clean))
        want = (Y, T) + abt.lr_adapters_bwd(clean["dY"], clean["X"], T, *of(clean))
        Y, T = abt.lr_adapters_fwd(d["X"], *of(d))
        got = (Y, T) + abt.lr_adapters_bwd(d["dY"], d["X"], T, *of(d))
        for x, y in zip(want, got):
            assert torch.equal(x, y)
        # one row of infinities and NaN: the other rows, and the gradients of adapters that it does not have, are what they were
        row = int(np.flatnonzero(c["ids"] == 4)[0])
        x, dy = c["X"].clone(), c["dY"].clone()
        x[row, 0::2], x[row, 1::2], dy[row, 0::2], dy[row, 1::2] = float("nan"), float("inf"), float("-inf"), float("nan")
        Y, T = abt.lr_adapters_fwd(x.cuda(), *of(clean))
        dX, dA, dB = abt.lr_adapters_bwd(dy.cuda(), x.cuda(), T, *of(clean))
        rest, others = torch.arange(M) != row, [0, 1, 2, 3]
        for p, q in ((Y, want[0]), (T, want[1]), (dX, want[2])):
            assert torch.equal(p[rest.cuda()], q[rest.cuda()])
        assert torch.equal(dA[others], want[3][others]) and torch.equal(dB[others], want[4][others])
        assert not bool(torch.isfinite(Y[row]).any())


def test_offsets_beyond_32_bits():
    """A stack of adapters of more than 2^32 bytes, and rows beyond 2^31 bytes of X."""
    m, n, r = 64, 4096, 128
    K = (1 << 32) // (n * r * 2) + 2
    B = torch.zeros((K, r, n), dtype=BF, device="cuda")
    A = torch.zeros((K, m, r), dtype=BF, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(3)
    B[-1], A[-1] = torch.randn((r, n), generator=g, device="cuda") * n ** -0.5, torch.randn((m, r), generator=g, device="cuda") * r ** -0.5
    M = (1 << 31) // (n * 2) + 500
    X = torch.zeros((M, n), dtype=BF, device="cuda")
    X[-300:] = torch.randn((300, n), generator=g, device="cuda").to(BF)
    dY = torch.zeros((M, m), dtype=BF, device="cuda")
    dY[-300:] = torch.randn((300, m), generator=g, device="cuda").to(BF)
    W = (torch.randn((m, n), generator=g, device="cuda") * n ** -0.5).to(BF)
    ids = torch.full((M,), -1, dtype=torch.int32, device="cuda")
    ids[-300:] = K - 1
    Y, T = abt.lr_adapters_fwd(X, W, A, B, ids)
    dX, dA, dB = abt.lr_adapters_bwd(dY, X, T, W, A, B, ids)
    c = dict(X=X[-300:].cpu(), W=W.cpu(), A=A[-1:].cpu(), B=B[-1:].cpu(), dY=dY[-300:].cpu(), scales=torch.ones(1), ids=np.zeros(300, np.int64), ranks=np.array([r]))
    o, b = reference(c, T[-300:].cpu())
    for got, k in ((Y[-300:], "Y"), (T[-300:], "T"), (dX[-300:], "dX"), (dA[-1:], "dA"), (dB[-1:], "dB")):
        within(got, o[k], b[k], k)
    assert not bool(Y[:-300].any()) and not bool(dA[:-1].any()) and not bool(dB[0].any())


def test_other_stream_and_captured_graph():
    c = make(333, 136, 72, 16, 4, "any", True, seed=9)
    d = gpu(c)
    args = (d["W"], d["A"], d["B"], d["row_adapter"], d["ranks"], d["scales"])
    Y, T = abt.lr_adapters_fwd(d["X"], *args)
    want = (Y, T) + abt.lr_adapters_bwd(d["dY"], d["X"], T, *args)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        Y, T = abt.lr_adapters_fwd(d["X"], *args)
        got = (Y, T) + abt.lr_adapters_bwd(d["dY"], d["X"], T, *args)
    side.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(want, got))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        Y, T = abt.lr_adapters_fwd(d["X"], *args)
        got = (Y, T) + abt.lr_adapters_bwd(d["dY"], d["X"], T, *args)
    for seed in (9, 10, 11):                                 # other rows and other adapters of the rows, without capturing again
        e = gpu(make(333, 136, 72, 16, 4, "any", True, seed=seed))
        for k in ("X", "dY", "row_adapter", "ranks", "scales"):
            d[k].copy_(e[k])
        graph.replay()
        torch.cuda.synchronize()
        eager_Y, eager_T = abt.lr_adapters_fwd(d["X"], *args)
        eager = (eager_Y, eager_T) + abt.lr_adapters_bwd(d["dY"], d["X"], eager_T, *args)
        assert all(torch.equal(x, y) for x, y in zip(eager, got))


def test_refusals():
    c = gpu(make(16, 64, 64, 16, 2, "any", False, seed=0))
    X, W, A, B, ids = (c[k] for k in ("X", "W", "A", "B", "row_adapter"))
    bad = [dict(X=X.float()), dict(W=W.float()), dict(ids=ids.long()), dict(ids=ids[:8].contiguous()), dict(A=A[:, :, :8].contiguous()), dict(B=B[:1].contiguous()),
           dict(X=X[:, :56].contiguous()), dict(X=X.t()), dict(A=A.float()), dict(ids=ids.cpu()), dict(X=X.cpu())]
    for change in bad:
        a = dict(dict(X=X, W=W, A=A, B=B, ids=ids), **change)
        with pytest.raises(abt.AbtError):
            abt.lr_adapters_fwd(a["X"], a["W"], a["A"], a["B"], a["ids"])
        with pytest.raises(abt.AbtError):
            abt.lr_adapters_bwd(c["dY"], a["X"], None, a["W"], a["A"], a["B"], a["ids"])
    with pytest.raises(abt.AbtError):
        abt.lr_adapters_bwd(c["dY"], X, None, W, A, B, ids, accumulate=True)
    with pytest.raises(abt.AbtError):
        abt.lr_adapters_fwd(X, W, A, B, ids, workspace=torch.empty(16, dtype=torch.uint8, device="cuda"))
    with pytest.raises(abt.AbtError):
        abt.lr_adapters_fwd(X, W, A, B, ids, ranks=torch.zeros(3, dtype=torch.int32, device="cuda"))
    one = torch.ones(16, device="cuda")
    with pytest.raises(abt.AbtError):
        abt.lr_adapters_fwd_q8(X, X, one, W, one, A, B, ids)
