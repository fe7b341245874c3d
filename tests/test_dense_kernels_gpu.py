"""Every kernel of the dense layer on whole numbers, whose sums are exact in fp32: a row, a column or a slab that is lost, counted twice or put in another's place shows."""
import pytest

from paper_2405_01067_amd import binding as abt
from kernel_sizes import DENSE_BACKWARD, DENSE_FORWARD
from test_dense_gpu import check_backward, check_forward
from test_dense_gpu import make as random_operands
from test_dense_precision_gpu import test_dW_has_all_of_dZ as dW_has_all_of_dZ
from test_dense_precision_gpu import test_dX_is_rounded_once as dX_is_rounded_once

pytestmark = pytest.mark.gpu


def whole_numbers(*shapes, seed):
    """Up to 3 in size: sums of 9 times 16384 of their products are below 2^24."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    return [torch.randint(-3, 4, s, generator=g, device="cuda").bfloat16() for s in shapes]


def half():
    """Dropout whose factor is 2, and that factor or 0 for every element."""
    import torch
    drop = abt.Dropout(0.5, torch.tensor([3, 1], dtype=torch.int64, device="cuda"), 2)
    return drop, lambda shape: abt.lr_dropout(torch.ones(shape, device="cuda"), drop).double()


def same(got, want, what):
    """`want` in 64 bits, rounded once."""
    off = (got != want.to(got.dtype)).nonzero()
    assert len(off) == 0, (what, len(off), off[0].tolist(), got[tuple(off[0])].item(), want[tuple(off[0])].item())


def off_by(a, b, step, values):
    """Bounds for the sums a^T b [r, c] of whole numbers up to 6 and 3, where every term of `a` has the smallest parts behind it, `values` in all.  A matrix instruction adds 16 products to a
    running sum; whole numbers alone are exact, beside the small parts it may be off by a unit in the last place of the largest number on its way, which is the sum so far (a piece's is the
    difference of two), and 16 products of 18.  So are fewer than 40 sums of partial sums."""
    import torch
    total, most = 0, 0
    for k in range(0, len(a), step):
        total = total + a[k:k + step].t().contiguous().float() @ b[k:k + step].float()
        most = torch.maximum(total.abs(), torch.as_tensor(most, device="cuda"))
    err = (values * len(a) / 16 + 40) * 2.0 ** -23 * (2 * most + 288).double()
    # a number that is lost or in another's place makes a difference of 1 or more to the sums of a row or a column: most of them show it
    assert float((err < 0.5).float().mean()) > 0.75
    return err


def near(got, want, err, what):
    """Between what want - err and want + err are rounded to."""
    off = (~((got >= (want - err).to(got.dtype)) & (got <= (want + err).to(got.dtype)))).nonzero()
    assert len(off) == 0, (what, len(off), off[0].tolist(), got[tuple(off[0])].item(), want[tuple(off[0])].item())


@pytest.mark.parametrize("size,more", [(s, more) for s, more, _, _ in DENSE_FORWARD], ids=str)
def test_forward(size, more):
    import torch
    M, m, n = size
    X, W, R, b = whole_numbers((M, n), (m, n), (M, m), (m,), seed=M + m)
    b = b.float()
    z = X.double() @ W.double().t().contiguous() + b.double()
    if not more:
        same(abt.lr_dense_fwd(X, W, b)[0], z, "Y")
        return
    drop, factors = half()
    Y, Z = abt.lr_dense_fwd(X, W, b, act="relu", dropout=drop, residual=R, save_Z=True)
    same(Z, z, "Z")
    want = R.double() + z.clamp(min=0) * factors((M, m))
    same(Y, want, "Y")
    same(abt.lr_dense_fwd(X, W, b, act="relu", dropout=drop, residual=R)[0], want, "Y without Z")
    same(abt.lr_dense_fwd(X, W, act="relu", save_Z=True)[1], z - b.double(), "Z without a bias")


@pytest.mark.parametrize("size", [s for s, more, _, _ in DENSE_FORWARD if more], ids=str)
def test_forward_of_any_numbers(size):
    check_forward(random_operands(*size, 8), "gelu", 0.1)


@pytest.mark.parametrize("size,values", [(s, values) for s, values, _, _, _ in DENSE_BACKWARD], ids=str)
@pytest.mark.parametrize("p", (None, 0.5))
def test_backward(size, values, p):
    """Without an activation (one value of dZ, and none that is written without dropout), or with slopes that are 0 or 1 (three)."""
    import torch
    M, m, n = size
    dY, X, W, Z = whole_numbers((M, m), (M, n), (m, n), (M, m), seed=M + n)
    drop, factors = half() if p else (None, lambda shape: 1.0)
    on = Z > 0
    Z = torch.where(on, 100.0, -100.0).bfloat16()
    act = "none" if values == 1 else "gelu_tanh"
    dZ = dY.double() * factors((M, m)) * (on if values == 3 else 1)
    dX, dW, db = abt.lr_dense_bwd(dY, X, W, Z if values == 3 else None, act=act, dropout=drop)
    same(db, dZ.sum(0), "dbias")
    want_x, want_w = dZ @ W.double(), dZ.t().contiguous() @ X.double()
    if values == 1:
        same(dX, want_x, "dX")
        same(dW, want_w, "dW")
        return
    near(dX, want_x, off_by(dZ.t(), W, 64, 2), "dX")
    near(dW, want_w, off_by(dZ, X, 32, 3), "dW")


@pytest.mark.parametrize("size", [s for s, values, _, _, _ in DENSE_BACKWARD if values == 1], ids=str)
def test_backward_of_relu(size):
    import torch
    M, m, n = size
    dY, X, W, Z = whole_numbers((M, m), (M, n), (m, n), (M, m), seed=M)
    drop, factors = half()
    dX, dW, db = abt.lr_dense_bwd(dY, X, W, Z, act="relu", dropout=drop)
    dZ = dY.double() * factors((M, m)) * (Z > 0)
    for got, want, what in ((dX, dZ @ W.double(), "dX"), (dW, dZ.t().contiguous() @ X.double(), "dW"), (db, dZ.sum(0), "dbias")):
        same(got, want, what)


@pytest.mark.parametrize("size", [s for s, values, _, _, _ in DENSE_BACKWARD if values == 3], ids=str)
def test_backward_of_any_numbers(size):
    if size[0] < 1000:
        check_backward(random_operands(*size, 9), "gelu", 0.1)
    dX_is_rounded_once(*size, "silu", 0.3)
    dW_has_all_of_dZ(*size, "gelu", 0.1)
