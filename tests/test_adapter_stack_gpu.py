"""AdapterStack (norm, layers with adapters, gradients, clipped step, 8-bit serving) against the same stack in fp64.

Tolerances, relative to the norm of the result (Frobenius).  Each of the L = 3 blocks rounds to bf16 the running sum, the norm's
output, T, the layer's output and, backwards, dN, dT and the running gradient: at most 2^-8 of the value each, so a result that is
reached through 2 (4 L + 2) of them is off by less than 28 * 2^-8 = 0.11 if all errors line up, and by about
sqrt(28) 2^-8 / sqrt(3) = 0.012 if they do not; the bound for outputs and gradients is 0.03.  8 bits (e4m3: 2^-4 at most, 2^-4 / sqrt(3) on
average, in each operand) add sqrt(2) 0.036 = 0.05 per layer's output, sqrt(3) 0.05 = 0.09 after three: the bound is 0.15."""
import pytest
import torch

from paper_2405_01067_amd import binding as abt
from paper_2405_01067_amd.adapter_stack import AdapterStack

pytestmark = pytest.mark.gpu

L, D, R, K = 3, 256, 16, 5


def make(M, seed):
    g = torch.Generator().manual_seed(seed)
    t = lambda *s: torch.randn(s, generator=g)
    W = [(t(D, D) * D ** -0.5).bfloat16() for _ in range(L)]
    factors = [((t(K, D, R) * R ** -0.5).bfloat16().float(), (t(K, R, D) * D ** -0.5).bfloat16().float()) for _ in range(L)]
    gains = [1 + 0.1 * t(D) for _ in range(L + 1)]
    ids = torch.randint(-1, K, (M,), generator=g)
    ranks = torch.randint(0, R + 1, (K,), generator=g)
    scales = torch.rand((K,), generator=g) + 0.5
    return W, factors, gains, t(M, D).bfloat16(), ids, ranks, scales, (t(M, D) * 1e-2).bfloat16()


def on_gpu(W, factors, gains, ranks, scales):
    return AdapterStack([w.cuda() for w in W], [(a.cuda(), b.cuda()) for a, b in factors], ranks.int().cuda(), scales.cuda(), [g.cuda() for g in gains])


def plain(W, factors, gains, X, ids, ranks, scales):
    """fp64, differentiable in the factors and gains that it returns."""
    A = [a.double().requires_grad_() for a, _ in factors]
    B = [b.double().requires_grad_() for _, b in factors]
    gains = [g.double().requires_grad_() for g in gains]
    mask = (torch.arange(R)[None] < ranks[:, None]).double()
    norm = lambda h, g: h / torch.sqrt((h * h).mean(1, keepdim=True) + 1e-6) * g
    x = X.double().requires_grad_()
    H = x
    has, a = ids >= 0, ids.clamp_min(0)
    for l in range(L):
        N = norm(H, gains[l])
        T = torch.einsum("ird,id->ir", B[l][a], N) * (mask[a] * (scales.double()[a] * has)[:, None])
        H = H + N @ W[l].double().T + torch.einsum("idr,ir->id", A[l][a], T)
    return norm(H, gains[L]), x, A, B, gains


def off(got, want):
    want = want.detach()
    return float((got.detach().double().cpu() - want).norm() / want.norm().clamp_min(1e-30))


@pytest.mark.parametrize("M", [1, 48, 300, 2100])
def test_forward_and_gradients(M):
    W, factors, gains, X, ids, ranks, scales, dout = make(M, M)
    out, x, A, B, g64 = plain(W, factors, gains, X, ids, ranks, scales)
    out.backward(dout.double())
    stack = on_gpu(W, factors, gains, ranks, scales)
    rows = ids.int().cuda()
    got, kept = stack.forward(X.cuda(), rows, keep=True)
    dX = stack.backward(dout.cuda(), kept, rows)
    assert off(got, out) < 0.03 and off(dX, x.grad) < 0.03
    for l in range(L):
        assert off(stack.dA[l], A[l].grad) < 0.03 and off(stack.dB[l], B[l].grad) < 0.03, l
    for l in range(L + 1):
        assert off(stack.dgains[l], g64[l].grad) < 0.03, l
    assert torch.equal(stack.forward(X.cuda(), rows), got)
    stack.freeze()
    assert off(stack.serve(X.cuda(), rows), out) < 0.15


def test_steps_lower_the_loss_and_leave_the_weights():
    W, factors, gains, X, ids, ranks, scales, _ = make(512, 1)
    ranks = torch.full((K,), R)
    stack = on_gpu(W, factors, gains, ranks, scales)
    before = [w.clone() for w in stack.W]
    other = on_gpu(W, [(a + 0.3 * torch.randn(a.shape, generator=torch.Generator().manual_seed(2)), b) for a, b in factors], gains, ranks, scales)
    x, rows = X.cuda(), ids.int().cuda()
    aim = other.forward(x, rows).float()
    losses, norms = [], []

    def loss_grad(out):
        d = out.float() - aim
        losses.append(float((d * d).mean()))
        return (2 * d / d.numel()).bfloat16()

    for _ in range(30):
        norms.append(stack.train_step(x, rows, loss_grad, lr=1e-2, max_norm=1e-3, weight_decay=0.0))
    assert losses[-1] < 0.5 * losses[0], losses
    assert all(float(n) > 0 for n in norms)
    for l in range(L):
        assert torch.equal(stack.W[l], before[l]) and torch.equal(stack.Ab[l], stack.A[l].bfloat16()) and torch.equal(stack.Bb[l], stack.B[l].bfloat16())
    # a step whose gradients are not finite changes nothing
    kept = [t.clone() for t in stack.A + stack.B + stack.gains]
    norm = stack.train_step(x, rows, lambda out: torch.full_like(out, float("inf")), lr=1e-2)
    assert not bool(torch.isfinite(norm)) and all(torch.equal(a, b) for a, b in zip(kept, stack.A + stack.B + stack.gains))


def test_refusals():
    W, factors, gains, X, ids, ranks, scales, _ = make(8, 3)
    cuda = lambda fs: [(a.cuda(), b.cuda()) for a, b in fs]
    with pytest.raises(abt.AbtError):
        AdapterStack([], [])
    with pytest.raises(abt.AbtError):
        AdapterStack([w.cuda() for w in W], cuda(factors[:2]))
    with pytest.raises(abt.AbtError):
        AdapterStack([w.float().cuda() for w in W], cuda(factors))
    with pytest.raises(abt.AbtError):
        AdapterStack([w.cuda() for w in W], [(a.bfloat16(), b.bfloat16()) for a, b in cuda(factors)])
    stack = on_gpu(W, factors, gains, ranks, scales)
    with pytest.raises(abt.AbtError):
        stack.serve(X.cuda(), ids.int().cuda())
    with pytest.raises(abt.AbtError):
        stack.forward(X.cuda(), ids.cuda())
    with pytest.raises(abt.AbtError):
        stack.forward(X[:, :128].contiguous().cuda(), ids.int().cuda())
