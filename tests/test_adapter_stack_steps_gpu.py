"""AdapterStack.train_step: a step whose gradients are not finite leaves the stack as if it had not been asked for, the count of steps in the bias corrections
of the following ones included."""
import pytest
import torch

from test_adapter_stack_gpu import make, on_gpu

pytestmark = pytest.mark.gpu


# True: a step that can be taken
@pytest.mark.parametrize("steps", [(False, True), (False, False, True, True), (True, False, True), (True, True, False)])
def test_a_refused_step_is_not_counted(steps):
    W, factors, gains, X, ids, ranks, scales, dout = make(96, 7)
    copies = lambda: on_gpu(W, [(a.clone(), b.clone()) for a, b in factors], [g.clone() for g in gains], ranks, scales)
    one, two = copies(), copies()
    x, rows, dout = X.cuda(), ids.int().cuda(), dout.cuda()
    good, bad = lambda out: dout, lambda out: torch.full_like(out, float("inf"))
    for taken in steps:
        norm = one.train_step(x, rows, good if taken else bad, lr=1e-2)
        assert bool(torch.isfinite(norm)) == taken
        if taken:
            two.train_step(x, rows, good, lr=1e-2)
    assert one.steps == two.steps == sum(steps)
    one.steps = 7
    one.train_step(x, rows, bad, lr=1e-2)
    assert one.steps == 7
    for p, q in zip(one.A + one.B + one.gains + one.Ab + one.Bb, two.A + two.B + two.gains + two.Ab + two.Bb):
        assert torch.equal(p, q)
