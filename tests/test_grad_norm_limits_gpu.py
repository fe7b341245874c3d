"""Clipping where the global norm, or the factor, leaves the range of fp32."""
import pytest
import torch

from paper_2405_01067_amd import binding as abt

pytestmark = pytest.mark.gpu

DTYPES = [torch.float32, torch.bfloat16]


def step_table(grads):
    one = lambda g, dt=torch.float32: torch.ones(g.shape, dtype=dt, device="cuda")
    return [dict(param=one(g), grad=g, exp_avg=one(g), exp_avg_sq=one(g), param_bf16=one(g, torch.bfloat16)) for g in grads]


@pytest.mark.parametrize("dtype", DTYPES)
def test_a_norm_that_is_reported_as_infinite_changes_nothing(dtype):
    """Finite in fp64, not in the fp32 value that the caller gets."""
    g = [torch.full((40,), 3e38, device="cuda").to(dtype), torch.full((7,), -3e38, device="cuda").to(dtype)]
    kept = [t.clone() for t in g]
    assert float(abt.ab_grad_norm(g)) == float("inf")
    out = [torch.zeros_like(t) for t in g]
    assert float(abt.ab_clip_grads(abt.GradPlan(g, out=out), 1.0)) == float("inf")
    assert all(torch.equal(o, k) and torch.equal(t, k) for o, t, k in zip(out, g, kept))
    assert float(abt.ab_clip_grads(g, 1.0)) == float("inf") and all(torch.equal(t, k) for t, k in zip(g, kept))
    if dtype == torch.float32:
        table = step_table(g)
        assert float(abt.ab_adamw_step_clipped(table, max_norm=1.0, step=1, lr=0.1)) == float("inf")
        for t in table:
            assert all(bool((t[k] == 1).all()) for k in ("param", "exp_avg", "exp_avg_sq", "param_bf16"))
