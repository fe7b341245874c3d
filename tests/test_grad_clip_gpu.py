"""Clipping by the global norm on the GPU (ab_grad_norm, ab_clip_grads, ab_adamw_step_clipped) against fp64.

Bounds.  The squares are summed in fp64, so the norm is off by its one rounding to fp32 (2^-24, 1.001 of it allowed).  The factor rounds once to fp32
and its product with an fp32 gradient once more: 2^-23 of the value; bf16 adds 2^-8.  The step is ab_adamw_step on fp32 gradients that are the
clipped ones to 2^-23; it is compared with ab_adamw_step on the output of ab_clip_grads, which rounds alike, bit for bit."""
import numpy as np
import pytest
import torch

from paper_2405_01067_amd import binding as abt

pytestmark = pytest.mark.gpu

SETS = {"one": [1], "few": [3, 8, 4, 1, 7], "chunks": [4095, 4096, 4097, 16383, 16384, 16385, 5], "empty": [0, 10, 0], "many": [17 + 3 * i for i in range(300)],
        "large": [3_000_001, 128, 1_000_000], "nothing": [0, 0], "none": []}


def make(counts, dtype, seed, std=1.0):
    g = torch.Generator().manual_seed(seed)
    return [(torch.randn((c,), generator=g) * std).to(dtype) for c in counts]


def norm64(ts):
    return float(np.sqrt(sum(float((t.double() ** 2).sum()) for t in ts)))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("name", sorted(SETS))
def test_norm_and_clip(name, dtype):
    host = make(SETS[name], dtype, seed=len(name))
    dev = [t.cuda() for t in host]
    N = norm64(host)
    got = abt.ab_grad_norm(dev)
    assert got.dtype == torch.float32 and got.shape == () and abs(float(got) - N) <= 1.001 * 2.0 ** -24 * N
    for max_norm in (0.25 * N, N * 2, 0.0):
        out = [torch.full_like(t, 7) for t in dev]
        M = abt.ab_clip_grads(abt.GradPlan(dev, out=out), max_norm)
        assert torch.equal(M, got)
        c = max_norm / N if N > max_norm else 1.0
        for h, d, o in zip(host, dev, out):
            assert torch.equal(d.cpu(), h)                       # the gradients themselves stay
            want = h.double() * c
            u = (2.0 ** -23 if dtype == torch.float32 else 2.0 ** -8 + 2.0 ** -22) if c != 1.0 else 0.0
            assert bool(((o.double().cpu() - want).abs() <= u * want.abs() + 1e-45).all())
        place = [t.clone() for t in dev]
        abt.ab_clip_grads(place, max_norm)
        assert all(torch.equal(p, o) for p, o in zip(place, out))


def test_types_side_by_side():
    a, b = make([5000], torch.float32, 1)[0], make([3001], torch.bfloat16, 2)[0]
    N = norm64([a, b])
    assert abs(float(abt.ab_grad_norm([a.cuda(), b.cuda()])) - N) <= 1.001 * 2.0 ** -24 * N


def test_squares_beyond_the_range_of_fp32():
    for std in (1e30, 1e-30):
        t = make([10000], torch.float32, 3, std)
        N = norm64(t)
        assert abs(float(abt.ab_grad_norm([t[0].cuda()])) - N) <= 1.001 * 2.0 ** -24 * N


@pytest.mark.parametrize("bad", [float("inf"), float("-inf"), float("nan")])
def test_a_norm_that_is_not_finite_changes_nothing(bad):
    host = make([5000, 70], torch.float32, 4)
    host[1][69] = bad
    dev = [t.cuda() for t in host]
    N = abt.ab_clip_grads(dev, 1.0)
    assert not bool(torch.isfinite(N)) and all(torch.equal(torch.nan_to_num(d.cpu()), torch.nan_to_num(h)) for d, h in zip(dev, host))
    table = [dict(param=torch.ones_like(d), grad=d, exp_avg=torch.ones_like(d), exp_avg_sq=torch.ones_like(d), param_bf16=torch.ones_like(d, dtype=torch.bfloat16)) for d in dev]
    N = abt.ab_adamw_step_clipped(table, max_norm=1.0, step=1, lr=0.1)
    assert not bool(torch.isfinite(N))
    for t in table:
        assert all(bool((t[k] == 1).all()) for k in ("param", "exp_avg", "exp_avg_sq", "param_bf16"))


@pytest.mark.parametrize("name", ["one", "few", "chunks", "empty", "many", "large"])
@pytest.mark.parametrize("factor", [0.3, 3.0])
def test_step_on_clipped_gradients(name, factor):
    host = make(SETS[name], torch.float32, seed=8)
    grads = [t.cuda() for t in host]
    max_norm = factor * norm64(host)
    state = lambda: [dict(param=p.cuda(), exp_avg=m.cuda(), exp_avg_sq=v.cuda().square(), param_bf16=torch.zeros(len(p), dtype=torch.bfloat16, device="cuda"))
                     for p, m, v in zip(*(make(SETS[name], torch.float32, seed=s) for s in (11, 12, 13)))]
    hyper = dict(step=5, lr=1e-2, lr_scale=0.5, beta1=0.8, beta2=0.95, eps=1e-7, weight_decay=0.1)
    one, two = state(), state()
    kept = [g.clone() for g in grads]
    N = abt.ab_adamw_step_clipped([dict(t, grad=g) for t, g in zip(one, grads)], max_norm=max_norm, **hyper)
    assert torch.equal(N, abt.ab_grad_norm(grads)) and all(torch.equal(g, k) for g, k in zip(grads, kept))
    abt.ab_clip_grads(grads, max_norm)
    abt.ab_adamw_step([dict(t, grad=g) for t, g in zip(two, grads)], **hyper)
    for x, y in zip(one, two):
        assert all(torch.equal(x[k], y[k]) for k in x)


def test_captured():
    g = make([70000, 33], torch.float32, 5)
    dev = [t.cuda() for t in g]
    plan = abt.GradPlan(dev, out=[torch.empty_like(t) for t in dev])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        N = abt.ab_clip_grads(plan, 2.0)
    for k in range(3):
        dev[0].mul_(0.5)
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in plan.tensors[1]]
        M = abt.ab_clip_grads(plan, 2.0)
        assert torch.equal(M, N) and all(torch.equal(x, y) for x, y in zip(got, plan.tensors[1]))


def test_refusals():
    t = torch.zeros(64, device="cuda")
    for f in (lambda: abt.ab_clip_grads([t], -1.0), lambda: abt.ab_clip_grads([t], float("inf")), lambda: abt.ab_clip_grads([t], float("nan")),
              lambda: abt.ab_grad_norm([t.half()]), lambda: abt.ab_grad_norm([t[::2]]), lambda: abt.ab_grad_norm([t.cpu()]), lambda: abt.ab_grad_norm([t[1:]]),
              lambda: abt.GradPlan([t], out=[]), lambda: abt.GradPlan([t], out=[t.bfloat16()]), lambda: abt.GradPlan([t], out=[t[:32]])):
        with pytest.raises(abt.AbtError):
            f()
    table = [dict(param=t, grad=t, exp_avg=t, exp_avg_sq=t)]
    for kw in (dict(max_norm=-1.0, step=1, lr=0.1), dict(max_norm=float("nan"), step=1, lr=0.1), dict(max_norm=1.0, step=0, lr=0.1)):
        with pytest.raises(abt.AbtError):
            abt.ab_adamw_step_clipped(table, **kw)
