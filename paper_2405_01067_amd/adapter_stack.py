"""A stack of frozen layers with low-rank adapters for several tasks, trained and served through the C ABI of the library.

One block normalises the running sum and adds the layer's output to it,

    N_l = norm(H_l),   Y_l = W_l N_l + scale_a A_a B_a N_l,   H_{l+1} = H_l + Y_l,        out = norm(H_L)

with a frozen W_l [d, d] and, per row, the adapter `a` of the row's task: the pair of factors that a group phase or ab_factorize
leaves for that task.  Rows of any number of tasks lie in one batch.  This module holds control flow only:

    H_{l+1} = H_l + Y_l and its norm             lr_rms_norm_fwd (the sum and the norm in one pass)
    the layer for all tasks                       lr_adapters_fwd, or lr_adapters_fwd_q8 on the 8-bit output of the norm
    gradients                                     lr_adapters_bwd, lr_rms_norm_bwd (the running sum's gradient is added in it)
    step of every factor and gain, clipped        ab_adamw_step_clipped
"""
from typing import Optional, Sequence

from . import binding as abt


class AdapterStack:
    """weights: L frozen bf16 matrices [d, d].  factors: per layer (A [count, d, r], B [count, r, d]), fp32, trained in place;
    ranks (int32) and scales (fp32), both [count], hold for all layers (None: all r, and 1).  gains: L + 1 fp32 vectors [d], trained in place (None: ones)."""

    def __init__(self, weights: Sequence, factors: Sequence, ranks=None, scales=None, gains: Optional[Sequence] = None, eps: float = 1e-6):
        torch = self.torch = abt._torch()
        if not weights or len(factors) != len(weights):
            raise abt.AbtError("one pair of stacked factors per layer, and one layer at least")
        d = weights[0].shape[0]
        for l, (W, (A, B)) in enumerate(zip(weights, factors)):
            if W.dtype != torch.bfloat16 or W.shape != (d, d):
                raise abt.AbtError(f"weight {l} must be a bf16 matrix [{d}, {d}]")
            for t, nm in ((A, "A"), (B, "B")):
                abt._dev_tensor(t, f"{nm}[{l}]")
                if t.dtype != torch.float32:
                    raise abt.AbtError(f"{nm}[{l}] must be fp32: the kernels read its bf16 copy")
        self.W, self.eps, self.ranks, self.scales = list(weights), float(eps), ranks, scales
        self.A, self.B = [a for a, _ in factors], [b for _, b in factors]
        self.gains = list(gains) if gains is not None else [torch.ones(d, device=weights[0].device) for _ in range(len(weights) + 1)]
        if len(self.gains) != len(self.W) + 1:
            raise abt.AbtError("one gain per layer and one behind the last")
        self.Ab, self.Bb = [a.bfloat16() for a in self.A], [b.bfloat16() for b in self.B]
        self.dA, self.dB, self.dgains = ([torch.empty_like(t) for t in ts] for ts in (self.A, self.B, self.gains))
        table = []
        for params, grads, copies in ((self.A, self.dA, self.Ab), (self.B, self.dB, self.Bb), (self.gains, self.dgains, [None] * len(self.gains))):
            table += [dict(param=p, grad=g, exp_avg=torch.zeros_like(p), exp_avg_sq=torch.zeros_like(p), param_bf16=c) for p, g, c in zip(params, grads, copies)]
        self.plan = abt.AdamwPlan(table)
        self._steps, self._asked = 0, None                   # steps known to have been taken, and the one behind them that may have been
        self.W8 = None

    @property
    def steps(self) -> int:
        """The steps that changed the stack (one that goes on from elsewhere sets it).  Waits for the norm of the last one."""
        if self._asked is not None:
            norm, done = self._asked
            done.synchronize()
            self._steps += bool(self.torch.isfinite(norm))
            self._asked = None
        return self._steps

    @steps.setter
    def steps(self, taken: int):
        self._steps, self._asked = int(taken), None

    def forward(self, X, row_adapter, keep: bool = False):
        """The output [M, d] (bf16); with keep, also what `backward` needs."""
        kept = []
        Y, H = X, None
        for l, W in enumerate(self.W):
            N, H, _, _ = abt.lr_rms_norm_fwd(Y, self.gains[l], self.eps, residual=H)
            Y, T = abt.lr_adapters_fwd(N, W, self.Ab[l], self.Bb[l], row_adapter, self.ranks, self.scales, save_T=keep)
            if keep:
                kept.append((H, N, T))
        out, H, _, _ = abt.lr_rms_norm_fwd(Y, self.gains[-1], self.eps, residual=H)
        return (out, (H, kept)) if keep else out

    def backward(self, dout, kept, row_adapter):
        """Fills dA, dB and dgains (self's) and returns the gradient of X."""
        H, layers = kept
        dH, _ = abt.lr_rms_norm_bwd(dout, H, self.gains[-1], self.eps, dgain=self.dgains[-1])
        for l in reversed(range(len(self.W))):
            H, N, T = layers[l]
            dN, _, _ = abt.lr_adapters_bwd(dH, N, T, self.W[l], self.Ab[l], self.Bb[l], row_adapter, self.ranks, self.scales, dA=self.dA[l], dB=self.dB[l])
            dH, _ = abt.lr_rms_norm_bwd(dN, H, self.gains[l], self.eps, dH=dH, dgain=self.dgains[l])
        return dH

    def train_step(self, X, row_adapter, loss_grad, lr: float, max_norm: float = 1.0, **hyper):
        """One step of every factor and gain: loss_grad(out) -> the gradient at the output (bf16).  Returns the gradients' global norm
        before clipping (a 0-d fp32 GPU tensor); a step whose norm is not finite changes nothing, and is not counted in the bias corrections
        of those after it.  So the host waits for the norm of the step before, once this one's gradients are enqueued."""
        out, kept = self.forward(X, row_adapter, keep=True)
        self.backward(loss_grad(out), kept, row_adapter)
        norm = abt.ab_adamw_step_clipped(self.plan, max_norm=max_norm, step=self.steps + 1, lr=lr, **hyper)
        on_host = self.torch.empty((), dtype=norm.dtype, pin_memory=True)
        on_host.copy_(norm, non_blocking=True)
        self._asked = (on_host, self.torch.cuda.Event())
        self._asked[1].record()
        return norm

    def freeze(self):
        """The dense weights once more in 8 bits (e4m3) with a scale per output, for `serve`."""
        torch = self.torch
        self.W8 = []
        for W in self.W:
            scale = W.abs().amax(1).float().clamp_min(1e-30) / 448.0
            self.W8.append(((W.float() / scale[:, None]).to(torch.float8_e4m3fn), scale))

    def serve(self, X, row_adapter):
        """`forward` with the dense products in 8 bits: the norm writes its output in 8 bits beside bf16, which the adapters read."""
        if self.W8 is None:
            raise abt.AbtError("freeze() before serve()")
        Y, H = X, None
        for l, (Wq, w_scale) in enumerate(self.W8):
            N, H, Nq, n_scale = abt.lr_rms_norm_fwd(Y, self.gains[l], self.eps, residual=H, quantize=True)
            Y = abt.lr_adapters_fwd_q8(N, Nq, n_scale, Wq, w_scale, self.Ab[l], self.Bb[l], row_adapter, self.ranks, self.scales)
        return abt.lr_rms_norm_fwd(Y, self.gains[-1], self.eps, residual=H)[0]
