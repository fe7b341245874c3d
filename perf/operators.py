"""Operators around a frozen linear layer that carries low-rank adapters, as cases that can be measured: the
layer itself for rows of many adapters (forward, with 8-bit operands too, and backward), the root-mean-square
norm in front of it (forward and backward), and the clipping of all gradients by their global norm.

A case is a dict of plain values; prepare() makes what a program holds before the call, run() makes one call,
work() states the bytes and operations that cannot be avoided and exact() gives the results from the definitions
in 64 bits.  `own` selects what run() computes with: elementary torch operations in 32 bits, or the entry points of
paper_2405_01067_amd.binding.

Kinds, with X [M, n], W [m, n], adapter a = row_adapter[i] of row i (-1: none), A [K, m, r], B [K, r, n]:
    fwd      T_i = B_a x_i,  Y_i = W x_i + s_a A_a T_i
    fwd_q8   the same, W x_i from 8-bit floats with a scale per row of X and per row of W
    bwd      dT_i = s_a A_a^T dY_i,  dX_i = W^T dY_i + B_a^T dT_i,  dA_a = sum_i s_a dY_i T_i^T,  dB_a = sum_i dT_i x_i^T
    norm     H = X + R,  Y = gain H / sqrt(mean H^2 + eps), optionally also as 8-bit floats with a scale per row
    norm_bwd dX = dH + d(norm)(dY), dgain
    clip     N = sqrt(sum g^2), g' = g min(1, max_norm / N)
    adamw    one AdamW step on the clipped gradients
"""
import math

import numpy as np
import torch

own = False

_DT = {"bf16": torch.bfloat16, "f32": torch.float32}
_F8 = torch.float8_e4m3fn
_F8_MAX = 448.0
_EPS = 1e-6
_ADAM = dict(step=7, lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.01)


def _layer(kind, M, m, n, r, adapters, prompts, mixed=False):
    """prompts: consecutive pieces of the rows, each of one adapter or of none; 0: every row by itself, a token of its own request.
    mixed: adapters of ranks r, r / 2 and r / 4."""
    return {"kind": kind, "M": M, "m": m, "n": n, "r": r, "adapters": adapters, "prompts": prompts, "mixed": mixed}


def _norm(kind, dtype, M, n, residual, q8=False):
    return {"kind": kind, "dtype": dtype, "M": M, "n": n, "residual": residual, "q8": q8}


def _grads(kind, dtype, layers, adapters, r, max_norm=1.0):
    """Gradients of the adapters [adapters, 2304, r], [adapters, r, 768] and the gain [768] of each of `layers` layers, 1e-2 each."""
    return {"kind": kind, "dtype": dtype, "layers": layers, "adapters": adapters, "r": r, "max_norm": max_norm}


def listed():
    return [
        # one new token of one request through the output projection of a ViT-B-sized block
        dict(_layer("fwd", 1, 768, 768, 8, 4, 0), name="fwd, 1 token"),
        # the next tokens of 48 requests, weights in 8 bits, adapters of several ranks
        dict(_layer("fwd_q8", 48, 4096, 4096, 16, 24, 0, True), name="fwd 8 bits, 48 tokens"),
        # seven prompts of different lengths
        dict(_layer("fwd", 1379, 2304, 768, 32, 5, 7, True), name="fwd, 1379 rows"),
        # a training batch, 64 images of 197 tokens, through the qkv projection, eight tasks
        dict(_layer("fwd", 12608, 2304, 768, 16, 8, 64), name="fwd, 12608 rows"),
        # long prompts through a wide layer in 8 bits
        dict(_layer("fwd_q8", 8190, 4096, 4096, 32, 6, 9, True), name="fwd 8 bits, 8190 rows"),
        # two images of two tasks
        dict(_layer("bwd", 394, 768, 768, 8, 2, 2), name="bwd, 394 rows"),
        # the training batch's backward
        dict(_layer("bwd", 12608, 2304, 768, 16, 8, 64), name="bwd, 12608 rows"),
        # the norm in front of the 8-bit layer, 48 tokens
        dict(_norm("norm", "bf16", 48, 4096, True, True), name="norm 8 bits, 48 rows"),
        # 256 images of 197 tokens
        dict(_norm("norm", "bf16", 50432, 768, True), name="norm, 50432 rows"),
        dict(_norm("norm_bwd", "bf16", 12608, 768, True), name="norm bwd, 12608 rows"),
        # one layer's gradients, kept beside the clipped ones
        dict(_grads("clip", "f32", 2, 2, 8), name="clip, 6 tensors"),
        # twelve layers, eight tasks
        dict(_grads("adamw", "f32", 12, 8, 64), name="adamw clipped, 36 tensors"),
    ]


def _log(rng, low, high, step=1):
    v = math.exp(rng.uniform(math.log(low), math.log(high)))
    v = max(low, int(v / step) * step)
    return v + step if v == 3072 else v


def draw(rng):
    kind = rng.choice(("fwd", "fwd", "fwd_q8", "fwd_q8", "bwd", "bwd", "norm", "norm_bwd", "clip", "adamw"))
    if kind in ("fwd", "fwd_q8", "bwd"):
        m, n = _log(rng, 64, 4096, 8), _log(rng, 64, 4096, 16 if kind == "fwd_q8" else 8)
        M = _log(rng, 1, 12608)
        if kind != "bwd" and rng.random() < 0.4:       # single tokens
            M = _log(rng, 1, 128)
            return _layer(kind, M, m, n, 8 * rng.randint(1, 8), rng.randint(1, 64), 0, rng.random() < 0.5)
        r, K = 8 * rng.randint(1, 16 if M > 512 else 8), rng.randint(1, 16)
        M = min(M, int(8190 * (4096 * 4096 + 192 * 8192) / (m * n + K * r * (m + n))))        # no more than the largest listed one
        return _layer(kind, M, m, n, r, K, rng.randint(1, min(M, 64)), rng.random() < 0.5)
    if kind in ("norm", "norm_bwd"):
        dtype = rng.choice(("bf16", "bf16", "f32"))
        n = _log(rng, 64, 8192, 8)
        M = _log(rng, 1, min(50432, 50432 * 768 // n))
        return _norm(kind, dtype, M, n, rng.random() < 0.7, kind == "norm" and rng.random() < 0.4)
    return _grads(kind, "f32" if kind == "adamw" else rng.choice(("f32", "bf16")), rng.randint(1, 12), rng.randint(1, 8), 8 * rng.randint(1, 8),
                  rng.choice((1.0, 1.0, 1000.0)))


# ------------------------------------------------------------------------------------------ inputs
def _normal(g, shape, std, dtype):
    return (torch.randn(shape, generator=g, device="cuda") * std).to(dtype)


def _row_adapters(case, seed):
    """Every tenth request or so has no adapter."""
    rs = np.random.RandomState(seed % (1 << 31))
    M, K, P = case["M"], case["adapters"], case["prompts"]
    pieces = M if P == 0 else P
    of = np.where(rs.rand(pieces) < 0.1, -1, rs.randint(0, K, pieces))
    if P:
        cuts = np.sort(rs.choice(np.arange(1, M), P - 1, replace=False)) if P > 1 else np.zeros(0, np.int64)
        of = np.repeat(of, np.diff(np.concatenate([[0], cuts, [M]])))
    ranks = np.full(K, case["r"])
    if case["mixed"]:
        ranks = rs.choice([case["r"], case["r"] // 2, case["r"] // 4], K)
    return torch.from_numpy(of.astype(np.int32)).cuda(), torch.from_numpy(ranks.astype(np.int32)).cuda()


def _to_8_bits(x):
    """x ~ q scale, one scale per row, the largest value of a row at the largest 8-bit one."""
    scale = x.float().abs().amax(1) / _F8_MAX
    return (x.float() / scale[:, None]).to(_F8), scale


def _spans(case):
    """(first, count) of each tensor in the flat buffers; every tensor starts at a multiple of 16 bytes."""
    K, r, at, spans = case["adapters"], case["r"], 0, []
    for _ in range(case["layers"]):
        for count in (K * 2304 * r, K * r * 768, 768):
            spans.append((at, count))
            at += (count + 7) // 8 * 8
    return spans, at


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    kind, bf = case["kind"], torch.bfloat16
    st = {"case": case}
    if kind in ("fwd", "fwd_q8", "bwd"):
        M, m, n, r, K = (case[k] for k in ("M", "m", "n", "r", "adapters"))
        st["row_adapter"], st["ranks"] = _row_adapters(case, seed)
        st["scales"] = torch.rand((K,), generator=g, device="cuda") + 0.5
        st["A"], st["B"] = _normal(g, (K, m, r), 0.5 * r ** -0.5, bf), _normal(g, (K, r, n), n ** -0.5, bf)
        st["X"], st["W"] = _normal(g, (M, n), 1.0, bf), _normal(g, (m, n), n ** -0.5, bf)
        if kind == "fwd_q8":
            st["Xq"], st["x_scale"] = _to_8_bits(st["X"])
            st["Wq"], st["w_scale"] = _to_8_bits(st.pop("W"))
        if kind == "bwd":
            st["dY"] = _normal(g, (M, m), 1e-2, bf)
            # what the forward keeps: columns past a row's rank and rows without an adapter are zero
            of = st["row_adapter"].long()
            T = torch.randn((M, r), generator=g, device="cuda")
            st["T"] = T * ((of >= 0)[:, None] & (torch.arange(r, device="cuda") < st["ranks"][of.clamp(min=0)][:, None]))
        return st
    if kind in ("norm", "norm_bwd"):
        M, n, dt = case["M"], case["n"], _DT[case["dtype"]]
        st["gain"] = 1 + _normal(g, (n,), 0.1, torch.float32)
        st["X"] = _normal(g, (M, n), 1.0, dt)
        st["R"] = _normal(g, (M, n), 2.0 if kind == "norm" else 1e-2, dt) if case["residual"] else None
        if kind == "norm_bwd":
            st["dY"] = _normal(g, (M, n), 1e-2, dt)
        return st
    spans, total = _spans(case)
    st["spans"], st["max_norm"] = spans, case["max_norm"]
    st["grad"] = torch.zeros(total, dtype=_DT[case["dtype"]], device="cuda")
    for at, count in spans:                                  # the paddings stay zero
        st["grad"][at:at + count] = _normal(g, (count,), 1e-2, torch.float32)
    views = lambda flat: [flat[at:at + count] for at, count in spans]
    st["grads"] = views(st["grad"])
    if kind == "clip":
        st["out"] = torch.zeros_like(st["grad"])
        st["outs"] = views(st["out"])
        return st
    st["param"] = _normal(g, (total,), 0.05, torch.float32)
    st["exp_avg"], st["exp_avg_sq"] = _normal(g, (total,), 1e-3, torch.float32), _normal(g, (total,), 1e-3, torch.float32).square()
    for at, end in zip([a + c for a, c in spans], [a for a, _ in spans[1:]] + [total]):
        for k in ("param", "exp_avg", "exp_avg_sq"):
            st[k][at:end] = 0
    st["param_bf16"] = st["param"].to(bf)
    st["table"] = [dict(param=p, grad=gr, exp_avg=a, exp_avg_sq=b, param_bf16=c) for p, gr, a, b, c in
                   zip(*(views(st[k]) for k in ("param", "grad", "exp_avg", "exp_avg_sq", "param_bf16")))]
    return st


# ------------------------------------------------------------------------------------------ one call
def run(state):
    return _library(state) if own else _plain(state)


def _library(st):
    from paper_2405_01067_amd import binding as abt
    kind = st["case"]["kind"]
    if kind in ("fwd", "fwd_q8", "bwd"):
        of = dict(ranks=st["ranks"], scales=st["scales"])
    if kind == "fwd":
        keep = st["case"]["prompts"] > 0                     # single tokens are not trained on
        Y, T = abt.lr_adapters_fwd(st["X"], st["W"], st["A"], st["B"], st["row_adapter"], save_T=keep, **of)
        return (Y, T) if keep else (Y,)
    if kind == "fwd_q8":
        return (abt.lr_adapters_fwd_q8(st["X"], st["Xq"], st["x_scale"], st["Wq"], st["w_scale"], st["A"], st["B"], st["row_adapter"], **of),)
    if kind == "bwd":
        return abt.lr_adapters_bwd(st["dY"], st["X"], st["T"], st["W"], st["A"], st["B"], st["row_adapter"], **of)
    if kind == "norm":
        Y, H, Yq, y_scale = abt.lr_rms_norm_fwd(st["X"], st["gain"], eps=_EPS, residual=st["R"], quantize=st["case"]["q8"])
        return [t for t in (Y, H if st["R"] is not None else None, Yq, y_scale) if t is not None]
    if kind == "norm_bwd":
        return abt.lr_rms_norm_bwd(st["dY"], st["X"], st["gain"], eps=_EPS, dH=st["R"])
    if kind == "clip":
        if "plan" not in st:                                 # the table of tensors that a training program keeps
            st["plan"] = abt.GradPlan(st["grads"], out=st["outs"])
        return abt.ab_clip_grads(st["plan"], st["max_norm"]), st["out"]
    if "plan" not in st:
        st["plan"] = abt.AdamwPlan(st["table"])
    N = abt.ab_adamw_step_clipped(st["plan"], max_norm=st["max_norm"], **_ADAM)
    return N, st["param"], st["exp_avg"], st["exp_avg_sq"], st["param_bf16"]


def _one_adapter_each(st):
    """[M, K r] truth: which columns of all adapters' T side by side belong to a row."""
    K, r = st["case"]["adapters"], st["case"]["r"]
    of, j = torch.arange(K * r, device="cuda") // r, torch.arange(K * r, device="cuda") % r
    return (st["row_adapter"][:, None] == of) & (j < st["ranks"][of])


def _plain(st):
    case = st["case"]
    kind = case["kind"]
    if kind in ("fwd", "fwd_q8", "bwd"):
        M, m, n, r, K = (case[k] for k in ("M", "m", "n", "r", "adapters"))
        mine = _one_adapter_each(st)
        A = st["A"].float().permute(1, 0, 2).reshape(m, K * r)
        B = st["B"].float().reshape(K * r, n)
        s = st["scales"].repeat_interleave(r)
        X = st["X"].float()
        if kind == "bwd":
            dY = st["dY"].float()
            dT = torch.where(mine, dY @ A * s, 0.0)
            T = torch.where(mine, st["T"].repeat(1, K) * s, 0.0)
            dA = (dY.t() @ T).reshape(m, K, r).permute(1, 0, 2).contiguous()
            dB = (dT.t() @ X).reshape(K, r, n)
            return (dY @ st["W"].float() + dT @ B).to(torch.bfloat16), dA, dB
        T = torch.where(mine, X @ B.t(), 0.0)
        if kind == "fwd":
            base = X @ st["W"].float().t()
        else:
            base = (st["Xq"].float() * st["x_scale"][:, None]) @ (st["Wq"].float() * st["w_scale"][:, None]).t()
        Y = (base + (T * s) @ A.t()).to(torch.bfloat16)
        return (Y, T.reshape(M, K, r).sum(1)) if kind == "fwd" and case["prompts"] > 0 else (Y,)
    if kind == "norm":
        H = st["X"].float() if st["R"] is None else st["X"].float() + st["R"].float()
        Y = H * torch.rsqrt(H.square().mean(1, keepdim=True) + _EPS) * st["gain"]
        out = [Y.to(st["X"].dtype)]
        if st["R"] is not None:
            out.append(H.to(st["X"].dtype))
        if case["q8"]:
            out += list(_to_8_bits(Y))
        return out
    if kind == "norm_bwd":
        H, dY = st["X"].float(), st["dY"].float()
        rs = torch.rsqrt(H.square().mean(1, keepdim=True) + _EPS)
        u = dY * st["gain"]
        dX = rs * u - H * rs ** 3 * (u * H).mean(1, keepdim=True)
        if st["R"] is not None:
            dX = dX + st["R"].float()
        return dX.to(st["X"].dtype), (dY * H * rs).sum(0)
    g = st["grad"].float()
    N = g.square().sum().sqrt()
    g = g * torch.where(N > st["max_norm"], st["max_norm"] / N, 1.0)
    if kind == "clip":
        st["out"].copy_(g)
        return N, st["out"]
    h, p = _ADAM, st["param"]
    st["exp_avg"].mul_(h["beta1"]).add_(g * (1 - h["beta1"]))
    st["exp_avg_sq"].mul_(h["beta2"]).add_(g * g * (1 - h["beta2"]))
    u = st["exp_avg"] / (1 - h["beta1"] ** h["step"]) / ((st["exp_avg_sq"] / (1 - h["beta2"] ** h["step"])).sqrt() + h["eps"])
    p.sub_((u + p * h["weight_decay"]) * h["lr"])
    st["param_bf16"].copy_(p)
    return N, p, st["exp_avg"], st["exp_avg_sq"], st["param_bf16"]


# ------------------------------------------------------------------------------------------ what it is, and what it needs
def exact(case, seed):
    """The definitions in 64 bits, adapter by adapter and tensor by tensor."""
    st = prepare(case, seed)
    kind = case["kind"]
    d = lambda k: st[k].double()
    if kind in ("fwd", "fwd_q8", "bwd"):
        M, m, n, r, K = (case[k] for k in ("M", "m", "n", "r", "adapters"))
        if kind == "fwd_q8":
            first = torch.addcmul(torch.zeros((), device="cuda", dtype=torch.float64), d("Xq"), d("x_scale").view(M, 1)).matmul(
                (d("Wq") * d("w_scale").view(m, 1)).t().contiguous())
        elif kind == "fwd":
            first = torch.mm(d("X"), d("W").t().contiguous())
        else:
            first = torch.mm(d("dY"), d("W"))
        T = torch.zeros((M, r), dtype=torch.float64, device="cuda")
        dA, dB = torch.zeros((K, m, r), dtype=torch.float64, device="cuda"), torch.zeros((K, r, n), dtype=torch.float64, device="cuda")
        for a in range(K):
            rows = torch.nonzero(st["row_adapter"] == a).flatten()
            k = int(st["ranks"][a])
            if rows.numel() == 0 or k == 0:
                continue
            Aa, Ba, s, X = d("A")[a, :, :k].contiguous(), d("B")[a, :k], float(st["scales"][a]), st["X"][rows].double()
            if kind == "bwd":
                dY = st["dY"][rows].double()
                dT = s * torch.mm(dY, Aa)
                first[rows] += torch.mm(dT, Ba)
                dA[a, :, :k] = s * torch.mm(dY.t().contiguous(), st["T"][rows, :k].double())
                dB[a, :k] = torch.mm(dT.t().contiguous(), X)
            else:
                T[rows, :k] = torch.mm(X, Ba.t().contiguous())
                first[rows] += s * torch.mm(T[rows, :k], Aa.t().contiguous())
        if kind == "bwd":
            return first, dA, dB
        return (first, T) if kind == "fwd" and case["prompts"] > 0 else (first,)
    if kind in ("norm", "norm_bwd"):
        n = case["n"]
        H = d("X") if kind == "norm_bwd" or st["R"] is None else d("X") + d("R")
        size = torch.sqrt(torch.einsum("ij,ij->i", H, H) / n + _EPS)[:, None]
        if kind == "norm":
            Y = H / size * d("gain")
            out = [Y] + ([H] if st["R"] is not None else [])
            return out + ([None, Y.abs().max(1).values / _F8_MAX] if case["q8"] else [])
        unit = H / size                                      # d(unit) = (I - unit unit^T / n) / size
        u = d("dY") * d("gain")
        dX = (u - unit * ((unit * u).sum(1, keepdim=True) / n)) / size
        return (dX if st["R"] is None else dX + d("R")), torch.einsum("ij,ij->j", d("dY"), unit)
    g = d("grad")
    N = math.sqrt(sum(float(g[at:at + c].dot(g[at:at + c])) for at, c in st["spans"]))
    if N > st["max_norm"]:
        g = g / (N / st["max_norm"])
    if kind == "clip":
        return torch.tensor(N, dtype=torch.float64), g
    h = _ADAM
    m1 = h["beta1"] * d("exp_avg") + (1 - h["beta1"]) * g
    v1 = h["beta2"] * d("exp_avg_sq") + (1 - h["beta2"]) * g ** 2
    mh, vh = m1 / (1 - h["beta1"] ** h["step"]), v1 / (1 - h["beta2"] ** h["step"])
    p = d("param") - h["lr"] * (mh / (vh ** 0.5 + h["eps"]) + h["weight_decay"] * d("param"))
    return torch.tensor(N, dtype=torch.float64), p, m1, v1, p


def work(case):
    kind = case["kind"]
    if kind in ("fwd", "fwd_q8", "bwd"):
        M, m, n, r = (case[k] for k in ("M", "m", "n", "r"))
        K = min(case["adapters"], M if case["prompts"] == 0 else case["prompts"])     # that rows ask for, at most
        pair = K * r * (m + n)
        if kind == "fwd":
            keep = 4 * M * r if case["prompts"] > 0 else 0
            return {"bytes": 2 * (M * n + m * n + M * m + pair) + keep + 4 * M, "flops": 2 * M * (m * n + r * (m + n))}
        if kind == "fwd_q8":
            return {"bytes": 3 * M * n + m * n + 2 * (M * m + pair) + 4 * (2 * M + m), "flops": 2 * M * (m * n + r * (m + n))}
        return {"bytes": 2 * (M * m + 2 * M * n + m * n + pair) + 4 * (M * r + case["adapters"] * r * (m + n) + M),
                "flops": 2 * M * (m * n + 2 * r * (m + n))}
    if kind in ("norm", "norm_bwd"):
        e, M, n = (2 if case["dtype"] == "bf16" else 4), case["M"], case["n"]
        if kind == "norm":
            return {"bytes": e * M * n * (4 if case["residual"] else 2) + 4 * n + ((n + 4) * M if case["q8"] else 0), "flops": 5 * M * n}
        return {"bytes": e * M * n * (4 if case["residual"] else 3) + 8 * n, "flops": 10 * M * n}
    count = sum(c for _, c in _spans(case)[0])
    e = 2 if case["dtype"] == "bf16" else 4
    if kind == "clip":
        return {"bytes": 2 * e * count, "flops": 3 * count}
    return {"bytes": (4 * 4 + 3 * 4 + 2) * count, "flops": 17 * count}
