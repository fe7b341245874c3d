"""Operators that stand between the products of a model trained layer by layer, as cases that can be measured: the dense layer of
the full-rank phases with bias, activation, dropout and residual in its epilogue (forward and backward), dropout from a counter-based
generator by itself, and the group norm with an activation behind a channels-last convolution (forward and backward).

A case is a dict of plain values; prepare() makes what a program holds before the call, run() makes one call,
work() states the bytes and operations that cannot be avoided and exact() gives the results from the definitions
in 64 bits.  `own` selects what run() computes with: elementary torch operations in 32 bits, or the entry points of
paper_2405_01067_amd.binding.

Kinds, with X [M, n], W [m, n]:
    dense        Z = X W^T + bias,  Y = residual + drop(act(Z))
    dense_bwd    dZ = act'(Z) drop(dY),  dX = dZ W,  dW = dZ^T X,  dbias = sum of the rows of dZ
    dropout      Y = residual + drop(X)
    group        Y = act(gain (X - mean) / sqrt(var + eps) + shift), mean and var over the pixels and the channels of a group of one image
    group_bwd    dX, dgain, dshift

drop(x) = x q / (q - t) with q = 2^16 and t = round(p q) where the element's random 16 bits are t or more, else 0.  The bits of elements
8 b .. 8 b + 7 (of the whole tensor, row by row) are the words of Philox4x32-10 (Salmon et al. 2011) in order, low half first, for the counter
(b, offset + site), both 64 bits, low word first, and the key (seed); seed and offset are given in memory.
"""
import math

import numpy as np
import torch

own = False

_DT = {"bf16": torch.bfloat16, "f32": torch.float32}
_EPS = 1e-5
_SITE = 5


def _dense(kind, M, m, n, act, bias=True, residual=False, p=0.0, keep=False):
    """keep: the sum before the activation is returned too, as the backward wants it."""
    return {"kind": kind, "M": M, "m": m, "n": n, "act": act, "bias": bias, "residual": residual, "p": p, "keep": keep}


def _dropout(dtype, M, n, residual, p):
    return {"kind": "dropout", "dtype": dtype, "M": M, "n": n, "residual": residual, "p": p}


def _group(kind, dtype, N, pixels, C, groups, act):
    return {"kind": kind, "dtype": dtype, "N": N, "pixels": pixels, "C": C, "groups": groups, "act": act}


def listed():
    return [
        # one row through the first layer of a head
        dict(_dense("dense", 1, 768, 768, "gelu"), name="dense, 1 row"),
        # the next tokens of 48 requests through a wide layer, added to the running sum
        dict(_dense("dense", 48, 4096, 4096, "silu", residual=True), name="dense, 48 rows"),
        # seven images of 197 tokens, trained: the sum before the activation is kept
        dict(_dense("dense", 1379, 2304, 768, "gelu", keep=True), name="dense, 1379 rows"),
        # a training batch of 64 images: the second layer of a block, back into the running sum
        dict(_dense("dense", 12608, 768, 2304, "none", residual=True, p=0.1), name="dense, 12608 rows"),
        # long sequences through a wide layer
        dict(_dense("dense", 8190, 4096, 4096, "gelu_tanh"), name="dense, 8190 rows"),
        # two images
        dict(_dense("dense_bwd", 394, 768, 768, "silu"), name="dense bwd, 394 rows"),
        # the training batch: the first layer of a block
        dict(_dense("dense_bwd", 12608, 2304, 768, "gelu"), name="dense bwd, 12608 rows"),
        # behind the embedding of one image
        dict(_dropout("bf16", 197, 768, False, 0.1), name="dropout, 197 rows"),
        # 256 images of 197 tokens, a product's result back into the running sum
        dict(_dropout("bf16", 50432, 768, True, 0.1), name="dropout, 50432 rows"),
        # one image at the last stage of a residual network
        dict(_group("group", "f32", 1, 49, 512, 32, "relu"), name="group norm, 1 image"),
        # 256 images behind a 14 x 14 convolution
        dict(_group("group", "bf16", 256, 196, 256, 32, "silu"), name="group norm, 256 images"),
        # the backward at 28 x 28
        dict(_group("group_bwd", "bf16", 128, 784, 128, 32, "relu"), name="group norm bwd, 128 images"),
    ]


_LARGEST = 8190 * 4096 * 4096


def _log(rng, low, high, step=1):
    v = math.exp(rng.uniform(math.log(low), math.log(high)))
    return max(low, int(v / step) * step)


def draw(rng):
    kind = rng.choice(("dense", "dense", "dense", "dense_bwd", "dense_bwd", "dropout", "group", "group_bwd"))
    p = rng.choice((0.0, 0.1, rng.uniform(0.01, 0.9)))
    if kind in ("dense", "dense_bwd"):
        m, n = _log(rng, 32, 6144, 8), _log(rng, 32, 6144, 8)
        M = _log(rng, 1, 16384) if rng.random() < 0.7 else _log(rng, 1, 128)
        M = max(1, min(M, _LARGEST // (m * n * (2 if kind == "dense_bwd" else 1))))
        act = rng.choice(("none", "relu", "gelu", "gelu", "gelu_tanh", "silu"))
        keep = kind == "dense" and act != "none" and rng.random() < 0.5
        return _dense(kind, M, m, n, act, rng.random() < 0.8, kind == "dense" and rng.random() < 0.5, p, keep)
    dtype = rng.choice(("bf16", "bf16", "f32"))
    if kind == "dropout":
        n = _log(rng, 32, 8192)
        return _dropout(dtype, _log(rng, 1, 50432 * 768 // n), n, rng.random() < 0.7, p or 0.1)
    C = 8 * _log(rng, 4, 256)
    pixels = _log(rng, 1, 4096)
    N = _log(rng, 1, max(1, 256 * 196 * 256 // (pixels * C)))
    divisors = [g for g in range(1, 65) if C % g == 0]
    return _group(kind, dtype, N, pixels, C, rng.choice(divisors), rng.choice(("none", "relu", "gelu", "gelu_tanh", "silu")))


# ------------------------------------------------------------------------------------------ inputs
def _normal(g, shape, std, dtype):
    return (torch.randn(shape, generator=g, device="cuda") * std).to(dtype)


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    kind, bf = case["kind"], torch.bfloat16
    st = {"case": case}
    if kind in ("dense", "dense_bwd"):
        M, m, n = (case[k] for k in ("M", "m", "n"))
        st["X"], st["W"] = _normal(g, (M, n), 1.0, bf), _normal(g, (m, n), n ** -0.5, bf)
        if kind == "dense":
            st["bias"] = _normal(g, (m,), 0.2, torch.float32) if case["bias"] else None
            st["residual"] = _normal(g, (M, m), 2.0, bf) if case["residual"] else None
        else:
            st["dY"] = _normal(g, (M, m), 1e-2, bf)
            st["Z"] = _normal(g, (M, m), 1.0, bf) if case["act"] != "none" else None
    elif kind == "dropout":
        st["X"] = _normal(g, (case["M"], case["n"]), 1.0, _DT[case["dtype"]])
        st["residual"] = _normal(g, (case["M"], case["n"]), 2.0, _DT[case["dtype"]]) if case["residual"] else None
    else:
        N, pixels, C, dt = case["N"], case["pixels"], case["C"], _DT[case["dtype"]]
        st["gain"], st["shift"] = 1 + _normal(g, (C,), 0.1, torch.float32), _normal(g, (C,), 0.2, torch.float32)
        # channels of different means and sizes, as a convolution leaves them
        st["X"] = (torch.randn((N, pixels, C), generator=g, device="cuda") * (0.5 + torch.rand((C,), generator=g, device="cuda"))
                   + torch.randn((C,), generator=g, device="cuda")).to(dt)
        if kind == "group_bwd":
            st["dY"] = _normal(g, (N, pixels, C), 1e-2, dt)
            mean, rstd = _statistics(st["X"].float(), case["groups"])
            st["mean"], st["rstd"] = mean.reshape(N, -1), rstd.reshape(N, -1)
    if case.get("p"):
        st["rng"] = torch.tensor([(seed * 0x9E3779B1 + 7) % (1 << 62), 1000 * (seed % 1000) + (1 << 33)], dtype=torch.int64, device="cuda")
    return st


# ------------------------------------------------------------------------------------------ one call
def run(state):
    return _library(state) if own else _plain(state)


def _library(st):
    from paper_2405_01067_amd import binding as abt
    case = st["case"]
    kind = case["kind"]
    if "rng" in st and "drop" not in st:
        st["drop"] = abt.Dropout(case["p"], st["rng"], site=_SITE)
    drop = st.get("drop")
    if kind == "dense":
        Y, Z = abt.lr_dense_fwd(st["X"], st["W"], st["bias"], act=case["act"], dropout=drop, residual=st["residual"], save_Z=case["keep"])
        return (Y, Z) if case["keep"] else (Y,)
    if kind == "dense_bwd":
        dX, dW, dbias = abt.lr_dense_bwd(st["dY"], st["X"], st["W"], st["Z"], act=case["act"], dropout=drop, need_dbias=case["bias"])
        return (dX, dW, dbias) if case["bias"] else (dX, dW)
    if kind == "dropout":
        return (abt.lr_dropout(st["X"], drop, residual=st["residual"]),)
    if kind == "group":
        return abt.lr_group_norm_fwd(st["X"], st["gain"], st["shift"], case["groups"], eps=_EPS, act=case["act"])
    return abt.lr_group_norm_bwd(st["dY"], st["X"], st["gain"], st["shift"], st["mean"], st["rstd"], act=case["act"])


def _words(seed, counter, blocks):
    """Philox4x32-10 in 64-bit whole numbers: a product's low and high word are its bits 0 .. 31 and 32 .. 63, also where it is taken modulo 2^64."""
    low = 0xFFFFFFFF
    b = torch.arange(blocks, device="cuda")
    c = [b & low, b >> 32, (counter & low).expand_as(b), ((counter >> 32) & low).expand_as(b)]
    k = [seed & low, (seed >> 32) & low]
    for _ in range(10):
        p, q = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57
        c = [((q >> 32) & low) ^ c[1] ^ k[0], q & low, ((p >> 32) & low) ^ c[3] ^ k[1], p & low]
        k = [(k[0] + 0x9E3779B9) & low, (k[1] + 0xBB67AE85) & low]
    return torch.stack(c, 1)


def _kept(st, shape):
    count = math.prod(shape)
    w = _words(st["rng"][0], st["rng"][1] + _SITE, (count + 7) // 8)
    return (torch.stack([w & 0xFFFF, w >> 16], 2).reshape(-1)[:count] >= round(st["case"]["p"] * 65536)).reshape(shape)


def _drop(st, x):
    if "rng" not in st:
        return x
    t = round(st["case"]["p"] * 65536)
    return torch.where(_kept(st, x.shape), x * (65536 / (65536 - t)), 0.0)


def _act(z, act):
    if act == "relu":
        return z.clamp(min=0)
    if act == "gelu":
        return 0.5 * z * (1 + torch.erf(z * 0.5 ** 0.5))
    if act == "gelu_tanh":
        return 0.5 * z * (1 + torch.tanh((2 / math.pi) ** 0.5 * (z + 0.044715 * z ** 3)))
    return z * torch.sigmoid(z) if act == "silu" else z


def _slope(z, act):
    if act == "relu":
        return (z > 0).float()
    if act == "gelu":
        return 0.5 * (1 + torch.erf(z * 0.5 ** 0.5)) + z * torch.exp(-0.5 * z * z) * (2 * math.pi) ** -0.5
    if act == "gelu_tanh":
        c = (2 / math.pi) ** 0.5
        t = torch.tanh(c * (z + 0.044715 * z ** 3))
        return 0.5 * (1 + t) + 0.5 * z * (1 - t * t) * c * (1 + 3 * 0.044715 * z * z)
    if act == "silu":
        s = torch.sigmoid(z)
        return s * (1 + z * (1 - s))
    return torch.ones_like(z)


def _statistics(x, groups):
    N, pixels, C = x.shape
    x = x.reshape(N, pixels, groups, C // groups)
    mean = x.mean((1, 3), keepdim=True)
    return mean, torch.rsqrt((x - mean).square().mean((1, 3), keepdim=True) + _EPS)


def _plain(st):
    case = st["case"]
    kind, bf = case["kind"], torch.bfloat16
    if kind == "dense":
        Z = st["X"].float() @ st["W"].float().t()
        if st["bias"] is not None:
            Z = Z + st["bias"]
        Y = _drop(st, _act(Z, case["act"]))
        if st["residual"] is not None:
            Y = st["residual"].float() + Y
        return (Y.to(bf), Z.to(bf)) if case["keep"] else (Y.to(bf),)
    if kind == "dense_bwd":
        dZ = _drop(st, st["dY"].float())
        if st["Z"] is not None:
            dZ = dZ * _slope(st["Z"].float(), case["act"])
        dX, dW = dZ @ st["W"].float(), dZ.t() @ st["X"].float()
        return (dX.to(bf), dW, dZ.sum(0)) if case["bias"] else (dX.to(bf), dW)
    if kind == "dropout":
        Y = _drop(st, st["X"].float())
        return ((Y if st["residual"] is None else st["residual"].float() + Y).to(st["X"].dtype),)
    X, groups = st["X"].float(), case["groups"]
    N, pixels, C = X.shape
    split = (N, pixels, groups, C // groups)
    if kind == "group":
        mean, rstd = _statistics(X, groups)
        unit = ((X.reshape(split) - mean) * rstd).reshape(X.shape)
        return _act(unit * st["gain"] + st["shift"], case["act"]).to(st["X"].dtype), mean.reshape(N, groups), rstd.reshape(N, groups)
    mean, rstd = (st[k].reshape(N, 1, groups, 1) for k in ("mean", "rstd"))
    unit = (X.reshape(split) - mean) * rstd
    d = st["dY"].float()
    if case["act"] != "none":
        d = d * _slope(unit.reshape(X.shape) * st["gain"] + st["shift"], case["act"])
    u = (d * st["gain"]).reshape(split)
    dX = rstd * (u - u.mean((1, 3), keepdim=True) - unit * (u * unit).mean((1, 3), keepdim=True))
    return dX.reshape(X.shape).to(st["X"].dtype), (d * unit.reshape(X.shape)).sum((0, 1)), d.sum((0, 1))


# ------------------------------------------------------------------------------------------ what it is, and what it needs
def _multipliers(st, shape):
    """What drop() multiplies every element with, in 64 bits: the generator in unsigned whole numbers on the host."""
    if "rng" not in st:
        return 1.0
    count = math.prod(shape)
    seed, offset = (int(v) for v in st["rng"].tolist())
    counter, u, low = (offset + _SITE) % (1 << 64), np.uint64, np.uint64(0xFFFFFFFF)
    x0 = np.arange((count + 7) // 8, dtype=u)
    x1, x0 = x0 >> u(32), x0 & low
    x2, x3 = np.full_like(x0, counter % (1 << 32)), np.full_like(x0, counter >> 32)
    for i in range(10):
        k0, k1 = u((seed + i * 0x9E3779B9) % (1 << 32)), u(((seed >> 32) + i * 0xBB67AE85) % (1 << 32))
        first, second = x0 * u(0xD2511F53), x2 * u(0xCD9E8D57)
        x0, x1, x2, x3 = (second >> u(32)) ^ x1 ^ k0, second & low, (first >> u(32)) ^ x3 ^ k1, first & low
    halves = np.stack([x0, x1, x2, x3], 1).astype("<u4").view("<u2").reshape(-1)[:count]
    t = round(st["case"]["p"] * 65536)
    return torch.from_numpy(np.where(halves >= t, 65536 / (65536 - t), 0.0)).cuda().reshape(shape)


def _value_and_slope(z, act):
    """act and its derivative in 64 bits."""
    if act == "relu":
        return torch.where(z > 0, z, 0.0), torch.where(z > 0, 1.0, 0.0).double()
    if act == "gelu":
        below = torch.erfc(-z / math.sqrt(2)) / 2
        return z * below, below + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    if act == "gelu_tanh":                                   # (1 + tanh a) / 2 = 1 / (1 + exp(-2 a))
        twice = math.sqrt(8 / math.pi) * (z + 0.044715 * z * z * z)
        s = 1 / (1 + torch.exp(-twice))
        return z * s, s + z * s * (1 - s) * math.sqrt(8 / math.pi) * (1 + 0.134145 * z * z)
    if act == "silu":
        s = 1 / (1 + torch.exp(-z))
        return z * s, s + z * s * (1 - s)
    return z, torch.ones_like(z)


def exact(case, seed):
    """The definitions in 64 bits."""
    st = prepare(case, seed)
    kind = case["kind"]
    d = lambda k: st[k].double()
    if kind == "dense":
        Z = torch.mm(d("X"), d("W").t().contiguous())
        if st["bias"] is not None:
            Z += d("bias")
        Y = _value_and_slope(Z, case["act"])[0] * _multipliers(st, Z.shape)
        if st["residual"] is not None:
            Y = Y + d("residual")
        return (Y, Z) if case["keep"] else (Y,)
    if kind == "dense_bwd":
        dZ = d("dY") * _multipliers(st, st["dY"].shape)
        if st["Z"] is not None:
            dZ = dZ * _value_and_slope(d("Z"), case["act"])[1]
        out = torch.mm(dZ, d("W")), torch.mm(dZ.t().contiguous(), d("X"))
        return out + (torch.einsum("ij->j", dZ),) if case["bias"] else out
    if kind == "dropout":
        Y = d("X") * _multipliers(st, st["X"].shape)
        return (Y if st["residual"] is None else Y + d("residual"),)
    N, pixels, C, G = case["N"], case["pixels"], case["C"], case["groups"]
    by_group = lambda t: t.reshape(N, pixels, G, C // G).transpose(1, 2).reshape(N, G, -1)
    back = lambda t: t.reshape(N, G, pixels, C // G).transpose(1, 2).reshape(N, pixels, C)
    x = by_group(d("X"))
    if kind == "group":
        mean = x.sum(2) / x.shape[2]
        rstd = 1 / torch.sqrt(torch.var(x, 2, correction=0) + _EPS)
    else:                                                    # what the forward left
        mean, rstd = d("mean"), d("rstd")
    unit = (x - mean[:, :, None]) * rstd[:, :, None]
    value, slope = _value_and_slope(back(unit) * d("gain") + d("shift"), case["act"])
    if kind == "group":
        return value, mean, rstd
    dpre = d("dY") * slope
    u = by_group(dpre * d("gain"))
    n = x.shape[2]                                           # d(unit) = rstd (I - 1 1^T / n - unit unit^T / n)
    dX = (u - u.sum(2, keepdim=True) / n - unit * ((u * unit).sum(2, keepdim=True) / n)) * rstd[:, :, None]
    return back(dX), torch.einsum("nij,nij->j", dpre, back(unit)), torch.einsum("nij->j", dpre)


def work(case):
    kind = case["kind"]
    if kind in ("dense", "dense_bwd"):
        M, m, n = (case[k] for k in ("M", "m", "n"))
        bias = 4 * m if case["bias"] else 0
        if kind == "dense":
            return {"bytes": 2 * (M * n + m * n + M * m * (1 + case["residual"] + case["keep"])) + bias, "flops": 2 * M * m * n}
        return {"bytes": 2 * (M * m * (2 if case["act"] != "none" else 1) + 2 * M * n + m * n) + 4 * m * n + bias, "flops": 4 * M * m * n}
    e = 2 if case["dtype"] == "bf16" else 4
    if kind == "dropout":
        return {"bytes": e * case["M"] * case["n"] * (3 if case["residual"] else 2), "flops": 2 * case["M"] * case["n"]}
    count = case["N"] * case["pixels"] * case["C"]
    small = 8 * (case["N"] * case["groups"] + case["C"])
    if kind == "group":
        return {"bytes": 2 * e * count + small, "flops": 8 * count}
    return {"bytes": 3 * e * count + 2 * small, "flops": 14 * count}
