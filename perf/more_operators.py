"""Operators of a training step round the pixelfly matrices of a gated block.

  gated      H = act(Zg) o Zu, Zg and Zu both pixelfly projections of one X
             (block-sparse + low-rank + bias), in one kernel
             (pf_linear_gated_fwd).  The two projections are one matrix of 2 N
             rows whose b-row blocks alternate gate, up: [Zg Zu] = X (M o W)^T +
             (X V^T) U^T + bias.  A training program also keeps Z = [Zg Zu].
  gated_bwd  the way back through that product: dZg = dH o Zu o act'(Zg), dZu =
             dH o act(Zg), and dbias = the column sums of dZ
             (pf_linear_gated_bwd).
  norm       layer normalisation of token rows: Y = (X - mean) rstd weight +
             bias; a training program also keeps mean and rstd
             (pf_layernorm_fwd).
  norm_bwd   its gradients dX (with the gradient that went round the
             normalisation added), dweight and dbias (pf_layernorm_bwd).
  clip       the norm over all gradients of a model and the gradients scaled to
             at most a given norm, into the buffer of an optimizer
             (pf_grads_clip).

The ranges that `draw` covers, and that the listed cases stand for:

  gated      256 .. 4096 in-features, 256 .. 16384 features of H, block size 32 /
             64 / 128, maximum stride 1 .. 64, rank 0 .. 256, 1 .. 16384 tokens of
             any count, bf16 and fp32 (fp32 up to 2048 tokens and features); every
             activation, with and without bias and kept Z
  gated_bwd  1 .. 16384 tokens, 256 .. 16384 features, bf16 and fp32, with and
             without bias
  norm       1 .. 16384 tokens, 48 .. 16384 features of any count, rows one after
             the other or taken out of wider ones, bf16 and fp32, with and
             without kept statistics
  norm_bwd   the same, with and without an added gradient
  clip       the gradients of 1 .. 24 blocks of 256 .. 2048 features, 12 tensors
             each from one element to tens of millions, bf16 or fp32 into the
             same type or fp32; norms above and below the limit

Keys of a case:

  gated      dtype T (tokens) K N b ms r act bias pre (Z is kept)
  gated_bwd  dtype T N b act bias
  norm       dtype T N pad (elements between rows) stats
  norm_bwd   dtype T N pad add (a gradient to add)
  clip       dtype out (type of the scaled gradients) layers K N b ms r extra
             (elements of one more tensor) norm (of the gradients, about; the
             limit is 1)
"""
from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False

EPS = 1e-5
LIMIT = 1.0
ACTS = ("none", "gelu", "gelu_tanh", "silu", "relu")


def listed():
    return [
        # Serving: one token through a gated feed-forward's first half; latency.
        dict(name="gated_decode_1024x4096_t1", kind="gated", dtype="bf16", T=1, K=1024, N=4096, b=64,
             ms=16, r=128, act="silu", bias=False, pre=False),
        # A small fp32 block (256 tokens) of a training program.
        dict(name="gated_fp32_768x2048_t256", kind="gated", dtype="fp32", T=256, K=768, N=2048, b=32,
             ms=16, r=32, act="gelu", bias=True, pre=True),
        # Training forward at the smallest block, a ragged micro-batch.
        dict(name="gated_train_1024x4096_b32_t2509", kind="gated", dtype="bf16", T=2509, K=1024, N=4096,
             b=32, ms=16, r=64, act="gelu_tanh", bias=True, pre=True),
        # Training forward of the widest block, full batch: the largest call.
        dict(name="gated_train_4096x16384_b128_t16384", kind="gated", dtype="bf16", T=16384, K=4096,
             N=16384, b=128, ms=32, r=256, act="silu", bias=True, pre=True),
        # The way back of a ragged micro-batch, and of the widest block.
        dict(name="gated_bwd_4096_t2100", kind="gated_bwd", dtype="bf16", T=2100, N=4096, b=32,
             act="gelu", bias=True),
        dict(name="gated_bwd_16384_t16384", kind="gated_bwd", dtype="bf16", T=16384, N=16384, b=128,
             act="silu", bias=True),
        # Serving: one token's normalisation; latency.
        dict(name="norm_1024_t1", kind="norm", dtype="bf16", T=1, N=1024, pad=0, stats=False),
        # Training forward, full batch.
        dict(name="norm_4096_t16384", kind="norm", dtype="bf16", T=16384, N=4096, pad=0, stats=True),
        # Way back of a ragged micro-batch, the residual's gradient added.
        dict(name="norm_bwd_768_t2509", kind="norm_bwd", dtype="bf16", T=2509, N=768, pad=0, add=True),
        # Way back of the full batch.
        dict(name="norm_bwd_4096_t16384", kind="norm_bwd", dtype="bf16", T=16384, N=4096, pad=0,
             add=True),
        # Clipping the gradients of one small fp32 block.
        dict(name="clip_fp32_1x768", kind="clip", dtype="fp32", out="fp32", layers=1, K=768, N=2048, b=32,
             ms=16, r=64, extra=1001, norm=4.0),
        # Clipping all gradients of a 24-block model: 289 tensors, bf16 into fp32
        # for the optimizer.
        dict(name="clip_bf16_24x1536", kind="clip", dtype="bf16", out="fp32", layers=24, K=1536, N=6144,
             b=64, ms=16, r=256, extra=33333333, norm=4.0),
    ]


def _log(rng, lo, hi):
    return math.exp(rng.uniform(math.log(lo), math.log(hi)))


def _tokens(rng, lo, hi):
    t = max(lo, min(hi, int(round(_log(rng, lo, hi)))))
    # Half of the larger counts fill whole tiles (sequence length x batch).
    return t // 128 * 128 if t >= 256 and rng.random() < 0.5 else t


def _width(rng, b, lo, hi):
    return max(2 * b, int(round(_log(rng, lo, hi) / b)) * b)


def _rank(rng, b, K, N):
    most = min(256, K // 2, N // 2) // b
    return b * rng.randint(0, most)


def draw(rng: random.Random):
    kind = rng.choice(["gated", "gated", "gated_bwd", "norm", "norm_bwd", "clip"])
    while True:
        fp32 = rng.random() < 0.25
        b = rng.choice([32, 64, 128])
        c = dict(kind=kind, dtype="fp32" if fp32 else "bf16")
        if kind == "gated":
            c.update(T=_tokens(rng, 1, 2048 if fp32 else 16384),
                     K=_width(rng, b, 256, 2048 if fp32 else 4096),
                     N=_width(rng, b, 256, 2048 if fp32 else 16384), b=b, ms=2 ** rng.randint(0, 6),
                     act=rng.choice(ACTS), bias=rng.random() < 0.6, pre=rng.random() < 0.6)
            c["r"] = _rank(rng, b, c["K"], c["N"])
        elif kind == "gated_bwd":
            c.update(T=_tokens(rng, 1, 16384), N=_width(rng, b, 256, 16384), b=b, act=rng.choice(ACTS),
                     bias=rng.random() < 0.7)
        elif kind == "clip":
            K = _width(rng, b, 256, 2048)
            c.update(out="fp32" if fp32 or rng.random() < 0.5 else "bf16",
                     layers=int(round(_log(rng, 1, 24))), K=K, N=_width(rng, b, K, 4 * K), b=b,
                     ms=2 ** rng.randint(0, 6), extra=int(_log(rng, 1, 3e7)),
                     norm=rng.choice([0.3, 4.0, 50.0]))
            c["r"] = _rank(rng, b, c["K"], c["N"])
        else:
            n = int(round(_log(rng, 48, 16384)))
            # Most widths are those of matrices; the others anything.
            n = n if rng.random() < 0.3 else max(32, n // 32 * 32)
            c.update(T=_tokens(rng, 1, 16384), N=n, pad=rng.choice([0, 0, 0, 64, rng.randint(1, 99)]))
            if kind == "norm":
                c["stats"] = rng.random() < 0.6
            else:
                c["add"] = rng.random() < 0.6
        w = work(c)
        # No dearer than the largest listed case (fp32 runs at a fraction of
        # the bf16 rate).
        if w["flops"] * (16 if fp32 and kind == "gated" else 1) < 1.1e12 and w["bytes"] < 2.6e9:
            return c


# ---- masks and sizes: properties of the case -------------------------------

def _butterfly_mask(nbo, nbi, ms):
    """Flat block butterfly: (i mod s) XOR (j mod s) is 0 or a power of two
    below ms, s the shorter side in blocks."""
    s = min(nbo, nbi)
    x = (np.arange(nbo)[:, None] % s) ^ (np.arange(nbi)[None, :] % s)
    return ((x & (x - 1)) == 0) & (x < ms)


def _kept(c):
    return int(_butterfly_mask(c["N"] // c["b"], c["K"] // c["b"], c["ms"]).sum())


def _sizes(c):
    """Elements of every gradient: per block two normalisations' vectors, the
    gated layer and the layer back (blocks, factors, bias), a position table, a
    mixing weight; then one more tensor.  Odd sizes come last, so that only they
    lie at odd places of a buffer that holds all."""
    K, N, r, w = c["K"], c["N"], c["r"], _kept(c) * c["b"] ** 2
    block = [K, K, 2 * w, 2 * N * r, r * K, 2 * N, w, K * r, r * N, K, 12 * 33, 1]
    return sorted((n for n in block * c["layers"] + [c["extra"]] if n), key=lambda n: n % 64 != 0)


def work(case):
    c = case
    es = 4 if c["dtype"] == "fp32" else 2
    if c["kind"] == "gated":
        T, K, N, r = c["T"], c["K"], c["N"], c["r"]
        nnz = 2 * _kept(c) * c["b"] ** 2
        outs = 1 + 2 * int(c["pre"])
        return {"bytes": es * (T * K + nnz + T * r + r * (2 * N + K) + outs * T * N + 2 * N * c["bias"]),
                "flops": 2.0 * T * (nnz + r * (2 * N + K))}
    if c["kind"] == "gated_bwd":
        return {"bytes": es * c["N"] * (5 * c["T"] + 2 * c["bias"]), "flops": 16.0 * c["T"] * c["N"]}
    if c["kind"] == "norm":
        return {"bytes": es * c["N"] * (2 * c["T"] + 2) + 8 * c["T"] * c["stats"],
                "flops": 8.0 * c["T"] * c["N"]}
    if c["kind"] == "norm_bwd":
        return {"bytes": es * c["N"] * ((3 + c["add"]) * c["T"] + 3) + 8 * c["T"],
                "flops": 14.0 * c["T"] * c["N"]}
    # Every gradient is read for the norm and once more to be scaled.
    n = sum(_sizes(c))
    return {"bytes": n * (2 * es + (4 if c["out"] == "fp32" else 2)) + 4, "flops": 3.0 * n}


# ---- prepare ---------------------------------------------------------------

def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _randn(g, shape, std, dtype):
    return torch.randn(shape, generator=g, device="cuda").mul_(std).to(dtype)


def _type(name):
    return torch.float32 if name == "fp32" else torch.bfloat16


def _empty(shape, dtype):
    return torch.empty(shape, dtype=dtype, device="cuda")


def _gated_inputs(c, seed):
    """Unit-variance activations; weights at the scale of an initialised
    network: unit-variance block-sparse outputs, low-rank ones of half that."""
    g, dt = _gen(seed), _type(c["dtype"])
    T, K, N, b, r = c["T"], c["K"], c["N"], c["b"], c["r"]
    mask = _butterfly_mask(N // b, K // b, c["ms"])
    nnzb = int(mask.sum())
    x = _randn(g, (T, K), 1.0, dt)
    w = _randn(g, (2 * nnzb, b, b), (nnzb / (N // b) * b) ** -0.5, dt)
    u = _randn(g, (2 * N, r), 0.5 * r ** -0.5, dt) if r else None
    v = _randn(g, (r, K), K ** -0.5, dt) if r else None
    bias = _randn(g, (2 * N,), 0.3, dt) if c["bias"] else None
    return mask, x, w, u, v, bias


def _gated_bwd_inputs(c, seed):
    g, dt = _gen(seed), _type(c["dtype"])
    dh = _randn(g, (c["T"], c["N"]), 1.0, dt)
    return dh, _randn(g, (c["T"], 2 * c["N"]), 1.2, dt)


def _rows(c):
    """A T x N view, its rows N + pad elements apart."""
    return _empty((c["T"], c["N"] + c["pad"]), _type(c["dtype"]))[:, : c["N"]]


def _norm_inputs(c, seed):
    """A residual stream: features of different spread and centre."""
    g, dt, N = _gen(seed), _type(c["dtype"]), c["N"]
    x = _rows(c)
    spread = torch.exp(0.5 * torch.randn((N,), generator=g, device="cuda"))
    centre = 0.5 * torch.randn((N,), generator=g, device="cuda")
    x.copy_(torch.randn((c["T"], N), generator=g, device="cuda") * spread + centre)
    weight = (1 + 0.2 * torch.randn((N,), generator=g, device="cuda")).to(dt)
    bias = _randn(g, (N,), 0.2, dt)
    dy = add = None
    if c["kind"] == "norm_bwd":
        dy = _rows(c)
        dy.copy_(torch.randn((c["T"], N), generator=g, device="cuda"))
        if c["add"]:
            add = _rows(c)
            add.copy_(torch.randn((c["T"], N), generator=g, device="cuda"))
    return x, weight, bias, dy, add


def _grads(c, seed):
    """Gradients whose spread differs from tensor to tensor, of about the case's
    norm together."""
    g, dt = _gen(seed), _type(c["dtype"])
    sizes = _sizes(c)
    std = c["norm"] * sum(sizes) ** -0.5
    return [_randn(g, (n,), std * (0.5 + i % 3 / 2), dt) for i, n in enumerate(sizes)]


def prepare(case, seed):
    c = case
    s = {"c": c}
    pf = None
    if own:
        from paper_2112_00029_amd import pixelfly as pf
        s["pf"] = pf
    dt = _type(c["dtype"])
    if c["kind"] == "gated":
        mask, s["x"], s["w"], s["u"], s["v"], s["bias"] = _gated_inputs(c, seed)
        i, j = np.nonzero(np.repeat(mask, 2, axis=0))
        s["blocks"] = 2 * mask.shape[0], mask.shape[1]
        s["ij"] = torch.from_numpy(i).cuda(), torch.from_numpy(j).cuda()
        if own:
            s["L"] = pf.pf_layout_create_gated(c["N"], c["K"], c["b"], c["ms"])
            pf.pf_layout_upload(s["L"])
            s["act"] = getattr(pf, "PF_ACT_" + c["act"].upper())
            s["wsb"] = pf.pf_workspace_bytes(s["L"], c["T"], c["r"], c["dtype"])
            s["h"] = _empty((c["T"], c["N"]), dt)
            s["z"] = _empty((c["T"], 2 * c["N"]), dt) if c["pre"] else None
            s["t"] = _empty((c["T"], c["r"]), dt) if c["r"] else None
    elif c["kind"] == "gated_bwd":
        s["dh"], s["z"] = _gated_bwd_inputs(c, seed)
        if own:
            s["act"] = getattr(pf, "PF_ACT_" + c["act"].upper())
            s["wsb"] = pf.pf_linear_gated_workspace_bytes(c["dtype"], c["T"], c["N"]) if c["bias"] else 0
            s["dz"] = torch.empty_like(s["z"])
            s["db"] = _empty((2 * c["N"],), dt) if c["bias"] else None
    elif c["kind"] == "clip":
        s["g"] = _grads(c, seed)
        if own:
            s["out"] = _empty((sum(_sizes(c)),), _type(c["out"]))
            s["G"] = pf.pf_grads_create(list(zip(s["g"], s["out"].split(_sizes(c)))))
            pf.pf_grads_upload(s["G"])
            s["wsb"] = pf.pf_grads_workspace_bytes(s["G"])
            s["norm"] = _empty((1,), torch.float32)
    else:
        s["x"], s["weight"], s["bias"], s["dy"], s["add"] = _norm_inputs(c, seed)
        if c["kind"] == "norm_bwd":
            # What the forward left: the rows' statistics in fp32.
            s["mean"], s["rstd"] = _stats(s["x"].float())
        if own and c["kind"] == "norm":
            s["y"] = _rows(c)
            s["mean"], s["rstd"] = ((_empty((c["T"],), torch.float32) for _ in range(2)) if c["stats"]
                                    else (None, None))
        elif own:
            s["wsb"] = pf.pf_layernorm_workspace_bytes(c["dtype"], c["T"], c["N"])
            s["dx"] = _rows(c)
            s["dw"], s["db"] = _empty((c["N"],), dt), _empty((c["N"],), dt)
    if own and c["kind"] != "norm":
        s["ws"] = _empty((max(s["wsb"], 256),), torch.uint8)
    return s


# ---- the plain form --------------------------------------------------------

def _act(z, act):
    if act == "gelu":
        return z * (0.5 + 0.5 * torch.erf(z * 0.5 ** 0.5))
    if act == "gelu_tanh":
        return z * (0.5 + 0.5 * torch.tanh((2 / math.pi) ** 0.5 * (z + 0.044715 * z * z * z)))
    if act == "silu":
        return z / (1 + torch.exp(-z))
    if act == "relu":
        return z * (z > 0)
    return z


def _act_slope(z, act):
    if act == "gelu":
        return 0.5 + 0.5 * torch.erf(z * 0.5 ** 0.5) + z * torch.exp(-0.5 * z * z) * (2 * math.pi) ** -0.5
    if act == "gelu_tanh":
        k = (2 / math.pi) ** 0.5
        t = torch.tanh(k * (z + 0.044715 * z * z * z))
        return 0.5 * (1 + t) + 0.5 * z * (1 - t * t) * k * (1 + 3 * 0.044715 * z * z)
    if act == "silu":
        g = 1 / (1 + torch.exp(-z))
        return g + z * g * (1 - g)
    if act == "relu":
        return (z > 0).to(z.dtype)
    return torch.ones_like(z)


def _gated_plain(s):
    c, dt = s["c"], s["x"].dtype
    T, N, b = c["T"], c["N"], c["b"]
    nbo, nbi = s["blocks"]
    w = torch.zeros((nbo, nbi, b, b), device="cuda")
    w[s["ij"]] = s["w"].float()
    w = w.permute(0, 2, 1, 3).reshape(nbo * b, nbi * b)
    x = s["x"].float()
    z = x @ w.t()
    out = {}
    if c["r"]:
        t = x @ s["v"].float().t()
        z += t @ s["u"].float().t()
        out["t"] = t.to(dt)
    if c["bias"]:
        z += s["bias"].float()
    if c["pre"]:
        out["z"] = z.to(dt)
    z = z.view(T, N // b, 2, b)
    out["h"] = (_act(z[:, :, 0], c["act"]) * z[:, :, 1]).reshape(T, N).to(dt)
    return out


def _gated_bwd_plain(s):
    c, dt = s["c"], s["dh"].dtype
    T, N, b = c["T"], c["N"], c["b"]
    z = s["z"].view(T, N // b, 2, b)
    dh = s["dh"].view(T, N // b, b).float()
    zg = z[:, :, 0].float()
    dz = _empty((T, N // b, 2, b), torch.float32)
    dz[:, :, 0] = dh * z[:, :, 1].float() * _act_slope(zg, c["act"])
    dz[:, :, 1] = dh * _act(zg, c["act"])
    dz = dz.view(T, 2 * N)
    out = {"dz": dz.to(dt)}
    if c["bias"]:
        out["db"] = dz.sum(0).to(dt)
    return out


def _stats(x):
    mean = x.mean(-1)
    d = x - mean[:, None]
    return mean, 1 / torch.sqrt((d * d).mean(-1) + EPS)


def _norm_plain(s):
    x = s["x"].float()
    mean, rstd = _stats(x)
    y = (x - mean[:, None]) * rstd[:, None] * s["weight"].float() + s["bias"].float()
    out = {"y": y.to(s["x"].dtype)}
    if s["c"]["stats"]:
        out.update(mean=mean, rstd=rstd)
    return out


def _norm_bwd_plain(s):
    dt = s["x"].dtype
    dy = s["dy"].float()
    xh = (s["x"].float() - s["mean"][:, None]) * s["rstd"][:, None]
    g = dy * s["weight"].float()
    dx = (g - g.mean(-1, keepdim=True) - xh * (g * xh).mean(-1, keepdim=True)) * s["rstd"][:, None]
    if s["add"] is not None:
        dx = dx + s["add"].float()
    return {"dx": dx.to(dt), "dw": (dy * xh).sum(0).to(dt), "db": dy.sum(0).to(dt)}


def _clip_plain(s):
    total = torch.zeros((), dtype=torch.float64, device="cuda")
    for t in s["g"]:
        f = t.float()
        total += (f * f).sum(dtype=torch.float64)
    norm = torch.sqrt(total)
    scale = torch.clamp(LIMIT / norm, max=1.0).float()
    out = _empty((sum(_sizes(s["c"])),), _type(s["c"]["out"]))
    for t, part in zip(s["g"], out.split(_sizes(s["c"]))):
        part.copy_(t.float() * scale)
    return {"norm": norm.float().view(1), "g": out}


# ---- run -------------------------------------------------------------------

def _run_own(s):
    c, pf = s["c"], s["pf"]
    if c["kind"] == "gated":
        pf.pf_linear_gated_fwd(s["L"], c["dtype"], c["T"], c["r"], s["x"], s["w"], s["u"], s["v"],
                               s["bias"], s["act"], s["h"], s["z"], s["t"], s["ws"], s["wsb"])
        return {k: s[k] for k in ("t", "z", "h") if s[k] is not None}
    if c["kind"] == "gated_bwd":
        pf.pf_linear_gated_bwd(c["dtype"], c["T"], c["N"], c["b"], s["act"], s["dh"], s["z"], s["dz"],
                               s["db"], s["ws"], s["wsb"])
        return {k: s[k] for k in ("dz", "db") if s[k] is not None}
    if c["kind"] == "clip":
        pf.pf_grads_clip(s["G"], LIMIT, s["norm"], s["ws"], s["wsb"])
        return {"norm": s["norm"], "g": s["out"]}
    ld = c["N"] + c["pad"]
    if c["kind"] == "norm":
        pf.pf_layernorm_fwd(c["dtype"], c["T"], c["N"], EPS, s["x"], ld, s["weight"], s["bias"], s["y"],
                            ld, s["mean"], s["rstd"])
        return {k: s[k] for k in ("y", "mean", "rstd") if s[k] is not None}
    pf.pf_layernorm_bwd(c["dtype"], c["T"], c["N"], s["dy"], ld, s["x"], ld, s["weight"], s["mean"],
                        s["rstd"], s["add"], ld, s["dx"], ld, s["dw"], s["db"], s["ws"], s["wsb"])
    return {k: s[k] for k in ("dx", "dw", "db")}


def run(state):
    if own:
        return _run_own(state)
    plain = {"gated": _gated_plain, "gated_bwd": _gated_bwd_plain, "norm": _norm_plain,
             "norm_bwd": _norm_bwd_plain, "clip": _clip_plain}
    return plain[state["c"]["kind"]](state)


# ---- exact: from the definitions, in 64 bits -------------------------------

def _phi(z):
    return 0.5 * torch.special.erfc(-z / math.sqrt(2.0))


def _exact_act(z, act):
    if act == "gelu":
        return z * _phi(z)
    if act == "gelu_tanh":
        return z * torch.sigmoid(math.sqrt(8 / math.pi) * (z + 0.044715 * z ** 3))
    if act == "silu":
        return z * torch.sigmoid(z)
    if act == "relu":
        return torch.clamp(z, min=0)
    return z


def _exact_slope(z, act):
    if act == "gelu":
        return _phi(z) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    if act == "gelu_tanh":
        a = math.sqrt(8 / math.pi)
        g = torch.sigmoid(a * (z + 0.044715 * z ** 3))
        return g + z * g * torch.sigmoid(-a * (z + 0.044715 * z ** 3)) * a * (1 + 0.134145 * z ** 2)
    if act == "silu":
        g = torch.sigmoid(z)
        return g * (1 + z * torch.sigmoid(-z))
    if act == "relu":
        return torch.where(z > 0, 1.0, 0.0).to(z.dtype)
    return torch.full_like(z, 1.0)


def _exact_gated(c, seed):
    """Block row by block row of the two projections: the kept blocks of the
    gate's row come before those of the other projection's."""
    mask, x, w, u, v, bias = _gated_inputs(c, seed)
    b = c["b"]
    x = x.double()
    t = torch.matmul(x, v.double().t()) if c["r"] else None
    h = torch.empty((c["T"], c["N"]), dtype=torch.float64, device="cuda")
    z = torch.empty((c["T"], 2 * c["N"]), dtype=torch.float64, device="cuda") if c["pre"] else None
    p = 0
    for i, row in enumerate(mask):
        cols = np.flatnonzero(row)
        xs = torch.cat([x[:, j * b:(j + 1) * b] for j in cols], 1)
        part = []
        for k in (2 * i, 2 * i + 1):
            y = xs @ torch.cat([w[p + n].double() for n in range(len(cols))], 1).t()
            p += len(cols)
            if t is not None:
                y = y + t @ u[k * b:(k + 1) * b].double().t()
            if bias is not None:
                y = y + bias[k * b:(k + 1) * b].double()
            if z is not None:
                z[:, k * b:(k + 1) * b] = y
            part.append(y)
        h[:, i * b:(i + 1) * b] = _exact_act(part[0], c["act"]) * part[1]
    out = {"t": t, "z": z, "h": h}
    return {k: o for k, o in out.items() if o is not None}


def _exact_gated_bwd(c, seed):
    dh, z = _gated_bwd_inputs(c, seed)
    b = c["b"]
    dz = torch.empty(z.shape, dtype=torch.float64, device="cuda")
    for i in range(c["N"] // b):
        g, u = slice(2 * i * b, (2 * i + 1) * b), slice((2 * i + 1) * b, (2 * i + 2) * b)
        d, zg, zu = dh[:, i * b:(i + 1) * b].double(), z[:, g].double(), z[:, u].double()
        dz[:, g] = d * zu * _exact_slope(zg, c["act"])
        dz[:, u] = d * _exact_act(zg, c["act"])
    out = {"dz": dz}
    if c["bias"]:
        out["db"] = dz.sum(0)
    return out


def _exact_norm(c, seed):
    x, weight, bias, _, _ = _norm_inputs(c, seed)
    x = x.double()
    mean = x.sum(-1) / c["N"]
    rstd = torch.rsqrt(x.var(-1, unbiased=False) + EPS)
    y = torch.addcmul(bias.double(), (x - mean[:, None]) * rstd[:, None], weight.double())
    return {"y": y, "mean": mean, "rstd": rstd} if c["stats"] else {"y": y}


def _exact_norm_bwd(c, seed):
    """dX = rstd (I - 11^T / N - n n^T / N) (dY o weight), n the normalised row
    of the statistics the forward left."""
    s = prepare(c, seed)
    r = s["rstd"].double()
    n = (s["x"].double() - s["mean"].double()[:, None]) * r[:, None]
    dy = s["dy"].double()
    q = dy * s["weight"].double()
    a = torch.sum(q, 1) / c["N"]
    k = torch.sum(q * n, 1) / c["N"]
    dx = r[:, None] * (q - torch.addcmul(a[:, None].expand_as(n), n, k[:, None]))
    if c["add"]:
        dx += s["add"].double()
    return {"dx": dx, "dw": torch.sum(dy * n, 0), "db": torch.sum(dy, 0)}


def _exact_clip(c, seed):
    g = _grads(c, seed)
    norm = math.sqrt(math.fsum(float(torch.dot(t.double(), t.double())) for t in g))
    scale = LIMIT / norm if norm > LIMIT else 1.0
    return {"norm": torch.tensor([norm], dtype=torch.float64, device="cuda"),
            "g": torch.cat([t.double() * scale for t in g])}


def exact(case, seed):
    of = {"gated": _exact_gated, "gated_bwd": _exact_gated_bwd, "norm": _exact_norm,
          "norm_bwd": _exact_norm_bwd, "clip": _exact_clip}
    return of[case["kind"]](case, seed)
