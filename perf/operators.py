"""Operators round the pixelfly matrices of a Transformer block.

  layer      Y = residual + act(X (M o W)^T + (X V^T) U^T + bias): the block-
             sparse + low-rank layer with bias, activation and residual in its
             epilogue (pf_linear_fwd_act).  A training program also keeps the
             pre-activation.
  layer_bwd  the way back through that epilogue: dY_pre = dY o act'(Y_pre) and
             dbias = the column sums of dY_pre (pf_linear_act_bwd).
  attn       block-sparse attention with a learned relative position bias by
             buckets: S = scale Q K^T + table[head][bucket(key - query)] on the
             kept blocks, softmax, O = P V, lse (pf_relpos_bias and
             pf_attn_relpos_fwd); of whole sequences, or of the newest query
             rows of every sequence against all its keys (serving).
  attn_bwd   its gradients dQ, dK, dV and the gradient of the table
             (pf_attn_relpos_bwd).

The ranges that `draw` covers, and that the listed cases stand for:

  layer      as the layer of perf/cases.py: 256 .. 4096 in-features, 256 .. 16384
             out-features, block size 32 / 64 / 128, maximum stride 1 .. 64,
             rank 0 .. 256, 1 .. 16384 tokens of any count, bf16 and fp32 (fp32 up
             to 2048 tokens and features); every activation, with and without
             bias, residual and kept pre-activation
  layer_bwd  1 .. 16384 tokens, 256 .. 16384 columns, bf16 and fp32
  attn       1 .. 4096 tokens of any count, 1 .. 8 sequences of any lengths, 4 .. 16
             query heads of 64 on as many or fewer key/value heads, maximum
             stride 1 .. 64 blocks or every block kept, 0 .. 2 global blocks,
             logarithmic or clipped-distance buckets (8 .. 129), causal or not,
             head-major or token-major tensors; serving: 1 .. 64 sequences, the
             newest 1 .. 200 rows of each
  attn_bwd   as the whole sequences of attn, 16 .. 4096 tokens

A case is a dict of plain values.  Keys by kind:
  layer      dtype T K N b ms r act bias res pre
  layer_bwd  dtype T N act
  attn       B H Hkv S ms (0: every block) glob map buckets reach causal lens
             (ragged lengths) tm (token-major tensors) rows (newest query rows;
             0: all)
  attn_bwd   the same, rows 0

Buckets come from integer arithmetic; a pair that the causal map leaves out
has bucket -1.
"""
from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False

D = 64
BLK = 64
ACTS = ("none", "gelu", "gelu_tanh", "silu", "relu")


def listed():
    return [
        # Serving: one token through the first layer of an MLP (bias, GELU);
        # two small launches, latency.
        dict(name="layer_decode_1024x4096_t1", kind="layer", dtype="bf16", T=1, K=1024, N=4096, b=64,
             ms=16, r=128, act="gelu", bias=True, res=False, pre=False),
        # Serving: the MLP's second layer for eight sequences, added to the
        # residual stream.
        dict(name="layer_decode_4096x1024_t8", kind="layer", dtype="bf16", T=8, K=4096, N=1024, b=64,
             ms=16, r=128, act="none", bias=True, res=True, pre=False),
        # A small fp32 layer (256 tokens, 1024 square) of a training program.
        dict(name="layer_fp32_1024_t256", kind="layer", dtype="fp32", T=256, K=1024, N=1024, b=32,
             ms=32, r=32, act="silu", bias=True, res=True, pre=True),
        # Training forward of an MLP's second layer with the residual, one
        # batch of 8192 tokens.
        dict(name="layer_train_4096x1024_t8192", kind="layer", dtype="bf16", T=8192, K=4096, N=1024,
             b=64, ms=16, r=128, act="none", bias=True, res=True, pre=False),
        # Training forward of the widest layer at the smallest block, a ragged
        # micro-batch.
        dict(name="layer_train_4096x16384_b32_t2509", kind="layer", dtype="bf16", T=2509, K=4096,
             N=16384, b=32, ms=32, r=256, act="gelu_tanh", bias=True, res=False, pre=True),
        # Training forward of the widest layer, full batch: the largest call.
        dict(name="layer_train_4096x16384_b128_t16384", kind="layer", dtype="bf16", T=16384, K=4096,
             N=16384, b=128, ms=32, r=256, act="gelu", bias=True, res=False, pre=True),
        # The way back through a small layer's epilogue (ragged tokens), and
        # through the widest layer's.
        dict(name="layer_bwd_4096_t2100", kind="layer_bwd", dtype="bf16", T=2100, N=4096, act="silu"),
        dict(name="layer_bwd_16384_t16384", kind="layer_bwd", dtype="bf16", T=16384, N=16384,
             act="gelu"),
        # Serving: 16 sequences decode one token each against caches of up to
        # 4096 tokens, every block kept, four query heads on each key/value head.
        dict(name="attn_decode_16x16x4096", kind="attn", B=16, H=16, Hkv=4, S=4096, ms=0, glob=0,
             map="log", buckets=32, reach=128, causal=True, lens=True, tm=True, rows=1),
        # Training forward, batch 8, 12 heads, 4096 tokens, butterfly mask,
        # buckets as an encoder has them.
        dict(name="attn_train_8x12x4096", kind="attn", B=8, H=12, Hkv=12, S=4096, ms=64, glob=0,
             map="log", buckets=32, reach=128, causal=False, lens=False, tm=False, rows=0),
        # Backward of the same.
        dict(name="attn_bwd_8x12x4096", kind="attn_bwd", B=8, H=12, Hkv=12, S=4096, ms=64, glob=0,
             map="log", buckets=32, reach=128, causal=False, lens=False, tm=False, rows=0),
        # Backward of a padded causal batch of an odd length, grouped heads,
        # one bucket per distance up to 64, a global stripe.
        dict(name="attn_bwd_4x16x1511", kind="attn_bwd", B=4, H=16, Hkv=4, S=1511, ms=32, glob=1,
             map="clip", buckets=129, reach=64, causal=True, lens=True, tm=True, rows=0),
    ]


def _log(rng, lo, hi):
    return math.exp(rng.uniform(math.log(lo), math.log(hi)))


def _tokens(rng, lo, hi):
    t = max(lo, min(hi, int(round(_log(rng, lo, hi)))))
    # Half of the larger counts fill whole tiles (sequence length x batch).
    return t // 128 * 128 if t >= 256 and rng.random() < 0.5 else t


def _width(rng, b, lo, hi):
    return max(2 * b, int(round(_log(rng, lo, hi) / b)) * b)


def draw(rng: random.Random):
    kind = rng.choice(["layer", "layer", "layer_bwd", "attn", "attn", "attn_bwd"])
    while True:
        fp32 = rng.random() < 0.25
        dtype = "fp32" if fp32 else "bf16"
        if kind == "layer":
            b = rng.choice([32, 64, 128])
            c = dict(kind=kind, dtype=dtype, T=_tokens(rng, 1, 2048 if fp32 else 16384),
                     K=_width(rng, b, 256, 2048 if fp32 else 4096),
                     N=_width(rng, b, 256, 2048 if fp32 else 16384), b=b, ms=2 ** rng.randint(0, 6),
                     r=0, act=rng.choice(ACTS), bias=rng.random() < 0.8, res=rng.random() < 0.5,
                     pre=False)
            rmax = min(256, c["K"] // 2, c["N"] // 2) // b
            c["r"] = b * rng.randint(0, rmax) if rmax else 0
            c["pre"] = c["act"] != "none" and rng.random() < 0.6
        elif kind == "layer_bwd":
            c = dict(kind=kind, dtype=dtype, T=_tokens(rng, 1, 16384), N=_width(rng, 32, 256, 16384),
                     act=rng.choice(ACTS))
        else:
            H = rng.choice([4, 8, 12, 16])
            m = rng.choice(["log", "clip"])
            c = dict(kind=kind, B=rng.randint(1, 8), H=H, Hkv=H // rng.choice([1, 1, 2, 4]),
                     S=_tokens(rng, 1 if kind == "attn" else 16, 4096), ms=2 ** rng.randint(0, 6),
                     glob=rng.choice([0, 0, 1, 2]), map=m, buckets=2 * rng.randint(4, 24),
                     reach=2 ** rng.randint(6, 9), causal=rng.random() < 0.5, lens=rng.random() < 0.5,
                     tm=rng.random() < 0.5, rows=0)
            if rng.random() < 0.25:
                c["ms"] = 0
            if m == "clip":
                c["reach"] = rng.randint(4, 64)
                c["buckets"] = 2 * c["reach"] + 1
            if kind == "attn" and rng.random() < 0.5:
                c["B"] = int(round(_log(rng, 1, 64)))
                c["rows"] = min(c["S"], 1 if rng.random() < 0.6 else int(round(_log(rng, 2, 200))))
            c["glob"] = min(c["glob"], _blocks(c["S"]))
        w = work(c)
        # No dearer than the largest listed case (fp32 runs at a fraction of
        # the bf16 rate).
        if w["flops"] * (16 if c.get("dtype") == "fp32" else 1) < 5.0e11 and w["bytes"] < 1.6e9:
            return c


# ---- masks, buckets, lengths: properties of the case -----------------------

def _blocks(s):
    return (s + BLK - 1) // BLK


def _butterfly_mask(nbo, nbi, ms):
    """Flat block butterfly: (i mod s) XOR (j mod s) is 0 or a power of two
    below ms, s the shorter side in blocks."""
    s = min(nbo, nbi)
    x = (np.arange(nbo)[:, None] % s) ^ (np.arange(nbi)[None, :] % s)
    return ((x & (x - 1)) == 0) & (x < ms)


def _attn_mask(c):
    nb = _blocks(c["S"])
    if c["ms"] == 0:
        return np.ones((nb, nb), dtype=bool)
    m = _butterfly_mask(nb, nb, c["ms"])
    m[:c["glob"]] = True
    m[:, :c["glob"]] = True
    return m


def _log_steps(n, reach):
    """Smallest distances of the buckets 1 .. n - 1 of one direction: the first
    half one distance each, then d enters bucket e + k (e = n // 2) as soon as
    (d / e)^(n - e) >= (reach / e)^k; in integers."""
    e = n // 2
    steps = list(range(1, e + 1))
    for k in range(1, n - e):
        d = steps[-1]
        while d ** (n - e) < reach ** k * e ** (n - e - k):
            d += 1
        steps.append(d)
    return np.array(steps[: n - 1], dtype=np.int64)


def _bucket_map(c):
    """Bucket of the distance key - query = -(side - 1) .. side - 1, side the
    sequence in whole blocks; -1 where the pair is left out."""
    side = _blocks(c["S"]) * BLK
    d = np.arange(-(side - 1), side)
    if c["map"] == "clip":
        b = np.clip(d, -c["reach"], c["reach"]) + c["reach"]
    elif c["causal"]:
        b = np.searchsorted(_log_steps(c["buckets"], c["reach"]), -d, side="right")
    else:
        half = c["buckets"] // 2
        b = np.searchsorted(_log_steps(half, c["reach"]), np.abs(d), side="right")
        b = b + half * (d > 0)
    if c["causal"]:
        b = np.where(d > 0, -1, b)
    return b.astype(np.int32)


def _lengths(c):
    """Tokens of each sequence: ragged ones spread over 1 .. S, the longest S."""
    if not c["lens"]:
        return [c["S"]] * c["B"]
    g = random.Random(c["B"] * 8191 + c["S"])
    return [c["S"]] + [g.randint((c["S"] + 3) // 4, c["S"]) for _ in range(c["B"] - 1)]


def _rows(c):
    return c["rows"] or c["S"]


def _starts(c):
    """Position of each sequence's first query row (its newest `rows` rows)."""
    return [max(0, n - c["rows"]) if c["rows"] else 0 for n in _lengths(c)]


# ---- work ------------------------------------------------------------------

def _pairs(c):
    """Attended (query, key) pairs of one head, all sequences."""
    kept = _attn_mask(c)
    nb = kept.shape[0]
    total = 0.0
    for n, st in zip(_lengths(c), _starts(c)):
        pos = np.arange(nb) * BLK
        q = np.clip(np.minimum(n, st + _rows(c)) - pos, 0, BLK) - np.clip(st - pos, 0, BLK)
        k = np.clip(n - pos, 0, BLK)
        cell = np.outer(np.maximum(q, 0), k) * kept
        if c["causal"]:
            cell = np.tril(cell, -1) + np.diag(np.diag(cell)) * 0.5
        total += float(cell.sum())
    return total


def work(case):
    c = case
    if c["kind"] == "layer":
        es = 4 if c["dtype"] == "fp32" else 2
        T, K, N, r = c["T"], c["K"], c["N"], c["r"]
        nnz = int(_butterfly_mask(N // c["b"], K // c["b"], c["ms"]).sum()) * c["b"] ** 2
        outs = 1 + int(c["pre"]) + int(c["res"])
        return {"bytes": es * (T * K + nnz + T * r + r * (N + K) + outs * T * N + N * c["bias"]),
                "flops": 2.0 * T * (nnz + r * (N + K))}
    if c["kind"] == "layer_bwd":
        es = 4 if c["dtype"] == "fp32" else 2
        n = 1 if c["act"] == "none" else 3
        return {"bytes": es * c["N"] * (n * c["T"] + 1), "flops": float(c["T"] * c["N"] * (1 + 10 * (n > 1)))}
    pairs = _pairs(c) * c["H"]
    q = sum(min(_rows(c), n) for n in _lengths(c)) * c["H"] * D * 2
    if c["rows"] and c["ms"]:
        # The key blocks that the query rows' block rows keep.
        kept, nb, k = _attn_mask(c), _blocks(c["S"]), 0
        for n, st in zip(_lengths(c), _starts(c)):
            rows = range(st // BLK, min(nb - 1, (max(n, st + 1) - 1) // BLK) + 1)
            cols = np.any([kept[i] for i in rows], axis=0)
            k += int((cols * np.clip(n - np.arange(nb) * BLK, 0, BLK)).sum())
    else:
        k = sum(_lengths(c))
    k *= c["Hkv"] * D * 2
    lse = q // (D * 2) * 4
    if c["kind"] == "attn":
        return {"bytes": 2 * q + 2 * k + lse, "flops": 4.0 * D * pairs}
    # Q, O, dO, dQ; K, V, dK, dV; five products.
    return {"bytes": 4 * q + 4 * k + lse + 8 * c["H"] * c["buckets"], "flops": 10.0 * D * pairs}


# ---- prepare ---------------------------------------------------------------

def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _randn(g, shape, std, dtype):
    return torch.randn(shape, generator=g, device="cuda").mul_(std).to(dtype)


def _dtype(c):
    return torch.float32 if c.get("dtype") == "fp32" else torch.bfloat16


def _empty(shape, dtype):
    return torch.empty(shape, dtype=dtype, device="cuda")


def _layer_inputs(c, seed):
    """Unit-variance activations; weights at the scale of an initialised
    network: unit-variance block-sparse outputs, low-rank ones of half that."""
    g, dt = _gen(seed), _dtype(c)
    T, K, N, b, r = c["T"], c["K"], c["N"], c["b"], c["r"]
    mask = _butterfly_mask(N // b, K // b, c["ms"])
    nnzb = int(mask.sum())
    fan = nnzb / (N // b) * b
    x = _randn(g, (T, K), 1.0, dt)
    w = _randn(g, (nnzb, b, b), fan ** -0.5, dt)
    u = _randn(g, (N, r), 0.5 * r ** -0.5, dt) if r else None
    v = _randn(g, (r, K), K ** -0.5, dt) if r else None
    bias = _randn(g, (N,), 0.3, dt) if c["bias"] else None
    res = _randn(g, (T, N), 1.0, dt) if c["res"] else None
    return mask, x, w, u, v, bias, res


def _attn_tensor(c, heads, s):
    """[B][heads][s][64], head-major or (tm) a view of [B][s][heads][64]."""
    if c["tm"]:
        return _empty((c["B"], s, heads, D), torch.bfloat16).transpose(1, 2)
    return _empty((c["B"], heads, s, D), torch.bfloat16)


def _attn_inputs(c, seed):
    g = _gen(seed)
    R, S = _rows(c), c["S"]
    q, k, v = _attn_tensor(c, c["H"], R), _attn_tensor(c, c["Hkv"], S), _attn_tensor(c, c["Hkv"], S)
    for t in (q, k, v):
        t.copy_(torch.randn(t.shape, generator=g, device="cuda"))
    table = torch.randn((c["H"], c["buckets"]), generator=g, device="cuda")
    do = None
    if c["kind"] == "attn_bwd":
        do = _attn_tensor(c, c["H"], R)
        do.copy_(torch.randn(do.shape, generator=g, device="cuda"))
    return q, k, v, table, do


def prepare(case, seed):
    c = case
    s = {"c": c}
    if c["kind"] == "layer":
        mask, s["x"], s["w"], s["u"], s["v"], s["bias"], s["res"] = _layer_inputs(c, seed)
        i, j = np.nonzero(mask)
        s["mask"] = mask.shape
        s["ij"] = torch.from_numpy(i).cuda(), torch.from_numpy(j).cuda()
        if own:
            from paper_2112_00029_amd import pixelfly as pf
            dt = s["x"].dtype
            s["pf"] = pf
            s["L"] = pf.pf_layout_create(c["N"], c["K"], c["b"], c["ms"])
            pf.pf_layout_upload(s["L"])
            s["act"] = getattr(pf, "PF_ACT_" + c["act"].upper())
            s["wsb"] = pf.pf_workspace_bytes(s["L"], c["T"], c["r"], c["dtype"])
            s["ws"] = _empty((max(s["wsb"], 256),), torch.uint8)
            s["y"] = _empty((c["T"], c["N"]), dt)
            s["ypre"] = torch.empty_like(s["y"]) if c["pre"] else None
            s["t"] = _empty((c["T"], c["r"]), dt) if c["r"] else None
        return s
    if c["kind"] == "layer_bwd":
        g, dt = _gen(seed), _dtype(c)
        s["dy"] = _randn(g, (c["T"], c["N"]), 1.0, dt)
        s["ypre"] = _randn(g, (c["T"], c["N"]), 1.2, dt) if c["act"] != "none" else None
        if own:
            from paper_2112_00029_amd import pixelfly as pf
            s["pf"] = pf
            s["act"] = getattr(pf, "PF_ACT_" + c["act"].upper())
            s["wsb"] = pf.pf_linear_act_workspace_bytes(c["dtype"], c["T"], c["N"])
            s["ws"] = _empty((max(s["wsb"], 256),), torch.uint8)
            s["dpre"] = torch.empty_like(s["dy"]) if c["act"] != "none" else None
            s["db"] = _empty((c["N"],), dt)
        return s
    s["q"], s["k"], s["v"], s["table"], s["do"] = _attn_inputs(c, seed)
    s["kept"] = torch.from_numpy(_attn_mask(c)).cuda()
    s["map"] = torch.from_numpy(_bucket_map(c)).cuda()
    s["len"] = torch.tensor(_lengths(c), dtype=torch.int32, device="cuda")
    s["start"] = torch.tensor(_starts(c), dtype=torch.int32, device="cuda")
    shape = (c["B"], c["H"], _rows(c))
    if c["kind"] == "attn_bwd":
        # What the forward left: its output in bf16 and the rows' log-sums.
        o, s["lse"] = _attn_plain(s)
        s["o"] = _attn_tensor(c, c["H"], _rows(c))
        s["o"].copy_(o)
    if own:
        from paper_2112_00029_amd import pixelfly as pf
        s["pf"] = pf
        side = _blocks(c["S"]) * BLK
        if c["ms"] == 0:
            s["L"] = pf.pf_layout_create_from_mask(side // BLK, side // BLK, BLK, _attn_mask(c))
        else:
            s["L"] = pf.pf_layout_create_attention(side, BLK, c["ms"], c["glob"])
        pf.pf_layout_upload(s["L"])
        if c["map"] == "log":
            s["R"] = pf.pf_relpos_create_log(side, c["buckets"], c["reach"], not c["causal"])
        else:
            s["R"] = pf.pf_relpos_create(side, c["buckets"], _bucket_map(c))
        pf.pf_relpos_upload(s["R"])
        s["bias"] = _empty((c["H"], pf.pf_relpos_bias_floats(s["R"])), torch.float32)
        s["wsb"] = pf.pf_attn_relpos_workspace_bytes(s["L"], s["R"], c["B"], c["H"], _rows(c))
        s["ws"] = _empty((max(s["wsb"], 256),), torch.uint8)
        if c["rows"] or c["kind"] == "attn_bwd":
            # Serving: the table does not change between calls.  Backward: the
            # forward has laid it out.
            pf.pf_relpos_bias(s["R"], c["H"], s["table"], s["bias"])
        if c["kind"] == "attn":
            s["o"] = _attn_tensor(c, c["H"], _rows(c))
            s["lse"] = _empty(shape, torch.float32)
        else:
            s["dq"] = _attn_tensor(c, c["H"], c["S"])
            s["dk"], s["dv"] = _attn_tensor(c, c["Hkv"], c["S"]), _attn_tensor(c, c["Hkv"], c["S"])
            s["dtable"] = torch.empty_like(s["table"])
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
    return (z > 0).to(z.dtype)


def _layer_plain(s):
    c, dt = s["c"], s["x"].dtype
    (nbo, nbi), b = s["mask"], c["b"]
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
        out["ypre"] = z.to(dt)
    z = _act(z, c["act"])
    if c["res"]:
        z = z + s["res"].float()
    out["y"] = z.to(dt)
    return out


def _layer_bwd_plain(s):
    c, dt = s["c"], s["dy"].dtype
    if c["act"] == "none":
        return {"db": s["dy"].float().sum(0).to(dt)}
    d = s["dy"].float() * _act_slope(s["ypre"].float(), c["act"])
    return {"dpre": d.to(dt), "db": d.sum(0).to(dt)}


def _scores(s, b0, b1):
    """Scores of the sequences b0 .. b1 - 1 with the bias, -inf where a pair is
    not attended; the pairs' buckets; which are attended."""
    c = s["c"]
    R, S, G = _rows(c), c["S"], c["H"] // c["Hkv"]
    side = (s["map"].numel() + 1) // 2
    pos = s["start"][b0:b1, None].long() + torch.arange(R, device="cuda")
    key = torch.arange(S, device="cuda")
    n = s["len"][b0:b1, None].long()
    p = pos.clamp(max=side - 1)
    bucket = s["map"].long()[key - p[:, :, None] + side - 1]
    ok = s["kept"][p // BLK][:, :, key // BLK] & (bucket >= 0)
    ok = ok & (key < n)[:, None, :] & (pos < n)[:, :, None]
    q = s["q"][b0:b1].float()
    k = s["k"][b0:b1].float().repeat_interleave(G, 1)
    sc = torch.matmul(q, k.transpose(-1, -2).contiguous()) * D ** -0.5
    sc += s["table"][:, bucket.clamp(min=0)].transpose(0, 1)
    sc.masked_fill_(~ok[:, None], -math.inf)
    return sc, bucket, ok


def _chunks(c):
    n = max(1, int(2 ** 28 // (c["H"] * _rows(c) * c["S"])))
    return [(i, min(c["B"], i + n)) for i in range(0, c["B"], n)]


def _attn_plain(s):
    c = s["c"]
    G = c["H"] // c["Hkv"]
    os, lses = [], []
    for b0, b1 in _chunks(c):
        sc, _, ok = _scores(s, b0, b1)
        m = sc.amax(-1, keepdim=True).clamp(min=-1e30)
        p = torch.exp(sc - m)
        z = p.sum(-1, keepdim=True)
        p /= torch.where(z > 0, z, torch.ones_like(z))
        os.append(torch.matmul(p, s["v"][b0:b1].float().repeat_interleave(G, 1)).to(s["q"].dtype))
        lses.append((m + torch.log(z)).squeeze(-1))
    return torch.cat(os), torch.cat(lses)


def _attn_bwd_plain(s):
    c = s["c"]
    G, H, S = c["H"] // c["Hkv"], c["H"], c["S"]
    dt, scale = s["q"].dtype, D ** -0.5
    outs = {"dq": [], "dk": [], "dv": []}
    dtable = torch.zeros((H, c["buckets"]), device="cuda")
    for b0, b1 in _chunks(c):
        sc, bucket, ok = _scores(s, b0, b1)
        lse = s["lse"][b0:b1, :, :, None]
        p = torch.exp(sc - torch.where(lse > -math.inf, lse, torch.zeros_like(lse)))
        del sc
        live = ok.any(-1)[:, None, :, None]
        do = s["do"][b0:b1].float() * live
        v = s["v"][b0:b1].float().repeat_interleave(G, 1)
        k = s["k"][b0:b1].float().repeat_interleave(G, 1)
        delta = (do * s["o"][b0:b1].float()).sum(-1, keepdim=True)
        dv = torch.matmul(p.transpose(-1, -2).contiguous(), do)
        ds = torch.matmul(do, v.transpose(-1, -2).contiguous())
        ds -= delta
        ds *= p
        del p
        dq = torch.matmul(ds, k) * scale
        dk = torch.matmul(ds.transpose(-1, -2).contiguous(), s["q"][b0:b1].float()) * scale
        n = b1 - b0
        outs["dq"].append(dq.to(dt))
        outs["dk"].append(dk.view(n, c["Hkv"], G, S, D).sum(2).to(dt))
        outs["dv"].append(dv.view(n, c["Hkv"], G, S, D).sum(2).to(dt))
        # Sums along the diagonals first: every diagonal is one distance.
        side = (s["map"].numel() + 1) // 2
        dist = torch.zeros((H, 2 * S - 1), dtype=torch.float64, device="cuda")
        total = ds.sum(0)
        for r0 in range(0, S, 64):
            r1 = min(S, r0 + 64)
            n = r1 - r0
            pad = torch.zeros((H, n, S + n), device="cuda")
            pad[:, :, :S] = total[:, r0:r1].flip(1)
            # Row i from the end read as rows of S + n - 1: shifted right by i, so
            # that equal distances share the column key - row + n - 1.
            skew = pad.view(H, -1)[:, : n * (S + n - 1)].reshape(H, n, S + n - 1)
            col = torch.arange(S + n - 1, device="cuda") - (n - 1) - r0
            dist.index_add_(1, col + S - 1, skew.sum(1, dtype=torch.float64))
        ids = s["map"].long()[torch.arange(-(S - 1), S, device="cuda") + side - 1]
        keep = ids >= 0
        dtable += torch.zeros((H, c["buckets"]), dtype=torch.float64, device="cuda").index_add_(
            1, ids[keep], dist[:, keep]).float()
    return {"dq": torch.cat(outs["dq"]), "dk": torch.cat(outs["dk"]), "dv": torch.cat(outs["dv"]),
            "dtable": dtable}


# ---- run -------------------------------------------------------------------

def _run_own(s):
    c, pf = s["c"], s["pf"]
    if c["kind"] == "layer":
        pf.pf_linear_fwd_act(s["L"], c["dtype"], c["T"], c["r"], s["x"], s["w"], s["u"], s["v"],
                             s["bias"], s["act"], s["res"], s["y"], s["ypre"], s["t"], s["ws"],
                             s["wsb"])
        return {k: s[k] for k in ("t", "ypre", "y") if s[k] is not None}
    if c["kind"] == "layer_bwd":
        pf.pf_linear_act_bwd(c["dtype"], c["T"], c["N"], s["act"], s["dy"], s["ypre"], s["dpre"],
                             s["db"], s["ws"], s["wsb"])
        return {k: s[k] for k in ("dpre", "db") if s[k] is not None}
    ragged = s["len"] if c["lens"] else None
    if c["kind"] == "attn":
        if not c["rows"]:
            pf.pf_relpos_bias(s["R"], c["H"], s["table"], s["bias"])
        pf.pf_attn_relpos_fwd(s["L"], s["R"], D ** -0.5, s["q"], s["k"], s["v"], s["bias"], s["o"],
                              s["lse"], s["start"] if c["rows"] else None, ragged, s["ws"], s["wsb"])
        return {"o": s["o"], "lse": s["lse"]}
    pf.pf_attn_relpos_bwd(s["L"], s["R"], D ** -0.5, s["q"], s["k"], s["v"], s["bias"], s["o"],
                          s["lse"], s["do"], s["dq"], s["dk"], s["dv"], s["dtable"], ragged, s["ws"],
                          s["wsb"])
    return {k: s[k] for k in ("dq", "dk", "dv", "dtable")}


def run(state):
    s = state
    if own:
        return _run_own(s)
    kind = s["c"]["kind"]
    if kind == "layer":
        return _layer_plain(s)
    if kind == "layer_bwd":
        return _layer_bwd_plain(s)
    if kind == "attn":
        o, lse = _attn_plain(s)
        return {"o": o, "lse": lse}
    return _attn_bwd_plain(s)


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
    return torch.where(z > 0, 1.0, 0.0).to(z.dtype)


def _exact_layer(c, seed):
    mask, x, w, u, v, bias, res = _layer_inputs(c, seed)
    b = c["b"]
    x = x.double()
    z = torch.zeros((c["T"], c["N"]), dtype=torch.float64, device="cuda")
    p = 0
    for i, row in enumerate(mask):
        for j in np.flatnonzero(row):
            z[:, i * b:(i + 1) * b] += x[:, j * b:(j + 1) * b] @ w[p].double().t()
            p += 1
    out = {}
    if c["r"]:
        t = torch.matmul(x, v.double().t())
        out["t"] = t
        z += torch.matmul(t, u.double().t())
    if bias is not None:
        z += bias.double()
    if c["pre"]:
        out["ypre"] = z
    y = _exact_act(z, c["act"])
    out["y"] = y if res is None else y + res.double()
    return out


def _exact_layer_bwd(c, seed):
    g, dt = _gen(seed), _dtype(c)
    dy = _randn(g, (c["T"], c["N"]), 1.0, dt).double()
    if c["act"] == "none":
        return {"db": dy.sum(0)}
    dy *= _exact_slope(_randn(g, (c["T"], c["N"]), 1.2, dt).double(), c["act"])
    return {"dpre": dy, "db": dy.sum(0)}


def _exact_attn(c, seed):
    """Head by head: the bias of every distance, then the whole score matrix."""
    s = None
    if c["kind"] == "attn_bwd":
        s = prepare(c, seed)
        q, k, v, table, do = (s[n] for n in ("q", "k", "v", "table", "do"))
    else:
        q, k, v, table, do = _attn_inputs(c, seed)
    B, H, G, R, S = c["B"], c["H"], c["H"] // c["Hkv"], _rows(c), c["S"]
    ids = _bucket_map(c)
    centre = (len(ids) - 1) // 2
    kept = np.kron(_attn_mask(c), np.ones((BLK, BLK), dtype=bool))
    f64 = dict(dtype=torch.float64, device="cuda")
    o, lse = torch.zeros((B, H, R, D), **f64), torch.full((B, H, R), -math.inf, **f64)
    dq = torch.zeros((B, H, R, D), **f64)
    dk, dv = torch.zeros((B, c["Hkv"], S, D), **f64), torch.zeros((B, c["Hkv"], S, D), **f64)
    dt = torch.zeros((H, c["buckets"]), **f64)
    for b, (n, st) in enumerate(zip(_lengths(c), _starts(c))):
        m = min(R, n - st)  # live query rows
        rows, keys = st + np.arange(m), np.arange(n)
        cell = ids[keys[None, :] - rows[:, None] + centre]
        live = torch.from_numpy(kept[rows][:, :n] & (cell >= 0)).cuda()
        cell = torch.from_numpy(np.maximum(cell, 0).astype(np.int64)).cuda()
        for h in range(H):
            kh, vh = k[b, h // G, :n].double(), v[b, h // G, :n].double()
            qh = q[b, h, :m].double()
            sc = qh @ kh.t() / math.sqrt(D) + table[h].double()[cell]
            sc = torch.where(live, sc, -math.inf)
            if c["kind"] == "attn":
                lse[b, h, :m] = torch.logsumexp(sc, -1)
                o[b, h, :m] = torch.nan_to_num(torch.softmax(sc, -1)) @ vh
                continue
            row = s["lse"][b, h, :m].double()
            p = torch.where(live, torch.exp(sc - row[:, None]), 0.0)
            dh = do[b, h, :m].double()
            ds = p * (dh @ vh.t() - (dh * s["o"][b, h, :m].double()).sum(-1, keepdim=True))
            dv[b, h // G, :n] += p.t() @ dh
            dk[b, h // G, :n] += ds.t() @ qh / math.sqrt(D)
            dq[b, h, :m] = ds @ kh / math.sqrt(D)
            dt[h].index_add_(0, cell[live], ds[live])
    if c["kind"] == "attn":
        return {"o": o, "lse": lse}
    return {"dq": dq, "dk": dk, "dv": dv, "dtable": dt}


def exact(case, seed):
    if case["kind"] == "layer":
        return _exact_layer(case, seed)
    if case["kind"] == "layer_bwd":
        return _exact_layer_bwd(case, seed)
    return _exact_attn(case, seed)
