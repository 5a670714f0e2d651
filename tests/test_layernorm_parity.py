"""GPU parity of layer normalisation, forward and backward, against float64.

Tolerances, element by element (u = finfo(t).eps / 2 of the stored type, e =
2^-24, N elements a row summed in fp32):
  * the mean is a sum in 64 bits, taken off as two fp32 numbers: the differences d = x
    - mean are off by their two roundings, td = 2 e (|x| + |mean|);
  * var: relative (2 N + 4) e, and 2 td's root mean square over std; rstd half of
    that and 4 e;
  * y: n = d rstd, one product and one sum, a rounding.
  * backward: n is off by 3 e (|x| + |mean|) rstd + 3 e |n| (the given fp32
    statistics are its inputs); sums over a row N e of the terms' mean absolute
    value; column sums T e."""
import numpy as np
import pytest

from tests._gpu_util import torch_cuda

pytestmark = pytest.mark.gpu
E = 2.0 ** -24
EPS = 1e-5

# Widths for every variant: one wave to sixteen, one or two chunks, odd ones.
WIDTHS = [1, 2, 7, 32, 64, 96, 100, 511, 512, 520, 768, 1000, 1023, 1024, 1032, 2048, 2056, 3001, 4096, 5120,
          8192, 8200, 12345, 16384]


def _types(t, dtype):
    return t.bfloat16 if dtype == "bf16" else t.float32


def _rows(t, T, N, pad, dt, fill=None):
    b = t.full((T, N + pad), 5.0 if fill is None else fill, dtype=dt, device="cuda")
    return b, b[:, :N]


def _inputs(t, dtype, T, N, pad, seed, shift=0.5):
    g = t.Generator(device="cuda").manual_seed(seed)
    dt = _types(t, dtype)
    spread = t.exp(0.5 * t.randn((N,), generator=g, device="cuda"))
    base, x = _rows(t, T, N, pad, dt)
    x.copy_(t.randn((T, N), generator=g, device="cuda") * spread + shift)
    w = (1 + 0.3 * t.randn((N,), generator=g, device="cuda")).to(dt)
    b = (0.3 * t.randn((N,), generator=g, device="cuda")).to(dt)
    return g, base, x, w, b


def _forward(t, dtype, x, w, b, pad, stats=True, out=None, stream=None):
    from paper_2112_00029_amd import pixelfly as pf
    T, N = x.shape
    base, y = (None, out) if out is not None else _rows(t, T, N, pad, x.dtype)
    mean, rstd = (t.full((T,), float("nan"), device="cuda") for _ in range(2)) if stats else (None, None)
    pf.pf_layernorm_fwd(dtype, T, N, EPS, x, x.stride(0) if T > 1 else N, w, b, y, y.stride(0) if T > 1 else N,
                        mean, rstd, stream)
    return base, y, mean, rstd


def _check_fwd(t, x, w, b, y, mean, rstd):
    N = x.shape[1]
    u = t.finfo(x.dtype).eps / 2
    X = x.double()
    m = X.mean(1, keepdim=True)
    d = X - m
    var = (d * d).mean(1, keepdim=True)
    r = (var + EPS) ** -0.5
    ax = X.abs()
    td = 2 * E * (ax + m.abs())
    rms = (td * td).mean(1, keepdim=True) ** 0.5
    std = var ** 0.5
    rv = (2 * N + 4) * E + (2 * rms * std + rms * rms) / (var + EPS)
    rr = 0.5 * rv * (1 + rv) + 4 * E
    if mean is not None:
        bad = (mean.double() - m[:, 0]).abs() - (E + 1e-12) * m[:, 0].abs() - 1e-13 * ax.mean(1)
        assert not (bad > 0).any(), ("mean", float(bad.max()))
        bad = (rstd.double() / r[:, 0] - 1).abs() - (rr[:, 0] + E)
        assert not (bad > 0).any(), ("rstd", float(bad.max()))
    n = d * r
    tn = td * r * (1 + rr) + n.abs() * (rr + E)
    W = w.double() if w is not None else t.ones((N,), dtype=t.float64, device="cuda")
    B = b.double() if b is not None else t.zeros((N,), dtype=t.float64, device="cuda")
    want = n * W + B
    tol = W.abs() * tn + 2 * E * ((n * W).abs() + B.abs())
    bad = (y.double() - want).abs() - (u * want.abs() + (1 + u) * tol)
    assert not (bad > 0).any() and not y.isnan().any(), ("y", float(bad.max()))


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("N", WIDTHS)
def test_forward(dtype, N):
    t = torch_cuda()
    for T, pad in ((1, 0), (5, 0), (300, 0), (37, 8), (11, 3)):
        _, xb, x, w, b = _inputs(t, dtype, T, N, pad, N + T)
        yb, y, mean, rstd = _forward(t, dtype, x, w, b, pad)
        _check_fwd(t, x, w, b, y, mean, rstd)
        if pad:
            assert bool((yb[:, N:] == 5).all()) and bool((xb[:, N:] == 5).all())
        _, y2, _, _ = _forward(t, dtype, x, w, b, 0, stats=False)
        assert t.equal(y2, y)
    _, y, mean, rstd = _forward(t, dtype, x, None, None, 0)
    _check_fwd(t, x, None, None, y, mean, rstd)
    want = y.clone()
    # In place.
    z = _rows(t, T, N, pad, x.dtype)[1].copy_(x)
    _, y, _, _ = _forward(t, dtype, z, None, None, 0, out=z)
    assert t.equal(y, want)


@pytest.mark.parametrize("N", [64, 1000, 4096])
def test_rows_far_from_zero(N):
    """A mean of a thousand standard deviations, and rows of one value."""
    t = torch_cuda()
    _, _, x, w, b = _inputs(t, "fp32", 40, N, 0, 3, shift=3000.0)
    _, y, mean, rstd = _forward(t, "fp32", x, w, b, 0)
    _check_fwd(t, x, w, b, y, mean, rstd)
    for v in (0.0, -7.25, 1e6, 0.1):
        x = t.full((3, N), v, device="cuda")
        _, y, mean, rstd = _forward(t, "fp32", x, w, b, 0)
        # Sums of N equal numbers: off by roundings in 64 bits alone.
        assert bool(((mean - v).abs() <= 2 * E * abs(v)).all())
        assert bool(((y - b).abs() <= (4 * E * abs(v) * EPS ** -0.5 + 2 * E) * w.abs() + 2 * E * b.abs()).all())


def test_not_a_number_stays_in_its_row():
    t = torch_cuda()
    for N in (96, 1024, 3000):
        _, _, x, w, b = _inputs(t, "bf16", 9, N, 0, 1)
        _, want, _, _ = _forward(t, "bf16", x, w, b, 0)
        x[2, 5], x[4, N - 1], x[6, 0] = float("nan"), float("inf"), -float("inf")
        _, y, mean, rstd = _forward(t, "bf16", x, w, b, 0)
        for i in range(9):
            if i in (2, 4, 6):
                assert y[i].isnan().all() and bool(rstd[i].isnan()), i
            else:
                assert t.equal(y[i], want[i]), i


def _backward(t, dtype, dy, x, w, mean, rstd, dr, pad, sums=True, dx=None, fill=255):
    from paper_2112_00029_amd import pixelfly as pf
    T, N = x.shape
    ld = lambda a: a.stride(0) if T > 1 else N
    base, out = (None, dx) if dx is not None else _rows(t, T, N, pad, x.dtype)
    wsb = pf.pf_layernorm_workspace_bytes(dtype, T, N)
    ws = t.full((wsb,), fill, dtype=t.uint8, device="cuda")
    dw, db = (t.full((N,), float("nan"), dtype=x.dtype, device="cuda") for _ in range(2)) if sums else (None, None)
    pf.pf_layernorm_bwd(dtype, T, N, dy, ld(dy), x, ld(x), w, mean, rstd, dr, ld(dr) if dr is not None else 0, out,
                        ld(out), dw, db, ws if sums else None, wsb if sums else 0)
    return base, out, dw, db


def _check_bwd(t, dy, x, w, mean, rstd, dr, dx, dw, db):
    T, N = x.shape
    u = t.finfo(x.dtype).eps / 2
    X, D = x.double(), dy.double()
    m, r = mean.double()[:, None], rstd.double()[:, None]
    n = (X - m) * r
    tn = 2 * E * (X.abs() + m.abs()) * r + 2 * E * n.abs()
    W = w.double() if w is not None else t.ones((N,), dtype=t.float64, device="cuda")
    q = D * W
    c1, c2 = q.mean(1, keepdim=True), (q * n).mean(1, keepdim=True)
    t1 = (N + 3) * E * q.abs().mean(1, keepdim=True)
    t2 = (N + 4) * E * (q * n).abs().mean(1, keepdim=True) + (q.abs() * tn).mean(1, keepdim=True)
    core = r * (q - c1 - n * c2)
    tol = r * (2 * E * q.abs() + t1 + n.abs() * t2 + tn * c2.abs() + tn * t2 +
               4 * E * (q.abs() + c1.abs() + (n * c2).abs())) + E * core.abs()
    want = core + dr.double() if dr is not None else core
    tol = tol + E * want.abs() + E * core.abs()
    bad = (dx.double() - want).abs() - (u * want.abs() + (1 + u) * tol)
    assert not (bad > 0).any() and not dx.isnan().any(), ("dx", float(bad.max()))
    if dw is None:
        return
    col = (D * n).sum(0)
    tc = (D.abs() * tn).sum(0) + (T + 2) * E * (D * n).abs().sum(0) * (1 + 1e-3)
    bad = (dw.double() - col).abs() - (u * col.abs() + (1 + u) * tc)
    assert not (bad > 0).any() and not dw.isnan().any(), ("dw", float(bad.max()))
    col = D.sum(0)
    bad = (db.double() - col).abs() - (u * col.abs() + (1 + u) * T * E * D.abs().sum(0))
    assert not (bad > 0).any() and not db.isnan().any(), ("db", float(bad.max()))


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("N", WIDTHS)
def test_backward(dtype, N):
    t = torch_cuda()
    from paper_2112_00029_amd import pixelfly as pf
    for T, pad in ((1, 0), (6, 0), (700, 0), (37, 8), (11, 3)):
        g, _, x, w, b = _inputs(t, dtype, T, N, pad, N + T)
        _, _, mean, rstd = _forward(t, dtype, x, w, b, 0)
        _, dy = _rows(t, T, N, pad, x.dtype)
        dy.copy_(t.randn((T, N), generator=g, device="cuda"))
        _, dr = _rows(t, T, N, pad, x.dtype)
        dr.copy_(t.randn((T, N), generator=g, device="cuda"))
        base, dx, dw, db = _backward(t, dtype, dy, x, w, mean, rstd, dr, pad)
        _check_bwd(t, dy, x, w, mean, rstd, dr, dx, dw, db)
        if pad:
            assert bool((base[:, N:] == 5).all())
        # Again, from other workspace contents; in place of each input; without
        # the column sums.
        _, dx2, dw2, db2 = _backward(t, dtype, dy, x, w, mean, rstd, dr, pad, fill=0)
        assert t.equal(dx2, dx) and t.equal(dw2, dw) and t.equal(db2, db)
        for k in range(3):
            a = [dy, x, dr]
            a[k] = _rows(t, T, N, pad, x.dtype)[1].copy_(a[k])
            _, dx2, dw2, db2 = _backward(t, dtype, a[0], a[1], w, mean, rstd, a[2], pad, dx=a[k])
            assert t.equal(dx2, dx) and t.equal(dw2, dw) and t.equal(db2, db), k
        _, dx2, _, _ = _backward(t, dtype, dy, x, w, mean, rstd, dr, pad, sums=False)
        assert t.equal(dx2, dx)
        # One of the column sums alone.
        wsb = pf.pf_layernorm_workspace_bytes(dtype, T, N)
        ws, ld = t.empty((wsb,), dtype=t.uint8, device="cuda"), x.stride(0) if T > 1 else N
        for k in range(2):
            o = [t.zeros_like(dw), None] if k == 0 else [None, t.zeros_like(db)]
            pf.pf_layernorm_bwd(dtype, T, N, dy, ld, x, ld, w, mean, rstd, dr, ld, dx2, ld, *o, ws, wsb)
            assert t.equal(dx2, dx) and t.equal(o[k], (dw, db)[k])
    _, dx, dw, db = _backward(t, dtype, dy, x, None, mean, rstd, None, pad)
    _check_bwd(t, dy, x, None, mean, rstd, None, dx, dw, db)


@pytest.mark.parametrize("dtype,T,N", [("bf16", 16384, 768), ("bf16", 9001, 4096), ("fp32", 5000, 1024)])
def test_many_rows(dtype, T, N):
    t = torch_cuda()
    g, _, x, w, b = _inputs(t, dtype, T, N, 0, 1)
    _, y, mean, rstd = _forward(t, dtype, x, w, b, 0)
    _check_fwd(t, x, w, b, y, mean, rstd)
    dy = t.randn((T, N), generator=g, device="cuda").to(x.dtype)
    _, dx, dw, db = _backward(t, dtype, dy, x, w, mean, rstd, None, 0)
    _check_bwd(t, dy, x, w, mean, rstd, None, dx, dw, db)


def test_gradients_against_differences():
    t = torch_cuda()
    T, N = 12, 100
    g, _, x, w, b = _inputs(t, "fp32", T, N, 0, 5)
    _, _, mean, rstd = _forward(t, "fp32", x, w, b, 0)
    G = t.randn((T, N), generator=g, device="cuda")
    _, dx, dw, db = _backward(t, "fp32", G, x, w, mean, rstd, None, 0)

    def loss(x, w, b):
        d = x - x.mean(1, keepdim=True)
        return float((G.double() * (d * ((d * d).mean(1, keepdim=True) + EPS) ** -0.5 * w + b)).sum())

    at = [p.double() for p in (x, w, b)]
    for k, grad in enumerate((dx, dw, db)):
        way = t.randn(at[k].shape, generator=g, device="cuda", dtype=t.float64)
        way /= way.norm()
        ends = []
        for s in (1, -1):
            p = list(at)
            p[k] = p[k] + s * 1e-4 * way
            ends.append(loss(*p))
        num, got = (ends[0] - ends[1]) / 2e-4, float((grad.double() * way).sum())
        # Differences: third order, below 1e-6; fp32: (N + T) roundings.
        assert abs(num - got) <= (1e-6 + 200 * E) * float(grad.double().norm()), (k, num, got)


def test_offsets_past_32_bits():
    """Rows whose elements lie past 2^32 bytes and 2^31 elements from the first."""
    t = torch_cuda()
    T, N, ld = 3, 512, (1 << 30) + 8
    buf = t.zeros((2 * ld + N,), dtype=t.bfloat16, device="cuda")
    x = buf.as_strided((T, N), (ld, 1))
    g = t.Generator(device="cuda").manual_seed(2)
    x.copy_(t.randn((T, N), generator=g, device="cuda"))
    w, b = t.ones((N,), dtype=t.bfloat16, device="cuda"), t.zeros((N,), dtype=t.bfloat16, device="cuda")
    _, y, mean, rstd = _forward(t, "bf16", x, w, b, 0)
    _, want, m2, r2 = _forward(t, "bf16", x.contiguous(), w, b, 0)
    assert t.equal(y, want) and t.equal(mean, m2) and t.equal(rstd, r2)
    dy = want
    _, d2, w2, b2 = _backward(t, "bf16", dy, x.contiguous(), w, mean, rstd, None, 0)
    _, d1, w1, b1 = _backward(t, "bf16", dy, x, w, mean, rstd, None, 0, dx=x)
    assert t.equal(d1, d2) and t.equal(w1, w2) and t.equal(b1, b2)


def test_streams_and_graphs():
    t = torch_cuda()
    from paper_2112_00029_amd import pixelfly as pf
    T, N = 300, 768
    g, _, x, w, b = _inputs(t, "bf16", T, N, 0, 4)
    _, y, mean, rstd = _forward(t, "bf16", x, w, b, 0)
    dy = t.randn((T, N), generator=g, device="cuda").bfloat16()
    _, dx, dw, db = _backward(t, "bf16", dy, x, w, mean, rstd, None, 0)
    wsb = pf.pf_layernorm_workspace_bytes("bf16", T, N)
    y2, dx2, dw2, db2 = t.zeros_like(y), t.zeros_like(dx), t.zeros_like(dw), t.zeros_like(db)
    m2, r2, ws = t.zeros_like(mean), t.zeros_like(rstd), t.zeros((wsb,), dtype=t.uint8, device="cuda")
    st, graph = t.cuda.Stream(), t.cuda.CUDAGraph()
    with t.cuda.graph(graph, stream=st):
        pf.pf_layernorm_fwd("bf16", T, N, EPS, x, N, w, b, y2, N, m2, r2)
        pf.pf_layernorm_bwd("bf16", T, N, dy, N, x, N, w, m2, r2, None, 0, dx2, N, dw2, db2, ws, wsb)
    for _ in range(3):
        for o in (y2, dx2, dw2, db2, m2, r2):
            o.fill_(9.0)
        graph.replay()
        t.cuda.synchronize()
        assert t.equal(y2, y) and t.equal(dx2, dx) and t.equal(dw2, dw) and t.equal(db2, db)
