"""fp32 GELU and its derivative keep their digits where the CDF is small: every
entry point that computes them, at points of both signs, zeros, tails and the
largest values, against scipy's erfc in float64 (Phi(x) = erfc(-x / sqrt 2) / 2; the form
1 + erf cancels to 4 % at -5 and to nothing at -5.6).

Bounds, from the arithmetic (e = 2^-24).  Beyond |x| = 1.25 the CDF's tail is t Q(t)
exp(-x^2 / 2): the fit 4e-7 (7 e); the reciprocal and the exponential one unit in the last
place (2 e each); t's rounding, which tail at most doubles, the five steps of Q and the
products 20 e; the exponent's two roundings and its constant's, together at most 2.8 e of
x^2 / 2.  Nearer to zero it is a polynomial within 7.45e-8 (tests/test_gelu_cdf_host.py), 12 e of
the 0.1056 and more there.  So Phi is within e (1.4 x^2 + 32) of itself, GELU with a product
and a store e (1.4 x^2 + 34).  x times the density rounds with 1.4 x^2 e for the exponent, two
for the exponential and four in all for the constant and the products; the derivative is
within e (1.4 x^2 + 32) Phi + e (1.4 x^2 + 6) |x| phi + 2 e of itself.  What falls below 2^-126
on the way may flush, up to 15 times that in the results."""
import numpy as np
import pytest
from scipy.special import erfc

from tests._gpu_util import to_dev, to_host, torch_cuda

pytestmark = pytest.mark.gpu

E = 2.0 ** -24


def _points(n):
    g = np.concatenate([np.linspace(-14, 14, n - 48), [0.0, -0.0, 1e-30, -1e-30, 30.0, -30.0, 1e4, -1e4, 1e18, -1e18,
                                                       3e38, -3e38]])
    x = np.zeros(n, np.float32)
    x[:g.size] = g
    return x


def _value(x):
    return 0.5 * x * erfc(-x / np.sqrt(2.0))


def _slope(x):
    with np.errstate(all="ignore"):
        phi = np.exp(-0.5 * x * x) / np.sqrt(2 * np.pi)
        return 0.5 * erfc(-x / np.sqrt(2.0)), np.where(np.abs(x) < 40, x * phi, 0.0)


def _check(name, got, ref, bound):
    bad = np.abs(got - ref) - bound - 15 * 2.0 ** -126
    i = int(np.argmax(bad))
    assert np.isfinite(got).all() and (bad <= 0).all(), (name, i, got[i], ref[i], bound[i])


def _check_value(name, got, x):
    x2 = np.minimum(x * x, 200.0)
    _check(name, got, _value(x), E * (1.4 * x2 + 34) * np.abs(_value(x)))


def _check_slope(name, got, x):
    x2 = np.minimum(x * x, 200.0)
    cdf, den = _slope(x)
    _check(name, got, cdf + den, E * ((1.4 * x2 + 32) * cdf + (1.4 * x2 + 6) * np.abs(den) + 2 * np.abs(cdf + den)))


def _identity(t, pf, b, copies):
    """A layer whose every block row i copies block column i: identity."""
    L = pf.pf_layout_create(copies * b, copies * b, b, 1)
    pf.pf_layout_upload(L)
    return L, t.eye(b, device="cuda").repeat(copies, 1, 1).contiguous()


# Few output tiles and many: both forward kernels of fp32.
@pytest.mark.parametrize("T,b,copies", [(64, 32, 1), (2048, 32, 32), (2048, 64, 16), (2048, 128, 8)])
def test_value_of_the_layers(T, b, copies):
    t = torch_cuda()
    from paper_2112_00029_amd import pixelfly as pf
    L, w = _identity(t, pf, b, copies)
    N = copies * b
    x = np.resize(_points(min(T * N, 1 << 15)), (T, N))
    X, y, pre = to_dev(x), t.empty((T, N), device="cuda"), t.empty((T, N), device="cuda")
    x = x.astype(np.float64)
    n = pf.pf_workspace_bytes(L, T, 0, "fp32")
    ws = t.empty((max(n, 256),), dtype=t.uint8, device="cuda")
    print(f"[gelu fp32] forward T={T} b={b} N={N}", flush=True)
    pf.pf_linear_fwd_act(L, "fp32", T, 0, X, w, None, None, None, pf.PF_ACT_GELU, None, y, pre, None,
                         ws, n)
    assert t.equal(pre, X)
    _check_value("act", to_host(y).ravel(), x.ravel())
    y2 = t.empty_like(y)
    pf.pf_linear_fwd(L, "fp32", T, 0, X, w, None, None, y2, None, pf.PF_EPI_GELU, pre, ws, n)
    _check_value("plain", to_host(y2).ravel(), x.ravel())
    one = t.ones_like(X)
    pf.pf_linear_bwd_data(L, "fp32", T, 0, one, w, None, None, None, y, pf.PF_EPI_GELU, X, ws, n)
    _check_slope("backward-data", to_host(y).ravel(), x.ravel())


def test_slope_alone():
    t = torch_cuda()
    from paper_2112_00029_amd import pixelfly as pf
    x = _points(1 << 15)
    X = to_dev(x)
    one, out = t.ones_like(X), t.empty_like(X)
    print("[gelu fp32] derivative", flush=True)
    pf.pf_gelu_bwd("fp32", x.size, one, X, out)
    _check_slope("pf_gelu_bwd", to_host(out), x.astype(np.float64))
    db = t.empty((x.size // 64,), device="cuda")
    ws = t.empty((1 << 20,), dtype=t.uint8, device="cuda")
    out.fill_(float("nan"))
    pf.pf_linear_act_bwd("fp32", 64, x.size // 64, pf.PF_ACT_GELU, one, X, out, db, ws, 1 << 20)
    _check_slope("pf_linear_act_bwd", to_host(out), x.astype(np.float64))


def test_value_with_bias_and_residual():
    """Z = x through the bias of a layer of zeros; the residual is added last."""
    t = torch_cuda()
    from paper_2112_00029_amd import pixelfly as pf
    N = 4096
    x = _points(N)
    L = pf.pf_layout_create(N, 32, 32, 1)
    pf.pf_layout_upload(L)
    w, X = t.zeros((N // 32, 32, 32), device="cuda"), t.ones((1, 32), device="cuda")
    res = t.zeros((1, N), device="cuda")
    y, pre = t.empty((1, N), device="cuda"), t.empty((1, N), device="cuda")
    print("[gelu fp32] bias", flush=True)
    pf.pf_linear_fwd_act(L, "fp32", 1, 0, X, w, None, None, to_dev(x), pf.PF_ACT_GELU, res, y, pre, None)
    _check_value("bias", to_host(y).ravel(), x.astype(np.float64))
