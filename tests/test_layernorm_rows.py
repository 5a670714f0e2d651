"""GPU parity of layer normalisation where workgroups take many rows and where a
row's last chunk of 16 bytes overlaps the one before (odd widths): no element is
counted twice or left out, nothing leaves its row.  Tolerances:
tests/test_layernorm_parity.py."""
import pytest

from tests._gpu_util import torch_cuda
from tests.test_layernorm_parity import _backward, _check_bwd, _check_fwd, _forward, _inputs, _rows, _types

pytestmark = pytest.mark.gpu

# Of each number of threads a row (64 to 1024 forward, to 512 backward), in both
# types; widths that leave 1 to 7 elements over, and the smallest with a chunk.
TAILS = [9, 77, 257, 323, 513, 777, 1001, 1023, 1999, 3001, 5003, 8191, 9065, 12345, 16383]


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("T,N,pad", [(10543, 323, 0), (40001, 323, 0), (65537, 256, 0), (16501, 1101, 3), (3001, 1001, 5),
                                     (9001, 3001, 0), (5001, 5003, 1), (5000, 12345, 0), (33001, 1024, 0)])
def test_many_rows(dtype, T, N, pad):
    """Several rows for every workgroup in both directions, more workgroups per CU for
    many short ones; with strides, and in place."""
    t = torch_cuda()
    g, xb, x, w, b = _inputs(t, dtype, T, N, pad, 1)
    yb, y, mean, rstd = _forward(t, dtype, x, w, b, pad)
    _check_fwd(t, x, w, b, y, mean, rstd)
    _, dy = _rows(t, T, N, pad, x.dtype)
    dy.copy_(t.randn((T, N), generator=g, device="cuda"))
    base, dx, dw, db = _backward(t, dtype, dy, x, w, mean, rstd, None, pad)
    _check_bwd(t, dy, x, w, mean, rstd, None, dx, dw, db)
    if pad:
        assert all(bool((a[:, N:] == 5).all()) for a in (xb, yb, base))
    _, dx2, dw2, db2 = _backward(t, dtype, dy, x, w, mean, rstd, None, pad, dx=dy)
    assert dx2 is dy and t.equal(dx2, dx) and t.equal(dw2, dw) and t.equal(db2, db)
    _forward(t, dtype, x, w, b, pad, out=x)
    assert t.equal(x, y)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("N", TAILS)
def test_every_element_once(dtype, N):
    """One element of each row outweighs all others, from each place of the last two
    chunks in turn: counted twice or not at all it moves the row's mean, variance and
    both means of the way back by half and more, whatever the width."""
    t = torch_cuda()
    T = min(N, 17)
    g, _, x, w, b = _inputs(t, dtype, T, N, 0, N)
    big = t.zeros((T, N), device="cuda")
    i = t.arange(T, device="cuda")
    big[i, N - 1 - i] = 1000.0
    x += big.to(x.dtype)
    _, y, mean, rstd = _forward(t, dtype, x, w, b, 0)
    _check_fwd(t, x, w, b, y, mean, rstd)
    # The way back of ordinary rows, so that one gradient outweighs the others too.
    _, _, x, w, b = _inputs(t, dtype, T, N, 0, N + 1)
    _, _, mean, rstd = _forward(t, dtype, x, w, b, 0)
    dy = (t.randn((T, N), generator=g, device="cuda") + big).to(x.dtype)
    _, dx, dw, db = _backward(t, dtype, dy, x, w, mean, rstd, None, 0)
    _check_bwd(t, dy, x, w, mean, rstd, None, dx, dw, db)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("N", TAILS)
def test_not_a_number_in_the_last_chunks(dtype, N):
    """A NaN or an infinity, from each place of the last two chunks in turn: it takes its
    own row; of the column sums its column alone; of the weights its column."""
    t = torch_cuda()
    nan, dt = float("nan"), _types(t, dtype)
    V = 16 // dt.itemsize
    g, _, x, w, b = _inputs(t, dtype, 5, N, 0, 2)
    dy = t.randn((5, N), generator=g, device="cuda").to(dt)
    _, y, mean, rstd = _forward(t, dtype, x, w, b, 0)
    _, dx, dw, db = _backward(t, dtype, dy, x, w, mean, rstd, None, 0)
    for back in range(min(N, 2 * V)):
        k = N - 1 - back
        others = [i for i in range(N) if i != k] if N < 100 else t.arange(N, device="cuda") != k
        for v in (nan, float("inf")):
            x2 = x.clone()
            x2[3, k] = v
            _, y2, m2, r2 = _forward(t, dtype, x2, w, b, 0)
            assert y2[3].isnan().all() and bool(r2[3].isnan())
            assert t.equal(y2[[0, 1, 2, 4]], y[[0, 1, 2, 4]]) and t.equal(m2[[0, 1, 2, 4]], mean[[0, 1, 2, 4]])
        for which in range(2):
            a = [dy.clone(), x.clone()]
            a[which][3, k] = nan
            _, d2, w2, b2 = _backward(t, dtype, a[0], a[1], w, mean, rstd, None, 0)
            assert d2[3].isnan().all() and t.equal(d2[[0, 1, 2, 4]], dx[[0, 1, 2, 4]])
            assert bool(w2[k].isnan()) and t.equal(w2[others], dw[others])
            assert bool(b2[k].isnan()) == (which == 0) and t.equal(b2[others], db[others])
        # A gradient that is added stays in its element.
        dr = t.zeros_like(x)
        dr[3, k] = nan
        _, d2, w2, b2 = _backward(t, dtype, dy, x, w, mean, rstd, dr, 0)
        assert d2.isnan().sum() == 1 and bool(d2[3, k].isnan()) and t.equal(w2, dw) and t.equal(b2, db)
        for which in range(2):
            a = [w.clone(), b.clone()]
            a[which][k] = nan
            _, y2, m2, r2 = _forward(t, dtype, x, a[0], a[1], 0)
            assert y2[:, k].isnan().all() and t.equal(y2[:, others], y[:, others])
            assert t.equal(m2, mean) and t.equal(r2, rstd)
