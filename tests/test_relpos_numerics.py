"""Position-bias attention over the range of scales that the calls accept, with
large scores, and its table gradient against differences that can fail.

Tolerances, pair by pair (u = 2^-8, half a step of bf16; e = 2^-24, of fp32; every
input is exact), in units of the natural score S = scale q.k + bias:
  * q.k is an fp32 sum of 64 products, which in dK/dV starts at the bias: 64 e of scale
    sum |q k| and of |bias|; scale log2(e) and the bias in log2 units round twice each,
    the bias of dK/dV three times more; the score, its difference from the running
    maximum and from lse round to at most 8 e |S| and, lse itself (the maximum plus a
    logarithm, times ln 2, and back times log2 e), 12 e |lse|; the hardware exponential and
    logarithm 1e-6.  So P is off by
        E = e (66 scale sum |q k| + 71 |bias| + 8 |S| + 12 |lse|) + 1e-6
    of itself, a row's sum of n of them by max E + n e, lse by as much;
  * O: each P rounded to bf16 before its product, the result once more;
  * gradients: dS off by P E (|dP| + |delta|) and 64 e of the sums in dP and delta, rounded
    to bf16 before its products, P before dV's; sums of n terms n e; the result once more;
  * dtable takes dS unrounded;
  * a P below the least normal number t = 2^-126 flushes to zero, and so may dS and the
    products' terms: P is off by t, dS by t (|dP| + |delta| + 1) more."""
import numpy as np
import pytest

from tests.test_relpos_parity import BLK, D, U, Case, butterfly, clip_map, log_map

pytestmark = pytest.mark.gpu

E32, TINY = 2.0 ** -24, 2.0 ** -126


class Scaled(Case):
    """A case with another scale, whose q and k are multiplied by qs and ks."""

    def __init__(self, *a, scale, qs=1.0, ks=1.0, **k):
        super().__init__(*a, **k)
        self.scale = float(np.float32(scale))
        self.q.mul_(qs)
        self.k.mul_(ks)

    def pairs(self, b, h):
        """Scores, pairs, buckets, key/value head, tokens, and the relative error of
        P with each row's (lse from the scores)."""
        t = self.t
        s, live, cell, hk, n, _ = self.head(b, h)
        lse = t.logsumexp(s, -1).nan_to_num(neginf=0.0)
        qk = self.scale * (self.q[b, h].double().abs() @ self.k[b, hk].double().abs().t())
        err = E32 * (66 * qk + 71 * self.table[h].double().abs()[cell] + 8 * s.nan_to_num(neginf=0.0).abs()
                     + 12 * lse.abs()[:, None]) + 1e-6
        return s, live, cell, hk, n, t.where(live, err, 0.0)

    def check_fwd(self, o, lse):
        t = self.t
        for b in range(self.B):
            for h in range(self.H):
                s, live, _, hk, n, err = self.pairs(b, h)
                some, row = live.any(-1), err.amax(-1) + n * E32
                ref = t.logsumexp(s, -1)
                p = t.nan_to_num(t.softmax(s, -1))
                v = t.where(live.any(0)[:, None], self.v[b, hk].double(), 0.0)
                ro, mag = p @ v, p @ v.abs()
                assert t.equal(lse[b, h] == -float("inf"), ~some) and not lse.isnan().any(), (b, h)
                bad = ((lse[b, h].double() - ref).abs() - row)[some]
                assert (bad <= 0).all(), ("lse", b, h, float(bad.max()))
                bad = (o[b, h].double() - ro).abs() - (U * ro.abs() + (1 + U) * (U + 2 * row)[:, None] * mag)
                assert (bad <= 0).all() and not o[b, h].isnan().any(), ("O", b, h, float(bad.max()))

    def check_bwd(self, o, lse, dq, dk, dv, dt):
        t, G = self.t, self.H // self.Hkv
        f64 = dict(dtype=t.float64, device="cuda")
        rt, tt = t.zeros((self.H, self.nbucket), **f64), t.zeros((self.H, self.nbucket), **f64)
        for b in range(self.B):
            rk, rv = t.zeros((self.Hkv, self.S, D), **f64), t.zeros((self.Hkv, self.S, D), **f64)
            tk, tv = t.zeros_like(rk), t.zeros_like(rv)
            for h in range(self.H):
                s, live, cell, hk, n, err = self.pairs(b, h)
                some = live.any(-1, keepdim=True)
                p = t.where(live, t.exp(s - t.where(some[:, 0], lse[b, h].double(), 0.0)[:, None]), 0.0)
                keys = (t.arange(self.S, device="cuda") < n)[:, None]
                cut = lambda x, m: t.where(m, x.double(), 0.0)
                k, v = cut(self.k[b, hk], keys), cut(self.v[b, hk], keys)
                q, do, oo = cut(self.q[b, h], some), cut(self.do[b, h], some), cut(o[b, h], some)
                delta, dp = (do * oo).sum(-1, keepdim=True), do @ v.t()
                ds = p * (dp - delta)
                eds = p * (err * (dp.abs() + delta.abs()) + 64 * E32 * (
                    do.abs() @ v.abs().t() + (do.abs() * oo.abs()).sum(-1, keepdim=True)))
                eds = eds + t.where(live, TINY * (dp.abs() + delta.abs() + 1), 0.0)
                low = (U + n * E32) * ds.abs() + (1 + U) * eds  # as bf16, in a sum of n
                rq, tq = ds @ k * self.scale, low @ k.abs() * self.scale
                bad = (dq[b, h].double() - rq).abs() - (U * rq.abs() + (1 + U) * tq + TINY)
                assert (bad <= 0).all() and not dq[b, h].isnan().any(), ("dQ", b, h, float(bad.max()))
                rk[hk] += ds.t() @ q * self.scale
                tk[hk] += (low + (G - 1) * n * E32 * ds.abs()).t() @ q.abs() * self.scale
                rv[hk] += p.t() @ do
                tv[hk] += (p * (U + G * n * E32 + (1 + U) * err) + TINY).t() @ do.abs()
                rt[h].index_add_(0, cell[live], ds[live])
                tt[h].index_add_(0, cell[live], (eds + self.B * n * E32 * ds.abs())[live])
            for name, got, r, tol in (("dK", dk, rk, tk), ("dV", dv, rv, tv)):
                bad = (got[b].double() - r).abs() - (U * r.abs() + (1 + U) * tol + TINY)
                assert (bad <= 0).all() and not got[b].isnan().any(), (name, b, float(bad.max()))
        bad = (dt.double() - rt).abs() - tt
        assert (bad <= 0).all() and not dt.isnan().any(), ("dtable", float(bad.max()))


# The ends of the accepted scales on inputs whose scores are ordinary; scales that
# are no power of two; scores of 50 and of some hundreds.
SCALES = [(2.0 ** -40, 2.0 ** 19, 2.0 ** 18), (2.0 ** 40, 2.0 ** -21, 2.0 ** -22), (0.11, 1.0, 1.0), (1.0, 1.0, 1.0),
          (7.3, 1.0, 1.0)]


@pytest.mark.parametrize("scale,qs,ks", SCALES)
@pytest.mark.parametrize("kind", ["clip", "log_causal"])
def test_scales(scale, qs, ks, kind):
    print(f"[relpos] scale {scale} {kind}", flush=True)
    if kind == "clip":
        c = Scaled(2, 4, 2, 450, clip_map(512, 20), 41, np.ones((8, 8), bool), [450, 130], scale=scale, qs=qs, ks=ks)
    else:
        c = Scaled(1, 2, 2, 640, log_map(640, 16, 96, False), 16, butterfly(10, 16, 1), None, True, scale=scale,
                   qs=qs, ks=ks)
    c.check()


@pytest.mark.parametrize("scale,qs,ks", SCALES)
def test_scales_of_one_row(scale, qs, ks):
    print(f"[relpos] one row, scale {scale}", flush=True)
    c = Scaled(3, 8, 2, 700, clip_map(704, 40, True), 81, np.ones((11, 11), bool), [700, 65, 300], True, 1,
               [699, 64, 200], scale=scale, qs=qs, ks=ks)
    c.check_fwd(*c.fwd())


@pytest.mark.parametrize("scale", [2.0 ** 20, 1.3 * 2.0 ** 24, 0.9 * 2.0 ** 30, 2.0 ** 33, 2.0 ** 40])
@pytest.mark.parametrize("rows", [None, 1, 90])
def test_large_scores(scale, rows):
    """q and k of small integers and a table in steps of scale / 512: of two scores
    that differ, the larger takes all (they differ by 2^11 or more, some hundred times
    fp32's rounding of them), and equal ones share.  O is the mean of V over a row's best
    keys, lse their score plus the logarithm of their number."""
    print(f"[relpos] scores of {scale} x 100, rows {rows}", flush=True)
    lens = [512, 200, 333]
    starts = None if rows is None else [n - rows for n in lens]
    c = Scaled(3, 4, 2, 512, clip_map(512, 20), 41, np.ones((8, 8), bool), lens, False, rows, starts, scale=scale)
    t = c.t
    for x in (c.q, c.k):
        x.copy_(x.float().round().clamp(-2, 2))
    g = np.random.default_rng(1)
    step = np.array([g.permutation(41) - 20 for _ in range(4)])
    c.table.copy_(t.from_numpy(step).cuda() * (c.scale / 512))
    c.pf.pf_relpos_bias(c.R, 4, c.table, c.bias)
    o, lse = c.fwd()
    for b in range(3):
        for h in range(4):
            s, live, _, hk, n, _ = c.head(b, h)
            some, top = live.any(-1), s.amax(-1, keepdim=True)
            best = t.where(live, s == top, False).double()
            num = best.sum(-1)
            w = best / num.clamp(min=1)[:, None]
            v = c.v[b, hk].double()
            ro, mag = w @ v, w @ v.abs()
            bad = (o[b, h].double() - ro).abs() - (U * ro.abs() + (1 + U) * 2 * n * E32 * mag)
            assert (bad <= 0).all() and not o[b, h].isnan().any(), ("O", b, h, float(bad.nan_to_num(1e9).max()))
            want = (top[:, 0] + t.log(num))[some]
            assert ((lse[b, h].double()[some] - want).abs() <= 8 * E32 * want.abs()).all(), (b, h)
            assert (lse[b, h][~some] == -float("inf")).all()


def _row_terms(c, h, o):
    """Head h of sequence 0: P, dP, the exact delta, the kernel's (from its O),
    pairs, buckets, relative error of P."""
    t = c.t
    s, live, cell, hk, n, err = c.pairs(0, h)
    p = t.nan_to_num(t.softmax(s, -1))
    do, v = c.do[0, h].double(), c.v[0, hk].double()
    dp = do @ v.t()
    return p, dp, (p * dp).sum(-1, keepdim=True), (do * o[0, h].double()).sum(-1, keepdim=True), live, cell, n, err


@pytest.mark.parametrize("kind,wide", [("clip", 0), ("clip", 40), ("log", 7), ("log", 15)])
def test_table_gradient_against_differences(kind, wide):
    """dtable by central differences of <dO, O> in float64 over the table, at each
    head's largest entries and at a bucket of many distances, along whose part of O the
    rows' dO lean, so that its entry is large too.

    delta takes O as it is stored: what its rounding moves dtable by, the sum over rows of
    P(bucket) (delta - <dO, O stored>), is computed and taken off, so that the bound is the
    fp32 part alone: P E (|dP| + |delta|), 64 e of the sums in dP and delta, n e of the sum.
    In one entry x the rows' O is linear in a logistic function of x, whose third
    derivative is at most its first: differences of step h are off by h^2 / 6 of the rows'
    absolute terms.  Bound and correction are at most 2 % of every entry checked: a dtable
    of zeros, one without delta, scaled or of the wrong bucket fails."""
    m, n = (clip_map(192, 20), 41) if kind == "clip" else (log_map(192, 16, 64, True), 16)
    c = Scaled(1, 2, 1, 190, m, n, butterfly(3, 4), [177], scale=0.125, seed=2)
    t = c.t
    o, lse = c.fwd()
    for hd in range(2):
        p, _, _, _, live, cell, _, _ = _row_terms(c, hd, o)
        v, mine = c.v[0, 0].double(), t.where(live & (cell == wide), p, 0.0)
        lean = mine @ v / mine.sum(-1, keepdim=True).clamp(min=1e-9) - p @ v
        c.do[0, hd] += (8 * lean / lean.norm(dim=-1, keepdim=True).clamp(min=1e-9)).bfloat16()
    _, _, _, dt = c.bwd(o, lse)
    tab, h = c.table.double(), 1e-3
    for hd in range(2):
        p, dp, delta, stored, live, cell, nk, err = _row_terms(c, hd, o)
        do, v = c.do[0, hd].double(), c.v[0, 0].double()

        def loss():
            s = c.head(0, hd)[0]
            return float((t.nan_to_num(t.softmax(s, -1)) @ v * do).sum())

        sums = lambda x: t.zeros(n, dtype=t.float64, device="cuda").index_add_(0, cell[live], x[live])
        exact = sums(p * (dp - delta))
        eds = p * (err * (dp.abs() + delta.abs()) + 64 * E32 * (do.abs() @ v.abs().t()
                                                              + (do.abs() * (p @ v.abs())).sum(-1, keepdim=True)))
        tol = sums(eds + nk * E32 * (p * (dp - stored)).abs())
        for cc in {wide, *exact.abs().argsort(descending=True)[:3].tolist()}:
            vals = []
            for sg in (1, -1):
                c.table = tab.clone()
                c.table[hd, cc] += sg * h
                vals.append(loss())
            c.table = tab
            num = (vals[0] - vals[1]) / (2 * h)
            mine = t.where(live & (cell == cc), p, 0.0)
            moved = float((mine * (delta - stored)).sum())
            bound = float(tol[cc]) + h * h / 6 * 1.01 * float((mine * (dp - delta)).sum(-1).abs().sum())
            got = float(dt[hd, cc])
            print(f"  head {hd} bucket {cc}: {got:.6f}, differences {num:.6f}, of the stored O {moved:.6f}, bound {bound:.1e}")
            assert bound + abs(moved) <= 0.02 * abs(num), (hd, cc)
            assert abs(got - moved - num) <= bound, (hd, cc, got, moved, num, bound)
