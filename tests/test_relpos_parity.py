"""GPU parity of block-sparse attention with a learned relative position bias
by buckets, forward and backward, against the formulas in float64.

Tolerances, derived row by row from the arithmetic (u = 2^-8, half a step of
bf16; every input is exact):
  * O = sum_j p_j v_j / sum p: each p is rounded to bf16 before the product, the
    result once more: u |O| + u (1 + u) sum_j p_j |v_j|, plus the fp32 part below;
  * the scores are fp32 sums of 64 products that start at the bias, scale sum |q k|
    below 9 and the bias below 6 for these inputs: 64 2^-24 15 = 5.8e-5, and with
    the running maximum (below 30 in log2 units: 2e-6) and the hardware
    exponential and logarithm (1 ulp) below F = 7e-5: p is off by F of itself, lse
    by F;
  * gradients: dS is rounded to bf16 before its products (u |dS|), P before dV's,
    and F (|P| (|dP| + |delta|)) for the fp32 part;
  * dtable: fp32 throughout: the fp32 part of dS only, plus n 2^-24 of sum |dS|
    for the sums."""
import numpy as np
import pytest

from tests._gpu_util import torch_cuda

pytestmark = pytest.mark.gpu

D, BLK = 64, 64
U = 2.0 ** -8
F = 7e-5


def log_map(side, n, reach, both):
    half = n // 2 if both else n
    e = half // 2
    steps = list(range(1, e + 1))
    for k in range(1, half - e):
        d = e
        while d ** (half - e) < reach ** k * e ** (half - e - k):
            d += 1
        steps.append(d)
    steps = np.array(steps[: half - 1])
    d = np.arange(-(side - 1), side)
    c = np.searchsorted(steps, np.abs(d), side="right")
    if both:
        return np.where(d > 0, half + c, c).astype(np.int32)
    return np.where(d > 0, -1, c).astype(np.int32)


def clip_map(side, reach, causal=False):
    d = np.arange(-(side - 1), side)
    c = np.clip(d, -reach, reach) + reach
    return np.where(causal & (d > 0), -1, c).astype(np.int32)


def butterfly(nb, ms, glob=0):
    x = np.arange(nb)[:, None] ^ np.arange(nb)[None, :]
    m = ((x & (x - 1)) == 0) & (x < ms)
    m[:glob] = True
    m[:, :glob] = True
    return m


class Case:
    def __init__(self, B, H, Hkv, S, bucket, nbucket, mask, lens=None, tm=False, Sq=None, starts=None,
                 seed=0, table_std=1.0, upload=True):
        t = self.t = torch_cuda()
        from paper_2112_00029_amd import pixelfly as pf
        self.pf, self.B, self.H, self.Hkv, self.S = pf, B, H, Hkv, S
        self.Sq = Sq or S
        nb = mask.shape[0]
        self.side, self.mask, self.nbucket = nb * BLK, mask, nbucket
        self.bucket = np.asarray(bucket, dtype=np.int32)
        g = t.Generator(device="cuda").manual_seed(seed)
        def rows(heads, s):
            x = t.randn((B, heads, s, D), generator=g, device="cuda").bfloat16()
            return x.transpose(1, 2).contiguous().transpose(1, 2) if tm else x
        self.q, self.do = rows(H, self.Sq), rows(H, self.Sq)
        self.k, self.v = rows(Hkv, S), rows(Hkv, S)
        self.table = t.randn((H, nbucket), generator=g, device="cuda") * table_std
        self.lens, self.starts = lens, starts
        self.scale = 0.125
        self.L = pf.pf_layout_create_from_mask(nb, nb, BLK, mask)
        self.R = pf.pf_relpos_create(self.side, nbucket, self.bucket)
        pf.pf_layout_upload(self.L)
        pf.pf_relpos_upload(self.R)
        self.bias = t.full((H, pf.pf_relpos_bias_floats(self.R)), float("nan"), device="cuda")
        pf.pf_relpos_bias(self.R, H, self.table, self.bias)
        self.wsb = pf.pf_attn_relpos_workspace_bytes(self.L, self.R, B, H, self.Sq)
        self.ws = t.full((max(self.wsb, 256),), 255, dtype=t.uint8, device="cuda")
        dev = lambda x: None if x is None else t.tensor(x, dtype=t.int32, device="cuda")
        self.dlens, self.dstarts = dev(lens), dev(starts)

    def fwd(self, q=None, k=None, v=None, o=None, stream=None):
        t = self.t
        o = t.full_like(self.q, float("nan")) if o is None else o
        lse = t.full((self.B, self.H, self.Sq), float("nan"), device="cuda")
        self.pf.pf_attn_relpos_fwd(self.L, self.R, self.scale, self.q if q is None else q,
                                   self.k if k is None else k, self.v if v is None else v, self.bias, o, lse,
                                   self.dstarts, self.dlens, self.ws, self.wsb, stream)
        return o, lse

    def bwd(self, o, lse, stream=None):
        t = self.t
        nan = lambda x: t.full_like(x, float("nan"))
        dq, dk, dv, dt = nan(self.q), nan(self.k), nan(self.v), nan(self.table)
        self.pf.pf_attn_relpos_bwd(self.L, self.R, self.scale, self.q, self.k, self.v, self.bias, o, lse,
                                   self.do, dq, dk, dv, dt, self.dlens, self.ws, self.wsb, stream)
        return dq, dk, dv, dt

    def head(self, b, h):
        """Scores (fp64, -inf where not attended), which pairs are, their bucket."""
        t = self.t
        n = self.S if self.lens is None else min(max(self.lens[b], 0), self.S)
        st = 0 if self.starts is None else min(max(self.starts[b], 0), self.side)
        pos, key = st + np.arange(self.Sq), np.arange(self.S)
        p = np.minimum(pos, self.side - 1)
        cell = self.bucket[key[None, :] - p[:, None] + self.side - 1]
        live = self.mask[p // BLK][:, key // BLK] & (cell >= 0) & (key < n)[None, :] & (pos < n)[:, None]
        live = t.from_numpy(live).cuda()
        cell = t.from_numpy(np.maximum(cell, 0).astype(np.int64)).cuda()
        hk = h // (self.H // self.Hkv)
        s = self.q[b, h].double() @ self.k[b, hk].double().t() * self.scale + self.table[h].double()[cell]
        return t.where(live, s, float("-inf")), live, cell, hk, n, t.from_numpy(pos < n).cuda()

    def check_fwd(self, o, lse):
        t = self.t
        for b in range(self.B):
            for h in range(self.H):
                s, live, _, hk, _, _ = self.head(b, h)
                ref = t.logsumexp(s, -1)
                some = live.any(-1)
                p = t.nan_to_num(t.softmax(s, -1))
                v = t.where(live.any(0)[:, None], self.v[b, hk].double(), 0.0)
                ro, mag = p @ v, p @ v.abs()
                assert t.equal(lse[b, h] == -float("inf"), ~some) and not lse.isnan().any(), (b, h)
                assert ((lse[b, h].double() - ref)[some].abs() <= F).all(), (b, h)
                bad = (o[b, h].double() - ro).abs() - (U * ro.abs() + (1 + U) * (U + 2 * F) * mag)
                assert (bad <= 0).all() and not o[b, h].isnan().any(), (b, h, float(bad.max()))
                assert (o[b, h][~some] == 0).all()

    def check_bwd(self, o, lse, dq, dk, dv, dt):
        t, G = self.t, self.H // self.Hkv
        f64 = dict(dtype=t.float64, device="cuda")
        rt, tt = t.zeros((self.H, self.nbucket), **f64), t.zeros((self.H, self.nbucket), **f64)
        for b in range(self.B):
            rk, rv = t.zeros((self.Hkv, self.S, D), **f64), t.zeros((self.Hkv, self.S, D), **f64)
            tk, tv = t.zeros_like(rk), t.zeros_like(rv)
            for h in range(self.H):
                s, live, cell, hk, n, rows = self.head(b, h)
                some = live.any(-1)
                row = t.where(some, lse[b, h].double(), 0.0)
                p = t.where(live, t.exp(s - row[:, None]), 0.0)
                do = t.where(some[:, None], self.do[b, h].double(), 0.0)
                k, v = self.k[b, hk].double(), self.v[b, hk].double()
                keys = (t.arange(self.S, device="cuda") < n)[:, None]
                k, v = t.where(keys, k, 0.0), t.where(keys, v, 0.0)
                q = t.where(some[:, None], self.q[b, h].double(), 0.0)
                delta = (do * t.where(some[:, None], o[b, h].double(), 0.0)).sum(-1, keepdim=True)
                dp = do @ v.t()
                ds = p * (dp - delta)
                # The fp32 part of dS, P off by F of itself and dP, delta by 64
                # terms' rounding.
                eds = p * (F * (dp.abs() + delta.abs()) + 64 * 2.0 ** -24 * (
                    do.abs() @ v.abs().t() + (do.abs() * o[b, h].double().nan_to_num().abs()).sum(-1, keepdim=True)))
                ads = ds.abs()
                rq, tq = ds @ k * self.scale, (U * ads + (1 + U) * eds) @ k.abs() * self.scale
                bad = (dq[b, h].double() - rq).abs() - (U * rq.abs() + (1 + U) * (tq + 1e-6 * (ads @ k.abs())))
                assert (bad <= 0).all() and not dq[b, h].isnan().any(), ("dQ", b, h, float(bad.max()))
                rk[hk] += ds.t() @ q * self.scale
                tk[hk] += (U * ads + (1 + U) * eds + 1e-6 * ads).t() @ q.abs() * self.scale
                rv[hk] += p.t() @ do
                tv[hk] += ((U + 2 * F) * p).t() @ do.abs()
                rt[h].index_add_(0, cell[live], ds[live])
                # Each bucket's sum: n terms in fp32 in a tree of sums; 4096 of
                # them in a row at most.
                tt[h].index_add_(0, cell[live], (eds + 4096 * 2.0 ** -24 * ads)[live])
            for name, got, r, tol in (("dK", dk, rk, tk), ("dV", dv, rv, tv)):
                bad = (got[b].double() - r).abs() - (U * r.abs() + (1 + U) * tol)
                assert (bad <= 0).all() and not got[b].isnan().any(), (name, b, float(bad.max()))
        bad = (dt.double() - rt).abs() - tt
        assert (bad <= 0).all() and not dt.isnan().any(), ("dtable", float(bad.max()))

    def check(self):
        o, lse = self.fwd()
        self.check_fwd(o, lse)
        out = self.bwd(o, lse)
        self.check_bwd(o, lse, *out)
        return o, lse, out


def _case(B, H, Hkv, S, kind, ms, lens=None, tm=False, glob=0, **kw):
    nb = (S + BLK - 1) // BLK
    side = nb * BLK
    mask = np.ones((nb, nb), bool) if ms == 0 else butterfly(nb, ms, min(glob, nb))
    bucket, n = {"log": (log_map(side, 32, 128, True), 32), "logc": (log_map(side, 16, 96, False), 16),
                 "far": (log_map(side, 64, max(side, 64), True), 64), "clip": (clip_map(side, 20), 41),
                 "clipc": (clip_map(side, 127, True), 255), "one": (np.zeros(2 * side - 1, np.int32), 1)}[kind]
    return Case(B, H, Hkv, S, bucket, n, mask, lens, tm, **kw)


CASES = {
    "one_token": (1, 1, 1, 1, "log", 1), "two_tokens": (2, 3, 1, 2, "clipc", 1),
    "one_block": (1, 2, 2, 64, "log", 1), "odd_65": (2, 4, 2, 65, "logc", 2),
    "butterfly_512": (2, 4, 4, 512, "log", 4), "far_buckets_640": (1, 2, 1, 640, "far", 8),
    "all_kept_300": (2, 2, 2, 300, "clip", 0), "causal_all_kept_449": (1, 4, 1, 449, "clipc", 0),
    "one_bucket_256": (1, 2, 2, 256, "one", 4), "stripe_1000": (1, 3, 3, 1000, "log", 4, None, True, 1),
    "lens": (4, 4, 2, 500, "log", 0, [500, 0, 1, 191]), "lens_causal": (3, 8, 2, 700, "logc", 8, [64, 700, 333], True),
    "lens_clamped": (3, 2, 2, 130, "clip", 2, [-5, 1 << 30, 128], True), "stripe_lens": (2, 2, 1, 1024, "clipc", 2, [900, 65], False, 2),
}


@pytest.mark.parametrize("name", CASES)
def test_whole_sequences(name):
    print(f"[relpos] {name} {CASES[name]}", flush=True)
    _case(*CASES[name]).check()


# Lists shared by several workgroups and joined: few blocks of long lists, long
# columns and rows of stripes, grouped heads; parts that get nothing.
SPLIT = {
    "all_kept_1300": (1, 2, 2, 1300, "log", 0), "causal_1411": (1, 4, 1, 1411, "clipc", 0, [1300], True),
    "stripe_1700": (2, 4, 2, 1700, "log", 2, [1700, 900], True, 1), "stripe_causal_1700": (1, 4, 1, 1700, "logc", 4, None, False, 2),
    "grouped_1100": (1, 8, 1, 1100, "log", 2), "short_lens_1300": (2, 2, 1, 1300, "clip", 0, [20, 0]),
    "all_stripes_1216": (1, 2, 2, 1216, "log", 1, None, False, 19),
}


@pytest.mark.parametrize("name", SPLIT)
def test_lists_in_parts(name):
    print(f"[relpos] {name} {SPLIT[name]}", flush=True)
    _case(*SPLIT[name]).check()


@pytest.mark.parametrize("H,Hkv,kind,ms,glob", [(8, 2, "logc", 0, 0), (4, 4, "clip", 0, 0), (32, 1, "log", 0, 0),
                                                (33, 1, "logc", 0, 0), (3, 3, "log", 4, 1), (40, 1, "log", 4, 0)])
def test_one_row_against_long_caches(H, Hkv, kind, ms, glob):
    lens = [1500, 1, 64, 65, 777, 1024, 0, 3]
    starts = [1499, 0, 63, 64, 776, 700, 5, 2]
    c = _case(8, H, Hkv, 1500, kind, ms, lens=lens, Sq=1, starts=starts, tm=True, glob=glob)
    c.check_fwd(*c.fwd())
    # Without q_start the one row is the first.
    c.dstarts = c.starts = None
    c.check_fwd(*c.fwd())


@pytest.mark.parametrize("rows", [2, 64, 130])
def test_few_rows_against_long_caches(rows):
    lens = [1500, 140, 200]
    c = _case(3, 4, 2, 1500, "logc", 0, lens=lens, Sq=rows, starts=[1500 - rows, 140 - rows, 10])
    c.check_fwd(*c.fwd())


def test_long_sequence():
    c = _case(1, 2, 1, 4096, "log", 64)
    c.check()


def test_map_of_any_shape():
    """Buckets in no order, masked distances in between, blocks wholly masked."""
    g = np.random.default_rng(5)
    side = 384
    b = g.integers(-1, 256, 2 * side - 1)
    b[100:260] = -1
    b[side - 1] = 3
    Case(2, 2, 1, 380, b, 256, np.ones((6, 6), bool), lens=[380, 200]).check()


def test_rows_that_attend_to_nothing():
    """A map that leaves out distance 0 and the near ones, blocks of the
    diagonal alone: most rows are empty, or all."""
    side = 256
    d = np.arange(-(side - 1), side)
    b = np.where((d >= -40) & (d < 63), -1, 0).astype(np.int32)
    o, lse, _ = Case(2, 2, 2, 250, b, 1, np.eye(4, dtype=bool), lens=[250, 30]).check()
    assert (lse == -float("inf")).any() and (lse[0] > -float("inf")).any()
    o, lse, (dq, dk, dv, dt) = Case(1, 2, 2, 250, np.full(2 * side - 1, -1), 4, np.eye(4, dtype=bool)).check()
    assert (lse == -float("inf")).all() and not (dq.any() or dk.any() or dv.any() or dt.any())


@pytest.mark.parametrize("low", [-float("inf"), -3.4028234e38])
def test_table_entries_that_mask(low):
    """Causal by the table: the bucket of every key after the query holds -inf,
    or the lowest fp32 value: the same bits as a map that leaves them out."""
    side = 320
    m = clip_map(side, 30)
    a = Case(2, 4, 2, 300, m, 61, np.ones((5, 5), bool), lens=[300, 100])
    b = Case(2, 4, 2, 300, np.where(np.arange(-(side - 1), side) > 0, -1, m), 61, np.ones((5, 5), bool),
             lens=[300, 100])
    a.table[:, 31:] = low
    b.table.copy_(a.table)
    for c in (a, b):
        c.pf.pf_relpos_bias(c.R, c.H, c.table, c.bias)
    oa, la = a.fwd()
    ob, lb = b.fwd()
    assert a.t.equal(oa, ob) and a.t.equal(la, lb)
    ga, gb = a.bwd(oa, la), b.bwd(ob, lb)
    for x, y in zip(ga[:3], gb[:3]):
        assert a.t.equal(x, y)
    assert not ga[3][:, 31:].any() and a.t.allclose(ga[3], gb[3], rtol=1e-4, atol=1e-4)


def test_garbage_past_the_tokens_is_not_used():
    c = _case(2, 4, 2, 300, "log", 0, lens=[130, 257], tm=True)
    o, lse = c.fwd()
    out = c.bwd(o, lse)
    for b, n in enumerate(c.lens):
        for x in (c.q, c.k, c.v, c.do):
            x[b, :, n:] = float("nan")
    o2, lse2 = c.fwd()
    for b, n in enumerate(c.lens):
        o2[b, :, n:] = float("inf")
        lse2[b, :, n:] = float("nan")
    out2 = c.bwd(o2, lse2)
    for b, n in enumerate(c.lens):
        assert c.t.equal(o[b, :, :n], o2[b, :, :n]) and c.t.equal(lse[b, :, :n], lse2[b, :, :n])
    for x, y in zip(out, out2):
        assert c.t.equal(x, y)


def test_strides_of_one_projection():
    """Q, K and V as views of one (B, S, H + 2 H_kv, 64) tensor, gradients into
    another: the bits of the separate tensors, and nothing else is written."""
    c = _case(2, 4, 2, 333, "clip", 2, lens=[333, 70])
    t, B, H, Hk, S = c.t, 2, 4, 2, 333
    o, lse = c.fwd()
    dq, dk, dv, dt = c.bwd(o, lse)
    qkv = t.full((B, S + 3, H + 2 * Hk + 1, D), 7.0, device="cuda").bfloat16()
    grad = qkv.clone()
    cut = lambda x: (x[:, :S, :H].transpose(1, 2), x[:, :S, H:H + Hk].transpose(1, 2),
                     x[:, :S, H + Hk:H + 2 * Hk].transpose(1, 2))
    for dst, src in zip(cut(qkv), (c.q, c.k, c.v)):
        dst.copy_(src)
    c.q, c.k, c.v = cut(qkv)
    o2 = t.full((B, S, H, D), 0.0, device="cuda").bfloat16().transpose(1, 2)
    _, lse2 = c.fwd(o=o2)
    assert t.equal(o, o2) and t.equal(lse, lse2)
    gq, gk, gv = cut(grad)
    dt2 = t.empty_like(dt)
    c.pf.pf_attn_relpos_bwd(c.L, c.R, c.scale, c.q, c.k, c.v, c.bias, o2, lse2, c.do, gq, gk, gv, dt2, c.dlens,
                            c.ws, c.wsb)
    for x, y in ((dq, gq), (dk, gk), (dv, gv), (dt, dt2)):
        assert t.equal(x, y)
    assert (grad[:, S:] == 7).all() and (grad[:, :, H + 2 * Hk:] == 7).all()


def test_offsets_past_32_bits():
    """Sequences 2^32 and heads 2^31 elements apart, of inputs and outputs: the
    bits of the separate tensors (whole sequences, and one row of each)."""
    for rows, starts in ((None, None), (1, [269, 99])):
        c = _case(2, 2, 2, 270, "log", 2, lens=[270, 100], Sq=rows, starts=starts)
        t = c.t
        if rows is None:
            big = t.empty((1 << 32) + (1 << 31) + (1 << 24), dtype=t.bfloat16, device="cuda")
        n = [0]
        def far(x):
            v = t.as_strided(big, tuple(x.shape), (1 << 32, 1 << 31, D, 1), n[0])
            n[0] += 1 << 20
            return v.copy_(x)
        o, lse = c.fwd()
        nan = t.full_like(o, float("nan"))
        q, k, v, o2 = far(c.q), far(c.k), far(c.v), far(nan)
        _, lse2 = c.fwd(q=q, k=k, v=v, o=o2)
        assert t.equal(o, o2) and t.equal(lse, lse2)
        if rows is None:
            grads = c.bwd(o, lse)
            far_grads = far(nan), far(nan), far(nan), t.empty_like(grads[3])
            c.pf.pf_attn_relpos_bwd(c.L, c.R, c.scale, q, k, v, c.bias, o2, lse2, far(c.do), *far_grads, c.dlens,
                                    c.ws, c.wsb)
            for x, y in zip(grads, far_grads):
                assert t.equal(x, y)


def test_strides_of_single_dimensions():
    """Strides of a dimension of one (any number, as views have them) do not
    matter."""
    c = _case(1, 1, 1, 1, "log", 0)
    odd = lambda x: c.t.as_strided(x, (1, 1, 1, D), (3, 5, 7, 1))
    o, lse = c.fwd()
    o2 = c.t.empty_like(o)
    c.q, c.k, c.v = odd(c.q), odd(c.k), odd(c.v)
    _, lse2 = c.fwd(o=odd(o2))
    assert c.t.equal(o, o2) and c.t.equal(lse, lse2)


def test_broadcast_keys_and_values():
    """One sequence's keys and values for the whole batch (stride 0)."""
    c = _case(3, 2, 2, 200, "log", 0)
    k, v = c.k[:1].expand(3, -1, -1, -1), c.v[:1].expand(3, -1, -1, -1)
    o, lse = c.fwd(k=k, v=v)
    o2, lse2 = c.fwd(k=k.contiguous(), v=v.contiguous())
    assert c.t.equal(o, o2) and c.t.equal(lse, lse2)


@pytest.mark.parametrize("rows,starts,lens", [
    (1, [0, 63, 64, 299], [1, 64, 65, 300]), (1, [299, 0, 5, 100], [300, 300, 0, 80]),
    (5, [0, 60, 127, 290], [5, 65, 132, 295]), (70, [0, 1, 63, 230], [70, 71, 133, 300]),
    (200, [0, 100, 64, 33], [200, 300, 264, 233]), (1, [-3, 320, 1 << 30, 10], [300, 300, 300, 1 << 30])])
@pytest.mark.parametrize("kind,ms", [("logc", 0), ("log", 4)])
def test_newest_rows(rows, starts, lens, kind, ms):
    c = _case(4, 4, 2, 300, kind, ms, lens=lens, Sq=rows, starts=starts, tm=True)
    o, lse = c.fwd()
    c.check_fwd(o, lse)


def test_newest_rows_are_the_rows_of_the_whole():
    """A sequence's rows in chunks against its cache: the whole call's results
    within the rounding of P (the order of the blocks is the same)."""
    c = _case(1, 4, 2, 400, "logc", 4)
    o, lse = c.fwd()
    for st, n in ((0, 64), (64, 100), (164, 1), (165, 235)):
        d = _case(1, 4, 2, 400, "logc", 4, Sq=n, starts=[st], lens=[st + n])
        d.k, d.v, d.q = c.k, c.v, c.q[:, :, st:st + n]
        d.table.copy_(c.table)
        d.pf.pf_relpos_bias(d.R, 4, d.table, d.bias)
        o2 = c.t.empty_like(d.q)
        _, lse2 = d.fwd(o=o2)
        assert (lse2 - lse[:, :, st:st + n]).abs().max() <= 2 * F
        assert (o2.double() - o[:, :, st:st + n].double()).abs().max() <= 2 * (U * 4.8 + (1 + U) * (U + 2 * F) * 4.8)


def test_gradient_against_differences():
    """dtable by central differences of <dO, O> in float64 over the table."""
    c = _case(1, 2, 1, 130, "clip", 2, lens=[120])
    t = c.t
    o, lse = c.fwd()
    _, _, _, dt = c.bwd(o, lse)
    tab = c.table.double()

    def loss(h):
        s, _, _, hk, _, _ = c.head(0, h)
        p = t.nan_to_num(t.softmax(s, -1))
        return float((p @ c.v[0, hk].double() * c.do[0, h].double()).sum())

    # The kernel's delta takes O in bf16 from probabilities in bf16: off by u
    # sum_d |dO| (|O| + sum_j p |v|) a row, times the row's probability of the
    # bucket; the fp32 part as above; differences of step h: h^2 / 6 of the third
    # derivative, at most 6 sum p |dP - delta|.
    for hd, cc in ((0, 20), (1, 0), (0, 40), (1, 33)):
        vals, h = [], 1e-3
        for sg in (1, -1):
            c.table = tab.clone()
            c.table[hd, cc] += sg * h
            vals.append(loss(hd))
        c.table = tab
        s, live, cell, hk, _, _ = c.head(0, hd)
        p = t.nan_to_num(t.softmax(s, -1))
        v, do = c.v[0, hk].double(), c.do[0, hd].double()
        mine = t.where(live & (cell == cc), p, 0.0).sum(-1)
        row = (do.abs() * ((p @ v).abs() + p @ v.abs())).sum(-1)
        big = (p * ((do @ v.t()).abs() + row[:, None])).sum()
        tol = float((mine * row).sum()) * (U + F) + float(big) * (h * h + F)
        num = (vals[0] - vals[1]) / (2 * h)
        assert abs(num - float(dt[hd, cc])) <= tol, (hd, cc, num, float(dt[hd, cc]), tol)


def test_repeat_streams_graph():
    """Bitwise repeatable, on a side stream, and captured once and replayed with
    the program's own work in between (lengths change between replays)."""
    c = _case(2, 4, 2, 500, "log", 4, lens=[500, 300])
    t = c.t
    o, lse = c.fwd()
    ref = (o, lse, *c.bwd(o, lse))
    t.cuda.synchronize()
    side = t.cuda.Stream()
    side.wait_stream(t.cuda.current_stream())
    with t.cuda.stream(side):
        o1, l1 = c.fwd()
        again = (o1, l1, *c.bwd(o1, l1))
    side.synchronize()
    for x, y in zip(ref, again):
        assert t.equal(x, y)
    bufs = [t.empty_like(x) for x in ref]
    o, lse, dq, dk, dv, dt = bufs
    graph = t.cuda.CUDAGraph()
    with t.cuda.graph(graph):
        c.pf.pf_relpos_bias(c.R, 4, c.table, c.bias)
        c.pf.pf_attn_relpos_fwd(c.L, c.R, c.scale, c.q, c.k, c.v, c.bias, o, lse, None, c.dlens, c.ws, c.wsb)
        c.pf.pf_attn_relpos_bwd(c.L, c.R, c.scale, c.q, c.k, c.v, c.bias, o, lse, c.do, dq, dk, dv, dt, c.dlens,
                                c.ws, c.wsb)
    tab = c.table.clone()
    for i in range(4):
        c.dlens.copy_(t.tensor([500, 300] if i % 2 == 0 else [77, 500], dtype=t.int32))
        c.table.copy_(tab if i % 2 == 0 else -tab)
        for x in bufs:
            x.fill_(float("nan"))
        graph.replay()
        t.cuda.synchronize()
        want = ref
        if i % 2:
            oo, ll = c.fwd()
            want = (oo, ll, *c.bwd(oo, ll))
        for x, y in zip(bufs, want):
            assert t.equal(x, y), i


def test_binding_checks_tensors():
    c = _case(1, 2, 2, 64, "log", 1)
    t, o = c.t, c.q.clone()
    lse = t.empty((1, 2, 64), device="cuda")
    call = lambda **k: c.pf.pf_attn_relpos_fwd(c.L, c.R, c.scale, k.get("q", c.q), k.get("k", c.k), c.v,
                                               k.get("bias", c.bias), o, k.get("lse", lse), k.get("st"), k.get("n"))
    call()
    for k, bad in (("q", c.q.float()), ("k", c.k[:, :, :32]), ("bias", c.bias[:1]), ("bias", c.bias.double()),
                   ("lse", lse[:, :1]), ("st", t.zeros(1, dtype=t.int64, device="cuda")),
                   ("n", t.zeros(1, dtype=t.int32)), ("n", t.zeros(0, dtype=t.int32, device="cuda"))):
        with pytest.raises(ValueError):
            call(**{k: bad})
    with pytest.raises(ValueError, match="contiguous"):
        call(q=c.q.transpose(2, 3))


def test_two_calls_at_once():
    """Two streams, a workspace each: the bits of the calls one by one."""
    a, b = _case(2, 4, 2, 500, "log", 4, lens=[500, 300]), _case(1, 4, 1, 1411, "clipc", 0, [1300], True)
    t = a.t
    want = []
    for c in (a, b):
        o, lse = c.fwd()
        want.append((o, lse, *c.bwd(o, lse)))
    t.cuda.synchronize()
    streams, got = [t.cuda.Stream(), t.cuda.Stream()], [None, None]
    for _ in range(3):
        for i, c in enumerate((a, b)):
            with t.cuda.stream(streams[i]):
                o, lse = c.fwd()
                got[i] = (o, lse, *c.bwd(o, lse))
        t.cuda.synchronize()
        for x, y in zip(want[0] + want[1], got[0] + got[1]):
            assert t.equal(x, y)
