"""A training step of a pre-norm gated feed-forward block as a program runs it: layer
normalisation, the gated layer, the layer back with bias and residual; their way back;
all gradients clipped.  Against float64 autograd of the formulas, eager and as one
captured graph.

Tolerance: relative to the whole tensor.  Of the roundings on the way to any one
tensor (the normalised rows, T_lr, Z, H, the second T_lr and Y; dH, S, dZ, S, the
input's gradient, the gradient itself) none is passed on with more than its own
relative size, and there are twelve: 12 u, u = finfo(t).eps / 2.  fp32 adds its sums'
errors, at most 1024 terms deep here: 1024 u."""
import math

import numpy as np
import pytest

from tests._gpu_util import torch_cuda
from tests.test_act_parity import _act, _mask

pytestmark = pytest.mark.gpu
EPS = 1e-5


class Step:
    def __init__(self, dtype, T, D, F, b, ms, r, act, seed=0):
        t = self.t = torch_cuda()
        from paper_2112_00029_amd import pixelfly as pf
        self.pf, self.dtype, self.act = pf, dtype, act
        self.T, self.D, self.F, self.b, self.ms, self.r = T, D, F, b, ms, r
        dt = self.dt = t.bfloat16 if dtype == "bf16" else t.float32
        g = t.Generator(device="cuda").manual_seed(seed)
        rnd = lambda shape, std=1.0: t.randn(shape, generator=g, device="cuda").mul_(std).to(dt)
        self.x, self.G = rnd((T, D)), rnd((T, D))
        n1, n2 = (int(_mask(*s, ms).sum()) for s in ((F // b, D // b), (D // b, F // b)))
        f1, f2 = n1 / (F // b) * b, n2 / (D // b) * b
        self.p = {"ln_w": (1 + rnd((D,), 0.2).float()).to(dt), "ln_b": rnd((D,), 0.2),
                  "w1": rnd((2 * n1, b, b), f1 ** -0.5), "u1": rnd((2 * F, r), 0.5 * r ** -0.5), "v1": rnd((r, D), D ** -0.5),
                  "b1": rnd((2 * F,), 0.2),
                  "w2": rnd((n2, b, b), f2 ** -0.5), "u2": rnd((D, r), 0.5 * r ** -0.5), "v2": rnd((r, F), F ** -0.5),
                  "b2": rnd((D,), 0.2)}
        self.g = {k: t.full_like(v, float("nan")) for k, v in self.p.items()}
        self.L1, self.L2 = pf.pf_layout_create_gated(F, D, b, ms), pf.pf_layout_create(D, F, b, ms)
        for L in (self.L1, self.L2):
            pf.pf_layout_upload(L)
        e = lambda *s: t.full(s, float("nan"), dtype=dt, device="cuda")
        self.n, self.h, self.z, self.t1, self.t2, self.y = e(T, D), e(T, F), e(T, 2 * F), e(T, r), e(T, r), e(T, D)
        self.mean, self.rstd = t.empty((T,), device="cuda"), t.empty((T,), device="cuda")
        self.s1, self.s2, self.dh, self.dz, self.dn, self.dx = e(T, r), e(T, r), e(T, F), e(T, 2 * F), e(T, D), e(T, D)
        # The optimizer's fp32 gradients: one buffer, back to back.
        sizes = [v.numel() for v in self.g.values()]
        self.flat = t.full((sum(sizes),), float("nan"), device="cuda")
        self.parts = dict(zip(self.g, self.flat.split(sizes)))
        self.grads = pf.pf_grads_create([(self.g[k].view(-1), self.parts[k]) for k in self.g])
        pf.pf_grads_upload(self.grads)
        self.norm = t.zeros((1,), device="cuda")
        self.wsb = max(pf.pf_workspace_bytes(self.L1, T, r, dtype), pf.pf_workspace_bytes(self.L2, T, r, dtype),
                       pf.pf_linear_gated_workspace_bytes(dtype, T, F), pf.pf_linear_act_workspace_bytes(dtype, T, D),
                       pf.pf_layernorm_workspace_bytes(dtype, T, D), pf.pf_grads_workspace_bytes(self.grads))
        self.ws = t.empty((self.wsb,), dtype=t.uint8, device="cuda")

    def outputs(self):
        return dict(y=self.y, dx=self.dx, norm=self.norm, flat=self.flat, **self.g)

    def run(self, limit):
        """One step; every call shares one workspace, as they follow one another."""
        pf, dt, T, D, F, b, r, p, g = (self.pf, self.dtype, self.T, self.D, self.F, self.b, self.r, self.p, self.g)
        act = getattr(pf, "PF_ACT_" + self.act.upper())
        ws = dict(workspace=self.ws, ws_bytes=self.wsb)
        pf.pf_layernorm_fwd(dt, T, D, EPS, self.x, D, p["ln_w"], p["ln_b"], self.n, D, self.mean, self.rstd)
        pf.pf_linear_gated_fwd(self.L1, dt, T, r, self.n, p["w1"], p["u1"], p["v1"], p["b1"], act, self.h, self.z,
                               self.t1, **ws)
        pf.pf_linear_fwd_act(self.L2, dt, T, r, self.h, p["w2"], p["u2"], p["v2"], p["b2"], pf.PF_ACT_NONE, self.x,
                             self.y, None, self.t2, **ws)
        # Way back.
        pf.pf_linear_act_bwd(dt, T, D, pf.PF_ACT_NONE, self.G, None, None, g["b2"], **ws)
        pf.pf_linear_bwd_data(self.L2, dt, T, r, self.G, p["w2"], p["u2"], p["v2"], self.s2, self.dh, **ws)
        pf.pf_linear_bwd_weight(self.L2, dt, T, r, self.G, self.h, self.t2, self.s2, g["w2"], g["u2"], g["v2"], **ws)
        pf.pf_linear_gated_bwd(dt, T, F, b, act, self.dh, self.z, self.dz, g["b1"], **ws)
        pf.pf_linear_bwd_data(self.L1, dt, T, r, self.dz, p["w1"], p["u1"], p["v1"], self.s1, self.dn, **ws)
        pf.pf_linear_bwd_weight(self.L1, dt, T, r, self.dz, self.n, self.t1, self.s1, g["w1"], g["u1"], g["v1"], **ws)
        pf.pf_layernorm_bwd(dt, T, D, self.dn, D, self.x, D, p["ln_w"], self.mean, self.rstd, self.G, D, self.dx, D,
                            g["ln_w"], g["ln_b"], **ws)
        pf.pf_grads_clip(self.grads, limit, self.norm, **ws)

    def reference(self):
        t, b = self.t, self.b
        p = {k: v.double().requires_grad_(True) for k, v in self.p.items()}
        x = self.x.double().requires_grad_(True)

        def dense(w, rows, cols, twice):
            m = _mask(rows // b, cols // b, self.ms)
            i, j = np.nonzero(np.repeat(m, 2, axis=0) if twice else m)
            W = t.zeros(((1 + twice) * rows // b, cols // b, b, b), dtype=t.float64, device="cuda")
            W = W.index_put((t.from_numpy(i).cuda(), t.from_numpy(j).cuda()), w)
            return W.permute(0, 2, 1, 3).reshape((1 + twice) * rows, cols)

        d = x - x.mean(1, keepdim=True)
        n = d * ((d * d).mean(1, keepdim=True) + EPS) ** -0.5 * p["ln_w"] + p["ln_b"]
        z = n @ dense(p["w1"], self.F, self.D, 1).t() + (n @ p["v1"].t()) @ p["u1"].t() + p["b1"]
        a, v = z.view(self.T, self.F // b, 2, b).unbind(2)
        h = (_act(t, a, self.act) * v).reshape(self.T, self.F)
        y = x + h @ dense(p["w2"], self.D, self.F, 0).t() + (h @ p["v2"].t()) @ p["u2"].t() + p["b2"]
        grads = t.autograd.grad((y * self.G.double()).sum(), [x, *p.values()])
        return y.detach(), dict(zip(["dx", *p], grads))


@pytest.mark.parametrize("dtype,T,D,F,b,ms,r,act", [
    ("fp32", 70, 128, 192, 32, 4, 32, "gelu"), ("fp32", 300, 256, 512, 64, 4, 64, "silu"),
    ("bf16", 130, 256, 512, 64, 4, 64, "silu"), ("bf16", 1000, 512, 1024, 32, 8, 32, "gelu_tanh"),
    ("bf16", 2300, 512, 1024, 128, 4, 128, "gelu"), ("bf16", 4200, 1024, 1024, 32, 16, 64, "silu")])
def test_step(dtype, T, D, F, b, ms, r, act):
    s = Step(dtype, T, D, F, b, ms, r, act)
    t = s.t
    s.run(1.0)
    y, ref = s.reference()
    u = t.finfo(s.dt).eps / 2
    tol = 12 * u if dtype == "bf16" else 1036 * u
    rel = lambda a, b: float((a.double().reshape(b.shape) - b).norm() / b.norm())
    assert rel(s.y, y) <= tol, rel(s.y, y)
    assert rel(s.dx, ref["dx"]) <= tol
    for k, v in s.g.items():
        assert rel(v, ref[k]) <= tol, (k, rel(v, ref[k]))
    # The norm is that of the gradients as they are stored, the copies theirs cut.
    norm = math.sqrt(sum(float((v.double() ** 2).sum()) for v in s.g.values()))
    assert abs(float(s.norm) / norm - 1) <= 2.0 ** -23 and norm > 1
    for k, v in s.g.items():
        want = v.double().view(-1) / norm
        assert not ((s.parts[k].double() - want).abs() > 2.1 * 2.0 ** -24 * want.abs()).any(), k
    assert abs(float(s.flat.double().norm()) - 1) < 1e-6


def test_captured_step():
    """The whole step as one graph, replayed with eager work between."""
    s = Step("bf16", 400, 256, 512, 32, 4, 32, "silu")
    t = s.t
    s.run(0.5)
    want = {k: v.clone() for k, v in s.outputs().items()}
    st, graph = t.cuda.Stream(), t.cuda.CUDAGraph()
    with t.cuda.graph(graph, stream=st):
        s.run(0.5)
    for i in range(4):
        for v in s.outputs().values():
            v.fill_(5.0)
        s.ws.fill_(i)
        graph.replay()
        t.cuda.synchronize()
        for k, v in s.outputs().items():
            assert t.equal(v, want[k]), (i, k)
        s.run(0.5)
        t.cuda.synchronize()
        assert all(t.equal(v, want[k]) for k, v in s.outputs().items())
