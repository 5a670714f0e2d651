"""GPU parity of the norm over all gradients and of their clipping, against
float64.

Tolerances: squares and sums are 64-bit, so the norm is its fp32 rounding (2^-24;
another 1e-12 for the order of the sum); the scale is rounded to fp32 once and the
product once, then the stored type: (2^-24 + 2^-24 + u) of the value, u zero for
fp32, whose product is the stored one."""
import math

import pytest

from tests._gpu_util import torch_cuda

pytestmark = pytest.mark.gpu
E = 2.0 ** -24


def _clip(t, pairs, limit, norm=True, upload=True):
    from paper_2112_00029_amd import pixelfly as pf
    G = pf.pf_grads_create(pairs)
    pf.pf_grads_upload(G)
    wsb = pf.pf_grads_workspace_bytes(G)
    ws = t.full((wsb,), 255, dtype=t.uint8, device="cuda")
    out = t.full((1,), -1.0, device="cuda") if norm else None
    pf.pf_grads_clip(G, limit, out, ws, wsb)
    return out


def _norm(t, gs):
    return math.sqrt(math.fsum(float((g.double() ** 2).sum()) for g in gs))


def _check(t, before, after, limit, norm):
    n = _norm(t, before)
    if norm is not None:
        assert abs(float(norm) - n) <= (E + 1e-12) * n, (float(norm), n)
    scale = limit / n if n > limit else 1.0
    for i, (g, a) in enumerate(zip(before, after)):
        want = g.double() * scale
        u = 0.0 if a.dtype == t.float32 else 2.0 ** -8
        tol = (u + 2.1 * E) * want.abs() + 1e-40
        if scale == 1.0 and a.dtype == g.dtype:
            tol = tol * 0
        bad = (a.double() - want).abs() - tol
        assert not (bad > 0).any(), (i, float(bad.max()))


SIZES = [1, 2, 7, 8, 9, 63, 64, 255, 256, 2047, 2048, 2049, 8191, 8192, 8193, 100003, 3]


@pytest.mark.parametrize("src", ["bf16", "fp32"])
@pytest.mark.parametrize("dst", ["same", "other", "place"])
@pytest.mark.parametrize("limit", [0.5, 1e6, 0.0])
def test_clip(src, dst, limit):
    t = torch_cuda()
    types = {"bf16": t.bfloat16, "fp32": t.float32}
    g = t.Generator(device="cuda").manual_seed(1)
    gs = [t.randn((n,), generator=g, device="cuda").to(types[src]) for n in SIZES]
    before = [x.clone() for x in gs]
    if dst == "place":
        pairs = after = gs
    else:
        to = types[src] if dst == "same" else types["fp32" if src == "bf16" else "bf16"]
        after = [t.full((n,), float("nan"), dtype=to, device="cuda") for n in SIZES]
        pairs = list(zip(gs, after))
    norm = _clip(t, pairs, limit)
    _check(t, before, after, limit, norm)
    if dst != "place":
        assert all(t.equal(x, y) for x, y in zip(gs, before))


@pytest.mark.parametrize("a,b", [(0, 0), (1, 0), (0, 1), (3, 1), (1, 5), (7, 7)])
@pytest.mark.parametrize("src,dst", [("bf16", "bf16"), ("bf16", "fp32"), ("fp32", "fp32"), ("fp32", "bf16")])
def test_slices_at_odd_places(a, b, src, dst):
    """Tensors that lie back to back in one buffer at any element; what is around
    them stays."""
    t = torch_cuda()
    types = {"bf16": t.bfloat16, "fp32": t.float32}
    g = t.Generator(device="cuda").manual_seed(3)
    sizes = [5, 4096, 1, 20001, 8192, 77]
    flat = t.randn((a + sum(sizes) + 9,), generator=g, device="cuda").to(types[src])
    out = t.full((b + sum(sizes) + 9,), 3.0, dtype=types[dst], device="cuda")
    gs, os_, i = [], [], 0
    for n in sizes:
        gs.append(flat[a + i:a + i + n])
        os_.append(out[b + i:b + i + n])
        i += n
    norm = _clip(t, list(zip(gs, os_)), 1.0)
    _check(t, gs, os_, 1.0, norm)
    assert bool((out[:b] == 3).all()) and bool((out[b + i:] == 3).all())


def test_mixed_empty_and_none():
    t = torch_cuda()
    g = t.Generator(device="cuda").manual_seed(4)
    gs = [t.randn((n,), generator=g, device="cuda").to(d) for n, d in
          ((0, t.float32), (1000, t.float32), (0, t.bfloat16), (333, t.bfloat16), (64, t.float32))]
    before = [x.clone() for x in gs]
    norm = _clip(t, gs, 1.0)
    _check(t, before, gs, 1.0, norm)
    again = [x.clone() for x in gs]
    # Already within the limit (by the rounding of the scale, just about): without a norm.
    _clip(t, gs, 2.0, norm=False)
    assert all(t.equal(x, y) for x, y in zip(gs, again))
    assert float(_clip(t, [], 1.0)) == 0.0
    z = t.zeros((70,), device="cuda")
    assert float(_clip(t, [z], 1.0)) == 0.0 and bool((z == 0).all())


@pytest.mark.parametrize("scale", [1e-30, 1e25, 3e38])
def test_very_small_and_large_gradients(scale):
    """Squares past fp32's range on both sides."""
    t = torch_cuda()
    g = t.Generator(device="cuda").manual_seed(5)
    x = (t.rand((5000,), generator=g, device="cuda") + 0.1) * (scale / 1.2)
    before = [x.clone()]
    limit = float(t.tensor(scale / 4, dtype=t.float32))
    norm = _clip(t, [x], limit)
    n = _norm(t, before)
    assert float(norm) == math.inf if n > 3.41e38 else abs(float(norm) / n - 1) <= E + 1e-12
    _check(t, before, [x], limit, None)


@pytest.mark.parametrize("limit", [1.0, 1e-3, 1e-6])
def test_scale_below_the_types_normal_numbers(limit):
    """limit / norm is 1e-40 and less: as one fp32 factor it would have lost its digits."""
    t = torch_cuda()
    g = t.Generator(device="cuda").manual_seed(6)
    for dt in (t.float32, t.bfloat16):
        x = ((t.rand((5000,), generator=g, device="cuda") + 0.1) * 3e38).to(dt)
        y = t.zeros((5000,), device="cuda")
        lim = float(t.tensor(limit, dtype=t.float32))
        before = [x.clone()]
        assert float(_clip(t, [(x, y)], lim)) == math.inf
        _check(t, before, [y], lim, None)


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_no_number_scales_nothing(bad):
    t = torch_cuda()
    x = t.randn((3000,), device="cuda")
    x[1234] = bad
    y = t.zeros((3000,), dtype=t.float32, device="cuda")
    before = x.clone()
    for pairs, after in (([x], x), ([(x, y)], y)):
        norm = _clip(t, pairs, 0.5)
        assert not math.isfinite(float(norm))
        assert t.equal(after.nan_to_num(1e30, 2e30, -2e30), before.nan_to_num(1e30, 2e30, -2e30))


def test_norm_then_scale():
    """The two halves, with another process's sum added in between."""
    t = torch_cuda()
    from paper_2112_00029_amd import pixelfly as pf
    g = t.Generator(device="cuda").manual_seed(6)
    gs = [t.randn((n,), generator=g, device="cuda") for n in (70000, 12, 8192)]
    before = [x.clone() for x in gs]
    G = pf.pf_grads_create(gs)
    pf.pf_grads_upload(G)
    wsb = pf.pf_grads_workspace_bytes(G)
    ws = t.empty((wsb,), dtype=t.uint8, device="cuda")
    sq, norm = t.zeros((1,), dtype=t.float64, device="cuda"), t.zeros((1,), device="cuda")
    pf.pf_grads_norm(G, sq, norm, ws, wsb)
    n = _norm(t, before)
    assert abs(float(sq) / n ** 2 - 1) <= 1e-12 and abs(float(norm) / n - 1) <= E + 1e-12
    assert all(t.equal(x, y) for x, y in zip(gs, before))
    first = float(sq)
    pf.pf_grads_norm(G, sq, None, ws, wsb)
    assert float(sq) == first
    sq += 3 * n ** 2
    pf.pf_grads_scale(G, 1.0, sq)
    for x, y in zip(gs, before):
        want = y.double() / (2 * n)
        assert not ((x.double() - want).abs() > 2.1 * E * want.abs()).any()


def test_many_tensors_repeats_and_graph():
    """More chunks than workgroups; repeat calls agree bitwise, captured too."""
    t = torch_cuda()
    from paper_2112_00029_amd import pixelfly as pf
    g = t.Generator(device="cuda").manual_seed(7)
    gs = [t.randn((n,), generator=g, device="cuda").bfloat16() for n in [30_000_001] + [517] * 1500]
    out = [t.zeros((x.numel(),), device="cuda") for x in gs]
    G = pf.pf_grads_create(list(zip(gs, out)))
    pf.pf_grads_upload(G)
    wsb = pf.pf_grads_workspace_bytes(G)
    ws, norm = t.empty((wsb,), dtype=t.uint8, device="cuda"), t.zeros((1,), device="cuda")
    pf.pf_grads_clip(G, 1.0, norm, ws, wsb)
    _check(t, gs, out, 1.0, norm)
    want, n0 = [o.clone() for o in out], float(norm)
    graph, st = t.cuda.CUDAGraph(), t.cuda.Stream()
    with t.cuda.graph(graph, stream=st):
        pf.pf_grads_clip(G, 1.0, norm, ws, wsb)
    for _ in range(3):
        for o in out[:3]:
            o.fill_(4.0)
        norm.zero_()
        graph.replay()
        t.cuda.synchronize()
        assert float(norm) == n0 and all(t.equal(x, y) for x, y in zip(out, want))


def test_offsets_past_32_bits():
    t = torch_cuda()
    x = t.zeros(((1 << 31) + 100,), dtype=t.bfloat16, device="cuda")
    x[-50:] = 2.0
    x[5] = 10.0
    norm = _clip(t, [x], 1.0)
    n = math.sqrt(300.0)
    assert abs(float(norm) / n - 1) <= E
    assert abs(float(x[-1]) - 2 / n) <= 2.0 ** -8 * 2 / n and abs(float(x[5]) - 10 / n) <= 2.0 ** -8 * 10 / n
    assert int((x != 0).sum()) == 51
