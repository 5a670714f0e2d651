"""Argument checks of the gated layer, layer normalisation and gradient clipping, on
the host: every refused call enqueues nothing, so plain integers stand in for device
addresses; and what a gated layout holds."""
import struct

import numpy as np
import pytest
import torch

from paper_2112_00029_amd import pixelfly as pf
from tests.test_block_host import A, _refused


@pytest.fixture(scope="module")
def layout():
    return pf.pf_layout_create_gated(512, 256, 64, 4)


# ---- gated layouts ----------------------------------------------------------

@pytest.mark.parametrize("N,K,b,ms", [(512, 256, 64, 4), (256, 512, 32, 8), (1024, 256, 128, 2), (416, 320, 32, 8),
                                      (32, 32, 32, 1), (768, 224, 32, 16), (640, 1920, 128, 16)])
def test_gated_layout_is_the_mask_twice(N, K, b, ms):
    one, two = (pf.pf_layout_info_get(f(N, K, b, ms)) for f in (pf.pf_layout_create, pf.pf_layout_create_gated))
    assert two["n_out"] == 2 * N and two["n_in"] == K and two["nnzb"] == 2 * one["nnzb"]
    rows = lambda i: [list(i["col_idx"][i["row_ptr"][r]:i["row_ptr"][r + 1]]) for r in range(i["nb_out"])]
    a, g = rows(one), rows(two)
    assert g[0::2] == a and g[1::2] == a
    L = pf.pf_layout_create_gated(N, K, b, ms)
    pf.pf_layout_check(L)
    # Every tile holds whole pairs: its rows come in even numbers.
    plan = pf.pf_layout_plan_get(L)
    assert b == 128 or plan["G_fwd"] % 2 == 0, plan


def test_gated_layout_from_mask():
    rng = np.random.default_rng(1)
    m = rng.random((9, 5)) < 0.5
    m[:, 2] = True
    g = pf.pf_layout_info_get(pf.pf_layout_create_gated_from_mask(9, 5, 64, m))
    assert g["nb_out"] == 18 and g["nnzb"] == 2 * m.sum()
    for r in range(18):
        assert list(g["col_idx"][g["row_ptr"][r]:g["row_ptr"][r + 1]]) == list(np.flatnonzero(m[r // 2]))
    m[4] = False
    with pytest.raises(pf.PixelflyError):
        pf.pf_layout_create_gated_from_mask(9, 5, 64, m)
    with pytest.raises(ValueError):
        pf.pf_layout_create_gated_from_mask(5, 9, 64, m)


@pytest.mark.parametrize("a", [(512, 256, 64, 3), (500, 256, 64, 4), (512, 250, 64, 4), (0, 256, 64, 4), (512, 256, 0, 4)])
def test_gated_layout_refusals(a):
    with pytest.raises(pf.PixelflyError) as e:
        pf.pf_layout_create_gated(*a)
    assert e.value.status == pf.PF_ERR_INVALID_ARG


# ---- gated forward and way back ---------------------------------------------

def _fwd(layout, **kw):
    d = dict(dtype="bf16", T=8, r=64, X=A, Wblk=A, U=A, V=A, bias=A, act=pf.PF_ACT_GELU, H=A, Z=A, T_lr=A,
             workspace=A, ws_bytes=1 << 30)
    d.update(kw)
    return (layout, *d.values())


@pytest.mark.parametrize("kw,text", [
    (dict(act=5), "bad activation"), (dict(act=-1), "bad activation"), (dict(bias=A + 2), "bias is not 16-byte"),
    (dict(Z=A + 4), "Z is not 16-byte"), (dict(H=None), "H is NULL"), (dict(H=A + 8), "H is not 16-byte"),
    (dict(X=None), "X is NULL"), (dict(Wblk=None), "Wblk is NULL"), (dict(T=0), "T must be"),
    (dict(r=32), "multiple of b"), (dict(r=-64), "multiple of b"), (dict(U=None), "U is NULL"),
    (dict(V=None), "V is NULL"), (dict(T_lr=None), "T_lr is NULL"), (dict(dtype=7), "bad dtype")])
def test_gated_forward_refusals(layout, kw, text):
    _refused(pf.PF_ERR_INVALID_ARG, text, pf.pf_linear_gated_fwd, *_fwd(layout, **kw))


def test_gated_forward_state_layout_and_gamma(layout):
    _refused(pf.PF_ERR_STATE, "not uploaded", pf.pf_linear_gated_fwd, *_fwd(layout))
    _refused(pf.PF_ERR_STATE, "not uploaded", pf.pf_linear_gated_fwd,
             *_fwd(layout, Z=None, bias=None, act=pf.PF_ACT_NONE, r=0, U=None, V=None, T_lr=None))
    other = pf.pf_layout_create(1024, 256, 64, 4)  # of the same size
    _refused(pf.PF_ERR_INVALID_ARG, "not a gated layout", pf.pf_linear_gated_fwd, *_fwd(other))
    _refused(pf.PF_ERR_UNSUPPORTED, "b in", pf.pf_linear_gated_fwd, *_fwd(pf.pf_layout_create_gated(64, 64, 16, 4)))
    a = _fwd(layout)
    for g in (float("nan"), float("inf")):
        _refused(pf.PF_ERR_INVALID_ARG, "gamma", pf.pf_linear_gated_fwd_mixed, *a[:4], g, *a[4:])
    # (1500 x 8192 to rank 256: T_lr is split.)
    big = pf.pf_layout_create_gated(256, 16384, 128, 2)
    need = pf.pf_workspace_bytes(big, 16384, 256, "fp32")
    assert need > 0
    a = _fwd(big, dtype="fp32", T=500, r=256, workspace=None, ws_bytes=0)
    with pytest.raises(pf.PixelflyError) as e:
        pf.pf_linear_gated_fwd(*a, stream=0)
    assert e.value.status in (pf.PF_ERR_WORKSPACE, pf.PF_ERR_STATE)


@pytest.mark.parametrize("dtype,T,K", [("bf16", 4096, 4096), ("bf16", 16384, 16384), ("fp32", 4096, 16384)])
def test_gated_forward_workspace(dtype, T, K):
    """Where T_lr's K list is split over workgroups (and has no kernel without a split),
    its fp32 partial sums are what the call needs; refused before the layout's state."""
    L, r = pf.pf_layout_create_gated(256, K, 128, 2), 256
    plan = pf.pf_linear_plan_get(L, dtype, T, r)
    need = plan["lowrank_t_split"] * T * r * 4
    assert plan["lowrank_t_split"] > 1 and need <= pf.pf_workspace_bytes(L, T, r, dtype)
    a = dict(dtype=dtype, T=T, r=r)
    _refused(pf.PF_ERR_WORKSPACE, f"workspace needs {need} bytes", pf.pf_linear_gated_fwd, *_fwd(L, **a, ws_bytes=need - 1))
    _refused(pf.PF_ERR_WORKSPACE, f"workspace needs {need} bytes", pf.pf_linear_gated_fwd,
             *_fwd(L, **a, workspace=None, ws_bytes=0))
    _refused(pf.PF_ERR_INVALID_ARG, "workspace is NULL", pf.pf_linear_gated_fwd, *_fwd(L, **a, workspace=None, ws_bytes=need))
    _refused(pf.PF_ERR_INVALID_ARG, "workspace is not", pf.pf_linear_gated_fwd, *_fwd(L, **a, workspace=A + 8, ws_bytes=need))
    _refused(pf.PF_ERR_STATE, "not uploaded", pf.pf_linear_gated_fwd, *_fwd(L, **a, ws_bytes=need))
    b = _fwd(L, **a, ws_bytes=need - 1)
    _refused(pf.PF_ERR_WORKSPACE, "workspace needs", pf.pf_linear_gated_fwd_mixed, *b[:4], 0.5, *b[4:])


def _bwd(**kw):
    d = dict(dtype="bf16", T=64, N=512, b=64, act=pf.PF_ACT_SILU, dH=A, Z=A, dZ=A, dbias=A, workspace=A,
             ws_bytes=1 << 30)
    d.update(kw)
    return d


@pytest.mark.parametrize("status,kw,text", [
    (pf.PF_ERR_INVALID_ARG, dict(act=9), "bad activation"), (pf.PF_ERR_INVALID_ARG, dict(T=0), "T must be"),
    (pf.PF_ERR_INVALID_ARG, dict(T=(1 << 30) + 1), "T must be"),
    (pf.PF_ERR_INVALID_ARG, dict(N=40), "multiple of 32"), (pf.PF_ERR_INVALID_ARG, dict(N=0), "multiple of 32"),
    (pf.PF_ERR_INVALID_ARG, dict(N=(1 << 24) + 64), "multiple of 32"),
    (pf.PF_ERR_UNSUPPORTED, dict(b=16), "b in"), (pf.PF_ERR_INVALID_ARG, dict(N=544), "b must divide"),
    (pf.PF_ERR_INVALID_ARG, dict(dtype=3), "bad dtype"), (pf.PF_ERR_INVALID_ARG, dict(dH=None), "dH is NULL"),
    (pf.PF_ERR_INVALID_ARG, dict(Z=A + 8), "Z is not"), (pf.PF_ERR_INVALID_ARG, dict(dZ=None), "dZ is NULL"),
    (pf.PF_ERR_INVALID_ARG, dict(dbias=A + 2), "dbias is not")])
def test_gated_backward_refusals(status, kw, text):
    _refused(status, text, pf.pf_linear_gated_bwd, **_bwd(**kw))


def test_gated_backward_workspace():
    need = pf.pf_linear_gated_workspace_bytes("bf16", 4096, 1024)
    assert need > 0 and need % (8 * 1024) == 0
    assert pf.pf_linear_gated_workspace_bytes("bf16", 0, 1024) == 0
    assert pf.pf_linear_gated_workspace_bytes("bf16", 64, 1000) == 0
    big = dict(T=4096, N=1024)
    _refused(pf.PF_ERR_WORKSPACE, "workspace needs", pf.pf_linear_gated_bwd, **_bwd(ws_bytes=need - 1, **big))
    _refused(pf.PF_ERR_INVALID_ARG, "workspace is NULL", pf.pf_linear_gated_bwd, **_bwd(workspace=None, **big))
    _refused(pf.PF_ERR_INVALID_ARG, "workspace is not", pf.pf_linear_gated_bwd, **_bwd(workspace=A + 4, **big))


# ---- layer normalisation ----------------------------------------------------

def _ln(**kw):
    d = dict(dtype="bf16", T=64, N=512, eps=1e-5, X=A, ldx=512, weight=A, bias=A, Y=A, ldy=512, mean=A, rstd=A)
    d.update(kw)
    return d


@pytest.mark.parametrize("status,kw,text", [
    (pf.PF_ERR_INVALID_ARG, dict(dtype=2), "bad dtype"), (pf.PF_ERR_INVALID_ARG, dict(T=0), "T must be"),
    (pf.PF_ERR_INVALID_ARG, dict(N=0), "T must be"), (pf.PF_ERR_UNSUPPORTED, dict(N=16385, ldx=1 << 20), "more than"),
    (pf.PF_ERR_INVALID_ARG, dict(eps=-1e-9), "eps"), (pf.PF_ERR_INVALID_ARG, dict(eps=float("nan")), "eps"),
    (pf.PF_ERR_INVALID_ARG, dict(eps=float("inf")), "eps"), (pf.PF_ERR_INVALID_ARG, dict(X=None), "X is NULL"),
    (pf.PF_ERR_INVALID_ARG, dict(X=A + 2), "X is not"), (pf.PF_ERR_INVALID_ARG, dict(ldx=511), "X: row stride"),
    (pf.PF_ERR_INVALID_ARG, dict(ldy=(1 << 32) + 1), "Y: row stride"), (pf.PF_ERR_INVALID_ARG, dict(Y=None), "Y is NULL"),
    (pf.PF_ERR_INVALID_ARG, dict(weight=A + 4), "weight is not"), (pf.PF_ERR_INVALID_ARG, dict(bias=A + 4), "bias is not"),
    (pf.PF_ERR_INVALID_ARG, dict(mean=A + 4), "mean is not"), (pf.PF_ERR_INVALID_ARG, dict(rstd=A + 4), "rstd is not")])
def test_layernorm_forward_refusals(status, kw, text):
    _refused(status, text, pf.pf_layernorm_fwd, **_ln(**kw))


def _lnb(**kw):
    d = dict(dtype="bf16", T=64, N=512, dY=A, lddy=512, X=A, ldx=512, weight=A, mean=A, rstd=A, dR=A, lddr=512, dX=A,
             lddx=512, dweight=A, dbias=A, workspace=A, ws_bytes=1 << 30)
    d.update(kw)
    return d


@pytest.mark.parametrize("status,kw,text", [
    (pf.PF_ERR_INVALID_ARG, dict(dtype=2), "bad dtype"), (pf.PF_ERR_INVALID_ARG, dict(T=0), "T must be"),
    (pf.PF_ERR_UNSUPPORTED, dict(N=16400), "more than"), (pf.PF_ERR_INVALID_ARG, dict(dY=None), "dY is NULL"),
    (pf.PF_ERR_INVALID_ARG, dict(lddy=5), "dY: row stride"), (pf.PF_ERR_INVALID_ARG, dict(X=None), "X is NULL"),
    (pf.PF_ERR_INVALID_ARG, dict(mean=None), "mean is NULL"), (pf.PF_ERR_INVALID_ARG, dict(rstd=None), "rstd is NULL"),
    (pf.PF_ERR_INVALID_ARG, dict(dR=A + 2), "dR is not"), (pf.PF_ERR_INVALID_ARG, dict(lddr=0), "dR: row stride"),
    (pf.PF_ERR_INVALID_ARG, dict(dX=None), "dX is NULL"), (pf.PF_ERR_INVALID_ARG, dict(lddx=1), "dX: row stride"),
    (pf.PF_ERR_INVALID_ARG, dict(weight=A + 8), "weight is not"),
    (pf.PF_ERR_INVALID_ARG, dict(dweight=A + 8), "dweight is not"),
    (pf.PF_ERR_INVALID_ARG, dict(dbias=A + 8), "dbias is not"),
    (pf.PF_ERR_INVALID_ARG, dict(workspace=None), "workspace is NULL"),
    (pf.PF_ERR_WORKSPACE, dict(ws_bytes=100), "workspace needs")])
def test_layernorm_backward_refusals(status, kw, text):
    _refused(status, text, pf.pf_layernorm_bwd, **_lnb(**kw))


def test_layernorm_workspace():
    for dt in ("bf16", "fp32"):
        for T in (1, 2, 100, 5000, 1 << 30):
            for N in (1, 7, 768, 1001, 4096, 16384):
                need = pf.pf_layernorm_workspace_bytes(dt, T, N)
                assert need % (8 * N) == 0 and (T == 1) <= (need == 0) and need <= 512 * 4 * 8 * N
                if need:
                    _refused(pf.PF_ERR_INVALID_ARG, "workspace is not", pf.pf_layernorm_bwd,
                             **_lnb(dtype=dt, T=T, N=N, lddy=N, ldx=N, lddr=N, lddx=N, workspace=A + 4, ws_bytes=need))
    assert pf.pf_layernorm_workspace_bytes("bf16", 0, 64) == 0
    assert pf.pf_layernorm_workspace_bytes("bf16", 64, 20000) == 0


# ---- gradients --------------------------------------------------------------

def _create(*rows):
    """pf_grads_create from (src, dst, n, src type, dst type) as they are."""
    import ctypes
    raw = b"".join(struct.pack("PPqii", *r) for r in rows)
    h = ctypes.c_void_p()
    pf._check(pf._lib.pf_grads_create(len(rows), raw, ctypes.byref(h)))
    return pf.Grads(h.value, None)


@pytest.mark.parametrize("rows,text", [
    ([(A, A, 4, 2, 0)], "bad dtype"), ([(A, A, 4, 0, -1)], "bad dtype"), ([(A, A, -1, 0, 0)], "negative"),
    ([(A, A, (1 << 37) + 1, 0, 0)], "too many"), ([(A, A, (1 << 62), 0, 0)], "too many"), ([(0, A, 4, 0, 0)], "NULL"), ([(A, 0, 4, 0, 0)], "NULL"),
    ([(A + 1, A, 4, 0, 0)], "aligned"), ([(A + 2, A + 2, 4, 1, 1)], "aligned"), ([(A, A, 4, 0, 1)], "types differ"),
    # The same tensor twice; a slice of another; what is written over a gradient that
    # is still to be read, or shifted over itself.
    ([(A, A, 64, 0, 0), (A, A, 64, 0, 0)], "overlaps"), ([(A, A, 64, 0, 0), (A + 126, A + 126, 1, 0, 0)], "overlaps"),
    ([(A, A + 4096, 64, 0, 0), (A + 8192, A, 64, 0, 0)], "overlaps"), ([(A, A + 2, 64, 0, 0)], "overlaps"),
    ([(A, 2 * A, 64, 0, 1), (A + 512, 2 * A + 252, 8, 0, 1)], "overlaps")])
def test_gradient_list_refusals(rows, text):
    with pytest.raises(pf.PixelflyError) as e:
        _create(*rows)
    assert e.value.status == pf.PF_ERR_INVALID_ARG and text in str(e.value), str(e.value)


def test_gradient_lists_that_hold():
    _create()
    _create((0, 0, 0, 0, 0), (A, A, 5, 1, 1))
    # Neighbours; the same gradient read twice into two places.
    _create((A, A, 64, 0, 0), (A + 128, A + 128, 64, 0, 0), (A + 256, A + 8192, 3, 1, 0))
    _create((A, A + 4096, 64, 0, 0), (A, A + 8192, 64, 0, 1))


def test_gradient_calls():
    g = _create((A, A, 100000, 0, 0))
    need = pf.pf_grads_workspace_bytes(g)
    assert need >= 8 and need % 8 == 0
    ok = dict(workspace=A, ws_bytes=need)
    for bad in (float("nan"), float("inf"), -1.0):
        _refused(pf.PF_ERR_INVALID_ARG, "max_norm", pf.pf_grads_clip, g, bad, A, **ok)
        _refused(pf.PF_ERR_INVALID_ARG, "max_norm", pf.pf_grads_scale, g, bad, A)
    _refused(pf.PF_ERR_INVALID_ARG, "norm is misaligned", pf.pf_grads_clip, g, 1.0, A + 2, **ok)
    _refused(pf.PF_ERR_WORKSPACE, "workspace needs", pf.pf_grads_clip, g, 1.0, A, workspace=A, ws_bytes=need - 1)
    _refused(pf.PF_ERR_INVALID_ARG, "workspace is NULL", pf.pf_grads_clip, g, 1.0, A, workspace=None, ws_bytes=need)
    _refused(pf.PF_ERR_INVALID_ARG, "NULL", pf.pf_grads_norm, g, None, None, **ok)
    _refused(pf.PF_ERR_INVALID_ARG, "sumsq is misaligned", pf.pf_grads_norm, g, A + 4, None, **ok)
    _refused(pf.PF_ERR_INVALID_ARG, "sumsq is NULL", pf.pf_grads_scale, g, 1.0, None)
    for call in ((pf.pf_grads_clip, g, 1.0, A), (pf.pf_grads_norm, g, A, A)):
        _refused(pf.PF_ERR_STATE, "not uploaded", *call, **ok)
    _refused(pf.PF_ERR_STATE, "not uploaded", pf.pf_grads_scale, g, 1.0, A)
    pf.pf_grads_destroy(g)
    for call in ((pf.pf_grads_clip, g, 1.0, A), (pf.pf_grads_norm, g, A, A)):
        _refused(pf.PF_ERR_INVALID_ARG, "list is NULL", *call, **ok)


def test_gradient_tensors():
    """The binding's own checks."""
    a, b = torch.zeros(8), torch.zeros(8, dtype=torch.bfloat16)
    pf.pf_grads_create([a, (b, torch.zeros(8))])
    for bad in ([a.double()], [torch.zeros(4, 4).t()], [(a, torch.zeros(7))], [(a, b.half())],
                [(a, torch.zeros(16)[::2])]):
        with pytest.raises(ValueError):
            pf.pf_grads_create(bad)
    with pytest.raises(pf.PixelflyError):
        pf.pf_grads_create([a, a])
    # Kernels would read host memory.
    with pytest.raises(ValueError, match="not on the GPU"):
        pf.pf_grads_upload(pf.pf_grads_create([a]))
