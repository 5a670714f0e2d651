"""Argument checks of the operators round the layer's matrices (bias,
activation and residual; their way back; attention with a relative position
bias), on the host: every refused call enqueues nothing, so plain integers stand in for device addresses."""
import struct

import numpy as np
import pytest

from paper_2112_00029_amd import pixelfly as pf

A = 1 << 20  # a 16-byte aligned address that no kernel ever sees


def _refused(status, text, fn, *a, **k):
    with pytest.raises(pf.PixelflyError) as e:
        fn(*a, stream=0, **k)
    assert e.value.status == status and text in str(e.value), str(e.value)


@pytest.fixture(scope="module")
def layout():
    return pf.pf_layout_create(512, 256, 64, 4)


def _fwd(layout, **kw):
    d = dict(dtype="bf16", T=8, r=64, X=A, Wblk=A, U=A, V=A, bias=A, act=pf.PF_ACT_GELU, residual=A, Y=A,
             Y_pre=A, T_lr=A)
    d.update(kw)
    return (layout, *d.values())


@pytest.mark.parametrize("kw,text", [
    (dict(act=5), "bad activation"), (dict(act=-1), "bad activation"),
    (dict(act=pf.PF_ACT_NONE), "Y_pre given without"), (dict(bias=A + 2), "bias is not 16-byte"),
    (dict(residual=A + 8), "residual is not 16-byte"), (dict(Y_pre=A + 4), "Y_pre is not 16-byte"),
    (dict(Y=None), "Y is NULL"), (dict(X=None), "X is NULL"), (dict(T=0), "T must be"),
    (dict(r=32), "multiple of b"), (dict(U=None), "U is NULL"), (dict(dtype=7), "bad dtype")])
def test_forward_refusals(layout, kw, text):
    _refused(pf.PF_ERR_INVALID_ARG, text, pf.pf_linear_fwd_act, *_fwd(layout, **kw))


def test_forward_state_and_gamma(layout):
    _refused(pf.PF_ERR_STATE, "not uploaded", pf.pf_linear_fwd_act, *_fwd(layout))
    a = _fwd(layout)
    _refused(pf.PF_ERR_INVALID_ARG, "gamma", pf.pf_linear_fwd_act_mixed, *a[:4], float("nan"), *a[4:])


@pytest.mark.parametrize("epi", [-1, 2, 3])
def test_other_epilogues_of_the_plain_forward(layout, epi):
    a = (layout, "bf16", 8, 64)
    b = (A, A, A, A, A, A, epi)
    for y_pre in (None, A):
        _refused(pf.PF_ERR_INVALID_ARG, "bad epilogue", pf.pf_linear_fwd, *a, *b, y_pre)
        _refused(pf.PF_ERR_INVALID_ARG, "bad epilogue", pf.pf_linear_fwd_mixed, *a, 0.5, *b, y_pre)
        _refused(pf.PF_ERR_INVALID_ARG, "bad epilogue", pf.pf_linear_bwd_data, *a, A, A, A, A, A, A, epi, y_pre)


def _bwd(**kw):
    d = dict(dtype="bf16", T=64, N=512, act=pf.PF_ACT_SILU, dY=A, Y_pre=A, dY_pre=A, dbias=A, workspace=A,
             ws_bytes=1 << 30)
    d.update(kw)
    return d


@pytest.mark.parametrize("kw,text", [
    (dict(act=9), "bad activation"), (dict(T=0), "T must be"), (dict(N=40), "multiple of 32"),
    (dict(N=0), "multiple of 32"), (dict(dtype=3), "bad dtype"), (dict(dY=None), "dY is NULL"),
    (dict(Y_pre=None), "Y_pre is NULL"), (dict(dY_pre=None), "dY_pre is NULL"),
    (dict(dbias=A + 2), "dbias is not"), (dict(act=pf.PF_ACT_NONE), "without an activation"),
    (dict(act=pf.PF_ACT_NONE, Y_pre=None, dY_pre=None, dbias=None), "dbias is NULL")])
def test_backward_refusals(kw, text):
    _refused(pf.PF_ERR_INVALID_ARG, text, pf.pf_linear_act_bwd, **_bwd(**kw))


def test_backward_workspace():
    need = pf.pf_linear_act_workspace_bytes("bf16", 4096, 1024)
    assert need > 0 and need % (4 * 1024) == 0
    assert pf.pf_linear_act_workspace_bytes("bf16", 0, 1024) == 0
    assert pf.pf_linear_act_workspace_bytes("bf16", 64, 1000) == 0
    big = dict(T=4096, N=1024)
    _refused(pf.PF_ERR_WORKSPACE, "workspace needs", pf.pf_linear_act_bwd, **_bwd(ws_bytes=need - 1, **big))
    _refused(pf.PF_ERR_INVALID_ARG, "workspace is NULL", pf.pf_linear_act_bwd, **_bwd(workspace=None, **big))
    _refused(pf.PF_ERR_INVALID_ARG, "workspace is not", pf.pf_linear_act_bwd, **_bwd(workspace=A + 4, **big))


# ---- attention with a relative position bias --------------------------------

def test_log_map_thresholds():
    """Against the definition in integers, exact powers among them."""
    for n, reach, both in ((32, 128, True), (16, 128, False), (8, 64, True), (48, 512, True), (2, 5, False),
                           (4, 9, True), (256, 4096, False), (7, 50, False)):
        R = pf.pf_relpos_create_log(1024, n, reach, both)
        got, nb = pf.pf_relpos_buckets_get(R)
        assert nb == n and got.shape == (2047,)
        half = n // 2 if both else n
        e = half // 2
        want = np.empty(2047, np.int32)
        for i in range(2047):
            d = abs(i - 1023)
            c = d
            if d >= e:
                k = 0
                while k + 1 < half - e and d ** (half - e) >= reach ** (k + 1) * e ** (half - e - k - 1):
                    k += 1
                c = e + k
            c = min(c, half - 1)
            want[i] = c if i <= 1023 else (half + c if both else -1)
        assert np.array_equal(got, want), (n, reach, both)


def test_plan_refusals():
    ok = np.zeros(127, np.int32)
    pf.pf_relpos_create(64, 1, ok)
    for a in ((63, 1, np.zeros(125, np.int32)), (0, 1, np.zeros(0, np.int32)), (64, 0, ok), (64, 257, ok)):
        with pytest.raises(pf.PixelflyError) as e:
            pf.pf_relpos_create(*a)
        assert e.value.status == pf.PF_ERR_INVALID_ARG
    for bad in (1, -2):
        m = ok.copy()
        m[70] = bad
        with pytest.raises(pf.PixelflyError) as e:
            pf.pf_relpos_create(64, 1, m)
        assert "distance 7" in str(e.value)
    with pytest.raises(ValueError):
        pf.pf_relpos_create(64, 1, ok[:-1])
    for a in ((64, 3, 10, True), (64, 32, 8, True), (64, 1, 10, False), (64, 32, 1 << 40, True)):
        with pytest.raises(pf.PixelflyError) as e:
            pf.pf_relpos_create_log(*a)
        assert e.value.status == pf.PF_ERR_INVALID_ARG


class _Attn:
    """Raw calls with stand-in addresses."""

    def __init__(self):
        self.L = pf.pf_layout_create_attention(256, 64, 2)
        self.R = pf.pf_relpos_create_log(256, 32, 128, True)

    def rows(self, **kw):
        d = dict(data=A, seq=4 * 256 * 64, head=256 * 64, token=64)
        d.update(kw)
        return struct.pack("Pqqq", d["data"] or 0, d["seq"], d["head"], d["token"])

    def fwd(self, **kw):
        d = dict(L=self.L.handle, R=self.R.handle, B=2, H=4, Hkv=2, Sq=250, Skv=250, d=64, scale=0.125,
                 Q=self.rows(), K=self.rows(), V=self.rows(), bias=A, O=self.rows(), lse=A, q_start=None,
                 kv_len=None, ws=A, wsb=1 << 30, stream=None)
        d.update(kw)
        return pf._lib.pf_attn_relpos_fwd(*d.values())

    def bwd(self, **kw):
        d = dict(L=self.L.handle, R=self.R.handle, B=2, H=4, Hkv=2, S=250, d=64, scale=0.125)
        for n in ("Q", "K", "V"):
            d[n] = self.rows()
        d["bias"] = A
        d["O"] = self.rows()
        d["lse"] = A
        for n in ("dO", "dQ", "dK", "dV"):
            d[n] = self.rows()
        d.update(dtable=A, kv_len=None, ws=A, wsb=1 << 30, stream=None)
        d.update(kw)
        return pf._lib.pf_attn_relpos_bwd(*d.values())


@pytest.fixture(scope="module")
def attn():
    return _Attn()


SHARED = [(dict(B=0), -1, "B, H and H_kv"), (dict(Hkv=3), -1, "divide H"), (dict(H=0), -1, "B, H and H_kv"),
          (dict(d=128), -2, "d = 64"), (dict(scale=0.0), -1, "scale"), (dict(scale=float("nan")), -1, "scale"),
          (dict(scale=float("inf")), -1, "scale"), (dict(scale=-1.0), -1, "scale"), (dict(bias=None), -1, "bias is NULL"),
          (dict(bias=A + 4), -1, "bias is not"), (dict(lse=None), -1, "lse is NULL"), (dict(kv_len=A + 2), -1, "kv_len"),
          (dict(Q=None), -1, "Q is NULL"), (dict(L=None), -1, "layout is NULL"), (dict(R=None), -1, "plan is NULL")]
ROWS = [(dict(data=None), -1, "is NULL"), (dict(data=A + 8), -1, "16-byte"), (dict(token=60), -1, "multiples of 8"),
        (dict(token=56), -1, "below 64"), (dict(seq=-64), -1, "negative"), (dict(head=12), -1, "multiples of 8"),
        (dict(token=1 << 25), -2, "2^31"), (dict(token=1 << 22), -2, "2^31")]


@pytest.mark.parametrize("kw,status,text", SHARED)
def test_attention_refusals(attn, kw, status, text):
    for call in (attn.fwd, attn.bwd):
        assert call(**kw) == status and text in pf.pf_last_error(), pf.pf_last_error()


@pytest.mark.parametrize("kw,status,text", ROWS)
def test_attention_tensor_refusals(attn, kw, status, text):
    for call, names in ((attn.fwd, "Q K V O"), (attn.bwd, "Q K V O dO dQ dK dV")):
        for n in names.split():
            assert call(**{n: attn.rows(**kw)}) == status, n
            assert text in pf.pf_last_error() and pf.pf_last_error().startswith(n), pf.pf_last_error()


def test_attention_outputs_may_not_overlap(attn):
    assert attn.fwd(K=attn.rows(seq=0), V=attn.rows(head=0)) == pf.PF_ERR_STATE
    for n in ("seq", "head"):
        assert attn.fwd(O=attn.rows(**{n: 0})) == -1 and "overlap" in pf.pf_last_error()
        for g in ("dQ", "dK", "dV"):
            assert attn.bwd(**{g: attn.rows(**{n: 0})}) == -1 and "overlap" in pf.pf_last_error()


@pytest.mark.parametrize("kw", [dict(head=64), dict(head=249 * 64), dict(seq=64), dict(token=128, head=64),
                                dict(token=4 * 64, head=64, seq=249 * 4 * 64), dict(seq=3 * 256 * 64)])
def test_attention_output_rows_may_not_meet(attn, kw):
    for n in ("O", "dQ"):
        call = attn.fwd if n == "O" else attn.bwd
        assert call(**{n: attn.rows(**kw)}) == -1 and "overlap" in pf.pf_last_error()
    assert attn.fwd(Q=attn.rows(**kw)) == pf.PF_ERR_STATE


@pytest.mark.parametrize("kw", [dict(head=250 * 64), dict(token=4 * 64, head=64, seq=250 * 4 * 64),
                                dict(token=24 * 64, head=128, seq=250 * 24 * 64), dict(seq=64, head=128, token=512),
                                dict(seq=1 << 62)])
def test_attention_output_orders(attn, kw):
    assert attn.fwd(O=attn.rows(**kw)) == pf.PF_ERR_STATE
    assert attn.bwd(dQ=attn.rows(**kw)) == pf.PF_ERR_STATE


def test_attention_workspace_of_refused_heads(attn):
    assert pf.pf_attn_relpos_workspace_bytes(attn.L, attn.R, 1, 65535, 64) > 0
    assert pf.pf_attn_relpos_workspace_bytes(attn.L, attn.R, 1, 65536, 64) == 0


def test_attention_sizes_layouts_workspace(attn):
    for kw in (dict(Sq=0), dict(Sq=257), dict(Skv=0), dict(Skv=300)):
        assert attn.fwd(**kw) == -1 and "Sq and Skv" in pf.pf_last_error()
    assert attn.fwd(q_start=A + 1) == -1
    other = pf.pf_layout_create_attention(512, 64, 2)
    assert attn.fwd(L=other.handle) == -1 and "square" in pf.pf_last_error()
    rect = pf.pf_layout_create(256, 512, 64, 2)
    assert attn.bwd(L=rect.handle) == -1
    b32 = pf.pf_layout_create(256, 256, 32, 2)
    assert attn.fwd(L=b32.handle) == -2
    assert attn.fwd() == pf.PF_ERR_STATE and attn.bwd() == pf.PF_ERR_STATE
    need = pf.pf_attn_relpos_workspace_bytes(attn.L, attn.R, 2, 4, 250)
    assert need >= 2 * 4 * 250 * 4 and attn.bwd(wsb=need - 1) == pf.PF_ERR_WORKSPACE
    assert attn.bwd(ws=None) == -1 and attn.bwd(dtable=None) == -1
    assert pf.pf_attn_relpos_workspace_bytes(attn.L, attn.R, 0, 4, 250) == 0
    with pytest.raises(pf.PixelflyError):
        pf.pf_relpos_bias(attn.R, 0, A, A, stream=0)
    with pytest.raises(pf.PixelflyError) as e:
        pf.pf_relpos_bias(attn.R, 4, A, A, stream=0)
    assert e.value.status == pf.PF_ERR_STATE


def test_binding_refuses_host_and_odd_tensors(attn):
    import torch
    x = torch.zeros((1, 2, 8, 64), dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="on the GPU in use"):
        pf.pf_attn_relpos_fwd(attn.L, attn.R, 0.125, x, x, x, A, x, A)
    with pytest.raises(ValueError, match="4-d bfloat16"):
        pf.pf_attn_relpos_fwd(attn.L, attn.R, 0.125, x.float(), x, x, A, x, A)
