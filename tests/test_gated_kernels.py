"""Every kernel of the gated forward: which one a call takes
(pf_linear_gated_plan_get), and its results there against float64.  KERNELS names
for each a call that it serves: pipelines longer and shorter than their stages, odd
numbers of rows, tiles that are not full, workgroup bands; tests/test_gated_parity.py has
the tolerances.  The plan of each is checked on the host."""
import pytest

from paper_2112_00029_amd import pixelfly as pf

DMA, STAGED, SMALL = 1, 0, 2
# (family, tokens, columns of Z, K step, waves), of block size b: the call.
KERNELS = [
    ((DMA, 128, 64, 64, 4), ("bf16", 513, 4096, 1056, 32, 64, 64)),
    ((DMA, 256, 64, 64, 4), ("bf16", 4501, 1024, 1088, 32, 16, 32)),
    ((DMA, 128, 128, 32, 4), ("bf16", 2509, 2048, 4096, 32, 32, 64)),
    ((DMA, 128, 128, 64, 4), ("bf16", 2509, 1024, 4096, 32, 64, 256)),
    ((DMA, 256, 256, 64, 8), ("bf16", 8201, 1024, 4128, 32, 64, 256)),  # tiles of 8 blocks, one of 2
    ((DMA, 128, 128, 64, 4), ("bf16", 1001, 1024, 4096, 64, 16, 128)),
    ((DMA, 256, 256, 64, 8), ("bf16", 8201, 2048, 4160, 64, 64, 64)),   # tiles of 4 blocks, one of 2
    ((DMA, 128, 256, 32, 4), ("bf16", 4909, 1024, 1664, 128, 8, 128)),
    ((DMA, 128, 256, 32, 4), ("bf16", 4909, 128, 1664, 128, 1, 0)),     # four steps, three stages
    ((DMA, 256, 256, 64, 8), ("bf16", 1101, 512, 8192, 128, 2, 128)),   # 64 column tiles: bands
    ((STAGED, 128, 64, 32, 4), ("fp32", 2101, 512, 800, 32, 4, 32)),
    ((STAGED, 128, 128, 32, 4), ("fp32", 2047, 512, 1024, 32, 8, 32)),
    ((STAGED, 128, 128, 32, 4), ("fp32", 1501, 512, 1024, 64, 4, 64)),
    ((STAGED, 64, 256, 32, 4), ("fp32", 2001, 512, 1024, 128, 4, 128)),
    ((SMALL, 32, 64, 64, 4), ("bf16", 33, 320, 416, 32, 8, 32)),
    ((SMALL, 32, 64, 64, 8), ("bf16", 5, 2048, 256, 32, 64, 64)),
    ((SMALL, 32, 64, 64, 4), ("bf16", 33, 256, 4096, 64, 1, 0)),
    ((SMALL, 32, 64, 64, 8), ("bf16", 5, 512, 512, 64, 16, 64)),
    ((SMALL, 32, 64, 64, 4), ("bf16", 100, 512, 7296, 128, 2, 128)),
    ((SMALL, 32, 64, 64, 8), ("bf16", 8, 512, 256, 128, 2, 0)),
    ((SMALL, 32, 64, 32, 4), ("fp32", 301, 128, 512, 64, 1, 0)),
    ((SMALL, 32, 64, 32, 8), ("fp32", 3, 1024, 256, 32, 32, 32)),
]
IDS = ["-".join(map(str, s)) for _, s in KERNELS]


def _plan(dtype, T, K, N, b, ms, r):
    return tuple(pf.pf_linear_gated_plan_get(pf.pf_layout_create_gated(N, K, b, ms), dtype, T, r).values())


@pytest.mark.parametrize("kernel,shape", KERNELS, ids=IDS)
def test_plan(kernel, shape):
    assert _plan(*shape) == kernel


def test_plan_refusals():
    L = pf.pf_layout_create_gated(512, 256, 64, 4)
    for layout, args in ((pf.pf_layout_create(1024, 256, 64, 4), ("bf16", 8, 64)), (L, ("bf16", 0, 64)),
                         (L, ("bf16", 8, 32)), (L, ("bf16", 8, -64)), (L, (7, 8, 64))):
        with pytest.raises(pf.PixelflyError) as e:
            pf.pf_linear_gated_plan_get(layout, *args)
        assert e.value.status == pf.PF_ERR_INVALID_ARG
    with pytest.raises(pf.PixelflyError) as e:
        pf.pf_linear_gated_plan_get(pf.pf_layout_create_gated(64, 64, 16, 1), "bf16", 8, 0)
    assert e.value.status == pf.PF_ERR_UNSUPPORTED


@pytest.mark.gpu
@pytest.mark.parametrize("kernel,shape", KERNELS, ids=IDS)
def test_kernel(kernel, shape):
    from tests.test_gated_parity import Gated
    assert _plan(*shape) == kernel
    lay = Gated(*shape)
    for act in ("gelu_tanh", "none"):
        h, z, _ = lay.run(act)
        lay.check(h, z, act)
    h2, _, _ = lay.run("none", pre=False)
    assert lay.t.equal(h2, h)
    h, z, _ = lay.run("silu", bias=False)
    lay.check(h, z, "silu", bias=False)


@pytest.mark.gpu
@pytest.mark.parametrize("kernel,shape", KERNELS, ids=IDS)
def test_kernel_mixed(kernel, shape):
    from tests.test_gated_parity import Gated
    lay = Gated(*shape, gamma=0.3)
    h, z, _ = lay.run("gelu", gamma=0.3)
    lay.check(h, z, "gelu")


@pytest.mark.gpu
@pytest.mark.parametrize("kernel,shape", KERNELS, ids=IDS)
def test_kernel_rows_and_repeats(kernel, shape):
    """Rows past the last token stay as they were; a repeat gives the same bits."""
    from tests.test_gated_parity import Gated
    lay = Gated(*shape)
    t, T, N = lay.t, lay.T, lay.N
    h, z, tl = lay.run("silu")
    big_h, big_z = (t.full((T + 3, n), 7.0, dtype=lay.dt, device="cuda") for n in (N, 2 * N))
    pf.pf_linear_gated_fwd(lay.L, lay.dtype, T, lay.r, lay.x, lay.w, lay.U, lay.V, lay.bias, pf.PF_ACT_SILU, big_h,
                           big_z, tl, lay.ws, lay.ws_bytes)
    assert t.equal(big_h[:T], h) and t.equal(big_z[:T], z)
    assert bool((big_h[T:] == 7).all()) and bool((big_z[T:] == 7).all())
