"""The binding's checks of a bucket map, on the host."""
import numpy as np
import pytest

from paper_2112_00029_amd import pixelfly as pf


@pytest.mark.parametrize("dtype,value", [(np.int64, 1 << 32), (np.int64, (1 << 32) - 1), (np.int64, -(1 << 32)),
                                         (np.uint32, (1 << 32) - 1), (np.uint64, 1 << 63)])
def test_bucket_numbers_past_32_bits_are_refused(dtype, value):
    """They are 0 or -1 in their lowest 32 bits."""
    m = np.zeros(127, dtype)
    m[3] = value
    with pytest.raises(ValueError, match="bucket"):
        pf.pf_relpos_create(64, 2, m)


@pytest.mark.parametrize("bad", [np.full(127, 0.5), np.full(127, np.nan), [0.0] * 127, np.zeros(127, complex)])
def test_buckets_that_are_no_integers_are_refused(bad):
    with pytest.raises(ValueError, match="bucket"):
        pf.pf_relpos_create(64, 2, bad)


@pytest.mark.parametrize("ok", [[1] * 127, np.ones(127, np.uint8), np.ones(127, np.int64), np.ones(254, np.int16)[::2]])
def test_integers_of_any_kind(ok):
    got, n = pf.pf_relpos_buckets_get(pf.pf_relpos_create(64, 2, ok))
    assert n == 2 and (got == 1).all() and got.shape == (127,)
