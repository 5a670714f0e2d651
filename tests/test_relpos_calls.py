"""Calls of position-bias attention that its documentation allows beside the usual
ones, against the formulas in float64 (tolerances: tests/test_relpos_numerics.py):
layouts longer than the sequences, fewer or more rows than tokens, masks without symmetry
and with empty columns, many heads on one key/value head."""
import numpy as np
import pytest

from tests.test_relpos_numerics import Scaled
from tests.test_relpos_parity import butterfly, clip_map, log_map

pytestmark = pytest.mark.gpu


def _mask(nb, share, seed):
    g = np.random.default_rng(seed)
    m = g.random((nb, nb)) < share
    m[:, g.integers(0, nb, nb // 4)] = False  # keys that no row attends to
    for i in range(nb):
        m[i, g.integers(0, nb)] = True
    return m


# name: B, H, Hkv, S, map, buckets, mask, lengths
WHOLE = {
    "long_layout": (2, 2, 2, 100, log_map(1024, 16, 96, True), 16, butterfly(16, 16, 2), [100, 33]),
    "long_layout_causal": (1, 4, 1, 1, clip_map(4096, 100, True), 201, butterfly(64, 64, 1), None),
    "long_layout_parts": (1, 2, 1, 1300, clip_map(2048, 60), 121, np.ones((32, 32), bool), [1290]),
    "stripes_past_the_tokens": (1, 3, 3, 130, clip_map(1536, 5), 11, butterfly(24, 2, 20), None),
    "no_symmetry": (2, 4, 2, 630, log_map(640, 32, 128, True), 32, _mask(10, 0.4, 1), [630, 600]),
    "no_symmetry_causal_parts": (1, 4, 1, 1900, log_map(1920, 16, 200, False), 16, _mask(30, 0.7, 2), [1850]),
    "heads_33_on_1": (1, 33, 1, 200, clip_map(256, 30, True), 61, np.ones((4, 4), bool), [190]),
    "every_bucket": (1, 2, 1, 320, np.arange(639) % 256, 256, np.ones((5, 5), bool), [300]),
}


@pytest.mark.parametrize("name", WHOLE)
def test_whole_sequences(name):
    print(f"[relpos] {name}", flush=True)
    B, H, Hkv, S, m, n, mask, lens = WHOLE[name]
    Scaled(B, H, Hkv, S, m, n, mask, lens, True, scale=0.125).check()


@pytest.mark.parametrize("rows,tokens,lens", [(300, 100, None), (70, 500, None), (300, 100, [100, 7]), (1, 500, [500, 0]),
                                              (500, 1, None), (65, 64, [64, 63])])
@pytest.mark.parametrize("Hkv", [4, 1])
def test_other_numbers_of_rows_than_of_tokens(rows, tokens, lens, Hkv):
    """Without q_start: the rows stand at 0, 1, ...; those past the tokens are empty."""
    print(f"[relpos] {rows} rows, {tokens} tokens, {lens}", flush=True)
    c = Scaled(2, 4, Hkv, tokens, log_map(512, 32, 128, True), 32, _mask(8, 0.6, 3), lens, False, rows, scale=0.125)
    c.check_fwd(*c.fwd())


@pytest.mark.parametrize("starts", [[0, 1, 700], [63, 640, 767], [767, 64, 128]])
@pytest.mark.parametrize("rows", [1, 3, 64, 129])
def test_rows_that_run_past_the_layout(starts, rows):
    """Rows past the tokens, the caches and the layout itself are empty; masks without
    symmetry, stripes among them."""
    print(f"[relpos] rows {rows} from {starts}", flush=True)
    for mask in (_mask(12, 0.5, 4), butterfly(12, 4, 2)):
        c = Scaled(3, 4, 2, 760, clip_map(768, 25, True), 51, mask, [760, 700, 760], True, rows, starts, scale=0.125)
        c.check_fwd(*c.fwd())
