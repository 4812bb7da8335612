"""Paged attention with infinities in tokens that queries do see: the result is the definition's, wherever
mask, window and tile boundaries fall. An infinite latent makes a score of plus or minus infinity (or NaN,
with several) and a value that is not finite, so that 0 * inf or inf - inf is left whatever its sign: NaN."""
import numpy as np
import pytest

from tests._build_once import ensure_built

ensure_built()

import paper_2605_30351_amd  # noqa: E402, F401
from tests.gpu_common import bf16_to_f64, host_bits  # noqa: E402
from tests.paged_common import Batch, assert_within  # noqa: E402
from tests.test_gpu_paged import TEXT, attend  # noqa: E402
from workloads import TINY  # noqa: E402

pytestmark = pytest.mark.gpu

WIDTHS = [TINY, TEXT.replace(d_c=64), TEXT.replace(d_c=128), TEXT, TEXT.replace(d_c=256), TEXT.replace(d_c=512)]
IDS = [f"dc{d.d_c}" for d in WIDTHS]
INF, NEG = 0x7f80, 0xff80


def batch(dims, max_new, mask, window):
    return Batch(dims, [(40, 150, 3), (1, 70, 0)], page=20, mask=mask, window=window, seed=41, max_new=max_new)


def seers(b, j):
    return np.array([i for i in range(40) if j in b.seen(0, 110 + i)], int)


# cached token of sequence 0 that holds the infinity: in whole tiles of most masks, in the tiles that the
# causal limit or the window cross, the last one
@pytest.mark.parametrize("j", [5, 100, 121, 130, 149])
@pytest.mark.parametrize("max_new", [1, 40])
@pytest.mark.parametrize("dims", WIDTHS, ids=IDS)
def test_an_infinite_latent_reaches_every_query_that_sees_it(dims, max_new, j):
    for mask, window in ((1, 0), (0, 0), (16, 60)):
        b = batch(dims, max_new, mask, window)
        want, bound = b.attention()
        for bits, at in ((INF, 0), (NEG, dims.d_c - 1), (NEG, slice(None))):
            c = b.c_kv.reshape(-1, dims.d_c)
            r = b.pool_row(0, j)
            before = c[r].copy()
            c[r, at] = bits
            got = bf16_to_f64(host_bits(attend(b)))
            c[r] = before
            see = seers(b, j)
            label = f"{dims.d_c} token {j} mask {mask} window {window} {bits:#x} at {at}"
            assert np.isnan(got[see]).all(), (label, int(np.isfinite(got[see]).sum()))
            keep = np.setdiff1d(np.arange(b.rows), see)
            assert_within(got[keep], want[keep], bound[keep], label)
