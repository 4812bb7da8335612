"""Paged attention with infinities in tokens that queries do see: the result is the definition's, wherever
mask, window and tile boundaries fall. An infinite latent makes a score of plus or minus infinity (or NaN,
with several) and a value that is not finite, so that 0 * inf or inf - inf is left whatever its sign: NaN. An
infinite rotated key has a finite value: at plus infinity the row is NaN, at minus infinity the key has no
weight, as if it were hidden."""
import numpy as np
import pytest

from tests._build_once import ensure_built

ensure_built()

import paper_2605_30351_amd  # noqa: E402, F401
from tests.gpu_common import bf16_to_f64, host_bits  # noqa: E402
from tests.paged_common import Batch, assert_within, rope  # noqa: E402
from tests.test_gpu_paged import TEXT, attend  # noqa: E402
from workloads import TINY  # noqa: E402

pytestmark = pytest.mark.gpu

WIDTHS = [TINY, TEXT.replace(d_c=64), TEXT.replace(d_c=128), TEXT, TEXT.replace(d_c=256), TEXT.replace(d_c=512)]
IDS = [f"dc{d.d_c}" for d in WIDTHS]
INF, NEG = 0x7f80, 0xff80


class Without(Batch):
    """A batch whose queries do not see cached token `gone` of sequence 0."""
    gone = -1

    def seen(self, s, i):
        return [j for j in super().seen(s, i) if s or j != self.gone]


def batch(dims, max_new, mask, window, gone=-1, gain=1.0):
    b = Without(dims, [(40, 150, 3), (1, 70, 0)], page=20, mask=mask, window=window, seed=41, max_new=max_new, gain=gain)
    b.gone = gone
    return b


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


@pytest.mark.parametrize("j", [5, 121, 149])
@pytest.mark.parametrize("max_new,gain", [(1, 1.0), (40, 1.0), (40, 4.0)])
@pytest.mark.parametrize("dims", WIDTHS, ids=IDS)
def test_an_infinite_key_is_seen_by_the_sign_of_its_score(dims, max_new, gain, j):
    for mask, window in ((1, 0), (16, 60)):
        b, without = (batch(dims, max_new, mask, window, gone, gain) for gone in (-1, j))
        (want, bound), (want_gone, bound_gone) = b.attention(), without.attention()
        b.k_r.reshape(-1, dims.d_rope)[b.pool_row(0, j), 0] = INF
        got = bf16_to_f64(host_bits(attend(b)))
        see = seers(b, j)
        q = rope(dims, bf16_to_f64(b.q_r[see]), (3 + 110 + see)[:, None])[..., 0]
        for n, i in enumerate(see):
            for h in range(dims.n_heads):
                if q[n, h] > 0:
                    want[i, h] = np.nan
                    assert np.isnan(got[i, h]).all(), (dims.d_c, j, mask, i, h)
                else:
                    want[i, h], bound[i, h] = want_gone[i, h], bound_gone[i, h]
        assert_within(got, want, bound, f"{dims.d_c} key {j} mask {mask} window {window}")
