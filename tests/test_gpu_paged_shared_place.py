"""Two new tokens of one write that name the same place of the pool."""
import numpy as np
import pytest

from tests._build_once import ensure_built

ensure_built()

import paper_2605_30351_amd  # noqa: E402, F401
from tests.gpu_common import host_bits  # noqa: E402
from tests.paged_common import Batch  # noqa: E402
from tests.test_gpu_paged import TEXT, write  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("tokens", [2, 40, 9000])
def test_a_place_written_twice_holds_pieces_of_the_two(tokens):
    """Sequences 0 and 1 share their last page, with the same lengths: every 16-byte piece of the shared places is
    one of the two tokens' own, and everything else is as in a write without sequence 1."""
    dims = TEXT.replace(d_model=768)
    half = tokens // 2
    b = Batch(dims, [(half, half + 3, 0), (half, half + 3, 0), (5, 9, 2)], page=half + 3, seed=51)
    one, two = (write(b)[k] for k in (0, 1))
    apart = [host_bits(v).reshape(b.n_pages, b.page, -1) for v in (one, two)]
    first, second = int(b.table[0, 0]), int(b.table[1, 0])
    b.table[1, 0] = first
    shared = [host_bits(v).reshape(b.n_pages, b.page, -1) for v in write(b)]
    for before, got, own in zip((b.c_kv, b.k_r), shared, apart):
        pieces = lambda a: a[3:].reshape(half, -1, 8)  # noqa: E731
        x, y, z = (pieces(v) for v in (got[first], own[first], own[second]))
        assert ((x == y).all(2) | (x == z).all(2)).all()
        want = own.copy()
        want[first, 3:], want[second] = got[first, 3:], before[second]
        assert np.array_equal(got, want)
