"""Paged attention of calls with more row blocks than the plan keeps in LDS (512): whose workgroups look the rest up
in memory. Against the definition in 64 bits."""
import numpy as np
import pytest

from tests._build_once import ensure_built

ensure_built()

import paper_2605_30351_amd  # noqa: E402, F401
from tests.gpu_common import SENTINEL, bf16_to_f64, host_bits  # noqa: E402
from tests.paged_common import Batch, assert_within, attention_by_sequence  # noqa: E402
from tests.test_gpu_paged import TEXT, attend, check_attend  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n", [511, 512, 513, 1500])
@pytest.mark.parametrize("max_new", [1, 0])
def test_a_block_per_sequence(n, max_new):
    """Single tokens over contexts of very different lengths, by the kernel of few rows and that of many."""
    rng = np.random.default_rng(n)
    kv = np.where(rng.random(n) < 0.05, rng.integers(200, 900, n), rng.integers(1, 40, n))
    b = Batch(TEXT, [(1, int(k), int(f)) for k, f in zip(kv, rng.integers(0, 99, n))], page=16, pad=3, mask=1, seed=61,
              max_new=max_new)
    check_attend(b, f"{n} blocks, max_new {max_new}")


@pytest.mark.parametrize("tokens", [2730, 2731, 3300])
def test_many_blocks_of_one_sequence(tokens):
    """d_c = 512, 64 rows a block: 512 blocks, one more with 12 rows, and 619."""
    b = Batch(TEXT.replace(d_c=512, n_heads=12), [(tokens, tokens + 70, 5)], page=100, pad=2, mask=1, window=600, seed=62)
    want, bound = attention_by_sequence(b, "cuda")
    bits = host_bits(attend(b))
    assert_within(bf16_to_f64(bits), want, bound, f"{tokens} tokens")
    assert (bits[b.tokens:] == SENTINEL).all()
