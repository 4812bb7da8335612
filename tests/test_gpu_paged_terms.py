"""Paged attention of many rows: the second bf16 term of the absorbed queries is multiplied by what the scores
are, not by how the query and the cache share their scale."""
import numpy as np
import pytest
import torch

from tests._build_once import ensure_built

ensure_built()

import paper_2605_30351_amd  # noqa: E402, F401
from tests.gpu_common import bf16_to_f64, host_bits  # noqa: E402
from tests.paged_common import Batch, assert_within, attention_by_sequence  # noqa: E402
from tests.test_gpu_paged import TEXT, attend  # noqa: E402

pytestmark = pytest.mark.gpu

WIDTHS = [TEXT.replace(d_c=n, n_heads=12) for n in (64, 128, 192, 256, 512)]


def scaled(bits, factor):
    """bf16 bits times a power of two: exact."""
    v = torch.from_numpy(bits.view(np.int16)).view(torch.bfloat16) * factor
    return v.view(torch.int16).numpy().view(np.uint16)


# what is scaled, and by how much: scores of standard deviation 4 or more in each
SCALES = {
    "queries": dict(q_nope=4, q_r=4),
    "latents": dict(q_nope=4, q_r=4, c_kv=4, w_uk=0.25, w_uv=0.25),  # the first's scores, of shorter absorbed queries
    "small latents": dict(q_nope=4, q_r=4, c_kv=2.0 ** -10, w_uk=2.0 ** 10, w_uv=2.0 ** 10),
    "positional queries": dict(q_r=8),
    "positional keys": dict(k_r=8),
}


@pytest.mark.parametrize("max_new", [0, 1])
@pytest.mark.parametrize("scale", SCALES)
@pytest.mark.parametrize("dims", WIDTHS, ids=lambda d: f"dc{d.d_c}")
def test_peaked_scores_keep_their_precision(dims, scale, max_new):
    """With both terms the roundings left are the weights' and the output's own: a weight is off by as much of
    itself as the output is, so that the two together are at most sqrt(2) times the output's rounding in the
    2-norm; 1.5 for the sums."""
    b = Batch(dims, [(301, 900, 0), (61, 200, 7), (3, 40, 0)], page=48, mask=1, seed=37, max_new=max_new)
    for name, factor in SCALES[scale].items():
        setattr(b, name, scaled(getattr(b, name), factor))
    want, bound = attention_by_sequence(b, "cuda")
    got = bf16_to_f64(host_bits(attend(b)))
    assert_within(got, want, bound, f"{dims.d_c} {scale}")
    rounded = torch.from_numpy(want).to(torch.bfloat16).double().numpy()
    off = [np.linalg.norm(v - want) for v in (got, rounded)]
    print(f"{dims.d_c} {scale}: {off[0] / off[1]:.3f} of the output's rounding", flush=True)
    assert off[0] <= 1.5 * off[1], off


@pytest.mark.parametrize("tokens", [1, 25])
@pytest.mark.parametrize("dims", WIDTHS, ids=lambda d: f"dc{d.d_c}")
def test_keys_that_grow_within_a_sequence(dims, tokens):
    """More sequences than workgroups, so that one takes a sequence's tiles one after the other; from its middle
    on the keys are larger. Waves without rows (1 token: 12 of a workgroup's rows) and with."""
    b = Batch(dims, [(tokens, 190 + n % 60, n) for n in range(270)], page=16, mask=1, seed=38)
    keys = b.k_r.reshape(-1, dims.d_rope)
    for s, (_, kv, _) in enumerate(b.seqs):
        rows = [b.pool_row(s, j) for j in range(100, kv)]
        keys[rows] = scaled(keys[rows], 16)
    want, bound = attention_by_sequence(b, "cuda")
    got = bf16_to_f64(host_bits(attend(b)))
    assert_within(got, want, bound, f"{dims.d_c}")
    rounded = torch.from_numpy(want).to(torch.bfloat16).double().numpy()
    off = [np.linalg.norm(v - want) for v in (got, rounded)]
    print(f"{dims.d_c} growing keys: {off[0] / off[1]:.3f} of the output's rounding", flush=True)
    assert off[0] <= 1.5 * off[1], off
