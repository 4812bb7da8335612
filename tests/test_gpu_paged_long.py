"""Paged attention and writes on the GPU where other kernels take over: hundreds of tokens per call, rows
of two blocks, thousands of sequences, graphs that share a workspace. Against the definitions of
tests/paged_common.py."""
import numpy as np
import pytest
import torch

from tests._build_once import ensure_built

ensure_built()

import paper_2605_30351_amd as vm  # noqa: E402
from tests.gpu_common import SENTINEL, bf16_to_f64, dev, host_bits  # noqa: E402
from tests.paged_common import Batch, assert_within, attention_by_sequence  # noqa: E402
from tests.test_gpu_paged import FAR, TEXT, attend, check_attend, check_write  # noqa: E402
from workloads import TINY  # noqa: E402

pytestmark = pytest.mark.gpu

WIDTHS = [TINY, TEXT.replace(d_c=64, n_heads=12), TEXT.replace(d_c=128, n_heads=12), TEXT.replace(n_heads=12),
          TEXT.replace(d_c=256, n_heads=12), TEXT.replace(d_c=512, n_heads=12, d_v=192)]
IDS = [f"dc{d.d_c}" for d in WIDTHS]


@pytest.mark.parametrize("max_new", [0, 1])
@pytest.mark.parametrize("mask,window", [(1, 0), (1, 333), (100, 500), (0, 0)])
@pytest.mark.parametrize("dims", WIDTHS, ids=IDS)
def test_attend_many_tokens(dims, mask, window, max_new):
    """Row blocks that cross mask blocks, windows and the end of a sequence; with the wrong bound of one
    new token the few-row kernel does the same work."""
    b = Batch(dims, [(300, 1400, 0), (1, 900, 7), (0, 30, 0), (219, 219, FAR), (3, 50, 5)], page=48, pad=70,
              mask=mask, window=window, seed=30, max_new=max_new)
    want, bound = attention_by_sequence(b, "cuda")
    bits = host_bits(attend(b))
    assert_within(bf16_to_f64(bits), want, bound, f"{dims.d_c} mask {mask} window {window} max_new {max_new}")
    assert (bits[b.tokens:] == SENTINEL).all()


@pytest.mark.parametrize("dims", WIDTHS, ids=IDS)
def test_attend_two_tokens_per_sequence(dims):
    """24 rows per sequence: a second block of 16 rows that is half empty."""
    check_attend(Batch(dims, [(2, 700, 0), (1, 77, 3), (2, 2, FAR), (2, 321, 9), (0, 5, 0)], page=20, mask=1, seed=31,
                       pad=1, max_new=2), f"{dims.d_c}")


@pytest.mark.parametrize("n", [64, 65, 700, 4096])
def test_many_sequences(n):
    """More sequences than a wave has lanes, most of them without new tokens, and padding rows behind."""
    rng = np.random.default_rng(n)
    new = np.where(rng.random(n) < min(1.0, 500 / n), rng.integers(0, 3, n), 0)
    seqs = [(int(v), int(v) + int(k), int(f)) for v, k, f in zip(new, rng.integers(0, 40, n), rng.integers(0, 9, n))]
    for max_new in (2, 0):
        b = Batch(TEXT, seqs, page=8, pad=40, mask=1, seed=32, max_new=max_new)
        check_attend(b, f"{n} sequences, max_new {max_new}")
    check_write(b)


@pytest.mark.parametrize("max_new", [1, 0])
def test_no_sequence_has_a_new_token(max_new):
    b = Batch(TEXT, [(0, 30, 0), (0, 0, 0), (0, 7, 3)], page=16, pad=300, seed=33, max_new=max_new)
    assert (host_bits(attend(b)) == SENTINEL).all()
    check_write(b)


def test_two_graphs_share_a_workspace():
    """Two captured calls of different batches over one workspace, replayed in turn."""
    batches = [Batch(TEXT, [(4, 900, 0), (1, 300, 1)], page=32, mask=1, seed=34, max_new=4),
               Batch(TEXT, [(200, 600, 0)], page=50, mask=1, seed=35)]
    want = [host_bits(attend(b)) for b in batches]
    need = max(vm.paged_attend_workspace_bytes(TEXT, b.paged(vm)) for b in batches)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    sides = []
    for b in batches:
        p = b.paged(vm)
        args = [dev(t) for t in (b.q_nope, b.q_r, b.w_uk, b.w_uv, b.c_kv, b.k_r)]
        out = torch.zeros(b.rows, TEXT.n_heads, TEXT.d_v, dtype=torch.bfloat16, device="cuda")
        vm.paged_attend(TEXT, p, *args, out, ws)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            vm.paged_attend(TEXT, p, *args, out, ws)
        sides.append((graph, out, p, args))
    for n in range(6):
        graph, out = sides[n % 2][:2]
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert np.array_equal(host_bits(out), want[n % 2]), n


@pytest.mark.parametrize("max_new", [0, 1])
@pytest.mark.parametrize("dims", WIDTHS[1:5], ids=IDS[1:5])
def test_long_queries_keep_their_precision(dims, max_new):
    """Scores of standard deviation 4 in every other token, 1 in the rest. With both terms of a long query the
    roundings left are the weights' and the output's own: a weight is off by as much of itself as the output
    is, so that the two together are at most sqrt(2) times the output's rounding in the 2-norm (one term alone
    measures 2.2 times); 1.5 for the sums. The short queries' rounding adds as much as their output's."""
    seqs = [(301, 900, 0), (61, 200, 7), (3, 40, 0)]
    b, short = (Batch(dims, seqs, page=48, mask=1, seed=36, gain=g, max_new=max_new) for g in (4.0, 1.0))
    for long_q, short_q in ((b.q_nope, short.q_nope), (b.q_r, short.q_r)):
        long_q[1::2] = short_q[1::2]
    want, bound = attention_by_sequence(b, "cuda")
    got = bf16_to_f64(host_bits(attend(b)))
    assert_within(got, want, bound, f"{dims.d_c}")
    rounded = torch.from_numpy(want).to(torch.bfloat16).double().numpy()
    for name, part, most in (("long", slice(0, None, 2), 1.5), ("short", slice(1, None, 2), 1.5 * 2 ** 0.5)):
        off = [np.linalg.norm(v[part] - want[part]) for v in (got, rounded)]
        print(f"{dims.d_c} {name}: {off[0] / off[1]:.3f} of the output's rounding", flush=True)
        assert off[0] <= most * off[1], (name, off)
