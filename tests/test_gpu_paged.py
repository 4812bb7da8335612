"""Paged latent cache on the GPU: writes, attention and page copies against their definitions in 64
bits (tests/paged_common.py), at the lengths, page sizes and masks where they can go wrong."""
import numpy as np
import pytest
import torch

from tests._build_once import ensure_built

ensure_built()

import paper_2605_30351_amd as vm  # noqa: E402
from oracle import videomla_oracle as O  # noqa: E402
from tests.gpu_common import SENTINEL, bf16_to_f64, dev, host_bits, ulp_distance  # noqa: E402
from tests.paged_common import Batch, assert_within  # noqa: E402
from workloads import SMALL, SMALL_PAPER, TINY, WAN  # noqa: E402

pytestmark = pytest.mark.gpu

FAR = 1_000_003
TEXT = SMALL.replace(grid_h=1, grid_w=1, rope_pairs=(16, 0, 0))
SHAPES = [TINY, SMALL, SMALL_PAPER, TEXT.replace(d_c=64, n_heads=3), TEXT.replace(d_c=128),
          TEXT.replace(d_c=256), TEXT.replace(d_c=512), TEXT.replace(n_heads=16, d_v=64)]
IDS = [f"dc{d.d_c}h{d.n_heads}n{d.d_nope}" for d in SHAPES]


def attend(b, paged=None, ws=None, out=None):
    paged = paged or b.paged(vm)
    d = b.dims
    need = vm.paged_attend_workspace_bytes(d, paged)
    if ws is None:
        ws = torch.full((need,), 0xff, dtype=torch.uint8, device="cuda")
    if out is None:
        out = torch.full((b.rows, d.n_heads, d.d_v), SENTINEL, dtype=torch.int16, device="cuda").view(torch.bfloat16)
    vm.paged_attend(d, paged, dev(b.q_nope), dev(b.q_r), dev(b.w_uk), dev(b.w_uv), dev(b.c_kv), dev(b.k_r),
                    out, ws)
    torch.cuda.synchronize()
    return out


def check_attend(b, label, **kw):
    want, bound = b.attention()
    bits = host_bits(attend(b, **kw))
    assert_within(bf16_to_f64(bits), want, bound, label)
    assert (bits[b.tokens:] == SENTINEL).all(), "rows behind the last sequence were written"
    empty = (want == 0).all(axis=(1, 2))
    assert (bits[empty] == 0).all()


RAGGED = [(1, 1, 0), (1, 33, 5), (5, 5, FAR), (0, 7, 2), (3, 64, 0), (0, 0, 0), (7, 200, FAR), (1, 129, 31),
          (20, 300, 7)]


@pytest.mark.parametrize("mask,window", [(0, 0), (1, 0), (7, 0), (1, 20), (60, 45), (0, 33)])
@pytest.mark.parametrize("dims", SHAPES, ids=IDS)
def test_attend_ragged(dims, mask, window):
    check_attend(Batch(dims, RAGGED, page=16, pad=3, mask=mask, window=window, seed=1),
                 f"{dims.d_c} mask {mask} window {window}")


@pytest.mark.parametrize("page", [1, 3, 31, 32, 50, 64, 200, 1560])
def test_attend_page_sizes(page):
    check_attend(Batch(SMALL, RAGGED, page=page, pad=1, mask=1, seed=2), f"page {page}")


@pytest.mark.parametrize("kv", [1, 31, 32, 33, 127, 128, 129, 1000])
@pytest.mark.parametrize("dims", SHAPES, ids=IDS)
def test_attend_single_tokens(dims, kv):
    check_attend(Batch(dims, [(1, kv, 0), (1, 1, 9), (1, kv // 2 + 1, FAR)], page=24, mask=1, seed=kv, max_new=1),
                 f"{dims.d_c} kv {kv}")


@pytest.mark.parametrize("dims", [SMALL, TEXT.replace(d_c=512), TINY], ids=["dc192", "dc512", "dc16"])
def test_attend_one_token_over_many_keys(dims):
    """Every workgroup takes part in one row block: many partial results per row."""
    check_attend(Batch(dims, [(1, 40_001, 17)], page=64, mask=1, seed=4, max_new=1), "40,001 keys")


@pytest.mark.parametrize("max_new", [0, 1, 150])
@pytest.mark.parametrize("dims", [SMALL, TEXT.replace(d_c=512), TINY], ids=["dc192", "dc512", "dc16"])
def test_attend_mixed_lengths_whatever_the_hint(dims, max_new):
    """Single tokens beside chunks of 150, with the right, no and a wrong bound on the new tokens."""
    check_attend(Batch(dims, [(1, 700, 0), (150, 400, 3), (1, 3, 0), (150, 150, FAR), (2, 90, 1)], page=48,
                       mask=1, seed=5, max_new=max_new), f"max_new {max_new}")


@pytest.mark.parametrize("dims", [SMALL, TEXT.replace(d_c=512), TINY], ids=["dc192", "dc512", "dc16"])
def test_attend_rows_that_see_nothing(dims):
    """More new tokens than cached ones, sequences that are all holes, holes inside and at the end."""
    seqs = [(5, 3, 0), (4, 0, 0), (2, 40, 8), (3, 100, 0), (1, 65, 2)]
    holes = [(2, 0, -1), (2, 1, 999), (2, 2, -7), (3, 1, -1), (3, 4, 1 << 30), (4, 4, -1)]
    for mask, window in ((1, 0), (0, 0), (16, 4), (1, 1)):
        check_attend(Batch(dims, seqs, page=16, pad=2, mask=mask, window=window, seed=6, holes=holes),
                     f"mask {mask} window {window}")


def test_attend_peaked_and_flat_scores():
    for gain in (0.0, 4.0, 30.0):
        check_attend(Batch(SMALL, [(9, 500, 0), (1, 300, 5)], page=32, mask=1, seed=7, gain=gain), f"gain {gain}")


def test_attend_without_first_positions():
    check_attend(Batch(SMALL, [(9, 70, 0), (1, 300, 0)], page=32, mask=1, seed=8, with_first=False), "first_pos NULL")


@pytest.mark.parametrize("bits", [0x7fc0, 0x7f80, 0xff80, 0xff7f, 0x7f7f])
def test_what_no_query_sees_reaches_none(bits):
    """NaN, infinities and the largest values in later tokens of a chunk, behind a window, behind the
    end of a sequence and in unused pages."""
    for max_new in (1, 0):
        b = Batch(SMALL, [(6, 70, 0), (1, 45, 3), (12, 50, 0)], page=16, mask=1, window=40, seed=9, max_new=max_new)
        want, bound = b.attention()
        c, k = b.c_kv.reshape(-1, b.dims.d_c), b.k_r.reshape(-1, b.dims.d_rope)
        used = set()
        for s, (n, kv, _) in enumerate(b.seqs):
            for t in range(n):
                used.update(b.pool_row(s, j) for j in b.seen(s, kv - n + t))
        for r in set(range(b.n_pages * b.page)) - used:
            c[r], k[r] = bits, bits
        got = bf16_to_f64(host_bits(attend(b)))
        assert_within(got, want, bound, f"{bits:#x} unseen by all")
        # the last new token of the first sequence: only its own query sees it
        r = b.pool_row(0, 69)
        c[r] = bits
        got = bf16_to_f64(host_bits(attend(b)))
        keep = np.ones(b.rows, bool)
        keep[5] = False
        assert_within(got[keep], want[keep], bound[keep], f"{bits:#x} seen by one")
        if bits == 0x7fc0:
            assert np.isnan(got[5]).all()


def test_attend_repeats_bit_for_bit_and_ignores_the_workspace_contents():
    b = Batch(SMALL, RAGGED, page=16, mask=1, seed=10)
    first = host_bits(attend(b))
    for fill in (0, 0x7f):
        ws = torch.full((vm.paged_attend_workspace_bytes(b.dims, b.paged(vm)),), fill, dtype=torch.uint8, device="cuda")
        assert np.array_equal(host_bits(attend(b, ws=ws)), first)


def test_lengths_out_of_range_stay_inside_the_buffers():
    """Offsets that go down or past the rows, lengths and positions out of range: the call returns, rows
    of no sequence and guard areas behind every buffer stay as they are."""
    b = Batch(SMALL, [(3, 40, 0), (5, 80, 0), (2, 20, 0)], page=16, mask=1, seed=11, pad=4)
    i32 = lambda *v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    i64 = lambda *v: torch.tensor(v, dtype=torch.int64, device="cuda")  # noqa: E731
    big = 2 ** 31 - 1
    for kw in (dict(cu_tokens=i32(0, 9, 2, 10)), dict(cu_tokens=i32(-5, 3, 8, 99)), dict(cu_tokens=i32(7, 7, 0, -1)),
               dict(kv_len=i32(big, -3, -big)), dict(first_pos=i64(-9, 2 ** 62, 2 ** 63 - 1)),
               dict(cu_tokens=i32(14, 14, 14, 14))):
        paged = b.paged(vm, **kw)
        need = vm.paged_attend_workspace_bytes(b.dims, paged)
        ws = torch.full((need + 4096,), 0x5a, dtype=torch.uint8, device="cuda")
        n = b.rows * b.dims.n_heads * b.dims.d_v
        flat = torch.full((n + 2048,), SENTINEL, dtype=torch.int16, device="cuda")
        out = flat[:n].view(torch.bfloat16).view(b.rows, b.dims.n_heads, b.dims.d_v)
        attend(b, paged, ws[:need], out)
        assert (ws[need:] == 0x5a).all() and (flat[n:] == SENTINEL).all(), kw
        write(b, paged)


# ---- writes -----------------------------------------------------------------------------------

def write(b, paged=None, pools=None, gamma=True):
    d = b.dims
    panel = torch.empty(vm.write_weights_bytes(d), dtype=torch.uint8, device="cuda")
    vm.prepare_write_weights(d, dev(b.w_dkv), dev(b.w_kr), panel)
    c, k = pools or (dev(b.c_kv), dev(b.k_r))
    vm.paged_cache_write(d, paged or b.paged(vm), dev(b.x), panel, dev(b.gamma) if gamma else None, c, k)
    torch.cuda.synchronize()
    return c, k


def check_write(b):
    """Written values within one bf16 step of the rounded definition (or, next to zero, 2^-16 of the
    row's size: the fp32 sums), everything else as it was."""
    rows, lat, key = b.written()
    for got, before, want in zip(write(b), (b.c_kv, b.k_r), (lat, key)):
        got, before = (v.reshape(-1, v.shape[-1]) for v in (host_bits(got), before))
        other = np.ones(len(got), bool)
        other[rows] = False
        assert np.array_equal(got[other], before[other]), "a row of no new token was written"
        if not len(rows):
            continue
        dist = ulp_distance(got[rows], O.round_to_bf16_bits(want))
        near = np.abs(bf16_to_f64(got[rows]) - want) <= 2.0 ** -16 * np.sqrt((want * want).mean(1, keepdims=True))
        assert ((dist <= 1) | near).all(), int(dist.max())


WRITE_DIMS = [TINY, SMALL, SMALL.replace(d_model=1536), SMALL.replace(d_model=320, d_c=64), TEXT.replace(d_c=512),
              TEXT.replace(d_c=256, d_model=2048), SMALL_PAPER.replace(d_model=768)]


@pytest.mark.parametrize("page", [1, 16, 50, 1560])
@pytest.mark.parametrize("dims", WRITE_DIMS, ids=lambda d: f"dc{d.d_c}m{d.d_model}")
def test_write_ragged(dims, page):
    check_write(Batch(dims, RAGGED + [(5, 3, 0), (4, 0, 0), (40, 100, FAR)], page=page, pad=5, seed=12,
                      holes=[(6, 199 // page, -1), (8, 299 // page, 1 << 29)]))


@pytest.mark.parametrize("dims", [TINY, SMALL.replace(d_model=1536), TEXT.replace(d_c=512)], ids=["dc16", "dc192", "dc512"])
def test_write_one_token(dims):
    check_write(Batch(dims, [(1, 1, 0)], page=16, seed=13))


def test_write_many_sequences():
    """More sequences than workgroups, some without new tokens."""
    rng = np.random.default_rng(0)
    check_write(Batch(SMALL, [(int(n), int(n) + 7, i) for i, n in enumerate(rng.integers(0, 3, 900))], page=8, seed=14))


@pytest.mark.parametrize("tokens", [8192, 8193, 9000, 14000, 21000])
def test_write_large_batches(tokens):
    """Around and above 32 tokens per compute unit, where more tokens share a workgroup."""
    b = Batch(SMALL.replace(d_model=768), [(tokens - 5000, tokens - 5000, 3), (0, 0, 0), (4990, 6000, FAR), (10, 12, 0)],
              page=100, pad=7, seed=15)
    check_write(b)


def test_write_without_norm():
    b = Batch(SMALL, [(5, 40, 3)], page=16, seed=16)
    rows, _, _ = b.written()
    got = host_bits(write(b, gamma=False)[0]).reshape(-1, b.dims.d_c)[rows]
    want = bf16_to_f64(b.x) @ bf16_to_f64(b.w_dkv).T
    assert np.abs(bf16_to_f64(got) - want).max() <= 2.0 ** -8 * np.abs(want).max()


# ---- copies -----------------------------------------------------------------------------------

@pytest.mark.parametrize("dims,page,pages,layers,n", [
    (TINY, 1, 3, 1, 1), (TINY, 16, 40, 3, 17), (WAN, 64, 32, 5, 4), (WAN, 1560, 7, 2, 3),
    (WAN.replace(d_c=512), 50, 60, 2, 30), (SMALL, 3, 2000, 1, 900)])
def test_copy(dims, page, pages, layers, n):
    gen = torch.Generator().manual_seed(page)
    c = torch.randint(-2 ** 15, 2 ** 15, (layers, pages, page, dims.d_c), generator=gen, dtype=torch.int16)
    k = torch.randint(-2 ** 15, 2 ** 15, (layers, pages, page, dims.d_rope), generator=gen, dtype=torch.int16)
    order = torch.randperm(pages, generator=gen).to(torch.int32)
    dst = order[:n].contiguous()
    src = order[n:][torch.randint(0, pages - n, (n,), generator=gen)].contiguous()  # some read twice
    got = [t.cuda() for t in (c, k)]
    vm.pages_copy(dims, page, *got, src, dst)
    torch.cuda.synchronize()
    for t, g in zip((c, k), got):
        want = t.clone()
        want[:, dst.long()] = t[:, src.long()]
        assert torch.equal(g.cpu(), want)


def test_copy_reaches_past_4_gib():
    """Byte offsets inside one layer past 32 bits."""
    page, pages = 64, 180_000  # 4.4 GB of latents
    c = torch.zeros(1, pages, page, WAN.d_c, dtype=torch.int16, device="cuda")
    k = torch.zeros(1, pages, page, WAN.d_rope, dtype=torch.int16, device="cuda")
    for t in (c, k):
        t[0, 1] = 7
        t[0, pages - 2] = 9
    vm.pages_copy(WAN, page, c, k, [1, pages - 2], [pages - 1, 0])
    torch.cuda.synchronize()
    for t in (c, k):
        assert (t[0, pages - 1] == 7).all() and (t[0, 0] == 9).all()
        assert int(t.ne(0).sum()) == 4 * page * t.shape[-1]


def test_attend_and_write_past_4_gib():
    """Pages at the end of a pool of more than 4 GiB."""
    b = Batch(SMALL, [(3, 90, 5)], page=64, mask=1, seed=17)
    pages = 180_000
    small = b.table.copy()
    far = {int(p): pages - 1 - int(p) for p in small[small >= 0]}
    b.table = np.where(small >= 0, pages - 1 - small, small).astype(np.int32)
    c = torch.zeros(pages, 64, b.dims.d_c, dtype=torch.bfloat16, device="cuda")
    k = torch.zeros(pages, 64, b.dims.d_rope, dtype=torch.bfloat16, device="cuda")
    paged = b.paged(vm, n_pages=pages)
    for p, q in far.items():
        c[q], k[q] = dev(b.c_kv[p]), dev(b.k_r[p])
    b.table = small
    want, bound = b.attention()
    ws = torch.empty(vm.paged_attend_workspace_bytes(b.dims, paged), dtype=torch.uint8, device="cuda")
    out = torch.empty(b.rows, b.dims.n_heads, b.dims.d_v, dtype=torch.bfloat16, device="cuda")
    vm.paged_attend(b.dims, paged, dev(b.q_nope), dev(b.q_r), dev(b.w_uk), dev(b.w_uv), c, k, out, ws)
    assert_within(bf16_to_f64(host_bits(out)), want, bound, "far pages")
    write(b, paged, (c, k))
    near = write(b)
    for p, q in far.items():
        assert torch.equal(c[q], near[0][p]) and torch.equal(k[q], near[1][p])


# ---- together ---------------------------------------------------------------------------------

def test_paged_equals_the_ring_bit_for_bit_in_the_cache_and_closely_in_the_output():
    """One video, a page per frame: the same chunk-steps through the ring and through pages that leave
    the table's front as frames are evicted."""
    from tests.gpu_common import layer_for
    from workloads import make_layer_inputs
    d = SMALL
    hw, W, C = d.hw, d.window_frames, d.chunk_frames
    inp = make_layer_inputs(d, seed=3, n_frames=12)
    ring = layer_for(vm, inp, "packed_weights")
    pages = 9
    c = torch.zeros(pages, hw, d.d_c, dtype=torch.bfloat16, device="cuda")
    k = torch.zeros(pages, hw, d.d_rope, dtype=torch.bfloat16, device="cuda")
    for fe in range(0, 12, C):
        lo = max(0, fe + C - W)
        frames = list(range(lo, fe + C))
        paged = vm.Paged(
            cu_tokens=torch.tensor([0, C * hw], dtype=torch.int32, device="cuda"),
            kv_len=torch.tensor([len(frames) * hw], dtype=torch.int32, device="cuda"),
            block_table=torch.tensor([[f * 5 % pages for f in frames]], dtype=torch.int32, device="cuda"),
            first_pos=torch.tensor([lo * hw], dtype=torch.int64, device="cuda"), n_tokens=C * hw,
            page_tokens=hw, n_pages=pages)
        ring.write(fe)
        x = ring.x[0, fe * hw:(fe + C) * hw].contiguous()
        vm.paged_cache_write(d, paged, x, ring.w_packed, ring.gamma, c, k)
        for f in frames:
            assert torch.equal(c[f * 5 % pages], ring.c_kv[0].view(W, hw, -1)[f % W])
            assert torch.equal(k[f * 5 % pages], ring.k_r[0].view(W, hw, -1)[f % W])
        want = ring.attend(fe)[0]
        out = torch.zeros(C * hw, d.n_heads, d.d_v, dtype=torch.bfloat16, device="cuda")
        ws = torch.empty(vm.paged_attend_workspace_bytes(d, paged), dtype=torch.uint8, device="cuda")
        vm.paged_attend(d, paged, ring.q_nope, ring.q_r, ring.w_uk, ring.w_uv, c, k, out, ws)
        got = bf16_to_f64(host_bits(out))
        assert np.linalg.norm(got - want) <= 1e-2 * np.linalg.norm(want)


def test_fork_decode_and_compact_in_a_replayed_graph():
    """Write and attention of one step captured once and replayed over steps whose lengths, positions and
    pages change in place; two continuations forked from one prefix; a compaction in between. Every replay
    equals the eager calls on the same cache."""
    d = SMALL
    P, n_pages, layers = 8, 40, 2
    gen = torch.Generator(device="cuda").manual_seed(0)
    rnd = lambda *s: torch.randn(*s, generator=gen, device="cuda").to(torch.bfloat16)  # noqa: E731
    w_dkv, w_kr = rnd(d.d_c, d.d_model) * d.d_model ** -0.5, rnd(d.d_rope, d.d_model) * d.d_model ** -0.5
    w_uk, w_uv = (rnd(d.n_heads * n, d.d_c) * d.d_c ** -0.5 for n in (d.d_nope, d.d_v))
    panel = torch.empty(vm.write_weights_bytes(d), dtype=torch.uint8, device="cuda")
    vm.prepare_write_weights(d, w_dkv, w_kr, panel)
    c, k = rnd(layers, n_pages, P, d.d_c), rnd(layers, n_pages, P, d.d_rope)
    rows = 6
    table = torch.full((3, 10), -1, dtype=torch.int32, device="cuda")
    cu, kv = (torch.zeros(n, dtype=torch.int32, device="cuda") for n in (4, 3))
    first = torch.zeros(3, dtype=torch.int64, device="cuda")
    paged = vm.Paged(cu_tokens=cu, kv_len=kv, block_table=table, first_pos=first, n_tokens=rows,
                     page_tokens=P, n_pages=n_pages, mask_block=1, max_new=4)
    x, qn, qr = (torch.empty(rows, n, dtype=torch.bfloat16, device="cuda")
                 for n in (d.d_model, d.n_heads * d.d_nope, d.n_heads * d.d_rope))
    out = torch.zeros(rows, d.n_heads, d.d_v, dtype=torch.bfloat16, device="cuda")
    ws = torch.empty(vm.paged_attend_workspace_bytes(d, paged), dtype=torch.uint8, device="cuda")

    def step(c, k, out, ws):
        for layer in range(layers):
            vm.paged_cache_write(d, paged, x, panel, None, c[layer], k[layer])
            vm.paged_attend(d, paged, qn, qr, w_uk, w_uv, c[layer], k[layer], out, ws)

    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        step(c, k, out, ws)  # (no sequence has a token yet: nothing is written)
    stream.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        step(c, k, out, ws)
    pages = [[0, 1, 2, 3], [], []]
    lens = [21, 0, 0]
    for n in range(8):
        new = [(2, 1, 1), (1, 0, 3), (1, 1, 1), (0, 2, 4)][n % 4]
        if n == 1:  # two continuations: full pages shared, the last one copied
            tail = lens[0] // P
            for s, p in ((1, 10), (2, 11)):
                vm.pages_copy(d, P, c, k, [pages[0][tail]], [p])
                pages[s], lens[s] = pages[0][:tail] + [p, 20 + s], lens[0]
        if n == 5:  # compaction: the second sequence's own pages move
            own = pages[1][2:]
            vm.pages_copy(d, P, c, k, own, [30 + i for i in range(len(own))])
            pages[1] = pages[1][:2] + [30 + i for i in range(len(own))]
        new = tuple(v if lens[s] else 0 for s, v in enumerate(new)) if n == 0 else new
        for s in range(3):
            lens[s] += new[s]
        cu.copy_(torch.tensor([0, *np.cumsum(new)], dtype=torch.int32))
        kv.copy_(torch.tensor(lens, dtype=torch.int32))
        first.fill_(100 * n)
        for s in range(3):
            row = torch.full((10,), -1, dtype=torch.int32)
            row[:len(pages[s])] = torch.tensor(pages[s], dtype=torch.int32)
            table[s] = row.cuda()
        for t in (x, qn, qr):
            t.copy_(torch.randn(t.shape, generator=gen, device="cuda"))
        out.fill_(3.0)
        mine, theirs, c2, k2 = out, out.clone(), c.clone(), k.clone()
        step(c2, k2, theirs, torch.empty_like(ws))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(c, c2) and torch.equal(k, k2), n
        assert torch.equal(mine, theirs), n
        assert (mine[sum(new):] == 3.0).all() and torch.isfinite(mine).all()


def test_two_streams_with_their_own_workspaces():
    a, b = (Batch(SMALL, [(4, 900, 0), (1, 300, 1)], page=32, mask=1, seed=s) for s in (20, 21))
    want = [host_bits(attend(v)) for v in (a, b)]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    sides = []
    for v in (a, b):
        p = v.paged(vm)
        args = [dev(t) for t in (v.q_nope, v.q_r, v.w_uk, v.w_uv, v.c_kv, v.k_r)]
        out = torch.zeros(v.rows, v.dims.n_heads, v.dims.d_v, dtype=torch.bfloat16, device="cuda")
        sides.append((p, args, out, torch.empty(vm.paged_attend_workspace_bytes(v.dims, p), dtype=torch.uint8, device="cuda")))
    torch.cuda.synchronize()
    for _ in range(5):
        for st, (p, args, out, ws) in zip(streams, sides):
            vm.paged_attend(SMALL, p, *args, out, ws, stream=st)
    torch.cuda.synchronize()
    for (_, _, out, _), w in zip(sides, want):
        assert np.array_equal(host_bits(out), w)


def test_timer_brackets_the_kernels():
    t = vm.Timer()
    b = Batch(SMALL, [(1, 40, 0)], page=16, mask=1, seed=22)
    p = b.paged(vm, timer=t)
    attend(b, p)
    write(b, p)
    for kernel in ("paged_absorb", "paged_attend", "paged_out", "paged_cache_write"):
        n, ms = t.read(kernel)
        assert n == 1 and ms > 0
    t.close()
