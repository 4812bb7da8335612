"""The paged latent cache's operators as measurable cases.

A program that serves streams of different lengths keeps the latents c_kv and the rotated keys k_r in
pages of a pool and, per stream, a row of a block table that names its pages. Per step and layer it
writes the new tokens of every stream (`write`) and attends their queries over the stream's pages
(`attend`); a stream that is forked, or a pool that is compacted, copies pages in every layer (`copy`).

Every case is a dict of plain values:
  op                      write | attend | copy
  d_model .. d_v, grid_*  the layer's shapes (videomla_dims)
  split                   RoPE channel split: wan (8, 4, 4 pairs), text (all pairs to the first axis) or
                          tiny (2, 1, 1)
  page, spare             tokens per page; the pool's pages beyond the used ones, in percent
  seqs                    sequences
  new_lo, new_hi          new tokens per sequence, spread evenly over this range
  kv_lo, kv_hi            cached tokens per sequence, new ones included, spread over this range
  pad                     rows behind the last sequence, which the call leaves alone
  first                   largest absolute position of a sequence's first cached token
  mask, window            block size of the causal mask (0: none), tokens of the sliding window (0: all)
  layers, pairs           copy: layers of the pool and copied pages
  gain                    factor on the queries (1: flat softmax, 4: peaked)
"""
from __future__ import annotations

import math
from types import SimpleNamespace

import torch

own = False

BF16 = torch.bfloat16

_WAN = dict(d_model=1536, n_heads=12, d_nope=128, d_rope=32, d_c=192, d_v=128, grid_h=30, grid_w=52,
            split="wan", page=64, spare=25, seqs=1, new_lo=1, new_hi=1, kv_lo=1, kv_hi=1, pad=0,
            first=0, mask=1, window=0, layers=1, pairs=0, gain=1.0)
_TINY = dict(_WAN, d_model=64, n_heads=2, d_nope=32, d_rope=8, d_c=16, d_v=32, grid_h=4, grid_w=4,
             split="tiny", page=16)
_TEXT = dict(_WAN, grid_h=1, grid_w=1, split="text")


def listed():
    """The listed cases: writes, attention and page copies, each smallest first."""
    def case(name, base, op, **kw):
        return dict(base, name=name, op=op, **kw)
    return [
        # one new token for each of 16 token streams: the write of a decoding step
        case("write-decode-16", _TEXT, "write", seqs=16, kv_lo=100, kv_hi=9000, first=100000),
        # ragged chunks of six streams, pages of an odd size, a padded batch
        case("write-ragged-6", _WAN, "write", seqs=6, new_lo=37, new_hi=1201, kv_lo=1300, kv_hi=6000,
             page=50, first=50000, pad=96),
        # a 3-frame video chunk for each of four streams at different frames, a page per frame
        case("write-chunk-4", _WAN, "write", seqs=4, new_lo=4680, new_hi=4680, kv_lo=4680, kv_hi=32760,
             page=1560, first=200000),
        # the smallest decoding step: one token over a few hundred
        case("decode-1", _TEXT, "attend", kv_lo=517, kv_hi=517),
        # a served batch: 32 streams of up to a whole video window, one token each
        case("decode-32", _TEXT, "attend", seqs=32, kv_lo=2000, kv_hi=32760, first=100000, pad=4),
        # the widest latent of the d_c sweep, decoding
        case("decode-16-dc512", _TEXT, "attend", seqs=16, d_c=512, kv_lo=4000, kv_hi=16000, page=128,
             gain=4.0),
        # four drafted tokens per stream checked at once, small pages
        case("verify-8", _TEXT, "attend", seqs=8, new_lo=4, new_hi=4, kv_lo=3000, kv_hi=16000, page=16),
        # ragged chunks of new tokens over their contexts, causal, pages that end inside a key tile
        case("chunk-ragged-6", _TEXT, "attend", seqs=6, new_lo=37, new_hi=900, kv_lo=1500, kv_hi=9000,
             page=50, first=50000),
        # a whole prompt under a sliding window
        case("prompt-window", _TEXT, "attend", new_lo=8190, new_hi=8190, kv_lo=8190, kv_hi=8190,
             window=4096, page=128),
        # one Wan2.1-1.3B layer's 3-frame chunk over the full 21-frame window, a page per frame
        case("video-chunk", _WAN, "attend", new_lo=4680, new_hi=4680, kv_lo=32760, kv_hi=32760,
             page=1560, mask=4680, first=182520),
        # four continuations of a stream get their own copy of its last page, 30 layers
        case("fork-4", _WAN, "copy", page=64, layers=30, pairs=4, spare=700),
        # a pool is compacted: half of its pages move, 30 layers
        case("compact-500", _WAN, "copy", page=64, layers=30, pairs=500, spare=100),
    ]


# A drawn case costs no more than the largest listed one, and its plain form fits the card.
_MAX_FLOPS, _MAX_BYTES, _MAX_SCORES = 1.5e12, 9e8, 1.84e9


def draw(rng):
    """One more case of the same ranges."""
    def log_int(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    while True:
        op = rng.choice(["write", "attend", "attend", "attend", "copy"])
        c = dict(_TINY if rng.random() < 0.1 else rng.choice([_TEXT, _WAN]), op=op)
        if c["d_c"] > 16:
            c["d_c"] = rng.choice([64, 128, 192, 192, 192, 256, 512])
            c["n_heads"] = rng.choice([8, 12, 12, 16])
            c["d_model"] = rng.choice([768, 1024, 1536, 1536])
            c["d_nope"] = rng.choice([96, 128, 128])
            if c["split"] == "wan":
                c.update(grid_h=log_int(6, 30), grid_w=log_int(8, 52))
        c["page"] = rng.choice([16, 32, 50, 64, 64, 100, 128, 256, log_int(17, 2000)])
        if op == "copy":
            c.update(layers=log_int(1, 30), pairs=log_int(1, 500), spare=rng.randint(100, 400),
                     page=min(c["page"], 256))
        else:
            kind = rng.choice(["one", "few", "chunk"])
            c["seqs"] = log_int(1, 64) if kind != "chunk" else log_int(1, 8)
            c["new_lo"] = {"one": 1, "few": rng.randint(1, 4), "chunk": log_int(20, 4000)}[kind]
            c["new_hi"] = {"one": 1, "few": rng.randint(4, 24), "chunk": c["new_lo"] + log_int(1, 1000)}[kind]
            c["kv_lo"] = c["new_hi"] + rng.choice([0, log_int(1, 4000)])
            c["kv_hi"] = c["kv_lo"] + rng.choice([0, log_int(1, 30000)])
            c["pad"] = rng.choice([0, 0, rng.randint(1, 100)])
            c["first"] = rng.choice([0, log_int(1, 1000000)])
            c["mask"] = rng.choice([1, 1, 0, log_int(2, 2000)])
            c["window"] = rng.choice([0, 0, log_int(16, 20000)])
            c["gain"] = rng.choice([1.0, 1.0, 4.0])
        w = work(c)
        if w["flops"] > _MAX_FLOPS or w["bytes"] > _MAX_BYTES:
            continue
        if op == "copy" or c["seqs"] * c["new_hi"] * c["n_heads"] * c["kv_hi"] <= _MAX_SCORES:
            return c


# ---- shapes ---------------------------------------------------------------------------------

_PAIRS = {"wan": (8, 4, 4), "text": (16, 0, 0), "tiny": (2, 1, 1)}


def _dims(c):
    return SimpleNamespace(
        d_model=c["d_model"], n_heads=c["n_heads"], d_nope=c["d_nope"], d_rope=c["d_rope"],
        d_c=c["d_c"], d_v=c["d_v"], grid_h=c["grid_h"], grid_w=c["grid_w"], window_frames=21,
        chunk_frames=3, rope_pairs=_PAIRS[c["split"]], rope_band_dim=(0, 0, 0), rope_base=10000.0,
        softmax_scale=0.0, kv_norm_eps=1e-6, sink_frames=0)


def _spread(lo, hi, n):
    """n whole numbers from lo to hi, evenly spaced, in a mixed order."""
    v = [lo + (hi - lo) * i // max(1, n - 1) for i in range(n)]
    return v[::2] + v[1::2]


def _lens(c):
    """(new tokens, cached tokens, absolute position of the first cached token) of every sequence."""
    n = c["seqs"]
    return (_spread(c["new_lo"], c["new_hi"], n), _spread(c["kv_lo"], c["kv_hi"], n)[::-1],
            _spread(0, c["first"], n) if n > 1 else [c["first"]])


def _pages(c):
    """Pages that the sequences use, the columns of the block table, the pool's pages."""
    if c["op"] == "copy":
        return c["pairs"], 0, 2 * c["pairs"] + c["pairs"] * (c["spare"] - 100) // 100
    per = [-(-k // c["page"]) for k in _lens(c)[1]]
    return sum(per), max(per), sum(per) + sum(per) * c["spare"] // 100 + 1


def _seen(c, n, kv, first):
    """(first, end) of the cached tokens that the query at cached index i sees, for the n last i."""
    out = []
    for i in range(kv - n, kv):
        end = ((first + i) // c["mask"] + 1) * c["mask"] - first if c["mask"] else kv
        out.append((max(0, end - c["window"]) if c["window"] else 0, min(kv, end)))
    return out


def work(case):
    c = case
    H, dm, dn, dr, dc, dv = c["n_heads"], c["d_model"], c["d_nope"], c["d_rope"], c["d_c"], c["d_v"]
    row = (dc + dr) * 2
    if c["op"] == "copy":
        return {"bytes": 2 * c["layers"] * c["pairs"] * c["page"] * row, "flops": 0}
    new, kv, first = _lens(c)
    tokens = sum(new)
    meta = c["seqs"] * 16 + 4 * _pages(c)[0]
    if c["op"] == "write":
        return {"bytes": tokens * (2 * dm + row) + (dc + dr) * dm * 2 + meta,
                "flops": 2 * tokens * (dc + dr) * dm}
    pairs, cached = 0, 0
    for n, k, f in zip(new, kv, first):
        seen = _seen(c, n, k, f)
        pairs += sum(max(0, e - b) for b, e in seen)
        cached += max(0, max(e for _, e in seen) - min(b for b, _ in seen))
    return {"bytes": tokens * H * (dn + dr + dv) * 2 + cached * row + H * (dn + dv) * dc * 2 + meta,
            "flops": 2 * tokens * H * (dn * dc + dc * dv) + 2 * pairs * H * (2 * dc + dr)}


# ---- inputs ---------------------------------------------------------------------------------

def prepare(case, seed):
    """Seeded inputs on the GPU: activations N(0, 1), weights N(0, 1 / fan_in), latents of unit RMS as the
    cache's norm leaves them, all bf16; pages in a shuffled order. With the framework's operators also what
    a program keeps from step to step: the packed weight panel, the workspace and the description of the
    batch, which holds the same tensors."""
    c = case
    gen = torch.Generator(device="cuda").manual_seed(seed)
    host = torch.Generator().manual_seed(seed)

    def normal(*shape, std=1.0):
        return (torch.randn(*shape, generator=gen, device="cuda") * std).to(BF16)

    dm, dn, dr, dc, dv, H = (c[k] for k in ("d_model", "d_nope", "d_rope", "d_c", "d_v", "n_heads"))
    used, cols, n_pages = _pages(c)
    s = SimpleNamespace(c=c, dims=_dims(c))
    s.c_kv = normal(c["layers"], n_pages, c["page"], dc)
    s.k_r = normal(c["layers"], n_pages, c["page"], dr)
    order = torch.randperm(n_pages, generator=host)
    if c["op"] == "copy":
        s.src, s.dst = (order[k * used:(k + 1) * used].to(torch.int32) for k in (0, 1))
        s.src_index, s.dst_index = s.src.long().cuda(), s.dst.long().cuda()
        if own:
            import paper_2605_30351_amd as vm
            s.vm = vm
        return s
    s.c_kv, s.k_r = s.c_kv[0], s.k_r[0]
    new, kv, first = _lens(c)
    s.tokens = sum(new)
    s.rows = s.tokens + c["pad"]
    table = torch.full((c["seqs"], cols), -1, dtype=torch.int32)
    at = 0
    for k, n in enumerate(kv):
        p = -(-n // c["page"])
        table[k, :p] = order[at:at + p]
        at += p
    s.table = table.cuda()
    s.cu = torch.tensor([0] + new, dtype=torch.int64).cumsum(0).to(torch.int32).cuda()
    s.kv = torch.tensor(kv, dtype=torch.int32).cuda()
    s.first = torch.tensor(first, dtype=torch.int64).cuda()
    s.max_new, s.max_kv = max(new), max(kv)
    if c["op"] == "write":
        s.x = normal(s.rows, dm)
        s.w_dkv, s.w_kr = normal(dc, dm, std=dm ** -0.5), normal(dr, dm, std=dm ** -0.5)
        s.gamma = (1 + 0.1 * torch.randn(dc, generator=gen, device="cuda")).to(BF16)
    else:
        s.q_nope, s.q_r = normal(s.rows, H, dn, std=c["gain"]), normal(s.rows, H, dr, std=c["gain"])
        s.w_uk, s.w_uv = normal(H * dn, dc, std=dc ** -0.5), normal(H * dv, dc, std=dc ** -0.5)
        s.out = torch.zeros(s.rows, H, dv, dtype=BF16, device="cuda")
    if own:
        import paper_2605_30351_amd as vm
        s.vm = vm
        s.paged = vm.Paged(
            cu_tokens=s.cu, kv_len=s.kv, first_pos=s.first, block_table=s.table, n_tokens=s.rows,
            page_tokens=c["page"], n_pages=n_pages, max_new=s.max_new, mask_block=c["mask"],
            window_tokens=c["window"])
        if c["op"] == "write":
            s.panel = torch.empty(vm.write_weights_bytes(s.dims), dtype=torch.uint8, device="cuda")
            vm.prepare_write_weights(s.dims, s.w_dkv, s.w_kr, s.panel)
        else:
            s.ws = torch.empty(vm.paged_attend_workspace_bytes(s.dims, s.paged), dtype=torch.uint8,
                               device="cuda")
    return s


# ---- one pass -------------------------------------------------------------------------------

def run(state):
    s = state
    op = s.c["op"]
    if op == "copy":
        if own:
            s.vm.pages_copy(s.dims, s.c["page"], s.c_kv, s.k_r, s.src, s.dst)
        else:
            _plain_copy(s)
        return s.c_kv, s.k_r
    if op == "write":
        if own:
            s.vm.paged_cache_write(s.dims, s.paged, s.x, s.panel, s.gamma, s.c_kv, s.k_r)
        else:
            _plain_write(s)
        return s.c_kv, s.k_r
    if own:
        s.vm.paged_attend(s.dims, s.paged, s.q_nope, s.q_r, s.w_uk, s.w_uv, s.c_kv, s.k_r, s.out, s.ws)
    else:
        _plain_attend(s)
    return s.out


def _plain_copy(s):
    s.c_kv[:, s.dst_index] = s.c_kv[:, s.src_index]
    s.k_r[:, s.dst_index] = s.k_r[:, s.src_index]


def _cos_sin(s, pos):
    """cos and sin [tokens][pairs] of the rotation at absolute token positions pos (angles in 64 bits)."""
    d, pairs = s.dims, s.dims.rope_pairs
    hw = d.grid_h * d.grid_w
    axes = torch.stack([pos // hw, pos % hw // d.grid_w, pos % d.grid_w], 1).double()
    n = torch.arange(max(pairs), device=pos.device, dtype=torch.float64)
    angle = torch.cat([axes[:, a:a + 1] * d.rope_base ** (-n[:p] / max(1, p)) for a, p in enumerate(pairs)], 1)
    return angle.cos().float(), angle.sin().float()


def _rotate(v, cos, sin):
    u, w = v[..., 0::2], v[..., 1::2]
    return torch.stack([u * cos - w * sin, u * sin + w * cos], -1).flatten(-2)


def _tokens(s):
    """(sequence, cached index) of every new token."""
    t = torch.arange(s.tokens, device="cuda", dtype=torch.int32)
    q = torch.searchsorted(s.cu, t, right=True) - 1
    return q, (s.kv[q] - s.cu[q + 1] + t).long()


def _plain_write(s):
    q, i = _tokens(s)
    y = s.x[:s.tokens].float() @ torch.cat([s.w_dkv, s.w_kr]).float().t()
    c, k = y.split([s.dims.d_c, s.dims.d_rope], 1)
    c = c * torch.rsqrt(c.square().mean(1, keepdim=True) + s.dims.kv_norm_eps) * s.gamma.float()
    cos, sin = _cos_sin(s, s.first[q] + i)
    P = s.c["page"]
    row = s.table[q, i // P].long() * P + i % P
    s.c_kv.view(-1, s.dims.d_c)[row] = c.to(BF16)
    s.k_r.view(-1, s.dims.d_rope)[row] = _rotate(k, cos, sin).to(BF16)


def _plain_attend(s):
    d, P = s.dims, s.c["page"]
    n, H, dev = s.c["seqs"], d.n_heads, s.table.device
    q, i = _tokens(s)
    slot = torch.arange(s.tokens, device=dev) - s.cu[q]
    # queries absorbed and rotated, padded to [sequence][max_new][head]
    lat = torch.bmm(s.q_nope[:s.tokens].float().transpose(0, 1),
                    s.w_uk.float().view(H, d.d_nope, d.d_c)).transpose(0, 1)
    cos, sin = _cos_sin(s, s.first[q] + i)
    rot = _rotate(s.q_r[:s.tokens].float(), cos[:, None], sin[:, None])
    qs = torch.zeros(n, s.max_new, H, d.d_c + d.d_rope, device=dev)
    qs[q, slot] = torch.cat([lat, rot], 2) * (d.d_nope + d.d_rope) ** -0.5
    # the context of every sequence, gathered from its pages and padded
    page = s.table[:, :-(-s.max_kv // P)].clamp(min=0).long()
    c = s.c_kv[page].flatten(1, 2)[:, :s.max_kv].float()
    k = torch.cat([c, s.k_r[page].flatten(1, 2)[:, :s.max_kv].float()], 2)
    # what each query sees: [sequence][max_new][key]
    at = torch.zeros(n, s.max_new, dtype=torch.int64, device=dev)
    at[q, slot] = i
    key = torch.arange(s.max_kv, device=dev)
    B, W = s.c["mask"], s.c["window"]
    end = ((s.first[:, None] + at) // B + 1) * B - s.first[:, None] if B else s.kv[:, None].expand(n, s.max_new)
    seen = (key < end[..., None]) & (key < s.kv[:, None, None])
    if W:
        seen &= key >= end[..., None] - W
    x = torch.bmm(qs.flatten(1, 2), k.transpose(1, 2)).view(n, s.max_new, H, s.max_kv)
    x.masked_fill_(~seen[:, :, None], -math.inf)
    x.sub_(x.amax(3, keepdim=True).clamp(min=-3e38)).exp_()
    o = torch.bmm(x.flatten(1, 2), c).view(n, s.max_new, H, d.d_c)
    o = (o / x.sum(3)[..., None].clamp(min=1e-30))[q, slot]
    out = torch.bmm(o.transpose(0, 1), s.w_uv.float().view(H, d.d_v, d.d_c).transpose(1, 2))
    s.out[:s.tokens] = out.transpose(0, 1).to(BF16)


# ---- the definition in 64 bits --------------------------------------------------------------

def exact(case, seed):
    """What run() returns, from the definitions in 64 bits: a sequence at a time, the attention in its
    per-head form (keys W_UK c and values W_UV c of every cached token), the rotation as a product of
    complex numbers."""
    c, s = case, prepare(case, seed)
    if c["op"] == "copy":
        a, b = s.c_kv.double(), s.k_r.double()
        for t in (a, b):
            t.index_copy_(1, s.dst_index, t.index_select(1, s.src_index))
        return a, b
    D = torch.float64
    new, kv, first = _lens(c)
    P, H, dr = c["page"], c["n_heads"], c["d_rope"]

    def turned(v, pos):
        """v [token][..][d_rope] rotated at the positions of its tokens."""
        coords = (pos // (c["grid_h"] * c["grid_w"]), pos // c["grid_w"] % c["grid_h"], pos % c["grid_w"])
        angle = [coords[a].to(D) * 10000.0 ** (-2.0 * j / (2 * n))
                 for a, n in enumerate(_PAIRS[c["split"]]) for j in range(n)]
        unit = torch.polar(torch.ones((), dtype=D, device="cuda"), torch.stack(angle, -1))
        z = torch.view_as_complex(v.unflatten(-1, (dr // 2, 2)).contiguous())
        return torch.view_as_real(z * unit.view(len(pos), *[1] * (v.dim() - 2), dr // 2)).flatten(-2)

    def rows_of(k):
        """Pool rows of all cached tokens of sequence k."""
        j = torch.arange(kv[k], device="cuda")
        return s.table[k].long()[torch.div(j, P, rounding_mode="floor")] * P + j % P

    at = 0
    if c["op"] == "write":
        ckv, kr = s.c_kv.double().view(-1, c["d_c"]), s.k_r.double().view(-1, dr)
        for k in range(c["seqs"]):
            n = new[k]
            x = s.x[at:at + n].double()
            lat = torch.mm(x, s.w_dkv.double().t())
            lat = lat / (lat.pow(2).sum(1, keepdim=True) / c["d_c"] + 1e-6).sqrt() * s.gamma.double()
            pos = torch.arange(first[k] + kv[k] - n, first[k] + kv[k], device="cuda")
            r = rows_of(k)[kv[k] - n:]
            ckv[r], kr[r] = lat, turned(torch.mm(x, s.w_kr.double().t()), pos)
            at += n
        return ckv.view(s.c_kv.shape), kr.view(s.k_r.shape)
    out = s.out.double()
    for k in range(c["seqs"]):
        n, r = new[k], rows_of(k)
        ctx, key_r = s.c_kv.view(-1, c["d_c"])[r].double(), s.k_r.view(-1, dr)[r].double()
        index = torch.arange(kv[k] - n, kv[k], device="cuda")
        q_r = turned(s.q_r[at:at + n].double(), first[k] + index)
        lo, hi = (torch.tensor(v, device="cuda")[:, None] for v in zip(*_seen(c, n, kv[k], first[k])))
        j = torch.arange(kv[k], device="cuda")[None]
        hidden = (j < lo) | (j >= hi)
        for h in range(H):
            up_k = s.w_uk[h * c["d_nope"]:(h + 1) * c["d_nope"]].double()
            up_v = s.w_uv[h * c["d_v"]:(h + 1) * c["d_v"]].double()
            score = torch.mm(s.q_nope[at:at + n, h].double(), torch.mm(ctx, up_k.t()).t())
            score = (score + torch.mm(q_r[:, h], key_r.t())) / math.sqrt(c["d_nope"] + dr)
            weight = score.masked_fill(hidden, -math.inf).softmax(1).nan_to_num(0.0)
            out[at:at + n, h] = torch.mm(weight, torch.mm(ctx, up_v.t()))
        at += n
    return out
