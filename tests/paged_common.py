"""A batch of sequences over a paged cache, and the definitions of its operators in 64 bits (numpy),
with the bounds that the roundings of the kernels' arithmetic give."""
import numpy as np
import torch

from oracle import videomla_oracle as O
from tests.gpu_common import bf16_to_f64
from workloads import _normal_bf16

U = 2.0 ** -8  # a rounding to bf16 is off by at most half a step, 2^-8 of the value


def rope(dims, v, pos):
    """v [..][d_rope] rotated at absolute token positions pos (broadcast against v[..., 0])."""
    hw = dims.grid_h * dims.grid_w
    axes = (pos // hw, pos % hw // dims.grid_w, pos % dims.grid_w)
    out = np.array(v, dtype=np.float64)
    p = 0
    for a, n in enumerate(dims.rope_pairs):
        band = dims.rope_band_dim[a] or 2 * n
        for k in range(n):
            ang = axes[a] * dims.rope_base ** (-2.0 * k / band)
            u, w = v[..., 2 * p], v[..., 2 * p + 1]
            out[..., 2 * p] = u * np.cos(ang) - w * np.sin(ang)
            out[..., 2 * p + 1] = u * np.sin(ang) + w * np.cos(ang)
            p += 1
    return out


class Batch:
    """seqs: (new tokens, cached tokens, absolute position of the first cached token) per sequence."""

    def __init__(self, dims, seqs, page, seed=0, pad=0, mask=0, window=0, spare=3, extra_cols=1, gain=1.0,
                 max_new=0, holes=(), with_first=True):
        self.dims, self.seqs, self.page, self.mask, self.window = dims, seqs, page, mask, window
        self.max_new, self.with_first = max_new, with_first
        rng = np.random.default_rng(seed)
        self.rng = rng
        per = [-(-kv // page) for _, kv, _ in seqs]
        self.cols = max(per) + extra_cols
        self.n_pages = sum(per) + spare
        order = rng.permutation(self.n_pages)
        self.table = np.full((len(seqs), self.cols), -1, np.int32)
        at = 0
        for s, n in enumerate(per):
            self.table[s, :n] = order[at:at + n]
            at += n
        for s, col, value in holes:
            self.table[s, col] = value
        self.cu = np.concatenate([[0], np.cumsum([n for n, _, _ in seqs])]).astype(np.int32)
        self.kv = np.array([k for _, k, _ in seqs], np.int32)
        self.first = np.array([f for _, _, f in seqs], np.int64)
        self.tokens = int(self.cu[-1])
        self.rows = self.tokens + pad
        d, H = dims, dims.n_heads
        self.x = _normal_bf16(rng, (self.rows, d.d_model))
        self.w_dkv = _normal_bf16(rng, (d.d_c, d.d_model), d.d_model ** -0.5)
        self.w_kr = _normal_bf16(rng, (d.d_rope, d.d_model), d.d_model ** -0.5)
        self.gamma = _normal_bf16(rng, (d.d_c,), 1.0)
        self.w_uk = _normal_bf16(rng, (H * d.d_nope, d.d_c), d.d_c ** -0.5)
        self.w_uv = _normal_bf16(rng, (H * d.d_v, d.d_c), d.d_c ** -0.5)
        self.q_nope = _normal_bf16(rng, (self.rows, H, d.d_nope), gain)
        self.q_r = _normal_bf16(rng, (self.rows, H, d.d_rope), gain)
        self.c_kv = _normal_bf16(rng, (self.n_pages, page, d.d_c))
        self.k_r = _normal_bf16(rng, (self.n_pages, page, d.d_rope))

    def pool_row(self, s, j):
        """Row of the flat pool of cached token j of sequence s, or -1."""
        if not 0 <= j < self.kv[s]:
            return -1
        p = self.table[s, j // self.page]
        return p * self.page + j % self.page if 0 <= p < self.n_pages else -1

    def paged(self, vm, **kw):
        """The description of the batch, its arrays on the device."""
        t = lambda a: torch.from_numpy(a).cuda()  # noqa: E731
        args = dict(cu_tokens=t(self.cu), kv_len=t(self.kv), block_table=t(self.table),
                    first_pos=t(self.first) if self.with_first else None, n_tokens=self.rows,
                    page_tokens=self.page, n_pages=self.n_pages, max_new=self.max_new,
                    mask_block=self.mask, window_tokens=self.window)
        return vm.Paged(**{**args, **kw})

    def seen(self, s, i):
        """The cached tokens, holes left out, that the query at cached index i of sequence s sees."""
        kv, first = int(self.kv[s]), int(self.first[s]) if self.with_first else 0
        end = (first + i) // self.mask * self.mask + self.mask - first if self.mask else kv
        beg = end - self.window if self.window else 0
        return [j for j in range(max(0, beg), min(kv, end)) if self.pool_row(s, j) >= 0]

    def attention(self):
        """(out, bound) [rows][H][d_v]: the attention of every token in its per-head form, NaN for rows
        of no sequence, and how far the kernels' roundings can move each value. With u = 2^-8:
          q_cat rounded to bf16 moves a score by at most u sum |q k| scale;
          p and the p that the sum takes are the same rounded values: p (1 + u) / sum;
          both move the weights: |d out| <= sum_j p_j d_j |v_j - out| with d_j the relative change;
          o_lat and out are each rounded: u sum |W| |o_lat| + u |out|.
        Twice the sum of the first-order terms covers the products of roundings and the fp32 sums."""
        d, H = self.dims, self.dims.n_heads
        f = bf16_to_f64
        uk, uv = f(self.w_uk).reshape(H, d.d_nope, d.d_c), f(self.w_uv).reshape(H, d.d_v, d.d_c)
        ckv, kr = f(self.c_kv).reshape(-1, d.d_c), f(self.k_r).reshape(-1, d.d_rope)
        scale = d.softmax_scale or (d.d_nope + d.d_rope) ** -0.5
        out = np.full((self.rows, H, d.d_v), np.nan)
        bound = np.zeros_like(out)
        for s in range(len(self.seqs)):
            n, first = int(self.cu[s + 1] - self.cu[s]), int(self.first[s]) if self.with_first else 0
            for t in range(n):
                i, row = int(self.kv[s]) - n + t, int(self.cu[s]) + t
                js = self.seen(s, i)
                out[row] = 0
                if not js:
                    continue
                r = np.array([self.pool_row(s, j) for j in js])
                qr = rope(d, f(self.q_r[row]), np.array(max(0, first + i)))
                lat = np.einsum("hn,hnc->hc", f(self.q_nope[row]), uk)
                c, k = ckv[r], kr[r]
                sc = (lat @ c.T + qr @ k.T) * scale
                ds = U * (np.abs(lat) @ np.abs(c).T + np.abs(qr) @ np.abs(k).T) * scale
                p = np.exp(sc - sc.max(1, keepdims=True))
                p /= p.sum(1, keepdims=True)
                o = p @ c
                v = np.einsum("jc,hvc->hjv", c, uv)
                out[row] = np.einsum("hj,hjv->hv", p, v)
                rel = ds + ds.max(1, keepdims=True) + 2 * U
                moved = np.einsum("hj,hjv->hv", p * rel, np.abs(v - out[row][:, None]))
                rounds = U * (np.einsum("hc,hvc->hv", np.abs(o), np.abs(uv)) + np.abs(out[row]))
                bound[row] = 2 * (moved + rounds) + 1e-6
        return out, bound

    def written(self):
        """(pool rows, latents, keys) of the new tokens that the write places."""
        d = self.dims
        f = bf16_to_f64
        rows, toks, pos = [], [], []
        for s in range(len(self.seqs)):
            n, first = int(self.cu[s + 1] - self.cu[s]), int(self.first[s]) if self.with_first else 0
            for t in range(n):
                i = int(self.kv[s]) - n + t
                if self.pool_row(s, i) >= 0:
                    rows.append(self.pool_row(s, i))
                    toks.append(int(self.cu[s]) + t)
                    pos.append(first + i)
        x = f(self.x[toks])
        c = x @ f(self.w_dkv).T
        c = c / np.sqrt((c * c).mean(1, keepdims=True) + d.kv_norm_eps) * f(self.gamma)
        return np.array(rows, int), c, rope(d, x @ f(self.w_kr).T, np.array(pos, int))


def attention_by_sequence(b, device):
    """Batch.attention for calls of many tokens: the same sums in torch, all heads' keys and values of a
    sequence at once, its tokens in blocks."""
    d, H = b.dims, b.dims.n_heads
    f = lambda a: torch.from_numpy(bf16_to_f64(a)).to(device)  # noqa: E731
    uk, uv = f(b.w_uk).view(H, d.d_nope, d.d_c), f(b.w_uv).view(H, d.d_v, d.d_c)
    ckv, kr = f(b.c_kv).view(-1, d.d_c), f(b.k_r).view(-1, d.d_rope)
    scale = d.softmax_scale or (d.d_nope + d.d_rope) ** -0.5
    out = np.full((b.rows, H, d.d_v), np.nan)
    bound = np.zeros_like(out)
    for s in range(len(b.seqs)):
        lo, hi, kv = int(b.cu[s]), int(b.cu[s + 1]), int(b.kv[s])
        rows = np.array([b.pool_row(s, j) for j in range(kv)], int)
        first = int(b.first[s]) if b.with_first else 0
        if kv == 0:
            out[lo:hi] = 0
            continue
        c, k = ckv[rows], kr[rows]
        for t0 in range(lo, hi, 32):
            toks = np.arange(t0, min(t0 + 32, hi))
            at = kv - hi + toks
            see = torch.zeros(len(toks), kv, dtype=torch.bool)
            for n, i in enumerate(at):
                see[n, b.seen(s, int(i))] = True
            see = see.to(device)
            qr = torch.from_numpy(rope(d, bf16_to_f64(b.q_r[toks]), np.maximum(0, first + at)[:, None])).to(device)
            qn = f(b.q_nope[toks])
            for h in range(H):
                lat = qn[:, h] @ uk[h]
                sc = ((lat @ c.t() + qr[:, h] @ k.t()) * scale).masked_fill(~see, -np.inf)
                ds = (lat.abs() @ c.abs().t() + qr[:, h].abs() @ k.abs().t()) * (U * scale)
                ds = ds.masked_fill(~see, 0.0)
                p = torch.where(see.any(1, keepdim=True), sc.softmax(1), 0.0)
                v = c @ uv[h].t()
                o = p @ v
                rel = ds + ds.amax(1, keepdim=True) + 2 * U
                moved = ((p * rel)[..., None] * (v[None] - o[:, None]).abs()).sum(1)
                rounds = U * ((p @ c).abs() @ uv[h].abs().t() + o.abs())
                out[toks, h] = o.cpu().numpy()
                bound[toks, h] = torch.where(see.any(1, keepdim=True), 2 * (moved + rounds) + 1e-6, 0.0).cpu().numpy()
    return out, bound


def assert_within(got, want, bound, label):
    """got (bf16 values) within the bound of every value, and 1e-2 of the whole in the 2-norm."""
    live = ~np.isnan(want)
    err = np.abs(got - want)[live]
    worst = (err / np.maximum(bound[live], 1e-300)).max() if err.size else 0.0  # (bound 0: exactly zero)
    norm = np.linalg.norm(want[live])
    rel = np.linalg.norm(err) / norm if norm else float(err.any())
    print(f"{label}: worst {worst:.3f} of the bound, relL2 {rel:.2e}, n {err.size}", flush=True)
    assert np.isfinite(got[live]).all(), label
    assert worst <= 1, (label, worst)
    assert rel <= 1e-2, (label, rel)
