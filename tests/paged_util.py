"""Inputs and 64-bit references shared by the tests of the rotary / paged-cache operators."""
import math

import torch

import paper_2302_01318_b200 as sps

DEV = "cuda"
F32, BF16 = torch.float32, torch.bfloat16
HALF = {F32: 2.0 ** -24, BF16: 2.0 ** -8}     # largest relative error of one rounding to the type


def normal(shape, dtype=F32, seed=0, std=1.0):
    g = torch.Generator(device=DEV).manual_seed(seed)
    return (torch.randn(shape, generator=g, device=DEV) * std).to(dtype)


def freqs(rot, base=10000.0, **kw):
    return torch.from_numpy(sps.sps_rotary_frequencies(rot, base, **kw)).to(DEV)


def rotate64(x, pos, freq, layout, gain=1.0, transposed=False):
    """x [rows, heads, d] in 64 bits, rotated element by element."""
    x = x.double()
    rot = 2 * freq.shape[0]
    a = pos.double()[:, None] * freq[None]
    c, s = a.cos()[:, None] * gain, a.sin()[:, None] * (-gain if transposed else gain)
    i = torch.arange(rot // 2, device=x.device)
    ia, ib = (2 * i, 2 * i + 1) if layout == "pairs" else (i, i + rot // 2)
    y = x.clone()
    y[..., ia] = x[..., ia] * c - x[..., ib] * s
    y[..., ib] = x[..., ia] * s + x[..., ib] * c
    return y


def rotate_tol(x, freq, layout, gain, out_dtype):
    """sincosf is within 2 ulp of a value of at most 1 (2^-22), products and their difference round to 2^-24 each: together
    under 2^-21 (|a| + |b|) |gain| per element of a pair, then the rounding to the output's type."""
    rot = 2 * freq.shape[0]
    i = torch.arange(rot // 2, device=x.device)
    ia, ib = (2 * i, 2 * i + 1) if layout == "pairs" else (i, i + rot // 2)
    t = torch.zeros_like(x, dtype=torch.float64)
    m = (x[..., ia].double().abs() + x[..., ib].double().abs()) * abs(gain)
    t[..., ia] = m
    t[..., ib] = m
    return t * 2.0 ** -21 + (t + x.double().abs()) * HALF[out_dtype] * (1.0 if out_dtype != F32 else 0.0)


class Pages:
    """A page pool and table for sequences of the given lengths; page numbers scattered, the pool's other slots hold `fill`."""

    def __init__(self, lens, Hkv, d, page, dtype, seed=0, order="head", fill=float("nan"), spare=2, n_pages=None, extra_cols=1):
        g = torch.Generator().manual_seed(seed)
        self.lens, self.page = list(lens), page
        need = [-(-max(L, 0) // page) for L in lens]
        total = sum(need) + spare
        self.n_pages = n_pages or total
        perm = torch.randperm(self.n_pages, generator=g)[:total].to(torch.int32)
        self.table = torch.full((len(lens), max(need + [0]) + extra_cols), 2 ** 31 - 1, dtype=torch.int32)   # unused entries: far out of range
        at = 0
        for b, n in enumerate(need):
            self.table[b, :n] = perm[at:at + n]
            at += n
        shape = (self.n_pages, Hkv, page, d) if order == "head" else (self.n_pages, page, Hkv, d)
        self.k = torch.full(shape, fill, dtype=dtype, device=DEV)
        self.v = torch.full(shape, fill, dtype=dtype, device=DEV)
        if order != "head":
            self.k, self.v = self.k.transpose(1, 2), self.v.transpose(1, 2)
        self.dense = []
        for b, L in enumerate(lens):
            k, v = normal((max(L, 0), Hkv, d), dtype, 2 * (seed + 17 * b)), normal((max(L, 0), Hkv, d), dtype, 2 * (seed + 17 * b) + 1)
            j = torch.arange(max(L, 0))
            p, s = self.table[b, j // page].long().to(DEV), (j % page).to(DEV)
            self.k[p, :, s] = k
            self.v[p, :, s] = v
            self.dense.append((k, v))
        self.cache = sps.PagedCache(self.k, self.v)

    def batch(self, news, lead=0, max_q=None):
        q_start = torch.tensor([lead] + list(news), dtype=torch.int32).cumsum(0).to(torch.int32).to(DEV)
        return sps.PagedBatch(q_start, torch.tensor(self.lens, dtype=torch.int32, device=DEV), self.table.to(DEV),
                              max_q=max(list(news) + [1]) if max_q is None else max_q)


def attention64(q, dense, news, lead=0, scale=None):
    """Per sequence and head in 64 bits: (out, lse, S) with S the sizes the tolerance needs: sum p |v|, sum over e of
    scale |q_e k_je| maximised over the visible j, visible tokens, largest |v|."""
    rows, H, d = q.shape
    scale = 1.0 / math.sqrt(d) if scale is None else scale
    out = torch.zeros((rows, H, d), dtype=torch.float64, device=q.device)
    lse = torch.full((rows, H), float("-inf"), dtype=torch.float64, device=q.device)
    pv, mag = torch.zeros_like(out), torch.zeros_like(lse)
    seen = torch.zeros((rows, H), dtype=torch.float64, device=q.device)
    a = lead
    for (k, v), n in zip(dense, news):
        L, Hkv = k.shape[0], k.shape[1]
        G = H // Hkv
        for i in range(n):
            p = L - n + i
            if p < 0:
                continue
            kk, vv = k[:p + 1].double().repeat_interleave(G, 1), v[:p + 1].double().repeat_interleave(G, 1)
            qq = q[a + i].double()
            s = torch.einsum("hd,jhd->hj", qq, kk) * scale
            w = torch.softmax(s, -1)
            out[a + i] = torch.einsum("hj,jhd->hd", w, vv)
            pv[a + i] = torch.einsum("hj,jhd->hd", w, vv.abs())
            lse[a + i] = torch.logsumexp(s, -1)
            mag[a + i] = (torch.einsum("hd,jhd->hj", qq.abs(), kk.abs()) * abs(scale)).amax(-1)
            seen[a + i] = p + 1
        a += n
    return out, lse, (pv, mag, seen)


def attention_tol(out, S, d, q_dtype, out_dtype):
    """Products are exact or rounded to 2^-24; each of the additions of a score (d of them), of the sum and of the output
    (as many as tokens are seen, or partial sums of them) is off by at most 2^-23 relative (tensor cores may cut instead of
    rounding).  A score's error is then (d + 8) 2^-23 times its terms' sum of magnitudes, twice that the relative error of a
    weight against its sum; sums add 2 seen 2^-23.  16-bit queries: weights round to bf16, 2^-8 each, in numerator and
    sum.  Everything multiplies sum p |v|; the output's own rounding comes last."""
    pv, mag, seen = S
    rel = 2 * (d + 8) * 2.0 ** -23 * mag + 2 * (seen + 16) * 2.0 ** -23
    if q_dtype == BF16:
        rel = rel + 2 * 2.0 ** -8
    return pv * rel[..., None] + out.abs() * HALF[out_dtype] + 1e-30


def workspace(cache, H, q_dtype):
    return torch.zeros(sps.sps_paged_attention_workspace_bytes(cache, H, q_dtype), dtype=torch.uint8, device=DEV)


def run_attention(pages, news, H, q_dtype, out_dtype=None, seed=5, lead=0, tail=0, q=None, ws=None, scale=None, max_q=None, std=1.5):
    """One call and its check against attention64, rows before and behind the batch untouched.  Returns (out, lse, batch, ws)."""
    d = pages.cache.k.shape[3]
    rows = lead + sum(news) + tail
    if q is None:
        q = normal((rows, H, d), q_dtype, seed, std)
    out = torch.full((rows, H, d), 7.0, dtype=out_dtype or q_dtype, device=DEV)
    lse = torch.full((rows, H), 7.0, device=DEV)
    ws = workspace(pages.cache, H, q_dtype) if ws is None else ws
    batch = pages.batch(news, lead, max_q)
    sps.sps_paged_attention(pages.cache, batch, q, out, ws, scale=scale or 0.0, lse=lse)
    torch.cuda.synchronize()
    check_attention(out, lse, q, pages.dense, news, lead, scale)
    assert int(batch.status) == 0
    return out, lse, batch, ws


def check_attention(out, lse, q, dense, news, lead=0, scale=None):
    d, end = q.shape[2], lead + sum(news)
    want, wl, S = attention64(q, dense, news, lead, scale)
    tol = attention_tol(want, S, d, q.dtype, out.dtype)
    inside = slice(lead, end)
    err = (out.double() - want).abs()[inside]
    assert torch.isfinite(out[inside].float()).all()
    assert (err <= tol[inside]).all(), float((err / tol[inside]).max())
    if lse is not None:
        empty = torch.isinf(wl[inside])
        assert torch.equal(empty, torch.isinf(lse[inside]))
        pv, mag, seen = S
        lt = 2 * (d + 8) * 2.0 ** -23 * mag + 2 * (seen + 16) * 2.0 ** -23 + wl.abs().nan_to_num(0, 0, 0) * 2.0 ** -22 + (2.0 ** -8 if q.dtype == BF16 else 0)
        assert ((lse.double() - wl)[inside][~empty].abs() <= lt[inside][~empty]).all()
        assert (lse[:lead] == 7).all() and (lse[end:] == 7).all()
    assert (out[:lead] == 7).all() and (out[end:] == 7).all()
