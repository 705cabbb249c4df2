"""How exact sps_paged_attention has to be: its error in the 2-norm against 64 bits, held to what a plain evaluation in
32 bits makes of the same inputs.  Runs on any device."""
import math

import torch

from paged_util import BF16, F32, HALF

MORE = 3.0     # times the plain form's error: both have the same sources (sums of d and of all tokens, an exponential)


def softmax_form(q, k, v, scale, ftype, together=False):
    """Causal attention of q [n, H, d] over k, v [L, Hkv, d] with the maximum taken first, all in `ftype`: (out, lse, root of
    sum p^2 v^2, or with `together` sum p |v|).  Every row sees something."""
    n, L, G = q.shape[0], k.shape[0], q.shape[1] // k.shape[1]
    kk, vv = k.to(ftype).repeat_interleave(G, 1), v.to(ftype).repeat_interleave(G, 1)
    s = torch.einsum("nhd,lhd->nhl", q.to(ftype), kk) * scale
    hidden = torch.arange(L, device=q.device)[None] > torch.arange(L - n, L, device=q.device)[:, None]
    s.masked_fill_(hidden[:, None], float("-inf"))
    m = s.amax(-1, keepdim=True)
    w = (s - m).exp_()
    t = w.sum(-1, keepdim=True)
    w /= t
    spread = torch.einsum("nhl,lhd->nhd", w, vv.abs()) if together else torch.einsum("nhl,lhd->nhd", w * w, vv * vv).sqrt()
    return torch.einsum("nhl,lhd->nhd", w, vv), (m + t.log())[..., 0], spread


def weight_rounding(q_dtype, cache_dtype, rows_of_a_key_head):
    """Largest relative rounding of a probability ahead of the second product: bf16 parts of 2^-8 each, three for fp32 queries
    (no less than fp32's own), two for bf16 ones, one in tiles of more than 64 rows."""
    if q_dtype == F32 or cache_dtype == F32:
        return 0.0
    return 2.0 ** -8 if rows_of_a_key_head > 64 else 2.0 ** -16


def precision(out, q, k, v, scale, rounding, together=False):
    """(error, allowed) of one sequence's rows.  Roundings of the probabilities are independent of each other: their errors
    add as squares to at most rounding * sqrt(sum p^2 v^2) -- or, where one weight is all tokens' (together), to rounding *
    sum p |v|; 2^-23 of the result stands in where the plain form's error is nil."""
    want, _, spread = softmax_form(q, k, v, scale, torch.float64, together)
    plain = softmax_form(q, k, v, scale, F32)[0].double()
    size = float(want.norm())
    allowed = MORE * (float((plain - want).norm()) + 2.0 ** -23 * size) + rounding * float(spread.norm())
    if together and k.dtype == BF16:
        allowed += float(cuts(q, k, v, scale, want, spread).norm())
    if out.dtype == BF16:
        allowed += HALF[BF16] * size
    return float((out.double() - want).norm()), allowed


def cuts(q, k, v, scale, want, spread):
    """Where all terms have one sign, what the tensor cores cut off running sums instead of rounding it adds up too: at most 2^-23
    of the sum so far at every step of 16.  A score has d / 16 steps (none, if one element is all there is to it), a tile's
    output 128 / 16; sums that grow evenly lose (steps + 1) / 2 times 2^-23.  A score's error moves its token's weight
    against the others'."""
    d, G = q.shape[2], q.shape[1] // k.shape[1]
    steps = 0.0 if int((k != 0).flatten(0, 1).any(0).sum()) <= 1 else (d // 16 + 1) / 2
    kk, vv = k.double().repeat_interleave(G, 1), v.double().repeat_interleave(G, 1)
    n, L = q.shape[0], k.shape[0]
    s = torch.einsum("nhd,lhd->nhl", q.double(), kk) * scale
    s.masked_fill_((torch.arange(L, device=q.device)[None] > torch.arange(L - n, L, device=q.device)[:, None])[:, None], float("-inf"))
    moved = torch.softmax(s, -1) * torch.einsum("nhd,lhd->nhl", q.double().abs(), kk.abs()) * abs(scale)
    by = torch.einsum("nhl,lhd->nhd", moved, vv.abs()) + moved.sum(-1, keepdim=True) * want.abs()
    return 2.0 ** -23 * ((128 // 16 + 1) / 2 * spread + steps * by)


def check_precision(out, lse, q, dense, news, scale=None, max_q=None, together=False):
    """Every sequence of a batch, its log-sum-exp too (which no rounding of the probabilities enters)."""
    scale = 1.0 / math.sqrt(q.shape[2]) if scale is None else scale
    at = 0
    for (k, v), n in zip(dense, news):
        if n:
            r = slice(at, at + n)
            rows = (max_q or max(news)) * (q.shape[1] // k.shape[1])
            err, allowed = precision(out[r], q[r], k, v, scale, weight_rounding(q.dtype, k.dtype, rows), together)
            assert err <= allowed, (err, allowed, err / allowed)
            if lse is not None:
                w64, w32 = (softmax_form(q[r], k, v, scale, t)[1].double() for t in (torch.float64, F32))
                off, may = float((lse[r].double() - w64).norm()), MORE * (float((w32 - w64).norm()) + 2.0 ** -23 * float(w64.norm() + w64.numel() ** 0.5))
                assert off <= may, (off, may)
        at += n


def hardest_weight(parts, dtype):
    """A score t of `dtype` in base 2, 0 < t < 1, whose weight 2^t is as far as can be from the sum of `parts` bf16 parts."""
    t = torch.linspace(0.01, 0.99, 20001, dtype=torch.float64).to(dtype).float()
    rest = w = torch.exp2(t.double()).float()
    for _ in range(parts):
        rest = rest - rest.to(BF16).float()
    return float(t[(rest / w).abs().argmax()])


def hardest_query(parts):
    """A number in 1 .. 2 as far as can be from the sum of `parts` bf16 parts."""
    q = torch.linspace(1.0, 1.99, 20001, dtype=torch.float64).float()
    rest = q
    for _ in range(parts):
        rest = rest - rest.to(BF16).float()
    return float(q[(rest / q).abs().argmax()])


def equal_weights(n, H, d, L, t, q_dtype, cache_dtype, device, seed=0):
    """Every token but the first has the score t in base 2 (with scale = ln 2), the first 0: roundings of the one weight add up
    instead of cancelling.  Values positive."""
    g = torch.Generator().manual_seed(seed)
    q = torch.zeros((n, H, d))
    q[..., 0] = t
    k = torch.zeros((L, 1, d))
    k[1:, :, 0] = 1.0
    v = torch.rand((L, 1, d), generator=g) * 0.5 + 0.5
    return q.to(q_dtype).to(device), k.to(cache_dtype).to(device), v.to(cache_dtype).to(device)


def one_query_number(n, H, d, L, c, q_dtype, cache_dtype, device, seed=0):
    """The queries are c in one element; one token in 350 scores about 6 (as much weight as the others together) and has values of
    the other sign: what is cut off c is cut off that score in proportion and moves the balance."""
    g = torch.Generator().manual_seed(seed)
    q, k = torch.zeros((n, H, d)), torch.zeros((L, 1, d))
    high = torch.arange(L) % 350 == 200
    q[..., 3] = c
    k[high, :, 3] = 6 / c
    v = torch.rand((L, 1, d), generator=g) * 0.5 + 0.5
    v[high] *= -1
    return q.to(q_dtype).to(device), k.to(cache_dtype).to(device), v.to(cache_dtype).to(device)


def lower(k, tokens, score, q):
    """Makes `score` (before the scale) of the given tokens through the last head element: 1 in every query, 0 in the other keys."""
    q[..., -1] = 1.0
    k[..., -1] = 0.0
    k[tokens, :, -1] = score
