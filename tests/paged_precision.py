"""How exact sps_paged_attention has to be: its error in the 2-norm against 64 bits, held to what a plain evaluation in
32 bits makes of the same inputs.  Runs on any device."""
import math

import torch

from paged_util import BF16, F32, HALF

MORE = 3.0     # times the plain form's error: both have the same sources (sums of d and of all tokens, an exponential)


def softmax_form(q, k, v, scale, ftype):
    """Causal attention of q [n, H, d] over k, v [L, Hkv, d] with the maximum taken first, all in `ftype`: (out, lse, root of
    sum p^2 v^2).  Every row sees something."""
    n, L, G = q.shape[0], k.shape[0], q.shape[1] // k.shape[1]
    kk, vv = k.to(ftype).repeat_interleave(G, 1), v.to(ftype).repeat_interleave(G, 1)
    s = torch.einsum("nhd,lhd->nhl", q.to(ftype), kk) * scale
    hidden = torch.arange(L, device=q.device)[None] > torch.arange(L - n, L, device=q.device)[:, None]
    s.masked_fill_(hidden[:, None], float("-inf"))
    m = s.amax(-1, keepdim=True)
    w = (s - m).exp_()
    t = w.sum(-1, keepdim=True)
    w /= t
    return torch.einsum("nhl,lhd->nhd", w, vv), (m + t.log())[..., 0], torch.einsum("nhl,lhd->nhd", w * w, vv * vv).sqrt()


def weight_rounding(q_dtype, cache_dtype, rows_of_a_key_head):
    """Largest relative rounding of a probability ahead of the second product: bf16 parts of 2^-8 each, three for fp32 queries
    (no less than fp32's own), two for bf16 ones, one in tiles of more than 64 rows."""
    if q_dtype == F32 or cache_dtype == F32:
        return 0.0
    return 2.0 ** -8 if rows_of_a_key_head > 64 else 2.0 ** -16


def precision(out, q, k, v, scale, rounding):
    """(error, allowed) of one sequence's rows.  Roundings of the probabilities are independent of each other: their errors
    add as squares to at most rounding * sqrt(sum p^2 v^2); 2^-23 of the result stands in where the plain form's error is nil."""
    want, _, spread = softmax_form(q, k, v, scale, torch.float64)
    plain = softmax_form(q, k, v, scale, F32)[0].double()
    size = float(want.norm())
    allowed = MORE * (float((plain - want).norm()) + 2.0 ** -23 * size) + rounding * float(spread.norm())
    if out.dtype == BF16:
        allowed += HALF[BF16] * size
    return float((out.double() - want).norm()), allowed


def check_precision(out, lse, q, dense, news, scale=None, max_q=None):
    """Every sequence of a batch, its log-sum-exp too (which no rounding of the probabilities enters)."""
    scale = 1.0 / math.sqrt(q.shape[2]) if scale is None else scale
    at = 0
    for (k, v), n in zip(dense, news):
        if n:
            r = slice(at, at + n)
            rows = (max_q or max(news)) * (q.shape[1] // k.shape[1])
            err, allowed = precision(out[r], q[r], k, v, scale, weight_rounding(q.dtype, k.dtype, rows))
            assert err <= allowed, (err, allowed, err / allowed)
            if lse is not None:
                w64, w32 = (softmax_form(q[r], k, v, scale, t)[1].double() for t in (torch.float64, F32))
                off, may = float((lse[r].double() - w64).norm()), MORE * (float((w32 - w64).norm()) + 2.0 ** -23 * float(w64.norm() + w64.numel() ** 0.5))
                assert off <= may, (off, may)
        at += n


def lower(k, tokens, score, q):
    """Makes `score` (before the scale) of the given tokens through the last head element: 1 in every query, 0 in the other keys."""
    q[..., -1] = 1.0
    k[..., -1] = 0.0
    k[tokens, :, -1] = score
