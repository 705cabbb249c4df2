"""The bound that sps_paged_attention's precision is held to, itself: a restatement of the kernels' arithmetic passes it, and the
same with a part of the queries or of the probabilities left out, a reference taken late or a sum that cuts does not."""
import math

import pytest
import torch

from paged_precision import equal_weights, hardest_query, hardest_weight, lower, one_query_number, precision, weight_rounding
from paged_util import BF16, F32


def parts_of(x, n):
    """x as a sum of n bf16 numbers, in 64 bits."""
    rest, total = x.float(), torch.zeros(x.shape, dtype=torch.float64)
    for _ in range(n):
        p = rest.to(BF16)
        total += p.double()
        rest = rest - p.float()
    return total


def kernel_form(q, k, v, scale, q_parts, p_parts, late=False, cut=0):
    """One row tile over one part, products in 64 bits: queries and probabilities in bf16 parts, scores relative to the first
    token's, that reference raised by 24 and more only.  late: the rise is taken off differences already rounded.
    cut: outputs summed tile by tile of `cut` tokens, low bits cut off at every step."""
    n, H, d = q.shape
    L, G = k.shape[0], H // k.shape[1]
    kk, vv = k.double().repeat_interleave(G, 1), v.double().repeat_interleave(G, 1)
    s = torch.einsum("nhd,lhd->nhl", parts_of(q, q_parts) if q.dtype == F32 else q.double(), kk).float().double() * (scale * 1.4426950408889634)
    s.masked_fill_((torch.arange(L)[None] > torch.arange(L - n, L)[:, None])[:, None], float("-inf"))
    m = s[..., :1].float().double()
    x = (s - m).float()
    rise = torch.where(x.amax(-1, keepdim=True) > 24, x.amax(-1, keepdim=True), torch.zeros(()))
    x = x - rise if late else (s - torch.where(rise > 0, s.amax(-1, keepdim=True), m).float().double()).float()
    w = torch.exp2(x.double()).float()
    p = parts_of(w, p_parts)
    if cut:
        o = torch.zeros((n, H, d), dtype=torch.float64)
        for t in range(0, L, cut):
            o = o + torch.einsum("nhl,lhd->nhd", p[..., t:t + cut], vv[t:t + cut])
            step = torch.exp2(torch.floor(torch.log2(o.abs().clamp_min(1e-30))) - 23)
            o = torch.trunc(o / step) * step
    else:
        o = torch.einsum("nhl,lhd->nhd", p, vv)
    return (o / w.double().sum(-1, keepdim=True)).float()


def within(out, q, k, v, scale, rows=8, together=False):
    err, allowed = precision(out, q, k, v, scale, weight_rounding(q.dtype, k.dtype, rows), together)
    return err <= allowed


@pytest.mark.parametrize("d", [64, 128])
def test_a_part_of_the_queries_left_out_shows(d):
    q, k, v = one_query_number(3, 4, d, 700, hardest_query(2), F32, BF16, "cpu")
    assert within(kernel_form(q, k, v, 1.0, 3, 3), q, k, v, 1.0, together=True)
    assert not within(kernel_form(q, k, v, 1.0, 2, 3), q, k, v, 1.0, together=True)


@pytest.mark.parametrize("L", [40, 700, 9000])
@pytest.mark.parametrize("q_dtype,parts", [(F32, 3), (BF16, 2)])
def test_a_part_of_the_probabilities_left_out_shows(L, q_dtype, parts):
    scale = math.log(2.0)
    q, k, v = equal_weights(3, 4, 64, L, hardest_weight(parts - 1, q_dtype), q_dtype, BF16, "cpu")
    assert within(kernel_form(q, k, v, scale, 3, parts), q, k, v, scale, together=True)
    assert not within(kernel_form(q, k, v, scale, 3, parts - 1), q, k, v, scale, together=True)


@pytest.mark.parametrize("score", [-1e4, -1e6, -1e9])
@pytest.mark.parametrize("d", [64, 128])
def test_a_reference_taken_late_shows(score, d):
    g = torch.Generator().manual_seed(3)
    q, k, v = torch.randn((2, 4, d), generator=g), torch.randn((400, 1, d), generator=g).to(BF16), torch.randn((400, 1, d), generator=g).to(BF16)
    lower(k, slice(0, 1), score, q)
    scale = d ** -0.5
    assert within(kernel_form(q, k, v, scale, 3, 3), q, k, v, scale)
    assert not within(kernel_form(q, k, v, scale, 3, 3, late=True), q, k, v, scale)


def test_a_running_sum_that_is_cut_shows():
    g = torch.Generator().manual_seed(4)
    q, k = torch.randn((1, 2, 64), generator=g), torch.randn((32768, 1, 64), generator=g).to(BF16)
    v = (torch.rand((32768, 1, 64), generator=g) * 0.5 + 0.5).to(BF16)
    assert within(kernel_form(q, k, v, 0.125, 3, 3), q, k, v, 0.125, together=True)
    assert not within(kernel_form(q, k, v, 0.125, 3, 3, cut=16), q, k, v, 0.125, together=True)
