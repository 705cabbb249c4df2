"""How exact sps_paged_attention is: low scores at the head of a context, of a tile or of a CTA's part; precision held to a
plain evaluation in 32 bits."""
import math

import pytest
import torch

import paper_2302_01318_b200 as sps
from paged_precision import check_precision, equal_weights, hardest_query, hardest_weight, lower, one_query_number
from paged_util import BF16, DEV, F32, Pages, normal, workspace

pytestmark = pytest.mark.gpu

TYPES = [(F32, F32, F32), (F32, BF16, F32), (BF16, BF16, BF16), (BF16, BF16, F32)]   # q, cache, out


def put(pages, b, k=None, v=None):
    """New keys or values of a sequence into its pages (the dense copies follow)."""
    for new, dense, pool in ((k, pages.dense[b][0], pages.k), (v, pages.dense[b][1], pages.v)):
        if new is not None:
            dense.copy_(new)
            j = torch.arange(dense.shape[0])
            pool[pages.table[b, j // pages.page].long().to(DEV), :, (j % pages.page).to(DEV)] = dense


def attend(pages, q, news, odt, scale=None, max_q=None):
    out = torch.full(q.shape, 7.0, dtype=odt, device=DEV)
    lse = torch.full(q.shape[:2], 7.0, device=DEV)
    batch = pages.batch(news, max_q=max_q)
    sps.sps_paged_attention(pages.cache, batch, q, out, workspace(pages.cache, q.shape[1], q.dtype), scale=scale or 0.0, lse=lse)
    torch.cuda.synchronize()
    assert int(batch.status) == 0
    return out, lse


# -3e38 twice over is beyond fp32: a score of -inf (an infinite key would be NaN in the parts of an fp32 query)
LOW = [-1e4, -1e6, -1e9, -3e38]


@pytest.mark.parametrize("score", LOW)
@pytest.mark.parametrize("new", [1, 3, 5, 7])                # 8, 24, 40 and 56 rows of a key head: every width of the few-row tiles
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("types", range(len(TYPES)))
def test_a_low_score_ahead_of_the_others(types, d, new, score):
    """The first token's, and in the second sequence every tile's first one: wherever a part begins."""
    qdt, cdt, odt = TYPES[types]
    pages = Pages([300, 9000], 1, d, 16, cdt)
    q = normal((2 * new, 8, d), qdt, 1, 1.5)
    for b, tokens in ((0, slice(0, 1)), (1, slice(0, 9000, 128))):
        k = pages.dense[b][0].clone()
        lower(k, tokens, score, q)
        put(pages, b, k)
    q[..., -1] = 2.0
    out, lse = attend(pages, q, [new, new], odt)
    check_precision(out, lse, q, pages.dense, [new, new])


@pytest.mark.parametrize("new", [1, 3, 5, 7])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("types", range(len(TYPES)))
def test_a_score_of_minus_infinity_ahead_of_very_low_ones(types, d, new):
    """No reference left at 0, where weights of scores around -300 would all vanish: the first tile's scores but one overflow to
    -inf (a later tile raises the reference), in the second sequence only the first token's of every tile."""
    qdt, cdt, odt = TYPES[types]
    pages = Pages([700, 9000], 1, d, 16, cdt)
    q = normal((2 * new, 8, d), qdt, 1, 1.5)
    scale = d ** -0.5
    for b, tokens in ((0, slice(0, 128)), (1, slice(0, 9000, 128))):
        k = pages.dense[b][0].clone()
        lower(k, tokens, -3e38, q)
        q[..., -2] = 16.0
        k[..., -2] = -300 / 16 / scale
        put(pages, b, k)
    q[..., -1] = 2.0
    out, lse = attend(pages, q, [new, new], odt)
    check_precision(out, lse, q, pages.dense, [new, new])


@pytest.mark.parametrize("score", LOW)
@pytest.mark.parametrize("below", [0.0, -300.0])             # of the other scores
@pytest.mark.parametrize("new", [9, 40])                     # 72 and 320 rows of a key head: one or both tiles of 128, several items
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("types", range(len(TYPES)))
def test_whole_tiles_of_low_scores_ahead_of_the_others(types, d, new, below, score):
    """The first 128 tokens, and in the second sequence every other tile of 128."""
    qdt, cdt, odt = TYPES[types]
    pages = Pages([700, 5000], 1, d, 16, cdt)
    q = normal((2 * new, 8, d), qdt, 1, 1.5)
    for b in range(2):
        L = pages.dense[b][0].shape[0]
        j = torch.arange(L, device=DEV)
        k = pages.dense[b][0].clone()
        lower(k, j // 128 % 2 == 0 if b else j < 128, score, q)
        if below:
            q[..., -2] = 16.0
            k[..., -2] = below / 16 * d ** 0.5
        put(pages, b, k)
    q[..., -1] = 2.0
    out, lse = attend(pages, q, [new, new], odt)
    check_precision(out, lse, q, pages.dense, [new, new])


# rows of a key head: every width of the few-row tiles, one and two tiles of 128, several items
ROWS = [(1, 4), (3, 8), (5, 8), (8, 8), (9, 8), (40, 8)]     # new rows, query heads (on one key head)


@pytest.mark.parametrize("new,H", ROWS)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("types", range(len(TYPES)))
def test_as_exact_as_a_plain_evaluation_in_32_bits(types, d, new, H):
    qdt, cdt, odt = TYPES[types]
    pages = Pages([50, 129, 9000], 1, d, 16, cdt)
    news = [new, min(new, 100), new]
    q = normal((sum(news), H, d), qdt, 2, 1.5)
    out, lse = attend(pages, q, news, odt)
    check_precision(out, lse, q, pages.dense, news)


@pytest.mark.parametrize("new,H", ROWS)
@pytest.mark.parametrize("L", [50, 700, 9000])
@pytest.mark.parametrize("types", range(len(TYPES)))
def test_no_part_of_the_probabilities_is_missing(types, L, new, H):
    qdt, cdt, odt = TYPES[types]
    parts = 3 if qdt == F32 else (1 if new * H > 64 else 2)
    pages = Pages([L], 1, 64, 16, cdt)
    q, k, v = equal_weights(new, H, 64, L, hardest_weight(max(parts - 1, 1), qdt), qdt, cdt, DEV)
    put(pages, 0, k, v)
    out, _ = attend(pages, q, [new], odt, scale=math.log(2.0))
    check_precision(out, None, q, pages.dense, [new], scale=math.log(2.0), together=True)


@pytest.mark.parametrize("new,H", ROWS)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("cdt", [F32, BF16])
def test_no_part_of_the_queries_is_missing(cdt, d, new, H):
    pages = Pages([700], 1, d, 16, cdt)
    q, k, v = one_query_number(new, H, d, 700, hardest_query(2), F32, cdt, DEV)
    put(pages, 0, k, v)
    out, _ = attend(pages, q, [new], F32, scale=1.0)
    check_precision(out, None, q, pages.dense, [new], scale=1.0, together=True)


@pytest.mark.parametrize("types", range(len(TYPES)))
def test_long_sums_are_not_cut(types):
    qdt, cdt, odt = TYPES[types]
    pages = Pages([32768], 1, 64, 64, cdt)
    v = torch.rand((32768, 1, 64), generator=torch.Generator().manual_seed(4)) * 0.5 + 0.5
    put(pages, 0, v=v.to(DEV).to(cdt))
    q = normal((1, 2, 64), qdt, 3)
    out, _ = attend(pages, q, [1], odt)
    check_precision(out, None, q, pages.dense, [1], together=True)
