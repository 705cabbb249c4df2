"""Beams that are alike -- one score, the same logits -- tie in every candidate, and places decide, wherever their rows lie; and
what a selection returns is looked up: each candidate's own score in 64 bits."""
import math

import pytest
import torch

import paper_2302_01318_b200 as sps
from pages_util import BF16, DEV, F32, I32, run_select

pytestmark = pytest.mark.gpu
INF = math.inf


def rows(shape, dtype=F32, seed=0, pad=0, offset=0):
    """Normal logits; rows pad elements apart, the first one offset elements behind an allocation's begin."""
    B, W, V = shape
    g = torch.Generator(device=DEV).manual_seed(seed)
    store = torch.randn(offset + B * W * (V + pad), generator=g, device=DEV).mul_(3.0).to(dtype)
    return store[offset:].view(B, W, V + pad)[..., :V]


def check(o, logits, scores, done=None, end=-1, N=4, T=1.0):
    """Beams fall into classes of alike ones.  A class orders its candidates exactly: by logit, then beam.  What a selection takes of a
    class has to be the first of that order, in that order; and its scores are the N best, within rounding, in 64 bits.

    Tolerance of a score: a beam's sum of exponentials is of V fp32 terms.  Their exponents have one rounding of a difference at
    most (3 2^-24 |l - max| / T with the factors', the same once more for parts' own maxima), each exponential is within 2^-22, a
    lane adds up at most V / 256 + 32 of them and 13 partial sums follow: relative to the sum this is the log's error.  Two sums
    may differ by twice that, and the result is rounded once."""
    B, W, V = logits.shape
    out_s, out_p, out_t = (x.tolist() for x in o[:3])
    score, top = scores.tolist(), logits.amax(-1).tolist()
    ended = [[0] * W] * B if done is None else done.tolist()
    for b in range(B):
        c = torch.full((W, V), -INF, dtype=torch.float64, device=DEV)
        tol, classes = 0.0, []
        for w in range(W):
            s = score[b][w]
            if not math.isfinite(s):
                continue
            like = [cl for cl in classes if not ended[b][w] and not ended[b][cl[0]] and score[b][cl[0]] == s and top[b][cl[0]] == top[b][w] and
                    bool((logits[b, cl[0]] == logits[b, w]).all())]
            if like:
                like[0].append(w)
            else:
                classes.append([w])
            if ended[b][w]:
                c[w, end] = s
                continue
            x = logits[b, w].double()
            below = (x - x.max()) / T
            lse = torch.exp(below).sum().log()
            c[w] = s + below - lse
            far = float((torch.exp(below - lse) * (-below).clamp(max=1e30)).sum())
            tol = max(tol, 2 * (6 * far + 8 + V / 256 + 32 + 13 + 1) * 2.0 ** -24)
        best = c.view(-1).topk(min(N, W * V)).values
        best = best[best > -INF].tolist()
        n = len(best)
        got = [(p - b * W, t) for p, t in zip(out_p[b], out_t[b])]
        assert all(x == (-1 - b * W, -1) for x in got[n:]) and all(0 <= w < W and 0 <= t < V for w, t in got[:n])
        for i, (w, t) in enumerate(got[:n]):
            own = float(c[w, t])
            assert abs(out_s[b][i] - best[i]) <= tol + abs(best[i]) * 2.0 ** -24
            assert abs(out_s[b][i] - own) <= tol + abs(own) * 2.0 ** -24
        for cl in classes:
            mine = [(w, t) for w, t in got[:n] if w in cl]
            x = c[cl[0]] if ended[b][cl[0]] else torch.where(logits[b, cl[0]] > -INF, logits[b, cl[0]].double(), -INF)
            k = min(len(mine) // len(cl) + 1, V)
            cut = x.topk(k).values[-1]
            at = (x >= cut).nonzero()[:, 0]
            order = sorted((-v, w, t) for v, t in zip(x[at].tolist(), at.tolist()) for w in cl)
            assert mine == [(w, t) for _, w, t in order[:len(mine)]], (b, cl)


SHAPES = [(8, 8, 32000, F32, 0, 0), (1, 8, 32000, F32, 0, 0), (1, 4, 32000, F32, 0, 0), (64, 4, 32000, F32, 0, 0), (64, 4, 131071, BF16, 1, 0), (1, 4, 32001, F32, 0, 0),
          (1, 4, 32001, BF16, 0, 0), (30, 4, 32001, F32, 0, 3), (5, 16, 4099, BF16, 0, 1), (32, 16, 32000, F32, 0, 0), (2, 128, 700, F32, 1, 0), (40, 3, 515, BF16, 0, 0),
          (3, 2, 1_000_003, F32, 0, 0), (1, 3, 7, F32, 0, 0)]


@pytest.mark.parametrize("B,W,V,dtype,pad,offset", SHAPES)
def test_all_beams_alike(B, W, V, dtype, pad, offset):
    x = rows((B, W, V), dtype, B + W + V, pad, offset)
    x.copy_(x[:, :1].clone().expand(B, W, V))
    s = torch.full((B, W), -1.25, device=DEV)
    for N, T in ((W, 1.0), (min(128, 3 * W + 1), 0.7)):
        check(run_select(x, s, N=N, T=T), x, s, N=N, T=T)


@pytest.mark.parametrize("B,W,V,dtype,pad,offset", SHAPES)
def test_some_beams_alike(B, W, V, dtype, pad, offset):
    """Every other beam is like the first, one more is like the second but for its score, the last one like the first but for an element."""
    x = rows((B, W, V), dtype, B + W + V + 1, pad, offset)
    x[:, 0::2] = x[:, :1].clone()
    s = torch.full((B, W), -1.25, device=DEV)
    if W > 3:
        x[:, 3] = x[:, 1].clone()
        s[:, 3] -= 2.0 ** -20
        x[:, -1] = x[:, 0].clone()
        x[:, -1, V // 2] -= 0.5
    N = min(2 * W, 128)
    check(run_select(x, s, N=N), x, s, N=N)


def test_rows_that_begin_alike():
    """Beams that differ in one place only, far behind: the first one, the last one, and one that is like a later beam."""
    B, W, V = 2, 6, 40000
    for dtype, pad in ((F32, 0), (F32, 1), (BF16, 3)):
        x = rows((B, W, V), dtype, 77, pad)
        x.copy_(x[:, :1].clone().expand(B, W, V))
        x[:, 1, V - 1] -= 2.0
        x[:, 3, V - 1] -= 2.0                                  # like beam 1, not like beam 0
        x[:, 2, 0] -= 2.0
        x[:, 5, 9000] -= 2.0
        s = torch.full((B, W), -3.0, device=DEV)
        check(run_select(x, s, N=60), x, s, N=60)


def test_masks_zeros_ended_and_missing_beams_among_alike_ones():
    B, W, V = 4, 8, 33001
    x = rows((B, W, V), F32, 5)
    x.copy_(x[:, :1].clone().expand(B, W, V))
    x[:, :, 300:] = -INF
    x[:, :, 40] = 0.0
    x[:, 4, 40] = -0.0                                         # (the same number)
    s = torch.full((B, W), -2.0, device=DEV)
    s[1, 0] = s[2, 2] = -INF
    s[3, 1] = math.nan
    done = torch.zeros((B, W), dtype=I32, device=DEV)
    done[0, 0] = done[2, 5] = done[2, 6] = 1
    check(run_select(x, s, done, 7, N=40), x, s, done, 7, N=40)
    none = s.clone()
    none[2, 1] = none[0, 3] = -INF                             # their logits make them no beams, whatever their scores are
    x[2, 1] = math.nan
    x[0, 3] = -INF
    check(run_select(x, s, done, 7, N=40), x, none, done, 7, N=40)


def test_beams_that_share_one_row_of_logits():
    """A stride of zero between rows."""
    x = rows((1, 1, 32000), F32, 6).expand(1, 5, 32000)
    s = torch.full((1, 5), -1.0, device=DEV)
    check(run_select(x, s, N=23), x, s, N=23)


def test_one_score_and_unlike_logits():
    """A program that starts W unlike beams from one score: scores alone make none alike."""
    for B, W, V, dtype in ((3, 128, 500, BF16), (20, 128, 500, BF16), (2, 16, 32000, F32)):
        x = rows((B, W, V), dtype, 11)
        s = torch.zeros((B, W), device=DEV)
        check(run_select(x, s, N=50), x, s, N=50)


@pytest.mark.parametrize("B", [2, 40])
def test_what_the_workspace_holds_never_matters(B):
    x, s = rows((B, 4, 20001), F32, 9), torch.tensor([[-1.0, -INF, -2.0, -1.0]], device=DEV).repeat(B, 1)
    want = run_select(x, s, N=6)
    ws = torch.full((sps.sps_beam_select_workspace_bytes(B, 4, 20001),), 255, dtype=torch.uint8, device=DEV)
    for _ in range(2):
        assert all(torch.equal(a, b) for a, b in zip(want, run_select(x, s, N=6, ws=ws)))
