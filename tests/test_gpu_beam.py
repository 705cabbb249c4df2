"""The selection of a beam step against 64-bit scores, and the cases where its order or its masks can go wrong."""
import math

import pytest
import torch

import paper_2302_01318_b200 as sps
from pages_util import BF16, DEV, F32, I32, check_select, run_select

pytestmark = pytest.mark.gpu
INF = math.inf


def normal(shape, dtype=F32, seed=0, std=3.0, pad=0):
    g = torch.Generator(device=DEV).manual_seed(seed)
    t = (torch.randn(shape[:-1] + (shape[-1] + pad,), generator=g, device=DEV) * std).to(dtype)
    return t[..., :shape[-1]]


def beams(B, W, seed=0):
    g = torch.Generator().manual_seed(seed)
    return (-(torch.rand((B, W), generator=g) * 12 + 1)).to(DEV)


def run_and_check(logits, scores, done=None, end=-1, N=4, T=1.0, exact_ties=False):
    o = run_select(logits, scores, done, end, N, T)
    check_select(o, logits, scores, done, end, N, T, exact_ties)
    return o


@pytest.mark.parametrize("B,W,V,N,dtype,pad,T", [(1, 1, 1, 1, F32, 0, 1.0), (1, 1, 16, 16, F32, 0, 1.0), (3, 2, 5, 8, BF16, 0, 1.0), (1, 4, 32000, 4, F32, 0, 1.0),
                                                 (8, 8, 1024, 16, F32, 0, 0.7), (2, 4, 127, 8, F32, 1, 1.0), (2, 4, 129, 8, BF16, 1, 1.0), (5, 3, 8193, 7, F32, 3, 1.5),
                                                 (4, 5, 32001, 10, BF16, 3, 1.0), (2, 3, 131071, 6, BF16, 1, 0.7), (2, 2, 131072, 128, F32, 0, 1.0),
                                                 (1, 128, 777, 128, F32, 0, 1.0), (70, 2, 300, 4, BF16, 8, 1.0), (1, 2, 1_000_003, 5, F32, 0, 1.0), (300, 1, 64, 1, F32, 0, 2.0)])
def test_against_64_bits(B, W, V, N, dtype, pad, T):
    run_and_check(normal((B, W, V), dtype, B + V, pad=pad), beams(B, W, V), N=N, T=T)


@pytest.mark.parametrize("B,W,V,N,dtype,pad", [(8192, 1, 33, 2, F32, 0), (1, 128, 32000, 128, F32, 0), (20, 4, 32001, 6, BF16, 3), (19, 5, 8001, 64, F32, 1),
                                               (40, 3, 515, 5, BF16, 0), (3, 7, 90_001, 100, BF16, 7)])
def test_many_sequences_wide_beams_and_unaligned_rows_in_both_forms(B, W, V, N, dtype, pad):
    run_and_check(normal((B, W, V), dtype, B + V, pad=pad), beams(B, W, V), N=N)


@pytest.mark.parametrize("B,W,V,N,dtype", [(3, 15, 873, 13, BF16), (20, 15, 873, 13, BF16), (2, 1, 15000, 128, F32), (20, 1, 15000, 127, F32), (2, 3, 500, 100, BF16),
                                           (20, 2, 4097, 64, F32), (1, 1, 9000, 65, BF16)])
def test_fewer_segments_than_candidates_or_about_as_many(B, W, V, N, dtype):
    """The segments' maxima then say little, or nothing, about the N-th candidate; one beam may hold them all."""
    s = beams(B, W, V)
    run_and_check(normal((B, W, V), dtype, B + V), s, N=N)
    s[:, 0] += 40
    run_and_check(normal((B, W, V), dtype, B + V + 1, std=0.5), s, N=N)


def test_sequences_of_which_many_beams_are_dead_or_done():
    """Whole runs of rows are skipped, and parts begin and end beside them."""
    B, W, V = 60, 16, 3001
    x, s = normal((B, W, V), seed=31), beams(B, W, 3)
    g = torch.Generator().manual_seed(9)
    s[(torch.rand((B, W), generator=g) < 0.5).to(DEV)] = -INF
    s[7:25] = -INF
    s[25, 15] = -1.0
    done = (torch.rand((B, W), generator=g) < 0.3).to(I32).to(DEV)
    done[40:44] = 1
    run_and_check(x, s, done, 11, N=9)


def test_two_calls_at_once_on_streams_and_workspaces_of_their_own():
    shapes = [(2, 4, 32000), (70, 4, 32000)]
    data = [(normal(sh, seed=i), beams(*sh[:2], i)) for i, sh in enumerate(shapes)]
    want = [run_select(x, s, N=4) for x, s in data]
    streams = [torch.cuda.Stream() for _ in shapes]
    got, ws = [], []
    for x, s in data:
        got.append([torch.zeros((x.shape[0], 4), device=DEV)] + [torch.zeros((x.shape[0], 4), dtype=I32, device=DEV) for _ in range(2)])
        ws.append(torch.zeros(sps.sps_beam_select_workspace_bytes(*x.shape), dtype=torch.uint8, device=DEV))
    torch.cuda.synchronize()
    for _ in range(20):
        for (x, s), o, w, st in zip(data, got, ws, streams):
            sps.sps_beam_select(x, s, *o, w, stream=st.cuda_stream)
    torch.cuda.synchronize()
    for a, b in zip(got, want):
        assert all(torch.equal(p, q) for p, q in zip(a, b))


@pytest.mark.parametrize("offset", [1, 2, 3, 5])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_rows_of_any_alignment(offset, dtype):
    B, W, V = 2, 3, 4099
    flat = normal((B * W * V + offset,), dtype, 7)
    run_and_check(flat[offset:].view(B, W, V), beams(B, W), N=6)


@pytest.mark.parametrize("V", [1, 7, 250, 4093])
@pytest.mark.parametrize("dtype,pad,offset", [(F32, 1, 1), (F32, 5, 0), (BF16, 13, 3), (BF16, 8, 0), (BF16, 1, 7)])
def test_what_lies_between_the_rows_never_matters(V, dtype, pad, offset):
    """NaN ahead of the first row, between rows and behind the last one; both forms of the call."""
    for B, W in ((2, 3), (40, 3)):
        store = torch.full((offset + B * W * (V + pad) + 8,), math.nan, dtype=dtype, device=DEV)
        x = store[offset:offset + B * W * (V + pad)].view(B, W, V + pad)[..., :V]
        x.copy_(normal((B, W, V), dtype, V))
        run_and_check(x, beams(B, W), N=5)


def test_one_beam_rows_may_lie_a_batch_stride_apart():
    x = normal((4, 3, 500))[:, 1:2]
    run_and_check(x, beams(4, 1), N=3)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("V,N", [(700, 9), (40000, 128)])
def test_equal_logits_fall_to_the_lowest_place(dtype, V, N):
    """Whole rows of one value, rows of a few values, and beams that are alike: everything ties, places decide."""
    flat = torch.full((2, 3, V), 1.25, dtype=dtype, device=DEV)
    o = run_and_check(flat, torch.full((2, 3), -2.0, device=DEV), N=N, exact_ties=True)
    assert o[2][0].tolist() == list(range(N)) and (o[1][0] == 0).all() and (o[1][1] == 3).all()
    few = torch.randint(0, 3, (2, 1, V), generator=torch.Generator().manual_seed(1)).to(DEV, dtype).expand(2, 3, V).contiguous()
    run_and_check(few, torch.full((2, 3), -2.0, device=DEV), N=N, exact_ties=True)


def test_rising_and_falling_rows():
    """Every element betters all before it (each segment is a new best one), and the other way round."""
    up = torch.arange(20000, device=DEV, dtype=F32) * 1e-3
    for x in (up, up.flip(0)):
        run_and_check(x.view(1, 1, -1).repeat(1, 2, 1), torch.tensor([[-1.0, -1.5]], device=DEV), N=50)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("V,N", [(200_000, 5), (150_001, 128)])
def test_more_equal_segments_than_the_list_holds(dtype, V, N):
    """Thousands of segments tie: they are taken in rounds, as are their elements."""
    flat = torch.full((2, 3, V), -0.75, dtype=dtype, device=DEV)
    o = run_and_check(flat, torch.full((2, 3), -2.0, device=DEV), N=N, exact_ties=True)
    assert o[2][1].tolist() == list(range(N)) and (o[1][1] == 3).all()
    flat[0, 1, V - 9:] = 0.5
    flat[1, 2, 7] = 0.5
    run_and_check(flat, torch.full((2, 3), -2.0, device=DEV), N=N)
    flat[:, 2, V - 3:] = 0.5                                   # (better ones in the last round alone)
    run_and_check(flat, torch.full((2, 3), -2.0, device=DEV), N=N)


def test_long_rising_and_falling_rows():
    """The same with every segment better than all before it, or worse: each round brings better ones, or none."""
    up = torch.arange(400_000, device=DEV, dtype=F32) * 2.0 ** -20
    for x in (up, up.flip(0)):
        for N in (1, 33, 128):
            run_and_check(x.view(1, 1, -1).repeat(1, 2, 1), torch.tensor([[-1.0, -1.125]], device=DEV), N=N)


def test_the_best_ones_in_one_segment_and_in_the_last_element():
    x = normal((2, 2, 5000), seed=3)
    x[:, 1, 1024:1088] += 30
    x[:, 0, 4999] = 60
    run_and_check(x, beams(2, 2), N=40)


def test_masked_logits():
    """-inf and the lowest finite values are masks; beams that keep fewer tokens than asked for; none at all."""
    x = normal((6, 3, 2000), seed=4)
    x[0, :, 10:] = -INF
    x[1, 0] = -INF
    x[2] = -INF
    x[3, :, 5:] = torch.finfo(F32).min
    x[4, 1] = torch.finfo(F32).min
    x[5, :, :1999] = -INF
    o = run_and_check(x, beams(6, 3), N=37)
    assert (o[1][2] == -1).all() and (o[1][1] != 3).all()
    assert (o[1][5][3:] == -1).all() and (o[2][5][:3] == 1999).all()
    assert (o[0][5][:3].sort(descending=True).values == beams(6, 3)[5].sort(descending=True).values).all()   # the one token has all the mass


def test_not_finite_logits_end_their_beam_alone():
    for bad in (math.nan, INF):
        for at in (0, 31, 777, 1999):
            x = normal((2, 3, 2000), seed=5)
            x[0, 1, at] = bad
            o = run_and_check(x, beams(2, 3), N=20)
            assert (o[1][0] != 1).all()
        x = normal((1, 2, 2000), seed=6)
        x[0, 0] = -INF
        x[0, 0, 77] = bad                                      # (a lane that holds nothing else)
        o = run_and_check(x, beams(1, 2), N=5)
        assert (o[1] == 1).all()


def test_scores_that_are_not_finite_are_no_beams():
    s = beams(3, 4)
    s[0, 1:] = -INF
    s[1, 2] = math.nan
    s[1, 3] = INF
    s[2] = -INF
    x = normal((3, 4, 900), seed=8)
    x[0, 1:] = math.nan                                        # never read as candidates
    o = run_and_check(x, s, N=6)
    assert (o[1][0] == 0).all() and (o[1][2] == -1).all()


def test_done_beams_stand_as_they_are():
    x = normal((3, 4, 900), seed=9)
    done = torch.tensor([[0, 1, 0, 0], [1, 1, 1, 1], [0, 0, 1, 1]], dtype=I32, device=DEV)
    s = beams(3, 4)
    s[2, 3] = -INF
    x[0, 1] = math.nan                                         # a done beam's logits are not read
    o = run_and_check(x, s, done, 5, N=6)
    assert o[1][1].tolist()[4:] == [-1, -1] and sorted(o[1][1].tolist()[:4]) == [4, 5, 6, 7]
    assert o[3][1].tolist() == [1, 1, 1, 1, 0, 0] and (o[2][1][:4] == 5).all()
    assert sorted(o[0][1][:4].tolist()) == sorted(s[1].tolist())
    x[2, 0, 5] = 40.0                                          # ends now
    o = run_and_check(x, s, done, 5, N=6)
    assert o[2][2][0] == 5 and o[3][2][0] == 1


def test_far_scores_keep_their_order():
    """Scores of thousands, where fp32 sums would tie: candidates are told apart by logits that differ in their last bits."""
    x = torch.zeros((1, 2, 300), device=DEV)
    x[0, 0, 100:140] = torch.tensor([1.0 + i * 2.0 ** -23 for i in range(40)], device=DEV)
    x[0, 1] = -50.0
    o = run_select(x, torch.tensor([[-40000.0, -90000.0]], device=DEV), N=40)
    assert o[2][0].tolist() == list(range(139, 99, -1)) and (o[1] == 0).all()


def test_large_and_small_logits():
    for scale in (1e4, 1e30, 1e-30):
        run_and_check(normal((2, 2, 3000), seed=10, std=scale), beams(2, 2), N=5)


@pytest.mark.parametrize("std,T", [(100.0, 1e-36), (100.0, 1e-30), (3.0, 1e-3), (3.0, 1e30), (1e30, 1e30)])
def test_temperatures_at_both_ends(std, T):
    """Scaled logits beyond fp32's range, and logits that temperature levels."""
    run_and_check(normal((3, 4, 3000), seed=13, std=std), beams(3, 4), N=7, T=T)
    run_and_check(normal((30, 4, 3000), seed=14, std=std), beams(30, 4), N=7, T=T)


def test_rows_that_lie_far_apart():
    """Offsets that pass 2^31 elements."""
    store = torch.empty(2 ** 31 + 4096, dtype=BF16, device=DEV)
    x = store.as_strided((1, 3, 2000), (3 * 2 ** 30, 2 ** 30, 1))
    x.copy_(normal((1, 3, 2000), BF16, 17))
    run_and_check(x, beams(1, 3), N=6)


@pytest.mark.skipif(torch.cuda.device_count() < 2, reason="needs two visible GPUs")
def test_on_a_device_that_is_not_the_current_one():
    x, s = normal((2, 3, 4000), seed=18), beams(2, 3)
    want = run_select(x, s, N=4)
    o = [torch.zeros((2, 4), device="cuda:1")] + [torch.zeros((2, 4), dtype=I32, device="cuda:1") for _ in range(2)]
    ws = torch.zeros(sps.sps_beam_select_workspace_bytes(2, 3, 4000), dtype=torch.uint8, device="cuda:1")
    sps.sps_beam_select(x.to("cuda:1"), s.to("cuda:1"), *o, ws)
    assert all(torch.equal(a, b.to(DEV)) for a, b in zip(want, o))
    with pytest.raises(ValueError):
        sps.sps_beam_select(x, s, *o, ws)


def test_in_place_scores_and_done():
    B, W, V = 5, 4, 3000
    x, s = normal((B, W, V), seed=11), beams(B, W)
    done = (torch.rand((B, W), generator=torch.Generator().manual_seed(0)) < 0.4).to(I32).to(DEV)
    want = run_select(x, s, done, 3, W)
    ws = torch.zeros(sps.sps_beam_select_workspace_bytes(B, W, V), dtype=torch.uint8, device=DEV)
    p, t = (torch.zeros((B, W), dtype=I32, device=DEV) for _ in range(2))
    sps.sps_beam_select(x, s, s, p, t, ws, done=done, out_done=done, end_token=3)
    assert all(torch.equal(a, b) for a, b in zip(want, (s, p, t, done)))


def test_one_workspace_serves_calls_of_any_shape_and_results_repeat():
    ws = torch.zeros(sps.sps_beam_select_workspace_bytes(16, 8, 32000), dtype=torch.uint8, device=DEV)
    first = {}
    for rep in range(3):
        for B, W, V, dt in ((16, 8, 32000, F32), (1, 4, 32000, F32), (3, 5, 777, BF16), (2, 1, 32000, BF16)):
            x, s = normal((B, W, V), dt, V + B), beams(B, W)
            o = run_select(x, s, N=W, ws=ws)
            if rep == 0:
                check_select(o, x, s, N=W)
                first[(B, W, V)] = o
            assert all(torch.equal(a, b) for a, b in zip(o, first[(B, W, V)]))


def test_one_workspace_serves_few_and_many_sequences_in_turn():
    """Arrivals are counted at the same place whatever the shape: what a call of few sequences leaves is no count of one of many."""
    ws = torch.zeros(sps.sps_beam_select_workspace_bytes(600, 2, 500), dtype=torch.uint8, device=DEV)
    for B, W, V in ((1, 8, 5000), (600, 2, 500), (2, 2, 9000), (600, 2, 500)):
        x, s = normal((B, W, V), seed=B + V), beams(B, W)
        check_select(run_select(x, s, N=3, ws=ws), x, s, N=3)


def test_captured_and_replayed_on_another_stream():
    B, W, V = 3, 4, 32000
    x, s = normal((B, W, V), seed=12), beams(B, W)
    ws = torch.zeros(sps.sps_beam_select_workspace_bytes(B, W, V), dtype=torch.uint8, device=DEV)
    o = [torch.zeros((B, W), device=DEV)] + [torch.zeros((B, W), dtype=I32, device=DEV) for _ in range(3)]
    st, g = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(g, stream=st):
        sps.sps_beam_select(x, s, *o[:3], ws, out_done=o[3], end_token=9)
    for seed in range(4):
        x.copy_(normal((B, W, V), seed=20 + seed))
        s.copy_(beams(B, W, seed))
        g.replay()
        torch.cuda.synchronize()
        check_select(o, x, s, end=9, N=W)


def test_the_binding_refuses_what_it_can_see():
    x, s = normal((2, 3, 50)), beams(2, 3)
    ws = torch.zeros(sps.sps_beam_select_workspace_bytes(2, 3, 50), dtype=torch.uint8, device=DEV)
    o, p, t = torch.zeros((2, 4), device=DEV), torch.zeros((2, 4), dtype=I32, device=DEV), torch.zeros((2, 4), dtype=I32, device=DEV)
    sps.sps_beam_select(x, s, o, p, t, ws)
    for bad in (dict(logits=x.double()), dict(logits=x.transpose(1, 2)), dict(logits=x[:, ::2]), dict(logits=x.half()), dict(scores=s[:, :2]), dict(scores=s.double()),
                dict(out_scores=o[0]), dict(out_parents=p[:, :3]), dict(out_tokens=t.long()), dict(workspace=ws[:-16]), dict(done=p), dict(out_done=t.cpu())):
        kw = dict(logits=x, scores=s, out_scores=o, out_parents=p, out_tokens=t, workspace=ws, end_token=1)
        kw.update(bad)
        with pytest.raises(ValueError):
            sps.sps_beam_select(**kw)
