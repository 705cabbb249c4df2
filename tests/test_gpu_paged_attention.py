"""sps_paged_attention on the GPU against per-row softmax attention in 64 bits."""
import pytest
import torch

import paper_2302_01318_b200 as sps
from paged_util import BF16, DEV, F32, Pages, attention64, attention_tol, check_attention, normal, run_attention, workspace

pytestmark = pytest.mark.gpu

TYPES = [(F32, F32, F32), (F32, BF16, F32), (BF16, BF16, BF16), (BF16, BF16, F32)]   # q, cache, out

# lens, news, Hkv, G, page
SHAPES = [
    ([1], [1], 1, 1, 8),                                     # one token that sees itself
    ([2, 1, 1], [1, 1, 1], 2, 1, 16),
    ([127, 128, 129, 130], [1, 1, 1, 1], 1, 8, 16),          # contexts around a tile's end
    ([64, 63, 65], [5, 5, 5], 2, 3, 32),                     # a group of three heads, 15 rows
    ([0, 3, 0, 200], [0, 2, 0, 4], 1, 4, 8),                 # sequences without rows and without tokens
    ([2, 40, 0], [5, 1, 3], 2, 2, 16),                       # rows at negative positions: they see nothing
    ([700], [1], 1, 1, 64),                                  # one row over a long context: split over CTAs
    ([1500, 3], [2, 3], 1, 5, 128),
    ([257, 511], [33, 17], 2, 6, 512),                       # many rows: several row tiles, groups that do not divide them
    ([150, 1, 90], [150, 1, 1], 1, 4, 16),                   # a prompt beside decode rows
    ([1], [1], 3, 16, 8),
    ([400], [7], 1, 20, 16),                                 # 140 rows of one key head
]


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("types", range(len(TYPES)))
@pytest.mark.parametrize("shape", range(len(SHAPES)))
def test_matches_64_bits(d, types, shape):
    lens, news, Hkv, G, page = SHAPES[shape]
    qdt, cdt, odt = TYPES[types]
    pages = Pages(lens, Hkv, d, page, cdt, seed=shape, order="head" if shape % 2 else "slot")   # every other slot is NaN
    run_attention(pages, news, Hkv * G, qdt, odt, lead=shape % 3, tail=2)


@pytest.mark.parametrize("types", range(3))
@pytest.mark.parametrize("max_q", [1, 64, 100000])
def test_max_q_is_a_hint_only(types, max_q):
    qdt, cdt, odt = TYPES[types]
    pages = Pages([300, 40], 2, 128, 16, cdt)
    run_attention(pages, [70, 1], 8, qdt, odt, max_q=max_q)


@pytest.mark.parametrize("types", range(3))
@pytest.mark.parametrize("d", [64, 128])
def test_one_workspace_serves_every_batch_in_turn(types, d):
    """Counters and parts left by one call do not reach the next, whatever its shape; the same call twice gives the same bits."""
    qdt, cdt, odt = TYPES[types]
    pools = [Pages(lens, 2, d, 16, cdt, seed=i) for i, lens in enumerate(([2000], [5, 900, 31], [64] * 20, [1]))]
    ws = workspace(pools[0].cache, 8, qdt)
    news = ([3], [2, 1, 9], [1] * 20, [1])
    for turn in range(2):
        for p, n in zip(pools, news):
            a = run_attention(p, n, 8, qdt, odt, ws=ws)
            b = run_attention(p, n, 8, qdt, odt, ws=ws)
            assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


@pytest.mark.parametrize("types", range(3))
def test_large_scores_small_scores_and_given_scale(types):
    qdt, cdt, odt = TYPES[types]
    pages = Pages([600, 90], 1, 64, 32, cdt)
    run_attention(pages, [4, 30], 4, qdt, odt, std=40.0)       # one token takes nearly all the weight
    run_attention(pages, [4, 30], 4, qdt, odt, std=1e-3)       # every token the same weight
    run_attention(pages, [4, 30], 4, qdt, odt, scale=0.7)
    run_attention(pages, [4, 30], 4, qdt, odt, scale=-0.25)


@pytest.mark.parametrize("types", range(3))
@pytest.mark.parametrize("rising", [False, True])
def test_scores_that_rise_and_fall_along_the_context(types, rising):
    """Maxima that keep moving: a key's score grows (or falls) by far more than a rescaling step from tile to tile."""
    qdt, cdt, odt = TYPES[types]
    pages = Pages([1000], 1, 64, 16, cdt)
    k, v = pages.dense[0]
    ramp = torch.linspace(0, 1, 1000, device=DEV)
    if not rising:
        ramp = ramp.flip(0)
    k.copy_((ramp[:, None, None] * torch.ones_like(k).float() * 6).to(cdt))
    j = torch.arange(1000)
    pages.k[pages.table[0, j // 16].long().to(DEV), :, (j % 16).to(DEV)] = k
    q = torch.ones((5, 4, 64), device=DEV).mul_(torch.tensor([1., 3., 0.2, -2.], device=DEV)[None, :, None]).to(qdt)
    run_attention(pages, [5], 4, qdt, odt, q=q)


@pytest.mark.parametrize("types", range(3))
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
def test_what_a_row_does_not_see_never_reaches_it(types, bad):
    """The last of the new tokens has a bad key and value: the rows before it are exact, its own is not finite."""
    qdt, cdt, odt = TYPES[types]
    pages = Pages([205, 70], 1, 64, 8, cdt, fill=bad)
    news = [9, 3]
    clean = [(k.clone(), v.clone()) for k, v in pages.dense]
    pg, sl = int(pages.table[0, 204 // 8]), 204 % 8
    pages.v[pg, 0, sl, 5] = bad
    q = normal((12, 2, 64), qdt, 1)
    out, ws = torch.empty((12, 2, 64), dtype=odt, device=DEV), workspace(pages.cache, 2, qdt)
    for key in (False, True):
        if key:
            pages.k[pg, 0, sl, 7] = bad
        sps.sps_paged_attention(pages.cache, pages.batch(news), q, out, ws)
        torch.cuda.synchronize()
        keep = [r for r in range(12) if r != 8]
        assert not torch.isfinite(out[8].float()).all() or (key and bad == float("-inf"))
        want, _, S = attention64(q, clean, news)

        tol = attention_tol(want, S, 64, qdt, odt)
        assert ((out.double() - want).abs() <= tol)[keep].all()


@pytest.mark.parametrize("types", range(3))
@pytest.mark.parametrize("new", [2, 150])
def test_an_infinite_value_stays_in_its_element(types, new):
    """Of an older token: every row sees it, and every other element is what it is without it."""
    qdt, cdt, odt = TYPES[types]
    pages = Pages([600], 1, 64, 16, cdt)
    q = normal((new, 2, 64), qdt, 1)
    ws, batch = workspace(pages.cache, 2, qdt), pages.batch([new])
    out, clean = (torch.empty((new, 2, 64), dtype=odt, device=DEV) for _ in range(2))
    sps.sps_paged_attention(pages.cache, batch, q, clean, ws)
    pages.v[int(pages.table[0, 5]), 0, 3, 21] = float("inf")    # token 83
    sps.sps_paged_attention(pages.cache, batch, q, out, ws)
    others = [e for e in range(64) if e != 21]
    assert not torch.isfinite(out[..., 21].float()).any()
    assert torch.equal(out[..., others], clean[..., others]) and torch.isfinite(out[..., others].float()).all()


@pytest.mark.parametrize("types", range(3))
@pytest.mark.parametrize("B,max_q", [(33, 2), (150, 64), (1100, 2)])
def test_batches_of_many_sequences(types, B, max_q):
    """More than a warp reads at once, and more than 32 blocks of 32: ragged lengths, sequences without rows or tokens among
    them; then one whose length does not fit the table."""
    qdt, cdt, odt = TYPES[types]
    g = torch.Generator().manual_seed(B)
    lens = torch.randint(0, 40, (B,), generator=g).tolist()
    lens[B // 2] = 1000                                          # cut between CTAs
    news = [min(n, L + 1) for n, L in zip(torch.randint(0, 3, (B,), generator=g).tolist(), lens)]
    pages = Pages(lens, 1, 64, 16, cdt)
    out, lse, _, ws = run_attention(pages, news, 4, qdt, odt, max_q=max_q, lead=1, tail=1)
    batch = pages.batch(news, 1, max_q)
    last = max(b for b in range(B) if news[b])
    batch.kv_len[last] = 10 ** 6
    rows = out.shape[0]
    q, again = normal((rows, 4, 64), qdt, 5, 1.5), out.clone()   # run_attention's queries
    sps.sps_paged_attention(pages.cache, batch, q, again, ws)
    assert int(batch.status) & sps.PAGED_BAD_LENGTH
    end = 1 + sum(news[:last])
    want, _, S = attention64(q, pages.dense, news, 1)
    assert ((again.double() - want).abs() <= attention_tol(want, S, 64, qdt, odt))[1:end].all()


@pytest.mark.parametrize("types", range(3))
def test_sequences_that_share_a_prefix(types):
    """Two sequences whose tables begin with the same pages, each with a last page of its own."""
    qdt, cdt, odt = TYPES[types]
    pages = Pages([160, 150], 2, 128, 16, cdt)
    pages.table[1, :8] = pages.table[0, :8]
    for own, other in zip(pages.dense[1], pages.dense[0]):
        own[:128] = other[:128]
    run_attention(pages, [5, 3], 8, qdt, odt)


@pytest.mark.parametrize("types", range(3))
def test_bad_pages_and_lengths_are_flagged_and_harm_no_other_sequence(types):
    qdt, cdt, odt = TYPES[types]
    pages = Pages([100, 300, 50], 2, 64, 16, cdt)
    batch = pages.batch([2, 2, 2])
    batch.pages[0, 3] = pages.n_pages
    batch.pages[2, 1] = -5
    q, ws = normal((6, 4, 64), qdt, 1), workspace(pages.cache, 4, qdt)
    out = torch.empty((6, 4, 64), dtype=odt, device=DEV)
    sps.sps_paged_attention(pages.cache, batch, q, out, ws)
    assert int(batch.status) == sps.PAGED_BAD_PAGE
    assert torch.isfinite(out.float()).all()
    check_attention(out[2:4], None, q[2:4], pages.dense[1:2], [2])
    # a bad page's tokens read as zeros: score 0, value 0
    zeroed = [(k.clone(), v.clone()) for k, v in pages.dense]
    zeroed[0][0][48:64], zeroed[0][1][48:64] = 0, 0
    zeroed[2][0][16:32], zeroed[2][1][16:32] = 0, 0
    check_attention(out, None, q, zeroed, [2, 2, 2])
    batch2 = pages.batch([2, 2, 2])
    batch2.kv_len[1] = 10 ** 6
    sps.sps_paged_attention(pages.cache, batch2, q, out, ws)
    assert int(batch2.status) & sps.PAGED_BAD_LENGTH
    check_attention(out[:2], None, q[:2], pages.dense[:1], [2])
    check_attention(out[4:], None, q[4:], pages.dense[2:], [2])
    # row numbers outside the buffers and out of order are cut, not followed
    batch3 = pages.batch([2, 2, 2])
    batch3.q_start.copy_(torch.tensor([-7, 2, 1, 5000], dtype=torch.int32))
    sps.sps_paged_attention(pages.cache, batch3, q, out, ws)
    torch.cuda.synchronize()


@pytest.mark.parametrize("types", range(3))
def test_strides_and_unaligned_rows(types):
    qdt, cdt, odt = TYPES[types]
    pages = Pages([77, 140], 2, 64, 8, cdt)
    news, rows, H = [3, 20], 23, 4
    big = normal((rows, H + 2, 67), qdt, 3)
    for q in (big[:, 1:1 + H, :64], big[:, 1:1 + H, 3:67], normal((H, rows, 64), qdt, 4).transpose(0, 1)):
        ob = torch.full((rows, H + 1, 69), 7.0, dtype=odt, device=DEV)
        out = ob[:, 1:, 5:]
        sps.sps_paged_attention(pages.cache, pages.batch(news), q, out, workspace(pages.cache, H, qdt))
        check_attention(out, None, q, pages.dense, news)
        assert (ob[:, 0] == 7).all() and (ob[..., :5] == 7).all()


@pytest.mark.parametrize("types", range(3))
def test_replayed_in_a_graph_with_moved_lengths(types):
    qdt, cdt, odt = TYPES[types]
    pages = Pages([900, 333], 1, 128, 16, cdt)
    q, ws = normal((4, 4, 128), qdt, 1), workspace(pages.cache, 4, qdt)
    out = torch.zeros((4, 4, 128), dtype=odt, device=DEV)
    batch = pages.batch([2, 2])
    sps.sps_paged_attention(pages.cache, batch, q, out, ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        sps.sps_paged_attention(pages.cache, batch, q, out, ws)
    for lens, starts in (([900, 333], [0, 2, 4]), ([2, 300], [0, 1, 4]), ([513, 129], [0, 4, 4]), ([1, 0], [0, 1, 1])):
        batch.kv_len.copy_(torch.tensor(lens, dtype=torch.int32))
        batch.q_start.copy_(torch.tensor(starts, dtype=torch.int32))
        q.copy_(normal((4, 4, 128), qdt, lens[0]))
        out.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        check_attention(out, None, q, [(k[:L], v[:L]) for (k, v), L in zip(pages.dense, lens)], [b - a for a, b in zip(starts, starts[1:])])
    assert int(batch.status) == 0


def test_two_streams_with_two_workspaces():
    pages = [Pages([1500, 20], 2, 128, 16, BF16, seed=s) for s in (0, 1)]
    qs = [normal((3, 8, 128), F32, s) for s in (0, 1)]
    outs = [torch.zeros_like(q) for q in qs]
    wss = [workspace(p.cache, 8, F32) for p in pages]
    batches = [p.batch([2, 1]) for p in pages]
    streams = [torch.cuda.Stream() for _ in pages]
    torch.cuda.synchronize()
    for _ in range(20):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                sps.sps_paged_attention(pages[i].cache, batches[i], qs[i], outs[i], wss[i])
    torch.cuda.synchronize()
    for i in range(2):
        check_attention(outs[i], None, qs[i], pages[i].dense, [2, 1])


@pytest.mark.parametrize("types", range(3))
def test_offsets_past_32_bits(types):
    """The pool holds more than 2^31 elements; the sequences' pages lie at both of its ends."""
    qdt, cdt, odt = TYPES[types]
    n_pages, page, d = (2 ** 31 + 2 ** 20) // (64 * 128), 64, 128
    k = torch.empty((n_pages, 1, page, d), dtype=cdt, device=DEV)
    v = torch.empty((n_pages, 1, page, d), dtype=cdt, device=DEV)
    lens = [200, 130]
    ids = [n_pages - 1, 0, n_pages - 2, 5, 3, n_pages - 3, 1]
    table = torch.tensor([ids[:4], ids[4:] + [0]], dtype=torch.int32)
    dense = []
    for b, L in enumerate(lens):
        kk, vv = normal((L, 1, d), cdt, b), normal((L, 1, d), cdt, b + 9)
        j = torch.arange(L)
        p, s = table[b, j // page].long().to(DEV), (j % page).to(DEV)
        k[p, :, s], v[p, :, s] = kk, vv
        dense.append((kk, vv))
    cache = sps.PagedCache(k, v)
    news = [3, 2]
    batch = sps.PagedBatch(torch.tensor([0, 3, 5], dtype=torch.int32, device=DEV), torch.tensor(lens, dtype=torch.int32, device=DEV), table.to(DEV), max_q=3)
    kn, vn = torch.cat([dense[0][0][-3:], dense[1][0][-2:]]), torch.cat([dense[0][1][-3:], dense[1][1][-2:]])
    for b, n in ((0, 3), (1, 2)):
        for i in range(n):
            at = lens[b] - n + i
            k[int(table[b, at // page]), :, at % page] = 0
    sps.sps_paged_append(cache, batch, kn.contiguous(), vn.contiguous())
    q = normal((5, 4, d), qdt, 3)
    out = torch.empty((5, 4, d), dtype=odt, device=DEV)
    sps.sps_paged_attention(cache, batch, q, out, workspace(cache, 4, qdt))
    check_attention(out, None, q, dense, news)
    del k, v, cache
    torch.cuda.empty_cache()


def test_a_large_batch_and_a_long_context_against_sums_over_chunks():
    """Many sequences of one token each, and one context of 70 000 tokens: every element against 64 bits, per head."""
    pages = Pages([1 + 7 * i for i in range(150)], 1, 64, 16, BF16)
    run_attention(pages, [1] * 150, 2, BF16)
    L = 70000
    pages = Pages([L], 1, 128, 64, BF16)
    run_attention(pages, [2], 2, F32)


@pytest.mark.parametrize("types", range(3))
@pytest.mark.parametrize("new", [1, 40])
def test_in_place(types, new):
    qdt, cdt, odt = TYPES[types]
    pages = Pages([700, 90], 2, 64, 16, cdt)
    q = normal((2 * new, 8, 64), qdt, 1)
    buf = q.clone()
    sps.sps_paged_attention(pages.cache, pages.batch([new, new]), buf, buf, workspace(pages.cache, 8, qdt))
    check_attention(buf, None, q, pages.dense, [new, new])


@pytest.mark.parametrize("types", range(3))
@pytest.mark.parametrize("order", [(0, 1, 2), (0, 2, 1), (1, 0, 2), (1, 2, 0), (2, 0, 1), (2, 1, 0)])
def test_pools_of_any_order(types, order):
    """Pages, heads and slots in any order of strides, with gaps: the pool is a view of a larger tensor."""
    qdt, cdt, odt = TYPES[types]
    src = Pages([100, 37], 3, 64, 8, cdt)
    size = [src.k.shape[i] for i in order]
    back = [order.index(i) for i in range(3)] + [3]
    pools = []
    for t in (src.k, src.v):
        big = torch.full([s + 1 for s in size] + [72], float("nan"), dtype=cdt, device=DEV)
        view = big[:size[0], :size[1], :size[2], :64]
        view.copy_(t.permute(*order, 3))
        pools.append(view.permute(*back))
    cache = sps.PagedCache(*pools)
    news = [5, 2]
    q = normal((7, 6, 64), qdt, 2)
    out = torch.empty((7, 6, 64), dtype=odt, device=DEV)
    sps.sps_paged_attention(cache, src.batch(news), q, out, workspace(cache, 6, qdt))
    check_attention(out, None, q, src.dense, news)


@pytest.mark.parametrize("qdt,new,lens", [(F32, 2, [60000, 90]), (BF16, 2, [60000, 90]), (F32, 6, [30000, 90]), (BF16, 100, [6000, 300])])
@pytest.mark.parametrize("stage", [0, 1, 2])
def test_a_wait_that_runs_out_ends_the_call_with_a_status(qdt, new, lens, stage):
    """The first CTA's copies leave out one half-tile (keys of its first tile, values of it, keys of the next): the call gives
    up within the bound, says so, and the next one on a fresh workspace is right."""
    pages = Pages(lens, 2, 128, 16, BF16)
    news = [new, new]
    q = normal((2 * new, 16, 128), qdt, 1)
    out, ws, batch = torch.empty_like(q), workspace(pages.cache, 16, qdt), pages.batch(news)
    try:
        sps.sps_debug_set_wait(20000, stage)
        sps.sps_paged_attention(pages.cache, batch, q, out, ws)
        torch.cuda.synchronize()
    finally:
        sps.sps_debug_set_wait()
    assert int(batch.status) == sps.PAGED_TIMEOUT
    batch.status.zero_()
    ws.zero_()
    sps.sps_paged_attention(pages.cache, batch, q, out, ws)
    torch.cuda.synchronize()
    assert int(batch.status) == 0
    check_attention(out, None, q, pages.dense, news)


@pytest.mark.parametrize("qdt,new,lens", [(F32, 2, [60000, 90]), (BF16, 2, [60000, 90]), (BF16, 100, [6000, 300])])
@pytest.mark.parametrize("watched", [True, False])
def test_a_call_that_gave_up_is_seen_without_its_status(qdt, new, lens, watched):
    """Whether or not the caller passes a status: what the call did not finish is NaN, and so is everything of the next calls on
    the same workspace, whose arrival counters are part-way, until it is zeroed."""
    pages = Pages(lens, 2, 128, 16, BF16)
    news, rows = [new, new], 2 * new + 3
    q = normal((rows, 16, 128), qdt, 1)
    ws, batch = workspace(pages.cache, 16, qdt), pages.batch(news, lead=1)
    status = batch.status
    if not watched:
        batch._c.status = None
    want, _, S = attention64(q, pages.dense, news, 1)
    tol = attention_tol(want, S, 128, qdt, qdt)
    inside = slice(1, 1 + 2 * new)

    def call(cache=pages.cache, over=batch, x=q):
        out, lse = torch.full_like(x, 7.0), torch.full((rows, 16), 7.0, device=DEV)
        sps.sps_paged_attention(cache, over, x, out, ws, lse=lse)
        torch.cuda.synchronize()
        for t in (out, lse):
            assert (t[:1] == 7).all() and (t[1 + 2 * new:] == 7).all()
        return out[inside], lse[inside]

    try:
        sps.sps_debug_set_wait(20000, 1)
        out, _ = call()
    finally:
        sps.sps_debug_set_wait()
    lost = torch.isnan(out.float())
    assert lost.any() and ((out.double() - want[inside]).abs() <= tol[inside])[~lost].all()
    for _ in range(2):
        status.zero_()
        out, lse = call()
        assert torch.isnan(out.float()).all() and torch.isnan(lse).all()
        assert int(status) == (sps.PAGED_TIMEOUT if watched else 0)
    # the kernels over an fp32 cache read the same counters
    other = Pages([70, 20], 2, 64, 16, F32)
    x = normal((rows, 16, 64), F32, 2)
    if ws.nbytes >= workspace(other.cache, 16, F32).nbytes and new < 20:
        small = other.batch(news, lead=1)
        out, lse = call(other.cache, small, x)
        assert torch.isnan(out).all() and torch.isnan(lse).all() and int(small.status) == sps.PAGED_TIMEOUT
    ws.zero_()
    status.zero_()
    out, _ = call()
    assert int(status) == 0 and ((out.double() - want[inside]).abs() <= tol[inside]).all()


def test_a_workspace_that_repeats_its_bytes_is_refused():
    """An expanded tensor claims more bytes than it has."""
    pages = Pages([20], 1, 64, 8, F32)
    q = normal((1, 2, 64), F32, 1)
    n = workspace(pages.cache, 2, F32).nbytes
    for ws in (torch.zeros((1, 16), dtype=torch.uint8, device=DEV).expand(n // 16 + 1, 16), torch.zeros((n, 2), dtype=torch.uint8, device=DEV)[:, 0],
               torch.zeros(n - 1, dtype=torch.uint8, device=DEV)):
        with pytest.raises(ValueError, match="workspace"):
            sps.sps_paged_attention(pages.cache, pages.batch([1]), q, torch.empty_like(q), ws)


@pytest.mark.parametrize("types", range(len(TYPES)))
@pytest.mark.parametrize("d", [64, 128])
def test_many_rows_with_strides_and_unaligned_rows(types, d):
    """More than 64 rows of a key head, of short sequences (items in one piece) and a long one (cut between CTAs and joined)."""
    qdt, cdt, odt = TYPES[types]
    pages = Pages([77, 6000, 150], 2, d, 8, cdt)
    news, rows, H = [3, 150, 90], 243, 4
    big = normal((rows, H + 2, d + 3), qdt, 3)
    for q in (big[:, 1:1 + H, :d], big[:, 1:1 + H, 3:], normal((H, rows, d), qdt, 4).transpose(0, 1)):
        for shift in (5, 8):                                     # outputs element by element, and whole pieces
            ob = torch.full((rows, H + 1, d + 8), 7.0, dtype=odt, device=DEV)
            out = ob[:, 1:, shift:shift + d]
            lse = torch.full((rows, H), 7.0, device=DEV)
            sps.sps_paged_attention(pages.cache, pages.batch(news), q, out, workspace(pages.cache, H, qdt), lse=lse)
            check_attention(out, lse, q, pages.dense, news)
            assert (ob[:, 0] == 7).all() and (ob[..., :shift] == 7).all() and (ob[..., shift + d:] == 7).all()


@pytest.mark.parametrize("types", range(len(TYPES)))
def test_many_rows_replayed_in_a_graph_with_moved_lengths(types):
    """Attention and the join of its parts, captured together; two captured calls that take turns on one workspace."""
    qdt, cdt, odt = TYPES[types]
    pages = Pages([5000, 333], 1, 128, 16, cdt)
    rows = 200
    q, ws = normal((rows, 4, 128), qdt, 1), workspace(pages.cache, 4, qdt)
    out, second = (torch.zeros((rows, 4, 128), dtype=odt, device=DEV) for _ in range(2))
    batch, other = pages.batch([150, 50]), pages.batch([1, 1], max_q=1)
    sps.sps_paged_attention(pages.cache, batch, q, out, ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        sps.sps_paged_attention(pages.cache, batch, q, out, ws)
        sps.sps_paged_attention(pages.cache, other, q, second, ws)
    for lens, starts in (([5000, 333], [0, 150, 200]), ([200, 300], [0, 1, 200]), ([4000, 129], [0, 71, 200]), ([170, 0], [0, 170, 170]), ([1, 333], [0, 1, 140])):
        batch.kv_len.copy_(torch.tensor(lens, dtype=torch.int32))
        batch.q_start.copy_(torch.tensor(starts, dtype=torch.int32))
        q.copy_(normal((rows, 4, 128), qdt, lens[0]))
        out.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        check_attention(out, None, q, [(k[:L], v[:L]) for (k, v), L in zip(pages.dense, lens)], [b - a for a, b in zip(starts, starts[1:])])
        check_attention(second[:2], None, q[:2], pages.dense, [1, 1])
    assert int(batch.status) == 0 and int(other.status) == 0


@pytest.mark.parametrize("types", range(3))
@pytest.mark.parametrize("news,lead", [([4, 3, 9], 0), ([4, 3, 90], -2), ([40, 3, 7], -5)])
def test_rows_outside_the_buffers_are_skipped_and_move_no_other(types, news, lead):
    """A call on the first rows only, row numbers before and behind them: a row's position goes by its sequence's rows, there or
    not, and what it sees with it."""
    qdt, cdt, odt = TYPES[types]
    lens = [300, 40, 260]
    pages = Pages(lens, 2, 64, 16, cdt)
    total = lead + sum(news)
    q, ws = normal((total, 8, 64), qdt, 1), workspace(pages.cache, 8, qdt)
    want, _, S = attention64(torch.cat([q[:1].expand(-lead, -1, -1), q]), pages.dense, news)
    tol = attention_tol(want, S, 64, qdt, odt)
    batch = pages.batch(news, lead=lead)
    for rows in (total, total - 2, total - news[2], total - news[2] - 1, 1):
        out, lse = torch.full((rows, 8, 64), 7.0, dtype=odt, device=DEV), torch.empty((rows, 8), device=DEV)
        sps.sps_paged_attention(pages.cache, batch, q[:rows], out, ws, lse=lse)
        assert ((out.double() - want[-lead:][:rows]).abs() <= tol[-lead:][:rows]).all()
