"""Fork, reserve, compact and copy of a paged cache's pages against plain lists: long random histories, and the cases where
each can go wrong."""
import random

import pytest
import torch

import paper_2302_01318_b200 as sps
from pages_util import BF16, DEV, F32, I32, Device, Model, consistent, ints

pytestmark = pytest.mark.gpu


def grown(n_pages, page, lens, ld=None, seed=0):
    """A model and its device twin with private pages for rows of the given lengths, page numbers scattered."""
    m = Model(n_pages, page, len(lens))
    perm = list(range(n_pages))
    random.Random(seed).shuffle(perm)
    for i, n in enumerate(lens):
        for _ in range(-(-n // page)):
            p = perm.pop()
            m.refs[p] = 1
            m.rows[i].append(p)
    m.lens = list(lens)
    d = Device(n_pages, page, len(lens), ld or max([len(r) for r in m.rows] + [0]) + 3)
    d.load(m)
    return m, d


# --------------------------------------------------------------------------------------------------------------- history
@pytest.mark.parametrize("n_pages,page,B,top", [(24, 8, 3, 60), (200, 8, 16, 90), (64, 16, 33, 40), (5000, 32, 40, 1500), (40000, 16, 130, 900)])
def test_a_random_history(n_pages, page, B, top):
    """Beams come and go, grow, roll back and run out of pages; pools of one tile and of several CTAs."""
    rng = random.Random(n_pages)
    m, d = Model(n_pages, page, B), Device(n_pages, page, B, top // page + 2)
    d.load(m)
    status = 0
    for _ in range(25):
        kind = rng.random()
        if kind < 0.35:
            parents = [rng.choice([-1] + list(range(B)) * 2) if rng.random() < 0.4 else i for i in range(B)]
            m.fork(parents)
            d.fork(parents)
        elif kind < 0.45:
            moves = m.compact(n_pages // 2 + 1)
            d.compact()
            assert d.listed() == moves
        else:
            for i in range(B):                               # what was reserved is filled, wholly or in part
                m.lens[i] = rng.randint(0, min(len(m.rows[i]) * page, top)) if rng.random() < 0.2 else min(len(m.rows[i]) * page, m.lens[i] + rng.randint(0, 9))
            d.t.lens.copy_(ints(m.lens))
            want = [rng.choice([0, 0, rng.randint(0, top)]) if rng.random() < 0.1 else min(top, n + rng.choice([0, 1, 1, 5, 40])) for n in m.lens]
            moves, short = m.reserve(want)
            status |= sps.PAGED_NO_PAGE if short else 0
            d.reserve(want)
            assert d.listed() == moves
        d.check(m, status)
        consistent(m)


# ------------------------------------------------------------------------------------------------------------------ fork
@pytest.mark.parametrize("B,Bd,ld", [(1, 1, 1), (1, 8, 5), (8, 1, 5), (7, 300, 130), (300, 7, 130), (2, 3, 2048), (3, 2, 5001), (8192, 8192, 3)])
def test_fork_shapes(B, Bd, ld):
    g = torch.Generator().manual_seed(B + Bd + ld)
    n_pages = 4 * B + ld
    held = torch.randint(0, ld + 1, (B,), generator=g).to(I32)
    held[0] = ld
    pages = torch.randint(0, n_pages, (B, ld), generator=g).to(I32)      # (rows share pages at random)
    inside = torch.arange(ld)[None] < held[:, None]
    refs = torch.zeros(n_pages, dtype=I32).index_add_(0, pages[inside].long(), torch.ones(int(inside.sum()), dtype=I32))
    pages[~inside] = 2 ** 31 - 1
    lens = torch.randint(0, 1000, (B,), generator=g).to(I32)
    parents = torch.randint(-1, B, (Bd,), generator=g).to(I32)
    src = sps.PageTable(pages.to(DEV), held.to(DEV), lens.to(DEV))
    dst = Device.table(Bd, ld + 2)
    pool = sps.PagePool(refs.to(DEV), 16)
    sps.sps_paged_fork(pool, src, dst, parents.to(DEV))
    want = torch.full((Bd, ld + 2), -9, dtype=I32)
    p = parents.long().clamp(min=0)
    wh = torch.where(parents >= 0, held[p], 0)
    there = torch.arange(ld)[None] < wh[:, None]
    want[:, :ld] = torch.where(there, pages[p], want[:, :ld])
    wr = torch.zeros(n_pages, dtype=I32).index_add_(0, want[:, :ld][there].long(), torch.ones(int(there.sum()), dtype=I32))
    assert torch.equal(dst.pages.cpu(), want) and torch.equal(dst.held.cpu(), wh) and torch.equal(dst.lens.cpu(), torch.where(parents >= 0, lens[p], 0))
    assert torch.equal(pool.refs.cpu(), wr) and int(pool.status) == 0
    assert torch.equal(src.pages.cpu(), pages) and torch.equal(src.held.cpu(), held)


def test_fork_of_nothing_and_into_nothing():
    m, d = grown(20, 8, [30, 9])
    empty = Device.table(0, d.ld)
    sps.sps_paged_fork(d.pool, d.t, empty, ints([]))
    assert not d.pool.refs.any()
    dst = Device.table(2, 4)
    sps.sps_paged_fork(d.pool, Device.table(0, 4), dst, ints([0, -1]))
    assert dst.held.tolist() == [0, 0] and int(d.pool.status) == sps.PAGED_BAD_ROW


@pytest.mark.parametrize("n_pages", [12, 30000])
def test_tables_without_rows(n_pages):
    d = Device(n_pages, 8, 0, 4, capacity=3)
    d.moves.count.fill_(9)
    d.reserve([])
    assert int(d.moves.count) == 0 and not d.pool.refs.any() and int(d.pool.status) == 0
    d = Device(n_pages, 8, 3, 0)
    d.reserve([0, 0, 0])
    assert int(d.pool.status) == 0
    d.reserve([0, 1, 0])                                       # rows without entries have room for nothing
    assert int(d.pool.status) == sps.PAGED_BAD_LENGTH and d.t.held.tolist() == [0, 0, 0]


@pytest.mark.parametrize("n_pages", [60, 30000])
def test_want_may_be_the_lengths_themselves(n_pages):
    """What was reserved ahead is given up: the lengths are both kept and wanted."""
    m, d = grown(n_pages, 8, [60, 41, 7, 0], ld=16)
    m.reserve([90, 41, 50, 3])
    d.reserve([90, 41, 50, 3])
    m.reserve([60, 41, 7, 0])
    sps.sps_paged_reserve(d.pool, d.t, d.t.lens, d.moves, d.ws, room=d.room)
    d.check(m)


@pytest.mark.skipif(torch.cuda.device_count() < 2, reason="needs two visible GPUs")
def test_on_a_device_that_is_not_the_current_one():
    m, d = grown(64, 8, [21, 13], ld=9)
    to = lambda t: t.to("cuda:1")
    pool = sps.PagePool(to(d.pool.refs), 8)
    tables = [sps.PageTable(to(t.pages), to(t.held), to(t.lens)) for t in d.tables]
    moves, ws = sps.PageMoves(to(d.moves.list), to(d.moves.count)), to(d.ws)
    sps.sps_paged_fork(pool, tables[0], tables[1], to(ints([1, 1])))
    sps.sps_paged_reserve(pool, tables[1], to(ints([14, 20])), moves, ws)
    m.fork([1, 1])
    want, _ = m.reserve([14, 20])
    assert moves.list[:int(moves.count)].tolist() == want and pool.refs.tolist() == m.refs
    with pytest.raises(ValueError):
        sps.sps_paged_fork(d.pool, tables[0], d.tables[1], ints([1, 1]))


def test_two_pools_at_once_on_streams_of_their_own():
    ms = [grown(n, 8, [60, 41, 7, 0], ld=16, seed=n) for n in (200, 40000)]
    streams = [torch.cuda.Stream() for _ in ms]
    wants = [ints([w + 3 * i for w in (60, 41, 7, 1)]) for i in range(8)]
    parents = ints([0, 1, 1, 2])
    torch.cuda.synchronize()
    for want in wants:
        for (m, d), st in zip(ms, streams):
            sps.sps_paged_reserve(d.pool, d.t, want, d.moves, d.ws, stream=st.cuda_stream)
            sps.sps_paged_fork(d.pool, d.t, d.tables[1 - d.at], parents, stream=st.cuda_stream)
            d.at = 1 - d.at
    torch.cuda.synchronize()
    for m, d in ms:
        for want in wants:
            m.reserve(want.tolist())
            m.fork([0, 1, 1, 2])
        d.check(m)


def test_fork_skips_what_does_not_fit():
    m, d = grown(20, 8, [30, 9, 17])
    d.t.pages[0, 1] = 20
    d.t.pages[2, 0] = -1
    refs = d.pool.refs.tolist()
    lost = m.rows[0][1], m.rows[2][0]
    d.fork([0, 0, 7])
    want = [r + (1 if p in m.rows[0] else -1 if p in m.rows[1] + m.rows[2] else 0) for p, r in enumerate(refs)]
    for p in lost:
        want[p] = 1                                            # (its entry no longer names it)
    assert d.pool.refs.tolist() == want and int(d.pool.status) == sps.PAGED_BAD_PAGE | sps.PAGED_BAD_ROW
    assert d.t.held.tolist() == [4, 4, 0] and d.t.pages[1, 1] == 20
    m, d = grown(20, 8, [30, 9])
    d.t.held[0], d.t.held[1] = d.ld + 5, -3
    d.t.pages[0] = ints(m.rows[0][:1] * d.ld)
    d.fork([0, 1])
    assert d.t.held.tolist() == [d.ld, 0] and int(d.pool.status) == sps.PAGED_BAD_LENGTH


# --------------------------------------------------------------------------------------------------------------- reserve
def test_the_first_of_all_who_write_keeps_the_page_and_readers_leave_it():
    for writers, keeps in (([0, 1, 2], 0), ([1, 2], None), ([2], None), ([], None)):
        m, d = grown(40, 8, [21, 0, 0])
        m.fork([0, 0, 0])
        d.fork([0, 0, 0])
        want = [22 if i in writers else 21 for i in range(3)]
        moves, short = m.reserve(want)
        d.reserve(want)
        assert not short and d.listed() == moves and len(moves) == len(writers) - (keeps is not None)
        assert all(n == 5 for _, _, n in moves)
        d.check(m)
        consistent(m)


@pytest.mark.parametrize("length", [0, 1, 7, 8, 9, 16])
def test_room_at_page_borders(length):
    """Nothing is exchanged at a border, whoever shares the page before it."""
    for want in (0, 1, 7, 8, 9, 15, 16, 17, 24, 25):
        m, d = grown(30, 8, [length, 0], ld=5)
        m.fork([0, 0])
        d.fork([0, 0])
        moves, short = m.reserve([want, length])
        d.reserve([want, length])
        assert d.listed() == moves and not short
        d.check(m)


def test_what_is_given_up_is_there_for_others_in_the_same_call():
    m, d = grown(10, 8, [40, 40], ld=10)                       # the pool is full
    for want in ([0, 80], [40, 40], [80, 0], [1, 72]):
        m.lens = [len(r) * 8 for r in m.rows]
        d.t.lens.copy_(ints(m.lens))
        moves, short = m.reserve(want)
        d.reserve(want)
        d.check(m)
        assert not short


def test_a_row_without_pages_keeps_its_tokens_and_stops_those_behind_it():
    m, d = grown(12, 8, [13, 13, 13, 13], ld=8)
    m.fork([0, 1, 2, 3])
    d.fork([0, 1, 2, 3])
    want = [17, 60, 13, 14]                                    # 4 free: row 0 gets one, row 1 asks for 6, row 3 for none
    moves, short = m.reserve(want)
    d.reserve(want)
    assert short
    d.check(m, sps.PAGED_NO_PAGE)
    want = [17, 13, 33, 41]                                    # 3 free: row 2 takes them, row 3 goes without
    moves, short = m.reserve(want)
    d.reserve(want)
    assert short and len(m.rows[2]) == 5 and len(m.rows[3]) == 2
    d.check(m, sps.PAGED_NO_PAGE)


def test_a_row_left_without_its_copy_still_shares():
    m, d = grown(2, 8, [12, 0], ld=4)
    m.fork([0, 0])
    d.fork([0, 0])
    moves, short = m.reserve([13, 13])                         # row 0 may keep the page, row 1's copy has no room
    d.reserve([13, 13])
    assert short and moves == [] and d.listed() == []
    d.check(m, sps.PAGED_NO_PAGE)
    assert m.rows[0] == m.rows[1] and d.room.tolist() == [13, 12]
    want = ints([13, 13])
    sps.sps_paged_reserve(d.pool, d.t, want, d.moves, d.ws, room=want)   # (room may be want)
    assert want.tolist() == [13, 12]


@pytest.mark.parametrize("B,n_pages", [(1, 1), (1025, 4096), (2500, 4097), (8192, 70001)])
def test_many_rows(B, n_pages):
    rng = random.Random(B)
    m, d = Model(n_pages, 8, B), Device(n_pages, 8, B, 12)
    d.load(m)
    status = 0
    for want in ([rng.randint(0, 16) for _ in range(B)], [rng.randint(0, 40) for _ in range(B)], [0] * B, [8 + i % 3 for i in range(B)]):
        moves, short = m.reserve(want)
        status |= sps.PAGED_NO_PAGE if short else 0
        d.reserve(want)
        d.check(m, status)
        m.lens = [min(w, 8 * len(r)) for w, r in zip(want, m.rows)]
        d.t.lens.copy_(ints(m.lens))


@pytest.mark.parametrize("n_pages", [31, 33, 2999, 3071, 3500, 4095, 4600, 5121, 24575, 24576, 24577, 32769])
def test_pools_of_any_size(n_pages):
    """Both kernels and every request for shared memory: pages at both ends of the pool, taken, shared, exchanged and given up."""
    page, top = 8, min(60, n_pages // 8)
    m, d = Model(n_pages, page, 9), Device(n_pages, page, 9, n_pages)
    d.load(m)
    status = 0
    for want in ([8 * top] * 8 + [8 * (n_pages - 8 * top)], [8 * top + 3] * 4 + [0] * 4 + [8 * (n_pages - 8 * top)], [5] * 8 + [0], [7] * 9):
        moves, short = m.reserve(want)
        status |= sps.PAGED_NO_PAGE if short else 0
        d.reserve(want)
        assert d.listed() == moves
        d.check(m, status)
        m.lens = [min(w, page * len(r)) for w, r in zip(want, m.rows)]
        d.t.lens.copy_(ints(m.lens))
        parents = [0, 0, 2, 3, 3, 5, 6, 7, 8]
        m.fork(parents)
        d.fork(parents)
        d.check(m, status)


@pytest.mark.parametrize("offset", [1, 2, 3])
def test_references_of_any_alignment(offset):
    m, d = grown(300, 8, [90, 41, 7, 500], ld=120)
    store = torch.zeros(300 + offset, dtype=I32, device=DEV)
    store[offset:] = d.pool.refs
    d.pool = sps.PagePool(store[offset:], 8)
    for want in ([91, 60, 0, 900], [3, 3, 3, 3]):
        m.reserve(want)
        d.reserve(want)
        d.check(m)
    assert d.listed() == []
    moves = m.compact(10 ** 9)
    d.compact()
    assert d.listed() == moves
    d.check(m)


def test_a_pool_of_several_rounds():
    """More pages than a CTA has threads for words of them (8 x 32768)."""
    n_pages = 600_001
    m, d = Model(n_pages, 8, 40), Device(n_pages, 8, 40, 60000)
    d.load(m)
    lens = [8 * 14900 + 3 * i for i in range(40)]
    status = 0
    for want in (lens, [0 if i % 3 == 0 else n + 1 for i, n in enumerate(lens)], [n + 90000 * (i % 3 == 0) for i, n in enumerate(lens)], [i % 2 * n for i, n in enumerate(lens)]):
        moves, short = m.reserve(want)
        status |= sps.PAGED_NO_PAGE if short else 0
        d.reserve(want)
        d.check(m, status)
        m.lens = [min(w, 8 * len(r)) for w, r in zip(want, m.rows)]
        d.t.lens.copy_(ints(m.lens))
    assert status == sps.PAGED_NO_PAGE
    moves = m.compact(10 ** 9)
    d.compact()
    assert d.listed() == moves and len(moves) > 100_000
    d.check(m, status)


def test_long_rows():
    """Thousands of pages to a row, taken and given up; the first call asks for one page more than there are."""
    m, d = Model(30000, 8, 3), Device(30000, 8, 3, 20000)
    d.load(m)
    for want, without in (([160000, 1, 79999], True), ([7, 160000, 0], False), ([80000, 80000, 79999], False), ([0, 0, 0], False)):
        moves, short = m.reserve(want)
        d.reserve(want)
        assert short == without
        d.check(m, sps.PAGED_NO_PAGE)
        m.lens = [min(w, 8 * len(r)) for w, r in zip(want, m.rows)]
        d.t.lens.copy_(ints(m.lens))


def test_reserve_clips_and_skips_what_does_not_fit():
    m, d = grown(20, 8, [30, 9, 17], ld=6)
    d.t.pages[0, 3] = 20                                       # given up: skipped
    d.reserve([8, 9, 17])
    assert int(d.pool.status) == sps.PAGED_BAD_PAGE and d.t.held.tolist() == [1, 2, 3]
    assert d.pool.refs.tolist()[m.rows[0][3]] == 1 and d.pool.refs.sum() == 1 + 2 + 3 + 1
    m, d = grown(20, 8, [30, 9], ld=6)
    d.t.pages[1, 1] = -5                                       # about to be written: not exchanged
    d.reserve([30, 20])
    assert int(d.pool.status) == sps.PAGED_BAD_PAGE and d.t.held.tolist() == [4, 3] and d.listed() == []
    m, d = grown(20, 8, [30, 9], ld=6)
    d.t.lens[0], d.t.lens[1] = 33, -4                          # more tokens than pages; fewer than none
    d.reserve([40, 3])
    assert int(d.pool.status) == sps.PAGED_BAD_LENGTH and d.t.lens.tolist() == [32, 0] and d.t.held.tolist() == [5, 1]
    m, d = grown(60, 8, [30, 9], ld=6)
    d.reserve([2 ** 31 - 1, -7])                               # as much as the row can hold; nothing
    assert int(d.pool.status) == sps.PAGED_BAD_LENGTH and d.t.held.tolist() == [6, 0] and d.t.lens.tolist() == [30, 0]
    m, d = grown(20, 8, [30, 9], ld=6)
    d.t.held[0], d.t.held[1] = 99, -1
    d.t.pages[0, 4:] = ints(m.rows[1])
    d.reserve([30, 0])
    assert int(d.pool.status) == sps.PAGED_BAD_LENGTH and d.t.held.tolist() == [4, 0]


def test_entries_behind_a_row_are_neither_read_nor_written():
    m, d = grown(40, 8, [21, 3], ld=9)
    d.reserve([25, 3])
    assert (d.t.pages[0, 4:] == 2 ** 31 - 1).all() and (d.t.pages[1, 1:] == 2 ** 31 - 1).all()
    assert (d.moves.list == -7).all()


# --------------------------------------------------------------------------------------------------------------- compact
@pytest.mark.parametrize("n_pages,share", [(1, 1.0), (1, 0.0), (37, 0.5), (4096, 0.3), (4097, 0.9), (33000, 0.1), (33000, 0.66), (33000, 1.0), (33000, 0.0)])
@pytest.mark.parametrize("inplace", [False, True])
def test_compact(n_pages, share, inplace):
    rng = random.Random(n_pages)
    lens = []
    left = int(n_pages * share)
    while left > 0:
        lens.append(8 * rng.randint(1, min(left, 900)))
        left -= lens[-1] // 8
    m, d = grown(n_pages, 8, lens or [0], seed=3)
    parents = [rng.randrange(len(m.rows)) if rng.random() < 0.2 else i for i in range(len(m.rows))]
    m.fork(parents)
    d.fork(parents)
    if inplace:
        moves = m.compact(10 ** 9)
        d.compact()
        d.check(m)
    else:
        before = [t.clone() for t in (d.t.pages, d.t.held, d.t.lens, d.pool.refs)]
        moves = m.compact(10 ** 9)
        out, refs = Device.table(d.B, d.ld + 1), torch.full_like(d.pool.refs, -3)
        sps.sps_paged_compact(d.pool, d.t, out, refs, d.moves, d.ws)
        assert all(torch.equal(a, b) for a, b in zip(before, (d.t.pages, d.t.held, d.t.lens, d.pool.refs)))
        assert [r[:h] for r, h in zip(out.pages.tolist(), out.held.tolist())] == m.rows
        assert all(x == -9 for r, h in zip(out.pages.tolist(), out.held.tolist()) for x in r[h:])
        assert out.lens.tolist() == m.lens and refs.tolist() == m.refs
    assert d.listed() == moves
    consistent(m)


def test_compact_in_steps_of_a_short_list():
    m, d = grown(600, 8, [8 * 60] * 4, seed=1)
    short = Device(600, 8, 4, d.ld, capacity=7)
    short.load(m)
    for _ in range(100):
        moves = m.compact(7)
        short.compact()
        assert short.listed() == moves
        short.check(m)
        if not moves:
            break
    assert not moves and sorted(p for r in m.rows for p in r) == list(range(240))


@pytest.mark.parametrize("n_pages", [50, 20000])
def test_compact_without_rows_moves_what_is_in_use(n_pages):
    """Pages that no table of this call names: their references and contents move all the same."""
    d = Device(n_pages, 8, 0, 0)
    d.pool.refs[n_pages - 7:] = 3
    d.compact()
    assert d.listed() == [[n_pages - 7 + i, i, 8] for i in range(7)]
    assert d.pool.refs[:7].tolist() == [3] * 7 and not d.pool.refs[7:].any()
    d = Device(n_pages, 8, 2, 0)
    d.pool.refs[n_pages - 1] = 1
    d.compact()
    assert d.listed() == [[n_pages - 1, 0, 8]] and d.t.held.tolist() == [0, 0]


def test_compact_keeps_entries_that_name_no_page():
    m, d = grown(40, 8, [30, 30], seed=2)
    d.t.pages[0, 0], d.t.pages[1, 2] = 40, -2
    d.compact()
    assert int(d.pool.status) == sps.PAGED_BAD_PAGE and d.t.pages[0, 0] == 40 and d.t.pages[1, 2] == -2


# ------------------------------------------------------------------------------------------------------------------ copy
def caches(L, n_pages, H, page, d, dtype, order, seed=0, gap=0):
    """gap: elements between slots' ends (of the innermost two dimensions' row) and the next."""
    g = torch.Generator(device=DEV).manual_seed(seed)
    out = []
    for _ in range(2 * L):
        shape = (n_pages, H, page, d + gap) if order == "head" else (n_pages, page, H, d + gap)
        t = torch.randn(shape, generator=g, device=DEV).to(dtype)[..., :d]
        out.append(t if order == "head" else t.transpose(1, 2))
    return out[:L], out[L:]


def copied(t, moves):
    t = t.clone()
    for a, b, n in moves:
        t[b, :, :n] = t[a, :, :n]
    return t


@pytest.mark.parametrize("L,H,page,d,dtype,order,gap", [(1, 1, 8, 64, BF16, "head", 0), (2, 3, 16, 128, BF16, "head", 0), (2, 3, 16, 128, BF16, "slot", 0),
                                                        (3, 8, 32, 64, F32, "slot", 0), (2, 5, 64, 128, F32, "head", 8), (1, 2, 512, 128, F32, "slot", 4),
                                                        (2, 40, 64, 128, BF16, "head", 0), (65, 2, 8, 64, BF16, "head", 0), (130, 1, 8, 64, F32, "slot", 0)])
def test_copy(L, H, page, d, dtype, order, gap):
    n_pages = 40
    k, v = caches(L, n_pages, H, page, d, dtype, order, gap=gap)
    perm = torch.randperm(n_pages, generator=torch.Generator().manual_seed(L)).tolist()
    slots = [1, page, page - 1, 0, page // 2, 3, page]
    moves = [[perm[2 * i], perm[2 * i + 1], n] for i, n in enumerate(slots)]
    want = [[copied(t, moves) for t in x] for x in (k, v)]
    layers = sps.PagedLayers([sps.PagedCache(a, b) for a, b in zip(k, v)])
    sps.sps_paged_copy(layers, sps.PageMoves(ints(moves + [[0, 1, page]]), ints([len(moves)])))
    for got, w in zip(k + v, want[0] + want[1]):
        assert torch.equal(got, w)


@pytest.mark.parametrize("L,H,page,d,dtype,order,gap", [(2, 3, 16, 128, BF16, "head", 0), (2, 3, 16, 128, BF16, "slot", 0), (1, 9, 64, 128, F32, "head", 8),
                                                        (66, 2, 8, 64, BF16, "slot", 0)])
def test_copy_of_a_long_list_little_of_which_is_used(L, H, page, d, dtype, order, gap):
    """A list that could hold more than half a gigabyte: the other kernel."""
    n_pages = 40
    k, v = caches(L, n_pages, H, page, d, dtype, order, gap=gap)
    capacity = 600_000_000 // (2 * min(L, 2) * H * page * d * k[0].element_size())
    perm = torch.randperm(n_pages, generator=torch.Generator().manual_seed(L)).tolist()
    slots = [1, page, page - 1, 0, page // 2, 3, page]
    moves = [[perm[2 * i], perm[2 * i + 1], n] for i, n in enumerate(slots)]
    want = [copied(t, moves) for t in k + v]
    layers = sps.PagedLayers([sps.PagedCache(a, b) for a, b in zip(k, v)])
    list_ = torch.full((capacity, 3), -1, dtype=I32, device=DEV)
    list_[:len(moves)] = ints(moves)
    sps.sps_paged_copy(layers, sps.PageMoves(list_, ints([len(moves)])))
    assert all(torch.equal(a, b) for a, b in zip(k + v, want))


def test_copy_of_pages_of_more_places_than_ctas():
    k, v = caches(40, 6, 8, 512, 64, BF16, "head")
    moves = [[5, 0, 512], [3, 1, 77], [4, 2, 511]]
    want = [copied(t, moves) for t in k + v]
    layers = sps.PagedLayers([sps.PagedCache(a, b) for a, b in zip(k, v)])
    for capacity in (3, 9):
        list_ = torch.zeros((capacity, 3), dtype=I32, device=DEV)
        list_[:3] = ints(moves)
        sps.sps_paged_copy(layers, sps.PageMoves(list_, ints([3])))
        assert all(torch.equal(a, b) for a, b in zip(k + v, want))


def test_copy_skips_what_does_not_fit():
    k, v = caches(2, 6, 2, 8, 64, BF16, "head")
    moves = [[0, 6, 8], [-1, 1, 8], [6, 2, 8], [3, -5, 8], [4, 5, 99], [2, 1, -3]]
    want = [copied(t, [[4, 5, 8]]) for t in k + v]
    layers = sps.PagedLayers([sps.PagedCache(a, b) for a, b in zip(k, v)])
    for count in (6, 1000, 5):                                 # (a count above the list's capacity is taken as that)
        sps.sps_paged_copy(layers, sps.PageMoves(ints(moves), ints([count])))
        assert all(torch.equal(a, b) for a, b in zip(k + v, want))
    before = [t.clone() for t in k + v]
    for count in (0, -4):
        sps.sps_paged_copy(layers, sps.PageMoves(ints([[0, 1, 8]]), ints([count])))
    assert all(torch.equal(a, b) for a, b in zip(k + v, before))


def test_copy_of_far_pages():
    """Offsets that pass 2^31 elements."""
    n_pages, H, page, d = 70000, 4, 64, 128
    t = torch.zeros((n_pages, H, page, d), dtype=BF16, device=DEV)
    t[n_pages - 1].normal_()
    t[n_pages - 2].normal_()
    layers = sps.PagedLayers([sps.PagedCache(t, t)])
    sps.sps_paged_copy(layers, sps.PageMoves(ints([[n_pages - 1, 3, 64], [n_pages - 2, n_pages - 5, 9]]), ints([2])))
    assert torch.equal(t[3], t[n_pages - 1]) and torch.equal(t[n_pages - 5, :, :9], t[n_pages - 2, :, :9]) and not t[n_pages - 5, :, 9:].any()


# ----------------------------------------------------------------------------------------------------- streams and graphs
def test_a_captured_step_replays_on_changed_state():
    """Fork, reserve and copy captured once, replayed while parents, lengths and tables move."""
    page, B, L = 8, 6, 2
    m, d = grown(120, page, [21, 13, 8, 40, 0, 5], ld=12)
    k, v = caches(L, 120, 2, page, 64, BF16, "head")
    layers = sps.PagedLayers([sps.PagedCache(a, b) for a, b in zip(k, v)])
    parents, want = ints(list(range(B))), ints([0] * B)
    a, b = d.tables
    st = torch.cuda.Stream()
    refs0 = d.pool.refs.clone()
    with torch.cuda.stream(st):
        def step(s, t):
            sps.sps_paged_fork(d.pool, s, t, parents)
            sps.sps_paged_reserve(d.pool, t, want, d.moves, d.ws)
            sps.sps_paged_copy(layers, d.moves)
        graphs = [torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()]
        for g, (s, t) in zip(graphs, ((a, b), (b, a))):
            with torch.cuda.graph(g, stream=st):
                step(s, t)
    assert torch.equal(refs0, d.pool.refs)
    rng = random.Random(5)
    for i in range(10):
        p = [rng.choice([x, rng.randrange(B)]) for x in range(B)]
        m.fork(p)
        w = [min(90, n + rng.randint(0, 3)) for n in m.lens]
        before = [t.clone() for t in k + v]
        moves, short = m.reserve(w)
        assert not short
        with torch.cuda.stream(st):
            parents.copy_(ints(p))
            want.copy_(ints(w))
            graphs[i % 2].replay()
        st.synchronize()
        d.at = 1 - i % 2
        d.check(m)
        assert d.listed() == moves and all(torch.equal(x, copied(y, moves)) for x, y in zip(k + v, before))
        m.lens = list(w)
        d.t.lens.copy_(ints(w))
        torch.cuda.synchronize()


def test_calls_on_a_stream_of_their_own():
    m, d = grown(64, 8, [21, 13], ld=9)
    st = torch.cuda.Stream()
    torch.cuda.synchronize()
    parents, want = ints([1, 1]), ints([14, 20])
    torch.cuda.synchronize()
    sps.sps_paged_fork(d.pool, d.tables[0], d.tables[1], parents, stream=st.cuda_stream)
    sps.sps_paged_reserve(d.pool, d.tables[1], want, d.moves, d.ws, stream=st.cuda_stream)
    st.synchronize()
    d.at = 1
    m.fork([1, 1])
    assert d.listed() == m.reserve([14, 20])[0]
    d.check(m)


def test_the_binding_refuses_what_it_can_see():
    m, d = grown(20, 8, [9, 9])
    with pytest.raises(ValueError):
        sps.PagePool(d.pool.refs.long(), 8)
    with pytest.raises(ValueError):
        sps.PagePool(d.pool.refs.cpu(), 8)
    with pytest.raises(ValueError):
        sps.PageTable(d.t.pages, d.t.held[:1], d.t.lens)
    with pytest.raises(ValueError):
        sps.PageTable(d.t.pages.t(), d.t.held, d.t.lens)
    with pytest.raises(ValueError):
        sps.PageMoves(torch.zeros((4, 2), dtype=I32, device=DEV), d.moves.count)
    with pytest.raises(ValueError):
        sps.sps_paged_fork(d.pool, d.t, d.tables[1], ints([0]))
    with pytest.raises(ValueError):
        sps.sps_paged_reserve(d.pool, d.t, ints([1, 2, 3]), d.moves, d.ws)
    with pytest.raises(ValueError):
        sps.sps_paged_reserve(d.pool, d.t, ints([1, 2]), d.moves, d.ws[:-16])
    with pytest.raises(ValueError):
        sps.sps_paged_compact(d.pool, d.t, d.t, d.pool.refs[:-1], d.moves, d.ws)
    with pytest.raises(ValueError):
        sps.PagedLayers([])
