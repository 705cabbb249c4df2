"""What rows keep when pages run out: every token that a row has is followed through forks, reserves, copies and appends, told
apart by a number of its own in the cache.  Nothing here says which page a row gets: only what the calls promise -- a row keeps the
tokens that it kept, whatever the others write within the room that they were given."""
import random

import pytest
import torch

import paper_2302_01318_b200 as sps
from pages_util import DEV, F32, I32, ints

pytestmark = pytest.mark.gpu


class Cache:
    """A pool, two tables and one layer's keys and values, whose first element is the token's number; texts: what each row has."""

    def __init__(self, n_pages, page, B, ld):
        self.page, self.n_pages, self.B, self.ld = page, n_pages, B, ld
        self.pool = sps.PagePool(torch.zeros(n_pages, dtype=I32, device=DEV), page)
        self.tables = [sps.PageTable(torch.full((B, ld), -1, dtype=I32, device=DEV), torch.zeros(B, dtype=I32, device=DEV), torch.zeros(B, dtype=I32, device=DEV))
                       for _ in range(2)]
        self.k, self.v = (torch.zeros((n_pages, 1, page, 64), dtype=F32, device=DEV) for _ in range(2))
        self.layers = sps.PagedLayers([sps.PagedCache(self.k, self.v)])
        self.moves = sps.PageMoves(torch.zeros((max(B, 1), 3), dtype=I32, device=DEV), torch.zeros(1, dtype=I32, device=DEV))
        self.ws = torch.zeros(sps.sps_paged_pool_workspace_bytes(n_pages), dtype=torch.uint8, device=DEV)
        self.texts, self.number, self.short = [[] for _ in range(B)], 0, False

    @property
    def t(self):
        return self.tables[0]

    def places(self, row, pages, first, last):
        at = torch.arange(first, last)
        return torch.tensor(pages[row], dtype=torch.int64)[at // self.page] * self.page + at % self.page

    def step(self, want):
        """Reserve, copy, and every row filled up to the room that it has.  Returns the room."""
        kept = [min(len(x), max(w, 0)) for x, w in zip(self.texts, want)]
        room = torch.full((self.B,), -4, dtype=I32, device=DEV)
        self.pool.status.zero_()
        sps.sps_paged_reserve(self.pool, self.t, ints(want), self.moves, self.ws, room=room)
        sps.sps_paged_copy(self.layers, self.moves)
        room = room.tolist()
        self.short = bool(int(self.pool.status) & sps.PAGED_NO_PAGE)
        assert int(self.pool.status) & ~sps.PAGED_NO_PAGE == 0
        assert self.t.lens.tolist() == kept
        for n, w, r in zip(kept, want, room):
            assert r == w or (r == n and self.short and w > n)
        assert self.short == any(r < w for r, w in zip(room, want))
        self.texts = [x[:n] for x, n in zip(self.texts, kept)]
        pages, held = self.t.pages.tolist(), self.t.held.tolist()
        where, what = [], []
        for i, r in enumerate(room):
            assert held[i] == -(-r // self.page)
            if r == kept[i]:
                continue
            new = list(range(self.number + 1, self.number + 1 + r - kept[i]))
            self.number += len(new)
            where.append(self.places(i, pages, kept[i], r))
            what += new
            self.texts[i] = self.texts[i] + new
        where = torch.cat([torch.zeros(0, dtype=torch.int64)] + where)
        assert where.unique().numel() == where.numel()                      # no two rows write to one place
        x = torch.tensor(what, dtype=F32, device=DEV)
        self.k.view(-1, 64)[where.to(DEV), 0] = x
        self.v.view(-1, 64)[where.to(DEV), 0] = -x
        self.t.lens.copy_(ints(room))
        self.check()
        return room

    def fork(self, parents):
        sps.sps_paged_fork(self.pool, self.tables[0], self.tables[1], ints(parents))
        self.tables.reverse()
        self.texts = [list(self.texts[p]) if p >= 0 else [] for p in parents]
        self.check()

    def roll_back(self, lens):
        self.texts = [x[:n] for x, n in zip(self.texts, lens)]
        self.t.lens.copy_(ints([len(x) for x in self.texts]))

    def check(self):
        pages, held = self.t.pages.tolist(), self.t.held.tolist()
        assert self.t.lens.tolist() == [len(x) for x in self.texts]
        where = torch.cat([torch.zeros(0, dtype=torch.int64)] + [self.places(i, pages, 0, len(x)) for i, x in enumerate(self.texts) if x]).to(DEV)
        want = torch.tensor([a for x in self.texts for a in x], dtype=F32, device=DEV)
        assert torch.equal(self.k.view(-1, 64)[where, 0], want) and torch.equal(self.v.view(-1, 64)[where, 0], -want)
        refs = torch.zeros(self.n_pages, dtype=I32)
        for r, h in zip(pages, held):
            if h:
                refs.index_add_(0, torch.tensor(r[:h], dtype=torch.int64), torch.ones(h, dtype=I32))
        assert torch.equal(refs, self.pool.refs.cpu())


def full(kind, B):
    """A cache whose pool will be full: one page for rows 0 .. B - 1, and a last row that holds all the others (none in a pool of one
    page).  The kernels: few rows and pages, a large pool, many rows."""
    n_pages, rows = {"small": (1, B), "large": (24577, B + 1), "rows": (1, 1030)}[kind]
    c = Cache(n_pages, 8, rows, max(n_pages, 3))
    c.step([0] * B + [8 * (n_pages - 1)] * (rows - B) if kind == "large" else [0] * rows)
    return c


KINDS = ["small", "large", "rows"]


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("lens,want", [((3, 5), (4, 6)), ((5, 3), (6, 4)), ((3, 5), (8, 8)), ((3, 5), (6, 6)), ((1, 7), (2, 8)), ((3, 5, 5, 4), (4, 6, 6, 5)),
                                       ((4, 3, 6, 2), (5, 5, 7, 7)), ((5, 5), (6, 6)), ((3, 5), (4, 9)), ((3, 5), (9, 6)), ((2, 6, 6), (3, 6, 7))])
def test_holders_of_unlike_lengths_and_no_free_page(kind, lens, want):
    c = full(kind, len(lens))
    rest = c.B - len(lens)
    others = [len(x) for x in c.texts[len(lens):]]
    c.step([max(lens)] + [0] * (len(lens) - 1) + others)                    # the one page, filled by row 0
    c.fork([0] * len(lens) + list(range(len(lens), c.B)))
    c.roll_back(list(lens) + others)
    c.step(list(want) + others)
    assert c.short and len(c.texts) == len(lens) + rest
    c.step([len(x) for x in c.texts])                                       # (nobody wants anything: all is as it was)


@pytest.mark.parametrize("kind", KINDS)
def test_a_sibling_ahead_is_not_overwritten_once_it_stands_behind(kind):
    """A shortage on equal lengths leaves one row a token ahead; a fork exchanges the two."""
    c = full(kind, 2)
    others = [len(x) for x in c.texts[2:]]
    c.step([5, 0] + others)
    c.fork([0, 0] + list(range(2, c.B)))
    for _ in range(3):
        c.step([min(len(x) + 1, 8) for x in c.texts[:2]] + others)
        c.fork([1, 0] + list(range(2, c.B)))


@pytest.mark.parametrize("kind", KINDS)
def test_of_alike_lengths_the_first_goes_on_and_of_unlike_ones_the_longest(kind):
    """Who holds the most tokens of the page can write behind all the others' -- and does: the pool's last page is not left idle."""
    c = full(kind, 3)
    others = [len(x) for x in c.texts[3:]]
    c.step([6, 0, 0] + others)
    c.fork([0, 0, 0] + list(range(3, c.B)))
    c.roll_back([4, 6, 6] + others)
    assert c.step([5, 7, 7] + others)[:3] == [4, 7, 6]


@pytest.mark.parametrize("kind", KINDS)
def test_one_who_only_reads_keeps_the_others_from_writing(kind):
    c = full(kind, 3)
    others = [len(x) for x in c.texts[3:]]
    c.step([6, 0, 0] + others)
    c.fork([0, 0, 0] + list(range(3, c.B)))
    c.roll_back([4, 3, 6] + others)
    assert c.step([5, 3, 7] + others)[:3] == [4, 3, 6]


@pytest.mark.parametrize("n_pages,page,B,top,hog", [(5, 8, 4, 40, 0), (6, 8, 7, 30, 0), (14, 16, 20, 90, 0), (25, 8, 1030, 40, 0), (20, 8, 8192, 60, 0), (24600, 8, 6, 40, 24590),
                                                    (40000, 16, 9, 70, 39985)])
def test_a_random_history_in_a_pool_that_is_short(n_pages, page, B, top, hog):
    """Forks, rollbacks and growth of rows that share pages, most reserves without pages enough; hog: pages that a row more
    holds throughout."""
    rng = random.Random(n_pages * 31 + B)
    c = Cache(n_pages, page, B + (hog > 0), max(hog, -(-top // page)) + 1)
    rest = [hog * page] * (hog > 0)
    live = min(B, 24)                                                       # the others stay empty
    spread = [B - 1 - i * (B // live) for i in range(live)]                 # ... and lie between
    c.step([0] * B + rest)
    shorts = 0
    for _ in range(40):
        kind = rng.random()
        parents, lens, want = list(range(c.B)), [len(x) for x in c.texts], [len(x) for x in c.texts]
        if kind < 0.35:
            for i in spread:
                if rng.random() < 0.6:
                    parents[i] = rng.choice(spread + [-1])
            c.fork(parents)
            continue
        if kind < 0.75:
            for i in spread:
                if rng.random() < 0.4:
                    lens[i] = max(0, lens[i] - rng.randint(0, page))
            c.roll_back(lens)
        for i in spread:
            want[i] = rng.choice([0, lens[i]]) if rng.random() < 0.2 else min(top, lens[i] + rng.choice([1, 1, 2, 3, page]))
        c.step(want)
        shorts += c.short
    assert shorts >= 5
