"""Beams over shared pages, as a serving program would search: whole models run through sps_paged_append and
sps_paged_attention, the selection over their logits, and fork, reserve and copy of the pages behind it; against a search that
runs every beam from scratch."""
import math

import numpy as np
import pytest
import torch

import paper_2302_01318_b200 as sps
import sps_synth
from gpu_util import oracle_model
from pages_util import DEV, I32, ints
from test_gpu_paged_model import TOL, PagedModel

pytestmark = pytest.mark.gpu


class Beams:
    """B prompts of W beams each over one pool; page 8."""

    def __init__(self, model, prompts, W, n_pages, top, end):
        self.model, self.W, self.B, self.end, page = model, W, len(prompts), end, 8
        rows, ld = self.B * W, -(-top // page)
        self.pool = sps.PagePool(torch.zeros(n_pages, dtype=I32, device=DEV), page)
        self.tables = [self.table(rows, ld), self.table(rows, ld)]
        self.moves = sps.PageMoves(torch.zeros((rows, 3), dtype=I32, device=DEV), torch.zeros(1, dtype=I32, device=DEV))
        self.ws = torch.zeros(sps.sps_paged_pool_workspace_bytes(n_pages), dtype=torch.uint8, device=DEV)
        self.layers = sps.PagedLayers(model.caches)
        V = model.cfg["vocab"]
        self.select_ws = torch.zeros(sps.sps_beam_select_workspace_bytes(self.B, W, V), dtype=torch.uint8, device=DEV)
        self.scores, self.done = torch.zeros((self.B, W), device=DEV), torch.zeros((self.B, W), dtype=I32, device=DEV)
        self.parents, self.tokens = (torch.zeros((self.B, W), dtype=I32, device=DEV) for _ in range(2))
        # the prompts, one row each; the first selection makes beams of them
        first = self.table(self.B, ld)
        lens = [len(p) for p in prompts]
        sps.sps_paged_reserve(self.pool, first, ints(lens), self.moves, self.ws)
        logits = self.forward(first, ints(lens), [t for p in prompts for t in p], lens)
        last = torch.tensor(lens).cumsum(0) - 1
        sps.sps_beam_select(logits[last].view(self.B, 1, V).contiguous(), torch.zeros((self.B, 1), device=DEV), self.scores, self.parents, self.tokens,
                            self.select_ws, out_done=self.done, end_token=end)
        sps.sps_paged_fork(self.pool, first, self.tables[0], self.parents.view(-1))
        self.t, self.text = self.tables[0], [[] for _ in range(rows)]
        self.note()

    @staticmethod
    def table(rows, ld):
        return sps.PageTable(torch.zeros((rows, ld), dtype=I32, device=DEV), torch.zeros(rows, dtype=I32, device=DEV), torch.zeros(rows, dtype=I32, device=DEV))

    def note(self):
        """What each beam has said so far, from parents and tokens (the first selection's parents are prompts)."""
        p, t = self.parents.view(-1).tolist(), self.tokens.view(-1).tolist()
        old = self.text
        self.text = [(list(old[a]) if any(old) and a >= 0 else []) + [x] for a, x in zip(p, t)]

    def forward(self, table, lens, tokens, news):
        sps.sps_paged_copy(self.layers, self.moves)
        q_start = torch.tensor([0] + list(news)).cumsum(0).to(torch.int32).to(DEV)
        batch = sps.PagedBatch(q_start, lens, table.pages, max_q=max(news))
        logits = self.model.forward(tokens, batch)
        assert int(batch.status) == 0
        table.lens.copy_(lens)
        return logits

    def step(self):
        rows = self.B * self.W
        want = self.t.lens + 1
        sps.sps_paged_reserve(self.pool, self.t, want, self.moves, self.ws)
        logits = self.forward(self.t, want, self.tokens.view(-1).tolist(), [1] * rows).view(self.B, self.W, -1)
        sps.sps_beam_select(logits, self.scores, self.scores, self.parents, self.tokens, self.select_ws, done=self.done, out_done=self.done, end_token=self.end)
        other = self.tables[1] if self.t is self.tables[0] else self.tables[0]
        sps.sps_paged_fork(self.pool, self.t, other, self.parents.view(-1))
        self.t = other
        self.note()
        assert int(self.pool.status) == 0
        refs = torch.zeros_like(self.pool.refs)
        for r in range(rows):
            h = int(self.t.held[r])
            refs.index_add_(0, self.t.pages[r, :h].long(), torch.ones(h, dtype=I32, device=DEV))
        assert torch.equal(refs, self.pool.refs)


def search(cfg, w, prompt, W, steps, end):
    """Beams of one prompt, every one of them evaluated from scratch in 64 bits; also the least distance that decided anything."""
    beams, gap = [([], 0.0, False)], math.inf
    for _ in range(steps):
        found = []
        for text, score, over in beams:
            if over:
                found.append((score, text + [end], True))
                continue
            seq = np.array(prompt + text, dtype=np.int32)
            x = oracle_model(cfg, w, 64).forward64(seq, np.arange(len(seq), dtype=np.int32))[-1]
            logp = x - x.max() - math.log(np.exp(x - x.max()).sum())
            found += [(score + logp[t], text + [int(t)], int(t) == end) for t in np.argsort(-logp)[:W + 1]]
        found.sort(key=lambda e: -e[0])
        gap = min([gap] + [a[0] - b[0] for a, b in zip(found[:W], found[1:])])
        beams = [(t, s, o) for s, t, o in found[:W]]
    return beams, gap


@pytest.mark.parametrize("name,W", [("tiny", 4), ("tiny_gqa", 3), ("tiny_bf16", 2)])
def test_beams_over_shared_pages_find_what_beams_from_scratch_find(name, W):
    cfg = sps_synth.CONFIGS[name]["target"]
    w = sps_synth.make_weights(cfg, seed=5)
    V, steps = cfg["vocab"], 6
    prompts = [list(map(int, sps_synth.make_prompt(i, n, V))) for i, n in enumerate((21, 8, 3))]
    n_pages, top = 60, 40
    model = PagedModel(cfg, sps_synth.weights_to(w, DEV), n_pages, 8)
    end = search(cfg, w, prompts[1], W, 2, -1)[0][0][0][1]            # a token that is found on the way: some beams end
    b = Beams(model, prompts, W, n_pages, top, end)
    for _ in range(steps - 1):
        b.step()
    assert (b.done != 0).any()
    for i, p in enumerate(prompts):
        want, gap = search(cfg, w, p, W, steps, end)
        got = [(b.text[i * W + j], float(b.scores[i, j]), bool(b.done[i, j])) for j in range(W)]
        tol = 2 * steps * TOL[name]                                   # each step's log-probability moves with its logits, twice at most
        for j in range(W):
            assert abs(got[j][1] - want[j][1]) < tol
        if gap > 2 * tol:
            assert [g[0] for g in got] == [x[0] for x in want] and [g[2] for g in got] == [x[2] for x in want]
        # whatever the order, a beam's score is the one its own tokens have from scratch
        for text, score, _ in got:
            said = 0.0
            for k, t in enumerate(text):
                if k > 0 and text[k - 1] == end:
                    break
                seq = np.array(p + text[:k], dtype=np.int32)
                x = oracle_model(cfg, w, 64).forward64(seq, np.arange(len(seq), dtype=np.int32))[-1]
                said += x[t] - x.max() - math.log(np.exp(x - x.max()).sum())
            assert abs(said - score) < tol
    # all rows given up: nothing is held, and the pool serves another prompt
    b.t.lens.zero_()
    sps.sps_paged_reserve(b.pool, b.t, torch.zeros_like(b.t.lens), b.moves, b.ws)
    assert not b.pool.refs.any() and not b.t.held.any()


def test_a_pool_compacted_between_steps_changes_nothing():
    """Two rows of unlike lengths decode; a third leaves, the pool moves together, and the next logits are those of a pool that
    never did."""
    cfg = sps_synth.CONFIGS["tiny"]["target"]
    w = sps_synth.weights_to(sps_synth.make_weights(cfg, seed=6), DEV)
    V, n_pages = cfg["vocab"], 30
    prompts = [list(map(int, sps_synth.make_prompt(i, n, V))) for i, n in enumerate((40, 50, 21))]
    out = []
    for compact in (False, True):
        model = PagedModel(cfg, w, n_pages, 8)
        b = Beams.__new__(Beams)
        b.model, b.layers = model, sps.PagedLayers(model.caches)
        pool = sps.PagePool(torch.zeros(n_pages, dtype=I32, device=DEV), 8)
        t = Beams.table(3, 8)
        b.moves = sps.PageMoves(torch.zeros((n_pages, 3), dtype=I32, device=DEV), torch.zeros(1, dtype=I32, device=DEV))
        ws = torch.zeros(sps.sps_paged_pool_workspace_bytes(n_pages), dtype=torch.uint8, device=DEV)
        lens = ints([len(p) for p in prompts])
        sps.sps_paged_reserve(pool, t, lens, b.moves, ws)
        b.forward(t, lens, [x for p in prompts for x in p], [len(p) for p in prompts])
        keep = ints([40, 0, 21])
        t.lens.copy_(keep)
        sps.sps_paged_reserve(pool, t, keep, b.moves, ws)             # the second row leaves
        if compact:
            sps.sps_paged_compact(pool, t, t, pool.refs, b.moves, ws)
            assert int(b.moves.count) == 3 and int((pool.refs != 0).sum()) == 8 and bool((pool.refs[:8] == 1).all())
            sps.sps_paged_copy(b.layers, b.moves)
        want = ints([41, 0, 22])
        sps.sps_paged_reserve(pool, t, want, b.moves, ws)
        out.append(b.forward(t, want, [7, 9], [1, 0, 1]))
        assert int(pool.status) == 0
    assert torch.equal(*out)
