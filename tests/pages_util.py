"""The pages of a cache and the selection of a beam step as plain Python over lists and 64-bit numbers, shared by their tests."""
import math

import torch

import paper_2302_01318_b200 as sps

DEV = "cuda"
F32, BF16, I32 = torch.float32, torch.bfloat16, torch.int32


def ints(x, shape=None):
    t = torch.tensor(x, dtype=I32)
    return (t if shape is None else t.reshape(shape)).to(DEV)


# ----------------------------------------------------------------------------------------------------------------- pages
class Model:
    """refs: references of each page; rows: pages of each row; lens: tokens of each row."""

    def __init__(self, n_pages, page, B):
        self.refs, self.page, self.rows, self.lens = [0] * n_pages, page, [[] for _ in range(B)], [0] * B

    def fork(self, parents):
        rows = [list(self.rows[p]) if p >= 0 else [] for p in parents]
        for r in self.rows:
            for p in r:
                self.refs[p] -= 1
        for r in rows:
            for p in r:
                self.refs[p] += 1
        self.lens = [self.lens[p] if p >= 0 else 0 for p in parents]
        self.rows = rows

    def reserve(self, want):
        """Returns (moves, a row went without); self.room: the tokens that each row may be written up to."""
        ps = self.page
        self.room = [max(w, 0) for w in want]
        for i, w in enumerate(want):
            self.lens[i] = min(self.lens[i], max(w, 0))
            while len(self.rows[i]) * ps >= self.lens[i] + ps:
                self.refs[self.rows[i].pop()] -= 1
        writes = [w > n and n % ps != 0 for n, w in zip(self.lens, want)]
        before = list(self.refs)
        fresh = []
        for i, r in enumerate(self.rows):
            q = r[-1] if writes[i] else None
            if q is None or before[q] < 2:
                fresh.append(False)
                continue
            writers = [j for j, s in enumerate(self.rows) if writes[j] and s[-1] == q]
            fresh.append(not (len(writers) == before[q] and writers[0] == i))
        free, moves, short = [p for p, n in enumerate(before) if n == 0], [], False
        for i, r in enumerate(self.rows):
            need = max(math.ceil(want[i] / ps) - len(r), 0) + fresh[i]
            if need == 0:
                continue
            if short or need > len(free):
                short = True
                self.room[i] = self.lens[i]
                continue
            mine, free = free[:need], free[need:]
            if fresh[i]:
                q = r.pop()
                self.refs[q] -= 1
                moves.append([q, mine[0], self.lens[i] % ps])
            r += mine
            for p in mine:
                self.refs[p] = 1
        return moves, short

    def compact(self, capacity):
        used = sum(1 for n in self.refs if n)
        moves = [[a, b, self.page] for a, b in zip([p for p in range(used, len(self.refs)) if self.refs[p]], [p for p in range(used) if not self.refs[p]])][:capacity]
        to = {a: b for a, b, _ in moves}
        for a, b in to.items():
            self.refs[a], self.refs[b] = 0, self.refs[a]
        self.rows = [[to.get(p, p) for p in r] for r in self.rows]
        return moves


class Device:
    """The same state on the GPU, with guards around every array."""

    def __init__(self, n_pages, page, B, ld, capacity=None):
        self.n_pages, self.page, self.B, self.ld = n_pages, page, B, ld
        self.pool = sps.PagePool(torch.zeros(n_pages, dtype=I32, device=DEV), page)
        self.tables = [self.table(B, ld), self.table(B, ld)]
        self.at, self.reserved = 0, False                      # reserved: the last call, whose room is to be checked
        cap = max(B, n_pages // 2 + 1) if capacity is None else capacity
        self.moves = sps.PageMoves(torch.full((cap, 3), -7, dtype=I32, device=DEV), torch.zeros(1, dtype=I32, device=DEV))
        self.ws = torch.zeros(sps.sps_paged_pool_workspace_bytes(n_pages), dtype=torch.uint8, device=DEV)

    @staticmethod
    def table(B, ld):
        return sps.PageTable(torch.full((B, ld), -9, dtype=I32, device=DEV), torch.zeros(B, dtype=I32, device=DEV), torch.zeros(B, dtype=I32, device=DEV))

    @property
    def t(self):
        return self.tables[self.at]

    def load(self, model):
        """The model's state, entries behind a row's own far out of range."""
        pages = torch.full((self.B, self.ld), 2 ** 31 - 1, dtype=I32)
        for i, r in enumerate(model.rows):
            pages[i, :len(r)] = torch.tensor(r, dtype=I32)
        self.t.pages.copy_(pages)
        self.t.held.copy_(ints([len(r) for r in model.rows]))
        self.t.lens.copy_(ints(model.lens))
        self.pool.refs.copy_(ints(model.refs))

    def fork(self, parents):
        self.reserved = False
        sps.sps_paged_fork(self.pool, self.t, self.tables[1 - self.at], ints(parents))
        self.at = 1 - self.at

    def reserve(self, want):
        self.reserved = True
        self.room = torch.full((self.B,), -4, dtype=I32, device=DEV)
        sps.sps_paged_reserve(self.pool, self.t, ints(want), self.moves, self.ws, room=self.room)

    def compact(self):
        self.reserved = False
        sps.sps_paged_compact(self.pool, self.t, self.t, self.pool.refs, self.moves, self.ws)

    def listed(self):
        return self.moves.list[:int(self.moves.count)].tolist()

    def check(self, model, status=0):
        rows = [r[:h] for r, h in zip(self.t.pages.tolist(), self.t.held.tolist())]
        assert rows == model.rows
        assert self.t.lens.tolist() == model.lens and self.t.held.tolist() == [len(r) for r in model.rows]
        assert self.pool.refs.tolist() == model.refs
        if self.reserved:
            assert self.room.tolist() == model.room
        assert int(self.pool.status) == status
        assert not self.ws[256:256 + 8 * ((self.n_pages + 63) // 64 * 64)].any()   # marks are zero between calls


def consistent(model):
    count = [0] * len(model.refs)
    for r in model.rows:
        for p in r:
            count[p] += 1
    assert count == model.refs


# ---------------------------------------------------------------------------------------------------------------- select
def select64(logits, scores, done, end, N, T):
    """Candidates of one sequence in 64 bits, best first: [(score, beam, token)], and each beam's tolerance.

    A term exp((l - max) / T) is worked out with three roundings of its exponent (difference, log2(e) / T, product), 2^-24 of
    it each, and an exponential within 2^-22: 3 2^-24 |l - max| / T + 2^-22 relative.  Parts have maxima of their own, so the
    same once more for the factor between them.  A lane adds up at most V / 256 + 32 terms, then 5 + 8 partial sums: 2^-24
    each.  The sum's relative error is the log's absolute one."""
    out, tols = [], []
    for w in range(logits.shape[0]):
        s = float(scores[w])
        tols.append(0.0)
        if not math.isfinite(s):
            continue
        if done is not None and int(done[w]):
            out.append((s, w, end))
            continue
        x = logits[w].double() / T
        if torch.isnan(x).any() or float(x.max()) == math.inf or float(x.max()) == -math.inf:
            continue
        below = x - x.max()               # (log sum exp(x) itself would lose log V next to the lowest value of the type: its ulp is 7e22)
        logp = below - torch.log(torch.exp(below).sum())
        c = s + logp
        far = float((torch.exp(logp) * (-below).clamp(max=1e30)).sum())
        tols[-1] = (6 * far + 8 + logits.shape[1] / 256 + 32 + 13 + 1) * 2.0 ** -24
        k = min(N, x.shape[0])
        cut = c.topk(k).values[-1]
        at = ((c >= cut) & (x > -math.inf)).nonzero()[:, 0]
        out += [(v, w, t) for v, t in zip(c[at].tolist(), at.tolist())]
    out.sort(key=lambda e: (-e[0], e[1], e[2]))
    return out, tols


def run_select(logits, scores, done=None, end=-1, N=4, T=1.0, ws=None):
    B, W, V = logits.shape
    o = [torch.full((B, N), 77.0, device=DEV)] + [torch.full((B, N), 77, dtype=I32, device=DEV) for _ in range(3)]
    ws = torch.zeros(sps.sps_beam_select_workspace_bytes(B, W, V), dtype=torch.uint8, device=DEV) if ws is None else ws
    sps.sps_beam_select(logits, scores, *o[:3], ws, done=done, out_done=o[3], end_token=end, temperature=T)
    torch.cuda.synchronize()
    return o


def check_select(o, logits, scores, done=None, end=-1, N=4, T=1.0, exact_ties=False):
    """Whole numbers are the reference's wherever its neighbours in the order are further away than both tolerances."""
    B, W, V = logits.shape
    out_s, out_p, out_t, out_d = [x.tolist() for x in o]
    for b in range(B):
        want, tols = select64(logits[b], scores[b], None if done is None else done[b], end, N, T)
        tol = 2 * max(tols) + 1e-13
        n = min(N, len(want))
        for i in range(N):
            if i >= n:
                assert (out_s[b][i], out_p[b][i], out_t[b][i], out_d[b][i]) == (-math.inf, -1, -1, 0), (b, i)
                continue
            s, w, t = want[i]
            assert abs(out_s[b][i] - s) <= tol + abs(s) * 2.0 ** -24, (b, i, out_s[b][i], s, tol)
            near = not exact_ties and any(0 < abs(want[j][0] - s) <= tol or (j != i and want[j][0] == s and want[j][1] != w)
                                          for j in (i - 1, i + 1) if 0 <= j < len(want))
            if not near:
                assert (out_p[b][i], out_t[b][i]) == (b * W + w, t), (b, i)
            p, t = out_p[b][i] - b * W, out_t[b][i]
            assert out_d[b][i] == int(t == end or (done is not None and int(done[b, p]) != 0))
        found = [(p, t) for p, t in zip(out_p[b][:n], out_t[b][:n])]
        assert len(set(found)) == n
