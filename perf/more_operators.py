"""The operators of this package that decide what a paged cache holds, as cases to measure: the selection of a beam step over
beams and vocabulary, the fork of page tables by parents, the reservation of pages (rollback, copy-on-write, fresh pages), the
compaction of a pool and the copies that these leave to do.

`run` computes an operator in its plain form -- elementary torch operations; scores in 64 bits, since the order of candidates
is decided by their last bits -- or, where `own` is true, through the package's entry points.  `exact` restates each operator
from its definition, scores in 64 bits, page lists element by element.

Select, for beams w of sequence b with scores s and logits l, at temperature T:

    c[b, w, v] = s[b, w] + l[b, w, v] / T - log sum_u exp(l[b, w, u] / T)

the N best (w, v) of each sequence, best first, equal ones in the order of w V + v.  A beam that is done offers one candidate,
(end_token, s); one whose score is -inf offers none.  Parents are rows b W + w.

Pages: refs[p] counts the table rows that hold page p (0: free).  Row r holds entries 0 .. held[r] - 1 of its table row and
has len[r] tokens in them.

    fork      row i of the new table is row parent[i] of the old one; the old rows give their pages up
    reserve   a row keeps the pages of its len tokens and gives up those behind; where it wants room for more, its last page,
              if partly filled and shared, is exchanged for a fresh one and listed to be copied (if all who hold it write to
              it, the first of them keeps it), and fresh pages follow up to `want` tokens: the lowest free ones, row after row
    compact   of U pages in use, those numbered U and above go to the free ones below U, both in ascending order
    copy      the listed (from, to, slots), in every layer's keys and values
"""
from __future__ import annotations

import math

import torch

own = False

F32, BF16, I32 = torch.float32, torch.bfloat16, torch.int32
DT = {"fp32": F32, "bf16": BF16}


# ---------------------------------------------------------------------------------------------------------------- cases
def _select(name, B, W, V, N, dtype, pad, T, live):
    """pad: elements between the end of a row of logits and the next.  live: "all" beams score, only the "first" of each
    sequence does (the step after the prompt), or "some" of them are done."""
    return {"name": name, "op": "select", "B": B, "W": W, "V": V, "N": N, "dtype": dtype, "pad": pad, "T": T, "live": live}


def _step(name, B, W, prompt, made, L, H, d, cache, page, order):
    """The pages' part of a beam step: B sequences of W beams, prompts of up to `prompt` tokens shared by a sequence's beams and
    `made` tokens of each beam's own; fork by parents, room for one more token, copies in L layers."""
    return {"name": name, "op": "step", "B": B, "W": W, "prompt": prompt, "made": made, "L": L, "H": H, "d": d, "cache": cache,
            "page": page, "order": order}


def _reserve(name, B, length, room, turn, page, spare):
    """B sequences of up to `length` tokens that want room for `room` more, back and forth; every turn-th comes and goes
    (0: none does).  spare: free pages, of every 16 in use."""
    return {"name": name, "op": "reserve", "B": B, "length": length, "room": room, "turn": turn, "page": page, "spare": spare}


def _compact(name, B, length, gone, L, H, d, cache, page, order):
    """A pool with room for B sequences of up to `length` tokens, every gone-th of which has left; the rest move together."""
    return {"name": name, "op": "compact", "B": B, "length": length, "gone": gone, "L": L, "H": H, "d": d, "cache": cache,
            "page": page, "order": order}


def _copy(name, n, slots, L, H, d, cache, page, order):
    """n pages of `slots` tokens (0: ragged)."""
    return {"name": name, "op": "copy", "n": n, "slots": slots, "L": L, "H": H, "d": d, "cache": cache, "page": page, "order": order}


def listed():
    return [
        # four beams of one prompt: the smallest step, latency-bound
        _select("select_one_prompt", 1, 4, 32000, 4, "fp32", 0, 1.0, "all"),
        # eight sequences' beams, some of them done, twice as many candidates as beams
        _select("select_batch", 8, 8, 32000, 16, "fp32", 0, 1.0, "some"),
        # a serving batch over a large odd vocabulary, 16-bit logits in padded rows
        _select("select_large_vocab_bf16", 64, 4, 131071, 8, "bf16", 1, 0.7, "all"),
        # wide beams, the largest read
        _select("select_wide", 32, 16, 32000, 32, "fp32", 0, 1.0, "all"),
        # one prompt's four beams on the mid-sized target: 24 layers, 16 heads
        _step("step_one_prompt", 1, 4, 370, 13, 24, 16, 128, "bf16", 16, "head"),
        # eight prompts of eight beams on the same target
        _step("step_batch", 8, 8, 1000, 27, 24, 16, 128, "bf16", 16, "head"),
        # a scoring pass's room and its rollback for a serving batch: bookkeeping alone
        _reserve("reserve_scoring_rows", 64, 8191, 5, 0, 16, 2),
        # many sequences, a quarter of which come and go, in a large pool
        _reserve("reserve_churn", 1024, 4096, 1, 4, 16, 4),
        # a small fp32 pool after a few sequences left
        _compact("compact_small", 6, 300, 3, 2, 4, 64, "fp32", 16, "slot"),
        # a serving pool, a third of it given up; 8 layers of 8 heads (the grouped draft's cache)
        _compact("compact_pool", 96, 2048, 3, 8, 8, 128, "bf16", 32, "head"),
        # the ragged last pages of a few sequences
        _copy("copy_few_ragged", 5, 0, 8, 8, 128, "bf16", 16, "slot"),
        # a long prompt's pages for a reader of its own: as large as copies get
        _copy("copy_prompt", 256, 16, 24, 16, 128, "bf16", 16, "head"),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["select", "select", "select", "step", "reserve", "compact", "copy"])
    if op == "select":
        B, W, V = _log_int(rng, 1, 64), _log_int(rng, 1, 16), _log_int(rng, 64, 131072)
        V = max(64, min(V, 33_000_000 // (B * W)))
        c = _select("", B, W, V, rng.randint(1, min(64, max(1, 2 * W + rng.randint(0, 4)))), rng.choice(["fp32", "bf16"]),
                    rng.choice([0, 0, 1, 3, 8]), rng.choice([1.0, 1.0, 0.7, 1.5]), rng.choice(["all", "some", "first"]))
        del c["name"]
        return c
    H, d, cache = rng.choice([1, 2, 4, 8, 16]), rng.choice([64, 128]), rng.choice(["bf16", "bf16", "fp32"])
    page, L, order = rng.choice([8, 16, 32, 64]), _log_int(rng, 1, 24), rng.choice(["head", "slot"])
    size = L * H * d * page * 2 * (2 if cache == "bf16" else 4)           # bytes of a page in all layers
    most = max(8, 2_000_000_000 // size)                                  # pages of a pool
    if op == "step":
        W, made = rng.randint(2, 12), rng.randint(1, 60)
        B = max(1, min(_log_int(rng, 1, 24), most // (W * (2 + made // page) + 4)))
        prompt = max(1, min(_log_int(rng, 8, 3000), (most // B - W * (2 + made // page) - 2) * page))
        c = _step("", B, W, prompt, made, L, H, d, cache, page, order)
    elif op == "reserve":
        B = _log_int(rng, 1, 1024)
        c = _reserve("", B, _log_int(rng, 1, 8192 if B < 512 else 4096), rng.randint(1, 20), rng.choice([0, 2, 3, 5]), max(page, 16),
                     rng.randint(1, 8))
    elif op == "compact":
        B = _log_int(rng, 2, 96)
        c = _compact("", B, max(1, min(_log_int(rng, 8, 2048), (most // B - 1) * page)), rng.choice([2, 3, 5]), L, H, d, cache, page, order)
        while B > 2 and B * (-(-c["length"] // page)) > most:
            B = c["B"] = B // 2
    else:
        c = _copy("", max(1, min(_log_int(rng, 1, 512), most // 3)), rng.choice([0, page, rng.randint(1, page)]), L, H, d, cache, page, order)
    del c["name"]
    return c


# --------------------------------------------------------------------------------------------------------------- inputs
def _spread(n, lo, hi):
    """n whole numbers spread evenly over lo .. hi in a scattered order, the first of them hi: the same for every seed (the work
    of a case is fixed, its numbers are not)."""
    return [hi] + [lo + int((hi - lo) * ((0.61803398875 * (i + 1)) % 1.0)) for i in range(1, n)]


def _parents(B, W):
    """Parents of a step: low beams have several children, some beams none."""
    return [b * W + min(W - 1, int(W * ((0.7548776662 * (i + 1) + 0.3 * b) % 1.0) ** 2)) for b in range(B) for i in range(W)]


def _lens(case):
    if case["op"] == "step":
        return [p + case["made"] for p in _spread(case["B"], max(1, case["prompt"] // 4), case["prompt"])]
    return _spread(case["B"], max(1, case["length"] // 8), case["length"])


def _slots(case):
    return [case["slots"]] * case["n"] if case["slots"] else [max(1, s) for s in _spread(case["n"], 1, case["page"] - 1)]


def _caches(case, n_pages, gd):
    shape = (case["L"], n_pages, case["H"], case["page"], case["d"])
    if case["order"] == "slot":
        shape = (shape[0], shape[1], shape[3], shape[2], shape[4])
    out = []
    for _ in "kv":
        t = torch.empty(shape, dtype=DT[case["cache"]], device="cuda")
        t.normal_(generator=gd)
        out.append(t if case["order"] == "head" else t.transpose(2, 3))
    return out


def _dev(x):
    return torch.tensor(x, dtype=I32).to("cuda")


def prepare(case, seed):
    op = case["op"]
    g = torch.Generator().manual_seed(seed * 2 + 1)
    gd = torch.Generator(device="cuda").manual_seed(seed * 2 + 1)
    s = {"case": case}
    if op == "select":
        B, W, V, N = case["B"], case["W"], case["V"], case["N"]
        rows = torch.empty((B, W, V + case["pad"]), device="cuda").normal_(0.0, 3.0, generator=gd).to(DT[case["dtype"]])
        s["logits"] = rows[:, :, :V]
        scores = -(torch.rand((B, W), generator=g) * 20.0 + 2.0)
        if case["live"] == "first":
            scores[:, 0] = 0.0
            scores[:, 1:] = float("-inf")
        done = torch.zeros((B, W), dtype=I32)
        if case["live"] == "some":
            done = (torch.rand((B, W), generator=g) < 0.3).to(I32)
            scores = torch.where(done.bool(), scores * 0.25, scores)        # what has ended is ahead of what goes on
        s["scores"], s["done"], s["end"] = scores.cuda(), done.cuda(), min(2, V - 1)
        s["out_scores"] = torch.empty((B, N), device="cuda")
        s["out_parents"], s["out_tokens"], s["out_done"] = (torch.empty((B, N), dtype=I32, device="cuda") for _ in range(3))
        if own:
            import paper_2302_01318_b200 as sps
            s["ws"] = torch.zeros(sps.sps_beam_select_workspace_bytes(B, W, V), dtype=torch.uint8, device="cuda")
        return s

    ps = case["page"]
    if op == "copy":
        n_pages = 3 * case["n"]
        perm = torch.randperm(n_pages, generator=g).tolist()
        moves = [[perm[i], perm[case["n"] + i], m] for i, m in enumerate(_slots(case))]
        s["k"], s["v"] = _caches(case, n_pages, gd)
        s["moves"], s["count"] = _dev(moves), _dev([len(moves)])
    elif op == "step":
        B, W = case["B"], case["W"]
        lens = _lens(case)
        rows, full = B * W, [(n - case["made"]) // ps for n in lens]        # pages that a prompt fills
        own_pages = [-(-n // ps) - f for n, f in zip(lens, full)]
        used = sum(full) + W * sum(own_pages)
        n_pages = used + rows * 2 + 1
        perm, at = torch.randperm(n_pages, generator=g).tolist(), 0
        ld = max(-(-(n + 1) // ps) for n in lens)
        table = torch.zeros((rows, ld), dtype=I32)
        refs = torch.zeros(n_pages, dtype=I32)
        for b in range(B):
            shared = perm[at:at + full[b]]
            at += full[b]
            refs[shared] = W
            for w in range(W):
                mine = perm[at:at + own_pages[b]]
                at += own_pages[b]
                refs[mine] = 1
                table[b * W + w, :len(shared) + len(mine)] = torch.tensor(shared + mine, dtype=I32)
        s["refs"] = refs.cuda()
        held, row_len = [x for n in lens for x in [-(-n // ps)] * W], [n for n in lens for _ in range(W)]
        s["tables"] = [{"pages": table.cuda(), "held": _dev(held), "len": _dev(row_len)},
                       {"pages": torch.zeros_like(table).cuda(), "held": _dev([0] * rows), "len": _dev([0] * rows)}]
        s["flip"], s["parents"], s["want"] = 0, _dev(_parents(B, W)), _dev([n + 1 for n in row_len])
        s["moves"], s["count"] = _dev([[0, 0, 0]] * rows), _dev([0])
        s["k"], s["v"] = _caches(case, n_pages, gd)
    else:
        B, lens = case["B"], _lens(case)
        if op == "reserve":
            need = [-(-(n + case["room"]) // ps) for n in lens]
            turn = case["turn"]
            comes = [turn > 0 and b % turn == 1 for b in range(B)]          # these are away at the start
            goes = [turn > 0 and b % turn == 0 for b in range(B)]           # these leave first
            have = [0 if c else -(-n // ps) for n, c in zip(lens, comes)]
            n_pages = sum(need) + sum(need) * case["spare"] // 16 + 1
            s["want"] = [_dev([0 if x else n + case["room"] for x, n in zip(goes, lens)]),
                         _dev([0 if x else n for x, n in zip(comes, lens)])]
            s["flip"] = 0
            start = [0 if c else n for n, c in zip(lens, comes)]
        else:
            need = [-(-n // ps) for n in lens]
            have = [0 if b % case["gone"] == case["gone"] - 1 else k for b, k in enumerate(need)]
            n_pages = sum(need)
            start = [n if k else 0 for n, k in zip(lens, have)]
        perm, at = torch.randperm(n_pages, generator=g).tolist(), 0
        table, refs = torch.zeros((B, max(need)), dtype=I32), torch.zeros(n_pages, dtype=I32)
        for b, k in enumerate(have):
            table[b, :k] = torch.tensor(perm[at:at + k], dtype=I32)
            refs[perm[at:at + k]] = 1
            at += k
        s["refs"] = refs.cuda()
        s["table"] = {"pages": table.cuda(), "held": _dev(have), "len": _dev(start)}
        s["moves"], s["count"] = _dev([[0, 0, 0]] * (B if op == "reserve" else n_pages // 2 + 1)), _dev([0])
        if op == "compact":
            s["out"] = {"pages": torch.zeros_like(table).cuda(), "held": _dev([0] * B), "len": _dev([0] * B)}
            s["refs_out"] = torch.zeros_like(s["refs"])
            s["k"], s["v"] = _caches(case, n_pages, gd)
    if own:
        import paper_2302_01318_b200 as sps
        s["c_moves"] = sps.PageMoves(s["moves"], s["count"])
        if "k" in s:
            s["c_layers"] = sps.PagedLayers([sps.PagedCache(k, v) for k, v in zip(s["k"], s["v"])])
        if op != "copy":
            s["c_pool"] = sps.PagePool(s["refs"], ps)
            s["c_tables"] = [sps.PageTable(t["pages"], t["held"], t["len"])
                             for t in (s["tables"] if op == "step" else [s["table"]] + ([s["out"]] if op == "compact" else []))]
            s["ws"] = torch.zeros(sps.sps_paged_pool_workspace_bytes(s["refs"].numel()), dtype=torch.uint8, device="cuda")
    return s


# ----------------------------------------------------------------------------------------------------------- plain forms
def _plain_select(s):
    c = s["case"]
    B, W, V, N = c["B"], c["W"], c["V"], c["N"]
    x = s["logits"].double() / c["T"]
    m = x.amax(-1, keepdim=True)
    base = s["scores"].double() - m[..., 0] - (x - m).exp().sum(-1).log()
    x += base[..., None]
    x[s["done"].bool()] = float("-inf")
    x[..., s["end"]] = torch.where(s["done"].bool(), s["scores"].double(), x[..., s["end"]])
    x = x.view(B, W * V)
    if W * V < N:
        x = torch.cat((x, torch.full((B, N - W * V), float("-inf"), dtype=x.dtype, device=x.device)), 1)
    best, at = torch.sort(x, dim=1, descending=True, stable=True)
    best, at = best[:, :N], at[:, :N]
    there = best > float("-inf")
    parent = at // V + (torch.arange(B, device=at.device) * W)[:, None]
    token = at % V
    over = there & ((s["done"].view(-1)[parent.clamp(max=B * W - 1)] != 0) | (token == s["end"]))
    s["out_scores"].copy_(best)
    s["out_parents"].copy_(torch.where(there, parent, -1))
    s["out_tokens"].copy_(torch.where(there, token, -1))
    s["out_done"].copy_(over)
    return s["out_scores"], s["out_parents"], s["out_tokens"], s["out_done"]


def _plain_fork(refs, src, dst, parents):
    rows, ld = src["pages"].shape
    at = torch.arange(ld, device=refs.device)
    p = parents.long()
    children = torch.zeros(rows, dtype=I32, device=refs.device).index_add_(0, p, torch.ones_like(parents))
    change = torch.where(at[None] < src["held"][:, None], (children - 1)[:, None], 0)
    refs.index_add_(0, src["pages"].reshape(-1).long(), change.reshape(-1))
    dst["held"].copy_(src["held"][p])
    dst["len"].copy_(src["len"][p])
    dst["pages"].copy_(torch.where(at[None] < dst["held"][:, None], src["pages"][p], dst["pages"]))


def _plain_reserve(refs, table, want, ps, moves, count):
    pages, held = table["pages"], table["held"]
    rows, ld = pages.shape
    at = torch.arange(ld, device=refs.device)
    n = torch.minimum(table["len"], want)
    keep = (n + ps - 1) // ps
    behind = (at[None] >= keep[:, None]) & (at[None] < held[:, None])
    refs.index_add_(0, pages.reshape(-1).long(), -behind.reshape(-1).to(I32))
    # the partly filled last page of a row that goes on
    row = torch.arange(rows, device=refs.device)
    last = pages[row, (keep - 1).clamp(min=0).long()].long()
    writes = (want > n) & (n % ps != 0)
    writers = torch.zeros_like(refs).index_add_(0, last, writes.to(I32))
    first = torch.full_like(refs, rows).scatter_reduce_(0, last, torch.where(writes, row, rows).to(I32), "amin")
    fresh = writes & (refs[last] > 1) & ~((writers[last] == refs[last]) & (first[last] == row))
    need = (want + ps - 1) // ps - keep + fresh
    end = need.cumsum(0)
    free = torch.argsort((refs != 0).to(I32), stable=True)                    # free pages first, ascending
    served = (need > 0) & (end <= (refs == 0).sum())
    start, fresh = end - need, fresh & served
    new_held = torch.where(served, (want + ps - 1) // ps, keep)
    lo = keep - fresh.to(keep.dtype)
    mine = (at[None] >= lo[:, None]) & (at[None] < new_held[:, None])
    page = free[(start[:, None] + at[None] - lo[:, None]).clamp(0, refs.numel() - 1)].to(I32)
    refs.index_add_(0, last, -fresh.to(I32))
    refs.index_add_(0, torch.where(mine, page, 0).reshape(-1).long(), mine.reshape(-1).to(I32))
    pages.copy_(torch.where(mine, page, pages))
    held.copy_(new_held)
    table["len"].copy_(n)
    place = torch.where(fresh, fresh.cumsum(0) - 1, moves.shape[0])
    item = torch.stack((last.to(I32), pages[row, (keep - 1).clamp(min=0).long()], (n % ps).to(I32)), 1)
    moves.copy_(torch.cat((moves, moves[:1])).index_copy_(0, place[fresh], item[fresh])[:-1])
    count.copy_(fresh.sum())


def _plain_compact(refs, src, dst, refs_out, ps, moves, count):
    n = refs.numel()
    used = refs != 0
    total = used.sum()
    p = torch.arange(n, device=refs.device)
    goes, hole = used & (p >= total), ~used & (p < total)
    rank = torch.where(hole, hole.cumsum(0) - 1, n)
    to = torch.zeros(n + 1, dtype=torch.int64, device=refs.device).index_copy_(0, rank, p)    # the rank-th hole (entry n: the rest)
    new = torch.where(goes, to[(goes.cumsum(0) - 1).clamp(min=0)], p)
    refs_out.zero_().index_add_(0, new, refs)
    rows, ld = src["pages"].shape
    inside = torch.arange(ld, device=refs.device)[None] < src["held"][:, None]
    dst["pages"].copy_(torch.where(inside, new[src["pages"].long()].to(I32), dst["pages"]))
    dst["held"].copy_(src["held"])
    dst["len"].copy_(src["len"])
    item = torch.stack((p[goes], new[goes], torch.full_like(p[goes], ps)), 1).to(I32)
    moves[:item.shape[0]] = item
    count.fill_(item.shape[0])


def _plain_copy(k, v, moves, count):
    m = moves[:int(count)].long()
    ps = k.shape[3]
    copied = (torch.arange(ps, device=k.device)[None] < m[:, 2:]).view(1, -1, 1, ps, 1)
    for t in (k, v):
        t[:, m[:, 1]] = torch.where(copied, t[:, m[:, 0]], t[:, m[:, 1]])


def run(s):
    c = s["case"]
    op = c["op"]
    if op == "select":
        if not own:
            return _plain_select(s)
        import paper_2302_01318_b200 as sps
        sps.sps_beam_select(s["logits"], s["scores"], s["out_scores"], s["out_parents"], s["out_tokens"], s["ws"], done=s["done"],
                            out_done=s["out_done"], end_token=s["end"], temperature=c["T"])
        return s["out_scores"], s["out_parents"], s["out_tokens"], s["out_done"]
    if op == "copy":
        if own:
            import paper_2302_01318_b200 as sps
            sps.sps_paged_copy(s["c_layers"], s["c_moves"])
        else:
            _plain_copy(s["k"], s["v"], s["moves"], s["count"])
        return s["k"], s["v"]
    if op == "step":
        a = s["flip"]
        s["flip"] = 1 - a
        src, dst = s["tables"][a], s["tables"][1 - a]
        if own:
            import paper_2302_01318_b200 as sps
            sps.sps_paged_fork(s["c_pool"], s["c_tables"][a], s["c_tables"][1 - a], s["parents"])
            sps.sps_paged_reserve(s["c_pool"], s["c_tables"][1 - a], s["want"], s["c_moves"], s["ws"])
            sps.sps_paged_copy(s["c_layers"], s["c_moves"])
        else:
            _plain_fork(s["refs"], src, dst, s["parents"])
            _plain_reserve(s["refs"], dst, s["want"], c["page"], s["moves"], s["count"])
            _plain_copy(s["k"], s["v"], s["moves"], s["count"])
        return dst["pages"], dst["held"], dst["len"], s["refs"], s["moves"], s["count"], s["k"], s["v"]
    if op == "reserve":
        want = s["want"][s["flip"]]
        s["flip"] = 1 - s["flip"]
        t = s["table"]
        if own:
            import paper_2302_01318_b200 as sps
            sps.sps_paged_reserve(s["c_pool"], s["c_tables"][0], want, s["c_moves"], s["ws"])
        else:
            _plain_reserve(s["refs"], t, want, c["page"], s["moves"], s["count"])
        return t["pages"], t["held"], t["len"], s["refs"], s["count"]
    if own:
        import paper_2302_01318_b200 as sps
        sps.sps_paged_compact(s["c_pool"], s["c_tables"][0], s["c_tables"][1], s["refs_out"], s["c_moves"], s["ws"])
        sps.sps_paged_copy(s["c_layers"], s["c_moves"])
    else:
        _plain_compact(s["refs"], s["table"], s["out"], s["refs_out"], c["page"], s["moves"], s["count"])
        _plain_copy(s["k"], s["v"], s["moves"], s["count"])
    o = s["out"]
    return o["pages"], o["held"], o["len"], s["refs_out"], s["moves"], s["count"], s["k"], s["v"]


# ----------------------------------------------------------------------------------------------------------------- work
def _slot_bytes(case):
    return case["L"] * 2 * case["H"] * case["d"] * (2 if case["cache"] == "bf16" else 4)


def work(case):
    op = case["op"]
    if op == "select":
        B, W, V, N = case["B"], case["W"], case["V"], case["N"]
        live = {"all": 1.0, "some": 0.7, "first": 1.0 / W}[case["live"]]      # a beam that is done or dead has no logits to read
        size = 4 if case["dtype"] == "fp32" else 2
        return {"bytes": int(B * W * live) * V * size + 4 * (2 * B * W + 4 * B * N), "flops": 4 * int(B * W * live) * V}
    ps = case["page"]
    if op == "copy":
        n = sum(_slots(case)) * _slot_bytes(case)
        return {"bytes": 2 * n + 12 * case["n"], "flops": 0}
    lens = _lens(case)
    if op == "step":
        B, W, parents = case["B"], case["W"], _parents(case["B"], case["W"])
        held, slots = sum(-(-n // ps) for n in lens) * W, 0
        for b, n in enumerate(lens):                                          # every child but one of a parent copies its last page
            slots += (W - len(set(parents[b * W:(b + 1) * W]))) * (n % ps)
        return {"bytes": 2 * slots * _slot_bytes(case) + 2 * 4 * held + 8 * B * W * 3, "flops": 0}
    if op == "reserve":
        pages = sum(-(-(n + case["room"]) // ps) for n in lens)
        pool = pages + pages * case["spare"] // 16 + 1
        turn = case["turn"]
        moved = sum(-(-n // ps) for b, n in enumerate(lens) if turn and b % turn < 2)
        return {"bytes": 4 * pool + 3 * 4 * moved + 4 * 5 * case["B"], "flops": 0}
    need = [-(-n // ps) for n in lens]
    left = [k for b, k in enumerate(need) if b % case["gone"] != case["gone"] - 1]
    moved = (sum(need) - sum(left)) * sum(left) // sum(need)                  # what lies above, the pool being scattered
    return {"bytes": 2 * moved * ps * _slot_bytes(case) + 2 * 4 * sum(need) + 2 * 4 * sum(left) + 12 * moved, "flops": 0}


# ---------------------------------------------------------------------------------------------------------------- exact
def _exact_select(s):
    c = s["case"]
    B, W, V, N = c["B"], c["W"], c["V"], c["N"]
    out = [torch.full((B, N), float("-inf"), dtype=torch.float64)] + [torch.full((B, N), x, dtype=torch.int64) for x in (-1, -1, 0)]
    scores, done = s["scores"].double().cpu(), s["done"].cpu()
    for b in range(B):
        found = []
        for w in range(W):
            if scores[b, w] == float("-inf"):
                continue
            if done[b, w]:
                found.append((-scores[b, w].item(), w, s["end"], 1))
                continue
            p = torch.log_softmax(s["logits"][b, w].double() / c["T"], 0)
            cut = p.topk(min(N, V)).values[-1]
            at = (p >= cut).nonzero()[:, 0]
            val = (p[at] + scores[b, w].item()).cpu().tolist()
            found += [(-x, w, v, int(v == s["end"])) for x, v in zip(val, at.cpu().tolist())]
        for i, (x, w, v, d) in enumerate(sorted(found)[:N]):
            out[0][b, i], out[1][b, i], out[2][b, i], out[3][b, i] = -x, b * W + w, v, d
    return tuple(t.cuda() for t in out)


def _exact_reserve(refs, rows, lens, want, ps):
    """refs: list, rows: list of page lists; both changed.  Returns (moves, lens)."""
    lens = [min(n, w) for n, w in zip(lens, want)]
    for r, n in zip(rows, lens):
        while len(r) > -(-n // ps):
            refs[r.pop()] -= 1
    writers = {}
    for i, (r, n, w) in enumerate(zip(rows, lens, want)):
        if w > n and n % ps:
            writers.setdefault(r[-1], []).append(i)
    fresh = set()
    for p, who in writers.items():
        if refs[p] > 1:
            fresh.update(who[1:] if len(who) == refs[p] else who)
    free = [p for p, x in enumerate(refs) if x == 0]
    at, dry, moves = 0, False, []
    for i, (r, n, w) in enumerate(zip(rows, lens, want)):
        need = -(-w // ps) - len(r) + (i in fresh)
        if need <= 0 or dry:
            continue
        if at + need > len(free):
            dry = True
            continue
        got = free[at:at + need]
        at += need
        if i in fresh:
            moves.append([r[-1], got[0], n % ps])
            refs[r[-1]] -= 1
            r.pop()
        r += got
        for p in got:
            refs[p] += 1
    return moves, lens


def _exact_copied(t, moves):
    t = t.clone()
    for a, b, n in moves:
        t[:, b, :, :n] = t[:, a, :, :n]
    return t


def _rows_of(table):
    pages = table["pages"].tolist()
    return [r[:h] for r, h in zip(pages, table["held"].tolist())]


def _table_like(before, rows):
    out = before.clone()
    for i, r in enumerate(rows):
        out[i, :len(r)] = torch.tensor(r, dtype=I32)
    return out


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "select":
        return _exact_select(s)
    if op == "copy":
        return tuple(_exact_copied(t, s["moves"].tolist()) for t in (s["k"], s["v"]))
    ps, refs = case["page"], s["refs"].tolist()
    if op == "step":
        old, lens, parents = _rows_of(s["tables"][0]), s["tables"][0]["len"].tolist(), s["parents"].tolist()
        for r in old:
            for p in r:
                refs[p] -= 1
        rows = [list(old[p]) for p in parents]
        for r in rows:
            for p in r:
                refs[p] += 1
        stale = _table_like(s["tables"][1]["pages"], rows)
        moves, lens = _exact_reserve(refs, rows, [lens[p] for p in parents], s["want"].tolist(), ps)
        listed_moves = s["moves"].clone()
        if moves:
            listed_moves[:len(moves)] = _dev(moves)
        return (_table_like(stale, rows), _dev([len(r) for r in rows]), _dev(lens), _dev(refs), listed_moves, _dev([len(moves)]),
                _exact_copied(s["k"], moves), _exact_copied(s["v"], moves))
    t = s["table"]
    rows, lens = _rows_of(t), t["len"].tolist()
    if op == "reserve":
        moves, lens = _exact_reserve(refs, rows, lens, s["want"][0].tolist(), ps)
        return _table_like(t["pages"], rows), _dev([len(r) for r in rows]), _dev(lens), _dev(refs), _dev([len(moves)])
    used = sum(x != 0 for x in refs)
    holes = [p for p in range(used) if refs[p] == 0]
    moves = [[p, q, ps] for p, q in zip((p for p in range(used, len(refs)) if refs[p] != 0), holes)]
    to = {a: b for a, b, _ in moves}
    for a, b, _ in moves:
        refs[b], refs[a] = refs[a], 0
    rows = [[to.get(p, p) for p in r] for r in rows]
    listed_moves = s["moves"].clone()
    if moves:
        listed_moves[:len(moves)] = _dev(moves)
    return (_table_like(s["out"]["pages"], rows), _dev([len(r) for r in rows]), _dev(lens), _dev(refs), listed_moves, _dev([len(moves)]),
            _exact_copied(s["k"], moves), _exact_copied(s["v"], moves))
