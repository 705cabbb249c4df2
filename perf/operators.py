"""The paged serving operators of this package, as cases to measure: rotary positions of given rows, the append of new
keys and values to a paged cache (rotated on the way, the queries with them), and the attention of every sequence's new
rows over its pages.

`run` computes an operator in its plain form -- elementary torch operations in 32 bits, angles in 64 -- or, where `own`
is true, through the package's entry points.  `exact` restates each operator from its definition in 64 bits.

Formulas, for a row at position p, frequencies f_i (64 bits) and gain g, over the first `rot` elements of a head:

    pair (x_a, x_b) -> g (x_a cos(p f_i) - x_b sin(p f_i),  x_a sin(p f_i) + x_b cos(p f_i))
    "pairs" layout: (a, b) = (2 i, 2 i + 1);   "halves" layout: (a, b) = (i, i + rot / 2)

Sequence b owns the rows q_start[b] .. q_start[b + 1] - 1 of q / k / v and has kv_len[b] tokens, its new rows included;
the last row is at position kv_len[b] - 1.  Token j of it lies in page pages[b][j / page_size], slot j % page_size.

    out[row, h] = sum_{j <= p} softmax_j(scale q[row, h] . K[j, h / G]) V[j, h / G],   G = query heads / key heads
"""
from __future__ import annotations

import math

import torch

own = False

F32, BF16 = torch.float32, torch.bfloat16
DT = {"fp32": F32, "bf16": BF16}


# ---------------------------------------------------------------------------------------------------------------- cases
def _rotary(name, rows, heads, d_head, rot, layout, dtype, far, bands, transposed):
    """bands: frequencies stretched by bands (factor 8 over a trained length of 4096), else the plain ones."""
    return {"name": name, "op": "rotary", "rows": rows, "heads": heads, "d_head": d_head, "rot": rot, "layout": layout,
            "dtype": dtype, "far": far, "bands": bands, "transposed": transposed}


def _append(name, B, new, old, H, Hkv, d_head, rot, layout, act, qdt, cache, page, packed):
    """new / old: the largest number of new rows / of older tokens; ragged below that when B > 1.
    packed: q | k | v are slices of one buffer (what a fused projection leaves), else tensors of their own."""
    return {"name": name, "op": "append", "B": B, "new": new, "old": old, "H": H, "Hkv": Hkv, "d_head": d_head, "rot": rot,
            "layout": layout, "act": act, "q_out": qdt, "cache": cache, "page": page, "packed": packed}


def _attn(name, B, new, old, H, Hkv, d_head, act, cache, page, shape):
    """shape: how lengths are spread.  "same": every sequence has `new` new rows over `old` older tokens; "ragged": older
    tokens log-uniform in 1 .. old; "mixed": the first sequence brings `new` rows over `old` older tokens, the others one row
    each over ragged lengths."""
    return {"name": name, "op": "attention", "B": B, "new": new, "old": old, "H": H, "Hkv": Hkv, "d_head": d_head, "act": act,
            "cache": cache, "page": page, "shape": shape}


def listed():
    return [
        # the K + 1 = 5 rows of one scoring pass of the large grouped-query pair: queries and keys, latency-bound
        _rotary("rotary_verify_rows", 5, 72, 128, 128, "pairs", "fp32", 4096, False, False),
        # a long prompt's rows in 16 bits, half layout, positions far beyond the trained length
        _rotary("rotary_prompt_bf16", 8190, 40, 128, 128, "halves", "bf16", 131072, True, False),
        # part of a small head, an odd number of rows, the transposed rotation (its gradient, or un-rotating keys)
        _rotary("rotary_partial_transposed", 4095, 6, 64, 32, "halves", "fp32", 8192, False, True),
        # one scoring pass of eight sequences: 5 new rows each, 8 key heads, fp32 projections into a bf16 cache
        _append("append_verify_rows", 8, 5, 4000, 64, 8, 128, 128, "pairs", "fp32", "fp32", "bf16", 16, True),
        # a prompt chunk of the draft shape (48 heads): fp32 projections, queries handed on in 16 bits
        _append("append_prompt_chunk", 1, 4096, 1000, 48, 48, 128, 128, "pairs", "fp32", "bf16", "bf16", 64, True),
        # one token of the mid-sized target (16 heads) late in its generation: the smallest call
        _attn("decode_mid", 1, 1, 383, 16, 16, 128, "fp32", "bf16", 16, "same"),
        # eight sequences' scoring pass, 64 query heads on 8 key heads, ragged contexts
        _attn("verify_gqa_ragged", 8, 5, 4096, 64, 8, 128, "fp32", "bf16", 16, "ragged"),
        # one scoring pass over a long context, a key head per query head: the largest read
        _attn("verify_long", 1, 5, 32763, 64, 64, 128, "fp32", "bf16", 64, "same"),
        # a serving batch, one token each, contexts from one token to thousands, 16-bit activations
        _attn("decode_ragged_bf16", 64, 1, 8191, 64, 8, 128, "bf16", "bf16", 32, "ragged"),
        # a prompt chunk over its own earlier chunks: bound by the tensor cores
        _attn("chunk_bf16", 1, 2048, 6144, 64, 8, 128, "bf16", "bf16", 64, "same"),
        # a prompt chunk of fp32 activations beside one-token rows of other sequences
        _attn("mixed_fp32", 12, 333, 2047, 32, 8, 64, "fp32", "bf16", 32, "mixed"),
        # the fp32 pairs (fp32 cache): scoring passes of eight sequences, grouped heads
        _attn("verify_fp32_cache", 8, 5, 1195, 4, 2, 64, "fp32", "fp32", 16, "ragged"),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["rotary", "append", "attention", "attention"])
    d_head = rng.choice([64, 128])
    layout = rng.choice(["pairs", "halves"])
    rot = rng.choice([d_head, d_head, d_head // 2, d_head // 4])
    if op == "rotary":
        rows, heads = _log_int(rng, 1, 8192), rng.randint(1, 72)
        rows = max(1, min(rows, 42_000_000 // (heads * d_head)))
        c = _rotary("", rows, heads, d_head, rot, layout, rng.choice(["fp32", "bf16"]), _log_int(rng, 4, 200000),
                    rng.random() < 0.5, rng.random() < 0.3)
    else:
        Hkv = rng.choice([1, 2, 4, 8, 16])
        H = Hkv * rng.choice([1, 2, 4, 8])
        page = rng.choice([8, 16, 32, 64, 128])
        act, cache = rng.choice([("fp32", "bf16"), ("bf16", "bf16"), ("fp32", "bf16"), ("bf16", "bf16"), ("fp32", "fp32")])
        B = _log_int(rng, 1, 48)
        if op == "append":
            new = _log_int(rng, 1, max(1, min(2048, 16_000_000 // (B * (H + 2 * Hkv) * d_head))))
            c = _append("", B, new, _log_int(rng, 1, 4096), H, Hkv, d_head, rot, layout, act,
                        "fp32" if act == "fp32" and rng.random() < 0.5 else "bf16", cache, page, rng.random() < 0.5)
        else:
            shape = rng.choice(["same", "ragged", "mixed"])
            new = _log_int(rng, 1, 16) if shape != "mixed" else _log_int(rng, 16, 600)
            if B == 1 and rng.random() < 0.5:
                new = _log_int(rng, 16, 1500)
            old = _log_int(rng, 1, 12000 if new <= 16 else 6000)
            if cache == "fp32":                       # fp32 pairs are small ones
                H, Hkv, B, new, old = min(H, 4 * min(Hkv, 4)), min(Hkv, 4), min(B, 8), min(new, 128), min(old, 2000)
            B = max(1, min(B, 250_000_000 // ((old + new) * Hkv * d_head), 500_000_000 // ((old + new) * H * new)))
            c = _attn("", B, new, old, H, Hkv, d_head, act, cache, page, shape)
    del c["name"]
    return c


# --------------------------------------------------------------------------------------------------------------- inputs
def _frequencies(rot, bands, device):
    """base 10000; by bands: a pair that turns r times within the trained length of 4096 keeps its frequency above
    r = 32, has it divided by 8 below r = 1, and a linear blend between; gain 0.1 ln 8 + 1."""
    f = 10000.0 ** (-2.0 * torch.arange(rot // 2, dtype=torch.float64) / rot)
    gain = 1.0
    if bands:
        turns = 4096 * f / (2.0 * math.pi)
        keep = ((turns - 1.0) / (32.0 - 1.0)).clamp(0.0, 1.0)
        f = keep * f + (1.0 - keep) * f / 8.0
        gain = 0.1 * math.log(8.0) + 1.0
    return f.to(device), gain


def _lengths(case):
    """(new rows, tokens) of every sequence, as lists: spread evenly over their ranges in a scattered order, the same
    for every seed (the work of a case is fixed; its numbers are not)."""
    B, new, old = case["B"], case["new"], case["old"]
    u = [(0.61803398875 * (b + 1)) % 1.0 for b in range(B)]
    if case["op"] == "append":
        n = [new] + [max(1, int(round(new * x))) for x in u[1:]]
        o = [old] + [int(old * (1.0 - x)) for x in u[1:]]
    elif case["shape"] == "same":
        n, o = [new] * B, [old] * B
    else:
        o = [old] + [max(1, int(round(old ** x))) for x in u[1:]]
        n = [new] * B if case["shape"] == "ragged" else [new] + [1] * (B - 1)
    return n, [a + b for a, b in zip(n, o)]


def prepare(case, seed):
    dev = "cuda"
    g = torch.Generator().manual_seed(seed * 2 + 1)
    gd = torch.Generator(device=dev).manual_seed(seed * 2 + 1)

    def normal(shape, dtype, std=1.0):
        return (torch.randn(shape, generator=gd, device=dev) * std).to(dtype)

    if case["op"] == "rotary":
        rows, heads, d = case["rows"], case["heads"], case["d_head"]
        x = normal((rows, heads, d), DT[case["dtype"]])
        pos = torch.randint(0, case["far"] + 1, (rows,), generator=g).to(torch.int32).to(dev)
        freq, gain = _frequencies(case["rot"], case["bands"], dev)
        s = {"case": case, "x": x, "y": torch.zeros_like(x), "pos": pos, "freq": freq, "gain": gain}
        if own:
            import paper_2302_01318_b200 as sps
            s["rope"] = sps.Rotary(freq, layout=case["layout"], gain=gain)
        return s

    B, H, Hkv, d, ps = case["B"], case["H"], case["Hkv"], case["d_head"], case["page"]
    n, L = _lengths(case)
    q_start = torch.tensor([0] + n, dtype=torch.int64).cumsum(0).to(torch.int32)
    rows = int(q_start[-1])
    need = [-(-x // ps) for x in L]
    n_pages = sum(need) + 3
    table = torch.zeros((B, max(need)), dtype=torch.int32)
    perm, at = torch.randperm(n_pages, generator=g).to(torch.int32), 0
    for b in range(B):
        table[b, :need[b]] = perm[at:at + need[b]]
        at += need[b]
    act, cdt = DT[case["act"]], DT[case["cache"]]
    s = {"case": case, "q_start": q_start.to(dev), "kv_len": torch.tensor(L, dtype=torch.int32).to(dev), "pages": table.to(dev),
         "rows": rows, "max_q": max(n), "max_len": max(L),
         "kp": normal((n_pages, Hkv, ps, d), cdt), "vp": normal((n_pages, Hkv, ps, d), cdt)}
    if case["op"] == "append":
        if case["packed"]:
            qkv = normal((rows, H + 2 * Hkv, d), act)
            s["q"], s["k"], s["v"] = qkv[:, :H], qkv[:, H:H + Hkv], qkv[:, H + Hkv:]
        else:
            s["q"], s["k"], s["v"] = normal((rows, H, d), act), normal((rows, Hkv, d), act), normal((rows, Hkv, d), act)
        s["freq"], s["gain"] = _frequencies(case["rot"], False, dev)
        s["q_rot"] = torch.zeros((rows, H, d), dtype=DT[case["q_out"]], device=dev)
    else:
        s["q"] = normal((rows, H, d), act, 1.5)
        s["out"] = torch.zeros((rows, H, d), dtype=act, device=dev)
    if own:
        import paper_2302_01318_b200 as sps
        s["cache"] = sps.PagedCache(s["kp"], s["vp"])
        s["batch"] = sps.PagedBatch(s["q_start"], s["kv_len"], s["pages"], max_q=s["max_q"])
        if case["op"] == "append":
            s["rope"] = sps.Rotary(s["freq"], layout=case["layout"], gain=s["gain"])
        else:
            s["ws"] = torch.zeros(sps.sps_paged_attention_workspace_bytes(s["cache"], H, act), dtype=torch.uint8, device=dev)
    return s


# ----------------------------------------------------------------------------------------------------------- plain forms
def _rotate(x, angle, rot, layout, gain, transposed):
    """x [rows, heads, d] fp32, angle [rows, rot / 2] fp64."""
    c = (angle.cos() * gain).float()[:, None, :]
    s = (angle.sin() * (-gain if transposed else gain)).float()[:, None, :]
    y = x.clone()
    if layout == "pairs":
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
        y[..., 0:rot:2], y[..., 1:rot:2] = a * c - b * s, a * s + b * c
    else:
        a, b = x[..., :rot // 2], x[..., rot // 2:rot]
        y[..., :rot // 2], y[..., rot // 2:rot] = a * c - b * s, a * s + b * c
    return y


def _row_places(s):
    """sequence and position of every row."""
    row = torch.arange(s["rows"], device=s["q_start"].device, dtype=torch.int32)
    seq = torch.searchsorted(s["q_start"], row, right=True) - 1
    pos = s["kv_len"][seq] - s["q_start"][seq + 1] + row
    return seq, pos.long()


def _plain_rotary(s):
    c = s["case"]
    angle = s["pos"].double()[:, None] * s["freq"][None]
    s["y"].copy_(_rotate(s["x"].float(), angle, c["rot"], c["layout"], s["gain"], c["transposed"]))
    return s["y"]


def _plain_append(s):
    c = s["case"]
    seq, pos = _row_places(s)
    angle = pos.double()[:, None] * s["freq"][None]
    s["q_rot"].copy_(_rotate(s["q"].float(), angle, c["rot"], c["layout"], s["gain"], False))
    k = _rotate(s["k"].float(), angle, c["rot"], c["layout"], s["gain"], False)
    page, slot = s["pages"][seq, pos // c["page"]].long(), pos % c["page"]
    s["kp"][page, :, slot] = k.to(s["kp"].dtype)
    s["vp"][page, :, slot] = s["v"].to(s["vp"].dtype)
    return s["q_rot"], s["kp"], s["vp"]


def _plain_attention(s):
    c = s["case"]
    B, H, Hkv, d, Q, L = c["B"], c["H"], c["Hkv"], c["d_head"], s["max_q"], s["max_len"]
    G, dev = H // Hkv, s["q"].device
    seq, pos = _row_places(s)
    inside = (torch.arange(s["rows"], device=dev, dtype=torch.int32) - s["q_start"][seq]).long()
    q = torch.zeros((B, Q, H, d), device=dev)
    q[seq, inside] = s["q"].float()
    limit = torch.full((B, Q), -1, dtype=torch.int64, device=dev)
    limit[seq, inside] = pos
    table = s["pages"].long()
    k = s["kp"][table].permute(0, 2, 1, 3, 4).reshape(B, Hkv, -1, d)[:, :, :L].float()
    v = s["vp"][table].permute(0, 2, 1, 3, 4).reshape(B, Hkv, -1, d)[:, :, :L].float()
    qg = q.view(B, Q, Hkv, G, d).permute(0, 2, 1, 3, 4).reshape(B, Hkv, Q * G, d)
    w = (qg @ k.transpose(-1, -2)).mul_(1.0 / math.sqrt(d)).view(B, Hkv, Q, G, L)
    w.masked_fill_((torch.arange(L, device=dev)[None, None] > limit[:, :, None])[:, None, :, None], float("-inf"))
    w = w.sub_(w.amax(-1, keepdim=True).clamp_min(-3e38)).exp_()
    total = w.sum(-1, keepdim=True).clamp_min(1e-30)
    o = (w.view(B, Hkv, Q * G, L) @ v).view(B, Hkv, Q, G, d) / total
    s["out"].copy_(o.permute(0, 2, 1, 3, 4).reshape(B, Q, H, d)[seq, inside])
    return s["out"]


def run(s):
    c = s["case"]
    if own:
        import paper_2302_01318_b200 as sps
        if c["op"] == "rotary":
            sps.sps_rotary(s["x"], s["y"], s["pos"], s["rope"], transposed=c["transposed"])
            return s["y"]
        if c["op"] == "append":
            sps.sps_paged_append(s["cache"], s["batch"], s["k"], s["v"], s["rope"], s["q"], s["q_rot"])
            return s["q_rot"], s["kp"], s["vp"]
        sps.sps_paged_attention(s["cache"], s["batch"], s["q"], s["out"], s["ws"])
        return s["out"]
    return {"rotary": _plain_rotary, "append": _plain_append, "attention": _plain_attention}[c["op"]](s)


# ----------------------------------------------------------------------------------------------------------------- work
def work(case):
    d = case["d_head"]
    size = {"fp32": 4, "bf16": 2}
    if case["op"] == "rotary":
        n = case["rows"] * case["heads"] * d
        return {"bytes": 2 * n * size[case["dtype"]] + 4 * case["rows"], "flops": 3 * case["rows"] * case["heads"] * case["rot"]}
    H, Hkv, (n, L) = case["H"], case["Hkv"], _lengths(case)
    rows = sum(n)
    if case["op"] == "append":
        return {"bytes": rows * d * ((H + 2 * Hkv) * size[case["act"]] + H * size[case["q_out"]] + 2 * Hkv * size[case["cache"]]),
                "flops": 3 * rows * (H + Hkv) * case["rot"]}
    pairs = sum(a * (b - a) + a * (a + 1) // 2 for a, b in zip(n, L))
    return {"bytes": 2 * sum(L) * Hkv * d * size[case["cache"]] + 2 * rows * H * d * size[case["act"]], "flops": 4 * pairs * H * d}


# ---------------------------------------------------------------------------------------------------------------- exact
def _exact_turn(x, pos, freq, rot, layout, gain, transposed):
    """The rotation as a product of complex numbers: z -> g e^{+- i p f} z."""
    x = x.double()
    z = torch.complex(x[..., 0:rot:2], x[..., 1:rot:2]) if layout == "pairs" else torch.complex(x[..., :rot // 2], x[..., rot // 2:rot])
    w = torch.polar(torch.full_like(pos, gain, dtype=torch.float64)[:, None].expand(-1, rot // 2).contiguous(),
                    pos.double()[:, None] * freq[None] * (-1.0 if transposed else 1.0))
    z = z * w[:, None, :]
    turned = torch.stack((z.real, z.imag), -1).flatten(-2) if layout == "pairs" else torch.cat((z.real, z.imag), -1)
    return torch.cat((turned, x[..., rot:]), -1)


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "rotary":
        return _exact_turn(s["x"], s["pos"], s["freq"], case["rot"], case["layout"], s["gain"], case["transposed"])
    d, ps = case["d_head"], case["page"]
    starts, lens, table = s["q_start"].tolist(), s["kv_len"].tolist(), s["pages"].long()
    if case["op"] == "append":
        pos = torch.cat([torch.arange(L - (e - a), L) for a, e, L in zip(starts, starts[1:], lens)]).to(s["q"].device)
        turn = (s["freq"], case["rot"], case["layout"], s["gain"], False)
        q, k, v = _exact_turn(s["q"], pos, *turn), _exact_turn(s["k"], pos, *turn), s["v"].double()
        kp, vp = s["kp"].double(), s["vp"].double()
        for b, (a, e, L) in enumerate(zip(starts, starts[1:], lens)):
            at = pos[a:e]
            kp[table[b, at // ps], :, at % ps] = k[a:e]
            vp[table[b, at // ps], :, at % ps] = v[a:e]
        return q, kp, vp
    H, Hkv = case["H"], case["Hkv"]
    G = H // Hkv
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=s["q"].device)
    for b, (a, e, L) in enumerate(zip(starts, starts[1:], lens)):
        at = torch.arange(L, device=out.device)
        hidden = at[None] > torch.arange(L - (e - a), L, device=out.device)[:, None]
        for h in range(Hkv):
            k, v = s["kp"][table[b, at // ps], h, at % ps].double(), s["vp"][table[b, at // ps], h, at % ps].double()
            for g in range(h * G, (h + 1) * G):
                w = torch.softmax((s["q"][a:e, g].double() @ k.T / math.sqrt(d)).masked_fill(hidden, float("-inf")), -1)
                out[a:e, g] = w @ v
    return out
