"""sps_rotary and sps_paged_append on the GPU against 64-bit restatements."""
import math

import pytest
import torch

import paper_2302_01318_b200 as sps
from paged_util import BF16, DEV, F32, Pages, freqs, normal, rotate64, rotate_tol

pytestmark = pytest.mark.gpu


def positions(n, far, seed=3):
    g = torch.Generator().manual_seed(seed)
    return torch.randint(0, far, (n,), generator=g).to(torch.int32).to(DEV)


@pytest.mark.parametrize("layout", ["pairs", "halves"])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,heads,d,rot", [(1, 1, 2, 2), (1, 72, 128, 128), (5, 72, 128, 128), (7, 3, 64, 32), (333, 6, 64, 16), (1031, 9, 128, 64),
                                              (3, 5, 96, 96), (2, 3, 80, 20), (4, 2, 1024, 1024), (6000, 1, 64, 64), (17, 4, 10, 6)])
def test_rotary_matches_64_bits(layout, dtype, rows, heads, d, rot):
    x, pos, f = normal((rows, heads, d), dtype, 1), positions(rows, 5000), freqs(rot)
    for transposed in (False, True):
        y = torch.full_like(x, 3.0)
        sps.sps_rotary(x, y, pos, sps.Rotary(f, layout, 1.25), transposed=transposed)
        want = rotate64(x, pos, f, layout, 1.25, transposed)
        assert ((y.double() - want).abs() <= rotate_tol(x, f, layout, 1.25, dtype)).all()
        assert torch.equal(y[..., rot:], x[..., rot:])


@pytest.mark.parametrize("layout", ["pairs", "halves"])
def test_rotary_far_and_negative_positions_keep_their_phase(layout):
    pos = torch.tensor([0, 1, -1, 131072, 1000003, 2 ** 24 + 1, 2 ** 31 - 1, -2 ** 31], dtype=torch.int64).to(torch.int32).to(DEV)
    x, f = normal((8, 4, 128), F32, 2), freqs(128, 500000.0)
    y = torch.empty_like(x)
    sps.sps_rotary(x, y, pos, sps.Rotary(f, layout))
    # the 64-bit angle itself is off by up to |angle| 2^-53 on either side: 2^31 * 2^-52 = 5e-7 on top
    tol = rotate_tol(x, f, layout, 1.0, F32) + 2.0 ** 31 * 2.0 ** -52 * x.double().abs().amax()
    assert ((y.double() - rotate64(x, pos, f, layout)).abs() <= tol).all()


@pytest.mark.parametrize("layout", ["pairs", "halves"])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_rotary_strides_alignment_and_in_place(layout, dtype):
    rows, heads, d, rot = 37, 5, 64, 48
    f, pos = freqs(rot), positions(rows, 999)
    plan = sps.Rotary(f, layout)
    big = normal((rows, heads + 3, d + 3), dtype, 4)
    for x in (big[:, 2:2 + heads, :d], big[:, 2:2 + heads, 3:], normal((heads, rows, d), dtype, 5).transpose(0, 1), normal((rows, heads, d), dtype, 6)):
        want, tol = rotate64(x, pos, f, layout), rotate_tol(x, f, layout, 1.0, dtype)
        y = torch.zeros((rows, heads, d), dtype=dtype, device=DEV)
        sps.sps_rotary(x, y, pos, plan)
        assert ((y.double() - want).abs() <= tol).all()
        before = big.clone()
        sps.sps_rotary(x, x, pos, plan)
        assert torch.equal(x, y)
        if x.data_ptr() >= big.data_ptr() and x.data_ptr() < big.data_ptr() + big.numel() * big.element_size():
            mask = torch.ones_like(big, dtype=torch.bool)
            mask[:, 2:2 + heads, (3 if x.storage_offset() % (d + 3) == 3 else 0):][..., :d] = False
            assert torch.equal(big[mask], before[mask])


@pytest.mark.parametrize("layout", ["pairs", "halves"])
def test_rotary_gradient(layout):
    """The transposed call is the gradient: against the formula's (autograd in 64 bits) and against differences."""
    rows, heads, d, rot = 3, 2, 16, 12
    f, pos, plan = freqs(rot), positions(rows, 50), None
    plan = sps.Rotary(f, layout, 0.75)
    x, g = normal((rows, heads, d), F32, 7), normal((rows, heads, d), F32, 8)
    dx = torch.empty_like(x)
    sps.sps_rotary(g, dx, pos, plan, transposed=True)
    xd = x.double().requires_grad_(True)
    (rotate64(xd, pos, f, layout, 0.75) * g.double()).sum().backward()
    assert ((dx.double() - xd.grad).abs() <= rotate_tol(g, f, layout, 0.75, F32)).all()
    # the map is linear, so a difference over a whole unit is the derivative: sum of g . (y(x + e) - y(x)) for every element
    eye = torch.eye(heads * d, device=DEV).view(heads * d, 1, heads, d)
    for r in range(rows):
        e = eye.expand(-1, 1, -1, -1).reshape(heads * d, heads, d).contiguous()
        p = pos[r:r + 1].expand(heads * d).contiguous()
        y1, y0 = torch.empty_like(e), torch.empty_like(e)
        xr = x[r:r + 1].expand(heads * d, -1, -1)
        sps.sps_rotary((xr + e).contiguous(), y1, p, plan)
        sps.sps_rotary(xr.contiguous(), y0, p, plan)
        diff = ((y1 - y0).double() * g[r].double()).sum((1, 2)).view(heads, d)
        # each y is off by 2^-21 (|a| + |b|), x + e rounds to 2^-24 |x + e|; summed over the pair's two elements and |g|
        tol = 16 * 2.0 ** -21 * (x.abs().max().item() + 1) * g.abs().max().item()
        assert (diff - dx[r].double()).abs().max().item() <= tol


def test_rotary_empty_and_other_stream_and_graph():
    f = freqs(64)
    plan = sps.Rotary(f)
    sps.sps_rotary(torch.empty((0, 3, 64), device=DEV), torch.empty((0, 3, 64), device=DEV), torch.empty(0, dtype=torch.int32, device=DEV), plan)
    x, pos, y = normal((50, 3, 64), F32, 9), positions(50, 100), torch.zeros((50, 3, 64), device=DEV)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        sps.sps_rotary(x, y, pos, plan)
    s.synchronize()
    tol = rotate_tol(x, f, "pairs", 1.0, F32)
    assert ((y.double() - rotate64(x, pos, f, "pairs")).abs() <= tol).all()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        sps.sps_rotary(x, y, pos, plan)
    pos.add_(1000)
    graph.replay()
    torch.cuda.synchronize()
    assert ((y.double() - rotate64(x, pos, f, "pairs")).abs() <= tol).all()


# ------------------------------------------------------------------------------------------------------------ append
def append_reference(pages, news, lead, k, v, q, f, layout, gain):
    """(expected rotated q, expected pools in 64 bits, which slots are written) -- rows at negative positions are skipped."""
    kp, vp = pages.k.double(), pages.v.double()
    rows = k.shape[0]
    written = torch.zeros(pages.k.shape[:3], dtype=torch.bool, device=DEV)
    rowmask = torch.zeros(rows, dtype=torch.bool, device=DEV)
    pos = torch.zeros(rows, dtype=torch.int64)
    where = []
    a = lead
    for b, (n, L) in enumerate(zip(news, pages.lens)):
        for i in range(n):
            p = L - n + i
            pos[a + i] = p
            if p >= 0:
                where.append((a + i, int(pages.table[b, p // pages.page]), p % pages.page))
                rowmask[a + i] = True
        a += n
    pos = pos.to(DEV)
    kr = rotate64(k, pos, f, layout, gain) if f is not None else k.double()
    qr = rotate64(q, pos, f, layout, gain) if q is not None else None
    for r, p, s in where:
        kp[p, :, s] = kr[r]
        vp[p, :, s] = v[r].double()
        written[p, :, s] = True
    return qr, kp, vp, written, rowmask


CASES = [  # lens, news, Hkv, H, d, rot, page
    ([1], [1], 1, 1, 64, 64, 8),
    ([5, 40, 7, 129], [5, 1, 0, 3], 2, 8, 128, 128, 16),
    ([300, 16, 33], [97, 16, 1], 4, 4, 64, 32, 32),
    ([6, 2, 64], [6, 5, 64], 8, 8, 128, 32, 64),            # the second sequence has more rows than tokens
    ([17] * 40, [3] * 40, 1, 3, 64, 64, 16),                # more sequences than a warp has lanes
    ([1100], [1100], 2, 2, 128, 128, 512),
]


@pytest.mark.parametrize("layout", ["pairs", "halves"])
@pytest.mark.parametrize("types", [(F32, F32, F32), (F32, F32, BF16), (F32, BF16, BF16), (F32, BF16, F32), (BF16, BF16, BF16)])
@pytest.mark.parametrize("case", range(len(CASES)))
def test_append_matches_64_bits(layout, types, case):
    lens, news, Hkv, H, d, rot, page = CASES[case]
    act, qdt, cdt = types
    lead, tail = (2, 3) if case % 2 else (0, 0)
    rows = lead + sum(news) + tail
    pages = Pages(lens, Hkv, d, page, cdt, seed=case, order="head" if case % 2 else "slot", fill=3.0)
    f, gain = freqs(rot), 1.5
    qkv = normal((rows, H + 2 * Hkv, d), act, 11)
    q, k, v = qkv[:, :H], qkv[:, H:H + Hkv], qkv[:, H + Hkv:]
    qr, kp, vp, written, rowmask = append_reference(pages, news, lead, k, v, q, f, layout, gain)
    k0, v0 = pages.k.clone(), pages.v.clone()
    q_out = torch.full((rows, H, d), 7.0, dtype=qdt, device=DEV)
    batch = pages.batch(news, lead)
    sps.sps_paged_append(pages.cache, batch, k, v, sps.Rotary(f, layout, gain), q, q_out)
    torch.cuda.synchronize()
    assert int(batch.status) == 0
    # untouched: every other slot, rows outside the batch, rows at negative positions
    assert torch.equal(pages.k[~written], k0[~written]) and torch.equal(pages.v[~written], v0[~written])
    assert (q_out[~rowmask] == 7).all()
    assert torch.equal(pages.v[written], vp[written].to(cdt))
    assert ((q_out.double() - qr).abs() <= rotate_tol(q, f, layout, gain, qdt))[rowmask].all()
    # of a written key, the tolerance of its own pair: |a| + |b| <= sqrt(2) of the rotated pair's length over the gain
    kmag = kp.abs()
    i = torch.arange(rot // 2, device=DEV)
    ia, ib = (2 * i, 2 * i + 1) if layout == "pairs" else (i, i + rot // 2)
    pair = (kp[..., ia] ** 2 + kp[..., ib] ** 2).sqrt() * 2 ** 0.5
    tol = torch.zeros_like(kp)
    tol[..., ia], tol[..., ib] = pair * 2.0 ** -21, pair * 2.0 ** -21
    tol = tol + (kmag + tol) * (2.0 ** -8 if cdt == BF16 else 0.0)
    assert ((pages.k.double() - kp).abs() <= tol)[written].all()


def test_append_without_rotation_and_without_queries():
    pages = Pages([9, 20], 2, 64, 8, BF16, fill=1.0)
    k, v = normal((7, 2, 64), F32, 1), normal((7, 2, 64), F32, 2)
    _, kp, vp, written, _ = append_reference(pages, [3, 4], 0, k, v, None, None, "pairs", 1.0)
    sps.sps_paged_append(pages.cache, pages.batch([3, 4]), k, v)
    assert torch.equal(pages.k[written], kp[written].to(BF16)) and torch.equal(pages.v[written], vp[written].to(BF16))
    f = freqs(32)
    sps.sps_paged_append(pages.cache, pages.batch([3, 4]), k, v, sps.Rotary(f, "halves"))
    _, kp, _, _, _ = append_reference(pages, [3, 4], 0, k, v, None, f, "halves", 1.0)
    assert ((pages.k.double() - kp).abs() <= (kp.abs() + 1e-5) * 2.0 ** -8 + 1e-5)[written].all()


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_append_in_place_and_unaligned_rows(dtype):
    pages = Pages([13], 1, 64, 8, BF16 if dtype == BF16 else F32, fill=0.0)
    buf = normal((13, 4, 67), dtype, 3)
    q, k, v = buf[:, 0:2, 1:65], buf[:, 2:3, 1:65], buf[:, 3:4, 1:65]
    f = freqs(64)
    qr, kp, vp, written, _ = append_reference(pages, [13], 0, k, v, q, f, "pairs", 1.0)
    tol, rest = rotate_tol(q, f, "pairs", 1.0, dtype), buf[..., 65:].clone()
    sps.sps_paged_append(pages.cache, pages.batch([13]), k, v, sps.Rotary(f), q, q)
    assert ((q.double() - qr).abs() <= tol).all() and torch.equal(buf[..., 65:], rest)
    assert torch.equal(pages.v[written], vp[written].to(pages.v.dtype))


def test_append_bad_pages_and_lengths_are_skipped_and_flagged():
    pages = Pages([20, 20, 20], 2, 64, 8, F32, fill=4.0, spare=0, extra_cols=0)
    pages.table[0, 2] = pages.n_pages          # one past the last page
    pages.table[1, 2] = -1
    k, v = normal((18, 2, 64), F32, 1), normal((18, 2, 64), F32, 2)
    k0 = pages.k.clone()
    batch = pages.batch([6, 6, 6])
    sps.sps_paged_append(pages.cache, batch, k, v)
    assert int(batch.status) == sps.PAGED_BAD_PAGE
    # sequences 0 and 1: positions 14, 15 are on a good page, 16 .. 19 are dropped; sequence 2 is whole
    for b, good in ((0, 2), (1, 2), (2, 6)):
        for i in range(6):
            p = 14 + i
            if i < good:
                pg = int(pages.table[b, p // 8])
                assert torch.equal(pages.k[pg, :, p % 8], k[6 * b + i]) and torch.equal(pages.v[pg, :, p % 8], v[6 * b + i])
    assert int((pages.k != k0).any(-1).any(1).sum()) == 2 + 2 + 6
    # a length beyond the table's three pages: nothing of that sequence past them is written
    pages2 = Pages([20], 2, 64, 8, F32, fill=4.0, extra_cols=0)
    b2 = pages2.batch([4])
    b2.kv_len.fill_(26)                        # positions 22 .. 25: two of them fit 24 slots
    before = pages2.k.clone()
    sps.sps_paged_append(pages2.cache, b2, k[:4], v[:4])
    assert int(b2.status) == sps.PAGED_BAD_LENGTH
    changed = (pages2.k != before).any(-1).any(1)
    assert int(changed.sum()) == 2 and bool(changed[int(pages2.table[0, 2]), 6]) and bool(changed[int(pages2.table[0, 2]), 7])


def test_append_replayed_in_a_graph_follows_lengths_and_tables():
    pages = Pages([10, 30], 1, 64, 8, F32, fill=0.0, spare=6, extra_cols=3)
    k, v = normal((2, 1, 64), F32, 1), normal((2, 1, 64), F32, 2)
    batch = pages.batch([1, 1])
    sps.sps_paged_append(pages.cache, batch, k, v)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        sps.sps_paged_append(pages.cache, batch, k, v)
    used = set(pages.table[0, :2].tolist()) | set(pages.table[1, :4].tolist())
    free = [p for p in range(pages.n_pages) if p not in used]
    for step in range(1, 9):
        k.copy_(normal((2, 1, 64), F32, 10 + step))
        batch.kv_len.add_(1)
        for b, L in ((0, 10 + step), (1, 30 + step)):
            if (L - 1) % 8 == 0:               # a new page begins
                pages.table[b, (L - 1) // 8] = free.pop()
        batch.pages.copy_(pages.table)
        graph.replay()
        torch.cuda.synchronize()
        for b, L in ((0, 10 + step), (1, 30 + step)):
            assert torch.equal(pages.k[int(pages.table[b, (L - 1) // 8]), 0, (L - 1) % 8], k[b, 0])
    assert int(batch.status) == 0


def test_rotary_as_many_rows_as_an_int_counts():
    """2^31 - 1 rows of one pair, in place (8.6 GB, and as much for the positions): a quarter turn at odd positions."""
    n = 2 ** 31 - 1
    plan = sps.Rotary(torch.tensor([math.pi / 2], dtype=torch.float64, device=DEV))
    x = torch.empty((n, 1, 2), dtype=BF16, device=DEV)
    x[..., 0], x[..., 1] = 1.0, 2.0
    pos = torch.zeros(n, dtype=torch.int32, device=DEV)
    pos[1::2] = 1
    sps.sps_rotary(x, x, pos, plan)
    for at, want in ((slice(0, None, 2), (1.0, 2.0)), (slice(1, None, 2), (-2.0, 1.0))):
        for e in range(2):
            assert bool((x[at, 0, e] == want[e]).all())
