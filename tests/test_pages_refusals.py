"""What the page and beam calls refuse.  No GPU needed: a refused call returns before anything is launched."""
import ctypes as C
import math

import pytest

import paper_2302_01318_b200 as sps

P = 1 << 20      # a 16-byte aligned number that is never followed


def make(kind, **kw):
    base = {sps.sps_page_pool: dict(refs=P, status=None, n_pages=8, page_size=16),
            sps.sps_page_table: dict(pages=P, held=2 * P, len=3 * P, B=4, ld=5),
            sps.sps_page_moves: dict(list=P, count=2 * P, capacity=4),
            sps.sps_paged_cache: dict(k=P, v=P, page_stride=64 * 16 * 2, head_stride=64 * 16, pos_stride=64, dtype=1, n_pages=8, page_size=16, n_kv_heads=2, d_head=64)}[kind]
    base.update(kw)
    return kind(*[base[n] for n, _ in kind._fields_])


def pool(**kw):
    return make(sps.sps_page_pool, **kw)


def table(**kw):
    return make(sps.sps_page_table, **kw)


def other(**kw):
    return make(sps.sps_page_table, **{"pages": 5 * P, "held": 6 * P, "len": 7 * P, **kw})


def moves(**kw):
    return make(sps.sps_page_moves, **kw)


def ref(x):
    return C.byref(x) if x is not None else None


def fork(p=None, s=None, d=None, parents=P):
    return sps.lib().sps_paged_fork(ref(p or pool()), ref(s or table()), ref(d or other()), parents, None)


def reserve(p=None, t=None, want=P, m=None, ws=P, room=None):
    return sps.lib().sps_paged_reserve(ref(p or pool()), ref(t or table()), want, room, ref(m or moves()), ws, None)


def compact(p=None, s=None, d=None, refs=P, m=None, ws=P):
    return sps.lib().sps_paged_compact(ref(p or pool()), ref(s or table()), ref(d or other()), refs, ref(m or moves()), ws, None)


def copy(layers, m=None, n=None):
    arr = (sps.sps_paged_cache * max(len(layers), 1))(*layers)
    return sps.lib().sps_paged_copy(C.addressof(arr), len(layers) if n is None else n, ref(m or moves()), None)


def select(**kw):
    f = dict(logits=P, dtype=0, row=100, B=2, W=3, V=100, T=1.0, scores=P, done=None, end=-1, N=4, os=P, op=P, ot=P, od=None, ws=P)
    f.update(kw)
    return sps.lib().sps_beam_select(*f.values(), None)


def refused(rc, word):
    msg = sps.lib().sps_last_error(None).decode()
    assert rc == sps.SPS_EINVAL and word in msg, (rc, msg)


@pytest.mark.parametrize("kw,word", [(dict(refs=None), "null"), (dict(refs=P + 2), "aligned"), (dict(status=P + 1), "aligned"), (dict(n_pages=0), "n_pages"), (dict(n_pages=(1 << 20) + 1), "n_pages"),
                                     (dict(page_size=12), "power of two"), (dict(page_size=4), "power of two"), (dict(page_size=1024), "power of two")])
def test_pools(kw, word):
    for rc in (fork(pool(**kw)), reserve(pool(**kw)), compact(pool(**kw))):
        refused(rc, word)


@pytest.mark.parametrize("kw,word", [(dict(B=-1), "B"), (dict(B=8193), "B"), (dict(ld=-1), "ld"), (dict(ld=(1 << 20) + 1), "ld"), (dict(B=8192, ld=262144), "2^31"), (dict(pages=None), "null"),
                                     (dict(held=None), "null"), (dict(len=None), "null"), (dict(len=P + 2), "aligned")])
def test_tables(kw, word):
    for rc in (fork(s=table(**kw)), fork(d=other(**kw)), reserve(t=table(**kw)), compact(s=table(**kw)), compact(d=other(**kw))):
        refused(rc, word)


@pytest.mark.parametrize("kw,word", [(dict(capacity=-1), "capacity"), (dict(count=None), "null"), (dict(list=None), "null"), (dict(list=P + 2), "aligned")])
def test_moves(kw, word):
    for rc in (reserve(m=moves(**kw)), compact(m=moves(**kw)), copy([make(sps.sps_paged_cache)], moves(**kw))):
        refused(rc, word)


def test_combinations():
    refused(fork(d=other(ld=4)), "shorter")
    refused(fork(d=other(pages=P)), "share")
    refused(fork(d=other(held=2 * P)), "share")
    refused(fork(d=other(len=3 * P)), "share")
    refused(fork(parents=None), "parents")
    refused(fork(parents=P + 2), "parents")
    refused(reserve(want=None), "want")
    refused(reserve(want=P + 1), "want")
    refused(reserve(room=P + 2), "room")
    refused(reserve(m=moves(capacity=3)), "capacity")
    refused(reserve(ws=None), "workspace")
    refused(reserve(ws=P + 8), "workspace")
    refused(compact(d=other(B=5)), "rows")
    refused(compact(d=other(ld=4)), "rows")
    refused(compact(d=table(ld=6)), "in place")
    refused(compact(refs=None), "refs_out")
    refused(compact(ws=P + 4), "workspace")
    L = sps.lib()
    assert L.sps_paged_fork(None, None, None, None, None) == sps.SPS_EINVAL
    assert L.sps_paged_reserve(None, None, None, None, None, None, None) == sps.SPS_EINVAL
    assert L.sps_paged_compact(None, None, None, None, None, None, None) == sps.SPS_EINVAL
    assert L.sps_paged_copy(None, 1, None, None) == sps.SPS_EINVAL
    assert L.sps_paged_pool_workspace_bytes(0) == -1 and L.sps_paged_pool_workspace_bytes((1 << 20) + 1) == -1
    with pytest.raises(sps.SpsError):
        sps.sps_paged_pool_workspace_bytes(-1)


def test_layers():
    c = make(sps.sps_paged_cache)
    for kw in (dict(dtype=0), dict(n_pages=9), dict(page_size=8), dict(n_kv_heads=1), dict(pos_stride=72), dict(page_stride=4096), dict(head_stride=2048)):
        refused(copy([c, make(sps.sps_paged_cache, **kw)]), "unlike")
    refused(copy([make(sps.sps_paged_cache, d_head=96)]), "d_head")
    refused(copy([c, make(sps.sps_paged_cache, v=None)]), "null")
    refused(copy([c], n=-1), "layers")


@pytest.mark.parametrize("kw,word", [(dict(B=-1), "B"), (dict(B=8193), "B"), (dict(W=0), "W"), (dict(W=129), "W"), (dict(V=0), "V"), (dict(V=(1 << 24) + 1), "V"),
                                     (dict(W=128, V=1 << 24), "2^31"), (dict(B=8192, W=128, V=(1 << 24) - 1), "W x V"), (dict(dtype=2), "dtype"), (dict(N=0), "N"),
                                     (dict(N=129), "N"), (dict(row=-1), "stride"), (dict(T=0.0), "temperature"), (dict(T=-1.0), "temperature"),
                                     (dict(T=math.nan), "temperature"), (dict(T=math.inf), "temperature"), (dict(T=1e-39), "temperature"), (dict(T=1e39), "temperature"),
                                     (dict(end=-2), "end_token"), (dict(end=100), "end_token"), (dict(done=P), "end_token"), (dict(logits=None), "null"),
                                     (dict(scores=None), "null"), (dict(os=None), "null"), (dict(op=None), "null"), (dict(ot=None), "null"),
                                     (dict(logits=P + 2), "aligned"), (dict(dtype=1, logits=P + 1), "aligned"), (dict(od=P + 2), "aligned"),
                                     (dict(ws=None), "workspace"), (dict(ws=P + 8), "workspace")])
def test_select(kw, word):
    refused(select(**kw), word)


def test_workspace_sizes_are_refused_with_the_shapes():
    L = sps.lib()
    for shape in ((-1, 1, 8), (1, 0, 8), (1, 129, 8), (1, 1, 0), (1, 128, 1 << 24)):
        assert L.sps_beam_select_workspace_bytes(*shape) == -1
    with pytest.raises(sps.SpsError):
        sps.sps_beam_select_workspace_bytes(1, 0, 8)


def test_nothing_to_do_is_no_error_and_launches_nothing():
    empty = dict(B=0, pages=None, held=None, len=None)
    assert fork(s=table(**empty), d=other(**empty), parents=None) == sps.SPS_OK
    assert copy([]) == sps.SPS_OK and copy([make(sps.sps_paged_cache)], moves(capacity=0, list=None)) == sps.SPS_OK
    assert select(B=0) == sps.SPS_OK


def test_struct_sizes_match_the_header():
    assert C.sizeof(sps.sps_page_pool) == 24 and C.sizeof(sps.sps_page_table) == 32 and C.sizeof(sps.sps_page_moves) == 24
