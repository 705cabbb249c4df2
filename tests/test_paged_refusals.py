"""What the rotary / paged-cache calls refuse, and the frequencies they compute on the host.  No GPU needed: a refused call
returns before anything is launched."""
import ctypes as C
import math

import numpy as np
import pytest

import paper_2302_01318_b200 as sps

P = 1 << 20      # a 16-byte aligned number that is never followed


def rows(p=P, row=256, head=64, dtype=0, heads=4):
    return sps.sps_rows(p, row, head, dtype, heads)


def cache(**kw):
    f = dict(k=P, v=P, page_stride=64 * 16 * 2, head_stride=64 * 16, pos_stride=64, dtype=1, n_pages=8, page_size=16, n_kv_heads=2, d_head=64)
    f.update(kw)
    return sps.sps_paged_cache(*[f[n] for n, _ in sps.sps_paged_cache._fields_])


def batch(**kw):
    f = dict(q_start=P, kv_len=P, pages=P, status=None, B=2, pages_ld=4, max_q=1)
    f.update(kw)
    return sps.sps_paged_batch(*[f[n] for n, _ in sps.sps_paged_batch._fields_])


def plan(**kw):
    f = dict(freq=P, rot_dim=64, layout=0, gain=1.0)
    f.update(kw)
    return sps.sps_rotary_plan(*[f[n] for n, _ in sps.sps_rotary_plan._fields_])


def ref(x):
    return C.byref(x) if x is not None else None


def rotary(pl=None, x=None, y=None, n=3, d=64, pos=P):
    return sps.lib().sps_rotary(ref(pl or plan()), ref(x or rows()), ref(y or rows(2 * P)), n, d, pos, 0, None)


def append(c=None, b=None, pl=True, n=3, k=None, v=None, q=None, qo=None):
    return sps.lib().sps_paged_append(ref(c or cache()), ref(b or batch()), ref(plan() if pl is True else pl), n,
                                      ref(k or rows(heads=2)), ref(v or rows(heads=2)), ref(q), ref(qo), None)


def attend(c=None, b=None, n=3, q=None, o=None, scale=0.0, lse=None, ws=P):
    return sps.lib().sps_paged_attention(ref(c or cache()), ref(b or batch()), n, ref(q or rows()), ref(o or rows(2 * P)), scale, lse, ws, None)


def refused(rc, word):
    msg = sps.lib().sps_last_error(None).decode()
    assert rc == sps.SPS_EINVAL and word in msg, (rc, msg)


BAD_CACHES = [(dict(d_head=96), "d_head"), (dict(page_size=24), "power of two"), (dict(page_size=4), "power of two"), (dict(page_size=1024), "power of two"),
              (dict(n_pages=0), "n_pages"), (dict(n_kv_heads=0), "n_kv_heads"), (dict(k=None), "null"), (dict(k=P + 8), "aligned"),
              (dict(page_stride=2047), "strides"), (dict(pos_stride=68), "strides"), (dict(pos_stride=56), "strides"), (dict(head_stride=0), "strides"),
              (dict(dtype=2), "dtype"), (dict(dtype=0, pos_stride=66), "strides")]
BAD_BATCHES = [(dict(B=-1), "B"), (dict(max_q=0), "max_q"), (dict(pages_ld=-1), "pages_ld"), (dict(q_start=None), "null"), (dict(kv_len=None), "null"),
               (dict(pages=None), "null"), (dict(kv_len=P + 2), "aligned"), (dict(status=P + 1), "aligned")]
BAD_PLANS = [(dict(freq=None), "freq"), (dict(freq=P + 4), "freq"), (dict(rot_dim=0), "rot_dim"), (dict(rot_dim=7), "rot_dim"), (dict(rot_dim=66), "rot_dim"),
             (dict(layout=2), "layout"), (dict(gain=math.nan), "gain"), (dict(gain=math.inf), "gain")]
BAD_ROWS = [(dict(dtype=2), "dtype"), (dict(heads=0), "heads"), (dict(row=-1), "stride"), (dict(p=None), "null"), (dict(p=P + 2), "aligned")]


@pytest.mark.parametrize("kw,word", BAD_CACHES)
def test_caches(kw, word):
    refused(append(cache(**kw)), word)
    refused(attend(cache(**kw)), word)
    assert sps.lib().sps_paged_attention_workspace_bytes(C.byref(cache(**kw)), 4, 0) == -1


@pytest.mark.parametrize("kw,word", BAD_BATCHES)
def test_batches(kw, word):
    refused(append(b=batch(**kw)), word)
    refused(attend(b=batch(**kw)), word)


@pytest.mark.parametrize("kw,word", BAD_PLANS)
def test_plans(kw, word):
    refused(rotary(plan(**kw)), word)
    refused(append(pl=plan(**kw)), word)


@pytest.mark.parametrize("kw,word", BAD_ROWS)
def test_rows(kw, word):
    refused(rotary(x=rows(**kw)), word)
    refused(rotary(y=rows(**kw)), word)
    refused(append(k=rows(**{"heads": 2, **kw})), word)
    refused(append(q=rows(**kw), qo=rows(2 * P)), word)
    refused(append(q=rows(), qo=rows(**kw)), word)
    refused(attend(q=rows(**kw)), word)
    refused(attend(o=rows(**kw)), word)


def test_combinations():
    refused(rotary(d=63), "d_head")
    refused(rotary(d=2048), "d_head")
    refused(rotary(n=-1), "rows")
    refused(rotary(pos=None), "positions")
    refused(rotary(y=rows(2 * P, dtype=1)), "dtype")
    refused(rotary(y=rows(2 * P, heads=3)), "heads")
    refused(rotary(y=rows(row=512)), "in place")
    refused(append(n=-1), "rows")
    refused(append(q=rows()), "null")
    refused(append(qo=rows()), "without q")
    refused(append(pl=None, q=rows(), qo=rows()), "plan")
    refused(append(k=rows(heads=3)), "heads")
    refused(append(v=rows(heads=2, dtype=1)), "dtype")
    refused(append(q=rows(dtype=1), qo=rows(dtype=1)), "dtype")
    refused(append(q=rows(), qo=rows(2 * P, heads=5)), "heads")
    refused(append(cache(dtype=0), k=rows(heads=2, dtype=1), v=rows(heads=2, dtype=1)), "fp32 cache")
    refused(append(k=rows(heads=2, dtype=1), v=rows(heads=2, dtype=1), q=rows(dtype=1), qo=rows(2 * P)), "q_out")
    refused(append(q=rows(), qo=rows(dtype=1)), "in place")
    refused(attend(n=-2), "rows")
    refused(attend(n=1 << 29), "2^31")
    refused(attend(q=rows(heads=3), o=rows(heads=3)), "multiple")
    refused(attend(o=rows(heads=2)), "heads")
    refused(attend(cache(dtype=0), q=rows(dtype=1)), "fp32 cache")
    refused(attend(o=rows(dtype=1)), "out")
    refused(attend(scale=math.nan), "scale")
    refused(attend(ws=None), "workspace")
    refused(attend(ws=P + 4), "workspace")
    refused(attend(lse=P + 2), "lse")
    L = sps.lib()
    assert L.sps_rotary(None, C.byref(rows()), C.byref(rows()), 1, 64, P, 0, None) == sps.SPS_EINVAL
    assert L.sps_paged_append(None, None, None, 1, None, None, None, None, None) == sps.SPS_EINVAL
    assert L.sps_paged_attention(None, None, 1, None, None, 0.0, None, None, None) == sps.SPS_EINVAL
    assert L.sps_paged_attention_workspace_bytes(None, 4, 0) == -1
    assert L.sps_paged_attention_workspace_bytes(C.byref(cache()), 3, 0) == -1
    assert L.sps_paged_attention_workspace_bytes(C.byref(cache(dtype=0)), 4, 1) == -1


def test_attention_in_place_wants_the_same_layout():
    refused(attend(q=rows(row=256), o=rows(row=512)), "in place")
    refused(attend(q=rows(head=64), o=rows(head=128)), "in place")
    refused(attend(q=rows(dtype=1), o=rows(dtype=0)), "in place")


def test_more_sequences_than_the_list_of_work_counts_are_refused():
    refused(attend(b=batch(B=(1 << 27) + 1)), "B")


def test_a_scale_that_overflows_in_base_2_is_refused():
    """Scores are kept in base 2: scale / ln 2 has to be a number too."""
    refused(attend(scale=3e38), "scale")


def test_nothing_to_do_is_no_error_and_launches_nothing():
    assert rotary(n=0) == sps.SPS_OK and append(n=0) == sps.SPS_OK and attend(n=0) == sps.SPS_OK
    assert append(b=batch(B=0, q_start=None, kv_len=None, pages=None)) == sps.SPS_OK
    assert attend(b=batch(B=0, q_start=None, kv_len=None, pages=None)) == sps.SPS_OK


def test_frequencies():
    f = sps.sps_rotary_frequencies
    i = np.arange(32)
    plain = 10000.0 ** (-2 * i / 64)
    assert np.allclose(f(64), plain, rtol=1e-14)
    assert np.allclose(f(64, scaling="linear", factor=4.0), plain / 4, rtol=1e-14)
    base = f(64, scaling="base", factor=8.0)
    assert math.isclose(base[0], plain[0], rel_tol=1e-13) and math.isclose(base[-1], plain[-1] / 8, rel_tol=1e-12)
    assert (np.diff(np.log(base)).std() < 1e-12)                          # still geometric
    bands = f(64, scaling="bands", factor=8.0, trained_len=4096, low_turns=1.0, high_turns=32.0)
    turns = 4096 * plain / (2 * np.pi)
    assert np.allclose(bands[turns >= 32], plain[turns >= 32], rtol=1e-14)
    assert np.allclose(bands[turns <= 1], plain[turns <= 1] / 8, rtol=1e-14)
    mid = (turns > 1) & (turns < 32)
    w = (turns - 1) / 31
    assert mid.any() and np.allclose(bands[mid], (w * plain + (1 - w) * plain / 8)[mid], rtol=1e-14)
    assert f(2).tolist() == [1.0] and f(2, scaling="base", factor=3.0).tolist() == [1.0]


@pytest.mark.parametrize("kw", [dict(rot_dim=0), dict(rot_dim=3), dict(rot_dim=2048), dict(base=1.0), dict(base=math.inf), dict(base=math.nan),
                                dict(scaling="linear", factor=0.5), dict(scaling="base", factor=math.nan), dict(scaling="bands", factor=2.0),
                                dict(scaling="bands", factor=2.0, trained_len=10, low_turns=2.0, high_turns=2.0),
                                dict(scaling="bands", factor=2.0, trained_len=10, low_turns=-1.0)])
def test_frequencies_refused(kw):
    kw = {"rot_dim": 64, **kw}
    with pytest.raises(sps.SpsError) as e:
        sps.sps_rotary_frequencies(**kw)
    assert e.value.code == sps.SPS_EINVAL
    with pytest.raises(ValueError):
        sps.sps_rotary_frequencies(64, scaling="other")


def test_struct_sizes_match_the_header():
    assert C.sizeof(sps.sps_rows) == 32 and C.sizeof(sps.sps_rotary_plan) == 24
    assert C.sizeof(sps.sps_paged_cache) == 2 * 8 + 3 * 8 + 5 * 4 + 4 and C.sizeof(sps.sps_paged_batch) == 4 * 8 + 3 * 4 + 4
