"""C entry points of serving from the key-value cache: what they refuse, on the host
and before anything is enqueued. Runs without a GPU."""
import ctypes
import math

import pytest

import paper_1402_3788_amd as km
from paper_1402_3788_amd.kv_serve import _Evict, _Tokens, _Turn
from test_kv_abi import BAD_DESC, ODD, P, desc

INVALID, UNSUPPORTED, WORKSPACE, OK = (km.KMEANS_EINVAL, km.KMEANS_EUNSUPPORTED,
                                       km.KMEANS_EWORKSPACE, km.KMEANS_OK)
lib = km._lib


def rotate(turn=True, q=P, qa=128, qb=64, q_heads=2, qo=P, qoa=128, qob=64, k=P, ka=64, kb=64,
           k_heads=1, ko=P, koa=64, kob=64, **kw):
    d = dict(positions=P, frequencies=P, tokens=3, dim=64, half=32, type=0, flags=0, amplitude=1.0)
    d.update(kw)
    return lib.kmeans_kv_rotate(_Turn(**d) if turn else None, q, qa, qb, q_heads, qo, qoa, qob, k, ka,
                                kb, k_heads, ko, koa, kob, None)


@pytest.mark.parametrize("kw,code", [
    (dict(turn=False), INVALID), (dict(tokens=-1), INVALID), (dict(dim=0), INVALID),
    (dict(half=-1), INVALID), (dict(half=33), INVALID), (dict(amplitude=math.nan), INVALID),
    (dict(amplitude=math.inf), INVALID), (dict(type=2), INVALID), (dict(flags=4), INVALID),
    (dict(dim=60, half=2), UNSUPPORTED), (dict(dim=520), UNSUPPORTED),
    (dict(tokens=1 << 31), UNSUPPORTED), (dict(q_heads=-1), INVALID), (dict(k_heads=-1), INVALID),
    (dict(q=None), INVALID), (dict(qo=None), INVALID), (dict(k=None), INVALID),
    (dict(ko=None), INVALID), (dict(q=ODD), INVALID), (dict(qo=ODD), INVALID), (dict(k=ODD), INVALID),
    (dict(ko=ODD), INVALID), (dict(qa=4), INVALID), (dict(qb=-8), INVALID), (dict(qoa=1), INVALID),
    (dict(qob=-64), INVALID), (dict(ka=7), INVALID), (dict(kob=9), INVALID),
    # in place with other strides
    (dict(qoa=256), INVALID), (dict(kob=128), INVALID),
    (dict(positions=None), INVALID), (dict(frequencies=None), INVALID),
    (dict(q_heads=4097), UNSUPPORTED),
    (dict(tokens=0), OK), (dict(q_heads=0, k_heads=0), OK),
    (dict(tokens=0, q=None, k=None, positions=None), OK),
    (dict(tokens=0, k_heads=-1), INVALID),
])
def test_rotate(kw, code):
    assert rotate(**kw) == code


def tokens(**kw):
    d = dict(bounds=P, table=P, table_stride=2, table_pages=2, lengths=P, starts=None, prefixes=None,
             slopes=None, tokens=5, seqs=3, q_heads=4, window=0, scale=0.1, cap=0.0)
    d.update(kw)
    return _Tokens(**d)


def attend(d, t=None, q=P, qa=256, qb=64, out=P, oa=256, ob=64, lse=None, ws=P, nbytes=1 << 40, **kw):
    t = tokens(**kw) if t is None else t
    return lib.kmeans_kv_attend_tokens(d, t, q, qa, qb, out, oa, ob, lse, ws, nbytes, None)


def weigh(d, t=None, q=P, qa=256, qb=64, lse=P, w=P, wa=64, wb=32, positions=32, add=0, **kw):
    t = tokens(**kw) if t is None else t
    return lib.kmeans_kv_weigh(d, t, q, qa, qb, lse, w, wa, wb, positions, add, None)


def evict(d, e=True, kept=P, lengths_out=P, out=P, oa=64, ob=32, **kw):
    x = dict(table=P, table_stride=2, table_pages=2, lengths=P, weights=P, weights_seq=64,
             weights_head=32, positions=32, seqs=3, keep=20, recent=4, first=2, to=None, to_stride=2,
             to_pages=2)
    x.update(kw)
    return lib.kmeans_kv_evict(d, _Evict(**x) if e else None, kept, lengths_out, out, oa, ob, None)


@pytest.mark.parametrize("kw,code", BAD_DESC)
def test_description(kw, code):
    d = ctypes.byref(desc(**kw))
    assert attend(d) == weigh(d) == evict(d) == code
    if not set(kw) & {"k_centres", "v_centres", "k_codes", "v_codes"}:
        assert lib.kmeans_kv_attend_tokens_workspace_bytes(d, tokens()) == 0


def test_nothing_given():
    d = ctypes.byref(desc())
    assert attend(None) == weigh(None) == evict(None) == INVALID
    assert lib.kmeans_kv_attend_tokens(d, None, P, 256, 64, P, 256, 64, None, P, 1 << 40, None) == INVALID
    assert lib.kmeans_kv_weigh(d, None, P, 256, 64, P, P, 64, 32, 32, 0, None) == INVALID
    assert evict(d, e=False) == INVALID
    assert lib.kmeans_kv_attend_tokens_workspace_bytes(None, tokens()) == 0
    assert lib.kmeans_kv_attend_tokens_workspace_bytes(d, None) == 0


@pytest.mark.parametrize("kw,code", [
    (dict(bounds=None), INVALID), (dict(table=None), INVALID), (dict(lengths=None), INVALID),
    (dict(q=None), INVALID), (dict(q=ODD), INVALID), (dict(qa=12), INVALID), (dict(qb=-8), INVALID),
    (dict(table_stride=-1), INVALID), (dict(table_pages=0), INVALID),
    (dict(table_pages=1 << 28), UNSUPPORTED), (dict(seqs=-1), INVALID),
    (dict(seqs=4097), UNSUPPORTED), (dict(tokens=-1), INVALID), (dict(tokens=1 << 30), UNSUPPORTED),
    (dict(tokens=1 << 28), UNSUPPORTED), (dict(window=-1), INVALID), (dict(q_heads=0), INVALID),
    (dict(q_heads=5), INVALID), (dict(q_heads=2 * 129), UNSUPPORTED),
    (dict(seqs=4096, table_pages=1 << 24), UNSUPPORTED),
    (dict(scale=math.nan), INVALID), (dict(scale=math.inf), INVALID), (dict(scale=3e38), INVALID),
    (dict(cap=-1.0), INVALID), (dict(cap=math.nan), INVALID), (dict(cap=math.inf), INVALID),
    (dict(cap=1e-44, scale=1.0), INVALID), (dict(cap=3e38), INVALID), (dict(seqs=0), OK),
    (dict(seqs=0, q=None, bounds=None), OK),
])
def test_new_tokens(kw, code):
    d = ctypes.byref(desc())
    assert attend(d, **kw) == weigh(d, **kw) == code
    if code != OK and not set(kw) & {"bounds", "table", "lengths", "q", "qa", "qb"}:
        assert lib.kmeans_kv_attend_tokens_workspace_bytes(d, tokens(**kw)) == 0


@pytest.mark.parametrize("scale,cap,code", [
    (2.0, 1.17e38, OK), (2.0, 1.19e38, INVALID), (2.0, 2.3e38, INVALID),
    (0.1, 8e36, OK), (0.1, 9e36, INVALID), (-1e-3, 1e37, INVALID), (0.0, 1e38, OK),
])
def test_the_limits_of_caps(scale, cap, code):
    """Twice the cap to base 2, which far scores are worked out with, is a finite fp32 number,
    and scale / cap has all bits of one."""
    d = ctypes.byref(desc())
    kw = dict(scale=scale, cap=cap, tokens=0)
    assert attend(d, **kw) == weigh(d, **kw, add=1) == code
    assert (lib.kmeans_kv_attend_tokens_workspace_bytes(d, tokens(**kw)) > 0) == (code == OK)


def test_the_limit_of_tokens_times_positions():
    """(seqs + tokens * q_heads / heads / 256) * (table_pages * page / 32 + 2) < 2^27"""
    size = lib.kmeans_kv_attend_tokens_workspace_bytes
    d = ctypes.byref(desc(page=32, pages=1 << 20))
    for seqs, new, pages in ((4096, 1, 32766), (1024, 1, (1 << 17) - 2), (1, (128 << 13) - 128, 16382)):
        t = dict(seqs=seqs, tokens=new, q_heads=4, table_pages=pages, table_stride=pages)
        assert size(d, tokens(**{**t, "table_pages": pages - 1})) > 0
        assert size(d, tokens(**t)) == 0
        assert attend(d, **t) == weigh(d, **t) == UNSUPPORTED


def test_workspaces():
    """Every number of rows has one, whichever units it is cut to."""
    size = lib.kmeans_kv_attend_tokens_workspace_bytes
    d = ctypes.byref(desc(page=32, pages=1 << 20))
    for seqs in (1, 3, 64, 65, 300, 4096):
        for new in (1, 2, 7, 31, 33, 64, 65, 128, 129, 1000, 5000):
            for pages in (1, 20, 1000):
                assert size(d, tokens(seqs=seqs, tokens=new, table_pages=pages, table_stride=pages)) > 0


@pytest.mark.parametrize("kw,code", [
    (dict(out=None), INVALID), (dict(out=ODD), INVALID), (dict(oa=7), INVALID), (dict(ob=-8), INVALID),
    (dict(ws=None), WORKSPACE), (dict(ws=ODD), WORKSPACE), (dict(nbytes=0), WORKSPACE),
    (dict(tokens=0), OK), (dict(tokens=0, q=None, out=None), OK),
])
def test_attend(kw, code):
    assert attend(ctypes.byref(desc()), **kw) == code


@pytest.mark.parametrize("kw,code", [
    (dict(w=None), INVALID), (dict(lse=None), INVALID), (dict(wa=-1), INVALID), (dict(wb=-1), INVALID),
    (dict(positions=-1), INVALID), (dict(positions=(1 << 30) + 1), UNSUPPORTED), (dict(add=2), INVALID),
    (dict(positions=0), OK), (dict(positions=0, w=None, lse=None), OK), (dict(tokens=0, add=1), OK),
    (dict(tokens=0, add=0, w=None), INVALID),
])
def test_weigh(kw, code):
    assert weigh(ctypes.byref(desc()), **kw) == code


@pytest.mark.parametrize("kw,code", [
    (dict(table=None), INVALID), (dict(lengths=None), INVALID), (dict(weights=None), INVALID),
    (dict(kept=None), INVALID), (dict(lengths_out=None), INVALID), (dict(out=None), INVALID),
    (dict(weights_seq=-1), INVALID), (dict(weights_head=-1), INVALID), (dict(oa=-1), INVALID),
    (dict(ob=-1), INVALID), (dict(oa=128), INVALID), (dict(ob=16), INVALID),
    (dict(positions=-1), INVALID), (dict(positions=(1 << 30) + 1), UNSUPPORTED),
    (dict(seqs=-1), INVALID), (dict(seqs=4097), UNSUPPORTED), (dict(table_pages=0), INVALID),
    (dict(table_stride=-1), INVALID), (dict(table_pages=1 << 28), UNSUPPORTED),
    (dict(keep=0), INVALID), (dict(keep=-4), INVALID), (dict(keep=(1 << 30) + 1), UNSUPPORTED),
    (dict(recent=-1), INVALID), (dict(first=-1), INVALID), (dict(recent=19), INVALID),
    (dict(recent=2 ** 31 - 1, first=2 ** 31 - 1), INVALID),
    (dict(to=P, to_pages=1), INVALID), (dict(to=P, to_pages=0), INVALID), (dict(to=P, to_stride=-1), INVALID),
    (dict(seqs=0), OK), (dict(seqs=0, table=None, kept=None), OK),
])
def test_evict(kw, code):
    assert evict(ctypes.byref(desc()), **kw) == code


def test_workspace_bytes():
    f = lib.kmeans_kv_attend_tokens_workspace_bytes
    d = ctypes.byref(desc(heads=8, dim=128, K=256))
    for kw in (dict(tokens=1, seqs=1), dict(tokens=4096, seqs=4096), dict(tokens=1 << 20, seqs=7),
               dict(tokens=0, seqs=1), dict(tokens=5, seqs=0)):
        n = f(d, tokens(q_heads=64, table_pages=1000, **kw))
        assert 0 < n < 1 << 30
        if kw["seqs"] and kw["tokens"]:
            assert attend(d, q_heads=64, table_pages=1000, nbytes=n - 1, **kw) == WORKSPACE
