"""C entry points of the key-value cache in K-means codes: what they refuse, on
the host and before anything is enqueued. Runs without a GPU."""
import ctypes
import math

import pytest

import paper_1402_3788_amd as km
from paper_1402_3788_amd.kv import _Desc

P, ODD = 0x10000, 0x10008               # never dereferenced: validation fails first


def desc(**kw):
    d = dict(k_centres=P, v_centres=P, k_codes=P, v_codes=P, pages=4, page=16, heads=2, dim=64,
             sub=4, K=16, type=0)
    d.update(kw)
    return _Desc(**d)


BAD_DESC = [
    (dict(k_centres=None), km.KMEANS_EINVAL), (dict(v_centres=None), km.KMEANS_EINVAL),
    (dict(k_codes=None), km.KMEANS_EINVAL), (dict(v_codes=None), km.KMEANS_EINVAL),
    (dict(k_centres=ODD), km.KMEANS_EINVAL), (dict(v_codes=ODD), km.KMEANS_EINVAL),
    (dict(pages=0), km.KMEANS_EINVAL), (dict(pages=-3), km.KMEANS_EINVAL),
    (dict(pages=1 << 40), km.KMEANS_EUNSUPPORTED),
    (dict(page=0), km.KMEANS_EINVAL), (dict(page=4), km.KMEANS_EUNSUPPORTED),
    (dict(page=24), km.KMEANS_EUNSUPPORTED), (dict(page=2048), km.KMEANS_EUNSUPPORTED),
    (dict(heads=0), km.KMEANS_EINVAL), (dict(heads=1025), km.KMEANS_EUNSUPPORTED),
    (dict(dim=80), km.KMEANS_EUNSUPPORTED), (dict(dim=0), km.KMEANS_EINVAL),
    (dict(sub=3), km.KMEANS_EUNSUPPORTED), (dict(sub=16), km.KMEANS_EUNSUPPORTED),
    (dict(K=0), km.KMEANS_EINVAL), (dict(K=257), km.KMEANS_EUNSUPPORTED),
    (dict(type=2), km.KMEANS_EINVAL),
]


def write(d, k=P, ka=128, kb=64, v=P, va=128, vb=64, slots=P, n=3):
    return km._lib.kmeans_kv_write(d, k, ka, kb, v, va, vb, slots, n, None)


def read(d, k=P, ka=128, kb=64, v=P, va=128, vb=64, slots=P, n=3):
    return km._lib.kmeans_kv_read(d, slots, n, k, ka, kb, v, va, vb, None)


def attend(d, q=P, qa=256, qb=64, seqs=3, q_heads=4, table=P, stride=2, width=2, lengths=P,
           starts=None, scale=0.1, out=P, oa=256, ob=64, lse=None, ws=P, nbytes=1 << 30):
    return km._lib.kmeans_kv_attend(d, q, qa, qb, seqs, q_heads, table, stride, width, lengths,
                                    starts, scale, out, oa, ob, lse, ws, nbytes, None)


@pytest.mark.parametrize("kw,code", BAD_DESC)
def test_description(kw, code):
    d = ctypes.byref(desc(**kw))
    assert write(d) == read(d) == attend(d) == code
    shape = [x for x in kw if x not in ("k_centres", "v_centres", "k_codes", "v_codes")]
    assert (km._lib.kmeans_kv_attend_workspace_bytes(d, 3, 4, 2) == 0) == bool(shape)


def test_no_description():
    assert write(None) == read(None) == attend(None) == km.KMEANS_EINVAL
    assert km._lib.kmeans_kv_attend_workspace_bytes(None, 3, 4, 2) == 0


@pytest.mark.parametrize("kw,code", [
    (dict(k=None), km.KMEANS_EINVAL), (dict(v=None), km.KMEANS_EINVAL),
    (dict(slots=None), km.KMEANS_EINVAL), (dict(k=ODD), km.KMEANS_EINVAL),
    (dict(v=ODD), km.KMEANS_EINVAL), (dict(ka=130), km.KMEANS_EINVAL),
    (dict(kb=-64), km.KMEANS_EINVAL), (dict(va=-8), km.KMEANS_EINVAL),
    (dict(vb=1), km.KMEANS_EINVAL), (dict(n=-1), km.KMEANS_EINVAL),
    (dict(n=2 ** 31), km.KMEANS_EUNSUPPORTED), (dict(n=0), km.KMEANS_OK),
    (dict(n=0, k=None, v=None, slots=None), km.KMEANS_OK),
])
def test_tokens(kw, code):
    d = ctypes.byref(desc())
    assert write(d, **kw) == read(d, **kw) == code


@pytest.mark.parametrize("kw,code", [
    (dict(q=None), km.KMEANS_EINVAL), (dict(out=None), km.KMEANS_EINVAL),
    (dict(table=None), km.KMEANS_EINVAL), (dict(lengths=None), km.KMEANS_EINVAL),
    (dict(q=ODD), km.KMEANS_EINVAL), (dict(out=ODD), km.KMEANS_EINVAL),
    (dict(qa=4), km.KMEANS_EINVAL), (dict(qb=-8), km.KMEANS_EINVAL),
    (dict(oa=7), km.KMEANS_EINVAL), (dict(ob=2), km.KMEANS_EINVAL),
    (dict(stride=-1), km.KMEANS_EINVAL), (dict(width=0), km.KMEANS_EINVAL),
    (dict(width=1 << 28), km.KMEANS_EUNSUPPORTED), (dict(seqs=-1), km.KMEANS_EINVAL),
    (dict(seqs=4097), km.KMEANS_EUNSUPPORTED), (dict(q_heads=0), km.KMEANS_EINVAL),
    (dict(q_heads=5), km.KMEANS_EINVAL), (dict(q_heads=2 * 129), km.KMEANS_EUNSUPPORTED),
    (dict(seqs=4096, width=1 << 24), km.KMEANS_EUNSUPPORTED),
    (dict(scale=math.nan), km.KMEANS_EINVAL), (dict(scale=math.inf), km.KMEANS_EINVAL),
    (dict(ws=None), km.KMEANS_EWORKSPACE), (dict(nbytes=0), km.KMEANS_EWORKSPACE),
    (dict(ws=ODD), km.KMEANS_EWORKSPACE), (dict(seqs=0), km.KMEANS_OK),
])
def test_attend(kw, code):
    assert attend(ctypes.byref(desc()), **kw) == code


def test_workspace_bytes():
    f = km._lib.kmeans_kv_attend_workspace_bytes
    d = ctypes.byref(desc(heads=8, dim=128, K=256))
    assert 0 < f(d, 1, 8, 1) <= f(d, 1, 8, 100) <= f(d, 64, 64, 1000) < 1 << 26
    assert f(d, 4096, 64, 1000) > 0 and f(d, 4097, 64, 1000) == 0
    assert f(d, 0, 8, 1) > 0 and f(d, 1, 9, 1) == 0 and f(d, 1, 8, 0) == 0
    assert attend(d, seqs=64, q_heads=64, width=1000, nbytes=f(d, 64, 64, 1000) - 1) == \
        km.KMEANS_EWORKSPACE
