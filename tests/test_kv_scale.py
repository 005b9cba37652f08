"""The attention's scale is taken to base 2 in fp32, which has to hold it."""
import ctypes

import pytest

import paper_1402_3788_amd as km
from paper_1402_3788_amd.kv import _Desc

P = 0x10000                             # never dereferenced: no workspace, no launch
MAX = 3.4028234663852886e38


@pytest.mark.parametrize("scale,code", [
    (MAX, km.KMEANS_EINVAL), (-MAX, km.KMEANS_EINVAL), (2.4e38, km.KMEANS_EINVAL),
    (2.35e38, km.KMEANS_EWORKSPACE), (-2.35e38, km.KMEANS_EWORKSPACE), (0.0, km.KMEANS_EWORKSPACE),
])
def test_scale(scale, code):
    d = _Desc(P, P, P, P, 4, 16, 2, 64, 4, 16, 0)
    assert km._lib.kmeans_kv_attend(ctypes.byref(d), P, 256, 64, 3, 4, P, 2, 2, P, None, scale,
                                    P, 256, 64, None, None, 0, None) == code
