"""The calls of the key-value cache carry no gradient: a query that would need one
is refused and not answered with a constant, the codes of a key are constants."""
import types

import pytest
import torch
import torch.autograd.forward_ad as fwd

import paper_1402_3788_amd as km
from paper_1402_3788_amd import kv

BF = torch.bfloat16
HOST = types.SimpleNamespace(dtype=BF, index=-1, device=torch.device("cpu"), dim=64)


def test_what_needs_a_gradient():
    plain = torch.zeros(3)
    kv._no_gradient(plain, "t")
    leaf = torch.zeros(3, requires_grad=True)
    for t in (leaf, leaf * 2):
        with pytest.raises(ValueError, match="gradient"):
            kv._no_gradient(t, "t")
        with torch.no_grad():
            kv._no_gradient(t, "t")
        kv._no_gradient(t.detach(), "t")
    with fwd.dual_level():
        kv._no_gradient(plain, "t")
        with pytest.raises(ValueError, match="gradient"):
            kv._no_gradient(fwd.make_dual(plain, plain), "t")


def test_outputs():
    t = torch.zeros(1, 2, 64, dtype=BF, requires_grad=True)
    with pytest.raises(ValueError, match="gradient"):
        kv._target(HOST, t, (1, 2, 64), "t")


@pytest.mark.gpu
def test_calls():
    dev = torch.device("cuda:0")
    g = torch.Generator().manual_seed(0)

    def rand(*shape):
        return torch.randn(shape, generator=g).to(BF).to(dev)

    cache = km.KVCodes.empty(rand(2, 16, 256, 4), rand(2, 16, 256, 4), 2, 16)
    slots = torch.arange(20, device=dev)
    k, v, q = rand(20, 2, 64), rand(20, 2, 64), rand(1, 4, 64)
    km.kmeans_kv_write(cache, k, v, slots)
    codes = cache.k_codes.clone()
    cache.k_codes.zero_()
    km.kmeans_kv_write(cache, k.clone().requires_grad_(), v, slots)
    assert torch.equal(cache.k_codes, codes)
    args = (torch.tensor([[1, 0]], dtype=torch.int32, device=dev),
            torch.tensor([20], dtype=torch.int32, device=dev))
    want = km.kmeans_kv_attend(cache, q, *args)
    leaf = q.clone().requires_grad_()
    buffers = dict(out=torch.empty_like(q), lse=torch.empty(1, 4, device=dev))
    for kw in ({}, buffers):
        for t in (leaf, leaf * 1):
            with pytest.raises(ValueError, match="gradient"):
                km.kmeans_kv_attend(cache, t, *args, **kw)
            with torch.no_grad():
                got = km.kmeans_kv_attend(cache, t, *args, **kw)
            assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
        with fwd.dual_level():
            with pytest.raises(ValueError, match="gradient"):
                km.kmeans_kv_attend(cache, fwd.make_dual(q, q), *args, **kw)
    for kw in (dict(out=leaf * 1), dict(lse=torch.empty(1, 4, device=dev, requires_grad=True))):
        with pytest.raises(ValueError, match="gradient"):
            km.kmeans_kv_attend(cache, q, *args, **kw)
    with pytest.raises(ValueError, match="gradient"):
        km.kmeans_kv_read(cache, slots, out=(k.clone().requires_grad_(), v))
